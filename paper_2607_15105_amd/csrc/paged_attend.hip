// Attention of a ragged batch of new rows over the paged cache: row r of
// sequence s, at position p = q_begin[s] + r - seq_rows[s], attends the cached
// positions t <= p whose page is present.
//
// The rows of a sequence and kv head are folded with its G query heads, so
// that one reading of K and V serves them all, and taken M folded rows at a
// time: an item is (sequence, kv head, row tile), a unit of work 32 or 64 keys
// of an item. Lengths live on the device; every workgroup counts the units of
// all sequences, takes an equal share of their concatenation and finds its
// first unit. However ragged the batch is, the shares are alike, and a long
// context of few rows spreads over the whole GPU. An item that lies in one
// share is finished there; one that several shares cut is left as partial
// results (unnormalised O with its maximum and sum), which a second kernel
// joins in the order of the keys: no atomics, the same bits every run.
//
// Softmax as in the routed kernels: S^T = K . Q^T, every lane holds scores of
// one row, running maximum and sum per lane, the maximum raised lazily (when
// it grows by over 2^8), O^T += V^T . P^T straight from the score registers;
// maxima, sums and O are float32.
#include "paged_device.h"

namespace hga {

namespace {

// The kernel's arguments, read where they are used: taken as the parameter they are
// loaded at the kernel's start and kept in scalars through the loops, of which they
// take as many as there are (the rest went through vector registers in every
// tile: 38 moves of 100 instructions that ask for a tile's rows).
__device__ __forceinline__ const PagedAttnArgs& args_here() {
  auto p = (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const PagedAttnArgs*)p;
}

// ---------------------------------------------------------------- the shares

// The items of a sequence: per kv head nt row tiles of T tokens; row tile j has
// tiles(j) units of 2^KS keys. Positions and tile numbers are 32-bit (kMaxPos).
template <int KS>
struct SeqShape {
  int first, n;   // rows of the call
  int qb, cap;    // position of the first row; positions that the page table covers
  int shift;      // row tiles hold 2^shift tokens
  bool plain;     // all positions inside [0, cap)

  __device__ inline int nt() const { return ((n - 1) >> shift) + 1; }
  // position of row i, clamped to 32 bits
  __device__ inline int pos(int64_t i) const { return (int)(qb + i < kMaxPos ? qb + i : kMaxPos); }
  // one past the last position that row tile j attends
  __device__ inline int end(int j) const {
    const int64_t rows = (int64_t)(j + 1) << shift, e = qb + (plain && rows < n ? rows : n);
    return e < 0 ? 0 : (e > cap ? cap : (int)e);
  }
  // at least one, so that rows with nothing to attend are written too
  __device__ inline int tiles(int j) const {
    const int e = end(j);
    return e > 0 ? (e + (1 << KS) - 1) >> KS : 1;
  }
  // units of the row tiles before j <= nt - 1: sum over i < j of ceil((qb + (i+1) T) / 2^KS)
  __device__ inline int64_t before(int64_t j) const {
    if (j == 0) return 0;
    if (!plain) return j * tiles(0);
    constexpr int up = (1 << KS) - 1;
    if (shift >= KS) return j * ((qb + up) >> KS) + (((j * (j + 1)) >> 1) << (shift - KS));
    const int q = 1 << (KS - shift);  // row tiles in which the sum's terms grow by one
    const int64_t a = j >> (KS - shift);
    const int b = (int)(j & (q - 1));
    int64_t period = 0, rest = 0;
    for (int i = 1; i <= q; ++i) {
      const int64_t term = ((int64_t)qb + up + ((int64_t)i << shift)) >> KS;
      period += term;
      if (i <= b) rest += term;
    }
    return q * (a * (a - 1) / 2) + a * period + rest + a * b;
  }
  // With `over` units ahead of each item's for its start and end: where item j's
  // begin, and all of them.
  __device__ inline int64_t start(int j, int over) const { return before(j) + (int64_t)j * over; }
  __device__ inline int64_t units(int over) const {
    return n == 0 ? 0 : start(nt() - 1, over) + over + tiles(nt() - 1);
  }
};

template <int KS>
__device__ inline SeqShape<KS> shape_of(const PagedAttnArgs& a, int s, int shift) {
  SeqShape<KS> q;
  rows_of(a.p, s, q.first, q.n);
  if (q.n < a.min_rows || q.n > a.max_rows) q.n = 0;
  q.qb = a.p.q_begin[s];
  const int64_t cap = a.p.table_cap << a.p.page_shift;
  q.cap = (int)(cap < kMaxPos ? cap : kMaxPos);
  q.shift = shift;
  q.plain = q.qb >= 0 && (int64_t)q.qb + q.n <= q.cap;
  return q;
}

// A workgroup's share of the units: `left` of them, and where it begins.
template <int KS>
struct Share {
  int64_t left, per;
  int s, h, j;
  int kt;           // first unit within the item; below zero: so many of its start are left
  SeqShape<KS> q;   // of sequence s
};

// NT threads, W workgroups; `lds` holds NT / 64 + 2 int64. A share is a multiple
// of `step` units, `least` at least. An item counts as OVER units more than it
// has, about what its start and end take, so that shares of many short items are
// not the last to end. (Not for few rows: four units there made 64 ragged contexts
// 179 -> 171 us, but eight equal ones of 131K 381 -> 388, and sixteen of 1,000
// positions, which fill the shares evenly without, 20 -> 25.)
template <int NT, int W, int KS, int OVER>
__device__ inline Share<KS> take_share(int wg, int shift, int step, int least, int64_t* lds) {
  constexpr int NW = NT / 64;
  const PagedAttnArgs& a = args_here();
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n_seqs = a.p.n_seqs, c = (n_seqs + NT - 1) / NT;
  int64_t sum = 0;
  for (int k = 0; k < c; ++k) {
    const int s = tid * c + k;
    if (s < n_seqs) sum += a.p.n_kv_heads * shape_of<KS>(a, s, shift).units(OVER);
  }
  int64_t inc = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t up = __shfl_up(inc, o, 64);
    if (lane >= o) inc += up;
  }
  if (lane == 63) lds[wave] = inc;
  __syncthreads();
  int64_t total = 0, base = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    if (w < wave) base += lds[w];
    total += lds[w];
  }
  Share<KS> sh;
  sh.per = (total + W - 1) / W;
  sh.per = sh.per < least ? least : (sh.per + step - 1) / step * step;
  const int64_t u0 = wg * sh.per;
  sh.left = u0 >= total ? 0 : total - u0 < sh.per ? total - u0 : sh.per;
  int64_t off = u0 - (base + inc - sum);
  if (sh.left > 0 && off >= 0 && off < sum) {  // this thread's sequences hold the first unit
    int s = tid * c;
    for (; s < n_seqs - 1; ++s) {
      const int64_t m = a.p.n_kv_heads * shape_of<KS>(a, s, shift).units(OVER);
      if (off < m) break;
      off -= m;
    }
    lds[NW] = s;
    lds[NW + 1] = off;
  }
  __syncthreads();
  sh.s = sh.h = sh.j = sh.kt = 0;
  if (sh.left > 0) {
    sh.s = __builtin_amdgcn_readfirstlane((int)lds[NW]);
    off = lds[NW + 1];
    sh.q = shape_of<KS>(a, sh.s, shift);
    const int64_t m = sh.q.units(OVER);
    // kv head and rest: 32-bit division where it will do
    const bool narrow = m < ((int64_t)1 << 31) && off < ((int64_t)1 << 31);
    sh.h = __builtin_amdgcn_readfirstlane(narrow ? (int)((uint32_t)off / (uint32_t)m) : (int)(off / m));
    off -= sh.h * m;
    int lo = 0, hi = sh.q.nt() - 1;  // the last row tile that begins at or before off
    while (lo < hi) {
      const int mid = (int)(((int64_t)lo + hi + 1) >> 1);
      if (sh.q.start(mid, OVER) <= off) lo = mid;
      else hi = mid - 1;
    }
    sh.j = __builtin_amdgcn_readfirstlane(lo);
    sh.kt = __builtin_amdgcn_readfirstlane((int)(off - sh.q.start(sh.j, OVER)) - OVER);
  }
  __syncthreads();
  return sh;
}

// ---------------------------------------------------------------- key tiles

// An item's cached rows: sequence, kv head and last position resolved, in as
// few scalars as the loops over its tiles need (with the call's arguments in
// their place 200 of them went through vector registers).
struct KvItem {
  const int32_t* table;   // of the sequence
  const char* k;          // of the kv head
  const char* v;
  const uint8_t* k_scale;
  const uint8_t* v_scale;
  uint32_t k_page, k_tok, v_page, v_tok, scale_page;  // bytes
  int n_pages, shift, mask;
  int end;                // one past the last position that the item attends

  __device__ inline KvItem(const PagedArgs& a, int s, int h, int end_)
      : table(a.table + (int64_t)s * a.table_cap), k(a.k + h * a.k_head), v(a.v + h * a.v_head),
        k_scale(a.k_scale + ((int64_t)h << a.page_shift)), v_scale(a.v_scale + ((int64_t)h << a.page_shift)),
        k_page((uint32_t)a.k_page), k_tok((uint32_t)a.k_tok), v_page((uint32_t)a.v_page), v_tok((uint32_t)a.v_tok),
        scale_page((uint32_t)a.n_kv_heads << a.page_shift), n_pages(a.n_pages), shift(a.page_shift),
        mask((1 << a.page_shift) - 1), end(end_) {}

  // V's row of position t, which is present.
  __device__ inline const char* v_row(int t) const { return v + page_off(table[t >> shift], t & mask, v_page, v_tok); }
  // Its scale, of 8-bit rows.
  __device__ inline float v_row_scale(int t) const {
    return __uint_as_float((uint32_t)v_scale[(uint64_t)(uint32_t)table[t >> shift] * scale_page + (uint32_t)(t & mask)] << 23);
  }
};

// Where 64 tiles of an item lie: lane i has the pages of tile x0 + i * STRIDE, a tile
// of KT positions, for the BLOCKS blocks of 16 rows from block b0 on; page 0
// where there is none. Asked for 64 tiles at a time, so that a tile costs a lane
// read and a bit test. (Asked for tile by tile, beside the tile before: 64
// ragged contexts in 8 bits 187 us, a 2,048-token chunk at the end of 32K 1,097 us;
// waited for where it was asked for: 343 and 1,383 us.)
template <int KT, int STRIDE, int BLOCKS>
struct TileMap {
  int page[BLOCKS];
  uint64_t full;   // bit i: every position of tile x0 + i * STRIDE is present and before the item's end

  __device__ inline void fill(const KvItem& a, int x0, int b0, int lane) {
    const int64_t t = ((int64_t)x0 + (int64_t)STRIDE * lane) * KT;
    bool all = t + KT <= a.end;
    int e[KT / 16];
#pragma unroll
    for (int b = 0; b < KT / 16; ++b) {
      e[b] = -1;
      if (t + 16 * b < a.end) e[b] = a.table[(int)(t + 16 * b) >> a.shift];
    }
#pragma unroll
    for (int b = 0; b < KT / 16; ++b) {
      if ((uint32_t)e[b] >= (uint32_t)a.n_pages) {
        all = false;
        e[b] = 0;
      }
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) page[b] = e[b];
    if constexpr (BLOCKS == 1) {
#pragma unroll
      for (int b = 1; b < KT / 16; ++b)
        if (b == b0) page[0] = e[b];
    }
    full = __ballot(all);
  }
};

template <int KT>
__device__ inline constexpr uint64_t all_keys() { return KT == 64 ? ~0ull : (1ull << (KT & 63)) - 1; }

// The positions of a tile that are present and before the item's end.
template <int KT>
__device__ inline uint64_t present(const KvItem& a, int tile, int lane) {
  const int t = tile * KT + lane;
  int e = -1;
  if (lane < KT && t < a.end) e = a.table[t >> a.shift];
  return __ballot((uint32_t)e < (uint32_t)a.n_pages);
}

template <typename T>
__device__ inline bool finite16(const uint4& w) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  bool fine = true;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (Elem<T>::kBytes == 2)
      fine = fine && (u[j] & 0x7f80u) != 0x7f80u && (u[j] & 0x7f800000u) != 0x7f800000u;
    else
      fine = fine && (u[j] & 0x7f800000u) != 0x7f800000u;
  }
  return fine;
}
// The finite elements of 16 bytes, zeros for the others.
template <typename T>
__device__ inline uint4 only_finite(const uint4& w) {
  uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (Elem<T>::kBytes == 2) {
      if ((u[j] & 0x7f80u) == 0x7f80u) u[j] &= 0xffff0000u;
      if ((u[j] & 0x7f800000u) == 0x7f800000u) u[j] &= 0xffffu;
    } else if ((u[j] & 0x7f800000u) == 0x7f800000u) {
      u[j] = 0;
    }
  }
  return make_uint4(u[0], u[1], u[2], u[3]);
}

// One LDS stage of a KT-key tile: K rows, then V (rows, or transposed for
// float32, which has no transposing LDS load).
template <typename T, int D, int KT_>
struct Stage {
  using TL = Tile<T, D>;
  static constexpr int KT = KT_;
  static constexpr bool TR = Elem<T>::kBytes == 2;
  static constexpr int kV = KT * TL::kRowPitch;  // offset of V
  static constexpr int kBytes = kV + (TR ? KT * TL::kRowPitch : D * (KT + 1) * 4);
  // element (d, kpos) of the transposed V
  __device__ static inline int t_off(int d, int kpos) { return kV + (d * (KT + 1) + kpos) * 4; }
  // 16 bytes of row `row` from element e on
  __device__ static inline void put(char* st, bool v, int row, int e, const uint4& w) {
    if (TR || !v) {
      *reinterpret_cast<uint4*>(st + (v ? kV : 0) + TL::row_off(row, e)) = w;
    } else {
      const uint32_t x[4] = {w.x, w.y, w.z, w.w};
      const int kp = kpos_of<Elem<T>::E>(row);
#pragma unroll
      for (int y = 0; y < 4; ++y) *reinterpret_cast<uint32_t*>(st + t_off(e + y, kp)) = x[y];
    }
  }
};

// The same for the 16-row products: both tensors in rows. An operand load of K
// takes one 16-byte piece of 16 rows, whose rows 16 bytes over a multiple of 256 (or
// 128) put them on all banks. bf16 V is read transposed, 32 lanes taking 32 bytes
// of eight consecutive rows: those 32 bytes over do the same. float32 V is
// read as it lies, 64 bytes of rows four apart, for which 16 bytes over are right.
template <typename T, int D>
struct FewStage {
  static constexpr int KT = 32, EB = Elem<T>::kBytes;
  static constexpr int kPitch = D * EB + 16, kVPitch = D * EB + (EB == 2 ? 32 : 16);
  static constexpr int kV = KT * kPitch, kBytes = kV + KT * kVPitch;
  __device__ static inline int k_off(int row, int e) { return row * kPitch + e * EB; }
  __device__ static inline int v_off(int row, int e) { return kV + row * kVPitch + e * EB; }
  __device__ static inline void put(char* st, bool v, int row, int e, const uint4& w) {
    *reinterpret_cast<uint4*>(st + (v ? v_off(row, e) : k_off(row, e))) = w;
  }
};

// One wave's share (of NW waves) of a KT-key tile of K and V, in registers. A
// load instruction covers R whole rows; pages hold 16 tokens or more, so 16 rows
// lie in one page and have one scalar address.
template <typename T, int D, typename ST, bool F8, int NW>
struct TileRegs {
  static constexpr int KT = ST::KT;
  static constexpr int EB = Elem<T>::kBytes;
  static constexpr int PPR = (F8 ? D : D * EB) / 16;  // 16-byte pieces of a held row
  static constexpr int R = 64 / PPR;
  static constexpr int NI = KT / R;                   // instructions per tensor
  static constexpr int IPW = 2 * NI / NW;
  static constexpr int IPB = 16 / R;                  // instructions per 16 rows
  static constexpr int PE = F8 ? 16 : 16 / EB;        // elements of a piece
  static_assert(IPW % IPB == 0, "a wave loads whole blocks of 16 rows");
  static constexpr int BLOCKS = NW == 1 ? KT / 16 : 1;  // blocks of 16 rows of a tensor that the wave loads
  u32x4 w[IPW];
  uint32_t sc;  // F8: scale byte of K's row `lane`, or V's row lane - KT (NW == 1); of the wave's row lane % 16

  // `page`: of the wave's blocks.
  __device__ inline void load(const KvItem& a, int tile, const int (&page)[BLOCKS], int wave, int lane) {
    if constexpr (F8) {
      const uint32_t low = (uint32_t)page[0], high = (uint32_t)page[BLOCKS - 1];
      uint32_t pg = low, row;
      const uint8_t* base;
      if constexpr (NW == 1) {
        static_assert(KT == 32, "K's and V's scales fill a wave");
        row = lane & 31;
        pg = row & 16 ? high : low;
        base = lane & 32 ? a.v_scale : a.k_scale;
      } else {
        row = (wave * IPW % NI) * R + (lane & 15);
        base = wave * IPW >= NI ? a.v_scale : a.k_scale;
      }
      sc = base[(uint64_t)pg * a.scale_page + (uint32_t)((tile * KT + row) & a.mask)];
    }
#pragma unroll
    for (int b = 0; b < IPW / IPB; ++b) {
      const int j = wave * IPW + b * IPB, row = (j % NI) * R;
      const bool v = j >= NI;
      const uint32_t pg = (uint32_t)page[NW == 1 ? b % BLOCKS : 0], slot = (uint32_t)((tile * KT + row) & a.mask);
      const uint32_t tok = v ? a.v_tok : a.k_tok;
      const char* base = (v ? a.v : a.k) + ((uint64_t)pg * (v ? a.v_page : a.k_page) + (uint64_t)slot * tok);
#pragma unroll
      for (int i = 0; i < IPB; ++i)
        w[b * IPB + i] =
            *reinterpret_cast<const u32x4*>(base + (uint32_t)((lane / PPR + i * R) * tok + (lane % PPR) * 16));
    }
  }

  // Into the LDS stage. masked: rows that are not ok are zeros, and what is not
  // finite in V is left out; returns whether there was such in the wave's rows.
  __device__ __forceinline__ bool store(char* st, uint64_t ok_rows, bool masked, int wave, int lane) const {
    if (masked) return put<true>(st, ok_rows, wave, lane);
    return put<false>(st, ok_rows, wave, lane);
  }
  template <bool MASKED>
  __device__ __forceinline__ bool put(char* st, uint64_t ok_rows, int wave, int lane) const {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < IPW; ++i) {
      const int j = wave * IPW + i, row0 = (j % NI) * R, row = row0 + lane / PPR;
      const bool v = j >= NI;
      uint4 out[PE * EB / 16];
      if constexpr (F8) {
        const int from = NW == 1 ? (v ? KT : 0) + row : row & 15;
        const float scale = __uint_as_float((uint32_t)__shfl((int)sc, from, 64) << 23);
#pragma unroll
        for (int o = 0; o < PE * EB / 16; ++o) {
          uint32_t c[Codes<T>::kWords];
#pragma unroll
          for (int x = 0; x < Codes<T>::kWords; ++x) c[x] = w[i][o * Codes<T>::kWords + x];
          out[o] = Codes<T>::decode(c, scale);
        }
      } else {
        out[0] = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
      }
      if constexpr (MASKED) {
        const bool ok = (ok_rows >> row) & 1;
#pragma unroll
        for (int o = 0; o < PE * EB / 16; ++o) {
          if (!ok) out[o] = make_uint4(0u, 0u, 0u, 0u);
          if (v && !finite16<T>(out[o])) {
            bad = true;
            out[o] = only_finite<T>(out[o]);
          }
        }
      }
#pragma unroll
      for (int o = 0; o < PE * EB / 16; ++o) {
        ST::put(st, v, row, (lane % PPR) * PE + o * 16 / EB, out[o]);
      }
    }
    if constexpr (MASKED) return __any(bad);
    return false;
  }
};

// Element e of a held row of V where it is not finite, else 0: judged by its value, as
// the tiles' rows are (8 bits: a code and its scale may stand for 2^128 and more).
template <typename T, bool F8>
__device__ inline float not_finite(const char* row, float scale, int e) {
  float x;
  if constexpr (F8) x = Codes<T>::one((uint8_t)row[e], scale);
  else if constexpr (Elem<T>::kBytes == 2) x = bf16_bits_to_float(*reinterpret_cast<const uint16_t*>(row + 2 * e));
  else x = *reinterpret_cast<const float*>(row + 4 * e);
  return fabsf(x) < __builtin_inff() ? 0.0f : x;
}

// Whether a held row of V is finite.
template <typename T, int D, bool F8>
__device__ inline bool finite_row(const char* row, float scale) {
  bool fine = true;
#pragma unroll 1
  for (int i = 0; i < D * (F8 ? 1 : Elem<T>::kBytes) / 16; ++i) {
    const uint4 w = *reinterpret_cast<const uint4*>(row + 16 * i);
    if constexpr (F8) {
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 4; j += Codes<T>::kWords) fine = fine && finite16<T>(Codes<T>::decode(u + j, scale));
    } else {
      fine = fine && finite16<T>(w);
    }
  }
  return fine;
}

// What is not finite in V is left out of masked tiles (a product with p = 0
// would bring it to rows that do not attend its key). Where there was such, the
// units first, first + stride, ... before `last`, of `sub` tiles each, are looked
// through again after the loop, the masked tiles or all of them, and add(position,
// row, its scale) adds it to the rows that do attend it. Rare, and apart from the
// loop: inside it, it cost the loop its registers.
template <typename T, int D, int KT, bool F8, typename Add>
__device__ inline void bad_rows(const KvItem& a, int first, int last, int stride, int sub, int first_pos, bool all,
                                int lane, Add&& add) {
  for (int i = 0, y = first * sub; y < last * sub; i = i + 1 == sub ? 0 : i + 1, y += i ? 1 : (stride - 1) * sub + 1) {
    const uint64_t ok = present<KT>(a, y, lane);
    if (!all && ok == all_keys<KT>() && y * KT + KT - 1 <= first_pos) continue;  // not masked
    bool fine = true;
    if ((ok >> lane) & 1) {  // a row per lane
      const int t = y * KT + lane;
      fine = finite_row<T, D, F8>(a.v_row(t), F8 ? a.v_row_scale(t) : 1.0f);
    }
    uint64_t bad = __ballot(!fine);
    while (bad) {
      const int t = y * KT + __builtin_ctzll(bad);
      bad &= bad - 1;
      add(t, a.v_row(t), F8 ? a.v_row_scale(t) : 1.0f);
    }
  }
}

// Folded row f of kv head h of the sequence whose rows begin at `first`.
__device__ inline const char* query_row(const PagedAttnArgs& a, int first, int h, int64_t f) {
  const int hq = (h << a.gqa_shift) + (int)(f & ((1 << a.gqa_shift) - 1));
  return row_ptr(a.Q, first + (f >> a.gqa_shift), a.q_tok) + hq * a.q_head;
}

// How far, in raw scores, a row's maximum may lie above the one in use: 2^8 in
// p. Finite for any scale, so that a score is above -inf plus it.
__device__ inline float slack(float c) { return fminf(8.0f / c, 3.0e38f); }

// ---------------------------------------------------------------- one wave's rows

// 32 folded rows of one wave, over KT-key tiles: lane l holds (half the head
// dim of) row l % 32.
template <typename T, int D, int KT>
struct WaveRows {
  using EL = Elem<T>;
  using Frag = typename EL::Frag;
  using TL = Tile<T, D>;
  static constexpr int E = EL::E, KS = EL::KSTEP, EB = EL::kBytes;
  static constexpr int NKS = D / KS, NDT = D / 32, VPS = 16 / E;
  using ST = Stage<T, D, KT>;

  Frag qf[NKS];
  f32x16 oacc[NDT];
  float m, l;
  int pos;  // of the lane's row; -1 for a row past the item's rows

  // Rows of the item from folded row f0 on (of nf rows of the sequence).
  template <typename Q>
  __device__ inline void begin(const PagedAttnArgs& a, const Q& q, int h, int64_t f0, int lane) {
    const int hh = lane >> 5;
    const int64_t nf = (int64_t)q.n << a.gqa_shift;
    const int64_t f = f0 + (lane & 31);
    pos = f < nf ? q.pos(f >> a.gqa_shift) : -1;
    const char* p = query_row(a, q.first, h, f < nf ? f : nf - 1);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[ks] = EL::load_frag(p + (ks * KS + E * hh) * EB);
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) oacc[dt] = f32x16{};
    m = -__builtin_inff();
    l = 0.0f;
  }

  using Probs = Frag[VPS];  // P of 32 keys, as the operand of P.V

  // Raw scores of keys 32 t ... of the stage.
  __device__ __forceinline__ void scores(f32x16& s, const char* st, int t, int lane) const {
    s = f32x16{};
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      const Frag kf = EL::load_frag(st + TL::row_off(32 * t + (lane & 31), ks * KS + E * (lane >> 5)));
      s = EL::mma(kf, qf[ks], s);
    }
  }
  // Keys of them that are not ok or after the row do not count.
  __device__ __forceinline__ void hide(f32x16& s, int tile, int t, uint64_t ok, int lane) const {
    const int rel = pos < 0 ? -1 : pos - tile * KT;  // keys 0 .. rel are at or before the row
    const uint64_t see = ok & (rel < 0 ? 0 : rel >= 63 ? ~0ull : (2ull << rel) - 1);
    const uint32_t mine = (uint32_t)(see >> (32 * t)) >> (4 * (lane >> 5));
#pragma unroll
    for (int v = 0; v < 16; ++v)
      if (!((mine >> (8 * (v >> 2) + (v & 3))) & 1)) s[v] = -__builtin_inff();
  }
  __device__ __forceinline__ static float row_max(const f32x16& s) {
    float mx = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
    return half_max(mx);
  }
  // The running maximum follows mx, O and the sum with it, where it grew by over 2^8.
  __device__ __forceinline__ void raise(float mx, float c) {
    const bool up = mx > m + slack(c);  // the first finite score too: m = -inf
    if (__any(up)) {
      const float mn = up ? mx : m;
      const float corr = up ? __builtin_amdgcn_exp2f((m - mn) * c) : 1.0f;
      m = mn;
      l *= corr;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) oacc[dt] *= corr;
    }
  }
  // float32: the scores' exponentials, and O^T += V^T . P^T over keys 32 t ... of the stage.
  __device__ __forceinline__ void probs(const f32x16& s, Probs& pf, float c) {
    const float mc = m == -__builtin_inff() ? 0.0f : m * c;  // nothing attended yet: every p is 0
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < VPS; ++k) {
      pf[k] = __builtin_amdgcn_exp2f(fmaf(s[k], c, -mc));
      sum += pf[k];
    }
    l += sum;
  }
  __device__ __forceinline__ void values(const Probs& pf, const char* st, int t, int lane) {
#pragma unroll
    for (int k = 0; k < VPS; ++k)
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        const Frag vf = EL::load_frag(st + ST::t_off(32 * dt + (lane & 31), KS * (t * VPS + k) + (lane >> 5)));
        oacc[dt] = EL::mma(vf, pf[k], oacc[dt]);
      }
  }

  // Operands of the products to come: the next four steps' (see half()).
  static constexpr int RING = 4, NB = NDT * VPS;
  __device__ __forceinline__ static Frag k_frag(const char* st, int t, int ks, int lane) {
    return EL::load_frag(st + TL::row_off(32 * t + (lane & 31), ks * KS + E * (lane >> 5)));
  }
  __device__ __forceinline__ static Frag v_frag(const char* st, int t, int i, int lane) {
    const int kk = t * VPS + i / NDT, hh = lane >> 5;
    return tr_frag<TL>(st + ST::kV, 32 * (i % NDT), 16 * kk + 4 * hh, 16 * kk + 8 + 4 * hh, lane);
  }

  // bf16: 32 keys whose scores are in s (V: half t of stage st), beside the
  // scores sn of the 32 after them (K: half tn of stage stn; MORE: there are
  // such). NKS + NB steps of one product each. The product's operand was read
  // from LDS four steps ahead; beside the first NKS products go the
  // exponentials, beside the others the maximum of sn. The order is fixed by
  // hand: left to itself the compiler gathers the products and waits for each
  // operand right after asking for it. fr holds the first operands on entry, and
  // those of the next call on return, whose K is half tk of stage stk.
  template <bool MORE, typename Hide>
  __device__ __forceinline__ void half(f32x16& s, f32x16& sn, Frag (&fr)[RING], const char* st, int t, const char* stn,
                                       int tn, const char* stk, int tk, float c, int lane, Hide&& hide_next) {
    const float mc = m == -__builtin_inff() ? 0.0f : m * c;  // nothing attended yet: every p is 0
    float sum = 0.0f;
    Probs pf;
    constexpr int PER = 16 / NKS;
#pragma unroll
    for (int i = 0; i < NKS; ++i) {
      if constexpr (MORE) sn = EL::mma(fr[i % RING], qf[i], i == 0 ? f32x16{} : sn);
      const int next = i + RING;
      if (next >= NKS) fr[i % RING] = v_frag(st, t, next - NKS, lane);
      else if constexpr (MORE) fr[i % RING] = k_frag(stn, tn, next, lane);
#pragma unroll
      for (int j = i * PER; j < (i + 1) * PER; ++j) {
        s[j] = __builtin_amdgcn_exp2f(fmaf(s[j], c, -mc));
        sum += s[j];
      }
      if ((i + 1) * PER % E == 0) {  // bf16: P is rounded to the inputs' precision, as in the routed forward
        const int k = ((i + 1) * PER - 1) / E;
        float pv[E];
#pragma unroll
        for (int j = 0; j < E; ++j) pv[j] = s[E * k + j];
        pf[k] = EL::frag_from(pv);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    l += sum;
#pragma unroll
    for (int k = 0; k < VPS; ++k) asm volatile("" : "+v"(pf[k]));  // here, and not past the branch
    hide_next();
    float mx = -__builtin_inff();
    constexpr int MAXES = 16 / (NB / 2);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      oacc[i % NDT] = EL::mma(fr[(NKS + i) % RING], pf[i / NDT], oacc[i % NDT]);
      const int next = i + RING;
      if (next < NB) fr[(NKS + i) % RING] = v_frag(st, t, next, lane);
      else if constexpr (MORE) fr[(NKS + i) % RING] = k_frag(stk, tk, next - NB, lane);
      if constexpr (MORE) {
        if (i >= NB / 2) {
#pragma unroll
          for (int j = (i - NB / 2) * MAXES; j < (i - NB / 2 + 1) * MAXES; ++j) mx = fmaxf(mx, sn[j]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (MORE) raise(half_max(mx), c);
  }

  template <bool F8>
  __device__ inline void add_bad(const KvItem& a, int first, int last, int first_pos, int lane) {
    bad_rows<T, D, KT, F8>(a, first, last, 1, 1, first_pos, false, lane, [&](int t, const char* row, float scale) {
      if (pos < t) return;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          oacc[dt][v] += not_finite<T, F8>(row, scale, 32 * dt + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3));
          __builtin_amdgcn_sched_barrier(0);
        }
    });
  }
};

__device__ inline void store4(char* p, f32x4 x, bool bf16) {
  if (bf16)
    *reinterpret_cast<uint2*>(p) = uint2{float_to_bf16_bits(x[0]) | (float_to_bf16_bits(x[1]) << 16),
                                         float_to_bf16_bits(x[2]) | (float_to_bf16_bits(x[3]) << 16)};
  else
    *reinterpret_cast<f32x4*>(p) = x;
}

// Output row of folded row f (of the sequence) of kv head h.
__device__ inline char* out_row(const PagedAttnArgs& a, int first, int h, int64_t f, float*& lse) {
  const int64_t row = first + (f >> a.gqa_shift);
  const int hq = (h << a.gqa_shift) + (int)(f & ((1 << a.gqa_shift) - 1));
  lse = a.lse + row * a.n_q_heads + hq;
  return a.O + (uint64_t)(uint32_t)row * (uint32_t)a.o_tok + hq * a.o_head;
}

__device__ inline float lse_of(float m, float l, float c) {
  return l == 0.0f ? -__builtin_inff() : (m * c + __log2f(l)) * kLn2;
}

// The workgroup's place in the concatenation of all units: consecutive shares on
// one XCD (workgroups are dealt round-robin to the eight), whose L2 then holds
// what they share (three of four reads of a 2,048-row chunk's keys).
__device__ inline int share_index() { return (blockIdx.x & 7) * (gridDim.x / 8) + (blockIdx.x >> 3); }

// Follows a share item by item: f(share at the item, tiles of it, whether that
// is all of it), and the record of the one left unfinished.
template <int OVER, int KS, typename F>
__device__ inline void walk(Share<KS> sh, int wg, int shift, F&& f) {
  if (threadIdx.x == 0) args_here().info[wg] = make_int4(0, 0, 0, 0);
  while (sh.left > 0) {
    if (OVER > 0 && sh.kt < 0) {
      sh.left += sh.kt;
      sh.kt = 0;
      if (sh.left <= 0) return;  // the item is the next share's
    }
    const int len = sh.q.tiles(sh.j), rest = len - sh.kt;
    const int n = rest < sh.left ? rest : (int)sh.left;
    if (sh.kt == 0 && n < len) {  // goes on in the next shares: this one joins it
      const int64_t more = len - n;
      if (threadIdx.x == 0) args_here().info[wg] = make_int4((int)(1 + (more + sh.per - 1) / sh.per), sh.s, sh.h, sh.j);
    }
    f(sh, n, n == len);
    sh.left -= n;
    sh.kt = -OVER;
    if (sh.left > 0 && ++sh.j == sh.q.nt()) {
      const PagedAttnArgs& a = args_here();
      sh.j = 0;
      if (++sh.h == a.p.n_kv_heads) {
        sh.h = 0;
        do {
          if (++sh.s >= a.p.n_seqs) return;  // not reached: units remain, so a sequence with rows does
          sh.q = shape_of<KS>(a, sh.s, shift);
        } while (sh.q.n == 0);
      }
    }
  }
}

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

// ---------------------------------------------------------------- few rows

// 16x16 products (lane l, quarter q = l / 16): A row and B column l % 16, k = E q + j; C
// column l % 16, row 4 q + v. bf16: k = 32, E = 8; float32: k = 4, E = 1.
template <typename T> struct Elem16;
template <> struct Elem16<__bf16> {
  using Frag = bf16x8;
  static constexpr int E = 8, KS = 32;
  __device__ static inline f32x4 mma(Frag a, Frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Elem16<float> {
  using Frag = float;
  static constexpr int E = 1, KS = 4;
  __device__ static inline f32x4 mma(Frag a, Frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  }
};

// NR groups of 16 folded rows: lane l holds (a quarter of the head dim of) row
// l % 16 of each. A 32-key tile's scores are two 16x16 tiles: of row l % 16 the lane has
// keys 4 q + v and 16 + 4 q + v, which in that order are P's operand.
template <typename T, int D, int NR>
struct FewRows {
  using EL = Elem16<T>;
  using Frag = typename EL::Frag;
  using ST = FewStage<T, D>;
  static constexpr int E = EL::E, KS = EL::KS, EB = Elem<T>::kBytes, NKS = D / KS, NDT = D / 16;

  Frag qf[NR][NKS];
  f32x4 oacc[NR][NDT];
  float m[NR], l[NR];
  int pos[NR];

  template <typename Q>
  __device__ inline void begin(const PagedAttnArgs& a, const Q& q, int h, int64_t f0, int lane) {
    const int64_t nf = (int64_t)q.n << a.gqa_shift;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const int64_t f = f0 + 16 * r + (lane & 15);
      pos[r] = f < nf ? q.pos(f >> a.gqa_shift) : -1;
      const char* p = query_row(a, q.first, h, f < nf ? f : nf - 1);
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) qf[r][ks] = *reinterpret_cast<const Frag*>(p + (ks * KS + E * (lane >> 4)) * EB);
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) oacc[r][dt] = f32x4{};
      m[r] = -__builtin_inff();
      l[r] = 0.0f;
    }
  }

  // A 32-key tile from its LDS stage. masked: keys that are not ok or after the row do not count.
  __device__ __forceinline__ void step(const char* st, int tile, uint64_t ok, bool masked, float c, int lane) {
    const int q = lane >> 4, l16 = lane & 15;
    f32x4 s[NR][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int r = 0; r < NR; ++r) s[r][t] = f32x4{};
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        const Frag kf = *reinterpret_cast<const Frag*>(st + ST::k_off(16 * t + l16, ks * KS + E * q));
#pragma unroll
        for (int r = 0; r < NR; ++r) s[r][t] = EL::mma(kf, qf[r][ks], s[r][t]);
      }
    }
    if (masked) {
      asm volatile("");  // a branch, not selects in every tile
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const int rel = pos[r] < 0 ? -1 : pos[r] - tile * 32;  // keys 0 .. rel are at or before the row
        const uint32_t see = ((uint32_t)ok & (rel < 0 ? 0u : rel >= 31 ? ~0u : (2u << rel) - 1)) >> (4 * q);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (!((see >> (16 * t + v)) & 1)) s[r][t][v] = -__builtin_inff();
      }
    }
    // bf16: P as a pair hi + lo, to about 2^-17, as in the per-query forward. The
    // second product takes 1% of the time here, and O's error is then its rounding's.
    Frag pf[NR], plo[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float mx = fmaxf(fmaxf(fmaxf(s[r][0][0], s[r][0][1]), fmaxf(s[r][0][2], s[r][0][3])),
                       fmaxf(fmaxf(s[r][1][0], s[r][1][1]), fmaxf(s[r][1][2], s[r][1][3])));
      float other = mx;
      swap16(mx, other);
      mx = half_max(fmaxf(mx, other));
      const bool up = mx > m[r] + slack(c);  // the first finite score too: m = -inf
      if (__any(up)) {
        const float mn = up ? mx : m[r];
        const float corr = up ? __builtin_amdgcn_exp2f((m[r] - mn) * c) : 1.0f;
        m[r] = mn;
        l[r] *= corr;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) oacc[r][dt] *= corr;
      }
      const float mc = m[r] == -__builtin_inff() ? 0.0f : m[r] * c;  // nothing attended yet: every p is 0
      float sum = 0.0f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          s[r][t][v] = __builtin_amdgcn_exp2f(fmaf(s[r][t][v], c, -mc));
          sum += s[r][t][v];
        }
      l[r] += sum;
      if constexpr (EB == 2)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = s[r][j >> 2][j & 3];
          pf[r][j] = (__bf16)p;
          plo[r][j] = (__bf16)(p - (float)pf[r][j]);
        }
    }
    if constexpr (EB == 2) {
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        typedef __attribute__((address_space(3))) s16x4* lds_s4;
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const char* p = st + ST::v_off(4 * q + (l16 >> 2), 16 * dt + 4 * (l16 & 3));
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)p);
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(p + 16 * ST::kVPitch));
        const Frag vf = __builtin_bit_cast(Frag, (s16x8)__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int r = 0; r < NR; ++r) oacc[r][dt] = EL::mma(vf, plo[r], EL::mma(vf, pf[r], oacc[r][dt]));
      }
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const float vf = *reinterpret_cast<const float*>(st + ST::v_off(16 * t + 4 * q + v, 16 * dt + l16));
#pragma unroll
            for (int r = 0; r < NR; ++r) oacc[r][dt] = EL::mma(vf, s[r][t][v], oacc[r][dt]);
          }
    }
  }

  // bf16: whether the products left O finite, by its sum (a sum that overflows only has
  // its tiles looked at). An infinity of V is one by P's high half, but NaN by a low half
  // of zero, or by one of the other sign.
  __device__ __forceinline__ bool finite() const {
    if constexpr (EB == 4) return true;
    f32x4 z = f32x4{};
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) z += oacc[r][dt];
    return !__any(!(fabsf((z[0] + z[1]) + (z[2] + z[3])) < __builtin_inff()));
  }

  // Adds what masked tiles left out, and puts it in the place of what the products made
  // of it in the others.
  template <bool F8>
  __device__ inline void add_bad(const KvItem& a, int first, int last, int stride, int sub, int first_pos, int lane) {
    static_assert(NR * NDT * 4 <= 32, "a bit for each element");
    uint32_t spoilt = 0;
    if constexpr (EB == 2) {
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (!(fabsf(oacc[r][dt][v]) < __builtin_inff())) spoilt |= 1u << ((r * NDT + dt) * 4 + v);
    }
    const bool all = __any(spoilt != 0);
    bad_rows<T, D, 32, F8>(a, first, last, stride, sub, first_pos, all, lane, [&](int t, const char* row, float scale) {
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float x = not_finite<T, F8>(row, scale, 16 * dt + 4 * (lane >> 4) + v);
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            if (x == 0.0f || pos[r] < t) continue;
            const uint32_t bit = 1u << ((r * NDT + dt) * 4 + v);
            oacc[r][dt][v] = spoilt & bit ? x : oacc[r][dt][v] + x;
            spoilt &= ~bit;
          }
        }
    });
  }
};

}  // namespace

// Up to 16 NR folded rows per item (NR = 2 with d = 64 only: with 128 the form of
// 256 rows was faster from 17 rows on): the four waves take every fourth unit
// each, on the same rows, with LDS of their own and no barrier; their results
// are joined at the item's end. Tiles of 32 keys, so that two workgroups fit a CU and
// one's rows are under way while the other begins or ends an item. A unit is a
// tile, or two of 8-bit rows, whose loads are under way at once: either way 16 KB a
// wave and 128 KB a CU, about what the memory's latency takes. 16-row products
// although the matrix cores have time to spare: it is the instructions beside
// them that count (with 32 rows, 64 ragged contexts in 8 bits took 180 us, with 16
// and P rounded 175). What bounds it: the memory where contexts are long (eight
// of 131K in 8 bits 380 us, 5.7 TB/s), the starts and ends of items beside it where
// they are not (64 of 1K to 16K 180 us, 4.8 TB/s), and a chain of round trips for
// one short context (2K: 10 us, of which 2 are the launch, 1.5 the share, 5 the tile).
template <typename T, int D, bool F8, int NR>
__global__ __launch_bounds__(256, 2) void paged_few_kernel(PagedAttnArgs) {
  constexpr int UK = few_unit_keys(F8), SUB = (1 << UK) / 32, KT = 32, NW = 4, M = 16 * NR, OP = D + 4;
  using W = FewRows<T, D, NR>;
  constexpr int SB = W::ST::kBytes > M * OP * 4 ? W::ST::kBytes : M * OP * 4;  // a wave's LDS: a stage, then its results
  __shared__ __attribute__((aligned(16))) char smem[NW * SB];
  __shared__ float s_m[NW][M], s_l[NW][M];
  __shared__ int64_t s_scan[NW + 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int shift = (NR == 1 ? 4 : 5) - args_here().gqa_shift, wg = share_index();
  const Share<UK> share = take_share<256, kPagedFewWorkgroups, UK, 0>(wg, shift, NW, NW, s_scan);
  const float c = args_here().scale_log2;
  char* st = smem + wave * SB;
  walk<0>(share, wg, shift, [&](const Share<UK>& sh, int n, bool whole) {
    const SeqShape<UK>& q = sh.q;
    const PagedAttnArgs& a0 = args_here();
    const int first_pos = q.pos((int64_t)sh.j << shift);
    const KvItem kv(a0.p, sh.s, sh.h, q.end(sh.j));
    W w;
    w.begin(a0, q, sh.h, (int64_t)sh.j * M, lane);
    const int last = sh.kt + n, x0 = sh.kt + wave;
    // slot i holds the rows of unit x's tile i; `map` the pages of the units to ask for
    TileRegs<T, D, typename W::ST, F8, 1> r[SUB];
    TileMap<(1 << UK), NW, 2 * SUB> map;
    bool full_now = false, full = false, bad = false;  // of unit x, and of the one asked for
    int x = x0, at = 0;
    auto ask = [&](int i, int u) __attribute__((always_inline)) {  // tile i of unit u
      if (i == 0) {
        if (at == 0) map.fill(kv, u, 0, lane);
        full = (map.full >> at) & 1;
      }
      const int page[2] = {__builtin_amdgcn_readlane(map.page[2 * i], at),
                           __builtin_amdgcn_readlane(map.page[2 * i + 1], at)};
      r[i].load(kv, u * SUB + i, page, 0, lane);
      if (i == SUB - 1) at = (at + 1) & 63;
    };
    auto tile = [&](int i, auto more) __attribute__((always_inline)) {
      // positions after the first row lie in this tile, or some are not there
      const int y = x * SUB + i;
      uint64_t ok = ~0ull;
      bool masked = y * KT + KT - 1 > first_pos;
      if (!full_now) {  // of the unit: this tile may be
        ok = present<KT>(kv, y, lane);
        masked = masked || ok != all_keys<KT>();
      }
      bad = r[i].store(st, ok, masked, 0, lane) || bad;
      __builtin_amdgcn_wave_barrier();
      if constexpr (more.value) ask(i, x + NW);
      w.step(st, y, ok, masked, c, lane);
      __builtin_amdgcn_wave_barrier();
    };
    if (x < last) {
#pragma unroll
      for (int i = 0; i < SUB; ++i) ask(i, x);
      // The last unit apart: where a slot may or may not be asked for again, the
      // compiler waits for both before it takes either.
      for (; x + NW < last; x += NW) {
        full_now = full;
#pragma unroll
        for (int i = 0; i < SUB; ++i) tile(i, Yes());
      }
      full_now = full;
#pragma unroll
      for (int i = 0; i < SUB; ++i) tile(i, No());
    }
    if (bad || !w.finite()) w.template add_bad<F8>(kv, x0, last, NW, SUB, first_pos, lane);
    // join the waves: rows as [wave][row][D] through the stages
    const PagedAttnArgs& a = args_here();
    __syncthreads();
    float* so = reinterpret_cast<float*>(smem);
    const int q4 = lane >> 4, l16 = lane & 15;
#pragma unroll
    for (int g = 0; g < NR; ++g) {
      float l = w.l[g], other = l;
      swap16(l, other);
      l = half_sum(l + other);
      if (q4 == 0) {
        s_m[wave][16 * g + l16] = w.m[g];
        s_l[wave][16 * g + l16] = l;
      }
#pragma unroll
      for (int dt = 0; dt < W::NDT; ++dt)
        *reinterpret_cast<f32x4*>(so + (wave * M + 16 * g + l16) * OP + 16 * dt + 4 * q4) = w.oacc[g][dt];
    }
    __syncthreads();
    const int64_t nf = (int64_t)q.n << a.gqa_shift, f0 = (int64_t)sh.j * M;
    const int rows = nf - f0 < M ? (int)(nf - f0) : M;
    const int64_t slot = (int64_t)wg * 2 + (sh.kt == 0 ? 1 : 0);
    for (int it = tid; it < rows * (D / 4); it += 256) {
      const int row = it / (D / 4), d4 = it % (D / 4);
      float mx = -__builtin_inff();
#pragma unroll
      for (int k = 0; k < NW; ++k) mx = fmaxf(mx, s_m[k][row]);
      float L = 0.0f;
      f32x4 o = f32x4{};
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        const float f = s_m[k][row] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((s_m[k][row] - mx) * c);
        L += s_l[k][row] * f;
        o += *reinterpret_cast<const f32x4*>(so + (k * M + row) * OP + 4 * d4) * f;
      }
      if (whole) {
        float* lse;
        char* dst = out_row(a, q.first, sh.h, f0 + row, lse);
        store4(dst + d4 * 4 * W::EB, o * (L == 0.0f ? 0.0f : 1.0f / L), W::EB == 2);
        if (d4 == 0) *lse = lse_of(mx, L, c);
      } else {
        *reinterpret_cast<f32x4*>(a.part + (slot * a.slot_rows + row) * D + 4 * d4) = o;
        if (d4 == 0) {
          a.part_ml[(slot * a.slot_rows + row) * 2] = mx;
          a.part_ml[(slot * a.slot_rows + row) * 2 + 1] = L;
        }
      }
    }
    __syncthreads();
  });
}

// ---------------------------------------------------------------- many rows

// 256 folded rows per item, 32 per wave; the waves share each tile through three
// LDS stages. A wave works on 32 keys at a time, in two phases that keep the
// matrix cores and the vector unit busy at once: the next 32 keys' scores beside
// these' exponentials, then these' P.V beside the next maximum. Tile x + 1 is
// staged before tile x is begun, so the phases run on across tiles; x + 2 goes
// to the third stage meanwhile. P is rounded to bf16, as in the routed forward (a
// pair would add half to the products).
//
// What bounds it: 2,048 rows of 32 heads at the end of 32K (bf16 rows) take
// 0.99 to 1.10 ms by the card, 0.97 to 1.07 PFLOP/s (0.87 ms on zeros: the clock
// falls under the power of products of real values, to 1.7 GHz where calls run one at
// a time). A product takes 32 cycles of a matrix core, which is busy half of the
// time, and there are 5.2 vector instructions beside each: 32 keys of a wave have 16
// products, 16 exponentials and some 70 others. 76 of 100 reads of keys are L2
// hits. Without the staging of tiles it took 0.71 ms on zeros. Longer operand
// queues, wave priorities, staggered waves and the exponentials spread over both
// kinds of product changed it by 1% at most; one phase after the other, 1.10 ms.
template <typename T, int D, bool F8>
__global__ __launch_bounds__(512) void paged_tile_kernel(PagedAttnArgs) {
  constexpr int KT = 1 << kPagedTileKeys, NW = 8;
  using W = WaveRows<T, D, KT>;
  using Frag = typename W::Frag;
  constexpr int SB = W::ST::kBytes;
  // the least share, in units: what a unit takes (bf16 2 us, float32 7) against a
  // partial result's writing and joining
  constexpr int kLeast = sizeof(T) == 2 ? 4 : 1;
  // units for an item's start and end (about 6 us): a prompt of 8,192 rows from its
  // beginning 695 us with none, 645 with two, 622 with three
  constexpr int kOver = sizeof(T) == 2 ? 3 : 1;
  __shared__ __attribute__((aligned(16))) char smem[3 * SB];
  __shared__ int64_t s_scan[NW + 2];
  __shared__ int s_bad[2];  // whether V had what is not finite in this item, and in the next
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int shift = kPagedTileRowsLog2 - args_here().gqa_shift, wg = share_index();
  const Share<kPagedTileKeys> share = take_share<512, kPagedTileWorkgroups, kPagedTileKeys, kOver>(wg, shift, 1, kLeast, s_scan);
  const float c = args_here().scale_log2;
  if (tid < 2) s_bad[tid] = 0;
  __syncthreads();
  int item = 0;
  walk<kOver>(share, wg, shift, [&](const Share<kPagedTileKeys>& sh, int n, bool whole) {
    const SeqShape<kPagedTileKeys>& q = sh.q;
    const PagedAttnArgs& a0 = args_here();
    const int first_pos = q.pos((int64_t)sh.j << shift);
    const KvItem kv(a0.p, sh.s, sh.h, q.end(sh.j));
    const int64_t nf = (int64_t)q.n << a0.gqa_shift, f0 = (int64_t)sh.j * kPagedTileRows + 32 * wave;
    W w;
    w.begin(a0, q, sh.h, f0, lane);
    const bool active = f0 < nf;  // else the wave only stages
    const int wave_first = q.pos(f0 >> a0.gqa_shift);
    const int last = sh.kt + n;
    int x = sh.kt;
    TileRegs<T, D, typename W::ST, F8, NW> r;
    constexpr int IPW = TileRegs<T, D, typename W::ST, F8, NW>::IPW, NI = TileRegs<T, D, typename W::ST, F8, NW>::NI;
    TileMap<KT, 1, 1> map;
    const int block = (wave * IPW % NI) * TileRegs<T, D, typename W::ST, F8, NW>::R / 16, x0 = x;
    int asked = 0;
    bool full = false;  // of the tile in r
    auto ask = [&]() __attribute__((always_inline)) {
      const int at = asked & 63;
      if (at == 0) map.fill(kv, x0 + asked, block, lane);
      const int page[1] = {__builtin_amdgcn_readlane(map.page[0], at)};
      full = (map.full >> at) & 1;
      r.load(kv, x0 + asked, page, wave, lane);
      ++asked;
    };
    // stages of tiles x, x + 1, x + 2, and which of their keys are there
    char *st0 = smem, *st1 = smem + SB, *st2 = smem + 2 * SB;
    uint64_t ok0, ok1 = 0, ok2 = 0;
    auto put = [&](int y, char* st, uint64_t& ok) __attribute__((always_inline)) {
      ok = ~0ull;
      if (!full) ok = present<KT>(kv, y, lane);
      const bool masked = y * KT + KT - 1 > first_pos || !full;
      if (r.store(st, ok, masked, wave, lane)) s_bad[item & 1] = 1;
    };
    ask();
    put(x, st0, ok0);
    if (x + 1 < last) {
      ask();
      put(x + 1, st1, ok1);
      if (x + 2 < last) ask();
    }
    __syncthreads();
    if (tid == 0) s_bad[(item + 1) & 1] = 0;  // read after the last item's loop, set in the next one's
    auto masked = [&](int y, uint64_t ok) { return y * KT + KT - 1 > wave_first || ok != ~0ull; };
    f32x16 s0, s1;
    typename W::Probs pf;
    constexpr Yes yes;
    constexpr No no;
    Frag fr[W::RING];
    // Keys of tile y that do not count, where it has such: a branch (its empty asm
    // keeps it one; as selects it would run in every tile). With a form of the loop for
    // tiles without masks the accumulators had two places, and 97 registers went to memory.
    auto hide = [&](f32x16& s, int y, int t, uint64_t ok) __attribute__((always_inline)) {
      if (masked(y, ok)) {
        asm volatile("");
        w.hide(s, y, t, ok, lane);
      }
    };
    // tile x, with the scores of its first half in s0; leaves those of the next tile's
    auto both = [&](auto more) __attribute__((always_inline)) {
      auto hide1 = [&]() __attribute__((always_inline)) { hide(s1, x, 1, ok0); };
      auto hide0 = [&]() __attribute__((always_inline)) { if constexpr (more.value) hide(s0, x + 1, 0, ok1); };
      if constexpr (sizeof(T) == 2) {
        w.template half<true>(s0, s1, fr, st0, 0, st0, 1, st1, 0, c, lane, hide1);
        w.template half<more.value>(s1, s0, fr, st0, 1, st1, 0, st1, 1, c, lane, hide0);
      } else {
        w.scores(s1, st0, 1, lane);
        w.probs(s0, pf, c);
        hide1();
        w.values(pf, st0, 0, lane);
        w.raise(W::row_max(s1), c);
        if constexpr (more.value) w.scores(s0, st1, 0, lane);
        w.probs(s1, pf, c);
        hide0();
        w.values(pf, st0, 1, lane);
        if constexpr (more.value) w.raise(W::row_max(s0), c);
      }
    };
    if (active) {
      w.scores(s0, st0, 0, lane);
      hide(s0, x, 0, ok0);
      w.raise(W::row_max(s0), c);
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < W::RING; ++i) fr[i] = W::k_frag(st0, 1, i, lane);
      }
    }
    for (; x + 1 < last; ++x) {
      if (active) both(yes);
      if (x + 2 < last) {
        put(x + 2, st2, ok2);
        if (x + 3 < last) ask();
      }
      __syncthreads();
      char* st = st0;
      st0 = st1; st1 = st2; st2 = st;
      ok0 = ok1; ok1 = ok2;
    }
    if (active) both(no);
    __syncthreads();  // the last stage is no longer read
    if (s_bad[item++ & 1] && active) w.template add_bad<F8>(kv, x0, last, first_pos, lane);
    // A lane holds half the head dim of one row, so stores from registers would
    // scatter over 32 rows each; the wave's rows go through its share of the
    // stages instead and leave with consecutive lanes on consecutive pieces.
    const PagedAttnArgs& a = args_here();
    const float l = half_sum(w.l);
    const int hh = lane >> 5, l32 = lane & 31;
    constexpr int EB = W::EB, SHARE = 3 * SB / NW / 16 * 16, OP = D * EB + 16, HP = D / 2 * 4 + 16;
    static_assert(32 * OP <= SHARE && 32 * HP <= SHARE, "a wave's rows fit its share");
    char* ost = smem + wave * SHARE;
    const int rows = nf - f0 < 32 ? (int)(nf - f0) : 32;  // of the wave; none if not active
    if (whole) {
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
      for (int dt = 0; dt < W::NDT; ++dt)
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4)
          store4(ost + l32 * OP + (32 * dt + 8 * v4 + 4 * hh) * EB,
                 f32x4{w.oacc[dt][4 * v4], w.oacc[dt][4 * v4 + 1], w.oacc[dt][4 * v4 + 2], w.oacc[dt][4 * v4 + 3]} *
                     inv,
                 EB == 2);
      float* lse;
      if (l32 < rows && hh == 0) {
        out_row(a, q.first, sh.h, f0 + l32, lse);
        *lse = lse_of(w.m, l, c);
      }
      __builtin_amdgcn_wave_barrier();
      constexpr int CPR = D * EB / 16;
#pragma unroll
      for (int i = 0; i < 32 * CPR / 64; ++i) {
        const int r = (lane + 64 * i) / CPR, p = (lane + 64 * i) % CPR;
        if (r < rows)
          *reinterpret_cast<u32x4*>(out_row(a, q.first, sh.h, f0 + r, lse) + p * 16) =
              *reinterpret_cast<const u32x4*>(ost + r * OP + p * 16);
      }
    } else {
      const int64_t at = ((int64_t)wg * 2 + (sh.kt == 0 ? 1 : 0)) * a.slot_rows + 32 * wave;
      if (l32 < rows && hh == 0) {
        a.part_ml[(at + l32) * 2] = w.m;
        a.part_ml[(at + l32) * 2 + 1] = l;
      }
      constexpr int HD = W::NDT / 2, CPR = D / 2 * 4 / 16;
#pragma unroll
      for (int half = 0; half < 2; ++half) {  // float32 rows: half the head dim at a time
#pragma unroll
        for (int dt = half * HD; dt < (half + 1) * HD; ++dt)
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4)
            *reinterpret_cast<f32x4*>(ost + l32 * HP + (32 * (dt - half * HD) + 8 * v4 + 4 * hh) * 4) =
                f32x4{w.oacc[dt][4 * v4], w.oacc[dt][4 * v4 + 1], w.oacc[dt][4 * v4 + 2], w.oacc[dt][4 * v4 + 3]};
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 32 * CPR / 64; ++i) {
          const int r = (lane + 64 * i) / CPR, p = (lane + 64 * i) % CPR;
          if (r < rows)
            *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(a.part + (at + r) * D + half * (D / 2)) + p * 16) =
                *reinterpret_cast<const u32x4*>(ost + r * HP + p * 16);
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
    __syncthreads();  // the stages are free again
  });
}

// ---------------------------------------------------------------- the joining

// Workgroups for the parts that one share may leave, of 8 / split rows each.
__host__ __device__ inline int join_groups(const PagedAttnArgs& a, int m_rows, int split) {
  const int rows = a.slot_rows < m_rows ? a.slot_rows : m_rows, per = 8 / split;
  return (rows + per - 1) / per;
}

// An item that shares w, w + 1, ... cut: its parts in the order of the keys. A
// workgroup joins eight rows by half a wave each, or two by `SPLIT` = four each
// (every fourth part): the lanes read 32 parts' maxima and sums at once and hand
// the weights round, and the parts' rows are read eight at a time. What bounds it
// is that chain of four round trips (4 us); where parts are many, several such (a
// row over 131,072 keys of two kv heads, 256 parts: 13 us by four, 41 by one); and
// where many rows are cut their bytes (20 us after a 2,048-row chunk's 256 shares).
// n_one: workgroups for the first form's parts.
template <typename T, int D, int SPLIT>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs one, int one_rows, int n_one, PagedAttnArgs two,
                                                         int two_rows) {
  constexpr int EB = Elem<T>::kBytes, V = D / 32;
  typedef float fV __attribute__((ext_vector_type(V)));
  const bool first = (int)blockIdx.x < n_one;
  const PagedAttnArgs& a = first ? one : two;
  const int m_rows = first ? one_rows : two_rows, groups = join_groups(a, m_rows, SPLIT);
  const int id = first ? blockIdx.x : blockIdx.x - n_one, wg = id / groups;
  const int4 rec = a.info[wg];
  if (rec.x == 0) return;
  const SeqShape<6> q = shape_of<6>(a, rec.y, 0);
  const int64_t nf = (int64_t)q.n << a.gqa_shift, f0 = (int64_t)rec.w * m_rows;
  const int half = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = id % groups * (8 / SPLIT) + half / SPLIT, begin = half % SPLIT;
  const bool live = row < m_rows && f0 + row < nf;
  if (SPLIT == 1 && !live) return;
  const int parts = SPLIT == 1 || live ? rec.x : 0;  // SPLIT == 1: the same in the whole workgroup
  const float c = a.scale_log2;
  // part k is the share wg + k's: the first one its last item, the others their first
  auto at = [&](int k) { return ((int64_t)(wg + k) * 2 + (k == 0 ? 1 : 0)) * a.slot_rows + row; };
  float M = -__builtin_inff(), L = 0.0f;
  fV o = fV{};
  auto raise = [&](float m) {
    if (m > M) {
      const float f = __builtin_amdgcn_exp2f((M - m) * c);
      L *= f;
      o *= f;
      M = m;
    }
  };
  auto weight = [&](float m) { return m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - M) * c); };
  for (int k0 = begin; k0 < parts; k0 += 32 * SPLIT) {
    const int rest = (parts - k0 + SPLIT - 1) / SPLIT, n = rest < 32 ? rest : 32;
    float m = -__builtin_inff(), l = 0.0f;
    if (lane < n) {
      m = a.part_ml[at(k0 + lane * SPLIT) * 2];
      l = a.part_ml[at(k0 + lane * SPLIT) * 2 + 1];
    }
    float mx = m;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d, 32));
    raise(mx);
    const float f = weight(m);
    l *= f;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) l += __shfl_xor(l, d, 32);
    L += l;
    for (int k = 0; k < n; k += 8) {
      fV x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x[i] = *reinterpret_cast<const fV*>(a.part + at(k0 + (k + i < n ? k + i : n - 1) * SPLIT) * D + lane * V);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float w = __shfl(f, k + i < n ? k + i : 0, 32);
        if (k + i < n) o += x[i] * w;
      }
    }
  }
  if constexpr (SPLIT > 1) {
    __shared__ fV s_o[8][32];
    __shared__ float s_m[8], s_l[8];
    s_o[half][lane] = o;
    if (lane == 0) {
      s_m[half] = M;
      s_l[half] = L;
    }
    __syncthreads();
    if (begin != 0) return;
    for (int j = 1; j < SPLIT; ++j) {
      raise(s_m[half + j]);
      const float f = weight(s_m[half + j]);
      L += s_l[half + j] * f;
      o += s_o[half + j][lane] * f;
    }
  }
  if (!live) return;
  o *= L == 0.0f ? 0.0f : 1.0f / L;
  float* lse;
  char* dst = out_row(a, q.first, rec.z, f0 + row, lse) + lane * V * EB;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if constexpr (EB == 2) reinterpret_cast<uint16_t*>(dst)[v] = (uint16_t)float_to_bf16_bits(o[v]);
    else reinterpret_cast<float*>(dst)[v] = o[v];
  }
  if (lane == 0) *lse = lse_of(M, L, c);
}

template <typename T, int D, bool F8>
static hipError_t attend_dispatch(const PagedAttnArgs* a, const PagedForm* form, int n, int split, hipStream_t s) {
  int join[2] = {0, 0};
  for (int i = 0; i < n; ++i) {
    const dim3 grid(paged_workgroups(form[i]));
    if (form[i] == PagedForm::kFew16) hipLaunchKernelGGL((paged_few_kernel<T, D, F8, 1>), grid, dim3(256), 0, s, a[i]);
    else if (form[i] == PagedForm::kTile) hipLaunchKernelGGL((paged_tile_kernel<T, D, F8>), grid, dim3(512), 0, s, a[i]);
    else if constexpr (D == 64) hipLaunchKernelGGL((paged_few_kernel<T, D, F8, 2>), grid, dim3(256), 0, s, a[i]);
    else return hipErrorInvalidValue;  // d = 128 has no form of 32 rows
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    join[i] = paged_workgroups(form[i]) * join_groups(a[i], paged_rows(form[i]), split);
  }
  auto* kernel = split == 1 ? paged_join_kernel<T, D, 1> : paged_join_kernel<T, D, 4>;
  hipLaunchKernelGGL(kernel, dim3(join[0] + join[1]), dim3(256), 0, s, a[0], paged_rows(form[0]), join[0], a[n - 1],
                     paged_rows(form[n - 1]));
  return hipGetLastError();
}

hipError_t launch_attend_paged(const PagedAttnArgs* a, const PagedForm* form, int n, int split, bool e4m3, bool bf16,
                               int head_dim, hipStream_t s) {
  auto* f = bf16 && head_dim == 128 ? (e4m3 ? attend_dispatch<__bf16, 128, true> : attend_dispatch<__bf16, 128, false>)
            : bf16                  ? (e4m3 ? attend_dispatch<__bf16, 64, true> : attend_dispatch<__bf16, 64, false>)
                                    : (e4m3 ? attend_dispatch<float, 64, true> : attend_dispatch<float, 64, false>);
  return f(a, form, n, split, s);  // float32: head_dim 64
}

}  // namespace hga
