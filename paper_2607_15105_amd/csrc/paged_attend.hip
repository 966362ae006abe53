// Attention of a ragged batch of new rows over the paged cache: row r of
// sequence s, at position p = q_begin[s] + r - seq_rows[s], attends the cached
// positions t <= p whose page is present.
//
// The rows of a sequence and kv head are folded with its G query heads, so
// that one reading of K and V serves them all, and taken M folded rows at a
// time: an item is (sequence, kv head, row tile), a unit of work one 64-key
// tile of an item. Lengths live on the device; every workgroup counts the
// units of all sequences, takes an equal share of their concatenation and
// finds its first unit. Shares differ by one unit at most however ragged the
// batch is, and a long context of few rows spreads over the whole GPU. An item that lies
// in one share is finished there; one that several shares cut is left as
// partial results (unnormalised O with its maximum and sum), which a second
// kernel joins in the order of the keys: no atomics, the same bits every run.
//
// Softmax as in the routed kernels: S^T = K . Q^T, every lane holds scores of
// one row, running maximum and sum per lane, the maximum raised lazily, O^T +=
// V^T . P^T straight from the score registers.
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

  __device__ inline int nt() const { return (n + (1 << shift) - 1) >> shift; }
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
  __device__ inline int64_t units() const { return n == 0 ? 0 : before(nt() - 1) + tiles(nt() - 1); }
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
  int kt;           // first unit within the item
  SeqShape<KS> q;   // of sequence s
};

// NT threads, W workgroups; `lds` holds NT / 64 + 2 int64. A share is a multiple of `step` units, `least` at least.
template <int NT, int W, int KS>
__device__ inline Share<KS> take_share(int wg, int shift, int step, int least, int64_t* lds) {
  constexpr int NW = NT / 64;
  const PagedAttnArgs& a = args_here();
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n_seqs = a.p.n_seqs, c = (n_seqs + NT - 1) / NT;
  int64_t sum = 0;
  for (int k = 0; k < c; ++k) {
    const int s = tid * c + k;
    if (s < n_seqs) sum += a.p.n_kv_heads * shape_of<KS>(a, s, shift).units();
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
      const int64_t m = a.p.n_kv_heads * shape_of<KS>(a, s, shift).units();
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
    const int64_t m = sh.q.units();
    // kv head and rest: 32-bit division where it will do
    int h = m < ((int64_t)1 << 31) && off < ((int64_t)1 << 31) ? (int)((uint32_t)off / (uint32_t)m) : (int)(off / m);
    sh.h = __builtin_amdgcn_readfirstlane(h);
    off -= sh.h * m;
    int lo = 0, hi = sh.q.nt() - 1;  // the last row tile that begins at or before off
    while (lo < hi) {
      const int mid = (int)(((int64_t)lo + hi + 1) >> 1);
      if (sh.q.before(mid) <= off) lo = mid;
      else hi = mid - 1;
    }
    sh.j = __builtin_amdgcn_readfirstlane(lo);
    sh.kt = __builtin_amdgcn_readfirstlane((int)(off - sh.q.before(sh.j)));
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
};

// Pages of a tile's KT positions (32 or 64), a position per lane. `entry` is the table's
// entry as loaded, or -1; nothing looks at it before use(), so the load can be
// under way beside the tile before it. (Loads return in order: a wait for the
// entry right after it was asked for is a wait for every row asked for before
// it. With that, 64 ragged contexts took 343 us, 8-bit rows; a 2,048-token chunk at the
// end of 32K 1,383 us.)
template <int KT>
struct TileKeys {
  static constexpr uint64_t kAll = KT == 64 ? ~0ull : (1ull << KT) - 1;
  int entry;
  int page;       // 0 where there is none
  uint64_t ok;    // positions that are present and before the item's end
  uint32_t ks, vs;  // the rows' scale bytes

  __device__ inline void ask(const KvItem& a, int tile, int lane) {
    const int t = tile * KT + lane;
    entry = -1;
    if (lane < KT && t < a.end) entry = a.table[t >> a.shift];
  }
  __device__ inline void use(const KvItem& a) {
    const bool there = (uint32_t)entry < (uint32_t)a.n_pages;
    ok = __ballot(there);
    page = there ? entry : 0;
  }
  template <bool F8>
  __device__ inline void ask_scales(const KvItem& a, int tile, int lane) {
    if constexpr (F8) {
      const uint64_t o = (uint64_t)(uint32_t)page * a.scale_page + (uint32_t)((tile * KT + lane) & a.mask);
      ks = a.k_scale[o];
      vs = a.v_scale[o];
    }
  }
};

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
template <typename T, int D, int KT>
struct Stage {
  using TL = Tile<T, D>;
  static constexpr bool TR = Elem<T>::kBytes == 2;
  static constexpr int kV = KT * TL::kRowPitch;  // offset of V
  static constexpr int kBytes = kV + (TR ? KT * TL::kRowPitch : D * (KT + 1) * 4);
  // element (d, kpos) of the transposed V
  __device__ static inline int t_off(int d, int kpos) { return kV + (d * (KT + 1) + kpos) * 4; }
};

// One wave's share (of NW waves) of a KT-key tile of K and V, in registers. A
// load instruction covers R whole rows; pages hold 16 tokens or more, so 16 rows
// lie in one page and have one scalar address.
template <typename T, int D, int KT, bool F8, int NW>
struct TileRegs {
  using TL = Tile<T, D>;
  using ST = Stage<T, D, KT>;
  static constexpr int EB = Elem<T>::kBytes;
  static constexpr int PPR = (F8 ? D : D * EB) / 16;  // 16-byte pieces of a held row
  static constexpr int R = 64 / PPR;
  static constexpr int NI = KT / R;                   // instructions per tensor
  static constexpr int IPW = 2 * NI / NW;
  static constexpr int IPB = 16 / R;                  // instructions per 16 rows
  static constexpr int PE = F8 ? 16 : 16 / EB;        // elements of a piece
  static_assert(IPW % IPB == 0, "a wave loads whole blocks of 16 rows");
  u32x4 w[IPW];

  __device__ inline void load(const KvItem& a, int tile, int page, int wave, int lane) {
#pragma unroll
    for (int b = 0; b < IPW / IPB; ++b) {
      const int j = wave * IPW + b * IPB, row = (j % NI) * R;
      const bool v = j >= NI;
      const uint32_t pg = (uint32_t)__builtin_amdgcn_readlane(page, row), slot = (uint32_t)((tile * KT + row) & a.mask);
      const uint32_t tok = v ? a.v_tok : a.k_tok;
      const char* base = (v ? a.v : a.k) + ((uint64_t)pg * (v ? a.v_page : a.k_page) + (uint64_t)slot * tok);
#pragma unroll
      for (int i = 0; i < IPB; ++i)
        w[b * IPB + i] = *reinterpret_cast<const u32x4*>(base + (uint32_t)((lane / PPR + i * R) * tok + (lane % PPR) * 16));
    }
  }

  // Into the LDS stage. masked: rows that are not ok are zeros, and what is not
  // finite in V is left out; returns the rows of V that have such elements.
  __device__ inline uint64_t store(char* st, const TileKeys<KT>& k, bool masked, int wave, int lane) const {
    uint64_t bad = 0;
#pragma unroll
    for (int i = 0; i < IPW; ++i) {
      const int j = wave * IPW + i, row0 = (j % NI) * R, row = row0 + lane / PPR;
      const bool v = j >= NI;
      uint4 out[PE * EB / 16];
      if constexpr (F8) {
        const float sc = __uint_as_float((uint32_t)__shfl((int)(v ? k.vs : k.ks), row, 64) << 23);
#pragma unroll
        for (int o = 0; o < PE * EB / 16; ++o) {
          uint32_t c[Codes<T>::kWords];
#pragma unroll
          for (int x = 0; x < Codes<T>::kWords; ++x) c[x] = w[i][o * Codes<T>::kWords + x];
          out[o] = Codes<T>::decode(c, sc);
        }
      } else {
        out[0] = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
      }
      if (masked) {
        const bool ok = (k.ok >> row) & 1;
        bool fine = true;
#pragma unroll
        for (int o = 0; o < PE * EB / 16; ++o) {
          if (!ok) out[o] = make_uint4(0u, 0u, 0u, 0u);
          if (v && !finite16<T>(out[o])) {
            fine = false;
            out[o] = only_finite<T>(out[o]);
          }
        }
        uint64_t lanes = __ballot(!fine);
        while (lanes) {
          const int l = __builtin_ctzll(lanes);
          lanes &= lanes - 1;
          bad |= 1ull << (row0 + l / PPR);
        }
      }
#pragma unroll
      for (int o = 0; o < PE * EB / 16; ++o) {
        const int e = (lane % PPR) * PE + o * 16 / EB;
        if (EB == 2 || !v) {
          *reinterpret_cast<uint4*>(st + (v ? ST::kV : 0) + TL::row_off(row, e)) = out[o];
        } else {
          const uint32_t x[4] = {out[o].x, out[o].y, out[o].z, out[o].w};
          const int kp = kpos_of<Elem<T>::E>(row);
#pragma unroll
          for (int y = 0; y < 4; ++y)
            *reinterpret_cast<uint32_t*>(st + ST::t_off(e + y, kp)) = x[y];
        }
      }
    }
    return bad;
  }
};

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
  static constexpr int NH = KT / 32;
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
    int64_t f = f0 + (lane & 31);
    pos = f < nf ? q.pos(f >> a.gqa_shift) : -1;
    if (f >= nf) f = nf - 1;
    const int64_t row = q.first + (f >> a.gqa_shift);
    const int hq = (h << a.gqa_shift) + (int)(f & ((1 << a.gqa_shift) - 1));
    const char* p = row_ptr(a.Q, row, a.q_tok) + hq * a.q_head;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[ks] = EL::load_frag(p + (ks * KS + E * hh) * EB);
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) oacc[dt] = f32x16{};
    m = -__builtin_inff();
    l = 0.0f;
  }

  // One tile from its LDS stage. masked: keys that are not ok or after the row do not count.
  __device__ __forceinline__ void step(const char* st, int tile, uint64_t ok, bool masked, float c, int lane) {
    const int hh = lane >> 5, l32 = lane & 31;
    const float lazy = 8.0f / c;
    f32x16 s[NH];
#pragma unroll
    for (int t = 0; t < NH; ++t) s[t] = f32x16{};
#pragma unroll
    for (int t = 0; t < NH; ++t)
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        const Frag kf = EL::load_frag(st + TL::row_off(32 * t + l32, ks * KS + E * hh));
        s[t] = EL::mma(kf, qf[ks], s[t]);
      }
    if (masked) {
      const int rel = pos < 0 ? -1 : pos - tile * KT;  // keys 0 .. rel are at or before the row
      const uint64_t see = (ok & (rel < 0 ? 0 : rel >= 63 ? ~0ull : (2ull << rel) - 1)) >> (4 * hh);
#pragma unroll
      for (int t = 0; t < NH; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (!((see >> (32 * t + 8 * (v >> 2) + (v & 3))) & 1)) s[t][v] = -__builtin_inff();
    }
#pragma unroll
    for (int t = 0; t < NH; ++t) {
      float mx = -__builtin_inff();
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[t][v]);
      mx = half_max(mx);
      const bool raise = mx > m + lazy;  // the first finite score too: m = -inf
      if (__any(raise)) {
        const float mn = raise ? mx : m;
        const float corr = raise ? __builtin_amdgcn_exp2f((m - mn) * c) : 1.0f;
        m = mn;
        l *= corr;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) oacc[dt] *= corr;
      }
      const float mc = m == -__builtin_inff() ? 0.0f : m * c;  // nothing attended yet: every p is 0
      float sum = 0.0f;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s[t][v] = __builtin_amdgcn_exp2f(fmaf(s[t][v], c, -mc));
        sum += s[t][v];
      }
      l += sum;
#pragma unroll
      for (int s2 = 0; s2 < VPS; ++s2) {
        const int k = t * VPS + s2;
        float pv[E];
#pragma unroll
        for (int j = 0; j < E; ++j) pv[j] = s[t][E * s2 + j];
        const Frag pf = EL::frag_from(pv);  // bf16: P is rounded to the inputs' precision, as in the routed forward
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
          Frag vf;
          if constexpr (ST::TR) vf = tr_frag<TL>(st + ST::kV, 32 * dt, 16 * k + 4 * hh, 16 * k + 8 + 4 * hh, lane);
          else vf = EL::load_frag(st + ST::t_off(32 * dt + l32, KS * k + E * hh));
          oacc[dt] = EL::mma(vf, pf, oacc[dt]);
        }
      }
    }
  }

  // What is not finite in V was left out of the tile (a product with p = 0
  // would bring it to rows that do not attend its key): added here to the
  // rows that do.
  template <bool F8>
  __device__ inline void add_bad(const KvItem& a, int tile, uint64_t bad, int lane) {
    const int hh = lane >> 5;
    while (bad) {
      const int kk = __builtin_ctzll(bad);
      bad &= bad - 1;
      const int t = tile * KT + kk;
      if (pos < t) continue;
      const char* row = a.v + page_off(a.table[t >> a.shift], t & a.mask, a.v_page, a.v_tok);  // a row of the tile: present
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int d = 32 * dt + 8 * (v >> 2) + 4 * hh + (v & 3);
          float x;
          if constexpr (F8) x = (row[d] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f;
          else if constexpr (EB == 2) x = bf16_bits_to_float(*reinterpret_cast<const uint16_t*>(row + 2 * d));
          else x = *reinterpret_cast<const float*>(row + 4 * d);
          if (!(fabsf(x) < __builtin_inff())) oacc[dt][v] += x;
          __builtin_amdgcn_sched_barrier(0);  // one at a time: all at once, the comparisons take the loops' scalars
        }
    }
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

// The workgroup's place in the concatenation of all units: consecutive shares
// on one XCD (workgroups are dealt round-robin to the eight), whose L2 then holds what they share.
__device__ inline int share_index() { return (blockIdx.x & 7) * (gridDim.x / 8) + (blockIdx.x >> 3); }

// Follows a share item by item: f(share at the item, tiles of it, whether that is all of it), and the record of the one left unfinished.
template <int KS, typename F>
__device__ inline void walk(Share<KS> sh, int wg, int shift, F&& f) {
  if (threadIdx.x == 0) args_here().info[wg] = make_int4(0, 0, 0, 0);
  while (sh.left > 0) {
    const int len = sh.q.tiles(sh.j), rest = len - sh.kt;
    const int n = rest < sh.left ? rest : (int)sh.left;
    if (sh.kt == 0 && n < len) {  // goes on in the next shares: this one joins it
      const int64_t more = len - n;
      if (threadIdx.x == 0) args_here().info[wg] = make_int4((int)(1 + (more + sh.per - 1) / sh.per), sh.s, sh.h, sh.j);
    }
    f(sh, n, n == len);
    sh.left -= n;
    sh.kt = 0;
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

}  // namespace

// ---------------------------------------------------------------- few rows

// Up to 32 folded rows per item: the four waves take every fourth tile each,
// on the same rows, with LDS of their own and no barrier; their results are
// joined at the item's end. 32-key tiles, so that two workgroups fit a CU and
// one's rows are under way while the other begins or ends an item. 8-bit rows
// are asked for two tiles ahead, which keeps as many bytes under way as one of
// bf16 rows does (16 KB a wave, 128 KB a CU).
template <typename T, int D, bool F8>
__global__ __launch_bounds__(256, 2) void paged_few_kernel(PagedAttnArgs) {
  constexpr int KT = 1 << kPagedFewKeys, NW = 4, OP = D + 4, DEPTH = F8 ? 2 : 1;
  using W = WaveRows<T, D, KT>;
  constexpr int SB = W::ST::kBytes > 32 * OP * 4 ? W::ST::kBytes : 32 * OP * 4;  // a wave's LDS: a stage, then its results
  __shared__ __attribute__((aligned(16))) char smem[NW * SB];
  __shared__ float s_m[NW][32], s_l[NW][32];
  __shared__ int64_t s_scan[NW + 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int shift = kPagedFewRowsLog2 - args_here().gqa_shift, wg = share_index();
  const Share<kPagedFewKeys> share = take_share<256, kPagedFewWorkgroups, kPagedFewKeys>(wg, shift, NW, NW, s_scan);
  const float c = args_here().scale_log2;
  char* st = smem + wave * SB;
  walk(share, wg, shift, [&](const Share<kPagedFewKeys>& sh, int n, bool whole) {
    const SeqShape<kPagedFewKeys>& q = sh.q;
    const PagedAttnArgs& a0 = args_here();
    const int first_pos = q.pos((int64_t)sh.j << shift);
    const KvItem kv(a0.p, sh.s, sh.h, q.end(sh.j));
    W w;
    w.begin(a0, q, sh.h, (int64_t)sh.j * kPagedFewRows, lane);
    const int last = sh.kt + n;
    int x = sh.kt + wave;
    // slot i holds a tile's rows and keys; `next` the pages of the one to ask for next
    TileRegs<T, D, KT, F8, 1> r[DEPTH];
    TileKeys<KT> key[DEPTH], next;
    auto ask = [&](int i, int y) __attribute__((always_inline)) {
      key[i].entry = next.entry;
      key[i].use(kv);
      next.ask(kv, y + NW, lane);
      key[i].template ask_scales<F8>(kv, y, lane);
      r[i].load(kv, y, key[i].page, 0, lane);
    };
    next.ask(kv, x, lane);
#pragma unroll
    for (int i = 0; i < DEPTH; ++i)
      if (x + i * NW < last) ask(i, x + i * NW);
    while (x < last) {
#pragma unroll
      for (int i = 0; i < DEPTH; ++i) {
        if (x >= last) break;
        // positions after the first row lie in this tile, or some are not there
        const uint64_t ok = key[i].ok;
        const bool masked = x * KT + KT - 1 > first_pos || ok != key[i].kAll;
        const uint64_t bad = r[i].store(st, key[i], masked, 0, lane);
        __builtin_amdgcn_wave_barrier();
        if (x + DEPTH * NW < last) ask(i, x + DEPTH * NW);
        w.step(st, x, ok, masked, c, lane);
        if (bad) w.template add_bad<F8>(kv, x, bad, lane);
        __builtin_amdgcn_wave_barrier();
        x += NW;
      }
    }
    // join the waves: rows as [wave][row][D] through the stages
    const PagedAttnArgs& a = args_here();
    const float l = half_sum(w.l);
    __syncthreads();
    float* so = reinterpret_cast<float*>(smem);
    const int hh = lane >> 5, l32 = lane & 31;
    if (hh == 0) {
      s_m[wave][l32] = w.m;
      s_l[wave][l32] = l;
    }
#pragma unroll
    for (int dt = 0; dt < W::NDT; ++dt)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4)
        *reinterpret_cast<f32x4*>(so + (wave * 32 + l32) * OP + 32 * dt + 8 * v4 + 4 * hh) =
            f32x4{w.oacc[dt][4 * v4], w.oacc[dt][4 * v4 + 1], w.oacc[dt][4 * v4 + 2], w.oacc[dt][4 * v4 + 3]};
    __syncthreads();
    const int64_t nf = (int64_t)q.n << a.gqa_shift, f0 = (int64_t)sh.j * kPagedFewRows;
    const int rows = nf - f0 < kPagedFewRows ? (int)(nf - f0) : kPagedFewRows;
    const int64_t slot = (int64_t)wg * 2 + (sh.kt == 0 ? 1 : 0);
    for (int it = tid; it < rows * (D / 4); it += 256) {
      const int row = it / (D / 4), d4 = it % (D / 4);
      float M = -__builtin_inff();
#pragma unroll
      for (int k = 0; k < NW; ++k) M = fmaxf(M, s_m[k][row]);
      float L = 0.0f;
      f32x4 o = f32x4{};
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        const float f = s_m[k][row] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((s_m[k][row] - M) * c);
        L += s_l[k][row] * f;
        o += *reinterpret_cast<const f32x4*>(so + (k * 32 + row) * OP + 4 * d4) * f;
      }
      if (whole) {
        float* lse;
        char* dst = out_row(a, q.first, sh.h, f0 + row, lse);
        store4(dst + d4 * 4 * W::EB, o * (L == 0.0f ? 0.0f : 1.0f / L), W::EB == 2);
        if (d4 == 0) *lse = lse_of(M, L, c);
      } else {
        *reinterpret_cast<f32x4*>(a.part + (slot * a.slot_rows + row) * D + 4 * d4) = o;
        if (d4 == 0) {
          a.part_ml[(slot * a.slot_rows + row) * 2] = M;
          a.part_ml[(slot * a.slot_rows + row) * 2 + 1] = L;
        }
      }
    }
    __syncthreads();
  });
}

// ---------------------------------------------------------------- many rows

// 256 folded rows per item, 32 per wave; the waves share each tile, which is
// staged in LDS while the one before it is computed.
template <typename T, int D, bool F8>
__global__ __launch_bounds__(512) void paged_tile_kernel(PagedAttnArgs) {
  constexpr int KT = 1 << kPagedTileKeys, NW = 8;
  using W = WaveRows<T, D, KT>;
  constexpr int SB = W::ST::kBytes;
  __shared__ __attribute__((aligned(16))) char smem[2 * SB];
  __shared__ int64_t s_scan[NW + 2];
  __shared__ uint64_t s_bad[2][NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int shift = kPagedTileRowsLog2 - args_here().gqa_shift, wg = share_index();
  const Share<kPagedTileKeys> share = take_share<512, kPagedTileWorkgroups, kPagedTileKeys>(wg, shift, 1, 4, s_scan);
  const float c = args_here().scale_log2;
  walk(share, wg, shift, [&](const Share<kPagedTileKeys>& sh, int n, bool whole) {
    const SeqShape<kPagedTileKeys>& q = sh.q;
    const PagedAttnArgs& a0 = args_here();
    const int first_pos = q.pos((int64_t)sh.j << shift);
    const KvItem kv(a0.p, sh.s, sh.h, q.end(sh.j));
    const int64_t nf = (int64_t)q.n << a0.gqa_shift, f0 = (int64_t)sh.j * kPagedTileRows + 32 * wave;
    W w;
    w.begin(a0, q, sh.h, f0, lane);
    // the wave's rows lie at positions wave_first .. wave_last; none if f0 >= nf
    const int64_t f1 = f0 + 31 < nf ? f0 + 31 : nf - 1;
    const int wave_first = q.pos(f0 >> a0.gqa_shift), wave_last = f0 < nf ? q.pos(f1 >> a0.gqa_shift) : -1;
    const int last = sh.kt + n;
    int x = sh.kt;
    TileRegs<T, D, KT, F8, NW> r;
    TileKeys<KT> cur, nxt;
    auto ask = [&](int y) {
      cur.use(kv);
      nxt.ask(kv, y + 1, lane);
      cur.template ask_scales<F8>(kv, y, lane);
      r.load(kv, y, cur.page, wave, lane);
    };
    cur.ask(kv, x, lane);
    ask(x);
    auto put = [&](int tile, const TileKeys<KT>& k) {
      const bool masked = tile * KT + KT - 1 > first_pos || k.ok != k.kAll;
      const uint64_t bad = r.store(smem + (tile & 1) * SB, k, masked, wave, lane);
      if (masked && lane == 0) s_bad[tile & 1][wave] = bad;
    };
    put(x, cur);
    uint64_t ok = cur.ok;
    if (x + 1 < last) {
      cur = nxt;
      ask(x + 1);
    }
    __syncthreads();
    for (; x < last; ++x) {
      const bool staged = x * KT + KT - 1 > first_pos || ok != cur.kAll;
      if (x * KT <= wave_last && ok != 0) {  // else no row of the wave attends a key of the tile
        w.step(smem + (x & 1) * SB, x, ok, x * KT + KT - 1 > wave_first || ok != cur.kAll, c, lane);
        if (staged) {
          uint64_t bad = 0;
#pragma unroll
          for (int k = 0; k < NW; ++k) bad |= s_bad[x & 1][k];
          if (bad) w.template add_bad<F8>(kv, x, bad, lane);
        }
      }
      if (x + 1 < last) {
        put(x + 1, cur);
        ok = cur.ok;
        if (x + 2 < last) {
          cur = nxt;
          ask(x + 2);
        }
      }
      __syncthreads();
    }
    const PagedAttnArgs& a = args_here();
    const float l = half_sum(w.l);
    const int hh = lane >> 5, l32 = lane & 31;
    const int64_t f = f0 + l32;
    if (f < nf) {
      if (whole) {
        float* lse;
        char* dst = out_row(a, q.first, sh.h, f, lse);
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        if (hh == 0) *lse = lse_of(w.m, l, c);
#pragma unroll
        for (int dt = 0; dt < W::NDT; ++dt)
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4)
            store4(dst + (32 * dt + 8 * v4 + 4 * hh) * W::EB,
                   f32x4{w.oacc[dt][4 * v4], w.oacc[dt][4 * v4 + 1], w.oacc[dt][4 * v4 + 2], w.oacc[dt][4 * v4 + 3]} * inv,
                   W::EB == 2);
      } else {
        const int64_t at = ((int64_t)wg * 2 + (sh.kt == 0 ? 1 : 0)) * a.slot_rows + 32 * wave + l32;
        float* dst = a.part + at * D;
#pragma unroll
        for (int dt = 0; dt < W::NDT; ++dt)
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4)
            *reinterpret_cast<f32x4*>(dst + 32 * dt + 8 * v4 + 4 * hh) =
                f32x4{w.oacc[dt][4 * v4], w.oacc[dt][4 * v4 + 1], w.oacc[dt][4 * v4 + 2], w.oacc[dt][4 * v4 + 3]};
        if (hh == 0) {
          a.part_ml[at * 2] = w.m;
          a.part_ml[at * 2 + 1] = l;
        }
      }
    }
  });
}

// ---------------------------------------------------------------- the joining

// An item that shares w, w + 1, ... cut: its parts in the order of the keys. A
// workgroup joins eight rows, 32 lanes each: the lanes read 32 parts' maxima and
// sums at once and hand the weights round, and the parts' rows are read eight
// at a time. What bounds it is that chain of four round trips.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a, int m_rows) {
  constexpr int EB = Elem<T>::kBytes, V = D / 32;
  typedef float fV __attribute__((ext_vector_type(V)));
  const int wg = blockIdx.x;
  const int4 rec = a.info[wg];
  if (rec.x == 0) return;
  const SeqShape<6> q = shape_of<6>(a, rec.y, 0);
  const int64_t nf = (int64_t)q.n << a.gqa_shift, f0 = (int64_t)rec.w * m_rows;
  const int row = blockIdx.y * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (row >= m_rows || f0 + row >= nf) return;
  const float c = a.scale_log2;
  // part k is the share wg + k's: the first one its last item, the others their first
  auto at = [&](int k) { return ((int64_t)(wg + k) * 2 + (k == 0 ? 1 : 0)) * a.slot_rows + row; };
  float M = -__builtin_inff(), L = 0.0f;
  fV o = fV{};
  for (int k0 = 0; k0 < rec.x; k0 += 32) {
    const int n = rec.x - k0 < 32 ? rec.x - k0 : 32;
    float m = -__builtin_inff(), l = 0.0f;
    if (lane < n) {
      m = a.part_ml[at(k0 + lane) * 2];
      l = a.part_ml[at(k0 + lane) * 2 + 1];
    }
    float mx = m;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d, 32));
    if (mx > M) {
      const float f = __builtin_amdgcn_exp2f((M - mx) * c);
      L *= f;
      o *= f;
      M = mx;
    }
    const float f = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - M) * c);
    l *= f;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) l += __shfl_xor(l, d, 32);
    L += l;
    for (int k = 0; k < n; k += 8) {
      fV x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x[i] = *reinterpret_cast<const fV*>(a.part + at(k0 + (k + i < n ? k + i : n - 1)) * D + lane * V);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float w = __shfl(f, k + i < n ? k + i : 0, 32);
        if (k + i < n) o += x[i] * w;
      }
    }
  }
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
static hipError_t attend_dispatch(const PagedAttnArgs& a, bool few, hipStream_t s) {
  const int m_rows = few ? kPagedFewRows : kPagedTileRows, n_wg = paged_workgroups(few);
  if (few) hipLaunchKernelGGL((paged_few_kernel<T, D, F8>), dim3(n_wg), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_tile_kernel<T, D, F8>), dim3(n_wg), dim3(512), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int rows = a.slot_rows < m_rows ? a.slot_rows : m_rows;
  hipLaunchKernelGGL((paged_join_kernel<T, D>), dim3(n_wg, (rows + 7) / 8), dim3(256), 0, s, a, m_rows);
  return hipGetLastError();
}

hipError_t launch_attend_paged(const PagedAttnArgs& a, bool few, bool e4m3, bool bf16, int head_dim, hipStream_t s) {
  if (bf16 && head_dim == 128)
    return e4m3 ? attend_dispatch<__bf16, 128, true>(a, few, s) : attend_dispatch<__bf16, 128, false>(a, few, s);
  if (bf16)
    return e4m3 ? attend_dispatch<__bf16, 64, true>(a, few, s) : attend_dispatch<__bf16, 64, false>(a, few, s);
  return e4m3 ? attend_dispatch<float, 64, true>(a, few, s) : attend_dispatch<float, 64, false>(a, few, s);  // float32: head_dim 64
}

}  // namespace hga
