// The paged cache's own kernels: rows written into it (and quantised on the
// way), rows read back, and the routed rows of one sequence gathered from it.
#include "paged_device.h"
#include "routed_tile.h"

namespace hga {

namespace {

// Largest finite magnitude of 16 bytes of T, and their values.
template <typename T>
__device__ inline float unpack(const uint4& w, float* x) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  constexpr int N = 16 / Elem<T>::kBytes;
  float m = 0.0f;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if constexpr (Elem<T>::kBytes == 2) x[j] = __uint_as_float((j & 1) ? u[j >> 1] & 0xffff0000u : u[j >> 1] << 16);
    else x[j] = __uint_as_float(u[j]);
    const float f = fabsf(x[j]);
    m = fmaxf(m, f < __builtin_inff() ? f : 0.0f);
  }
  return m;
}

// Row r of kv head h of the call's dense K (kv = 0) or V (1).
__device__ inline char* dense_row(const DenseRows& d, int kv, int64_t r, int h) {
  return kv ? d.v + (uint64_t)(uint32_t)r * (uint32_t)d.v_tok + h * d.v_head
            : d.k + (uint64_t)(uint32_t)r * (uint32_t)d.k_tok + h * d.k_head;
}

}  // namespace

// Where row r of the call lies in the cache; page -1: nowhere, seq -1: of no sequence.
struct RowPlace {
  int seq, page, slot;
};
__device__ inline RowPlace place_of(const PagedArgs& a, int64_t r, int lane) {
  RowPlace p = {__builtin_amdgcn_readfirstlane(seq_of_row(a, r, lane)), -1, 0};
  if (p.seq >= 0) {
    const int64_t t = (int64_t)a.q_begin[p.seq] + (r - a.seq_rows[p.seq]);
    p.page = page_of(a, p.seq, t);
    p.slot = (int)(t & ((1 << a.page_shift) - 1));
  }
  return p;
}

// 16 bytes of T of a cached row: piece `c` of the row at `src`.
template <typename T, bool F8>
__device__ inline uint4 load_piece(const char* src, int c, float scale) {
  if constexpr (!F8) {
    return *reinterpret_cast<const uint4*>(src + c * 16);
  } else if constexpr (Codes<T>::kWords == 2) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(src + c * 8);
    const uint32_t x[2] = {w[0], w[1]};
    return Codes<T>::decode(x, scale);
  } else {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(src + c * 4);
    return Codes<T>::decode(&w, scale);
  }
}

constexpr int kPasses = 2;  // head groups of a row whose pieces are under way at once

// Rows into the cache, one per wave. A row of a kv head is held by LPR
// consecutive lanes, 16 bytes each, so its largest magnitude is a reduction over
// LPR lanes. A call of few rows is bound by a chain of four round trips (the
// sequence, its position, the page, the store), one of many by the memory: 64
// rows of 8 heads, d = 128, bf16 to 8 bits take 4.8 us and 7,896 rows 11.7 (10.7 and
// 16.1 with four rows to a wave, one after the other). A wave for a row whatever its
// width: where Hkv * d * eb is below 1 KiB lanes are idle, and 32,768 rows of one
// head, d = 64, bf16 to 8 bits take 14.8 us where their bytes take 2.6.
template <typename T, int D, bool F8>
__global__ __launch_bounds__(256) void cache_write_kernel(PagedArgs a, DenseRows d, int64_t first) {
  constexpr int EB = Elem<T>::kBytes, LPR = D * EB / 16, HP = 64 / LPR, N = 16 / EB;
  const int lane = threadIdx.x & 63, c = lane % LPR;
  const int64_t r = first + (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (r >= a.n_rows) return;
  const RowPlace at = place_of(a, r, lane);
  if (at.page < 0) return;
  char* const kd = a.k + page_off(at.page, at.slot, a.k_page, a.k_tok);
  char* const vd = a.v + page_off(at.page, at.slot, a.v_page, a.v_tok);
  for (int h0 = 0; h0 < a.n_kv_heads; h0 += HP * kPasses) {
    uint4 w[kPasses][2];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int h = h0 + p * HP + lane / LPR;
      if (h < a.n_kv_heads) {
        w[p][0] = *reinterpret_cast<const uint4*>(dense_row(d, 0, r, h) + c * 16);
        w[p][1] = *reinterpret_cast<const uint4*>(dense_row(d, 1, r, h) + c * 16);
      }
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int h = h0 + p * HP + lane / LPR;
      if (h >= a.n_kv_heads) continue;  // whole groups of LPR lanes
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        char* dst = kv ? vd + h * a.v_head : kd + h * a.k_head;
        if constexpr (!F8) {
          *reinterpret_cast<uint4*>(dst + c * 16) = w[p][kv];
        } else {
          float x[N];
          float m = unpack<T>(w[p][kv], x);
#pragma unroll
          for (int o = LPR / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
          const int e = row_exponent(m);
          cap_values<N>(x, e);
          const float inv = exp2i(-e);
          if constexpr (N == 8) {
            const u32x2 y = {codes4(x, inv), codes4(x + 4, inv)};
            *reinterpret_cast<u32x2*>(dst + c * 8) = y;
          } else {
            *reinterpret_cast<uint32_t*>(dst + c * 4) = codes4(x, inv);
          }
          if (c == 0) (kv ? a.v_scale : a.k_scale)[scale_off(a, at.page, h, at.slot)] = (uint8_t)(e + 127);
        }
      }
    }
  }
}

// Rows out of the cache, one per wave; an absent page's rows are zeros.
template <typename T, int D, bool F8>
__global__ __launch_bounds__(256) void cache_read_kernel(PagedArgs a, DenseRows d, int64_t first) {
  constexpr int EB = Elem<T>::kBytes, LPR = D * EB / 16, HP = 64 / LPR;
  const int lane = threadIdx.x & 63, c = lane % LPR;
  const int64_t r = first + (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (r >= a.n_rows) return;
  const RowPlace at = place_of(a, r, lane);
  if (at.seq < 0) return;
  const bool there = at.page >= 0;
  const char* const ks = a.k + page_off(there ? at.page : 0, at.slot, a.k_page, a.k_tok);
  const char* const vs = a.v + page_off(there ? at.page : 0, at.slot, a.v_page, a.v_tok);
  for (int h0 = 0; h0 < a.n_kv_heads; h0 += HP * kPasses) {
    uint4 w[kPasses][2];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int h = h0 + p * HP + lane / LPR;
      w[p][0] = w[p][1] = make_uint4(0u, 0u, 0u, 0u);
      if (there && h < a.n_kv_heads) {
        float s[2] = {1.0f, 1.0f};
        if constexpr (F8) {
          const int64_t so = scale_off(a, at.page, h, at.slot);
          s[0] = __uint_as_float((uint32_t)a.k_scale[so] << 23);
          s[1] = __uint_as_float((uint32_t)a.v_scale[so] << 23);
        }
        w[p][0] = load_piece<T, F8>(ks + h * a.k_head, c, s[0]);
        w[p][1] = load_piece<T, F8>(vs + h * a.v_head, c, s[1]);
      }
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int h = h0 + p * HP + lane / LPR;
      if (h < a.n_kv_heads) {
        *reinterpret_cast<uint4*>(dense_row(d, 0, r, h) + c * 16) = w[p][0];
        *reinterpret_cast<uint4*>(dense_row(d, 1, r, h) + c * 16) = w[p][1];
      }
    }
  }
}

// hga_gather_routed over a cached sequence: one workgroup per (tile of 64
// positions, block, kv head).
template <typename T, int D, bool F8>
__global__ __launch_bounds__(256) void gather_paged_kernel(AttnArgs a, PagedArgs p, int seq, char* kc, char* vc) {
  constexpr int EB = Elem<T>::kBytes, CPR = D * EB / 16;
  __shared__ int s_sel[64];
  const int tid = threadIdx.x;
  const int h = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads;
  const RouteRow rrow = load_route_row(a, b, h, tid);
  const RoutedSet rs = make_routed_set(a, b, rrow, s_sel, tid);
  __syncthreads();  // s_sel
  const int tile = blockIdx.y;
  if (tile * 64 >= rs.R) return;
  const int64_t slot0 = (((int64_t)b * a.n_kv_heads + h) * a.r_cap + tile * 64) * D * EB;
  for (int item = tid; item < 64 * CPR; item += 256) {
    const int r = item / CPR, c = item % CPR;
    bool ok;
    const int64_t t = rs.token(tile * 64 + r, ok);
    const int page = ok ? page_of(p, seq, t) : -1;
    const int slot = (int)(t & ((1 << p.page_shift) - 1));
    uint4 wk = make_uint4(0u, 0u, 0u, 0u), wv = wk;
    if (page >= 0) {
      float sk = 1.0f, sv = 1.0f;
      if constexpr (F8) {
        const int64_t so = scale_off(p, page, h, slot);
        sk = __uint_as_float((uint32_t)p.k_scale[so] << 23);
        sv = __uint_as_float((uint32_t)p.v_scale[so] << 23);
      }
      wk = load_piece<T, F8>(p.k + page_off(page, slot, p.k_page, p.k_tok) + h * p.k_head, c, sk);
      wv = load_piece<T, F8>(p.v + page_off(page, slot, p.v_page, p.v_tok) + h * p.v_head, c, sv);
    }
    *reinterpret_cast<uint4*>(kc + slot0 + (int64_t)item * 16) = wk;
    *reinterpret_cast<uint4*>(vc + slot0 + (int64_t)item * 16) = wv;
  }
}

#define HGA_PAGED_DISPATCH(CALL)                     \
  do {                                               \
    if (bf16 && head_dim == 128) {                   \
      if (e4m3) CALL(__bf16, 128, true);             \
      else CALL(__bf16, 128, false);                 \
    } else if (bf16) {                               \
      if (e4m3) CALL(__bf16, 64, true);              \
      else CALL(__bf16, 64, false);                  \
    } else { /* float32: head_dim 64 */              \
      if (e4m3) CALL(float, 64, true);               \
      else CALL(float, 64, false);                   \
    }                                                \
  } while (0)

// Rows of a launch: a grid holds fewer than 2^32 threads, 64 to a row.
constexpr int64_t kLaunchRows = 1 << 25;
static unsigned row_workgroups(int64_t rows) { return (unsigned)(((rows < kLaunchRows ? rows : kLaunchRows) + 3) / 4); }

hipError_t launch_cache_write(const PagedArgs& a, const DenseRows& d, bool e4m3, bool bf16, int head_dim, hipStream_t s) {
#define HGA_CALL(T, D, F) hipLaunchKernelGGL((cache_write_kernel<T, D, F>), grid, dim3(256), 0, s, a, d, first)
  for (int64_t first = 0; first < a.n_rows; first += kLaunchRows) {
    const dim3 grid(row_workgroups(a.n_rows - first));
    HGA_PAGED_DISPATCH(HGA_CALL);
  }
#undef HGA_CALL
  return hipGetLastError();
}

hipError_t launch_cache_read(const PagedArgs& a, const DenseRows& d, bool e4m3, bool bf16, int head_dim, hipStream_t s) {
#define HGA_CALL(T, D, F) hipLaunchKernelGGL((cache_read_kernel<T, D, F>), grid, dim3(256), 0, s, a, d, first)
  for (int64_t first = 0; first < a.n_rows; first += kLaunchRows) {
    const dim3 grid(row_workgroups(a.n_rows - first));
    HGA_PAGED_DISPATCH(HGA_CALL);
  }
#undef HGA_CALL
  return hipGetLastError();
}

hipError_t launch_gather_paged(const AttnArgs& a, const PagedArgs& p, int seq, void* kc, void* vc, bool e4m3, bool bf16,
                               int head_dim, hipStream_t s) {
  // as many tiles as the longest set of the call has
  const int64_t end = a.q_begin + (int64_t)a.n_qb * 64;
  const int64_t sink = a.sink_tokens < end ? a.sink_tokens : end, local = a.local_tokens < end ? a.local_tokens : end;
  const int64_t rows = sink + local + ((int64_t)a.top_groups << a.group_shift);
  const dim3 grid(a.n_qb * a.n_kv_heads, (unsigned)((rows + 63) / 64));
#define HGA_CALL(T, D, F) \
  hipLaunchKernelGGL((gather_paged_kernel<T, D, F>), grid, dim3(256), 0, s, a, p, seq, (char*)kc, (char*)vc)
  HGA_PAGED_DISPATCH(HGA_CALL);
#undef HGA_CALL
  return hipGetLastError();
}

}  // namespace hga
