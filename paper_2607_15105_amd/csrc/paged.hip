// The paged cache's own kernels: rows written into it (and quantised on the
// way), rows read back, and the routed rows of one sequence gathered from it.
#include "paged_device.h"
#include "routed_tile.h"

namespace hga {

namespace {

constexpr int kRowsPerWave = 4;

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

// Rows into the cache. A row of a kv head is held by LPR consecutive lanes, 16
// bytes each, so its largest magnitude is a reduction over LPR lanes.
template <typename T, int D, bool F8>
__global__ __launch_bounds__(256) void cache_write_kernel(PagedArgs a, DenseRows d) {
  constexpr int EB = Elem<T>::kBytes, LPR = D * EB / 16, N = 16 / EB;
  const int lane = threadIdx.x & 63;
  const int64_t r0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * kRowsPerWave;
  if (r0 >= a.n_rows) return;
  int seq[kRowsPerWave];
  find_rows<kRowsPerWave>(a, r0, lane, seq);
  for (int i = 0; i < kRowsPerWave; ++i) {
    if (seq[i] < 0) continue;
    const int64_t t = (int64_t)a.q_begin[seq[i]] + (r0 + i - a.seq_rows[seq[i]]);
    const int page = page_of(a, seq[i], t);
    if (page < 0) continue;
    const int slot = (int)(t & ((1 << a.page_shift) - 1));
    for (int h = lane / LPR; h < a.n_kv_heads; h += 64 / LPR) {
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const char* src = dense_row(d, kv, r0 + i, h);
        char* dst = kv ? a.v + page_off(page, slot, a.v_page, a.v_tok) + h * a.v_head
                       : a.k + page_off(page, slot, a.k_page, a.k_tok) + h * a.k_head;
        const uint4 w = *reinterpret_cast<const uint4*>(src + (lane % LPR) * 16);
        if constexpr (!F8) {
          *reinterpret_cast<uint4*>(dst + (lane % LPR) * 16) = w;
        } else {
          float x[N];
          float m = unpack<T>(w, x);
#pragma unroll
          for (int o = LPR / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
          const int e = row_exponent(m);
          const float inv = exp2i(-e);
          if constexpr (N == 8) {
            const u32x2 c = {codes4(x, inv), codes4(x + 4, inv)};
            *reinterpret_cast<u32x2*>(dst + (lane % LPR) * 8) = c;
          } else {
            *reinterpret_cast<uint32_t*>(dst + (lane % LPR) * 4) = codes4(x, inv);
          }
          if (lane % LPR == 0) (kv ? a.v_scale : a.k_scale)[scale_off(a, page, h, slot)] = (uint8_t)(e + 127);
        }
      }
    }
  }
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

// Rows out of the cache; an absent page's rows are zeros.
template <typename T, int D, bool F8>
__global__ __launch_bounds__(256) void cache_read_kernel(PagedArgs a, DenseRows d) {
  constexpr int EB = Elem<T>::kBytes, LPR = D * EB / 16;
  const int lane = threadIdx.x & 63;
  const int64_t r0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * kRowsPerWave;
  if (r0 >= a.n_rows) return;
  int seq[kRowsPerWave];
  find_rows<kRowsPerWave>(a, r0, lane, seq);
  for (int i = 0; i < kRowsPerWave; ++i) {
    if (seq[i] < 0) continue;
    const int64_t t = (int64_t)a.q_begin[seq[i]] + (r0 + i - a.seq_rows[seq[i]]);
    const int page = page_of(a, seq[i], t);
    const int slot = (int)(t & ((1 << a.page_shift) - 1));
    for (int h = lane / LPR; h < a.n_kv_heads; h += 64 / LPR) {
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        char* dst = dense_row(d, kv, r0 + i, h);
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        if (page >= 0) {
          const char* src = kv ? a.v + page_off(page, slot, a.v_page, a.v_tok) + h * a.v_head
                               : a.k + page_off(page, slot, a.k_page, a.k_tok) + h * a.k_head;
          float scale = 1.0f;
          if constexpr (F8) scale = __uint_as_float((uint32_t)(kv ? a.v_scale : a.k_scale)[scale_off(a, page, h, slot)] << 23);
          w = load_piece<T, F8>(src, lane % LPR, scale);
        }
        *reinterpret_cast<uint4*>(dst + (lane % LPR) * 16) = w;
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

hipError_t launch_cache_write(const PagedArgs& a, const DenseRows& d, bool e4m3, bool bf16, int head_dim, hipStream_t s) {
  const dim3 grid((unsigned)((a.n_rows + 4 * kRowsPerWave - 1) / (4 * kRowsPerWave)));
#define HGA_CALL(T, D, F) hipLaunchKernelGGL((cache_write_kernel<T, D, F>), grid, dim3(256), 0, s, a, d)
  HGA_PAGED_DISPATCH(HGA_CALL);
#undef HGA_CALL
  return hipGetLastError();
}

hipError_t launch_cache_read(const PagedArgs& a, const DenseRows& d, bool e4m3, bool bf16, int head_dim, hipStream_t s) {
  const dim3 grid((unsigned)((a.n_rows + 4 * kRowsPerWave - 1) / (4 * kRowsPerWave)));
#define HGA_CALL(T, D, F) hipLaunchKernelGGL((cache_read_kernel<T, D, F>), grid, dim3(256), 0, s, a, d)
  HGA_PAGED_DISPATCH(HGA_CALL);
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
