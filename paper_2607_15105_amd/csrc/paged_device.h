// Device code of the paged key/value cache: where a position's rows lie, the
// 8-bit format, and the rows of a ragged batch.
//
// A cached row (one token, one kv head, K or V) is held either in the
// configuration's element type or in 8 bits: e4m3 codes and one power-of-two
// scale, code * 2^e with e the least integer >= kMinExp under which the row's
// largest finite magnitude is at most 448 * 2^e (magnitudes over 240 * 2^120
// count as that). x * 2^-e is exact, so a code is one rounding away from its
// value, and code * 2^e has four significant bits: it is exact in bf16, and
// reading back rounds nothing. (A scale of amax / 448 would round three times for
// a gain of less than one binade of range, which a floating format does not need.)
#pragma once
#include "hga_device.h"
#include "hga_kernels.h"

namespace hga {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int kMinExp = -100;  // 2^(kMinExp - 9), a code's least step, is normal in bf16 and float32
// What finite values over it are held as, in rows of the largest exponent: with four
// significant bits they would round to 2^128, which no type that a row is read back
// in has.
constexpr float kMaxHeld = 0x1.ep127f;  // 240 * 2^120: below the largest float by less than 1/16
constexpr int kMaxExp = 120;

// Exponent of a row whose largest finite magnitude is `amax` (>= 0).
__device__ inline int row_exponent(float amax) {
  // 448 = 1.75 * 2^8: carry into the exponent field when the mantissa is over .75
  const int k = (int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 127 - 8;
  return k < kMinExp ? kMinExp : k;
}
__device__ inline float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127

// x[0..N) of a row of exponent e with its finite values within kMaxHeld. A branch for
// the rows that need it: done in every row it made 7,896 rows 12.5 -> 13.2 us.
template <int N>
__device__ inline void cap_values(float* x, int e) {
  if (!__any(e >= kMaxExp)) return;
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (fabsf(x[j]) < __builtin_inff()) x[j] = fminf(fmaxf(x[j], -kMaxHeld), kMaxHeld);
}

// Codes of x[0..3] * inv (inv = 2^-e) in one word. The conversion gives NaN for NaN and
// for what overflows, of which there are only infinities: no finite quotient passes 448.
__device__ inline uint32_t codes4(const float* x, float inv) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
  return (uint32_t)w;
}

// 16 bytes of T from the codes that hold them: eight codes for bf16, four for float.
template <typename T> struct Codes;
template <> struct Codes<__bf16> {
  static constexpr int kWords = 2;
  __device__ static inline uint4 decode(const uint32_t* w, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, true);
    return make_uint4(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                      __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d));
  }
  __device__ static inline float one(uint8_t code, float scale) {
    return (float)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, scale, false)[0];
  }
};
template <> struct Codes<float> {
  static constexpr int kWords = 1;
  __device__ static inline uint4 decode(const uint32_t* w, float scale) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], false);
    const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], true);
    return make_uint4(__float_as_uint(a[0] * scale), __float_as_uint(a[1] * scale), __float_as_uint(b[0] * scale),
                      __float_as_uint(b[1] * scale));
  }
  __device__ static inline float one(uint8_t code, float scale) {
    return __builtin_amdgcn_cvt_pk_f32_fp8(code, false)[0] * scale;
  }
};

// Positions from here on count as outside the page table, so that a position, one
// past it and the tile that holds it fit 32 bits.
constexpr int kMaxPos = 0x7fffff80;

// Page of position t (any value) of sequence s, -1 if it is absent: outside the
// table, or an entry outside [0, n_pages).
__device__ inline int page_of(const PagedArgs& a, int s, int64_t t) {
  if (t < 0 || t >= kMaxPos || (t >> a.page_shift) >= a.table_cap) return -1;
  const int p = a.table[(int64_t)s * a.table_cap + (t >> a.page_shift)];
  return (uint32_t)p < (uint32_t)a.n_pages ? p : -1;
}

// Byte offset of slot `slot` of page `page` (page and token strides below 4 GB).
__device__ inline uint64_t page_off(int page, int slot, int64_t page_b, int64_t tok_b) {
  return (uint64_t)(uint32_t)page * (uint32_t)page_b + (uint64_t)(uint32_t)slot * (uint32_t)tok_b;
}
// Index of the scale byte of (page, kv head, slot).
__device__ inline int64_t scale_off(const PagedArgs& a, int page, int h, int slot) {
  return (((int64_t)page * a.n_kv_heads + h) << a.page_shift) + slot;
}

// Rows of sequence s: [first, first + n) within the call's rows, n >= 0 whatever seq_rows holds.
__device__ inline void rows_of(const PagedArgs& a, int s, int& first, int& n) {
  const int b = a.seq_rows[s], e = a.seq_rows[s + 1], last = (int)a.n_rows;
  first = b < 0 ? 0 : (b > last ? last : b);
  n = (e > last ? last : e) - first;
  if (n < 0 || b < 0) n = 0;
}

// Sequence of the call's row r (the same in the whole wave), -1 if it is of none:
// 64 entries of seq_rows at a time, counted by ballot, so that any number of
// sequences costs independent loads and no search.
__device__ inline int seq_of_row(const PagedArgs& a, int64_t r, int lane) {
  int cnt = 0;
  for (int base = 0; base <= a.n_seqs; base += 64) {
    const int v = base + lane <= a.n_seqs ? a.seq_rows[base + lane] : 0x7fffffff;
    cnt += __popcll(__ballot((int64_t)v <= r));
  }
  return r < a.n_rows && cnt >= 1 && cnt <= a.n_seqs ? cnt - 1 : -1;
}

}  // namespace hga
