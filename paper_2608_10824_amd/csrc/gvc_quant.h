// Internal declarations of the quantised paged cache's operators: a paged
// cache (gvc_paged.h) whose keys and values are e4m3 codes, with one power of
// two to each head of a slot.
#pragma once
#include "gvc_paged.h"

namespace gvc {

// The pages; PagedPool::k and v are not used.  Offsets inside one page fit 32
// bits, a page's own may not.
struct QuantPages {
  uint8_t *k, *v;               // [n_pages][Hk][page][dh], [n_pages][Hk][dh][page] e4m3
  uint8_t *k_scale, *v_scale;   // [n_pages][Hk][page] e8m0
};

struct QuantReadArgs {
  PagedPool pool;
  QuantPages pages;
  const int *row_seq, *row_slot;
  uint16_t *k_out, *v_out;      // nullptr: not wanted
  int64_t k_stride, v_stride;
  int n_rows;
};

hipError_t launch_quant_append(const PagedAppendArgs& a, const QuantPages& to, int dtype, hipStream_t s);
hipError_t launch_quant_read(const QuantReadArgs& a, int dtype, hipStream_t s);
PagedSplit quant_decode_split(const PagedPool& p, int n_rows, bool rows, int window, int n_sinks);
hipError_t launch_quant_decode(const PagedAttnArgs& a, const QuantPages& from, const PagedSplit& sp, int dtype,
                               void* workspace, hipStream_t s);
hipError_t launch_quant_prefill(const PagedAttnArgs& a, const QuantPages& from, const PagedSplit& sp, int dtype,
                                void* workspace, hipStream_t s);

#ifdef __HIPCC__
// ------------------------------------------------------------------ device
// A scale code as a factor: 2^(code - 127).  The conversions below take a
// float's exponent bits as such a code: 0 is 2^-127 and 255 NaN to them.
__device__ __forceinline__ float scale_of(uint32_t code) { return __uint_as_float(code << 23); }

// Codes 2 HI and 2 HI + 1 of w, times a scale, as a pair of the 16-bit type (rounded to nearest even once).
template <class T, bool HI>
__device__ __forceinline__ uint32_t decoded(uint32_t w, float scale);
template <>
__device__ __forceinline__ uint32_t decoded<Bf16, false>(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
}
template <>
__device__ __forceinline__ uint32_t decoded<Bf16, true>(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
}
template <>
__device__ __forceinline__ uint32_t decoded<Fp16, false>(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false));
}
template <>
__device__ __forceinline__ uint32_t decoded<Fp16, true>(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true));
}

// The largest value of a code that the 16-bit type holds (240 times a power of two: the next one, 256 times it, is past the type).
template <class T>
struct QuantMost;
template <>
struct QuantMost<Bf16> {
  static constexpr float value = 0x1.ep127f;
};
template <>
struct QuantMost<Fp16> {
  static constexpr float value = 61440.f;
};

// A value as it is quantised, and what it counts for the scale.
template <class T>
__device__ __forceinline__ float bounded(float x) {
  return fabsf(x) < INFINITY ? fminf(fmaxf(x, -QuantMost<T>::value), QuantMost<T>::value) : x;
}
__device__ __forceinline__ float counted(float bounded_x) { return fabsf(bounded_x) < INFINITY ? fabsf(bounded_x) : 0.f; }

// The scale code of a head whose largest magnitude is `most`: the least e >=
// -126 with most <= 448 * 2^e = 1.75 * 2^(e + 8), from the bits of most.
__device__ __forceinline__ int scale_code(float most) {
  const uint32_t bits = __float_as_uint(most);
  return max((int)(bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0), 1);
}
// 2^-e of a scale code from 1 to 253.
__device__ __forceinline__ float inverse_scale(int code) { return __uint_as_float((uint32_t)(254 - code) << 23); }

// Where a row goes: its page (-1: nowhere) and the slot in it.
struct QuantPlace {
  int page, off;
};
__device__ __forceinline__ QuantPlace quant_place(const PagedPool& p, int seq, int slot) {
  int page = -1;
  if ((unsigned)seq < (unsigned)p.n_seqs && slot >= 0 && (slot >> p.page_shift) < p.max_pages)
    page = p.table[(int64_t)seq * p.max_pages + (slot >> p.page_shift)];
  return {(unsigned)page < (unsigned)p.n_pages ? page : -1, slot & ((1 << p.page_shift) - 1)};
}
#endif

}  // namespace gvc
