// Internal declarations of the paged key-value cache's operators: what their
// kernels take, their launchers, and the device code that they share.
#pragma once
#include "gvc.h"
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gvc {

// Sets gvc_last_error and returns code (defined beside the error text).
int32_t set_error(int32_t code, const char* msg) noexcept;

// The pool as the kernels see it.  Offsets inside one page fit 32 bits (at
// most 1024 heads x 128 slots x 128 dimensions); a page's own offset may not.
struct PagedPool {
  uint16_t* k;         // [n_pages][Hk][page][dh]
  uint16_t* v;         // [n_pages][Hk][dh][page]
  const int* table;    // [n_seqs][max_pages]
  int n_seqs, max_pages, n_pages, page_shift;   // page = 1 << page_shift slots
  int H, Hk, dh;
};

constexpr int kPagedMaxPairs = 64;   // head_dim / 2
constexpr int kPagedMaxSeqs = 4096;  // every wave goes through their rows to find its work

struct PagedAppendArgs {
  PagedPool pool;
  const uint16_t *q, *kin, *vin, *q_norm, *k_norm;
  uint16_t* q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  const int *row_seq, *row_slot, *positions;   // positions: nullptr = the row's slot on every axis
  int64_t position_stride;
  int n_rows, n_pairs, end0, end1;             // pairs [0, end0) use axis 0, [end0, end1) axis 1, the others axis 2
  float eps;
  double turns[kPagedMaxPairs];                // pair i turns by position * turns[i] full turns
};

struct PagedAttnArgs {
  PagedPool pool;
  const uint16_t* q;
  uint16_t* out;
  int64_t q_stride, out_stride;
  const int* row_last;    // last slot of each row; decode: the sequences' lengths
  const int* row_begin;   // rows of each sequence, or nullptr: row s is sequence s, and row_last holds lengths
  int n_rows, window, n_sinks;
  float scale_log2e;      // scores in powers of two
  uint64_t tag;           // of the call (paged_tag)
};

// A number, not zero, that no other call of the process has, and that memory
// which no call has written holds with a probability of 2^-64.
uint64_t paged_tag() noexcept;

// How a call is cut into units of work, and the workspace of their partial results.
struct PagedSplit {
  bool split;       // a row's slots may be split over units
  int least;        // decode: the least tiles of a unit
  bool fused;       // decode: the units join their results themselves (else a second launch does)
  int64_t units;    // an upper bound: the grid
  int64_t tiles;    // prefill: row tiles, at most, and the parts that each one's slots are cut into
  int parts;
  size_t bytes;
};
// rows: lists of rows, else one row per sequence.
PagedSplit paged_decode_split(const PagedPool& p, int n_rows, bool rows, int window, int n_sinks);
PagedSplit paged_prefill_split(const PagedPool& p, int n_rows);
// Whether a call with lists of rows goes to the decode kernel.
bool paged_few_rows(const PagedPool& p, int n_rows, int window, int n_sinks);

hipError_t launch_paged_decode(const PagedAttnArgs& a, const PagedSplit& sp, int dtype, void* workspace, hipStream_t s);
hipError_t launch_paged_prefill(const PagedAttnArgs& a, const PagedSplit& sp, int dtype, void* workspace, hipStream_t s);
hipError_t launch_paged_append(const PagedAppendArgs& a, int dtype, hipStream_t s);

#ifdef __HIPCC__
// ------------------------------------------------------------------ device
typedef __bf16 pbf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 pf16x8 __attribute__((ext_vector_type(8)));
typedef float pf32x4 __attribute__((ext_vector_type(4)));
typedef float pf32x16 __attribute__((ext_vector_type(16)));
typedef float pf32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t pu32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t pu32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t pu16x4 __attribute__((ext_vector_type(4)));

// The running maximum may lag behind the true one by 2^kPagedLazy before output
// and sum are rescaled: a probability is at most 2^kPagedLazy.
constexpr float kPagedLazy = 8.f;

// Outputs are summed before they are divided by the sum of the probabilities, so in
// bf16, whose values reach 2^128, a sum may overflow where the output is finite.  A
// wave whose sums reach kPagedLarge, or are not finite, does them again relative to
// 2^spare_bits above its maximum: the probabilities of its slots then add up to at
// most 2^-13.  Either way a wave's sums are below 2^115, and the 4 x 1026 of them that
// are joined at most below 2^128.  (In such a wave products of a probability and a
// value under 2^-126 + spare_bits are lost.)
constexpr float kPagedLarge = 0x1p115f;

// The two 16-bit types.  Conversions to 16 bits round to nearest even.  What is
// rounded to them, once each: a rotated query or key (the pages hold 16 bits), a
// probability before the second product (whose operands are of one type: the matrix
// cores would need two products for more bits.  Half a step, at most 2^-8 of it in bf16
// and 2^-11 in fp16, averages out over the slots; the sum takes it unrounded) and an
// output.  (Relative difference of bf16 outputs from 64 bits: 0.0018 to 0.0023; with
// unrounded probabilities 0.0016 to 0.0017, the output's own rounding.)
struct Bf16 {
  typedef pbf16x8 x8;
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ float up(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }
  static __device__ __forceinline__ pf32x4 mfma16(pu32x4 a, pu32x4 b, pf32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ pf32x16 mfma32(pu32x4 a, pu32x4 b, pf32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static constexpr float kShift = 0.f;   // see Fp16
  static constexpr bool kOverflows = true;
  static constexpr float kMax = 0x1.fep127f;   // the largest value
};
struct Fp16 {
  typedef pf16x8 x8;
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ float up(uint16_t h) { return (float)__builtin_bit_cast(_Float16, h); }
  static __device__ __forceinline__ pf32x4 mfma16(pu32x4 a, pu32x4 b, pf32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ pf32x16 mfma32(pu32x4 a, pu32x4 b, pf32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  // Probabilities enter the product with V in 16 bits.  fp16 has few exponents
  // below 1: a long tail of probabilities under 2^-25 would vanish.  They are
  // scaled by 2^kShift, sum and output alike, and still fit: a probability is
  // at most 2^kPagedLazy before scaling.
  static constexpr float kShift = 6.f;
  // 2^30 slots at most, probabilities of 2^14, values of 2^16: sums are below 2^60.
  static constexpr bool kOverflows = false;
  static constexpr float kMax = 65504.f;
};

template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const pf32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, typename T::x2));
}

// Four outputs.  An average of values is not larger than the largest of them, but the
// rounded probabilities can carry it there: a finite one stays within the type.
template <class T>
__device__ __forceinline__ pu32x2 pack_out(pf32x4 o) {
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = fabsf(o[i]) < INFINITY ? fminf(fmaxf(o[i], -T::kMax), T::kMax) : o[i];
  return {pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
}

// For n tiles of 2^tile_log slots.
__device__ __forceinline__ int spare_bits(int n, int tile_log) { return 13 + tile_log + 32 - __builtin_clz(max(n, 1)); }

// The largest over the four 16-lane rows of a wave, lane by lane.
__device__ __forceinline__ float rows_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float rows_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
#endif

}  // namespace gvc
