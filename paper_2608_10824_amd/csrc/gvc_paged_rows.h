// Device code that the attention kernels of the paged cache share: a
// sequence's rows, and the join of partial results.
#pragma once
#include "gvc_kernels.h"
#include "gvc_paged.h"

namespace gvc {

// v, which is the same in every lane, as a scalar: loops and branches on it stay scalar.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// The lowest n of eight bits, for any n.
__device__ __forceinline__ uint32_t first8(int n) { return (1u << min(max(n, 0), 8)) - 1; }
// x if bit i is set, else -infinity: two instructions and no condition register.
__device__ __forceinline__ float seen_score(uint32_t bits, int i, float x) {
  const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)bits, i, 1);
  return __uint_as_float((__float_as_uint(x) & keep) | (0xff800000u & ~keep));
}

// A sequence's first row and number of virtual rows, and the last slot that its
// last row sees.
struct SeqRows {
  int begin, rows, last;
};

// ROWS: the call gives lists of rows (gvc_paged_prefill), else one row per sequence and lengths.
template <bool ROWS>
__device__ __forceinline__ SeqRows seq_rows(const PagedAttnArgs& a, int s, int G) {
  const int slots = a.pool.max_pages << a.pool.page_shift;
  if (!ROWS) return {s, G, min(max(a.row_last[s], 0), slots) - 1};
  const int begin = min(max(a.row_begin[s], 0), a.n_rows), n = max(min(a.row_begin[s + 1], a.n_rows) - begin, 0);
  return {begin, n * G, n ? min(max(a.row_last[begin + n - 1], -1), slots - 1) : -1};
}

// The sequence that a listed row belongs to (seq -1: none).
__device__ __forceinline__ SeqRows seq_of_row(const PagedAttnArgs& a, int row, int G, int lane, int& seq) {
  const int S = a.pool.n_seqs;
  seq = -1;
  for (int s0 = 0; s0 < S; s0 += 64) {
    const SeqRows r = seq_rows<true>(a, min(s0 + lane, S - 1), G);
    const uint64_t here = __ballot(r.begin <= row && row < r.begin + r.rows / G);
    if (!here) continue;
    const int l = __builtin_ctzll(here);
    seq = uniform(s0 + l);
    return {__builtin_amdgcn_readlane(r.begin, l), __builtin_amdgcn_readlane(r.rows, l),
            __builtin_amdgcn_readlane(r.last, l)};
  }
  return {0, 0, -1};
}

// Inclusive sum over the lanes of a wave, on DPP row shifts and broadcasts.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);   // within rows of 16: 1, 2, 4, 8 lanes down
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // the last lane of rows 0 and 2 to rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // the last lane of row 1 to rows 2 and 3
  return v;
}

// Joins n partial results of one row and head, `step` floats apart: maximum,
// sum, whether a slot was seen, nothing, DH outputs.  Weights of the parts from
// their maxima, then groups of DH / 4 threads add up the weighted outputs of every
// n-th part, and the groups' sums are added in LDS.
template <int DH, int NT, int MOST>
struct JoinLds {
  float weight[MOST], sums[3][NT / 64];
  pf32x4 part[NT / (DH / 4)][DH / 4];
};

template <class T, int DH, int NT, int MOST>
__device__ __forceinline__ void join_row(const float* from, int64_t step, int n, JoinLds<DH, NT, MOST>& lds, uint16_t* out) {
  constexpr int GT = DH / 4, NG = NT / GT;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  float m = -INFINITY;
  for (int c = tid; c < n; c += NT) {
    lds.weight[c] = from[c * step];
    m = fmaxf(m, lds.weight[c]);
  }
  m = wave_max(m);
  if (lane == 0) lds.sums[0][wv] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) m = fmaxf(m, lds.sums[0][w]);
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f, saw = 0.f;
  for (int c = tid; c < n; c += NT) {
    const float f = __builtin_amdgcn_exp2f(lds.weight[c] - ref);
    lds.weight[c] = f;
    l += from[c * step + 1] * f;
    saw += from[c * step + 2];
  }
  l = wave_sum(l);
  saw = wave_sum(saw);
  if (lane == 0) lds.sums[1][wv] = l, lds.sums[2][wv] = saw;
  __syncthreads();
  const int gr = tid / GT, d = tid % GT;
  pf32x4 o = {0, 0, 0, 0};
#pragma unroll 4
  for (int c = gr; c < n; c += NG) o += *(const pf32x4*)(from + c * step + 4 + 4 * d) * lds.weight[c];
  lds.part[gr][d] = o;
  __syncthreads();
  if (tid >= GT) return;
  o = lds.part[0][d];
#pragma unroll
  for (int k = 1; k < NG; ++k) o += lds.part[k][d];
  l = saw = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) l += lds.sums[1][w], saw += lds.sums[2][w];
  const float inv = 1.f / l;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = saw > 0.f ? o[k] * inv : 0.f;
  *(pu32x2*)(out + 4 * d) = pack_out<T>(o);
}

}  // namespace gvc
