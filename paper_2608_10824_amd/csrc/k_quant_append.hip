// Rows into the quantised paged cache, with the norm and rotation of queries
// and keys, and rows read back.
//
// The scale of a head is 2^e with the least e for which its largest magnitude is
// at most 448 * 2^e (from the bits of that magnitude), its codes are the values divided by it,
// which is exact, rounded once.  A key's norm and rotation are computed in double (rms_eps is its 32 bits) and
// not rounded before (high_word), so its codes are those of the exact key unless that is nearer to half way between two
// codes than the computation's error: 2^-44 of the pair that turns, and 2^-46 of it times the angle, from the turns' 64
// roundings (with bases of 10^4 and more less than 2^-51 times the position).  32 bits would take the other code in one value of
// two million.  (Double takes 1% of a long call of few key-value heads, 9% where every head has one.)  Queries are
// computed in 32 bits.  Angles are taken in full turns, in double, and reduced to [-1/2, 1/2].
//
// Everything is read and written once, so HBM bounds long calls and launch and
// load latency short ones.  One launch of append has two kinds of workgroups, as k_paged_append.hip:
//  * Queries and keys: a wave takes one row and every slices-th group of heads
//    of it, DH / 8 lanes to a head; a lane holds two chunks of four dimensions
//    that turn together, or past the rotated dimensions two neighbouring chunks.
//  * Values: a workgroup takes one head of 32 rows.  DH / 8 threads quantise a row and put its
//    codes into LDS; where eight rows fill eight slots in a row, a lane writes 8 bytes of one
//    dimension, rows that stand alone are written byte by byte, neighbouring lanes
//    taking neighbouring rows.
//
// Measured (bf16, 128 to a head): append of 21 627 rows of whole prompts, 32 heads on 8, norm and three axes 99 us,
// 488 MB at 4.9 TB/s, a copy's rate; of 2368 rows of 16 sequences, about every second slot, 32 heads 31 us, 3.1 TB/s
// (10 us of it bytes of V that stand alone); one row 4.0 us, 6.1 to 6.4 between two calls of a graph.  Two or four heads of values to a workgroup, kinds of
// workgroups in turns: 5 to 10% slower.  Read of 41 000 rows of 8 heads, fp16, 64 us, 303 MB at 4.8 TB/s, of every second
// slot 34 us (stores that stay in the caches 47); of 282 rows of 32 heads 5.1 us.
#include "gvc_kernels.h"
#include "gvc_quant.h"

#include <type_traits>

namespace gvc {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kRows = 32;      // rows of a workgroup of values, and 7 on both sides that its runs of eight may reach
constexpr int kReadThreads = 512, kReadRows = 64;   // (32 rows to 256 threads: 6% slower, 41 000 rows)
constexpr int kFill = 4096;    // waves of queries and keys that a call's rows are cut into, at least

// What a call reads and writes once: past the caches' least recent lines where the call is larger than
// the last of them (21 627 rows, 488 MB, one call after another 103 us for 111; where 97 MB stay in the cache 32.2 for 31.5).
constexpr int64_t kLastCache = 256 << 20;
template <bool STREAM, class V>
__device__ __forceinline__ V once(const V* from) {
  return STREAM ? __builtin_nontemporal_load(from) : *from;
}
template <bool STREAM, class V>
__device__ __forceinline__ void once(V* to, V v) {
  if (STREAM) __builtin_nontemporal_store(v, to);
  else *to = v;
}

constexpr float kMostCode = 240.f;   // QuantMost is this times a power of two

// Four values times a power of two, as codes.
__device__ __forceinline__ uint32_t encoded4(const float* x, float f) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, lo, true);
}

// Sine and cosine of t full turns, |t| <= 1/2: a quarter turn at most from a multiple of one, by Taylor's
// series to x^13 and x^14 (off by at most 2^-45).
__device__ __forceinline__ void sine_cosine(double t, double& sine, double& cosine) {
  const double q = rint(4 * t), x = (t - 0.25 * q) * 6.283185307179586477, y = x * x;
  double s = fma(y, 1. / 6227020800, -1. / 39916800), c = fma(y, -1. / 87178291200, 1. / 479001600);
  s = fma(y, s, 1. / 362880), c = fma(y, c, -1. / 3628800);
  s = fma(y, s, -1. / 5040), c = fma(y, c, 1. / 40320);
  s = fma(y, s, 1. / 120), c = fma(y, c, -1. / 720);
  s = fma(y, s, -1. / 6), c = fma(y, c, 1. / 24);
  s = fma(x * y, s, x), c = fma(y, fma(y, c, -0.5), 1.);
  const int i = (int)q;
  sine = i & 1 ? c : s;
  cosine = i & 1 ? s : c;
  if (i & 2) sine = -sine;             // q of 2, -2 and -1
  if ((i + 1) & 2) cosine = -cosine;   // q of 1, 2 and -2
}

// The sum over aligned groups of N lanes.
template <int CTRL>
__device__ __forceinline__ double other_lane(double v) {
  const uint64_t x = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, 0xF, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, 0xF, 0xF, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int N>
__device__ __forceinline__ double sum_of_group(double v) {
  v += other_lane<kDppXor1>(v);
  v += other_lane<kDppXor2>(v);
  v += other_lane<kDppHalfMirror>(v);
  if constexpr (N == 16) v += other_lane<kDppMirror>(v);
  return v;
}
template <int N>
__device__ __forceinline__ float sum_of_group(float v) {
  return group_sum<N>(v);
}

// 1 / sqrt(x).  In double one Newton step from the instruction's estimate (2^-24 at most): off by 2^-46.
__device__ __forceinline__ float inverse_root(float x) { return 1.f / sqrtf(x); }
__device__ __forceinline__ double inverse_root(double x) {
  const double r = __builtin_amdgcn_rsq(x);
  return x > 0 && x < INFINITY ? r * fma(-0.5 * x * r, r, 1.5) : r;
}

// Keys are quantised from doubles: a gain or a rotation can carry 16-bit values past the ends of a float's range, where it
// would be infinite or lose bits.  They are scaled in double too, and only then become floats.

// The high word of a double, its last bit set where the low one is not zero: rounding that to a few bits, or
// comparing it with a number of a few bits, is as exact as with the double.
__device__ __forceinline__ uint32_t high_word(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return (uint32_t)(b >> 32) | min((uint32_t)b, 1u);
}
// The size of a word's double where that is finite, else 0.
__device__ __forceinline__ uint32_t counted_word(uint32_t w) {
  const uint32_t size = w & 0x7fffffff;
  return size < 0x7ff00000 ? size : 0;
}
// As scale_code(), of the word of a head's largest magnitude.
__device__ __forceinline__ int scale_code_of_word(uint32_t most) {
  return max((int)(most >> 20) - 1023 + 127 - 8 + ((most & 0xfffff) > 0xc0000 ? 1 : 0), 1);
}
// Doubles, given by their words, divided by their scale.
__device__ __forceinline__ float scaled(uint32_t w, int scale_code) {
  return (float)__builtin_ldexp(__builtin_bit_cast(double, (uint64_t)w << 32), 127 - scale_code);
}
// The largest over aligned groups of N lanes.
template <int N>
__device__ __forceinline__ uint32_t max_of_group(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppXor1, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppXor2, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppHalfMirror, 0xF, 0xF, false));
  if constexpr (N == 16) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppMirror, 0xF, 0xF, false));
  return v;
}

template <class T, int DH, bool STREAM>
__device__ __forceinline__ void append_qk(const PagedAppendArgs& a, const QuantPages& pages, int wave, int slices) {
  constexpr int GL = DH / 8, HW = 64 / GL;   // lanes of a head, heads of a wave at a time
  constexpr int kAhead = 2, kAheadK = 1;     // groups of heads that are loaded at once, of queries and of keys
  const PagedPool& p = a.pool;
  const int row = wave / slices, slice = wave % slices;
  if (row >= a.n_rows) return;
  const int sub = (threadIdx.x & 63) / GL, j = threadIdx.x & (GL - 1);   // one of the wave's heads, a lane of it
  const bool turned = 4 * j < a.n_pairs;
  const int c0 = turned ? 4 * j : 8 * j, c1 = turned ? a.n_pairs + 4 * j : c0 + 4;
  const int slot = a.row_slot[row];
  const QuantPlace at = quant_place(p, a.row_seq[row], slot);
  double cs[4] = {}, sn[4] = {};
  if (turned) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pair = c0 + i, axis = pair < a.end0 ? 0 : pair < a.end1 ? 1 : 2;
      const int pos = a.positions ? a.positions[axis * a.position_stride + row] : slot;
      const double t = (double)pos * a.turns[pair];
      sine_cosine(t - rint(t), sn[i], cs[i]);
    }
  }
  // groups g0, g0 + slices, .. of the row's heads from `src`, AHEAD loaded at once, computed in the sines' type, each
  // handed to `put` with its two chunks
  auto heads_of = [&](auto ahead, const auto& sine, const auto& cosine, int g0, int heads, const uint16_t* src,
                      const uint16_t* gain, auto put) {
    constexpr int AHEAD = decltype(ahead)::value;
    typedef typename std::remove_const<typename std::remove_reference<decltype(sine[0])>::type>::type Real;
    pu16x4 w0 = {0, 0, 0, 0}, w1 = w0;
    if (gain) w0 = *(const pu16x4*)(gain + c0), w1 = *(const pu16x4*)(gain + c1);
    for (int g = g0; g * HW < heads; g += slices * AHEAD) {
      const int h0 = g * HW + sub;
      pu16x4 x0[AHEAD], x1[AHEAD];
#pragma unroll
      for (int s = 0; s < AHEAD; ++s) {   // past the last head: it again
        const int h = min(h0 + s * slices * HW, heads - 1);
        x0[s] = once<STREAM>((const pu16x4*)(src + h * DH + c0));
        x1[s] = once<STREAM>((const pu16x4*)(src + h * DH + c1));
      }
#pragma unroll
      for (int s = 0; s < AHEAD; ++s) {
        Real u[4], w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = T::up(x0[s][i]), w[i] = T::up(x1[s][i]);
        if (gain) {
          auto mean_square = [&](Real eps) {
            Real ss = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) ss += u[i] * u[i] + w[i] * w[i];
            return sum_of_group<GL>(ss) * (Real)(1.f / DH) + eps;
          };
          Real mean = mean_square(a.eps);
          // Squares that 32 bits may not hold: of the head times a power of two (the mean is the same in all its lanes).
          if constexpr (std::is_same<Real, float>::value)
            if (__builtin_expect(!(mean >= 0x1p-100f && mean <= 0x1p120f), 0)) {
              const float f = mean > 1.f ? 0x1p-100f : 0x1p100f;
#pragma unroll
              for (int i = 0; i < 4; ++i) u[i] *= f, w[i] *= f;
              mean = mean_square(a.eps * f * f);
            }
          const Real r = inverse_root(mean);
#pragma unroll
          for (int i = 0; i < 4; ++i) u[i] = u[i] * r * T::up(w0[i]), w[i] = w[i] * r * T::up(w1[i]);
        }
        if (turned)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const Real x = u[i], y = w[i];
            u[i] = x * cosine[i] - y * sine[i];
            w[i] = y * cosine[i] + x * sine[i];
          }
        put(h0 + s * slices * HW, u, w);
      }
    }
  };
  // keys first: what they need in double is not kept for the queries
  const int k_groups = (p.Hk + HW - 1) / HW;
  if (slice < k_groups)
    heads_of(std::integral_constant<int, kAheadK>{}, sn, cs, slice, p.Hk, a.kin + row * a.k_stride, a.k_norm,
             [&](int h, const double* u, const double* w) {
      constexpr uint32_t kMost = (uint32_t)(__builtin_bit_cast(uint64_t, (double)QuantMost<T>::value) >> 32);
      uint32_t x[4], y[4], most = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = high_word(u[i]);
        y[i] = high_word(w[i]);
        most = max(most, max(counted_word(x[i]), counted_word(y[i])));
      }
      most = max_of_group<GL>(most);
      if (h >= p.Hk || at.page < 0) return;
      const int64_t to = (((int64_t)at.page * p.Hk + h) << p.page_shift) + at.off;
      const int code = scale_code_of_word(min(most, kMost));
      float xs[4], ys[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) xs[i] = scaled(x[i], code), ys[i] = scaled(y[i], code);
      if (__builtin_expect(most > kMost, 0))   // finite values past the largest code
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (fabsf(xs[i]) < INFINITY) xs[i] = fminf(fmaxf(xs[i], -kMostCode), kMostCode);
          if (fabsf(ys[i]) < INFINITY) ys[i] = fminf(fmaxf(ys[i], -kMostCode), kMostCode);
        }
      *(uint32_t*)(pages.k + to * DH + c0) = encoded4(xs, 1.f);
      *(uint32_t*)(pages.k + to * DH + c1) = encoded4(ys, 1.f);
      if (c0 == 0) pages.k_scale[to] = (uint8_t)code;
    });
  if (!a.q_out) return;
  float cos_q[4], sin_q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) cos_q[i] = (float)cs[i], sin_q[i] = (float)sn[i];
  // query groups go on where the key groups ended
  const int g = slice < k_groups ? (slices - (k_groups - slice) % slices) % slices : slice - k_groups;
  heads_of(std::integral_constant<int, kAhead>{}, sin_q, cos_q, g, p.H, a.q + row * a.q_stride, a.q_norm,
           [&](int h, const float* u, const float* w) {
    uint16_t* to = a.q_out + row * a.q_out_stride + h * DH;
    if (h >= p.H) return;
    once<STREAM>((pu32x2*)(to + c0), pu32x2{pack2<T>(u[0], u[1]), pack2<T>(u[2], u[3])});
    once<STREAM>((pu32x2*)(to + c1), pu32x2{pack2<T>(w[0], w[1]), pack2<T>(w[2], w[3])});
  });
}

template <class T, int DH, bool STREAM>
__device__ __forceinline__ void append_v(const PagedAppendArgs& a, const QuantPages& pages, int block) {
  constexpr int R = kRows, LR = R + 7;   // rows in LDS: the last run of eight may reach past the workgroup's own
  constexpr int LS = DH + 8;             // bytes from row to row
  __shared__ __attribute__((aligned(16))) uint8_t codes[LR * LS];
  __shared__ int s_page[LR], s_off[LR];
  __shared__ uint64_t s_lead, s_lone;
  const PagedPool& p = a.pool;
  const int h = block % p.Hk, r0 = block / p.Hk * R, tid = threadIdx.x, lane = tid & 63;
  constexpr int C = DH / 8, L = (LR * C + kThreads - 1) / kThreads;   // 16-byte chunks of a row, of a thread
  pu32x4 x[L];
#pragma unroll
  for (int k = 0; k < L; ++k) {   // past the last row: it again
    const int i = tid + k * kThreads, r = min(r0 + min(i / C, LR - 1), a.n_rows - 1);
    x[k] = once<STREAM>((const pu32x4*)(a.vin + r * a.v_stride + h * DH + i % C * 8));
  }
  // Lane i of the first wave: row r0 - 7 + i.
  if (tid < 64) {
    const int r = r0 - 7 + lane;
    QuantPlace at{-1, 0};
    if (r >= 0 && r < a.n_rows && lane < LR + 7) at = quant_place(p, a.row_seq[r], a.row_slot[r]);
    const int page1 = __shfl_up(at.page, 1), off1 = __shfl_up(at.off, 1);
    const uint64_t here = __ballot(at.page >= 0), first = __ballot((at.off & 7) == 0);
    const uint64_t follows = __ballot(lane > 0 && at.page >= 0 && page1 == at.page && off1 + 1 == at.off);
    uint64_t lead = here & first;   // rows that start eight slots in a row
#pragma unroll
    for (int k = 1; k < 8; ++k) lead &= follows >> k;
    uint64_t run = lead;            // rows of such runs
#pragma unroll
    for (int k = 1; k < 8; ++k) run |= lead << k;
    if (lane >= 7 && lane < LR + 7) s_page[lane - 7] = at.page, s_off[lane - 7] = at.off;
    if (lane == 0) s_lead = lead >> 7 & (((uint64_t)1 << R) - 1), s_lone = (here & ~run) >> 7 & (((uint64_t)1 << R) - 1);
  }
  int scale[L];
#pragma unroll
  for (int k = 0; k < L; ++k) {
    const int i = tid + k * kThreads;
    float y[8], most = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = bounded<T>(T::up((uint16_t)(x[k][e >> 1] >> (16 * (e & 1)))));
      most = fmaxf(most, counted(y[e]));
    }
    scale[k] = scale_code(group_max<C>(most));
    const float f = inverse_scale(scale[k]);
    if (i < LR * C) *(pu32x2*)(codes + i / C * LS + i % C * 8) = pu32x2{encoded4(y, f), encoded4(y + 4, f)};
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < L; ++k) {
    const int i = tid + k * kThreads, r = i / C;
    if (i % C == 0 && r < R && s_page[r] >= 0)
      pages.v_scale[(((int64_t)s_page[r] * p.Hk + h) << p.page_shift) + s_off[r]] = (uint8_t)scale[k];
  }
  auto page_at = [&](int r) { return pages.v + ((((int64_t)s_page[r] * p.Hk + h) * DH) << p.page_shift) + s_off[r]; };
  // runs: pairs of dimensions, 8 bytes of each; DH / 2 threads to a run
  constexpr int PT = DH / 2, PR = kThreads / PT;
  int turn = 0;
  for (uint64_t m = s_lead; m; m &= m - 1, ++turn) {
    const int r = __builtin_ctzll(m), dim = tid % PT * 2;
    if (turn % PR == tid / PT) {
      uint32_t y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = *(const uint16_t*)(codes + (r + k) * LS + dim);
      pu32x2 even = {0, 0}, odd = {0, 0};
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        even[k >> 2] |= (y[k] & 0xff) << (8 * (k & 3));
        odd[k >> 2] |= (y[k] >> 8) << (8 * (k & 3));
      }
      uint8_t* to = page_at(r) + (dim << p.page_shift);
      *(pu32x2*)to = even;
      *(pu32x2*)(to + (1 << p.page_shift)) = odd;
    }
  }
  // rows that stand alone: 16 rows to a row of lanes
  if (const uint64_t lone = s_lone)
#pragma unroll
    for (int b = 0; b < R; b += 16) {
      const int r = b + (tid & 15), d0 = tid >> 4;
      if (!(lone >> r & 1)) continue;
      uint8_t* to = page_at(r) + (d0 << p.page_shift);
#pragma unroll
      for (int k = 0; k < DH; k += kThreads / 16) to[k << p.page_shift] = codes[r * LS + d0 + k];
    }
}

// (Seven waves to a SIMD, 72 registers.  With six, of 74, 21 627 rows took 100.9 us for 98.9.)
template <class T, int DH, bool STREAM>
__global__ __launch_bounds__(kThreads, 7) void k_quant_append(const PagedAppendArgs a, const QuantPages pages, int v_blocks,
                                                           int slices) {
  const int qk = gridDim.x - v_blocks;   // queries and keys first: 98 us for 103 (21 627 rows), 28.3 for 31.3 (2368)
  if ((int)blockIdx.x >= qk) append_v<T, DH, STREAM>(a, pages, blockIdx.x - qk);
  else append_qk<T, DH, STREAM>(a, pages, blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), slices);
}

// Reads 64 rows of one head.  Keys: DH / 16 threads to a row, 16 codes each.  Values: where sixteen
// rows are sixteen slots in a row, a thread loads 16 bytes of one dimension, else it gathers them
// byte by byte; they cross over to rows in LDS.
template <class T, int DH>
__global__ __launch_bounds__(kReadThreads) void k_quant_read(const QuantReadArgs a) {
  constexpr int R = kReadRows, CL = DH / 16;
  constexpr int LS = DH + 8;   // bytes from row to row
  __shared__ __attribute__((aligned(16))) uint8_t codes[R * LS];
  __shared__ int s_page[R], s_off[R];
  __shared__ uint64_t s_lead, s_lone;
  const PagedPool& p = a.pool;
  const int h = blockIdx.x % p.Hk, r0 = blockIdx.x / p.Hk * R, tid = threadIdx.x, lane = tid & 63;
  if (tid < 64) {
    const int r = r0 + lane;
    QuantPlace at{-1, 0};
    if (lane < R && r < a.n_rows) at = quant_place(p, a.row_seq[r], a.row_slot[r]);
    const int page1 = __shfl_up(at.page, 1), off1 = __shfl_up(at.off, 1);
    const uint64_t here = __ballot(at.page >= 0), first = __ballot((at.off & 15) == 0);
    const uint64_t follows = __ballot(lane > 0 && at.page >= 0 && page1 == at.page && off1 + 1 == at.off);
    uint64_t lead = here & first;   // rows that start sixteen slots in a row
#pragma unroll
    for (int k = 1; k < 16; ++k) lead &= follows >> k;
    uint64_t run = lead;
#pragma unroll
    for (int k = 1; k < 16; ++k) run |= lead << k;
    if (lane < R) s_page[lane] = at.page, s_off[lane] = at.off;
    if (lane == 0) s_lead = lead, s_lone = here & ~run;
  }
  __syncthreads();
  auto slot_at = [&](int r) { return (((int64_t)s_page[r] * p.Hk + h) << p.page_shift) + s_off[r]; };
  auto put = [&](uint16_t* out, int64_t stride, int i, pu32x4 c, float f) {   // 16 codes of row i / CL
    uint16_t* to = out + (int64_t)(r0 + i / CL) * stride + h * DH + i % CL * 16;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      __builtin_nontemporal_store(pu32x4{decoded<T, false>(c[2 * e], f), decoded<T, true>(c[2 * e], f),
                                         decoded<T, false>(c[2 * e + 1], f), decoded<T, true>(c[2 * e + 1], f)}, (pu32x4*)(to + 8 * e));
  };
  // The thread's key chunk and dimension of a run are under way together.
  static_assert(R * CL <= kReadThreads && R / 16 * DH <= kReadThreads, "one chunk and one dimension of a run to a thread");
  const bool mine = tid < R * CL && r0 + tid / CL < a.n_rows, here = mine && s_page[tid / CL] >= 0;
  pu32x4 kc = {0, 0, 0, 0}, vc = kc;
  float kf = 0.f, vf = 0.f;
  if (here && a.k_out) {
    kc = *(const pu32x4*)(a.pages.k + slot_at(tid / CL) * DH + tid % CL * 16);
    kf = scale_of(a.pages.k_scale[slot_at(tid / CL)]);
  }
  auto page_at = [&](int r) { return a.pages.v + ((((int64_t)s_page[r] * p.Hk + h) * DH) << p.page_shift) + s_off[r]; };
  uint64_t leads = s_lead;
  for (int k = tid / DH; k > 0; --k) leads &= leads - 1;
  const int run = leads ? __builtin_ctzll(leads) : -1, dim = tid % DH;
  if (a.v_out) {
    if (run >= 0) vc = *(const pu32x4*)(page_at(run) + (dim << p.page_shift));
    if (here) vf = scale_of(a.pages.v_scale[slot_at(tid / CL)]);
  }
  if (a.k_out && mine) put(a.k_out, a.k_stride, tid, kc, kf);
  if (!a.v_out) return;
  if (run >= 0)
#pragma unroll
    for (int k = 0; k < 16; ++k) codes[(run + k) * LS + dim] = (uint8_t)(vc[k >> 2] >> (8 * (k & 3)));
  if (const uint64_t lone = s_lone)
    for (int b = 0; b < R; b += 16) {
      const int r = b + (tid & 15), d0 = tid >> 4;
      if (!(lone >> r & 1)) continue;
      const uint8_t* from = page_at(r) + (d0 << p.page_shift);
#pragma unroll
      for (int k = 0; k < DH; k += kReadThreads / 16) codes[r * LS + d0 + k] = from[k << p.page_shift];
    }
  __syncthreads();
  if (!mine) return;
  const pu32x2* c = (const pu32x2*)(codes + tid / CL * LS + tid % CL * 16);
  put(a.v_out, a.v_stride, tid, here ? pu32x4{c[0][0], c[0][1], c[1][0], c[1][1]} : pu32x4{0, 0, 0, 0}, vf);
}

template <class T, int DH>
static hipError_t append(const PagedAppendArgs& a, const QuantPages& to, hipStream_t s) {
  constexpr int HW = 512 / DH;
  const int groups = (a.q_out ? (a.pool.H + HW - 1) / HW : 0) + (a.pool.Hk + HW - 1) / HW;
  const int want = (kFill + a.n_rows - 1) / a.n_rows, slices = want < groups ? want : groups;
  const int64_t v_blocks = (int64_t)((a.n_rows + kRows - 1) / kRows) * a.pool.Hk;
  const int64_t qk_blocks = ((int64_t)a.n_rows * slices + kWaves - 1) / kWaves;
  const int64_t bytes = (int64_t)a.n_rows * ((a.q_out ? 4 * a.pool.H : 0) + 6 * a.pool.Hk) * DH;
  const unsigned grid = (unsigned)(v_blocks + qk_blocks);
  if (bytes > kLastCache) k_quant_append<T, DH, true><<<grid, kThreads, 0, s>>>(a, to, (int)v_blocks, slices);
  else k_quant_append<T, DH, false><<<grid, kThreads, 0, s>>>(a, to, (int)v_blocks, slices);
  return hipGetLastError();
}

template <class T, int DH>
static hipError_t read(const QuantReadArgs& a, hipStream_t s) {
  k_quant_read<T, DH><<<(unsigned)((int64_t)((a.n_rows + kReadRows - 1) / kReadRows) * a.pool.Hk), kReadThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_quant_append(const PagedAppendArgs& a, const QuantPages& to, int dtype, hipStream_t s) {
  if (dtype == GVC_BF16) return a.pool.dh == 64 ? append<Bf16, 64>(a, to, s) : append<Bf16, 128>(a, to, s);
  return a.pool.dh == 64 ? append<Fp16, 64>(a, to, s) : append<Fp16, 128>(a, to, s);
}

hipError_t launch_quant_read(const QuantReadArgs& a, int dtype, hipStream_t s) {
  if (dtype == GVC_BF16) return a.pool.dh == 64 ? read<Bf16, 64>(a, s) : read<Bf16, 128>(a, s);
  return a.pool.dh == 64 ? read<Fp16, 64>(a, s) : read<Fp16, 128>(a, s);
}

}  // namespace gvc
