// Rows into the quantised paged cache, with the norm and rotation of queries
// and keys, and rows read back.
//
// The scale of a head is 2^e with the least e for which its largest magnitude is
// at most 448 * 2^e (from the bits of that magnitude), its codes are the values divided by it,
// which is exact, rounded once.  A rotated key is not rounded to 16 bits before.  The
// angle is taken in full turns in double precision and reduced to [-1/2, 1/2];
// what fp32 cuts from it then is made good in first order, so sine and cosine are off by
// little more than their own rounding.
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
#include "gvc_kernels.h"
#include "gvc_quant.h"

namespace gvc {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kRows = 32;      // rows of a workgroup of values, and 7 on both sides that its runs of eight may reach
constexpr int kReadThreads = 512, kReadRows = 64;   // (32 rows to 256 threads: 41 000 rows 70 us for 66)
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

// Four values times a power of two, as codes.
__device__ __forceinline__ uint32_t encoded4(const float* x, float f) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, lo, true);
}

template <class T, int DH, bool STREAM>
__device__ __forceinline__ void append_qk(const PagedAppendArgs& a, const QuantPages& pages, int wave, int slices) {
  constexpr int GL = DH / 8, HW = 64 / GL;   // lanes of a head, heads of a wave at a time
  constexpr int kAhead = 2;                  // groups of heads that are loaded at once
  const PagedPool& p = a.pool;
  const int row = wave / slices, slice = wave % slices;
  if (row >= a.n_rows) return;
  const int lane = threadIdx.x & 63, j = lane & (GL - 1);
  const bool turned = 4 * j < a.n_pairs;
  const int c0 = turned ? 4 * j : 8 * j, c1 = turned ? a.n_pairs + 4 * j : c0 + 4;
  const int slot = a.row_slot[row];
  const QuantPlace at = quant_place(p, a.row_seq[row], slot);
  float cs[4], sn[4];
  if (turned) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pair = c0 + i, axis = pair < a.end0 ? 0 : pair < a.end1 ? 1 : 2;
      const int pos = a.positions ? a.positions[axis * a.position_stride + row] : slot;
      double t = (double)pos * a.turns[pair];
      t = 2 * (t - rint(t));
      const float half = (float)t, rest = (float)(t - (double)half) * 3.14159274f;
      float s, c;
      sincospif(half, &s, &c);
      sn[i] = fmaf(c, rest, s);
      cs[i] = fmaf(-s, rest, c);
    }
  }
  // groups g0, g0 + slices, .. of the row's heads from `src`, each handed to `put` with its two chunks
  auto heads_of = [&](int g0, int heads, const uint16_t* src, const uint16_t* gain, auto put) {
    pu16x4 w0 = {0, 0, 0, 0}, w1 = w0;
    if (gain) w0 = *(const pu16x4*)(gain + c0), w1 = *(const pu16x4*)(gain + c1);
    for (int h0 = g0 * HW + lane / GL; h0 - lane / GL < heads; h0 += slices * HW * kAhead) {
      pu16x4 x0[kAhead], x1[kAhead];
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {   // past the last head: it again
        const int h = min(h0 + s * slices * HW, heads - 1);
        x0[s] = once<STREAM>((const pu16x4*)(src + h * DH + c0));
        x1[s] = once<STREAM>((const pu16x4*)(src + h * DH + c1));
      }
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        float u[4], w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = T::up(x0[s][i]), w[i] = T::up(x1[s][i]);
        if (gain) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) ss += u[i] * u[i] + w[i] * w[i];
          const float r = 1.f / sqrtf(group_sum<GL>(ss) * (1.f / DH) + a.eps);
#pragma unroll
          for (int i = 0; i < 4; ++i) u[i] = u[i] * r * T::up(w0[i]), w[i] = w[i] * r * T::up(w1[i]);
        }
        if (turned)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = u[i], y = w[i];
            u[i] = x * cs[i] - y * sn[i];
            w[i] = y * cs[i] + x * sn[i];
          }
        put(h0 + s * slices * HW, u, w);
      }
    }
  };
  const int q_groups = a.q_out ? (p.H + HW - 1) / HW : 0;
  if (slice < q_groups)
    heads_of(slice, p.H, a.q + row * a.q_stride, a.q_norm, [&](int h, const float* u, const float* w) {
      uint16_t* to = a.q_out + row * a.q_out_stride + h * DH;
      if (h >= p.H) return;
      once<STREAM>((pu32x2*)(to + c0), pu32x2{pack2<T>(u[0], u[1]), pack2<T>(u[2], u[3])});
      once<STREAM>((pu32x2*)(to + c1), pu32x2{pack2<T>(w[0], w[1]), pack2<T>(w[2], w[3])});
    });
  // key groups go on where the query groups ended
  const int g = slice < q_groups ? (slices - (q_groups - slice) % slices) % slices : slice - q_groups;
  heads_of(g, p.Hk, a.kin + row * a.k_stride, a.k_norm, [&](int h, float* u, float* w) {
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u[i] = bounded<T>(u[i]);
      w[i] = bounded<T>(w[i]);
      most = fmaxf(most, fmaxf(counted(u[i]), counted(w[i])));
    }
    const int code = scale_code(group_max<GL>(most));
    if (h >= p.Hk || at.page < 0) return;
    const int64_t to = (((int64_t)at.page * p.Hk + h) << p.page_shift) + at.off;
    const float f = inverse_scale(code);
    *(uint32_t*)(pages.k + to * DH + c0) = encoded4(u, f);
    *(uint32_t*)(pages.k + to * DH + c1) = encoded4(w, f);
    if (j == 0) pages.k_scale[to] = (uint8_t)code;
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

template <class T, int DH, bool STREAM>
__global__ __launch_bounds__(kThreads) void k_quant_append(const PagedAppendArgs a, const QuantPages pages, int v_blocks,
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
