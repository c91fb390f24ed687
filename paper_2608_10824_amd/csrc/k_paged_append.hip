// Rows into the paged cache, with the norm and rotation of queries and keys.
//
// q and k of a row: x' = x / sqrt(mean x^2 + eps) * gain per head, then pair i
// of dimensions (i, i + n) turns by position(axis of i) * theta^(-i/n); v goes
// in as it is.  The angle is taken in full turns in double precision and
// reduced to [-1/2, 1/2] before it is rounded to fp32, so a far position keeps
// its angle (fp32 alone is off by a radian at position 10^7).
//
// Everything is read and written once, so HBM bounds long calls and launch and
// load latency short ones.  One launch has two kinds of workgroups:
//  * Queries and keys: a wave takes one row and every slices-th group of heads
//    of it, DH / 8 lanes to a head, so the sines and cosines of a row are
//    computed once for the heads that follow.  A lane holds two chunks of four
//    dimensions that turn together (4 j.. and n + 4 j..), or past the rotated dimensions two
//    neighbouring chunks: a pair never crosses lanes.
//  * Values: pages hold them dim-major, so a row's values lie a page's width
//    apart.  A workgroup takes one head of 32 rows through LDS: where eight
//    rows fill eight slots in a row, a lane writes 16 bytes of one dimension;
//    rows that stand alone are written in 2-byte pieces, neighbouring lanes
//    taking neighbouring rows, so that pieces of one page meet in a cache line.
//
// Measured (bf16, 128 to a head): 19600 rows of whole prompts, 32 heads on 8, norm
// and three axes 107 us, 4.5 TB/s read and written, 88% of a copy; 2368 rows of 16
// sequences, about every second slot, 32 heads 36 us, 3.2 TB/s (parts of
// V's 32-byte sectors: 75 MB written for 58); one row 3.7 us.
#include "gvc_kernels.h"
#include "gvc_paged.h"

namespace gvc {

constexpr int kAppendThreads = 256, kAppendWaves = kAppendThreads / 64;
constexpr int kAppendRows = 32;      // rows of a workgroup of values, and 7 on both sides that its runs of eight may reach
constexpr int kAppendFill = 4096;    // waves of queries and keys that a call's rows are cut into, at least (8192: 5% slower at 750 rows)

// Where a row goes: its page (-1: nowhere) and the slot in it.
struct Place {
  int page, off;
};
__device__ __forceinline__ Place place_of(const PagedPool& p, int seq, int slot) {
  int page = -1;
  if ((unsigned)seq < (unsigned)p.n_seqs && slot >= 0 && (slot >> p.page_shift) < p.max_pages)
    page = p.table[(int64_t)seq * p.max_pages + (slot >> p.page_shift)];
  return {(unsigned)page < (unsigned)p.n_pages ? page : -1, slot & ((1 << p.page_shift) - 1)};
}

template <class T, int DH>
__device__ __forceinline__ void append_qk(const PagedAppendArgs& a, int wave, int slices) {
  constexpr int GL = DH / 8, HW = 64 / GL;   // lanes of a head, heads of a wave at a time
  constexpr int kAhead = 2;                  // groups of heads that are loaded at once
  const PagedPool& p = a.pool;
  const int row = wave / slices, slice = wave % slices;
  if (row >= a.n_rows) return;
  const int lane = threadIdx.x & 63, j = lane & (GL - 1);
  const bool turned = 4 * j < a.n_pairs;
  const int c0 = turned ? 4 * j : 8 * j, c1 = turned ? a.n_pairs + 4 * j : c0 + 4;
  const int slot = a.row_slot[row];
  const Place at = place_of(p, a.row_seq[row], slot);
  float cs[4], sn[4];
  if (turned) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pair = c0 + i, axis = pair < a.end0 ? 0 : pair < a.end1 ? 1 : 2;
      const int pos = a.positions ? a.positions[axis * a.position_stride + row] : slot;
      double t = (double)pos * a.turns[pair];
      t -= rint(t);
      sn[i] = __builtin_amdgcn_sinf((float)t);   // of a full turn's part, off by at most 2^-22.9 (measured)
      cs[i] = __builtin_amdgcn_cosf((float)t);
    }
  }
  // groups g0, g0 + slices, .. of the row's heads: from `src`, to `dst` where heads lie `step` apart (nullptr: nowhere)
  auto heads_of = [&](int g0, int heads, const uint16_t* src, uint16_t* dst, int64_t step, const uint16_t* gain) {
    pu16x4 w0 = {0, 0, 0, 0}, w1 = w0;
    if (gain) w0 = *(const pu16x4*)(gain + c0), w1 = *(const pu16x4*)(gain + c1);
    for (int h0 = g0 * HW + lane / GL; h0 - lane / GL < heads; h0 += slices * HW * kAhead) {
      pu16x4 x0[kAhead], x1[kAhead];
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {   // past the last head: it again
        const int h = min(h0 + s * slices * HW, heads - 1);
        x0[s] = *(const pu16x4*)(src + h * DH + c0);
        x1[s] = *(const pu16x4*)(src + h * DH + c1);
      }
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        const int h = h0 + s * slices * HW;
        float u[4], w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = T::up(x0[s][i]), w[i] = T::up(x1[s][i]);
        if (gain) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) ss += u[i] * u[i] + w[i] * w[i];
          const float r = rsqrtf(group_sum<GL>(ss) * (1.f / DH) + a.eps);
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
        if (h >= heads || !dst) continue;
        *(pu32x2*)(dst + h * step + c0) = pu32x2{pack2<T>(u[0], u[1]), pack2<T>(u[2], u[3])};
        *(pu32x2*)(dst + h * step + c1) = pu32x2{pack2<T>(w[0], w[1]), pack2<T>(w[2], w[3])};
      }
    }
  };
  const int q_groups = a.q_out ? (p.H + HW - 1) / HW : 0;
  if (slice < q_groups)
    heads_of(slice, p.H, a.q + row * a.q_stride, a.q_out + row * a.q_out_stride, DH, a.q_norm);
  // key groups go on where the query groups ended
  const int g = slice < q_groups ? (slices - (q_groups - slice) % slices) % slices : slice - q_groups;
  heads_of(g, p.Hk, a.kin + row * a.k_stride,
           at.page < 0 ? nullptr : p.k + (((int64_t)at.page * p.Hk << p.page_shift) + at.off) * DH, (int64_t)DH << p.page_shift,
           a.k_norm);
}

template <int DH>
__device__ __forceinline__ void append_v(const PagedAppendArgs& a, int block) {
  constexpr int R = kAppendRows, LR = R + 7;   // rows in LDS: the last run of eight may reach past the workgroup's own
  constexpr int LS = DH + 4;                   // 16-bit elements from row to row
  __shared__ __attribute__((aligned(16))) uint16_t vals[LR * LS + 4];
  __shared__ int s_page[LR], s_off[LR];
  __shared__ uint64_t s_lead, s_lone;
  const PagedPool& p = a.pool;
  const int h = block % p.Hk, r0 = block / p.Hk * R, tid = threadIdx.x, lane = tid & 63;
  constexpr int C = DH / 8, L = (LR * C + kAppendThreads - 1) / kAppendThreads;   // 16-byte chunks of a row, of a thread
  pu32x4 x[L];
#pragma unroll
  for (int k = 0; k < L; ++k) {   // past the last row: it again
    const int i = tid + k * kAppendThreads, r = min(r0 + min(i / C, LR - 1), a.n_rows - 1);
    x[k] = *(const pu32x4*)(a.vin + r * a.v_stride + h * DH + i % C * 8);
  }
  // Lane i of the first wave: row r0 - 7 + i.
  if (tid < 64) {
    const int r = r0 - 7 + lane;
    Place at{-1, 0};
    if (r >= 0 && r < a.n_rows && lane < LR + 7) at = place_of(p, a.row_seq[r], a.row_slot[r]);
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
#pragma unroll
  for (int k = 0; k < L; ++k) {
    const int i = tid + k * kAppendThreads;
    uint16_t* to = vals + i / C * LS + i % C * 8;
    if (i < LR * C) {
      *(pu32x2*)to = pu32x2{x[k][0], x[k][1]};
      *(pu32x2*)(to + 4) = pu32x2{x[k][2], x[k][3]};
    }
  }
  __syncthreads();
  auto page_at = [&](int r) { return p.v + ((((int64_t)s_page[r] * p.Hk + h) * DH) << p.page_shift) + s_off[r]; };
  // runs: pairs of dimensions, 16 bytes of each; DH / 2 threads to a run
  constexpr int PT = DH / 2, PR = kAppendThreads / PT;
  int turn = 0;
  for (uint64_t m = s_lead; m; m &= m - 1, ++turn) {
    const int r = __builtin_ctzll(m), dim = tid % PT * 2;
    if (turn % PR == tid / PT) {
      uint32_t y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = *(const uint32_t*)(vals + (r + k) * LS + dim);
      pu32x4 even, odd;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        even[k] = (y[2 * k] & 0xffff) | y[2 * k + 1] << 16;
        odd[k] = y[2 * k] >> 16 | (y[2 * k + 1] & 0xffff0000u);
      }
      uint16_t* to = page_at(r) + (dim << p.page_shift);
      *(pu32x4*)to = even;
      *(pu32x4*)(to + (1 << p.page_shift)) = odd;
    }
  }
  // rows that stand alone: 16 rows to a row of lanes
  if (const uint64_t lone = s_lone)
#pragma unroll
    for (int b = 0; b < R; b += 16) {
      const int r = b + (tid & 15), d0 = tid >> 4;
      if (!(lone >> r & 1)) continue;
      uint16_t* to = page_at(r) + (d0 << p.page_shift);
#pragma unroll
      for (int k = 0; k < DH; k += kAppendThreads / 16) to[k << p.page_shift] = vals[r * LS + d0 + k];
    }
}

template <class T, int DH>
__global__ __launch_bounds__(kAppendThreads) void k_paged_append(const PagedAppendArgs a, int v_blocks, int slices) {
  if ((int)blockIdx.x < v_blocks) append_v<DH>(a, blockIdx.x);
  else append_qk<T, DH>(a, (blockIdx.x - v_blocks) * kAppendWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), slices);
}

template <class T, int DH>
static hipError_t append(const PagedAppendArgs& a, hipStream_t s) {
  constexpr int HW = 512 / DH;
  const int groups = (a.q_out ? (a.pool.H + HW - 1) / HW : 0) + (a.pool.Hk + HW - 1) / HW;
  const int want = (kAppendFill + a.n_rows - 1) / a.n_rows, slices = want < groups ? want : groups;
  const int64_t v_blocks = (int64_t)((a.n_rows + kAppendRows - 1) / kAppendRows) * a.pool.Hk;
  const int64_t qk_blocks = ((int64_t)a.n_rows * slices + kAppendWaves - 1) / kAppendWaves;
  k_paged_append<T, DH><<<(unsigned)(v_blocks + qk_blocks), kAppendThreads, 0, s>>>(a, (int)v_blocks, slices);
  return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppendArgs& a, int dtype, hipStream_t s) {
  if (dtype == GVC_BF16) return a.pool.dh == 64 ? append<Bf16, 64>(a, s) : append<Bf16, 128>(a, s);
  return a.pool.dh == 64 ? append<Fp16, 64>(a, s) : append<Fp16, 128>(a, s);
}

}  // namespace gvc
