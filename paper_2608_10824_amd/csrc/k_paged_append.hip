// Rows into the paged cache, with the norm and rotation of queries and keys.
//
// q and k of a row: x' = x / sqrt(mean x^2 + eps) * gain per head, then pair i
// of dimensions (i, i + n) turns by position(axis of i) * theta^(-i/n); v goes
// in as it is.  The angle is taken in full turns in double precision and
// reduced to [-1/2, 1/2] before it is rounded to fp32, so a far position keeps
// its angle (fp32 alone is off by a radian at position 10^7).
#include "gvc_paged.h"

namespace gvc {

constexpr int kAppendThreads = 256;

// One group of DH / 8 lanes per (row, head).  A lane holds two chunks of four
// dimensions that turn together (4j.. and n + 4j.., j the lane of the group),
// or past the rotated dimensions two neighbouring chunks, so that a pair never
// crosses lanes.
template <class T, int DH>
__global__ __launch_bounds__(kAppendThreads) void k_paged_append(const PagedAppendArgs a) {
  constexpr int GL = DH / 8;   // lanes of a group
  const PagedPool& p = a.pool;
  const int heads = (a.q_out ? p.H : 0) + 2 * p.Hk;
  const int64_t item = ((int64_t)blockIdx.x * kAppendThreads + threadIdx.x) / GL;
  if (item >= (int64_t)a.n_rows * heads) return;   // uniform over a group
  const int row = (int)(item / heads), lane = threadIdx.x & (GL - 1);
  int h = (int)(item % heads) + (a.q_out ? 0 : p.H);
  const int slot = a.row_slot[row], seq = a.row_seq[row];
  // the place of the row in the pool, or none
  int page = -1;
  if ((unsigned)seq < (unsigned)p.n_seqs && slot >= 0 && (slot >> p.page_shift) < p.max_pages)
    page = p.table[(int64_t)seq * p.max_pages + (slot >> p.page_shift)];
  const bool stored = (unsigned)page < (unsigned)p.n_pages;
  const int off = slot & ((1 << p.page_shift) - 1);
  if (h >= p.H + p.Hk) {
    h -= p.H + p.Hk;
    if (!stored) return;
    const pu16x8 x = *(const pu16x8*)(a.vin + row * a.v_stride + h * DH + lane * 8);
    uint16_t* dst = p.v + (((int64_t)page * p.Hk + h) * DH << p.page_shift) + off;
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[(lane * 8 + i) << p.page_shift] = x[i];
    return;
  }
  const bool is_q = h < p.H;
  const uint16_t* src = is_q ? a.q + row * a.q_stride + h * DH : a.kin + row * a.k_stride + (h - p.H) * DH;
  const bool turned = 4 * lane < a.n_pairs;
  const int c0 = turned ? 4 * lane : 8 * lane, c1 = turned ? a.n_pairs + 4 * lane : c0 + 4;
  const pu16x4 x0 = *(const pu16x4*)(src + c0), x1 = *(const pu16x4*)(src + c1);
  float u[4], w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = T::up(x0[i]), w[i] = T::up(x1[i]);
  const uint16_t* gain = is_q ? a.q_norm : a.k_norm;
  if (gain) {   // uniform over a group
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) ss += u[i] * u[i] + w[i] * w[i];
#pragma unroll
    for (int m = 1; m < GL; m <<= 1) ss += __shfl_xor(ss, m);
    const float r = 1.f / sqrtf(ss * (1.f / DH) + a.eps);
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = u[i] * r * T::up(gain[c0 + i]), w[i] = w[i] * r * T::up(gain[c1 + i]);
  }
  if (turned) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pair = c0 + i;
      const int axis = pair < a.end0 ? 0 : pair < a.end1 ? 1 : 2;
      const int pos = a.positions ? a.positions[axis * a.position_stride + row] : slot;
      double t = (double)pos * a.turns[pair];
      t -= rint(t);
      float sn, cs;
      sincospif(2.f * (float)t, &sn, &cs);
      const float x = u[i], y = w[i];
      u[i] = x * cs - y * sn;
      w[i] = y * cs + x * sn;
    }
  }
  uint16_t* dst;
  if (is_q) {
    dst = a.q_out + row * a.q_out_stride + h * DH;
  } else {
    if (!stored) return;
    dst = p.k + ((((int64_t)page * p.Hk + h - p.H) << p.page_shift) + off) * DH;
  }
  *(pu32x2*)(dst + c0) = pu32x2{pack2<T>(u[0], u[1]), pack2<T>(u[2], u[3])};
  *(pu32x2*)(dst + c1) = pu32x2{pack2<T>(w[0], w[1]), pack2<T>(w[2], w[3])};
}

template <class T, int DH>
static hipError_t append(const PagedAppendArgs& a, hipStream_t s) {
  const int64_t lanes = (int64_t)a.n_rows * ((a.q_out ? a.pool.H : 0) + 2 * a.pool.Hk) * (DH / 8);
  const unsigned grid = (unsigned)((lanes + kAppendThreads - 1) / kAppendThreads);
  k_paged_append<T, DH><<<grid, kAppendThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppendArgs& a, int dtype, hipStream_t s) {
  if (dtype == GVC_BF16) return a.pool.dh == 64 ? append<Bf16, 64>(a, s) : append<Bf16, 128>(a, s);
  return a.pool.dh == 64 ? append<Fp16, 64>(a, s) : append<Fp16, 128>(a, s);
}

}  // namespace gvc
