// The quantised paged cache's operators in simple form: a wave for each head of each row.
#include "gvc_paged_rows.h"
#include "gvc_quant.h"

namespace gvc {

// Head `h` of a row: queries, then keys, then values.
template <class T, int DH>
__global__ __launch_bounds__(64) void k_quant_append(const PagedAppendArgs a, const QuantPages to) {
  constexpr int N = DH / 64;
  const PagedPool& p = a.pool;
  const int H = a.q_out ? p.H : 0, heads = H + 2 * p.Hk, row = blockIdx.x / heads, lane = threadIdx.x;
  int h = blockIdx.x % heads;
  const int kind = h < H ? 0 : h < H + p.Hk ? 1 : 2;
  h -= kind == 0 ? 0 : kind == 1 ? H : H + p.Hk;
  const uint16_t* src = kind == 0 ? a.q + row * a.q_stride : kind == 1 ? a.kin + row * a.k_stride : a.vin + row * a.v_stride;
  const uint16_t* gain = kind == 0 ? a.q_norm : kind == 1 ? a.k_norm : nullptr;
  const int slot = a.row_slot[row];
  const QuantPlace at = quant_place(p, a.row_seq[row], slot);
  __shared__ float lds[DH];
  float x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = T::up(src[h * DH + lane + 64 * i]);
  if (gain) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) ss += x[i] * x[i];
    const float r = 1.f / sqrtf(wave_sum(ss) * (1.f / DH) + a.eps);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = x[i] * r * T::up(gain[lane + 64 * i]);
  }
  if (kind < 2) {
#pragma unroll
    for (int i = 0; i < N; ++i) lds[lane + 64 * i] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int d = lane + 64 * i, n = a.n_pairs, pair = d < n ? d : d - n;
      if (d >= 2 * n) continue;
      const int axis = pair < a.end0 ? 0 : pair < a.end1 ? 1 : 2;
      const int pos = a.positions ? a.positions[axis * a.position_stride + row] : slot;
      double t = (double)pos * a.turns[pair];
      t -= rint(t);
      t *= 2;
      float sn, cs;
      sincospif((float)t, &sn, &cs);
      const float rest = (float)(t - (double)(float)t) * 3.14159274f, s0 = sn;   // what fp32 cut from the angle
      sn = fmaf(cs, rest, sn);
      cs = fmaf(-s0, rest, cs);
      x[i] = d < n ? x[i] * cs - lds[d + n] * sn : x[i] * cs + lds[d - n] * sn;
    }
  }
  if (kind == 0) {
    uint16_t* q = a.q_out + row * a.q_out_stride + h * DH;
#pragma unroll
    for (int i = 0; i < N; ++i) q[lane + 64 * i] = (uint16_t)pack2<T>(x[i], 0.f);
    return;
  }
  if (at.page < 0) return;
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = bounded<T>(x[i]);
    most = fmaxf(most, counted(x[i]));
  }
  const int code = scale_code(wave_max(most));
  const float inv = inverse_scale(code);
  const int64_t head = (int64_t)at.page * p.Hk + h;
  (kind == 1 ? to.k_scale : to.v_scale)[(head << p.page_shift) + at.off] = (uint8_t)code;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int d = lane + 64 * i;
    const uint8_t c = (uint8_t)encoded(x[i] * inv, 0.f);
    if (kind == 1) to.k[((head << p.page_shift) + at.off) * DH + d] = c;
    else to.v[((head * DH + d) << p.page_shift) + at.off] = c;
  }
}

template <class T, int DH>
__global__ __launch_bounds__(64) void k_quant_read(const QuantReadArgs a) {
  const PagedPool& p = a.pool;
  const int row = blockIdx.x / p.Hk, h = blockIdx.x % p.Hk, lane = threadIdx.x;
  const QuantPlace at = quant_place(p, a.row_seq[row], a.row_slot[row]);
  const int64_t head = (int64_t)max(at.page, 0) * p.Hk + h;
  for (int d = lane; d < DH; d += 64) {
    uint16_t k = 0, v = 0;
    if (at.page >= 0) {
      const int64_t j = (head << p.page_shift) + at.off;
      k = (uint16_t)decoded<T, false>(a.pages.k[j * DH + d], scale_of(a.pages.k_scale[j]));
      v = (uint16_t)decoded<T, false>(a.pages.v[((head * DH + d) << p.page_shift) + at.off], scale_of(a.pages.v_scale[j]));
    }
    if (a.k_out) a.k_out[row * a.k_stride + h * DH + d] = k;
    if (a.v_out) a.v_out[row * a.v_stride + h * DH + d] = v;
  }
}

#define GVC_QUANT_LAUNCH(kernel, dh, grid, ...)                                       \
  do {                                                                                \
    if ((grid) >= 1 << 26) return hipErrorInvalidConfiguration;                       \
    if (dtype == GVC_BF16) {                                                          \
      if (dh == 64) kernel<Bf16, 64><<<(unsigned)(grid), 64, 0, s>>>(__VA_ARGS__);    \
      else kernel<Bf16, 128><<<(unsigned)(grid), 64, 0, s>>>(__VA_ARGS__);            \
    } else {                                                                          \
      if (dh == 64) kernel<Fp16, 64><<<(unsigned)(grid), 64, 0, s>>>(__VA_ARGS__);    \
      else kernel<Fp16, 128><<<(unsigned)(grid), 64, 0, s>>>(__VA_ARGS__);            \
    }                                                                                 \
    return hipGetLastError();                                                         \
  } while (0)

hipError_t launch_quant_append(const PagedAppendArgs& a, const QuantPages& to, int dtype, hipStream_t s) {
  GVC_QUANT_LAUNCH(k_quant_append, a.pool.dh, (int64_t)a.n_rows * ((a.q_out ? a.pool.H : 0) + 2 * a.pool.Hk), a, to);
}
hipError_t launch_quant_read(const QuantReadArgs& a, int dtype, hipStream_t s) {
  GVC_QUANT_LAUNCH(k_quant_read, a.pool.dh, (int64_t)a.n_rows * a.pool.Hk, a);
}

}  // namespace gvc
