// Attention of rows over the paged cache.
//
// One wave per (sequence, tile of 16 query rows, key-value head), where the
// query heads that share a key-value head count as rows of one tile: virtual
// row v of a sequence is row v / G, head v % G of the group.  Keys go by in
// tiles of 32; S^T = K Q^T and O^T += V^T P^T run on 16x16x32 MFMA with an
// online softmax in fp32.  A lane's scores in S^T belong to one query, and the
// keys of a tile are taken in an order in which they are also the lane's
// operand of the second product, so probabilities never cross lanes.
#include "gvc_paged.h"

namespace gvc {

constexpr int kAttnThreads = 256;

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// A tile of 16 virtual rows: the lane's query and what it sees.
struct TileRows {
  int last;                // last slot of the lane's row (-1: none)
  int lo_all, hi_all;      // slots in (lo_all, hi_all] or below the sinks are seen by some row of the tile
  int lo_full, hi_full;    // slots in (lo_full, hi_full] or below sinks_full by every row
};

template <class T, int DH>
struct Tile16 {
  pf32x4 acc[DH / 16];   // O^T: dimensions 16 c + 4 g + i of the lane's query
  float m, l;            // running maximum (powers of two) and this lane's share of the sum
  bool any;              // the row saw a slot
};

// Visits the slots of tiles [t0, t1) of the tile's list (sink tiles, then the
// window's) for the lane's query.  CAREFUL: slots seen by some rows only are
// added key by key, so that NaN and infinities in V stay with the rows that
// see them.
template <class T, int DH, bool CAREFUL>
__device__ __forceinline__ void visit16(const PagedAttnArgs& a, int seq, int kvh, const pu32x4 (&qf)[DH / 32],
                                        const TileRows& r, int t0, int t1, int sink_tiles, int win_tile,
                                        Tile16<T, DH>& st) {
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  const int* table = p.table + (int64_t)seq * p.max_pages;
  const int in_page = (1 << p.page_shift) - 1;
#pragma unroll
  for (int c = 0; c < DH / 16; ++c) st.acc[c] = pf32x4{0, 0, 0, 0};
  st.m = -INFINITY;
  st.l = 0.f;
  st.any = false;
  float mb = 0.f;   // the maximum that scores are taken against: st.m, or 0 while that is -inf
  for (int t = t0; t < t1; ++t) {
    const int j0 = 32 * (t < sink_tiles ? t : t - sink_tiles + win_tile);
    // keys: row 4 g' + i of operand tile n is slot j0 + 8 g' + 4 n + i, so that lane group g's scores are those of
    // slots j0 + 8 g .. + 7
    const int jk = j0 + 8 * (col >> 2), jv = j0 + 8 * g;
    const int pk = table[min(jk >> p.page_shift, p.max_pages - 1)], pv = table[min(jv >> p.page_shift, p.max_pages - 1)];
    const bool okv = (unsigned)pv < (unsigned)p.n_pages;
    const uint16_t* kp = p.k + (((((int64_t)((unsigned)pk < (unsigned)p.n_pages ? pk : 0)) * p.Hk + kvh) << p.page_shift) +
                                (jk & in_page) + (col & 3)) * DH + g * 8;
    const uint16_t* vp = p.v + ((((int64_t)(okv ? pv : 0) * p.Hk + kvh) * DH + col) << p.page_shift) + (jv & in_page);
    pf32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
    for (int kk = 0; kk < DH / 32; ++kk)
#pragma unroll
      for (int n = 0; n < 2; ++n) s[n] = T::mfma16(*(const pu32x4*)(kp + n * 4 * DH + kk * 32), qf[kk], s[n]);
    pu32x4 vf[DH / 16];
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) vf[c] = *(const pu32x4*)(vp + ((16 * c) << p.page_shift));
    // seen by every row?
    const bool full = __all(okv) && j0 + 31 <= r.hi_full && j0 > r.lo_full;
    unsigned seen = 0xff;
    if (!full) {
      seen = 0;
      unsigned some = 0;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int j = jv + u;
        const bool in = j <= r.last && (a.window == 0 || j > r.last - a.window || j < a.n_sinks);
        const bool by = j <= r.hi_all && (j > r.lo_all || j < a.n_sinks);
        seen |= (unsigned)(okv && in) << u;
        some |= (unsigned)(okv && by) << u;
      }
      // values that no row of the tile sees become zeros (0 x NaN is NaN)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t keep = ((some >> (2 * w)) & 1 ? 0xffffu : 0u) | ((some >> (2 * w + 1)) & 1 ? 0xffff0000u : 0u);
#pragma unroll
        for (int c = 0; c < DH / 16; ++c) vf[c][w] &= keep;
      }
    }
    st.any |= seen != 0;
    float x[8], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      x[u] = (seen >> u) & 1 ? s[u >> 2][u & 3] * a.scale_log2e : -INFINITY;
      top = fmaxf(top, x[u]);
    }
    if (__any(top > st.m + kPagedLazy)) {
      const float mn = fmaxf(st.m, rows_max(top));
      const float nb = mn == -INFINITY ? 0.f : mn;
      const float f = __builtin_amdgcn_exp2f(st.m - nb);
      st.m = mn;
      mb = nb;
      st.l *= f;
#pragma unroll
      for (int c = 0; c < DH / 16; ++c) st.acc[c] *= f;
    }
    float pr[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      pr[u] = __builtin_amdgcn_exp2f(x[u] - mb + T::kShift);
      st.l += pr[u];
    }
    const pu32x4 pf = {pack2<T>(pr[0], pr[1]), pack2<T>(pr[2], pr[3]), pack2<T>(pr[4], pr[5]), pack2<T>(pr[6], pr[7])};
    if (!CAREFUL || full) {
#pragma unroll
      for (int c = 0; c < DH / 16; ++c) st.acc[c] = T::mfma16(vf[c], pf, st.acc[c]);
    } else {
      for (int u = 0; u < 32; ++u) {
        const bool mine = g == (u >> 3);
        const bool sees = ((unsigned)__shfl((int)seen, (u >> 3) * 16 + col) >> (u & 7)) & 1;
        const uint32_t half = u & 1 ? 0xffff0000u : 0xffffu;
        pu32x4 pu = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; ++w) pu[w] = mine && ((u & 7) >> 1) == w ? pf[w] & half : 0u;
#pragma unroll
        for (int c = 0; c < DH / 16; ++c) {
          pu32x4 vu;
#pragma unroll
          for (int w = 0; w < 4; ++w) vu[w] = mine && ((u & 7) >> 1) == w ? vf[c][w] & half : 0u;
          const pf32x4 o = T::mfma16(vu, pu, pf32x4{0, 0, 0, 0});
#pragma unroll
          for (int i = 0; i < 4; ++i) st.acc[c][i] += sees ? o[i] : 0.f;
        }
      }
    }
  }
}

template <class T, int DH>
__global__ __launch_bounds__(kAttnThreads) void k_paged_rows16(const PagedAttnArgs a) {
  __shared__ int first[kPagedMaxSeqs + 1];   // tiles before each sequence
  __shared__ int carry[kAttnThreads];
  const PagedPool& p = a.pool;
  const int G = p.H / p.Hk, S = p.n_seqs, tid = threadIdx.x;
  // tiles of a sequence's rows, summed over the sequences
  auto rows_of = [&](int s, int& begin) {
    if (!a.row_begin) {
      begin = s;
      return 1;
    }
    begin = min(max(a.row_begin[s], 0), a.n_rows);
    return max(min(a.row_begin[s + 1], a.n_rows) - begin, 0);
  };
  const int per = (S + kAttnThreads - 1) / kAttnThreads;
  int sum = 0, begin;
  for (int s = tid * per; s < min(S, (tid + 1) * per); ++s) sum += (rows_of(s, begin) * G + 15) >> 4;
  carry[tid] = sum;
  __syncthreads();
  int before = 0;
  for (int i = 0; i < tid; ++i) before += carry[i];
  for (int s = tid * per; s < min(S, (tid + 1) * per); ++s) {
    first[s] = before;
    before += (rows_of(s, begin) * G + 15) >> 4;
  }
  if (tid == kAttnThreads - 1) first[S] = before;
  __syncthreads();
  const int tile = blockIdx.x * (kAttnThreads / 64) + (tid >> 6), kvh = blockIdx.y;
  if (tile >= first[S]) return;
  int lo = 0, hi = S;   // first[lo] <= tile < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    (first[mid] <= tile ? lo : hi) = mid;
  }
  const int seq = lo, rows = rows_of(seq, begin);
  const int lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int v = (tile - first[seq]) * 16 + col;
  const bool live = v < rows * G;
  const int row = begin + min(v, rows * G - 1) / G, h = kvh * G + min(v, rows * G - 1) % G;
  TileRows r;
  const int slots = p.max_pages << p.page_shift;
  r.last = live ? min(a.row_begin ? max(a.row_last[row], -1) : max(a.row_last[row], 0) - 1, slots - 1) : -1;
  int big = r.last, small = r.last < 0 ? slots : r.last, least = live ? r.last : slots;
  for (int m = 1; m < 16; m <<= 1) {
    big = max(big, __shfl_xor(big, m));
    small = min(small, __shfl_xor(small, m));
    least = min(least, __shfl_xor(least, m));
  }
  r.hi_all = big;
  r.hi_full = least;
  r.lo_all = a.window ? small - a.window : -1;
  r.lo_full = a.window ? big - a.window : -1;
  // the tiles of 32 slots that some row sees: the sinks', then the window's
  const int end = (r.hi_all >> 5) + 1;
  const int win_lo = max(r.lo_all + 1, 0) >> 5;
  const int sink_tiles = a.window ? min(min((a.n_sinks + 31) >> 5, win_lo), end) : 0;
  const int win_tile = a.window ? max(win_lo, sink_tiles) : 0;
  const int tiles = r.hi_all < 0 ? 0 : sink_tiles + end - win_tile;
  pu32x4 qf[DH / 32];
#pragma unroll
  for (int kk = 0; kk < DH / 32; ++kk) qf[kk] = *(const pu32x4*)(a.q + row * a.q_stride + h * DH + g * 8 + kk * 32);
  Tile16<T, DH> st;
  visit16<T, DH, false>(a, seq, kvh, qf, r, 0, tiles, sink_tiles, win_tile, st);
  bool bad = false;
#pragma unroll
  for (int c = 0; c < DH / 16; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= !finite(st.acc[c][i]);
  if (__any(bad)) visit16<T, DH, true>(a, seq, kvh, qf, r, 0, tiles, sink_tiles, win_tile, st);
  const float l = rows_sum(st.l);
  const bool any = __shfl((int)st.any, col) | __shfl((int)st.any, col + 16) | __shfl((int)st.any, col + 32) |
                   __shfl((int)st.any, col + 48);
  if (!live) return;
  uint16_t* o = a.out + row * a.out_stride + h * DH + 4 * g;
  const float inv = 1.f / l;
#pragma unroll
  for (int c = 0; c < DH / 16; ++c) {
    pf32x4 x = st.acc[c] * inv;
    if (!any) x = pf32x4{0, 0, 0, 0};
    *(pu32x2*)(o + 16 * c) = pu32x2{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3])};
  }
}

template <class T, int DH>
static hipError_t rows16(const PagedAttnArgs& a, hipStream_t s) {
  const int64_t G = a.pool.H / a.pool.Hk;
  const int64_t tiles = a.row_begin ? (a.n_rows * G + 15) / 16 + a.pool.n_seqs : a.pool.n_seqs * ((G + 15) / 16);
  k_paged_rows16<T, DH><<<dim3((unsigned)((tiles + 3) / 4), a.pool.Hk), kAttnThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, int dtype, hipStream_t s) {
  if (dtype == GVC_BF16) return a.pool.dh == 64 ? rows16<Bf16, 64>(a, s) : rows16<Bf16, 128>(a, s);
  return a.pool.dh == 64 ? rows16<Fp16, 64>(a, s) : rows16<Fp16, 128>(a, s);
}

}  // namespace gvc
