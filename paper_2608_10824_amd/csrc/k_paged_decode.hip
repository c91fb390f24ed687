// Attention of one new token per sequence over the paged cache.
//
// The call reads every visible key and value once and computes little with
// them (about one multiply-add per byte and query head), so HBM bounds it: the
// kernel has to keep enough loads in flight on every compute unit, whatever the
// mix of lengths.  A workgroup takes one unit: a chunk of one sequence's 32-slot tiles for
// one key-value head, whose query heads (up to 16) are the columns of one MFMA
// tile.  The chunk length follows from the sum of the lengths, which only the
// GPU knows: every wave adds them up and finds its unit, so ragged batches come
// out in pieces of about equal work, and a batch that fills the GPU by itself
// is not split at all.  Within a unit the waves take tiles round robin, each
// with its own online softmax, and are joined in LDS; the chunks of a sequence
// are joined by a second launch, which the host leaves out where the page
// table cannot hold enough slots to be split.
//
// S^T = K Q^T and O^T += V^T P^T on 16x16x32 MFMA.  A lane's scores in S^T are
// of one query; the keys of a tile are ordered such that they are also the
// lane's operand of the second product, so probabilities stay in registers,
// and 16 bytes of V (dim-major pages) are one operand.  All queries of a unit
// see the same slots: what they do not see is zeroed in V (0 x NaN is NaN).
#include "gvc_paged.h"

namespace gvc {

constexpr int kDecWaves = 8;
constexpr int kDecMinChunk = 16;   // tiles: shorter sequences are not split
constexpr int kDecTarget = 1024;   // units that the chunk length aims at, four to a compute unit

// v, which is the same in every lane, as a scalar: loops and branches on it stay scalar.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// What a sequence's token sees, in tiles of 32 slots: tiles [0, sink_tiles) and from win_tile on.
struct SeqTiles {
  int last, sink_tiles, win_tile, tiles;
};

__device__ __forceinline__ SeqTiles seq_tiles(const PagedAttnArgs& a, int s) {
  SeqTiles t;
  t.last = min(max(a.row_last[s], 0), a.pool.max_pages << a.pool.page_shift) - 1;
  const int end = (t.last >> 5) + 1, win_lo = a.window ? max(t.last - a.window + 1, 0) >> 5 : 0;
  t.sink_tiles = a.window ? min((a.n_sinks + 31) >> 5, min(win_lo, end)) : 0;
  t.win_tile = max(win_lo, t.sink_tiles);
  t.tiles = t.last < 0 ? 0 : t.sink_tiles + end - t.win_tile;
  return t;
}

__device__ __forceinline__ int wave_scan(int v, int lane) {   // inclusive
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int o = __shfl_up(v, m);
    if (lane >= m) v += o;
  }
  return v;
}

// Tiles per chunk: the sum of the tiles over the units aimed at, in whole
// rounds of the workgroup's waves.  The same in every wave of both launches.
__device__ __forceinline__ int chunk_tiles(const PagedAttnArgs& a, int heads, int lane) {
  int total = 0;
  for (int s = lane; s < a.pool.n_seqs; s += 64) total += min(seq_tiles(a, s).tiles, 1 << 18);
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
  const long long c = ((long long)total * heads + kDecTarget - 1) / kDecTarget;
  return uniform(max((int)((c + kDecWaves - 1) / kDecWaves) * kDecWaves, kDecMinChunk));
}

__device__ __forceinline__ int chunks_of(int tiles, int chunk) { return max((tiles + chunk - 1) / chunk, 1); }

template <class T, int DH>
__global__ __launch_bounds__(kDecWaves * 64, 2) void k_paged_decode(const PagedAttnArgs a, float* part) {
  constexpr int NK = DH / 32, NO = DH / 16;
  extern __shared__ float lds[];   // [waves / 2][queries][DH + 4], then [waves][16][4]
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int G = p.H / p.Hk, blocks = (G + 15) >> 4, heads = p.Hk * blocks;
  const int chunk = chunk_tiles(a, heads, lane);
  // the sequence of this workgroup's chunk
  const int head = blockIdx.x % heads;
  int want = blockIdx.x / heads, seq = -1, c_idx = 0, n_chunks = 0;
  for (int s0 = 0; s0 < p.n_seqs && seq < 0; s0 += 64) {
    const int s = s0 + lane;
    const int n = s < p.n_seqs ? chunks_of(seq_tiles(a, s).tiles, chunk) : 0;
    const int sum = wave_scan(n, lane);
    const uint64_t past = __ballot(sum > want);
    if (past) {
      const int l = __builtin_ctzll(past);
      seq = s0 + l;
      n_chunks = __builtin_amdgcn_readlane(n, l);
      c_idx = want - (__builtin_amdgcn_readlane(sum, l) - n_chunks);
    } else {
      want -= __builtin_amdgcn_readlane(sum, 63);
    }
  }
  seq = uniform(seq);
  if (seq < 0) return;   // the grid is an upper bound; uniform over the workgroup
  c_idx = uniform(c_idx);
  n_chunks = uniform(n_chunks);
  SeqTiles st = seq_tiles(a, seq);
  st = {uniform(st.last), uniform(st.sink_tiles), uniform(st.win_tile), uniform(st.tiles)};
  const int t_end = min((c_idx + 1) * chunk, st.tiles);
  const int kvh = head / blocks, hb = head % blocks;
  const int qs = min(G - hb * 16, 16), h0 = kvh * G + hb * 16;
  const int* table = p.table + (int64_t)seq * p.max_pages;
  const int in_page = (1 << p.page_shift) - 1;
  auto tile_slot = [&](int t) { return 32 * (t < st.sink_tiles ? t : t - st.sink_tiles + st.win_tile); };

  pu32x4 qf[NK];
#pragma unroll
  for (int kk = 0; kk < NK; ++kk) {
    qf[kk] = *(const pu32x4*)(a.q + seq * a.q_stride + (h0 + min(col, qs - 1)) * DH + g * 8 + kk * 32);
    if (col >= qs) qf[kk] = pu32x4{0, 0, 0, 0};
  }
  pf32x4 acc[NO];
#pragma unroll
  for (int c = 0; c < NO; ++c) acc[c] = pf32x4{0, 0, 0, 0};
  float m = -INFINITY, mb = T::kShift, l = 0.f;   // maximum, what a score is shifted by, this lane's share of the sum
  unsigned any = 0;

  // The wave's tiles t0, t0 + waves, ...: page ids of 32 of them at a time, one
  // half tile (16 slots, always one page) to a lane.
  int ids = -1, ids_base = 0;
  const int t0 = c_idx * chunk + wv;
  auto load_ids = [&](int n) {   // of the wave's tiles n .. n + 31
    const int t = t0 + (n + (lane >> 1)) * kDecWaves;
    const int j = tile_slot(min(t, max(t_end - 1, 0))) + 16 * (lane & 1);
    const int id = table[min(j >> p.page_shift, p.max_pages - 1)];
    ids = (unsigned)id < (unsigned)p.n_pages ? id : -1;
    ids_base = n;
  };
  // operands of tile t, the wave's n-th: keys in rows 4 g' + i of operand e are slots 8 g' + 4 e + i
  pu32x4 kf[2][NK], vf[NO];
  int id0, id1;
  auto page_ids = [&](int n) {
    if (n - ids_base >= 32) load_ids(n);
    id0 = __builtin_amdgcn_readlane(ids, 2 * (n - ids_base));
    id1 = __builtin_amdgcn_readlane(ids, 2 * (n - ids_base) + 1);
  };
  auto load_k = [&](int t) {
    const int j = (tile_slot(t) & in_page) + 8 * (col >> 2) + (col & 3);   // slot of the lane's row in the pages of the tile
    const int64_t b0 = ((int64_t)max(id0, 0) * p.Hk + kvh) << p.page_shift, b1 = ((int64_t)max(id1, 0) * p.Hk + kvh) << p.page_shift;
    const uint16_t* kp = p.k + ((col < 8 ? b0 : b1) + (j & in_page)) * DH + g * 8;
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) kf[e][kk] = *(const pu32x4*)(kp + e * 4 * DH + kk * 32);
  };
  auto load_v = [&](int t) {
    const int j = (tile_slot(t) & in_page) + 8 * g;
    const int64_t b0 = ((int64_t)max(id0, 0) * p.Hk + kvh) * DH, b1 = ((int64_t)max(id1, 0) * p.Hk + kvh) * DH;
    const uint16_t* vp = p.v + (((g < 2 ? b0 : b1) + col) << p.page_shift) + (j & in_page);
#pragma unroll
    for (int c = 0; c < NO; ++c) vf[c] = *(const pu32x4*)(vp + ((16 * c) << p.page_shift));
  };
  if (t0 < t_end) {
    load_ids(0);
    page_ids(0);
    load_k(t0);
    // K before V here as in the loop, or every wait for K would wait for V as well
    __builtin_amdgcn_sched_barrier(0);
    load_v(t0);
  }
  int n = 0;
  for (int t = t0; t < t_end; t += kDecWaves, ++n) {
    const int j0 = tile_slot(t);
    const bool okv = (g < 2 ? id0 : id1) >= 0;
    const bool full = id0 >= 0 && id1 >= 0 && j0 + 31 <= st.last && (a.window == 0 || j0 > st.last - a.window);
    const bool more = t + kDecWaves < t_end;
    pf32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
    for (int kk = 0; kk < NK; ++kk)
#pragma unroll
      for (int e = 0; e < 2; ++e) s[e] = T::mfma16(kf[e][kk], qf[kk], s[e]);
    if (more) {
      page_ids(n + 1);
      load_k(t + kDecWaves);   // in flight over the softmax and the second product
    }
    float x[8], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = s[u >> 2][u & 3];
    if (full) {
      any = 1;
    } else {
      unsigned seen = 0;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int j = j0 + 8 * g + u;
        const bool in = okv && j <= st.last && (a.window == 0 || j > st.last - a.window || j < a.n_sinks);
        x[u] = in ? x[u] : -INFINITY;
        seen |= (unsigned)in << u;
      }
      any |= seen != 0;
      pu32x4 keep;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        keep[w] = ((seen >> (2 * w)) & 1 ? 0xffffu : 0u) | ((seen >> (2 * w + 1)) & 1 ? 0xffff0000u : 0u);
#pragma unroll
      for (int c = 0; c < NO; ++c) vf[c] &= keep;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) top = fmaxf(top, x[u]);
    top *= a.scale_log2e;   // positive
    if (__any(top > m + kPagedLazy)) {
      const float mn = fmaxf(m, rows_max(top)), nb = mn == -INFINITY ? 0.f : mn;
      const float f = __builtin_amdgcn_exp2f(m - nb);
      m = mn;
      mb = T::kShift - nb;
      l *= f;
#pragma unroll
      for (int c = 0; c < NO; ++c) acc[c] *= f;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      x[u] = __builtin_amdgcn_exp2f(fmaf(x[u], a.scale_log2e, mb));
      l += x[u];
    }
    const pu32x4 pf = {pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7])};
#pragma unroll
    for (int c = 0; c < NO; ++c) acc[c] = T::mfma16(vf[c], pf, acc[c]);
    if (more) load_v(t + kDecWaves);
  }

  // Join the waves: every wave scales its output to the common maximum; the
  // second half of them adds theirs to the first half's through LDS, then all
  // threads add up what is left.
  constexpr int kHalf = kDecWaves / 2;
  const int row = DH + 4;   // floats between queries: four apart in banks
  float* ml = lds + kHalf * qs * row;
  l = rows_sum(l);
  any = __any(any);
  if (lane < 16) *(pf32x4*)(ml + (wv * 16 + col) * 4) = pf32x4{m, l, any ? 1.f : 0.f, 0.f};
  __syncthreads();
  float mm = -INFINITY;
#pragma unroll
  for (int w = 0; w < kDecWaves; ++w) mm = fmaxf(mm, ml[(w * 16 + col) * 4]);
  const float mine = __builtin_amdgcn_exp2f(m - (mm == -INFINITY ? 0.f : mm));
#pragma unroll
  for (int c = 0; c < NO; ++c) acc[c] *= mine;
  float* o_row = lds + ((wv % kHalf) * qs + min(col, qs - 1)) * row + 4 * g;
  if (wv >= kHalf && col < qs)
#pragma unroll
    for (int c = 0; c < NO; ++c) *(pf32x4*)(o_row + 16 * c) = acc[c];
  __syncthreads();
  if (wv < kHalf && col < qs)
#pragma unroll
    for (int c = 0; c < NO; ++c) *(pf32x4*)(o_row + 16 * c) = acc[c] + *(const pf32x4*)(o_row + 16 * c);
  __syncthreads();
  for (int i = threadIdx.x; i < qs * (DH / 4); i += kDecWaves * 64) {
    const int q = i / (DH / 4), d = i % (DH / 4) * 4;
    float top = -INFINITY, ll = 0.f, saw = 0.f;
#pragma unroll
    for (int w = 0; w < kDecWaves; ++w) top = fmaxf(top, ml[(w * 16 + q) * 4]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < kDecWaves; ++w) {
      const pf32x4 x = *(const pf32x4*)(ml + (w * 16 + q) * 4);
      ll += x[1] * __builtin_amdgcn_exp2f(x[0] - ref);
      saw += x[2];
    }
    pf32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kHalf; ++w) o += *(const pf32x4*)(lds + (w * qs + q) * row + d);
    if (n_chunks == 1) {
      const float inv = 1.f / ll;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = saw > 0.f ? o[k] * inv : 0.f;
      *(pu32x2*)(a.out + seq * a.out_stride + (h0 + q) * DH + d) = pu32x2{pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
    } else {
      float* to = part + ((int64_t)blockIdx.x * min(G, 16) + q) * row;
      *(pf32x4*)(to + 4 + d) = o;
      if (d == 0) *(pf32x4*)to = pf32x4{top, ll, saw, 0.f};
    }
  }
}

// Joins the chunks of a sequence: a wave per query head, a workgroup's waves
// taking chunks round robin.
constexpr int kJoinWaves = 4;
template <class T, int DH>
__global__ __launch_bounds__(kJoinWaves * 64) void k_paged_join(const PagedAttnArgs a, const float* part) {
  __shared__ float o_w[kJoinWaves][DH], ml_w[kJoinWaves][3];
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = p.H / p.Hk, blocks = (G + 15) >> 4, heads = p.Hk * blocks;
  const int seq = blockIdx.x / p.H, h = blockIdx.x % p.H;
  const int chunk = chunk_tiles(a, heads, lane);
  const int n = chunks_of(seq_tiles(a, seq).tiles, chunk);
  if (n == 1) return;   // the unit has written the output
  int before = 0;       // chunks of earlier sequences
  for (int s = lane; s < seq; s += 64) before += chunks_of(seq_tiles(a, s).tiles, chunk);
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) before += __shfl_xor(before, k);
  const int head = h / G * blocks + h % G / 16, q = h % G % 16, row = DH + 4, wide = min(G, 16);
  constexpr int D = DH / 64;   // dimensions of a lane
  float m = -INFINITY, l = 0.f, saw = 0.f, o[D] = {};
  for (int c = wv; c < n; c += kJoinWaves) {
    const float* from = part + (((int64_t)(before + c) * heads + head) * wide + q) * row;
    const pf32x4 x = *(const pf32x4*)from;
    const float mn = fmaxf(m, x[0]), ref = mn == -INFINITY ? 0.f : mn;
    const float f = __builtin_amdgcn_exp2f(m - ref), e = __builtin_amdgcn_exp2f(x[0] - ref);
    m = mn;
    l = l * f + x[1] * e;
    saw += x[2];
#pragma unroll
    for (int d = 0; d < D; ++d) o[d] = o[d] * f + from[4 + lane * D + d] * e;
  }
#pragma unroll
  for (int d = 0; d < D; ++d) o_w[wv][lane * D + d] = o[d];
  if (lane == 0) ml_w[wv][0] = m, ml_w[wv][1] = l, ml_w[wv][2] = saw;
  __syncthreads();
  if (threadIdx.x >= DH / 2) return;
  m = -INFINITY;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) m = fmaxf(m, ml_w[w][0]);
  const float ref = m == -INFINITY ? 0.f : m;
  float x = 0.f, y = 0.f;
  l = saw = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) {
    const float f = __builtin_amdgcn_exp2f(ml_w[w][0] - ref);
    l += ml_w[w][1] * f;
    saw += ml_w[w][2];
    x += o_w[w][2 * threadIdx.x] * f;
    y += o_w[w][2 * threadIdx.x + 1] * f;
  }
  const float inv = 1.f / l;
  x = saw > 0.f ? x * inv : 0.f;
  y = saw > 0.f ? y * inv : 0.f;
  *(uint32_t*)(a.out + seq * a.out_stride + h * DH + 2 * threadIdx.x) = pack2<T>(x, y);
}

PagedSplit paged_decode_split(const PagedPool& p, int window, int n_sinks) {
  const int G = p.H / p.Hk, heads = p.Hk * ((G + 15) / 16);
  PagedSplit s{};
  // the most tiles that a token can see
  const int64_t slots = (int64_t)p.max_pages << p.page_shift, all = (slots + 31) / 32;
  const int64_t seen = window ? ((int64_t)window + 31) / 32 + 1 + ((int64_t)n_sinks + 31) / 32 : all;
  s.split = (seen < all ? seen : all) > kDecMinChunk;
  s.units = (int64_t)p.n_seqs * heads + (s.split ? kDecTarget : 0);
  s.bytes = s.split ? (size_t)s.units * (G < 16 ? G : 16) * (p.dh + 4) * sizeof(float) : 0;
  return s;
}

template <class T, int DH>
static hipError_t decode(const PagedAttnArgs& a, const PagedSplit& sp, void* workspace, hipStream_t s) {
  const int G = a.pool.H / a.pool.Hk, wide = G < 16 ? G : 16;
  const size_t lds = (size_t)kDecWaves * (wide * (DH + 4) / 2 + 16 * 4) * sizeof(float);
  k_paged_decode<T, DH><<<(unsigned)sp.units, kDecWaves * 64, lds, s>>>(a, (float*)workspace);
  if (sp.split) k_paged_join<T, DH><<<a.pool.n_seqs * a.pool.H, kJoinWaves * 64, 0, s>>>(a, (const float*)workspace);
  return hipGetLastError();
}

hipError_t launch_paged_decode(const PagedAttnArgs& a, const PagedSplit& sp, int dtype, void* workspace, hipStream_t s) {
  if (dtype == GVC_BF16)
    return a.pool.dh == 64 ? decode<Bf16, 64>(a, sp, workspace, s) : decode<Bf16, 128>(a, sp, workspace, s);
  return a.pool.dh == 64 ? decode<Fp16, 64>(a, sp, workspace, s) : decode<Fp16, 128>(a, sp, workspace, s);
}

}  // namespace gvc
