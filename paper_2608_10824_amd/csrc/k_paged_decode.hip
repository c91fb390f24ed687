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

// Waves of a workgroup; three fit a compute unit, and their starts, ends and
// loads overlap.  (One workgroup of 12 waves instead was slower at every size:
// 8.6 us against 7.3 for one sequence of 282 slots, 137 against 101 for 131072.)
constexpr int NW = 4;
// Units that the chunk length aims at (768 or 2048: 5% slower at one size or
// another), and the least tiles of a chunk: shorter sequences are not split.
constexpr int kDecTarget = 1024, kDecMinChunk = 16;

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

__device__ __forceinline__ int chunks_of(int tiles, int chunk) { return max((tiles + chunk - 1) / chunk, 1); }

// A unit of a call: chunk `index` of the `count` of sequence seq (-1: past the last one).
struct Unit {
  int seq, index, count, chunk;
  SeqTiles st;
};

// The chunk length is the sum of all tiles over the units aimed at, in whole
// rounds of the workgroup's waves (so no sequence has more chunks than that,
// and one); chunk numbers go through the sequences in
// order.  Every wave finds this out by itself.
__device__ __forceinline__ Unit find_unit(const PagedAttnArgs& a, int heads, int number, int lane) {
  const int S = a.pool.n_seqs;
  SeqTiles t = seq_tiles(a, min(lane, S - 1));
  int total = lane < S ? t.tiles : 0;   // at most 2^29: n_seqs * max_pages <= 2^27
  for (int s = lane + 64; s < S; s += 64) total += seq_tiles(a, s).tiles;
  total = __builtin_amdgcn_readlane(wave_scan(total), 63);
  const long long c = ((long long)total * heads + kDecTarget - 1) / kDecTarget;
  Unit u{-1, 0, 0, max((int)((c + NW - 1) / NW) * NW, kDecMinChunk), {}};
  for (int s0 = 0; s0 < S; s0 += 64) {
    if (s0) t = seq_tiles(a, min(s0 + lane, S - 1));
    const int n = s0 + lane < S ? chunks_of(t.tiles, u.chunk) : 0;
    const int sum = wave_scan(n);
    const uint64_t past = __ballot(sum > number);
    if (past) {
      const int l = __builtin_ctzll(past);
      u.seq = s0 + l;
      u.count = __builtin_amdgcn_readlane(n, l);
      u.index = number - (__builtin_amdgcn_readlane(sum, l) - u.count);
      u.st = {__builtin_amdgcn_readlane(t.last, l), __builtin_amdgcn_readlane(t.sink_tiles, l),
              __builtin_amdgcn_readlane(t.win_tile, l), __builtin_amdgcn_readlane(t.tiles, l)};
      break;
    }
    number -= __builtin_amdgcn_readlane(sum, 63);
  }
  u.seq = uniform(u.seq);
  u.index = uniform(u.index);
  u.count = uniform(u.count);
  u.st = {uniform(u.st.last), uniform(u.st.sink_tiles), uniform(u.st.win_tile), uniform(u.st.tiles)};
  return u;
}

// A split call's workspace: for each sequence the number of its first chunk
// and how many it has, then [chunk][key-value head, block of 16 queries][query]
// [DH + 4] floats: maximum, sum, whether a slot was seen, nothing, output.
__host__ __device__ __forceinline__ int64_t plan_bytes(int n_seqs) { return ((int64_t)n_seqs * 8 + 15) / 16 * 16; }

template <class T, int DH>
__global__ __launch_bounds__(NW * 64, 3) void k_paged_decode(const PagedAttnArgs a, char* work) {
  constexpr int NK = DH / 32, NO = DH / 16;
  extern __shared__ float lds[];   // [waves / 2][queries][DH + 4], then [waves][16][4]
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int G = p.H / p.Hk, blocks = (G + 15) >> 4, heads = p.Hk * blocks;
  const int head = blockIdx.x % heads, number = blockIdx.x / heads;
  const Unit unit = find_unit(a, heads, number, lane);
  if (unit.seq < 0) return;   // the grid is an upper bound; uniform over the workgroup
  const SeqTiles& st = unit.st;
  const int seq = unit.seq, t_end = min((unit.index + 1) * unit.chunk, st.tiles);
  if (work && head == 0 && unit.index == 0 && threadIdx.x == 0) ((int2*)work)[seq] = int2{number, unit.count};
  const int kvh = head / blocks, hb = head % blocks;
  const int qs = min(G - hb * 16, 16), h0 = kvh * G + hb * 16;
  const int* table = p.table + (int64_t)seq * p.max_pages;
  const int in_page = (1 << p.page_shift) - 1;
  auto tile_slot = [&](int t) { return 32 * (t < st.sink_tiles ? t : t - st.sink_tiles + st.win_tile); };

  const int lo = a.window ? st.last - a.window : -1;   // slots past lo are in the window

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

  // The wave's tiles go round the waves.  Page ids of 32 of them at a time, one
  // half tile (16 slots, always one page) to a lane.
  const int t0 = unit.index * unit.chunk + wv;
  int ids = -1, ids_base = 0;
  auto load_ids = [&](int n) {   // of the wave's tiles n .. n + 31
    const int t = t0 + (n + (lane >> 1)) * NW;
    const int j = tile_slot(min(t, max(t_end - 1, 0))) + 16 * (lane & 1);
    const int id = table[min(j >> p.page_shift, p.max_pages - 1)];
    ids = (unsigned)id < (unsigned)p.n_pages ? id : -1;
    ids_base = n;
  };
  // Operands of tile t, if there is one more; else the start of the pool, once
  // for all lanes: a branch around the loads would cost the waits for them
  // their order.  Keys in rows 4 g' + i of operand e are slots 8 g' + 4 e + i
  pu32x4 kf[2][NK], vf[NO];
  int id0, id1;
  auto page_ids = [&](int n) {
    if (n - ids_base >= 32) load_ids(n);
    id0 = __builtin_amdgcn_readlane(ids, 2 * (n - ids_base));
    id1 = __builtin_amdgcn_readlane(ids, 2 * (n - ids_base) + 1);
  };
  auto load_k = [&](int t, bool more) {
    const int j = (tile_slot(t) & in_page) + 8 * (col >> 2) + (col & 3);   // slot of the lane's row in the pages of the tile
    const int64_t b0 = ((int64_t)max(id0, 0) * p.Hk + kvh) << p.page_shift, b1 = ((int64_t)max(id1, 0) * p.Hk + kvh) << p.page_shift;
    const int64_t at = ((col < 8 ? b0 : b1) + (j & in_page)) * DH + g * 8;
    const uint16_t* kp = p.k + (more ? at : 0);
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) kf[e][kk] = *(const pu32x4*)(kp + e * 4 * DH + kk * 32);
  };
  auto load_v = [&](int t, bool more) {
    const int j = (tile_slot(t) & in_page) + 8 * g;
    const int64_t b0 = ((int64_t)max(id0, 0) * p.Hk + kvh) * DH, b1 = ((int64_t)max(id1, 0) * p.Hk + kvh) * DH;
    const int64_t at = (((g < 2 ? b0 : b1) + col) << p.page_shift) + (j & in_page);
    const uint16_t* vp = p.v + (more ? at : 0);
#pragma unroll
    for (int c = 0; c < NO; ++c) vf[c] = *(const pu32x4*)(vp + ((16 * c) << p.page_shift));
  };
  if (t0 < t_end) {
    load_ids(0);
    page_ids(0);
    load_k(t0, true);
    // K before V here as in the loop, or every wait for K there would wait for V as well
    __builtin_amdgcn_sched_barrier(0);
    load_v(t0, true);
  }
  // The next tile's K are loaded as soon as the scores are done, its V after the second product.
  for (int t = t0, n = 0; t < t_end; ++n) {
    const int j0 = tile_slot(t), next = t + NW;
    const bool more = next < t_end;
    const bool okv = (g < 2 ? id0 : id1) >= 0;
    const bool full = id0 >= 0 && id1 >= 0 && j0 + 31 <= st.last && j0 > lo;
    pf32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
    for (int kk = 0; kk < NK; ++kk)
#pragma unroll
      for (int e = 0; e < 2; ++e) s[e] = T::mfma16(kf[e][kk], qf[kk], s[e]);
    if (more) page_ids(n + 1);
    load_k(next, more);
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
        const bool in = okv & (j <= st.last) & ((j > lo) | (j < a.n_sinks));
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
    t = next;
    load_v(t, more);
  }

  // Join the waves: every wave scales its output to the common maximum; the
  // second half of them adds theirs to the first half's through LDS, then all
  // threads add up what is left.
  constexpr int kHalf = NW / 2;
  const int row = DH + 4;   // floats between queries: four apart in banks
  float* ml = lds + kHalf * qs * row;
  l = rows_sum(l);
  any = __any(any);
  if (lane < 16) *(pf32x4*)(ml + (wv * 16 + col) * 4) = pf32x4{m, l, any ? 1.f : 0.f, 0.f};
  __syncthreads();
  float mm = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) mm = fmaxf(mm, ml[(w * 16 + col) * 4]);
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
  for (int i = threadIdx.x; i < qs * (DH / 4); i += NW * 64) {
    const int q = i / (DH / 4), d = i % (DH / 4) * 4;
    float top = -INFINITY, ll = 0.f, saw = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, ml[(w * 16 + q) * 4]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const pf32x4 x = *(const pf32x4*)(ml + (w * 16 + q) * 4);
      ll += x[1] * __builtin_amdgcn_exp2f(x[0] - ref);
      saw += x[2];
    }
    pf32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kHalf; ++w) o += *(const pf32x4*)(lds + (w * qs + q) * row + d);
    if (unit.count == 1) {
      const float inv = 1.f / ll;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = saw > 0.f ? o[k] * inv : 0.f;
      *(pu32x2*)(a.out + seq * a.out_stride + (h0 + q) * DH + d) = pu32x2{pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
    } else {
      float* to = (float*)(work + plan_bytes(p.n_seqs)) + ((int64_t)blockIdx.x * min(G, 16) + q) * row;
      *(pf32x4*)(to + 4 + d) = o;
      if (d == 0) *(pf32x4*)to = pf32x4{top, ll, saw, 0.f};
    }
  }
}

// Joins the chunks of a sequence: a workgroup for each query head.  Weights of
// the chunks from their maxima, then groups of DH / 4 threads add up the
// weighted outputs of every n-th chunk, and the groups' sums are added in LDS.
template <class T, int DH, int NT>
__global__ __launch_bounds__(NT) void k_paged_join(const PagedAttnArgs a, const char* work) {
  constexpr int GT = DH / 4, NG = NT / GT;
  __shared__ float weight[kDecTarget + 1], sums[3][NT / 64];
  __shared__ pf32x4 part_o[NG][GT];
  const PagedPool& p = a.pool;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int seq = blockIdx.x / p.H, h = blockIdx.x % p.H;
  const int2 plan = ((const int2*)work)[seq];
  const int n = plan.y;
  if (n == 1) return;   // the unit has written the output; uniform
  const int G = p.H / p.Hk, blocks = (G + 15) >> 4, heads = p.Hk * blocks;
  const int head = h / G * blocks + h % G / 16, q = h % G % 16, wide = min(G, 16);
  const float* from = (const float*)(work + plan_bytes(p.n_seqs)) + (((int64_t)plan.x * heads + head) * wide + q) * (DH + 4);
  const int64_t step = (int64_t)heads * wide * (DH + 4);   // floats between chunks
  float m = -INFINITY;
  for (int c = tid; c < n; c += NT) {
    weight[c] = from[c * step];
    m = fmaxf(m, weight[c]);
  }
  m = fmaxf(m, __shfl_xor(m, 1));
  m = fmaxf(m, __shfl_xor(m, 2));
  m = fmaxf(m, __shfl_xor(m, 4));
  m = fmaxf(m, __shfl_xor(m, 8));
  m = rows_max(m);
  if (lane == 0) sums[0][wv] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) m = fmaxf(m, sums[0][w]);
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f, saw = 0.f;
  for (int c = tid; c < n; c += NT) {
    const float f = __builtin_amdgcn_exp2f(weight[c] - ref);
    weight[c] = f;
    l += from[c * step + 1] * f;
    saw += from[c * step + 2];
  }
#pragma unroll
  for (int k = 1; k < 16; k <<= 1) {
    l += __shfl_xor(l, k);
    saw += __shfl_xor(saw, k);
  }
  l = rows_sum(l);
  saw = rows_sum(saw);
  if (lane == 0) sums[1][wv] = l, sums[2][wv] = saw;
  __syncthreads();
  const int gr = tid / GT, d = tid % GT;
  pf32x4 o = {0, 0, 0, 0};
#pragma unroll 4
  for (int c = gr; c < n; c += NG) o += *(const pf32x4*)(from + c * step + 4 + 4 * d) * weight[c];
  part_o[gr][d] = o;
  __syncthreads();
  if (tid >= GT) return;
  o = part_o[0][d];
#pragma unroll
  for (int k = 1; k < NG; ++k) o += part_o[k][d];
  l = saw = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) l += sums[1][w], saw += sums[2][w];
  const float inv = 1.f / l;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = saw > 0.f ? o[k] * inv : 0.f;
  *(pu32x2*)(a.out + seq * a.out_stride + h * DH + 4 * d) = pu32x2{pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
}

PagedSplit paged_decode_split(const PagedPool& p, int window, int n_sinks) {
  const int G = p.H / p.Hk, heads = p.Hk * ((G + 15) / 16);
  // the most tiles that a token can see
  const int64_t slots = (int64_t)p.max_pages << p.page_shift, all = (slots + 31) / 32;
  const int64_t seen = window ? ((int64_t)window + 31) / 32 + 1 + ((int64_t)n_sinks + 31) / 32 : all;
  PagedSplit s{};
  s.split = (seen < all ? seen : all) > kDecMinChunk;
  s.units = (int64_t)p.n_seqs * heads + (s.split ? kDecTarget : 0);
  s.bytes = s.split ? (size_t)(plan_bytes(p.n_seqs) + s.units * (G < 16 ? G : 16) * (p.dh + 4) * (int64_t)sizeof(float)) : 0;
  return s;
}

template <class T, int DH>
static hipError_t decode(const PagedAttnArgs& a, const PagedSplit& sp, void* workspace, hipStream_t s) {
  const int G = a.pool.H / a.pool.Hk, wide = G < 16 ? G : 16;
  const size_t lds = (size_t)NW * (wide * (DH + 4) / 2 + 16 * 4) * sizeof(float);
  char* work = sp.split ? (char*)workspace : nullptr;
  k_paged_decode<T, DH><<<(unsigned)sp.units, NW * 64, lds, s>>>(a, work);
  if (sp.split) {
    const unsigned rows = a.pool.n_seqs * a.pool.H;
    if (rows <= 256) k_paged_join<T, DH, 1024><<<rows, 1024, 0, s>>>(a, work);   // many chunks each
    else k_paged_join<T, DH, 256><<<rows, 256, 0, s>>>(a, work);
  }
  return hipGetLastError();
}

hipError_t launch_paged_decode(const PagedAttnArgs& a, const PagedSplit& sp, int dtype, void* workspace, hipStream_t s) {
  if (dtype == GVC_BF16)
    return a.pool.dh == 64 ? decode<Bf16, 64>(a, sp, workspace, s) : decode<Bf16, 128>(a, sp, workspace, s);
  return a.pool.dh == 64 ? decode<Fp16, 64>(a, sp, workspace, s) : decode<Fp16, 128>(a, sp, workspace, s);
}

}  // namespace gvc
