// Units of work of the decode kernels: how a call whose lengths only the GPU
// knows is cut into chunks of about equal work, and how the chunks of a row are
// joined.  (k_paged_decode.hip says why; the figures here are of 16-bit pages unless
// another is named.  The quantised kernel, whose tiles have 64 slots and of whose workgroups
// with heads of 128 two fit a compute unit, takes the same numbers; they were not chosen for
// it.  One sequence, 32 heads on 8, which it splits from 961 slots on: 500 slots 8.0 us, 800
// 10.3, 1000 11.8, where 16-bit pages, split from 481 on, take 12.6, 11.8 and 12.5.)
#pragma once
#include "gvc_paged_rows.h"

namespace gvc {

// Waves of a workgroup; three fit a compute unit, and their starts, ends and
// loads overlap.  (One workgroup of 12 waves instead was slower at every size:
// 8.6 us against 7.3 for one sequence of 282 slots, 137 against 101 for 131072.)
constexpr int NW = 4;
// The least tiles of a chunk (a sequence of fewer than two is not split), and
// the units that splitting makes at most, besides one for each row tile.
constexpr int kDecMinChunk = 8, kDecTarget = 1024;
constexpr float kDecShare = 0.99999f / kDecTarget;   // (a rounded sum is no reason for longer chunks)
// Chunks that the last workgroup of a row tile joins, at most; a second
// launch spreads more of them over its workgroups, and costs 3 us of the host's time.
// (One sequence, 32 heads on 8, chunks of 16 tiles: two of them 12.4 us against 14.0, 8
// 14.7 against 14.7, 16 17 against 15; 16 sequences of 500 to 900 slots, 32 heads:
// 34.3 against 36.2.)
constexpr int kFuseChunks = 8;
static_assert(kFuseChunks <= 64, "a lane reads a chunk's flag");

// What rows see whose last slots lie in [least, most], in tiles of 2^TL slots:
// tiles [0, sinks) and from `win` on, `count` in all.
struct SlotTiles {
  int sinks, win, count;
};

template <int TL>
__device__ __forceinline__ SlotTiles slot_tiles(const PagedAttnArgs& a, int least, int most) {
  SlotTiles t;
  const int end = (most >> TL) + 1, win_lo = a.window ? max(least - a.window + 1, 0) >> TL : 0;
  t.sinks = a.window ? min((a.n_sinks + (1 << TL) - 1) >> TL, min(win_lo, end)) : 0;
  t.win = max(win_lo, t.sinks);
  t.count = most < 0 ? 0 : t.sinks + end - t.win;
  return t;
}

// The largest over each row of 16 lanes.
__device__ __forceinline__ int row16_max(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(0, v, kDppXor1, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, kDppXor2, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, kDppHalfMirror, 0xF, 0xF, false));
  return max(v, __builtin_amdgcn_update_dpp(0, v, kDppMirror, 0xF, 0xF, false));
}

// A unit of a call: chunk `index` of `count` of what tile `tile` of sequence
// seq's virtual rows sees (seq -1: past the last unit).
struct Unit {
  int seq, tile, index, count;
  SeqRows rows;
};

// Chunk lengths that are tried, one to a lane of 16: 8, 10, 12, 16, 20, 25, .. 203 and no splitting.
__device__ __forceinline__ int chunk_length(int k) {
  return k == 15 ? 1 << 27 : (int)(8.01f * __builtin_amdgcn_exp2f((float)k * (1.f / 3)));
}

// A call takes about as long as the compute unit with the most to do: its
// units, ceil(units / 256), by a chunk's tiles, the eight that a unit's start
// and end are worth, and as many for the join.  (Where a compute unit has more
// units than it holds, they come one by one as it gets room.)  Of the sixteen
// lengths this is the one for which that is least, and not so short that there
// are more units than kDecTarget and the row tiles.  It takes 0.7 us.  (Against
// chunks of at least 16 tiles that made 1024 units, 32 heads on 8: one sequence of 4096
// slots 13.0 us for 14.7, 12 of 2000 23.4 for 25.3, 64 of 700 38.4 for 45.8, 32 with a
// window of 1000, 28 heads on 4, 19.1 for 20.4; 64 of 500 29.7 for 28.5.)
// r, n: rows and tiles of sequence `lane`, or of the last one.
__device__ __forceinline__ int best_chunk(const PagedAttnArgs& a, int least, int lane, const SeqRows& r, int n) {
  const int S = a.pool.n_seqs, mine = chunk_length(lane & 15);
  const float part = 1.f / (float)mine, tiles = lane < S ? (float)((r.rows + 15) >> 4) : 0.f;
  float units = 0.f, total = 0.f, longest = 0.f;   // units, all tiles and the longest of every fourth sequence
  for (int i = 0; i < S; i += 32) {
#pragma unroll
    for (int k = 0; k < 32; k += 4) {
      const float t = __shfl(tiles, i + k + (lane >> 4)), m = (float)__shfl(n, i + k + (lane >> 4));
      units += t * (m < 2 * kDecMinChunk ? 1.f : fmaxf(ceilf(fmaf(m, part, -1e-4f)), 1.f));
      total = fmaf(t, m, total);
      longest = fmaxf(longest, t > 0.f ? m : 0.f);
    }
  }
  units = rows_sum(units) * (float)a.pool.Hk;
  total = rows_sum(total) * (float)a.pool.Hk;
  longest = rows_max(longest);
  const float share = total * kDecShare;
  if (__any(share > 200.f)) return share < 1 << 27 ? (int)ceilf(share) : 1 << 27;   // (the same in every lane)
  const bool allowed = (lane & 15) == 15 || (mine >= least && (float)mine >= share);
  const float rounds = units * (1.f / 256);
  const float cost = (rounds > 3.f ? rounds + 0.5f : ceilf(rounds)) * ((float)mine < longest ? (float)mine + 16.f : longest + 8.f);
  const int order = allowed ? -__float_as_int(cost) : -__float_as_int(INFINITY);   // of floats that are not negative
  const int most = row16_max(order);
  const uint64_t best = __ballot(order == most);
  return chunk_length((63 - __builtin_clzll(best)) & 15);
}

// More than 64 sequences: their chunks are long anyway, and looking for the best would cost more than
// it gives (200 sequences of 700 slots: 6 us of 110).
template <bool ROWS, int TL>
__device__ __forceinline__ int long_chunk(const PagedAttnArgs& a, int G, int least, int lane) {
  float total = 0.f;
#pragma unroll 8
  for (int s = lane; s < a.pool.n_seqs; s += 64) {
    const SeqRows r = seq_rows<ROWS>(a, s, G);
    total += (float)((r.rows + 15) >> 4) * (float)slot_tiles<TL>(a, r.last, r.last).count;
  }
  const float share = wave_sum(total) * (float)a.pool.Hk * kDecShare;
  return max(share < 1 << 27 ? (int)ceilf(share) : 1 << 27, max(least, 4 * kDecMinChunk));
}

// Units are numbered through the sequences in order, chunk by chunk; a
// sequence's row tiles all have the chunks that its last row would have.  Every
// wave finds its unit by itself.
// (4096 sequences of 100 slots, 32 heads on 8: 368 to 401 us where the table holds less
// than 512 slots each, so that none can be split; 985 to 1016 where it holds more and
// all lengths are gone through.)
template <bool ROWS, int TL>
__device__ __forceinline__ Unit find_unit(const PagedAttnArgs& a, int G, int number, bool split, int least, int lane) {
  const int S = a.pool.n_seqs;
  if (!ROWS && !split) {
    const int of = (G + 15) >> 4, seq = uniform(number / of);
    return {seq, uniform(number % of), 0, 1, seq_rows<false>(a, seq, G)};
  }
  SeqRows r = seq_rows<ROWS>(a, min(lane, S - 1), G);
  int chunk = chunk_length(15);
  if (S > 64 && split) {
    chunk = long_chunk<ROWS, TL>(a, G, least, lane);
  } else if (split) {
    const int n = slot_tiles<TL>(a, r.last, r.last).count;
    if (__any(n >= 2 * kDecMinChunk)) chunk = best_chunk(a, least, lane, r, n);
  }
  Unit u{-1, 0, 0, 0, {}};
  for (int s0 = 0; s0 < S; s0 += 64) {
    SeqRows next = r;   // lengths are on their way while these are counted (for lists of rows, two loads deep, 2% slower)
    if (!ROWS && s0 + 64 < S) next = seq_rows<ROWS>(a, min(s0 + 64 + lane, S - 1), G);
    const int n = slot_tiles<TL>(a, r.last, r.last).count;
    const int count = n < 2 * kDecMinChunk ? 1 : (n + chunk - 1) / chunk, tiles = (r.rows + 15) >> 4;
    const int units = s0 + lane < S ? count * tiles : 0;
    const int sum = wave_scan(units);
    const uint64_t past = __ballot(sum > number);
    if (past) {
      const int l = __builtin_ctzll(past);
      u.seq = s0 + l;
      u.count = __builtin_amdgcn_readlane(count, l);
      u.rows = {__builtin_amdgcn_readlane(r.begin, l), __builtin_amdgcn_readlane(r.rows, l),
                __builtin_amdgcn_readlane(r.last, l)};
      const int at = number - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(units, l));
      const int of = (u.rows.rows + 15) >> 4;
      u.index = at / of;
      u.tile = at % of;
      break;
    }
    number -= __builtin_amdgcn_readlane(sum, 63);
    r = ROWS ? seq_rows<ROWS>(a, min(s0 + 64 + lane, S - 1), G) : next;
  }
  return {uniform(u.seq), uniform(u.tile), uniform(u.index), uniform(u.count),
          {uniform(u.rows.begin), uniform(u.rows.rows), uniform(u.rows.last)}};
}

// A split call's workspace: for each unit and key-value head a flag; for each
// sequence the number of its first unit and its chunks; then [unit][key-value
// head][column][DH + 4] floats: maximum, sum, whether a slot was seen, nothing,
// output.  Columns: G, at most 16, for one row per sequence, else 16.
//
// A unit that is done sets its flag to the call's tag, and when that has come
// through reads the flags of its row tile's units: the last one finds them all
// set (two may, and write the same output), and clears them.  A tag is no other
// call's (see paged_tag), so what memory holds before does not matter, nor how
// often a captured call is replayed.  (A counter needs read-modify-writes of one
// address by all units, about 1 us each: 16 chunks took 13 us longer.)
__host__ __device__ __forceinline__ int64_t flag_bytes(int64_t units) { return (units * 8 + 15) / 16 * 16; }
__host__ __device__ __forceinline__ int64_t plan_bytes(int n_seqs) { return ((int64_t)n_seqs * 8 + 15) / 16 * 16; }
__host__ __device__ __forceinline__ int columns(bool rows, int G) { return rows || G > 16 ? 16 : G; }

// Partial results and flags pass between XCDs, whose L2 caches do not see each
// other's lines: they are written and read at agent scope.
__device__ __forceinline__ void put(uint64_t* to, uint64_t v) {
  __hip_atomic_store(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t get(const uint64_t* from) {
  return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put4(float* to, pf32x4 v) {
  const uint64_t* w = (const uint64_t*)&v;
  put((uint64_t*)to, w[0]);
  put((uint64_t*)to + 1, w[1]);
}
__device__ __forceinline__ pf32x4 get4(const float* from) {
  const uint64_t x = get((const uint64_t*)from), y = get((const uint64_t*)from + 1);
  return {__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32)), __uint_as_float((uint32_t)y),
          __uint_as_float((uint32_t)(y >> 32))};
}
// Waits until this wave's stores are where every XCD reads them.
__device__ __forceinline__ void stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// At least as large as every |acc|, NaN where one is NaN.
template <int N>
__device__ __forceinline__ float magnitude(const pf32x4 (&acc)[N]) {
  pf32x4 sum = {0, 0, 0, 0};
#pragma unroll
  for (int c = 0; c < N; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += fabsf(acc[c][i]);
  return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// The end of a unit whose waves hold running maxima m (powers of two), their lanes' shares l of the
// sums, whether a slot was seen, and outputs acc: lane (col, g) holds dimensions 16 c + 4 g .. + 3
// of column col.  lds: [NW / 2][columns][DH + 4], then [NW][16][4] floats.
template <class T, int DH, bool ROWS>
__device__ __forceinline__ void join_unit(const PagedAttnArgs& a, const Unit& unit, char* work, int64_t units, bool fused,
                                          pf32x4 (&acc)[DH / 16], float m, float l, bool any, float* lds) {
  constexpr int NO = DH / 16;
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
  const int G = p.H / p.Hk, kvh = blockIdx.x % p.Hk, number = blockIdx.x / p.Hk;
  const int v0 = unit.tile * 16, qs = min(unit.rows.rows - v0, 16);
  const char* plans = work + flag_bytes(units);
  auto row_of = [&](int q) { return ROWS ? unit.rows.begin + (v0 + q) / G : unit.rows.begin; };
  auto head_of = [&](int q) { return kvh * G + (ROWS ? (v0 + q) % G : v0 + q); };

  // Join the waves: every wave scales its output to the common maximum; the
  // second half of them adds theirs to the first half's through LDS, then all
  // threads add up what is left.
  constexpr int kHalf = NW / 2;
  const int row_len = DH + 4;   // floats between columns: four apart in banks
  float* ml = lds + kHalf * qs * row_len;
  l = rows_sum(l);
  const float saw_col = rows_max(any ? 1.f : 0.f);
  if (lane < 16) *(pf32x4*)(ml + (wv * 16 + col) * 4) = pf32x4{m, l, saw_col, 0.f};
  __syncthreads();
  float mm = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) mm = fmaxf(mm, ml[(w * 16 + col) * 4]);
  const float mine = __builtin_amdgcn_exp2f(m - (mm == -INFINITY ? 0.f : mm));
#pragma unroll
  for (int c = 0; c < NO; ++c) acc[c] *= mine;
  float* o_row = lds + ((wv % kHalf) * qs + min(col, qs - 1)) * row_len + 4 * g;
  if (wv >= kHalf && col < qs)
#pragma unroll
    for (int c = 0; c < NO; ++c) *(pf32x4*)(o_row + 16 * c) = acc[c];
  __syncthreads();
  if (wv < kHalf && col < qs)
#pragma unroll
    for (int c = 0; c < NO; ++c) *(pf32x4*)(o_row + 16 * c) = acc[c] + *(const pf32x4*)(o_row + 16 * c);
  __syncthreads();
  float* parts = (float*)(plans + plan_bytes(p.n_seqs));
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
    for (int w = 0; w < kHalf; ++w) o += *(const pf32x4*)(lds + (w * qs + q) * row_len + d);
    if (unit.count == 1) {
      const float inv = 1.f / ll;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = saw > 0.f ? o[k] * inv : 0.f;
      *(pu32x2*)(a.out + row_of(q) * a.out_stride + head_of(q) * DH + d) = pack_out<T>(o);
    } else {
      float* to = parts + ((int64_t)blockIdx.x * columns(ROWS, G) + q) * row_len;
      const pf32x4 stat = {top, ll, saw, 0.f};
      if (fused) {
        put4(to + 4 + d, o);
        if (d == 0) put4(to, stat);
      } else {
        *(pf32x4*)(to + 4 + d) = o;
        if (d == 0) *(pf32x4*)to = stat;
      }
    }
  }
  const int row_tiles = (unit.rows.rows + 15) >> 4, first = number - unit.index * row_tiles;   // the row tile's first unit
  // (rows' bounds that do not rise can name more units than there are: nobody joins such a tile)
  if (unit.count == 1 || !fused || first + (int64_t)(unit.count - 1) * row_tiles >= units / p.Hk) return;
  stores_done();
  __syncthreads();
  int* join = (int*)lds;
  if (wv == 0) {
    uint64_t* flags = (uint64_t*)work;
    if (lane == 0) {   // an exchange whose answer is there has been seen by every XCD
      const uint64_t held = __hip_atomic_exchange(flags + blockIdx.x, a.tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("" ::"v"(held));
    }
    stores_done();
    uint64_t* theirs = flags + (first + (int64_t)min(lane, unit.count - 1) * row_tiles) * p.Hk + kvh;   // chunk `lane`'s
    const bool all = __all(get(theirs) == a.tag);
    if (all) put(theirs, 0);
    if (lane == 0) *join = all;
  }
  __syncthreads();
  if (!*join) return;   // uniform
  const float* from = parts + ((int64_t)first * p.Hk + kvh) * columns(ROWS, G) * row_len;
  const int64_t step = (int64_t)row_tiles * p.Hk * columns(ROWS, G) * row_len;   // floats between chunks
  for (int i = threadIdx.x; i < qs * (DH / 4); i += NW * 64) {
    const int q = i / (DH / 4), d = i % (DH / 4) * 4;
    pf32x4 stat[kFuseChunks], x[kFuseChunks];   // all at once: a load takes 1 us
#pragma unroll
    for (int c = 0; c < kFuseChunks; ++c) {
      const float* part = from + min(c, unit.count - 1) * step + q * row_len;
      stat[c] = get4(part);
      x[c] = get4(part + 4 + d);
    }
    float top = -INFINITY, ll = 0.f, saw = 0.f;
    pf32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < kFuseChunks; ++c) top = fmaxf(top, stat[c][0]);   // the last chunk several times is no harm here
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int c = 0; c < kFuseChunks; ++c)
      if (c < unit.count) {
        const float f = __builtin_amdgcn_exp2f(stat[c][0] - ref);
        ll += stat[c][1] * f;
        saw += stat[c][2];
        o += x[c] * f;
      }
    const float inv = 1.f / ll;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = saw > 0.f ? o[k] * inv : 0.f;
    *(pu32x2*)(a.out + row_of(q) * a.out_stride + head_of(q) * DH + d) = pack_out<T>(o);
  }
}

// Joins the chunks of a sequence: a workgroup for each row and query head.
template <class T, int DH, int NT, bool ROWS>
__global__ __launch_bounds__(NT) void k_paged_join(const PagedAttnArgs a, const char* plans, int limit) {
  __shared__ JoinLds<DH, NT, kDecTarget + 2> lds;
  const PagedPool& p = a.pool;
  const int row = blockIdx.x / p.H, h = blockIdx.x % p.H, G = p.H / p.Hk;
  int seq = row, begin = row, rows = G;
  if (ROWS) {
    const SeqRows r = seq_of_row(a, row, G, threadIdx.x & 63, seq);
    if (seq < 0) return;   // a row of no sequence; uniform
    begin = r.begin;
    rows = r.rows;
  }
  const int2 plan = ((const int2*)plans)[seq];
  const int n = plan.y;
  if (n == 1) return;   // the unit has written the output; uniform
  const int v = (row - begin) * G + h % G, wide = columns(ROWS, G), tiles = (rows + 15) >> 4, first = plan.x + v / 16;
  // rows' bounds that do not rise can name more units than there are: such a sequence's plan may be missing
  if (n < 1 || n > kDecTarget + 2 || first < 0 || first + (int64_t)(n - 1) * tiles >= limit) return;
  const float* from = (const float*)(plans + plan_bytes(p.n_seqs)) + (((int64_t)first * p.Hk + h / G) * wide + v % 16) * (DH + 4);
  join_row<T, DH, NT>(from, (int64_t)tiles * p.Hk * wide * (DH + 4), n, lds, a.out + row * a.out_stride + h * DH);
}

template <int TL>
PagedSplit decode_split(const PagedPool& p, int n_rows, bool rows, int window, int n_sinks) {
  constexpr int64_t T = 1 << TL;
  const int64_t G = p.H / p.Hk;
  // the most tiles of rows, and the most tiles of slots that a row sees
  const int64_t partial = p.n_seqs < n_rows ? p.n_seqs : n_rows;
  const int64_t tiles = rows ? n_rows * G / 16 + partial : n_rows * ((G + 15) / 16);
  const int64_t slots = (int64_t)p.max_pages << p.page_shift, all = (slots + T - 1) / T;
  const int64_t seen = window ? (window + T - 1) / T + 1 + (n_sinks + T - 1) / T : all;
  PagedSplit s{};
  const int64_t most = seen < all ? seen : all;
  s.split = most >= 2 * kDecMinChunk;
  // The units join their results where a sequence has at most kFuseChunks chunks of the least length, or
  // where few longer ones are enough to fill the GPU.
  const int64_t least = (most + kFuseChunks - 1) / kFuseChunks;
  s.fused = least <= kDecMinChunk || (least <= 4 * kDecMinChunk && p.Hk * kFuseChunks >= 256);
  s.least = s.fused && least > kDecMinChunk ? (int)least : kDecMinChunk;
  s.units = tiles * p.Hk + (s.split ? kDecTarget + p.Hk : 0);
  s.bytes = s.split ? (size_t)(flag_bytes(s.units) + plan_bytes(p.n_seqs) + s.units * columns(rows, G) * (p.dh + 4) * (int64_t)sizeof(float)) : 0;
  return s;
}

// The second launch of a call whose units do not join their chunks themselves.
template <class T, int DH, bool ROWS>
static void launch_join(const PagedAttnArgs& a, const PagedSplit& sp, const char* work, hipStream_t s) {
  const char* plans = work + flag_bytes(sp.units);
  const unsigned rows = (unsigned)a.n_rows * a.pool.H;
  const int limit = (int)(sp.units / a.pool.Hk);
  if (rows <= 256) k_paged_join<T, DH, 1024, ROWS><<<rows, 1024, 0, s>>>(a, plans, limit);   // many chunks each
  else k_paged_join<T, DH, 256, ROWS><<<rows, 256, 0, s>>>(a, plans, limit);
}

}  // namespace gvc
