// Attention over the paged cache for one new token per sequence, and for calls
// of few rows.
//
// Such a call reads every visible key and value once and computes little with
// them (about one multiply-add per byte and query head), so HBM bounds it: the
// kernel has to keep enough loads in flight on every compute unit, whatever the
// mix of lengths.  The query heads that share a key-value head count as rows:
// virtual row v of a sequence is row v / G, head v % G of the group, and 16 of
// them are the columns of one MFMA tile.  A workgroup takes one unit: a chunk
// of the 32-slot tiles that such a tile of rows sees, for one key-value head.
// The chunk length follows from the lengths, which only the GPU knows: every
// wave looks for the one with which the compute units have the least to do (see
// best_chunk) and finds its unit, so ragged batches come out in pieces of
// about equal work, and a batch that fills the GPU by itself is not split at
// all.  Within a unit the waves take tiles round robin, each with its own
// online softmax, and are joined in LDS.  The chunks of a row tile are
// joined by the workgroup that is done last, in the order of the chunks, so a
// result does not depend on which one that is; where there may be more than
// kFuseChunks of them, by a second launch with a workgroup for each row.
//
// Measured (bf16, 128 to a head): one sequence of 282 slots, 32 heads, 7.2 us (a
// chain of launch, table, keys, values: 4.8 us for one slot); of 131072, 32 heads on
// 8, 102.6 us, 5.2 TB/s; 16 sequences of 500 to 900 slots, 32 heads, 32.5 to 33.8 us, 4.3 to
// 4.5 TB/s; 64 of 5 to 16384 slots, 64 heads on 8, fp16, 120 to 123 us, 4.5 TB/s.
//
// How a call is cut follows the table's width, which alone is known before the launch
// (these figures: tables as wide as the longest sequence needs).  In a table of 8192
// slots the 282 take 7.6 us, of 131072, with a second launch, 9.1 us.
//
// S^T = K Q^T and O^T += V^T P^T on 16x16x32 MFMA.  A lane's scores in S^T are
// of one query; the keys of a tile are ordered such that they are also the
// lane's operand of the second product, so probabilities stay in registers,
// and 16 bytes of V (dim-major pages) are one operand.  What no row of a tile sees
// is zeroed in V (0 x NaN is NaN).
#include "gvc_kernels.h"
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

// What rows see whose last slots lie in [least, most], in tiles of 32 slots:
// tiles [0, sinks) and from `win` on, `count` in all.
struct SlotTiles {
  int sinks, win, count;
};

__device__ __forceinline__ SlotTiles slot_tiles(const PagedAttnArgs& a, int least, int most) {
  SlotTiles t;
  const int end = (most >> 5) + 1, win_lo = a.window ? max(least - a.window + 1, 0) >> 5 : 0;
  t.sinks = a.window ? min((a.n_sinks + 31) >> 5, min(win_lo, end)) : 0;
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
template <bool ROWS>
__device__ __forceinline__ int long_chunk(const PagedAttnArgs& a, int G, int least, int lane) {
  float total = 0.f;
#pragma unroll 8
  for (int s = lane; s < a.pool.n_seqs; s += 64) {
    const SeqRows r = seq_rows<ROWS>(a, s, G);
    total += (float)((r.rows + 15) >> 4) * (float)slot_tiles(a, r.last, r.last).count;
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
template <bool ROWS>
__device__ __forceinline__ Unit find_unit(const PagedAttnArgs& a, int G, int number, bool split, int least, int lane) {
  const int S = a.pool.n_seqs;
  if (!ROWS && !split) {
    const int of = (G + 15) >> 4, seq = uniform(number / of);
    return {seq, uniform(number % of), 0, 1, seq_rows<false>(a, seq, G)};
  }
  SeqRows r = seq_rows<ROWS>(a, min(lane, S - 1), G);
  int chunk = chunk_length(15);
  if (S > 64 && split) {
    chunk = long_chunk<ROWS>(a, G, least, lane);
  } else if (split) {
    const int n = slot_tiles(a, r.last, r.last).count;
    if (__any(n >= 2 * kDecMinChunk)) chunk = best_chunk(a, least, lane, r, n);
  }
  Unit u{-1, 0, 0, 0, {}};
  for (int s0 = 0; s0 < S; s0 += 64) {
    SeqRows next = r;   // lengths are on their way while these are counted (for lists of rows, two loads deep, 2% slower)
    if (!ROWS && s0 + 64 < S) next = seq_rows<ROWS>(a, min(s0 + 64 + lane, S - 1), G);
    const int n = slot_tiles(a, r.last, r.last).count;
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

template <class T, int DH, bool ROWS>
__global__ __launch_bounds__(NW * 64, 3) void k_paged_decode(const PagedAttnArgs a, char* work, int64_t units, bool fused,
                                                              int least_chunk) {
  constexpr int NK = DH / 32, NO = DH / 16;
  extern __shared__ float lds[];   // [waves / 2][columns][DH + 4], then [waves][16][4]
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int G = p.H / p.Hk, kvh = blockIdx.x % p.Hk, number = blockIdx.x / p.Hk;
  const Unit unit = find_unit<ROWS>(a, G, number, work != nullptr, least_chunk, lane);
  if (unit.seq < 0) return;   // the grid is an upper bound; uniform over the workgroup
  const int seq = unit.seq, v0 = unit.tile * 16, qs = min(unit.rows.rows - v0, 16);
  char* plans = work + flag_bytes(units);
  if (work && !fused && kvh == 0 && unit.index == 0 && unit.tile == 0 && threadIdx.x == 0)
    ((int2*)plans)[seq] = int2{number, unit.count};
  auto row_of = [&](int q) { return ROWS ? unit.rows.begin + (v0 + q) / G : unit.rows.begin; };
  auto head_of = [&](int q) { return kvh * G + (ROWS ? (v0 + q) % G : v0 + q); };
  const int* table = p.table + (int64_t)seq * p.max_pages;
  const int in_page = (1 << p.page_shift) - 1;
  const int row = row_of(min(col, qs - 1));
  pu32x4 qf[NK];
  auto load_q = [&]() {
    const uint16_t* q = a.q;
    asm volatile("" : "+s"(q));   // an address of its own: the second call loads, and keeps no registers until then
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      qf[kk] = *(const pu32x4*)(q + row * a.q_stride + head_of(min(col, qs - 1)) * DH + g * 8 + kk * 32);
      if (col >= qs) qf[kk] = pu32x4{0, 0, 0, 0};
    }
  };
  load_q();
  // The last slot of the lane's row, and what the tile's rows see: slots in
  // (lo_some, hi_some] (or below the sinks) some row, in (lo_all, hi_all] every row.
  int last = unit.rows.last, hi_some = last, hi_all = last, least = last;
  if (ROWS) {
    const int slots = p.max_pages << p.page_shift;
    last = col < qs ? min(max(a.row_last[row], -1), slots - 1) : -1;
    hi_some = uniform(row16_max(last));
    hi_all = uniform(-row16_max(col < qs ? -last : -slots));
    least = uniform(-row16_max(last < 0 ? -slots : -last));
  }
  const int lo = a.window ? last - a.window : -1, lo_some = a.window ? least - a.window : -1;
  const int lo_all = a.window ? hi_some - a.window : -1;
  const SlotTiles st = slot_tiles(a, least, hi_some);
  const int chunk = ((st.count + unit.count - 1) / unit.count + NW - 1) / NW * NW;   // equal parts, in whole rounds
  const int t0 = unit.index * chunk + wv, t_end = min((unit.index + 1) * chunk, st.count);
  auto tile_slot = [&](int t) { return 32 * (t < st.sinks ? t : t - st.sinks + st.win); };

  pf32x4 acc[NO];
  float m = -INFINITY, l = 0.f;   // maximum (powers of two), this lane's share of the sum
  bool any = false;
  // The wave's tiles go round the waves.  Page ids of 32 of them at a time, one
  // half tile (16 slots, always one page) to a lane.
  int ids = -1, ids_base = 0, id0, id1;
  auto load_ids = [&](int n) {   // of the wave's tiles n .. n + 31
    const int t = t0 + (n + (lane >> 1)) * NW;
    const int j = tile_slot(min(t, max(t_end - 1, 0))) + 16 * (lane & 1);
    const int id = table[min(j >> p.page_shift, p.max_pages - 1)];
    ids = (unsigned)id < (unsigned)p.n_pages ? id : -1;
    ids_base = n;
  };
  auto page_ids = [&](int n) {
    if (n - ids_base >= 32) load_ids(n);
    id0 = __builtin_amdgcn_readlane(ids, 2 * (n - ids_base));
    id1 = __builtin_amdgcn_readlane(ids, 2 * (n - ids_base) + 1);
  };
  // Operands of tile t, if there is one more; else the start of the pool, once
  // for all lanes: a branch around the loads would cost the waits for them
  // their order.  Keys in rows 4 g' + i of operand e are slots 8 g' + 4 e + i.
  pu32x4 kf[2][NK], vf[NO];
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
#pragma unroll
  for (int c = 0; c < NO; ++c) acc[c] = pf32x4{0, 0, 0, 0};
  float shift = T::kShift;   // a score's exponent is score * scale + shift
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
    const bool full = id0 >= 0 && id1 >= 0 && j0 + 31 <= hi_all && j0 > lo_all;
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
    unsigned seen = 0xff;
    if (full) {
      any = true;
    } else {
      const int j = j0 + 8 * g;
      const unsigned sinks = first8(a.n_sinks - j), page = okv ? ~0u : 0u;
      seen = first8(last + 1 - j) & (~first8(lo + 1 - j) | sinks) & page;
      // one token: all rows see the same
      const unsigned some = ROWS ? first8(hi_some + 1 - j) & (~first8(lo_some + 1 - j) | sinks) & page : seen;
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = seen_score(seen, u, x[u]);
      any |= seen != 0;
      pu32x4 keep;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        keep[w] = ((some >> (2 * w)) & 1 ? 0xffffu : 0u) | ((some >> (2 * w + 1)) & 1 ? 0xffff0000u : 0u);
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
      shift = T::kShift - nb;
      l *= f;
#pragma unroll
      for (int c = 0; c < NO; ++c) acc[c] *= f;
    }
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      x[u] = __builtin_amdgcn_exp2f(fmaf(x[u], a.scale_log2e, shift));
      sum += x[u];
    }
    l += sum;
    const pu32x4 pf = {pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7])};
#pragma unroll
    for (int c = 0; c < NO; ++c) acc[c] = T::mfma16(vf[c], pf, acc[c]);
    t = next;
    load_v(t, more);
  }
  // Where a sum is not finite, or too large to be joined with others (kPagedLarge),
  // the wave does its tiles again, slowly, with the true maximum and the spare bits.
  // In lists of rows a slot that only some rows of the tile see is then added to those
  // alone, by its unrounded probability, so that NaN and infinities in its values
  // stay with them; with one token all rows see the same.  (The test takes 0.1 to 0.25 us
  // of a call; out of the way and with q loaded anew: registers that it would keep made
  // the wave wait for the last round's unused loads, 0.5 us.)
  if (ROWS || T::kOverflows) {
    if (__builtin_expect(__any((col < qs) & !(magnitude(acc) < kPagedLarge)), 0)) {
      const float spare = (float)spare_bits(t_end - t0, 5);
#pragma unroll
      for (int c = 0; c < NO; ++c) acc[c] = pf32x4{0, 0, 0, 0};
      m = -INFINITY;
      l = 0.f;
      load_q();
      load_ids(0);
#pragma unroll 1
      for (int t = t0, n = 0; t < t_end; t += NW, ++n) {
        const int j0 = tile_slot(t);
        page_ids(n);
        load_k(t, true);
        pf32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
#pragma unroll
          for (int e = 0; e < 2; ++e) s[e] = T::mfma16(kf[e][kk], qf[kk], s[e]);
        float x[8], top = -INFINITY;
        unsigned seen = 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int j = j0 + 8 * g + u;
          const bool in = ((g < 2 ? id0 : id1) >= 0) & (j <= last) & ((j > lo) | (j < a.n_sinks));
          x[u] = in ? s[u >> 2][u & 3] : -INFINITY;
          seen |= (unsigned)in << u;
          top = fmaxf(top, x[u]);
        }
        const float mn = fmaxf(m, rows_max(top * a.scale_log2e)), nb = mn == -INFINITY ? 0.f : mn;
        const float f = __builtin_amdgcn_exp2f(m - nb);
        m = mn;
        shift = T::kShift - nb - spare;
        l *= f;
#pragma unroll
        for (int c = 0; c < NO; ++c) acc[c] *= f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          x[u] = __builtin_amdgcn_exp2f(fmaf(x[u], a.scale_log2e, shift));
          l += x[u];
        }
        if constexpr (!ROWS) {
          load_v(t, true);
          pu32x4 keep;
#pragma unroll
          for (int w = 0; w < 4; ++w)
            keep[w] = ((seen >> (2 * w)) & 1 ? 0xffffu : 0u) | ((seen >> (2 * w + 1)) & 1 ? 0xffff0000u : 0u);
          const pu32x4 pf = {pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7])};
#pragma unroll
          for (int c = 0; c < NO; ++c) acc[c] = T::mfma16(vf[c] & keep, pf, acc[c]);
        } else {
#pragma unroll 1
          for (int o = 0; o < 4; ++o) {   // the slots of lane group o
            const unsigned bits = (unsigned)__shfl((int)seen, 16 * o + col);
            const int64_t page = o < 2 ? max(id0, 0) : max(id1, 0);
            const uint16_t* vp = p.v + (((page * p.Hk + kvh) * DH + 4 * g) << p.page_shift) + ((j0 + 8 * o) & in_page);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const float pr = __shfl(x[u], 16 * o + col);
              if ((bits >> u) & 1)
#pragma unroll
                for (int c = 0; c < NO; ++c)
#pragma unroll
                  for (int i = 0; i < 4; ++i) acc[c][i] = fmaf(pr, T::up(vp[((16 * c + i) << p.page_shift) + u]), acc[c][i]);
            }
          }
        }
      }
      m += spare;
    }
  }

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

// Lists of rows come here rather than to the 128-row tiles of the prefill
// kernel where there is little to do in all, for all that a table of this width lets
// them see (148 rows over 276 slots, 32 heads: 9.6 us, and 20 in the tiles, where they go
// once the table holds 886 slots; 276 rows over 276 slots, 32 heads: 13.1 us
// against 17.8; 300 over 300, 32 heads on 8: 13.8 against 17.1; 8 over 16000: 23.7
// against 28.7; on the other side of the bound 128 over 2000: 28.9 against 25.6, 16
// lists of 148 over 276, 32 heads: 77 against 37), or few sequences have one
// tile of rows each (2 rows of 32 heads on 8, 8 sequences of 8000 slots: 56 us
// against 65; 64 such sequences of 600 slots: the same).
bool paged_few_rows(const PagedPool& p, int n_rows, int window, int n_sinks) {
  const int64_t slots = (int64_t)p.max_pages << p.page_shift, seen = (int64_t)window + n_sinks + 64;
  const int64_t most = window && seen < slots ? seen : slots;
  if ((int64_t)n_rows * p.H * most <= 1 << 22) return true;
  return (int64_t)n_rows * (p.H / p.Hk) <= (int64_t)p.n_seqs * 16 && p.n_seqs * p.Hk <= 128;
}

PagedSplit paged_decode_split(const PagedPool& p, int n_rows, bool rows, int window, int n_sinks) {
  const int64_t G = p.H / p.Hk;
  // the most tiles of rows, and the most tiles of slots that a row sees
  const int64_t partial = p.n_seqs < n_rows ? p.n_seqs : n_rows;
  const int64_t tiles = rows ? n_rows * G / 16 + partial : n_rows * ((G + 15) / 16);
  const int64_t slots = (int64_t)p.max_pages << p.page_shift, all = (slots + 31) / 32;
  const int64_t seen = window ? ((int64_t)window + 31) / 32 + 1 + ((int64_t)n_sinks + 31) / 32 : all;
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

template <class T, int DH, bool ROWS>
static hipError_t decode(const PagedAttnArgs& a, const PagedSplit& sp, void* workspace, hipStream_t s) {
  const size_t lds = (size_t)NW * (columns(ROWS, a.pool.H / a.pool.Hk) * (DH + 4) / 2 + 16 * 4) * sizeof(float);
  char* work = sp.split ? (char*)workspace : nullptr;
  k_paged_decode<T, DH, ROWS><<<(unsigned)sp.units, NW * 64, lds, s>>>(a, work, sp.units, sp.fused, sp.least);
  if (sp.split && !sp.fused) {
    const char* plans = work + flag_bytes(sp.units);
    const unsigned rows = (unsigned)a.n_rows * a.pool.H;
    const int limit = (int)(sp.units / a.pool.Hk);
    if (rows <= 256) k_paged_join<T, DH, 1024, ROWS><<<rows, 1024, 0, s>>>(a, plans, limit);   // many chunks each
    else k_paged_join<T, DH, 256, ROWS><<<rows, 256, 0, s>>>(a, plans, limit);
  }
  return hipGetLastError();
}

template <class T, int DH>
static hipError_t decode_or_rows(const PagedAttnArgs& a, const PagedSplit& sp, void* workspace, hipStream_t s) {
  return a.row_begin ? decode<T, DH, true>(a, sp, workspace, s) : decode<T, DH, false>(a, sp, workspace, s);
}

hipError_t launch_paged_decode(const PagedAttnArgs& a, const PagedSplit& sp, int dtype, void* workspace, hipStream_t s) {
  if (dtype == GVC_BF16)
    return a.pool.dh == 64 ? decode_or_rows<Bf16, 64>(a, sp, workspace, s) : decode_or_rows<Bf16, 128>(a, sp, workspace, s);
  return a.pool.dh == 64 ? decode_or_rows<Fp16, 64>(a, sp, workspace, s) : decode_or_rows<Fp16, 128>(a, sp, workspace, s);
}

}  // namespace gvc
