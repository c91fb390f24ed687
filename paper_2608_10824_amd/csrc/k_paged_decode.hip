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
#include "gvc_paged_units.h"

namespace gvc {

constexpr int kTileLog = 5;   // slots of a tile

template <class T, int DH, bool ROWS>
__global__ __launch_bounds__(NW * 64, 3) void k_paged_decode(const PagedAttnArgs a, char* work, int64_t units, bool fused,
                                                              int least_chunk) {
  constexpr int NK = DH / 32, NO = DH / 16;
  extern __shared__ float lds[];   // [waves / 2][columns][DH + 4], then [waves][16][4]
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int G = p.H / p.Hk, kvh = blockIdx.x % p.Hk, number = blockIdx.x / p.Hk;
  const Unit unit = find_unit<ROWS, kTileLog>(a, G, number, work != nullptr, least_chunk, lane);
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
  const SlotTiles st = slot_tiles<kTileLog>(a, least, hi_some);
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

  join_unit<T, DH, ROWS>(a, unit, work, units, fused, acc, m, l, any, lds);
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
  return decode_split<kTileLog>(p, n_rows, rows, window, n_sinks);
}

template <class T, int DH, bool ROWS>
static hipError_t decode(const PagedAttnArgs& a, const PagedSplit& sp, void* workspace, hipStream_t s) {
  const size_t lds = (size_t)NW * (columns(ROWS, a.pool.H / a.pool.Hk) * (DH + 4) / 2 + 16 * 4) * sizeof(float);
  char* work = sp.split ? (char*)workspace : nullptr;
  k_paged_decode<T, DH, ROWS><<<(unsigned)sp.units, NW * 64, lds, s>>>(a, work, sp.units, sp.fused, sp.least);
  if (sp.split && !sp.fused) launch_join<T, DH, ROWS>(a, sp, work, s);
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
