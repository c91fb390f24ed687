// Attention over the quantised paged cache for one new token per sequence, and
// for calls of few rows.
//
// The work of k_paged_decode.hip on half the bytes: units of chunks, 16 virtual
// rows to a workgroup, an online softmax in each wave, joins as described there
// (gvc_paged_units.h).  HBM bounds it.  A tile is 64 slots, so it has the bytes of 32
// slots of 16 bits and the same loads are in flight.  Codes become 16-bit operands in
// registers (three conversions and merges to a pair of V, half of one to a pair of K: with
// scales of V on the probabilities instead, a third of these instructions, the same time):
//  * Sixteen bytes of a key are two operands of S^T = K Q^T: the lanes of a slot
//    take dimensions 16 g .. 16 g + 15 of each 64, and so do the queries.  A
//    lane's keys are of one slot, whose scale the conversion applies.
//  * Sixteen bytes of V (dim-major pages) are a dimension's values of sixteen
//    slots, two operands of O^T += V^T P^T.  Their scales differ from slot to slot: each
//    pair is converted twice, with either slot's scale, and a half taken of both.
// So the operands are what the cache's values are in 16 bits, rounded once; probabilities are rounded to 16 bits before the
// second product, as gvc_paged.h says (relative difference of outputs from 64 bits over the same codes: 0.0017 to 0.0021 in bf16,
// 0.0002 to 0.0003 in fp16; 32 bits rounded at the end 0.0016 to 0.0017 and 0.0002).
//
// Measured (128 to a head, pages not in the caches): one sequence of 282 slots, 32 heads, bf16, 7.4 us; of
// 200003, 32 heads on 8, 72.8 us and 4.7 for the join, 413 MB at 5.7 TB/s; 64 of 7 to
// 16000 slots, 64 heads on 8, fp16, 62 and 5.5 us, 4.5 TB/s (of equal length 5.0: a unit's
// start and end take 4 to 5 us, which two workgroups of a compute unit do not hide); 40 with a window of 1000,
// 28 heads on 4, 14.5 us.
//
// Two workgroups to a compute unit: the 187 to 196 registers of heads of 128 leave room for two, and in the 168 of three
// they spill (200003 slots 98 to 125 us for 78).  Both tiles' operands in flight at once instead
// of the next ones behind their use, 81 for 78; 2 or 8 waves to a workgroup 85 and 83.
//
// Lists of rows come here by the rule of 16-bit pages (paged_few_rows), else to the 128-row tiles.  Both ways over codes, heads of
// 128, 32 of them: at the rule's 2^22 row-head-slots or below, one sequence of 280 slots and 234 rows 11.1 us for the tiles' 18.5, four of
// 1000 and 32 rows each 15.5 for 26.8, one of 4000 and 32 rows 19.6 for 26.3; at twice that, one of 1000 and 262 rows 25.2 for 27.3, four of 280
// and 234 rows 30.0 for 16.3, one of 4000 and 65 rows 29.9 for 27.7; at four times, one of 1000 34.5 for 34.4, one of 4000 50.4 for 34.4.
#include "gvc_kernels.h"
#include "gvc_paged_units.h"
#include "gvc_quant.h"

namespace gvc {

constexpr int kTileLog = 6;   // slots of a tile

template <class T, int DH, bool ROWS>
__global__ __launch_bounds__(NW * 64, 2) void k_quant_decode(const PagedAttnArgs a, const QuantPages from, char* work,
                                                              int64_t units, bool fused, int least_chunk) {
  constexpr int NK = DH / 64, NO = DH / 16;
  extern __shared__ float lds[];   // [waves / 2][columns][DH + 4], then [waves][16][4]
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int G = p.H / p.Hk, kvh = blockIdx.x % p.Hk, number = blockIdx.x / p.Hk;
  const Unit unit = find_unit<ROWS, kTileLog>(a, G, number, work != nullptr, least_chunk, lane);
  if (unit.seq < 0) return;   // the grid is an upper bound; uniform over the workgroup
  const int seq = unit.seq, v0 = unit.tile * 16, qs = min(unit.rows.rows - v0, 16);
  if (work && !fused && kvh == 0 && unit.index == 0 && unit.tile == 0 && threadIdx.x == 0)
    ((int2*)(work + flag_bytes(units)))[seq] = int2{number, unit.count};
  auto row_of = [&](int q) { return ROWS ? unit.rows.begin + (v0 + q) / G : unit.rows.begin; };
  auto head_of = [&](int q) { return kvh * G + (ROWS ? (v0 + q) % G : v0 + q); };
  const int* table = p.table + (int64_t)seq * p.max_pages;
  const int in_page = (1 << p.page_shift) - 1;
  const int row = row_of(min(col, qs - 1));
  pu32x4 qf[2 * NK];   // operand 2 kk + i: dimensions 64 kk + 16 g + 8 i .. + 7
  auto load_q = [&]() {
    const uint16_t* q = a.q;
    asm volatile("" : "+s"(q));   // an address of its own: the second call loads, and keeps no registers until then
#pragma unroll
    for (int kk = 0; kk < 2 * NK; ++kk) {
      qf[kk] = *(const pu32x4*)(q + row * a.q_stride + head_of(min(col, qs - 1)) * DH + (kk >> 1) * 64 + g * 16 + (kk & 1) * 8);
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
  auto tile_slot = [&](int t) { return 64 * (t < st.sinks ? t : t - st.sinks + st.win); };

  pf32x4 acc[NO];
  float m = -INFINITY, l = 0.f;   // maximum (powers of two), this lane's share of the sum
  bool any = false;
  // The wave's tiles go round the waves.  Page ids of 16 of them at a time, a quarter
  // of a tile (16 slots, always one page) to a lane.
  int ids = -1, ids_base = 0, k_id = -1, v_id = -1;   // pages of the lane's keys and values
  auto load_ids = [&](int n) {   // of the wave's tiles n .. n + 15
    const int t = t0 + (n + (lane >> 2)) * NW;
    const int j = tile_slot(min(t, max(t_end - 1, 0))) + 16 * (lane & 3);
    const int page = table[min(j >> p.page_shift, p.max_pages - 1)];
    ids = (unsigned)page < (unsigned)p.n_pages ? page : -1;
    ids_base = n;
  };
  auto page_ids = [&](int n) {
    if (n - ids_base >= 16) load_ids(n);
    k_id = __shfl(ids, 4 * (n - ids_base) + (col >> 2));
    v_id = __shfl(ids, 4 * (n - ids_base) + g);
  };
  auto head_of_page = [&](int id) { return (int64_t)max(id, 0) * p.Hk + kvh; };
  // Operands of tile t, if there is one more; else the start of the pool, once
  // for all lanes: a branch around the loads would cost the waits for them
  // their order.  Keys in rows 4 g' + i of operand e are slots 16 g' + 4 e + i.
  pu32x4 kf[4][NK], vf[NO], ks, vs;
  auto load_k = [&](int t, bool more) {
    const int64_t head = head_of_page(k_id) << p.page_shift;
    const int j = (tile_slot(t) + 16 * (col >> 2)) & in_page;
    const uint8_t* kp = from.k + (more ? (head + j + (col & 3)) * DH + g * 16 : 0);
    ks = *(const pu32x4*)(from.k_scale + (more ? head + j : 0));
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) kf[e][kk] = *(const pu32x4*)(kp + e * 4 * DH + kk * 64);
  };
  auto load_v = [&](int t, bool more) {
    const int64_t head = head_of_page(v_id);
    const int j = (tile_slot(t) + 16 * g) & in_page;
    const uint8_t* vp = from.v + (more ? ((head * DH + col) << p.page_shift) + j : 0);
    vs = *(const pu32x4*)(from.v_scale + (more ? (head << p.page_shift) + j : 0));
#pragma unroll
    for (int c = 0; c < NO; ++c) vf[c] = *(const pu32x4*)(vp + ((16 * c) << p.page_shift));
  };
  auto scores = [&](pf32x4 (&s)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[e] = pf32x4{0, 0, 0, 0};
      const float scale = scale_of((ks[e] >> (8 * (col & 3))) & 0xff);
#pragma unroll
      for (int kk = 0; kk < 2 * NK; ++kk) {
        const uint32_t x = kf[e][kk >> 1][2 * (kk & 1)], y = kf[e][kk >> 1][2 * (kk & 1) + 1];
        s[e] = T::mfma16(pu32x4{decoded<T, false>(x, scale), decoded<T, true>(x, scale), decoded<T, false>(y, scale),
                                decoded<T, true>(y, scale)}, qf[kk], s[e]);
      }
    }
  };
  // acc += V^T P^T, of probabilities x of slots 16 g ..
  auto values = [&](const float (&x)[16]) {
    float scale[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) scale[u] = scale_of((vs[u >> 2] >> (8 * (u & 3))) & 0xff);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      pu32x4 pf;
#pragma unroll
      for (int i = 0; i < 4; ++i) pf[i] = pack2<T>(x[8 * h + 2 * i], x[8 * h + 2 * i + 1]);
#pragma unroll
      for (int c = 0; c < NO; ++c) {
        pu32x4 v;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t codes = vf[c][2 * h + w];
          const float* f = scale + 8 * h + 4 * w;
          v[2 * w] = (decoded<T, false>(codes, f[0]) & 0xffffu) | (decoded<T, false>(codes, f[1]) & 0xffff0000u);
          v[2 * w + 1] = (decoded<T, true>(codes, f[2]) & 0xffffu) | (decoded<T, true>(codes, f[3]) & 0xffff0000u);
        }
        acc[c] = T::mfma16(v, pf, acc[c]);
      }
    }
  };
  // codes and scales of slots whose bits are not set become zero
  auto keep_only = [&](uint32_t bits) {
    pu32x4 keep;
#pragma unroll
    for (int w = 0; w < 4; ++w) keep[w] = ((((bits >> (4 * w)) & 15) * 0x204081u) & 0x1010101u) * 0xffu;
    vs &= keep;
#pragma unroll
    for (int c = 0; c < NO; ++c) vf[c] &= keep;
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
    const bool okv = v_id >= 0;
    const bool full = __all(okv) && j0 + 63 <= hi_all && j0 > lo_all;
    pf32x4 s[4];
    scores(s);
    if (more) page_ids(n + 1);
    load_k(next, more);
    float x[16], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 16; ++u) x[u] = s[u >> 2][u & 3];
    if (full) {
      any = true;
    } else {
      const int j = j0 + 16 * g;
      const unsigned sinks = first16(a.n_sinks - j), page = okv ? ~0u : 0u;
      const unsigned seen = first16(last + 1 - j) & (~first16(lo + 1 - j) | sinks) & page;
      // one token: all rows see the same
      const unsigned some = ROWS ? first16(hi_some + 1 - j) & (~first16(lo_some + 1 - j) | sinks) & page : seen;
#pragma unroll
      for (int u = 0; u < 16; ++u) x[u] = seen_score(seen, u, x[u]);
      any |= seen != 0;
      keep_only(some);
    }
#pragma unroll
    for (int u = 0; u < 16; ++u) top = fmaxf(top, x[u]);
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
    for (int u = 0; u < 16; ++u) {
      x[u] = __builtin_amdgcn_exp2f(fmaf(x[u], a.scale_log2e, shift));
      sum += x[u];
    }
    l += sum;
    values(x);
    t = next;
    load_v(t, more);
  }
  // Where a sum is not finite, or too large to be joined with others (kPagedLarge),
  // the wave does its tiles again, slowly, with the true maximum and the spare bits.
  // In lists of rows a slot that only some rows of the tile see is then added to those
  // alone, by its unrounded probability, so that NaN and infinities in its values
  // stay with them; with one token all rows see the same.
  if (ROWS || T::kOverflows) {
    if (__builtin_expect(__any((col < qs) & !(magnitude(acc) < kPagedLarge)), 0)) {
      const float spare = (float)spare_bits(t_end - t0, kTileLog);
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
        pf32x4 s[4];
        scores(s);
        float x[16], top = -INFINITY;
        unsigned seen = 0;
#pragma unroll
        for (int u = 0; u < 16; ++u) {
          const int j = j0 + 16 * g + u;
          const bool in = (v_id >= 0) & (j <= last) & ((j > lo) | (j < a.n_sinks));
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
        for (int u = 0; u < 16; ++u) {
          x[u] = __builtin_amdgcn_exp2f(fmaf(x[u], a.scale_log2e, shift));
          l += x[u];
        }
        if constexpr (!ROWS) {
          load_v(t, true);
          keep_only(seen);
          values(x);
        } else {
#pragma unroll 1
          for (int o = 0; o < 4; ++o) {   // the slots of lane group o
            const unsigned bits = (unsigned)__shfl((int)seen, 16 * o + col);
            const int64_t head = head_of_page(__builtin_amdgcn_readlane(ids, 4 * (n - ids_base) + o));
            const int off = (j0 + 16 * o) & in_page;
            const uint8_t* vp = from.v + ((head * DH + 4 * g) << p.page_shift) + off;
            const uint8_t* sp = from.v_scale + (head << p.page_shift) + off;
#pragma unroll
            for (int u = 0; u < 16; ++u) {
              const float pr = __shfl(x[u], 16 * o + col), scale = scale_of(sp[u]);
              if ((bits >> u) & 1)
#pragma unroll
                for (int c = 0; c < NO; ++c)
#pragma unroll
                  for (int i = 0; i < 4; ++i)
                    acc[c][i] = fmaf(pr, T::up((uint16_t)decoded<T, false>(vp[((16 * c + i) << p.page_shift) + u], scale)),
                                     acc[c][i]);
            }
          }
        }
      }
      m += spare;
    }
  }
  join_unit<T, DH, ROWS>(a, unit, work, units, fused, acc, m, l, any, lds);
}

PagedSplit quant_decode_split(const PagedPool& p, int n_rows, bool rows, int window, int n_sinks) {
  return decode_split<kTileLog>(p, n_rows, rows, window, n_sinks);
}

template <class T, int DH, bool ROWS>
static hipError_t decode(const PagedAttnArgs& a, const QuantPages& from, const PagedSplit& sp, void* workspace, hipStream_t s) {
  const size_t lds = (size_t)NW * (columns(ROWS, a.pool.H / a.pool.Hk) * (DH + 4) / 2 + 16 * 4) * sizeof(float);
  char* work = sp.split ? (char*)workspace : nullptr;
  k_quant_decode<T, DH, ROWS><<<(unsigned)sp.units, NW * 64, lds, s>>>(a, from, work, sp.units, sp.fused, sp.least);
  if (sp.split && !sp.fused) launch_join<T, DH, ROWS>(a, sp, work, s);
  return hipGetLastError();
}

template <class T, int DH>
static hipError_t decode_or_rows(const PagedAttnArgs& a, const QuantPages& from, const PagedSplit& sp, void* workspace,
                                 hipStream_t s) {
  return a.row_begin ? decode<T, DH, true>(a, from, sp, workspace, s) : decode<T, DH, false>(a, from, sp, workspace, s);
}

hipError_t launch_quant_decode(const PagedAttnArgs& a, const QuantPages& from, const PagedSplit& sp, int dtype,
                               void* workspace, hipStream_t s) {
  if (dtype == GVC_BF16)
    return a.pool.dh == 64 ? decode_or_rows<Bf16, 64>(a, from, sp, workspace, s)
                           : decode_or_rows<Bf16, 128>(a, from, sp, workspace, s);
  return a.pool.dh == 64 ? decode_or_rows<Fp16, 64>(a, from, sp, workspace, s)
                         : decode_or_rows<Fp16, 128>(a, from, sp, workspace, s);
}

}  // namespace gvc
