// Attention of lists of rows over the quantised paged cache.
//
// The tiles, products and softmax of k_paged_prefill.hip: 128 virtual rows to a
// workgroup, 64 slots at a time in LDS, S^T = K Q^T and O^T += V^T P^T on 32x32x16
// MFMA.  LDS holds the values in 16 bits.  Each wave brings 16 slots of a tile: the codes of the
// next tile are loaded into registers before the products of this one, and
// converted and written into the other stage behind them, so a code is converted once
// for 128 rows and one barrier to a tile is enough.  A key's codes are converted with their slot's
// scale.  A dimension of V has a byte for each of the wave's 16 slots, whose scales are
// the same in all lanes (scalar registers): a pair is converted twice, with either slot's scale, and a
// half taken of both.  What no row sees is made zero on the way.
//
// Measured: 6000 rows behind 3000 slots, 32 heads of 128 on 8, bf16, 613 to 625 us, 945 to 962 TFLOP/s of the
// products that rows see; heads of 64 368 us, 802 TFLOP/s; 16 chunks with a window of 600, heads of 64, fp16, 33 us.
// The softmax and the products take turns as in the 16-bit kernel (matrix cores busy 42%, vector units 50% of the time); the
// conversions add a quarter to the vector instructions, and their way through LDS from registers takes as long
// as reading the operands (a write of 1 KiB 16 cycles for the read's 4).  Conversions beside the first product or between the two took
// the same time; 8 waves, which share them among 256 rows, 0 to 4% less for long lists and up to 50% more for shorter ones.
#include "gvc_paged_tiles.h"
#include "gvc_quant.h"
#include "gvc_sync.h"

namespace gvc {

// Kinds of instructions for sched_group_barrier.
constexpr int kMfma = 0x8, kDsRead = 0x100;

template <class T, int DH>
__global__ __launch_bounds__(kPreWaves * 64, 2) void k_quant_prefill(const PagedAttnArgs a, const QuantPages from,
                                                                     float* work, int parts) {
  constexpr int NK = DH / 16, ND = DH / 32;
  constexpr int CR = DH / 8;               // 16-byte chunks of a key's row in LDS
  constexpr int CL = DH / 16;              // of its codes
  constexpr int KR = kPreKeys / kPreWaves; // slots of a tile that a wave brings
  constexpr int KI = KR * CL / 64;         // its loads of K, and of V (16 bytes a lane)
  constexpr int kTile = kPreKeys * DH * 2; // bytes of K, and of V
  __shared__ __attribute__((aligned(16))) char lds[2][2][kTile];
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
  const int r32 = lane & 31, half = lane >> 5;
  const int G = p.H / p.Hk, kvh = blockIdx.x % p.Hk, part = blockIdx.x / p.Hk % parts;
  const RowTile rt = find_tile(a, G, blockIdx.x / p.Hk / parts, lane);
  if (rt.seq < 0) return;   // the grid is an upper bound; uniform over the workgroup
  const int v = rt.first + wv * 32 + r32;
  const bool live = v < rt.rows;
  const int row = rt.begin + min(v, rt.rows - 1) / G, h = kvh * G + min(v, rt.rows - 1) % G;
  const int slots = p.max_pages << p.page_shift;
  const int last = live ? min(max(a.row_last[row], -1), slots - 1) : -1;
  // What the wave's rows see: slots in (lo_some, hi_some] (or below the sinks)
  // some row, in (lo_all, hi_all] every row; dead rows do not count.
  int hi_some = last, lo_some = last < 0 ? slots : last, hi_all = live ? last : slots;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    hi_some = max(hi_some, __shfl_xor(hi_some, m));
    lo_some = min(lo_some, __shfl_xor(lo_some, m));
    hi_all = min(hi_all, __shfl_xor(hi_all, m));
  }
  int* shared_rows = (int*)lds;
  if (lane == 0) {
    shared_rows[wv] = hi_some;
    shared_rows[kPreWaves + wv] = lo_some;
  }
  __syncthreads();
  int hi = shared_rows[0], lo = shared_rows[kPreWaves];
#pragma unroll
  for (int w = 1; w < kPreWaves; ++w) {
    hi = max(hi, shared_rows[w]);
    lo = min(lo, shared_rows[kPreWaves + w]);
  }
  __syncthreads();
  hi = uniform(hi);
  lo = uniform(lo);
  const int lo_all = uniform(a.window ? hi_some - a.window : -1);
  hi_some = uniform(hi_some);
  hi_all = uniform(hi_all);
  lo_some = uniform(a.window ? lo_some - a.window : -1);
  const int lo_row = a.window ? last - a.window : -1, lo_wg = a.window ? lo - a.window : -1;
  // the workgroup's tiles: the sinks', then the window's; and this part of them
  const int end = (hi >> 6) + 1, win_lo = a.window ? max(lo - a.window + 1, 0) >> 6 : 0;
  const int sink_tiles = a.window ? min((a.n_sinks + 63) >> 6, min(win_lo, end)) : 0;
  const int win_tile = max(win_lo, sink_tiles);
  const int tiles = hi < 0 ? 0 : sink_tiles + end - win_tile;
  const int part_tiles = max((tiles + parts - 1) / parts, kPreMinTiles);
  const int n_parts = parts == 1 ? 1 : max((tiles + part_tiles - 1) / part_tiles, 1);
  if (part >= n_parts) return;
  const int t_begin = parts == 1 ? 0 : part * part_tiles, t_end = parts == 1 ? tiles : min(tiles, t_begin + part_tiles);

  const int* table = p.table + (int64_t)rt.seq * p.max_pages;
  const int in_page = (1 << p.page_shift) - 1;
  auto tile_slot = [&](int t) { return 64 * (t < sink_tiles ? t : t - sink_tiles + win_tile); };
  pu32x4 qf[NK];
#pragma unroll
  for (int kk = 0; kk < NK; ++kk) qf[kk] = *(const pu32x4*)(a.q + row * a.q_stride + h * DH + kk * 16 + half * 8);

  // LDS.  K: row n of a tile holds slot slot_of(n), the order of the operand's
  // rows (its own inverse); chunk c (16 bytes) of it is at c ^ turn(n).  V: operands of 32
  // dimensions by two chunks of eight slots, 1 KiB each; chunk c of dimension d is at c ^ (d / 8 & 1).  So
  // sixteen lanes that read an operand together hit different banks.
  auto slot_of = [](int n) { return (n & ~12) | ((n & 4) << 1) | ((n & 8) >> 1); };
  auto turn = [](int n) { return DH == 64 ? n >> 1 & 7 : n & 15; };
  // Codes of the wave's 16 slots (always of one page): load i of K has 16 dimensions of slot i * 64 / CL + lane / CL,
  // load i of V dimension 64 i + lane.
  auto load_ids = [&](int t) {   // the page of chunk lane % 8 of tile t (the last one's past it)
    const int j = tile_slot(min(t, t_end - 1)) + 8 * (lane & 7);
    return table[min(j >> p.page_shift, p.max_pages - 1)];
  };
  const int head_bytes = DH << p.page_shift;   // of a page
  pu32x4 k_in[KI], v_in[KI], v_scale;
  uint32_t k_scale[KI];
  auto load = [&](int t, int id) {
    const int page = __builtin_amdgcn_readlane(id, 2 * wv), off = (tile_slot(t) + 16 * wv) & in_page;
    const int64_t head = (int64_t)((unsigned)page < (unsigned)p.n_pages ? page : 0) * p.Hk + kvh;
    const auto k = __builtin_amdgcn_make_buffer_rsrc((char*)from.k + head * head_bytes, (short)0, head_bytes, 0x00020000);
    const auto v = __builtin_amdgcn_make_buffer_rsrc((char*)from.v + head * head_bytes, (short)0, head_bytes, 0x00020000);
    const int page_slots = in_page + 1;
    const auto ks = __builtin_amdgcn_make_buffer_rsrc((char*)from.k_scale + (head << p.page_shift), (short)0, page_slots, 0x00020000);
    const auto vs = __builtin_amdgcn_make_buffer_rsrc((char*)from.v_scale + (head << p.page_shift), (short)0, page_slots, 0x00020000);
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      k_in[i] = __builtin_amdgcn_raw_buffer_load_b128(k, lane * 16, off * DH + i * 1024, 0);
      k_scale[i] = __builtin_amdgcn_raw_buffer_load_b8(ks, lane / CL, off + i * (64 / CL), 0);
    }
#pragma unroll
    for (int i = 0; i < KI; ++i) v_in[i] = __builtin_amdgcn_raw_buffer_load_b128(v, lane << p.page_shift, off + (i << (p.page_shift + 6)), 0);
    v_scale = __builtin_amdgcn_raw_buffer_load_b128(vs, 0, off, 0);
  };
  // The loaded tile t, whose chunks' pages are `pages`, into its stage.
  auto store = [&](int t, unsigned pages) {
    char* to = lds[t & 1][0];
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const int n = slot_of(16 * wv + (i * 64 + lane) / CL), c = 2 * (lane & (CL - 1));
      const float f = scale_of(k_scale[i]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t x = k_in[i][2 * e], y = k_in[i][2 * e + 1];
        *(pu32x4*)(to + n * CR * 16 + (((c + e) ^ turn(n)) << 4)) =
            pu32x4{decoded<T, false>(x, f), decoded<T, true>(x, f), decoded<T, false>(y, f), decoded<T, true>(y, f)};
      }
    }
    // Values that no row of the workgroup sees become zeros: what memory holds
    // there, NaN perhaps, would pass a probability of zero (0 x NaN is NaN).
    const int j0 = tile_slot(t) + 16 * wv;
    uint32_t vs[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) vs[w] = (uint32_t)uniform((int)v_scale[w]);
    if (!((pages >> (2 * wv)) & 1) || j0 + 15 > hi || j0 <= lo_wg) {
      const uint32_t bits =
          ((pages >> (2 * wv)) & 1) ? first16(hi + 1 - j0) & (~first16(lo_wg + 1 - j0) | first16(a.n_sinks - j0)) : 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t keep = ((((bits >> (4 * w)) & 15) * 0x204081u) & 0x1010101u) * 0xffu;
        vs[w] &= keep;
#pragma unroll
        for (int i = 0; i < KI; ++i) v_in[i][w] &= keep;
      }
    }
    float f[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) f[u] = scale_of((vs[u >> 2] >> (8 * (u & 3))) & 0xff);
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const int d = i * 64 + lane;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        pu32x4 y;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t x = v_in[i][2 * e + w];
          const float* g = f + 8 * e + 4 * w;
          y[2 * w] = (decoded<T, false>(x, g[0]) & 0xffffu) | (decoded<T, false>(x, g[1]) & 0xffff0000u);
          y[2 * w + 1] = (decoded<T, true>(x, g[2]) & 0xffffu) | (decoded<T, true>(x, g[3]) & 0xffff0000u);
        }
        *(pu32x4*)(to + kTile + (wv * ND + (d >> 5)) * 1024 + (d & 31) * 32 + ((e ^ (d >> 3 & 1)) << 4)) = y;
      }
    }
  };
  // Where this lane's operands start in a stage: K's chunk 2 kk + half is at
  // k_at ^ (kk << 5), V's chunk half of slots 16 m.. and dimensions 32 d.. 1024 (ND m + d) behind v_at.
  const int k_at = r32 * (CR * 16) + ((half ^ turn(r32)) << 4);
  const int v_at = kTile + r32 * 32 + ((half ^ (r32 >> 3 & 1)) << 4);
  auto operand = [&](int at) { return *(const pu32x4*)((const char*)lds + at); };

  pf32x16 acc[ND];
  float m_run = -INFINITY, l_run = 0.f;   // maximum (powers of two), this lane's share of the sum
  bool any = false;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
  float shift = T::kShift;   // a score's exponent is score * scale + shift
  // The products and the softmax of tile t.
  auto attend = [&](int t, unsigned pages) {
    const int j0 = tile_slot(t);
    const bool full = pages == 0xff && j0 + 63 <= hi_all && j0 > lo_all;
    const int kt = (t & 1) * 2 * kTile + k_at, vt = (t & 1) * 2 * kTile + v_at;
    pf32x16 s[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[0][i] = s[1][i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < NK; ++kk)
#pragma unroll
      for (int e = 0; e < 2; ++e) s[e] = T::mfma32(operand((kt ^ (kk << 5)) + e * 32 * CR * 16), qf[kk], s[e]);
    // four operands ahead of the matrix cores
    __builtin_amdgcn_sched_group_barrier(kDsRead, 4, 0);
#pragma unroll
    for (int i = 0; i < 2 * NK; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
      if (i < 2 * NK - 4) __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
    }
    if (full) {
      any = true;
    } else {   // element 16 e + i is slot j0 + 32 e + 16 (i / 8) + 8 half + i % 8
      uint32_t seen = 0;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = 2 * g + half, j = j0 + 8 * c;
        seen |= (first8(last + 1 - j) & (~first8(lo_row + 1 - j) | first8(a.n_sinks - j)) & (0u - ((pages >> c) & 1)))
                << (8 * g);
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] = seen_score(seen, i, s[i >> 4][i & 15]);
      any |= seen != 0;
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = fmaxf(top, s[i >> 4][i & 15]);
    top *= a.scale_log2e;   // positive
    if (__any(top > m_run + kPagedLazy)) {
      const float mn = fmaxf(m_run, fmaxf(top, __shfl_xor(top, 32))), nb = mn == -INFINITY ? 0.f : mn;
      const float f = __builtin_amdgcn_exp2f(m_run - nb);
      m_run = mn;
      shift = T::kShift - nb;
      l_run *= f;
#pragma unroll
      for (int d = 0; d < ND; ++d) acc[d] *= f;
    }
    auto values = [&](int m, pu32x4 (&vf)[ND]) {
#pragma unroll
      for (int d = 0; d < ND; ++d) vf[d] = operand(vt + (m * ND + d) * 1024);
    };
    auto weights = [&](int m) {   // probabilities of slots 16 m + 8 half .. + 7, as the operand of the second product
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __builtin_amdgcn_exp2f(fmaf(s[m >> 1][8 * (m & 1) + i], a.scale_log2e, shift));
        l_run += x[i];
      }
      return pu32x4{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7])};
    };
    // the next weights are computed while the matrix cores are busy with the last ones
    pu32x4 vf[2][ND], pf = weights(0);
    values(0, vf[0]);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      pu32x4 next = pf;
      if (m < 3) values(m + 1, vf[(m + 1) & 1]);
      if (m < 3) next = weights(m + 1);
#pragma unroll
      for (int d = 0; d < ND; ++d) acc[d] = T::mfma32(vf[m & 1][d], pf, acc[d]);
      pf = next;
    }
  };
  auto exists = [&](int id) { return (unsigned)__ballot((unsigned)id < (unsigned)p.n_pages) & 0xff; };
  if (t_begin < t_end) {
    int id = load_ids(t_begin), next_id = load_ids(t_begin + 1);
    load(t_begin, id);
    unsigned pages = exists(id);
    store(t_begin, pages);
    for (int t = t_begin; t < t_end; ++t) {
      __builtin_amdgcn_s_waitcnt(0xC07F);   // this wave's part of tile t is in LDS
      lds_barrier();                        // everyone's, and everyone is done with tile t - 1
      const unsigned next_pages = exists(next_id);
      if (t + 1 < t_end) {
        load(t + 1, next_id);
        next_id = load_ids(t + 2);
      }
      const int j0 = tile_slot(t);
      if (!(j0 > hi_some || (j0 + 63 <= lo_some && j0 >= a.n_sinks))) attend(t, pages);   // else nothing for this wave
      pages = next_pages;
      if (t + 1 < t_end) store(t + 1, pages);
    }
  }
  // Where a sum is not finite, or too large to be joined with others (kPagedLarge),
  // the workgroup does its rows again, slowly, with the true maximum and the spare
  // bits: a slot that only some rows of a wave see is added to those alone, by its
  // unrounded probability, so that NaN and infinities in its values stay with them.
  bool bad = false;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) bad |= !(fabsf(acc[d][i]) < kPagedLarge);
  const int wave_bad = __any(bad && live);
  __syncthreads();   // LDS is free
  if (lane == 0) shared_rows[wv] = wave_bad;
  __syncthreads();
  bool again = false;
#pragma unroll
  for (int w = 0; w < kPreWaves; ++w) again |= shared_rows[w] != 0;
  __syncthreads();
  if (again) {
    const float spare = (float)spare_bits(t_end - t_begin, 6);
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll 1
    for (int t = t_begin; t < t_end; ++t) {
      const int id = load_ids(t);
      load(t, id);
      const unsigned pages = exists(id);
      store(t, pages);
      __syncthreads();
      const int j0 = tile_slot(t);
      const char* st = lds[t & 1][0];
      pf32x16 s[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[e][i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
          s[e] = T::mfma32(operand((((t & 1) * 2 * kTile + k_at) ^ (kk << 5)) + e * 32 * CR * 16), qf[kk], s[e]);
      }
      uint32_t seen = 0;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int c = 2 * (i >> 3) + half, j = j0 + 8 * c + (i & 7);
        const bool in = ((pages >> c) & 1) & (j <= last) & ((j > lo_row) | (j < a.n_sinks));
        s[i >> 4][i & 15] = in ? s[i >> 4][i & 15] : -INFINITY;
        seen |= (uint32_t)in << i;
        top = fmaxf(top, s[i >> 4][i & 15]);
      }
      const float mn = fmaxf(m_run, fmaxf(top, __shfl_xor(top, 32)) * a.scale_log2e), nb = mn == -INFINITY ? 0.f : mn;
      const float f = __builtin_amdgcn_exp2f(m_run - nb);
      m_run = mn;
      l_run *= f;
#pragma unroll
      for (int d = 0; d < ND; ++d) acc[d] *= f;
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = 8 * m + j;
          const float x = __builtin_amdgcn_exp2f(fmaf(s[i >> 4][i & 15], a.scale_log2e, T::kShift - nb - spare));
          l_run += x;
#pragma unroll 1
          for (int o = 0; o < 2; ++o) {   // slot 16 m + 8 o + j, of the lanes with half == o
            const float pr = __shfl(x, 32 * o + r32);
            if (!(((unsigned)__shfl((int)seen, 32 * o + r32) >> i) & 1)) continue;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
              for (int k = 0; k < 16; ++k) {
                const int dim = 32 * d + 8 * (k >> 2) + 4 * half + (k & 3);
                const char* vp = st + kTile + (m * ND + d) * 1024 + dim % 32 * 32 + ((o ^ (dim >> 3 & 1)) << 4) + 2 * j;
                acc[d][k] = fmaf(pr, T::up(*(const uint16_t*)vp), acc[d][k]);
              }
          }
        }
      __syncthreads();
    }
    m_run += spare;
  }

  const float l = l_run + __shfl_xor(l_run, 32);
  any |= __shfl_xor((int)any, 32) != 0;
  // [unit][virtual row][DH + 4]: maximum, sum, whether a slot was seen, the number of parts, output
  float* to = work + ((int64_t)blockIdx.x * kPreRows + wv * 32 + r32) * (DH + 4);
  if (parts > 1 && half == 0) *(pf32x4*)to = pf32x4{m_run, l, any ? 1.f : 0.f, (float)n_parts};
  if (n_parts == 1) {
    if (!live) return;
    uint16_t* o = a.out + row * a.out_stride + h * DH + 4 * half;
    const float inv = 1.f / l;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        pf32x4 y;
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = any ? acc[d][i + k] * inv : 0.f;
        *(pu32x2*)(o + 32 * d + 2 * i) = pack_out<T>(y);
      }
  } else {
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(pf32x4*)(to + 4 + 32 * d + 2 * i + 4 * half) = pf32x4{acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]};
  }
}

template <class T, int DH>
static hipError_t prefill(const PagedAttnArgs& a, const QuantPages& from, const PagedSplit& sp, void* workspace, hipStream_t s) {
  k_quant_prefill<T, DH><<<(unsigned)sp.units, kPreWaves * 64, 0, s>>>(a, from, (float*)workspace, sp.parts);
  if (sp.split) launch_join_tiles<T, DH>(a, sp, (const float*)workspace, s);
  return hipGetLastError();
}

hipError_t launch_quant_prefill(const PagedAttnArgs& a, const QuantPages& from, const PagedSplit& sp, int dtype,
                                void* workspace, hipStream_t s) {
  if (dtype == GVC_BF16)
    return a.pool.dh == 64 ? prefill<Bf16, 64>(a, from, sp, workspace, s) : prefill<Bf16, 128>(a, from, sp, workspace, s);
  return a.pool.dh == 64 ? prefill<Fp16, 64>(a, from, sp, workspace, s) : prefill<Fp16, 128>(a, from, sp, workspace, s);
}

}  // namespace gvc
