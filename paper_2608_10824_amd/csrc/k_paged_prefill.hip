// Attention of lists of rows over the paged cache.
//
// The query heads that share a key-value head count as rows: virtual row v of
// a sequence is row v / G, head v % G of the group.  A workgroup takes 128 of
// them, 32 to a wave, and goes through the slots that some of them see in
// tiles of 64, which are copied once for its waves straight into LDS, one tile
// ahead.  Long lists are bound by the matrix cores and the softmax between the
// two products.  S^T = K Q^T and O^T += V^T P^T run on 32x32x16 MFMA: a lane's
// scores are of one query, and the keys of a tile are taken in an order in
// which they are also the lane's operand of the second product, so
// probabilities stay in registers and a row's maximum and sum need one
// exchange between two lanes.
//
// Tiles of late rows see the most slots and start first.  Neighbouring
// workgroups take different key-value heads, so an XCD's L2 holds the keys and
// values of few heads.  Few rows over many slots are split over the slots as
// well; a second launch joins the parts.
//
// The copies go by buffer loads: beside loads of the other kind into LDS the compiler
// waits for all LDS reads where it needs one (5% slower), and a page's address
// stays in scalar registers.
//
// Measured: 8192 causal rows, 32 heads of 128 on 8, bf16, 524 to 568 us by the box, 968 to 1048
// TFLOP/s of the products that rows see, 80 to 86% of a large matrix product's rate (matrix cores busy 52%,
// vector units 46% of the time: the softmax costs as much as the products, and
// the two take turns); heads of 64 307 us, 896 TFLOP/s; 4 prompts of 1000 rows 58 us.
#include "gvc_paged_rows.h"
#include "gvc_sync.h"

#define LPA(p) ((void __attribute__((address_space(3)))*)(p))

namespace gvc {

constexpr int kPreWaves = 4, kPreRows = 32 * kPreWaves, kPreKeys = 64;
constexpr int kPreUnits = 512;   // calls with fewer units split the slots, into about as many
constexpr int kPreMinTiles = 4;  // tiles of a part, at least
constexpr int kPreMaxParts = kPreUnits;

// Kinds of instructions for sched_group_barrier.
constexpr int kMfma = 0x8, kDsRead = 0x100;

// The tile of virtual rows that a workgroup takes.
struct RowTile {
  int seq, first, begin, rows;   // sequence (-1: none), the tile's first virtual row, the sequence's first row, its virtual rows
};

// Tile `number` of the call, counted from the last sequence's last rows.
__device__ __forceinline__ RowTile find_tile(const PagedAttnArgs& a, int G, int number, int lane) {
  RowTile t{-1, 0, 0, 0};
  for (int s1 = a.pool.n_seqs; s1 > 0; s1 -= 64) {
    const int s = s1 - 1 - lane;
    const SeqRows r = seq_rows<true>(a, max(s, 0), G);
    const int n = s >= 0 ? (r.rows + kPreRows - 1) / kPreRows : 0;
    const int sum = wave_scan(n);
    const uint64_t past = __ballot(sum > number);
    if (past) {
      const int l = __builtin_ctzll(past);
      t.seq = s1 - 1 - l;
      t.begin = __builtin_amdgcn_readlane(r.begin, l);
      t.rows = __builtin_amdgcn_readlane(r.rows, l);
      t.first = (__builtin_amdgcn_readlane(sum, l) - 1 - number) * kPreRows;
      break;
    }
    number -= __builtin_amdgcn_readlane(sum, 63);
  }
  return {uniform(t.seq), uniform(t.first), uniform(t.begin), uniform(t.rows)};
}

template <class T, int DH>
__global__ __launch_bounds__(kPreWaves * 64, DH == 64 ? 3 : 2) void k_paged_prefill(const PagedAttnArgs a, float* work, int parts) {
  constexpr int NK = DH / 16, ND = DH / 32;
  constexpr int CR = DH / 8;               // 16-byte chunks of a key's row
  constexpr int RI = 64 / CR;              // keys of one copy (1 KiB)
  constexpr int KR = kPreKeys / kPreWaves; // keys of a tile that a wave copies
  constexpr int KI = KR / RI;              // its copies of K, and of V
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

  // Copies, of the 16 slots (always of one page) that are the wave's in every
  // tile.  K: LDS row n of a tile holds slot slot_of(n), the order of the operand's
  // rows; chunk c (16 bytes) of it is at c ^ turn(n).  V: a copy is one operand, 32
  // dimensions of two chunks of eight slots; chunk c of dimension d is at c ^ (d / 8 & 1).  So
  // sixteen lanes that read an operand together hit different banks.
  auto slot_of = [](int n) { return (n & ~12) | ((n & 4) << 1) | ((n & 8) >> 1); };
  auto turn = [](int n) { return DH == 64 ? n >> 1 & 7 : n & 15; };
  uint32_t k_off[KI];             // bytes from the first slot's
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    const int n = i * RI + lane / CR;
    k_off[i] = slot_of(n) * DH * 2 + ((lane & (CR - 1)) ^ turn(n)) * 16;
  }
  const uint32_t v_off = ((lane >> 1) << (p.page_shift + 1)) + ((lane & 1) ^ (lane >> 4 & 1)) * 16;
  auto load_ids = [&](int t) {   // the page of chunk lane % 8 of tile t (the last one's past it)
    const int j = tile_slot(min(t, t_end - 1)) + 8 * (lane & 7);
    return table[min(j >> p.page_shift, p.max_pages - 1)];
  };
  const int head_bytes = (DH * 2) << p.page_shift;   // of a page
  auto copy = [&](int t, int id) {
    char* to = lds[t & 1][0] + wv * KI * 1024;
    const int page = __builtin_amdgcn_readlane(id, 2 * wv), off = (tile_slot(t) + 16 * wv) & in_page;
    const int64_t at = ((int64_t)((unsigned)page < (unsigned)p.n_pages ? page : 0) * p.Hk + kvh) * head_bytes;
    const auto k = __builtin_amdgcn_make_buffer_rsrc((char*)p.k + at, (short)0, head_bytes, 0x00020000);
    const auto v = __builtin_amdgcn_make_buffer_rsrc((char*)p.v + at, (short)0, head_bytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < KI; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(k, LPA(to + i * 1024), 16, (int)k_off[i], off * DH * 2, 0, 0);
#pragma unroll
    for (int i = 0; i < KI; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(v, LPA(to + kTile + i * 1024), 16, (int)v_off, (i << (p.page_shift + 6)) + off * 2, 0, 0);
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
  int next_id = 0;
  uint64_t ok = 0;
  if (t_begin < t_end) {
    const int id = load_ids(t_begin);
    next_id = load_ids(t_begin + 1);
    copy(t_begin, id);
    ok = __ballot((unsigned)id < (unsigned)p.n_pages);
  }
  for (int t = t_begin; t < t_end; ++t) {
    wait_vmcnt<0>();   // this wave's copies of tile t
    lds_barrier();     // everyone's, and everyone is done with tile t - 1
    uint64_t next_ok = 0;
    if (t + 1 < t_end) {
      copy(t + 1, next_id);
      next_ok = __ballot((unsigned)next_id < (unsigned)p.n_pages);
      next_id = load_ids(t + 2);
    }
    const int j0 = tile_slot(t);
    const unsigned pages = (unsigned)ok & 0xff;   // of the tile's chunks
    ok = next_ok;
    // Values that no row of the workgroup sees become zeros: what memory holds
    // there, NaN perhaps, would pass a probability of zero (0 x NaN is NaN).
    if (pages != 0xff || j0 + 63 > hi || j0 <= lo_wg) {
#pragma unroll
      for (int i = 0; i < DH * 8; i += kPreWaves * 64) {
        pu32x4* v = (pu32x4*)(lds[t & 1][1]) + i + threadIdx.x;
        const int c = 2 * ((i + threadIdx.x) / (64 * ND)) + ((threadIdx.x & 1) ^ (threadIdx.x >> 4 & 1)), j = j0 + 8 * c;
        uint32_t b = first8(hi + 1 - j) & (~first8(lo_wg + 1 - j) | first8(a.n_sinks - j)) & (0u - ((pages >> c) & 1));
        pu32x4 keep;
#pragma unroll
        for (int w = 0; w < 4; ++w, b >>= 2) keep[w] = (b & 1 ? 0xffffu : 0u) | (b & 2 ? 0xffff0000u : 0u);
        *v &= keep;
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);   // LDS only: the next tile's copies go on
      lds_barrier();
    }
    if (j0 > hi_some || (j0 + 63 <= lo_some && j0 >= a.n_sinks)) continue;   // nothing for this wave
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
      copy(t, id);
      const unsigned pages = (unsigned)__ballot((unsigned)id < (unsigned)p.n_pages) & 0xff;
      wait_vmcnt<0>();
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

// Joins the parts of a split call.  RT threads to a row and head: a whole
// workgroup where there are many parts, else DH / 4.
template <class T, int DH, bool MANY>
__global__ __launch_bounds__(256) void k_paged_join_tiles(const PagedAttnArgs a, const float* work, int parts) {
  constexpr int RT = MANY ? 256 : DH / 4, R = 256 / RT;
  const PagedPool& p = a.pool;
  const int lane = threadIdx.x & 63, G = p.H / p.Hk;
  const int per_tile = kPreRows / R;
  const int piece = blockIdx.x % per_tile, kvh = blockIdx.x / per_tile % p.Hk, number = blockIdx.x / per_tile / p.Hk;
  const RowTile rt = find_tile(a, G, number, lane);
  const int r = piece * R + threadIdx.x / RT, v = rt.first + r;
  if (rt.seq < 0 || v >= rt.rows) return;   // MANY: uniform
  const float* from = work + (((int64_t)number * parts * p.Hk + kvh) * kPreRows + r) * (DH + 4);
  const int64_t step = (int64_t)p.Hk * kPreRows * (DH + 4);
  const int n = (int)from[3];   // written for every row of a call of several parts
  if (n == 1) return;           // part 0 has written the output
  uint16_t* out = a.out + (rt.begin + v / G) * a.out_stride + (kvh * G + v % G) * DH;
  if constexpr (MANY) {
    __shared__ JoinLds<DH, 256, kPreMaxParts> lds;
    join_row<T, DH, 256>(from, step, n, lds, out);
  } else {
    const int d = threadIdx.x % RT * 4;
    float m = -INFINITY;
#pragma unroll 4
    for (int c = 0; c < n; ++c) m = fmaxf(m, from[c * step]);
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f, saw = 0.f;
    pf32x4 o = {0, 0, 0, 0};
#pragma unroll 4
    for (int c = 0; c < n; ++c) {
      const pf32x4 x = *(const pf32x4*)(from + c * step);
      const float f = __builtin_amdgcn_exp2f(x[0] - ref);
      l += x[1] * f;
      saw += x[2];
      o += *(const pf32x4*)(from + c * step + 4 + d) * f;
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = saw > 0.f ? o[k] * inv : 0.f;
    *(pu32x2*)(out + d) = pack_out<T>(o);
  }
}

PagedSplit paged_prefill_split(const PagedPool& p, int n_rows) {
  const int64_t G = p.H / p.Hk, slots = (int64_t)p.max_pages << p.page_shift;
  const int64_t partial = p.n_seqs < n_rows ? p.n_seqs : n_rows;   // tiles that are not full, at most
  PagedSplit s{};
  s.tiles = (n_rows * G) / kPreRows + partial;
  s.parts = 1;
  const int64_t base = s.tiles * p.Hk, most = (slots + kPreKeys * kPreMinTiles - 1) / (kPreKeys * kPreMinTiles);
  if (base > 0 && base <= kPreUnits / 2) {
    const int64_t want = kPreUnits / base;
    s.parts = (int)(want < most ? want : most);
  }
  s.split = s.parts > 1;
  s.units = base * s.parts;
  s.bytes = s.split ? (size_t)s.units * kPreRows * (p.dh + 4) * sizeof(float) : 0;
  return s;
}

template <class T, int DH>
static hipError_t prefill(const PagedAttnArgs& a, const PagedSplit& sp, void* workspace, hipStream_t s) {
  k_paged_prefill<T, DH><<<(unsigned)sp.units, kPreWaves * 64, 0, s>>>(a, (float*)workspace, sp.parts);
  if (sp.split) {
    const unsigned rows = (unsigned)(sp.tiles * a.pool.Hk * kPreRows);
    if (sp.parts > 16) k_paged_join_tiles<T, DH, true><<<rows, 256, 0, s>>>(a, (const float*)workspace, sp.parts);
    else k_paged_join_tiles<T, DH, false><<<rows * (DH / 4) / 256, 256, 0, s>>>(a, (const float*)workspace, sp.parts);
  }
  return hipGetLastError();
}

hipError_t launch_paged_prefill(const PagedAttnArgs& a, const PagedSplit& sp, int dtype, void* workspace, hipStream_t s) {
  if (dtype == GVC_BF16)
    return a.pool.dh == 64 ? prefill<Bf16, 64>(a, sp, workspace, s) : prefill<Bf16, 128>(a, sp, workspace, s);
  return a.pool.dh == 64 ? prefill<Fp16, 64>(a, sp, workspace, s) : prefill<Fp16, 128>(a, sp, workspace, s);
}

}  // namespace gvc
