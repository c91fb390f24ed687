// Tiles of 128 virtual rows, which the prefill kernels share: how a call's lists
// are cut into them, which one a workgroup takes, and the join of parts.
#pragma once
#include "gvc_paged_rows.h"

namespace gvc {

constexpr int kPreWaves = 4, kPreRows = 32 * kPreWaves, kPreKeys = 64;
constexpr int kPreUnits = 512;   // calls with fewer units split the slots, into about as many
constexpr int kPreMinTiles = 4;  // tiles of a part, at least
constexpr int kPreMaxParts = kPreUnits;

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

// The second launch of a split call.
template <class T, int DH>
static void launch_join_tiles(const PagedAttnArgs& a, const PagedSplit& sp, const float* work, hipStream_t s) {
  const unsigned rows = (unsigned)(sp.tiles * a.pool.Hk * kPreRows);
  if (sp.parts > 16) k_paged_join_tiles<T, DH, true><<<rows, 256, 0, s>>>(a, work, sp.parts);
  else k_paged_join_tiles<T, DH, false><<<rows * (DH / 4) / 256, 256, 0, s>>>(a, work, sp.parts);
}

}  // namespace gvc
