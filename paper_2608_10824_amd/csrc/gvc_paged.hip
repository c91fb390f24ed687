// Host side of the paged caches' operators: argument checks and launches of
// the C ABI's gvc_paged_* and gvc_quant_* calls.
#include "gvc_quant.h"

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <chrono>
#include <cmath>
#include <cstdio>
#include <random>
#include <unordered_set>

using namespace gvc;

uint64_t gvc::paged_tag() noexcept {
  // a permutation (odd multiplications and xor-shifts) of a counter from a random start
  static std::atomic<uint64_t> next{[] {
    uint64_t seed = (uint64_t)std::chrono::steady_clock::now().time_since_epoch().count();
    try {
      std::random_device d;
      seed ^= (uint64_t)d() << 32 ^ d();
    } catch (...) {   // no entropy source: the clock alone
    }
    return seed;
  }()};
  for (;;) {
    uint64_t x = next.fetch_add(1, std::memory_order_relaxed);
    x ^= x >> 32;
    x *= 0x9e3779b97f4a7c15u;
    x ^= x >> 31;
    x *= 0xd1342543de82ef95u;
    x ^= x >> 32;
    if (x) return x;
  }
}

namespace {

int32_t fail(const char* msg) noexcept { return set_error(GVC_EINVAL, msg); }

int32_t device(hipError_t e) noexcept {
  return e == hipSuccess ? GVC_OK : set_error(GVC_EDEVICE, hipGetErrorString(e));
}

constexpr int64_t kMaxSlots = 1 << 30;
// A launch has less than 2^32 threads.  Attention takes two to a row and head and
// 256 to a sequence and key-value head, or at most 2^30 (short lists, and one row to
// each of 4096 sequences).  Append takes 64 to a row (a wave of queries and keys, more
// only for fewer than 4096 rows) and 8 to a row and key-value head (values), and less than
// 2^19 besides; with fewer than five heads in all that is more than the first bound allows.
constexpr int64_t kMaxHeadRows = 1 << 28;
constexpr int64_t kMaxAppendThreads = ((int64_t)1 << 32) - (1 << 19);

// nullptr, or what is wrong with d
const char* bad_desc(const gvc_paged_desc* d) noexcept {
  if (!d) return "null desc";
  if (d->dtype != GVC_BF16 && d->dtype != GVC_FP16) return "dtype must be GVC_BF16 or GVC_FP16";
  if (d->n_kv_heads < 1 || d->n_heads < 1 || d->n_heads > 1024 || d->n_heads % d->n_kv_heads)
    return "n_heads must be a multiple of n_kv_heads, at most 1024";
  if (d->head_dim != 64 && d->head_dim != 128) return "head_dim must be 64 or 128";
  if (d->page_size != 16 && d->page_size != 32 && d->page_size != 64 && d->page_size != 128)
    return "page_size must be 16, 32, 64 or 128";
  if (d->n_pages < 1) return "n_pages must be >= 1";
  if (d->n_seqs < 1 || d->n_seqs > kPagedMaxSeqs) return "n_seqs must be in [1, 4096]";
  if (d->max_pages < 1 || (int64_t)d->max_pages * d->page_size > kMaxSlots)
    return "max_pages * page_size must be in [1, 2^30]";
  if ((int64_t)d->n_seqs * d->max_pages > 1 << 27) return "n_seqs * max_pages must be at most 2^27";
  return nullptr;
}

// A call's pages: of 16 bits, or of codes with their scales.
struct Pages {
  const void *k, *v;
  bool quant;
  const void *k_scale, *v_scale;
};

PagedPool pool_of(const gvc_paged_desc& d, const Pages& pages, const int32_t* table) noexcept {
  PagedPool p{};
  if (!pages.quant) {
    p.k = static_cast<uint16_t*>(const_cast<void*>(pages.k));
    p.v = static_cast<uint16_t*>(const_cast<void*>(pages.v));
  }
  p.table = table;
  p.n_seqs = d.n_seqs;
  p.max_pages = d.max_pages;
  p.n_pages = d.n_pages;
  p.page_shift = d.page_size == 16 ? 4 : d.page_size == 32 ? 5 : d.page_size == 64 ? 6 : 7;
  p.H = d.n_heads;
  p.Hk = d.n_kv_heads;
  p.dh = d.head_dim;
  return p;
}

QuantPages quant_pages(const Pages& p) noexcept {
  auto bytes = [](const void* x) { return static_cast<uint8_t*>(const_cast<void*>(x)); };
  return {bytes(p.k), bytes(p.v), bytes(p.k_scale), bytes(p.v_scale)};
}

bool aligned(const void* p) noexcept { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

const char* bad_pages(const Pages& p, const int32_t* page_table) noexcept {
  if (!p.k || !p.v || !page_table || (p.quant && (!p.k_scale || !p.v_scale))) return "null argument";
  return aligned(p.k) && aligned(p.v) && aligned(p.k_scale) && aligned(p.v_scale) ? nullptr
                                                                                  : "pages must be 16-byte aligned";
}

// rows of `heads` heads, `stride` elements apart
const char* bad_rows(const void* p, int64_t stride, int heads, int dh, int n_rows) noexcept {
  if (!p) return "null argument";
  if (!aligned(p) || stride % 8) return "rows must be 16-byte aligned and their stride a multiple of 8";
  if (n_rows > 1 && (stride < (int64_t)heads * dh || stride > (int64_t)1 << 32))
    return "a row stride must be in [heads * head_dim, 2^32]";
  return nullptr;
}

const char* bad_reach(int32_t window, int32_t n_sinks) noexcept {
  return window < 0 || n_sinks < 0 ? "window and n_sinks must be >= 0" : nullptr;
}

const char* bad_row_count(const gvc_paged_desc& d, int32_t n_rows) noexcept {
  return n_rows < 0 || (int64_t)n_rows * d.n_heads >= kMaxHeadRows ? "n_rows must be >= 0, and n_rows * n_heads below 2^28"
                                                                   : nullptr;
}

// A window over every slot hides none.
struct Reach {
  int window, sinks;
};
Reach reach(const gvc_paged_desc& d, int32_t window, int32_t n_sinks) noexcept {
  const int slots = d.max_pages * d.page_size;
  return {window >= slots ? 0 : window, std::min(n_sinks, slots)};
}

// The kernel that a call takes (tiled: the prefill kernel) and how it is cut.
PagedSplit plan(const PagedPool& p, int n_rows, bool lists, const Reach& r, bool quant, bool& tiled) noexcept {
  tiled = lists && !paged_few_rows(p, n_rows, r.window, r.sinks);
  if (tiled) return paged_prefill_split(p, n_rows);
  return quant ? quant_decode_split(p, n_rows, lists, r.window, r.sinks)
               : paged_decode_split(p, n_rows, lists, r.window, r.sinks);
}

int32_t attend(const gvc_paged_desc* desc, float scale, int32_t window, int32_t n_sinks, const void* q,
               int64_t q_stride, const int32_t* row_last, const int32_t* row_begin, int32_t n_rows, const Pages& pages,
               const int32_t* page_table, void* out, int64_t out_stride, void* workspace, size_t workspace_bytes,
               void* stream) noexcept {
  const gvc_paged_desc& d = *desc;
  const float scale_log2e = scale * 1.44269504088896340736f;
  if (!(scale > 0.f) || !std::isfinite(scale_log2e)) return fail("scale must be positive and finite (in powers of two too)");
  if (const char* w = bad_reach(window, n_sinks)) return fail(w);
  if (n_rows == 0) return GVC_OK;
  if (!row_last) return fail("null argument");
  if (const char* w = bad_pages(pages, page_table)) return fail(w);
  if (const char* w = bad_rows(q, q_stride, d.n_heads, d.head_dim, n_rows)) return fail(w);
  if (const char* w = bad_rows(out, out_stride, d.n_heads, d.head_dim, n_rows)) return fail(w);
  const Reach seen = reach(d, window, n_sinks);
  PagedAttnArgs a{};
  a.pool = pool_of(d, pages, page_table);
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.row_last = row_last;
  a.row_begin = row_begin;
  a.n_rows = n_rows;
  a.window = seen.window;
  a.n_sinks = seen.sinks;
  a.tag = paged_tag();
  a.scale_log2e = scale_log2e;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  bool tiled;
  const PagedSplit sp = plan(a.pool, n_rows, row_begin != nullptr, seen, pages.quant, tiled);
  if (sp.bytes && (workspace_bytes < sp.bytes || !workspace || !aligned(workspace)))
    return set_error(GVC_ENOMEM, "the workspace is too small (or not 16-byte aligned)");
  if (pages.quant)
    return device(tiled ? launch_quant_prefill(a, quant_pages(pages), sp, d.dtype, workspace, s)
                        : launch_quant_decode(a, quant_pages(pages), sp, d.dtype, workspace, s));
  return device(tiled ? launch_paged_prefill(a, sp, d.dtype, workspace, s)
                      : launch_paged_decode(a, sp, d.dtype, workspace, s));
}

int32_t append(const gvc_paged_desc* desc, const gvc_paged_rope* rope, const void* q, int64_t q_stride, const void* k,
               int64_t k_stride, const void* v, int64_t v_stride, const int32_t* row_seq, const int32_t* row_slot,
               int32_t n_rows, const Pages& pages, const int32_t* page_table, void* q_out, int64_t q_out_stride,
               void* stream) noexcept {
  if (const char* w = bad_desc(desc)) return fail(w);
  if (!rope) return fail("null rope");
  const gvc_paged_desc& d = *desc;
  int64_t n = 0;
  for (int32_t x : rope->pairs) {
    if (x < 0) return fail("pairs must be >= 0");
    n += x;
  }
  if (n % 4 || 2 * n > d.head_dim) return fail("the sum of pairs must be a multiple of 4, at most head_dim / 2");
  // (a base below a float's range would turn by more than a double can reduce)
  if (!(rope->theta >= FLT_TRUE_MIN && rope->theta <= FLT_MAX)) return fail("theta must be positive and within a float's range");
  if (!(rope->rms_eps >= 0.f)) return fail("rms_eps must be >= 0");
  if (n_rows < 0 || (int64_t)n_rows * (d.n_heads + 2 * d.n_kv_heads) >= kMaxHeadRows ||
      (int64_t)n_rows * (64 + 8 * d.n_kv_heads) >= kMaxAppendThreads)
    return fail("n_rows must be >= 0, n_rows * (n_heads + 2 n_kv_heads) below 2^28 and n_rows * (8 + n_kv_heads) below 2^29 - 2^16");
  if ((q == nullptr) != (q_out == nullptr) && n_rows) return fail("q and q_out come together");
  if (n_rows == 0) return GVC_OK;
  if (!row_seq || !row_slot) return fail("null argument");
  if (const char* w = bad_pages(pages, page_table)) return fail(w);
  if (q) {
    if (const char* w = bad_rows(q, q_stride, d.n_heads, d.head_dim, n_rows)) return fail(w);
    if (const char* w = bad_rows(q_out, q_out_stride, d.n_heads, d.head_dim, n_rows)) return fail(w);
  }
  if (const char* w = bad_rows(k, k_stride, d.n_kv_heads, d.head_dim, n_rows)) return fail(w);
  if (const char* w = bad_rows(v, v_stride, d.n_kv_heads, d.head_dim, n_rows)) return fail(w);
  if (!aligned(rope->q_norm) || !aligned(rope->k_norm)) return fail("norm gains must be 16-byte aligned");
  if (rope->positions && rope->position_stride < n_rows) return fail("position_stride must be >= n_rows");
  PagedAppendArgs a{};
  a.pool = pool_of(d, pages, page_table);
  a.q = static_cast<const uint16_t*>(q);
  a.kin = static_cast<const uint16_t*>(k);
  a.vin = static_cast<const uint16_t*>(v);
  a.q_norm = static_cast<const uint16_t*>(rope->q_norm);
  a.k_norm = static_cast<const uint16_t*>(rope->k_norm);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out_stride = q_out_stride;
  a.row_seq = row_seq;
  a.row_slot = row_slot;
  a.positions = rope->positions;
  a.position_stride = rope->position_stride;
  a.n_rows = n_rows;
  a.n_pairs = (int)n;
  a.end0 = rope->pairs[0];
  a.end1 = rope->pairs[0] + rope->pairs[1];
  a.eps = rope->rms_eps;
  // theta^(-i/n) / 2 pi by repeated products: off by at most 64 roundings of a double
  const double step = n ? std::pow(rope->theta, -1.0 / (double)n) : 1.0;
  double turn = 0.15915494309189533577;
  for (int i = 0; i < n; ++i, turn *= step) a.turns[i] = turn;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return device(pages.quant ? launch_quant_append(a, quant_pages(pages), d.dtype, s) : launch_paged_append(a, d.dtype, s));
}

int32_t workspace_of(const gvc_paged_desc* desc, int32_t prefill, int32_t n_rows, int32_t window, int32_t n_sinks,
                     size_t* bytes, bool quant) noexcept {
  if (const char* w = bad_desc(desc)) return fail(w);
  if (const char* w = bad_reach(window, n_sinks)) return fail(w);
  if (!bytes) return fail("null bytes");
  if (prefill && bad_row_count(*desc, n_rows)) return fail(bad_row_count(*desc, n_rows));
  bool tiled;
  *bytes = plan(pool_of(*desc, {}, nullptr), prefill ? n_rows : desc->n_seqs, prefill != 0, reach(*desc, window, n_sinks),
                quant, tiled).bytes;
  return GVC_OK;
}

int32_t decode(const gvc_paged_desc* desc, float scale, int32_t window, int32_t n_sinks, const void* q, int64_t q_stride,
               const int32_t* lengths, const Pages& pages, const int32_t* page_table, void* out, int64_t out_stride,
               void* workspace, size_t workspace_bytes, void* stream) noexcept {
  if (const char* w = bad_desc(desc)) return fail(w);
  return attend(desc, scale, window, n_sinks, q, q_stride, lengths, nullptr, desc->n_seqs, pages, page_table, out,
                out_stride, workspace, workspace_bytes, stream);
}

int32_t prefill(const gvc_paged_desc* desc, float scale, int32_t window, int32_t n_sinks, const void* q,
                int64_t q_stride, const int32_t* row_last, const int32_t* row_begin, int32_t n_rows, const Pages& pages,
                const int32_t* page_table, void* out, int64_t out_stride, void* workspace, size_t workspace_bytes,
                void* stream) noexcept {
  if (const char* w = bad_desc(desc)) return fail(w);
  if (const char* w = bad_row_count(*desc, n_rows)) return fail(w);
  if (n_rows && !row_begin) return fail("null argument");
  return attend(desc, scale, window, n_sinks, q, q_stride, row_last, row_begin, n_rows, pages, page_table, out,
                out_stride, workspace, workspace_bytes, stream);
}

}  // namespace

extern "C" {

int32_t gvc_paged_append(const gvc_paged_desc* desc, const gvc_paged_rope* rope, const void* q, int64_t q_stride,
                         const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* row_seq,
                         const int32_t* row_slot, int32_t n_rows, void* k_pages, void* v_pages,
                         const int32_t* page_table, void* q_out, int64_t q_out_stride, void* stream) {
  return append(desc, rope, q, q_stride, k, k_stride, v, v_stride, row_seq, row_slot, n_rows, {k_pages, v_pages},
                page_table, q_out, q_out_stride, stream);
}

int32_t gvc_quant_append(const gvc_paged_desc* desc, const gvc_paged_rope* rope, const void* q, int64_t q_stride,
                         const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* row_seq,
                         const int32_t* row_slot, int32_t n_rows, void* k_pages, void* k_scales, void* v_pages,
                         void* v_scales, const int32_t* page_table, void* q_out, int64_t q_out_stride, void* stream) {
  return append(desc, rope, q, q_stride, k, k_stride, v, v_stride, row_seq, row_slot, n_rows,
                {k_pages, v_pages, true, k_scales, v_scales}, page_table, q_out, q_out_stride, stream);
}

int32_t gvc_paged_workspace(const gvc_paged_desc* desc, int32_t prefill, int32_t n_rows, int32_t window,
                            int32_t n_sinks, size_t* bytes) {
  return workspace_of(desc, prefill, n_rows, window, n_sinks, bytes, false);
}

int32_t gvc_quant_workspace(const gvc_paged_desc* desc, int32_t prefill, int32_t n_rows, int32_t window,
                            int32_t n_sinks, size_t* bytes) {
  return workspace_of(desc, prefill, n_rows, window, n_sinks, bytes, true);
}

int32_t gvc_paged_decode(const gvc_paged_desc* desc, float scale, int32_t window, int32_t n_sinks, const void* q,
                         int64_t q_stride, const int32_t* lengths, const void* k_pages, const void* v_pages,
                         const int32_t* page_table, void* out, int64_t out_stride, void* workspace,
                         size_t workspace_bytes, void* stream) {
  return decode(desc, scale, window, n_sinks, q, q_stride, lengths, {k_pages, v_pages}, page_table, out, out_stride,
                workspace, workspace_bytes, stream);
}

int32_t gvc_quant_decode(const gvc_paged_desc* desc, float scale, int32_t window, int32_t n_sinks, const void* q,
                         int64_t q_stride, const int32_t* lengths, const void* k_pages, const void* k_scales,
                         const void* v_pages, const void* v_scales, const int32_t* page_table, void* out,
                         int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream) {
  return decode(desc, scale, window, n_sinks, q, q_stride, lengths, {k_pages, v_pages, true, k_scales, v_scales},
                page_table, out, out_stride, workspace, workspace_bytes, stream);
}

int32_t gvc_paged_prefill(const gvc_paged_desc* desc, float scale, int32_t window, int32_t n_sinks, const void* q,
                          int64_t q_stride, const int32_t* row_last, const int32_t* row_begin, int32_t n_rows,
                          const void* k_pages, const void* v_pages, const int32_t* page_table, void* out,
                          int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream) {
  return prefill(desc, scale, window, n_sinks, q, q_stride, row_last, row_begin, n_rows, {k_pages, v_pages}, page_table,
                 out, out_stride, workspace, workspace_bytes, stream);
}

int32_t gvc_quant_prefill(const gvc_paged_desc* desc, float scale, int32_t window, int32_t n_sinks, const void* q,
                          int64_t q_stride, const int32_t* row_last, const int32_t* row_begin, int32_t n_rows,
                          const void* k_pages, const void* k_scales, const void* v_pages, const void* v_scales,
                          const int32_t* page_table, void* out, int64_t out_stride, void* workspace,
                          size_t workspace_bytes, void* stream) {
  return prefill(desc, scale, window, n_sinks, q, q_stride, row_last, row_begin, n_rows,
                 {k_pages, v_pages, true, k_scales, v_scales}, page_table, out, out_stride, workspace, workspace_bytes,
                 stream);
}

int32_t gvc_quant_read(const gvc_paged_desc* desc, const int32_t* row_seq, const int32_t* row_slot, int32_t n_rows,
                       const void* k_pages, const void* k_scales, const void* v_pages, const void* v_scales,
                       const int32_t* page_table, void* k_out, int64_t k_stride, void* v_out, int64_t v_stride,
                       void* stream) {
  if (const char* w = bad_desc(desc)) return fail(w);
  const gvc_paged_desc& d = *desc;
  if (n_rows < 0 || (int64_t)n_rows * d.n_kv_heads >= kMaxHeadRows)
    return fail("n_rows must be >= 0, and n_rows * n_kv_heads below 2^28");
  if (n_rows == 0 || (!k_out && !v_out)) return GVC_OK;
  if (!row_seq || !row_slot) return fail("null argument");
  const Pages pages{k_pages, v_pages, true, k_scales, v_scales};
  if (const char* w = bad_pages(pages, page_table)) return fail(w);
  if (k_out)
    if (const char* w = bad_rows(k_out, k_stride, d.n_kv_heads, d.head_dim, n_rows)) return fail(w);
  if (v_out)
    if (const char* w = bad_rows(v_out, v_stride, d.n_kv_heads, d.head_dim, n_rows)) return fail(w);
  QuantReadArgs a{};
  a.pool = pool_of(d, pages, page_table);
  a.pages = quant_pages(pages);
  a.row_seq = row_seq;
  a.row_slot = row_slot;
  a.n_rows = n_rows;
  a.k_out = static_cast<uint16_t*>(k_out);
  a.v_out = static_cast<uint16_t*>(v_out);
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  return device(launch_quant_read(a, d.dtype, static_cast<hipStream_t>(stream)));
}

int32_t gvc_paged_check(const gvc_paged_desc* desc, const int32_t* page_table, const int32_t* lengths,
                        const int32_t* row_seq, const int32_t* row_slot, int32_t n_rows) {
  if (const char* w = bad_desc(desc)) return fail(w);
  const gvc_paged_desc& d = *desc;
  if (!page_table || n_rows < 0 || (n_rows && (!row_seq || !row_slot))) return fail("null argument or negative n_rows");
  char msg[160];
  const int64_t slots = (int64_t)d.max_pages * d.page_size;
  auto page_of = [&](int s, int64_t j) { return page_table[(int64_t)s * d.max_pages + j / d.page_size]; };
  if (lengths)
    for (int s = 0; s < d.n_seqs; ++s) {
      if (lengths[s] < 0 || lengths[s] > slots) {
        std::snprintf(msg, sizeof msg, "sequence %d: length %d is not in [0, %lld]", s, lengths[s], (long long)slots);
        return fail(msg);
      }
      for (int64_t j = 0; j < lengths[s]; j += d.page_size)
        if (page_of(s, j) < 0 || page_of(s, j) >= d.n_pages) {
          std::snprintf(msg, sizeof msg, "sequence %d: slot %lld is on page %d of %d", s, (long long)j, page_of(s, j),
                        d.n_pages);
          return fail(msg);
        }
    }
  try {
    std::unordered_set<int64_t> taken;
    for (int r = 0; r < n_rows; ++r) {
      const int s = row_seq[r];
      const int64_t j = row_slot[r];
      if (s == -1) continue;
      if (s < -1 || s >= d.n_seqs || j < 0 || j >= slots) {
        std::snprintf(msg, sizeof msg, "row %d: no slot %lld of sequence %d", r, (long long)j, s);
        return fail(msg);
      }
      if (page_of(s, j) < 0 || page_of(s, j) >= d.n_pages) {
        std::snprintf(msg, sizeof msg, "row %d: slot %lld of sequence %d is on page %d of %d", r, (long long)j, s,
                      page_of(s, j), d.n_pages);
        return fail(msg);
      }
      if (!taken.insert((int64_t)page_of(s, j) * d.page_size + j % d.page_size).second) {
        std::snprintf(msg, sizeof msg, "row %d: another row has its place (slot %lld of sequence %d)", r, (long long)j,
                      s);
        return fail(msg);
      }
    }
  } catch (...) {
    return set_error(GVC_ENOMEM, "out of host memory");
  }
  return GVC_OK;
}

}  // extern "C"
