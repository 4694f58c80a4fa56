// Host side of the paged cache: configuration and argument checks, rotary frequencies, the workspace and the launch plan.
// Nothing about a sequence is kept here: lengths and page tables are read by the kernels.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "../../include/kvx.h"
#include "paged_dev.h"

using namespace kvx::paged;

struct kv_paged {
  kv_paged_config cfg{};
  int device = 0;
  int32_t n_cus = 256;
  int32_t group = 1;
  int32_t page_shift = 0;
  int32_t cache_elt = 2;        // bytes of a stored element
  float factor = 0.f;           // softmax scale * log2(e)
  uint8_t* mem = nullptr;
  int32_t* status = nullptr;
  int32_t* arrived = nullptr;   // [max_seqs]
  uint64_t* turns = nullptr;    // [rotary_dim / 2]
  float* lse = nullptr;         // [max_tokens][Hq], where the caller wants weights but no lse
  uint8_t* work = nullptr;      // partial results of an attention launch, or the moves of an eviction: calls are ordered
  int64_t part_rows_cap = 0;    // rows of partial results that fit
  float* logits = nullptr;      // of launches of few rows that collect weights
  int64_t logits_cap = 0;       // floats
  std::string err;
};

namespace {

thread_local std::string g_paged_error;

int fail(kv_paged* h, int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  try {
    (h ? h->err : g_paged_error) = buf;
  } catch (...) {      // no memory for the text: the code stands
  }
  return code;
}

int64_t align_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

int check_config(const kv_paged_config* c) {
  if (!c) return fail(nullptr, KV_E_INVAL, "kv_paged_init: cfg is NULL");
  if (c->n_kv_heads < 1 || c->n_kv_heads > 256) return fail(nullptr, KV_E_INVAL, "kv_paged_init: n_kv_heads must be in [1, 256]");
  if (c->n_q_heads < 1 || c->n_q_heads > 1024 || c->n_q_heads % c->n_kv_heads || c->n_q_heads / c->n_kv_heads > 128)
    return fail(nullptr, KV_E_INVAL, "kv_paged_init: n_q_heads must be a multiple of n_kv_heads, at most 128 times as many and at most 1024");
  if (c->head_dim != 64 && c->head_dim != 128) return fail(nullptr, KV_E_INVAL, "kv_paged_init: head_dim must be 64 or 128");
  if (c->page_size < 8 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
    return fail(nullptr, KV_E_INVAL, "kv_paged_init: page_size must be a power of two in [8, 1024]");
  if (c->dtype != KV_BF16 && c->dtype != KV_F16) return fail(nullptr, KV_E_INVAL, "kv_paged_init: dtype must be KV_BF16 or KV_F16");
  if (c->cache_dtype != c->dtype && c->cache_dtype != KV_E4M3)
    return fail(nullptr, KV_E_INVAL, "kv_paged_init: cache_dtype must be dtype or KV_E4M3");
  if (c->max_seqs < 1 || c->max_seqs > (1 << 16)) return fail(nullptr, KV_E_INVAL, "kv_paged_init: max_seqs must be in [1, 65536]");
  if (c->max_tokens < 1 || c->max_tokens > (1 << 22)) return fail(nullptr, KV_E_INVAL, "kv_paged_init: max_tokens must be in [1, 2^22]");
  if (c->max_len < 1 || c->max_len > (1 << 27)) return fail(nullptr, KV_E_INVAL, "kv_paged_init: max_len must be in [1, 2^27]");
  if (c->max_evicted < 0 || c->max_evicted > c->max_len) return fail(nullptr, KV_E_INVAL, "kv_paged_init: max_evicted must be in [0, max_len]");
  if (!(c->softmax_scale >= 0.f) || !std::isfinite(c->softmax_scale))
    return fail(nullptr, KV_E_INVAL, "kv_paged_init: softmax_scale must be finite and >= 0");
  if (c->rotary_dim < 0 || c->rotary_dim > c->head_dim || c->rotary_dim % 16)
    return fail(nullptr, KV_E_INVAL, "kv_paged_init: rotary_dim must be a multiple of 16 in [0, head_dim]");
  if (c->rope_layout != KV_ROPE_HALF && c->rope_layout != KV_ROPE_INTERLEAVED)
    return fail(nullptr, KV_E_INVAL, "kv_paged_init: rope_layout must be KV_ROPE_HALF or KV_ROPE_INTERLEAVED");
  if (c->rope_scaling < KV_ROPE_PLAIN || c->rope_scaling > KV_ROPE_PARTS) return fail(nullptr, KV_E_INVAL, "kv_paged_init: unknown rope_scaling");
  if (!(c->rope_base >= 0.0) || !std::isfinite(c->rope_base) || (c->rope_base > 0.0 && c->rope_base <= 1.0))
    return fail(nullptr, KV_E_INVAL, "kv_paged_init: rope_base must be above 1 (or 0 for 10000)");
  if (!(c->rope_factor >= 0.0) || !std::isfinite(c->rope_factor) || (c->rope_factor > 0.0 && c->rope_factor < 1.0))
    return fail(nullptr, KV_E_INVAL, "kv_paged_init: rope_factor must be at least 1 (or 0 for 1)");
  if (!(c->rope_magnitude >= 0.f) || !std::isfinite(c->rope_magnitude))
    return fail(nullptr, KV_E_INVAL, "kv_paged_init: rope_magnitude must be finite and >= 0");
  if (!(c->rope_low_turns >= 0.0) || !(c->rope_high_turns >= 0.0) || !std::isfinite(c->rope_low_turns) || !std::isfinite(c->rope_high_turns))
    return fail(nullptr, KV_E_INVAL, "kv_paged_init: rope_low_turns and rope_high_turns must be finite and >= 0");
  if (c->rotary_dim && !c->rope_freqs && c->rope_scaling == KV_ROPE_PARTS) {
    const double low = c->rope_low_turns > 0.0 ? c->rope_low_turns : 1.0, high = c->rope_high_turns > 0.0 ? c->rope_high_turns : 4.0;
    if (c->rope_original_len < 1) return fail(nullptr, KV_E_INVAL, "kv_paged_init: KV_ROPE_PARTS needs rope_original_len");
    if (!(high > low)) return fail(nullptr, KV_E_INVAL, "kv_paged_init: rope_high_turns must be above rope_low_turns");
  }
  if (c->rotary_dim && c->rope_freqs)
    for (int i = 0; i < c->rotary_dim / 2; ++i)
      if (!std::isfinite(c->rope_freqs[i])) return fail(nullptr, KV_E_INVAL, "kv_paged_init: rope_freqs[%d] is not finite", i);
  return KV_OK;
}

// Frequency of pair i in radians per position.
double frequency(const kv_paged_config& c, int i) {
  if (c.rope_freqs) return c.rope_freqs[i];
  const double r = c.rotary_dim, f = c.rope_factor > 0.0 ? c.rope_factor : 1.0;
  double base = c.rope_base > 0.0 ? c.rope_base : 10000.0;
  if (c.rope_scaling == KV_ROPE_BASE) base *= std::pow(f, r / (r - 2.0));
  const double w = std::pow(base, -2.0 * i / r);
  if (c.rope_scaling == KV_ROPE_LINEAR) return w / f;
  if (c.rope_scaling == KV_ROPE_PARTS) {
    const double low = c.rope_low_turns > 0.0 ? c.rope_low_turns : 1.0, high = c.rope_high_turns > 0.0 ? c.rope_high_turns : 4.0;
    const double turns = c.rope_original_len * w / 6.283185307179586476925286766559;
    const double keep = std::min(1.0, std::max(0.0, (turns - low) / (high - low)));
    return w / f * (1.0 - keep) + w * keep;
  }
  return w;
}

// Turns per position as a fraction of 2^64.
uint64_t turn_fraction(double radians) {
  const long double t = (long double)radians / 6.283185307179586476925286766559005768L;
  const long double f = t - floorl(t);
  return f >= 1.0L ? 0 : (uint64_t)(f * 18446744073709551616.0L);      // (f < 1, and the product of it is below 2^64 for every such f)
}

// ---- arguments of a call ----------------------------------------------------------------
int check_rows(kv_paged* h, const char* call, const char* name, const kv_paged_batch* b, const kv_rows* r, Rows* out) {
  if (b->n_tokens == 0) return KV_OK;      // no rows: nothing is read
  if (!r || !r->data) return fail(h, KV_E_INVAL, "%s: %s is NULL", call, name);
  const int d = h->cfg.head_dim;
  if (r->tok_stride < d || r->head_stride < d) return fail(h, KV_E_INVAL, "%s: strides of %s must be >= head_dim", call, name);
  if (r->tok_stride > (1ll << 40) || r->head_stride > (1ll << 40)) return fail(h, KV_E_INVAL, "%s: strides of %s are out of range", call, name);
  if (((uintptr_t)r->data & 15) || (r->tok_stride * 2) % 16 || (r->head_stride * 2) % 16)
    return fail(h, KV_E_INVAL, "%s: rows of %s must be 16-byte aligned", call, name);
  out->p = (uint8_t*)r->data;
  out->tok = r->tok_stride * 2;
  out->head = r->head_stride * 2;
  return KV_OK;
}

int check_device(kv_paged* h, const char* call) {
  int device = -1;
  if (hipGetDevice(&device) == hipSuccess && device == h->device) return KV_OK;
  (void)hipGetLastError();
  return fail(h, KV_E_STATE, "%s: device %d is current, the handle belongs to device %d", call, device, h->device);
}

int check_call(kv_paged* h, const char* call, const kv_pages* p, const kv_paged_batch* b, Call* out) {
  if (!p || !b) return fail(h, KV_E_INVAL, "%s: %s is NULL", call, p ? "batch" : "pages");
  const kv_paged_config& c = h->cfg;
  const int rc = check_device(h, call);
  if (rc != KV_OK) return rc;
  if (b->n_seqs < 1 || b->n_seqs > c.max_seqs) return fail(h, KV_E_RANGE, "%s: %d sequences, the handle takes 1..%d (max_seqs)", call, b->n_seqs, c.max_seqs);
  if (b->n_tokens < 0 || b->n_tokens > c.max_tokens)
    return fail(h, KV_E_RANGE, "%s: %d new tokens, the handle takes 0..%d (max_tokens)", call, b->n_tokens, c.max_tokens);
  if (b->max_new < 0 || b->max_new > b->n_tokens) return fail(h, KV_E_RANGE, "%s: max_new must be in [0, n_tokens]", call);
  if (b->max_len < 1 || b->max_len > c.max_len) return fail(h, KV_E_RANGE, "%s: max_len must be in [1, %d] (the handle's)", call, c.max_len);
  if (!b->q_start || !b->kv_lens) return fail(h, KV_E_INVAL, "%s: q_start or kv_lens is NULL", call);
  if (!p->k || !p->v || !p->page_table) return fail(h, KV_E_INVAL, "%s: pages: NULL pointer", call);
  if (p->n_pages < 1) return fail(h, KV_E_INVAL, "%s: n_pages must be >= 1", call);
  const int64_t d = c.head_dim, elt = h->cache_elt, most = (((1ll << 32) - 1) * 16) / elt;      // (kernels count in 16 bytes, 32 bits)
  if (p->page_stride < d || p->slot_stride < d || p->head_stride < d || p->page_stride > most || p->slot_stride > most || p->head_stride > most)
    return fail(h, KV_E_INVAL, "%s: strides of the pages must be >= head_dim and below 2^36 bytes", call);
  if ((((uintptr_t)p->k | (uintptr_t)p->v) & 15) || (p->page_stride * elt) % 16 || (p->slot_stride * elt) % 16 || (p->head_stride * elt) % 16)
    return fail(h, KV_E_INVAL, "%s: rows of the pages must be 16-byte aligned", call);
  if (p->pages_per_seq < 1 || p->table_stride < p->pages_per_seq)
    return fail(h, KV_E_INVAL, "%s: pages_per_seq must be >= 1 and table_stride no smaller", call);
  if (((int64_t)p->pages_per_seq << h->page_shift) < b->max_len)
    return fail(h, KV_E_RANGE, "%s: %d pages of %d slots hold fewer than max_len = %d tokens", call, p->pages_per_seq, c.page_size, b->max_len);
  if (((uintptr_t)p->page_table | (uintptr_t)b->q_start | (uintptr_t)b->kv_lens | (uintptr_t)b->seen | (uintptr_t)p->k_scale | (uintptr_t)p->v_scale) & 3)
    return fail(h, KV_E_INVAL, "%s: arrays must be 4-byte aligned", call);
  if (((uintptr_t)p->weights | (uintptr_t)p->ids) & 15) return fail(h, KV_E_INVAL, "%s: weights and ids must be 16-byte aligned", call);
  Call& o = *out;
  o.k = (uint8_t*)p->k;
  o.v = (uint8_t*)p->v;
  o.page_stride = (uint32_t)(p->page_stride * elt / 16);
  o.slot_stride = (uint32_t)(p->slot_stride * elt / 16);
  o.head_stride = (uint32_t)(p->head_stride * elt / 16);
  o.table = p->page_table;
  o.table_stride = p->table_stride;
  o.k_scale = p->k_scale;
  o.v_scale = p->v_scale;
  o.weights = p->weights;
  o.ids = p->ids;
  o.start = b->q_start;
  o.lens = b->kv_lens;
  o.seen = b->seen ? b->seen : b->kv_lens;
  o.status = h->status;
  o.n_pages = p->n_pages;
  o.n_seqs = b->n_seqs;
  o.n_tokens = b->n_tokens;
  o.max_new = b->max_new;
  o.max_len = b->max_len;
  o.hq = c.n_q_heads;
  o.hkv = c.n_kv_heads;
  o.group = h->group;
  o.page_shift = h->page_shift;
  return KV_OK;
}

int too_large(kv_paged* h, const char* call) { return fail(h, KV_E_RANGE, "%s: a launch of this call would need 2^32 threads or more", call); }

int launched(kv_paged* h, const char* call) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? KV_OK : fail(h, KV_E_HIP, "%s: launch failed: %s", call, hipGetErrorString(e));
}

// ---- the attention launch ------------------------------------------------------------------
// Row tiles: a sequence's rows (new tokens x heads of the group) in pieces of tile_rows.  Where every sequence may have the same
// number of tiles a tile's number is direct; where that would be more than the call's rows can fill, tiles are counted out in the kernel.
void plan_tiles(const kv_paged* h, AttendArgs& a, int tile_rows) {
  const int64_t per_seq = ((int64_t)a.c.max_new * h->group + tile_rows - 1) / tile_rows;
  const int64_t direct = per_seq * a.c.n_seqs, counted = (int64_t)a.c.n_tokens * h->group / tile_rows + a.c.n_seqs;
  a.tiles_per_seq = direct <= counted ? (int32_t)per_seq : 0;
  a.tiles = (int32_t)std::min(direct, counted);
  a.part_rows = (int32_t)std::min<int64_t>(tile_rows, (int64_t)a.c.max_new * h->group);
}

// Most keys that a row tile reads.
int64_t reach(const AttendArgs& a) {
  int64_t keys = a.c.max_len;
  if (a.window > 0) keys = std::min<int64_t>(keys, (int64_t)a.window + (a.causal ? std::min<int64_t>(a.c.max_new, kChunkRows) : a.c.max_new) + 64);
  return align_up(keys, 64);
}

// Launches of few rows: as many workers as the chip holds workgroups of that kernel (by its LDS and registers two on a compute unit
// where a row of d channels is 256 bytes or its outputs are, three else).  Short columns, or many that are not long, have a workgroup each
// and nothing to join.
int few_workers(const kv_paged* h) { return (h->cfg.head_dim == 128 ? 2 : 3) * h->n_cus; }
void plan_workers(const kv_paged* h, AttendArgs& a) {
  const int64_t keys = reach(a), columns = (int64_t)a.tiles * a.c.hkv;
  const int workers = few_workers(h);
  a.splits = 1;
  a.split_keys = (int32_t)keys;
  a.workers = keys <= 256 || (keys <= 1024 && columns >= 2 * workers) ? 0 : (int32_t)std::min<int64_t>(workers, columns * parts_of(keys, kFewKeys));
}

// Launches of more rows: key ranges per row tile, for the fewest rounds of the workgroups that the chip holds at a time; a workgroup costs
// about four tiles of 64 keys by itself, and fifty of them as much as one for what the merge reads.  A causal tile has only the ranges that it sees: where
// the last f of the keys are new, a range that begins at x of them is seen by (1 - x) / f of the tiles (16 heads of 128, 2048 new
// tokens of 2048: three ranges, 53 us; two, 62; one, 67.  12 heads on two of 128, 27 tokens on 10397: 33 ranges, 27; sixteen, 35; 58, 30).
void plan_splits(const kv_paged* h, AttendArgs& a) {
  const int64_t keys = reach(a), columns = (int64_t)a.tiles * a.c.hkv;
  const int64_t fit = std::max<int64_t>(1, h->part_rows_cap / std::max<int64_t>(1, columns * a.part_rows));
  const int64_t slots = (h->cfg.head_dim == 128 ? 2ll : 3ll) * h->n_cus, tiles = keys / 64;
  const double fresh = a.causal && keys >= a.c.max_len ? std::min(1.0, (double)a.c.max_new / a.c.max_len) : 0.0;
  int64_t range = keys;
  double best = 0.0;
  for (int64_t s = 1; s <= std::min<int64_t>(64, tiles); ++s) {
    const int64_t all = std::min(s, (int64_t)((double)s * (1.0 - fresh)) + 1), some = s - all;
    const double seen = (double)all + (some > 0 ? (double)(some * (some + 1)) / (2.0 * (double)s * fresh) : 0.0);
    const int64_t blocks = (int64_t)((double)columns * seen);
    const double cost = (double)((blocks + slots - 1) / slots) * ((double)((tiles + s - 1) / s) + 4.0) + (s > 1 ? 4.0 + 0.02 * (double)blocks : 0.0);
    if (s == 1 || cost < 0.97 * best) {
      best = cost;
      range = (tiles + s - 1) / s * 64;
    }
  }
  int64_t splits = (keys + range - 1) / range;
  if (splits > fit) {
    range = align_up((keys + fit - 1) / fit, 64);
    splits = (keys + range - 1) / range;
  }
  a.split_keys = (int32_t)range;
  a.splits = (int32_t)splits;
}

// Parts of the rows in the launch that forms weights again: as many as give a compute unit eight workgroups (a key late in a causal call
// has few rows, and its workgroups end at once), of at least 128 rows.  12 heads on two of 64, three sequences of 2330 tokens, 1985 of
// them new: 112 us for the call, 120 at four workgroups, 218 at one, 327 in one part.  The sums lie where attention's partial results were, which the merge in
// front of this launch has read.
void plan_weights(const kv_paged* h, AttendArgs& a) {
  const int64_t stride = align_up(a.c.max_len, kWeightKeys), blocks = stride / kWeightKeys * a.c.hkv * a.c.n_seqs;
  const int64_t rows = (int64_t)a.c.max_new * h->group, fit = h->part_rows_cap * h->cfg.head_dim / (kWeightKeys * blocks);
  const int64_t splits = std::min(std::min<int64_t>(8ll * h->n_cus / blocks, rows / 128), std::min<int64_t>(fit, 32));
  a.weight_splits = (int32_t)std::max<int64_t>(1, splits);
  a.weight_rows = (int32_t)align_up((rows + a.weight_splits - 1) / a.weight_splits, 64);
  a.weight_stride = (int32_t)stride;
  a.weight_part = (float*)h->work;
}

}  // namespace

extern "C" {

int kv_paged_init(const kv_paged_config* cfg, kv_paged** out) {
  if (!out) return fail(nullptr, KV_E_INVAL, "kv_paged_init: out is NULL");
  *out = nullptr;
  int rc = check_config(cfg);
  if (rc != KV_OK) return rc;
  kv_paged* h = new (std::nothrow) kv_paged();
  if (!h) return fail(nullptr, KV_E_NOMEM, "kv_paged_init: host allocation failed");
  h->cfg = *cfg;
  kv_paged_config& c = h->cfg;
  if (c.max_evicted == 0) c.max_evicted = std::max(1, c.max_len / 2);
  h->group = c.n_q_heads / c.n_kv_heads;
  while ((1 << h->page_shift) < c.page_size) ++h->page_shift;
  h->cache_elt = c.cache_dtype == KV_E4M3 ? 1 : 2;
  const float scale = c.softmax_scale > 0.f ? c.softmax_scale : 1.0f / std::sqrt((float)c.head_dim);
  h->factor = scale * 1.4426950408889634f;

  int cus = 0;
  hipError_t e = hipGetDevice(&h->device);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, h->device);
  if (e == hipSuccess && cus < 1) e = hipErrorInvalidDevice;
  if (e != hipSuccess) {
    rc = fail(nullptr, KV_E_HIP, "kv_paged_init: no HIP device: %s", hipGetErrorString(e));
    (void)hipGetLastError();
    delete h;
    return rc;
  }
  h->n_cus = cus;

  // partial results: two places a worker, and what plan_splits can ask for up to 256 K rows (calls that would need more get fewer ranges)
  const int64_t few_rows = (int64_t)c.n_kv_heads * c.max_seqs * std::min<int64_t>(kFewRows, (int64_t)c.max_tokens * h->group);
  const int64_t chunk_rows = (int64_t)c.max_tokens * h->group > kFewRows
                                 ? c.n_kv_heads * ((int64_t)c.max_tokens * h->group + (int64_t)kChunkRows * c.max_seqs) : 0;
  h->part_rows_cap = std::max<int64_t>(2ll * few_workers(h) * std::min<int64_t>(kFewRows, (int64_t)c.max_tokens * h->group),
                                       std::min<int64_t>(1 << 18, chunk_rows * ((c.max_len + 127) / 128)));
  const int64_t part_bytes = h->part_rows_cap * (c.head_dim * 4 + 8);
  const int64_t move_bytes = (int64_t)c.max_seqs * c.n_kv_heads * ((int64_t)c.max_evicted * 8 + 4);
  // logits: for the largest such launch, up to 128 MB (calls that would need more form them twice)
  h->logits_cap = std::min<int64_t>(1 << 25, few_rows * align_up(c.max_len, 64));
  const int64_t head_bytes = align_up(256 + 64 * 8 + (int64_t)c.max_seqs * 4, 256);
  const int64_t lse_bytes = align_up((int64_t)c.max_tokens * c.n_q_heads * 4, 256);
  const int64_t logit_bytes = align_up(h->logits_cap * 4, 256);
  const int64_t bytes = head_bytes + lse_bytes + logit_bytes + align_up(std::max(part_bytes, move_bytes), 256);
  e = hipMalloc((void**)&h->mem, (size_t)bytes);
  if (e != hipSuccess) {
    rc = fail(nullptr, e == hipErrorOutOfMemory ? KV_E_NOMEM : KV_E_HIP, "kv_paged_init: device allocation of %lld bytes failed: %s", (long long)bytes,
              hipGetErrorString(e));
    (void)hipGetLastError();
    h->mem = nullptr;
    kv_paged_destroy(h);
    return rc;
  }
  h->status = (int32_t*)h->mem;
  h->turns = (uint64_t*)(h->mem + 256);
  h->arrived = (int32_t*)(h->mem + 256 + 64 * 8);
  h->lse = (float*)(h->mem + head_bytes);
  h->logits = (float*)(h->mem + head_bytes + lse_bytes);
  h->work = h->mem + head_bytes + lse_bytes + logit_bytes;
  uint8_t* head = new (std::nothrow) uint8_t[(size_t)head_bytes];
  if (!head) {
    kv_paged_destroy(h);
    return fail(nullptr, KV_E_NOMEM, "kv_paged_init: host allocation failed");
  }
  memset(head, 0, (size_t)head_bytes);
  for (int i = 0; i < c.rotary_dim / 2; ++i) {
    const uint64_t f = turn_fraction(frequency(c, i));
    memcpy(head + 256 + 8 * i, &f, 8);
  }
  c.rope_freqs = nullptr;                 // the caller's array
  e = hipMemcpy(h->mem, head, (size_t)head_bytes, hipMemcpyHostToDevice);
  delete[] head;
  if (e != hipSuccess) {
    rc = fail(nullptr, KV_E_HIP, "kv_paged_init: copying the rotary frequencies failed: %s", hipGetErrorString(e));
    (void)hipGetLastError();
    kv_paged_destroy(h);
    return rc;
  }
  *out = h;
  return KV_OK;
}

int kv_paged_append(kv_paged* h, const kv_pages* pages, const kv_paged_batch* batch, const int32_t* positions, const kv_rows* q,
                    const kv_rows* q_out, const kv_rows* k, const kv_rows* v, void* hip_stream) {
  if (!h) return KV_E_INVAL;
  AppendArgs a{};
  int rc = check_call(h, "kv_paged_append", pages, batch, &a.c);
  if (rc != KV_OK) return rc;
  if ((q == nullptr) != (q_out == nullptr)) return fail(h, KV_E_INVAL, "kv_paged_append: q and q_out must both be given or both be NULL");
  if (q && ((rc = check_rows(h, "kv_paged_append", "q", batch, q, &a.q)) != KV_OK || (rc = check_rows(h, "kv_paged_append", "q_out", batch, q_out, &a.q_out)) != KV_OK)) return rc;
  if (q && batch->n_tokens > 0 && q->data == q_out->data && (q->tok_stride != q_out->tok_stride || q->head_stride != q_out->head_stride))
    return fail(h, KV_E_INVAL, "kv_paged_append: q_out in the place of q needs its strides");
  if ((rc = check_rows(h, "kv_paged_append", "k", batch, k, &a.k)) != KV_OK || (rc = check_rows(h, "kv_paged_append", "v", batch, v, &a.v)) != KV_OK) return rc;
  if ((uintptr_t)positions & 3) return fail(h, KV_E_INVAL, "kv_paged_append: positions must be 4-byte aligned");
  a.positions = positions;
  a.turns = h->turns;
  a.magnitude = h->cfg.rope_magnitude > 0.f ? h->cfg.rope_magnitude : 1.f;
  a.rotary = h->cfg.rotary_dim;
  if (a.c.n_tokens == 0 || a.c.max_new == 0) return KV_OK;
  if (!append_grid(a, h->cfg.head_dim).fits()) return too_large(h, "kv_paged_append");
  launch_append(a, h->cfg.head_dim, h->cfg.dtype, h->cfg.cache_dtype == KV_E4M3, h->cfg.rope_layout == KV_ROPE_INTERLEAVED, (hipStream_t)hip_stream);
  return launched(h, "kv_paged_append");
}

int kv_paged_attend(kv_paged* h, const kv_pages* pages, const kv_paged_batch* batch, const kv_rows* q, const kv_rows* out, float* lse,
                    int32_t causal, int32_t window, float* weights_out, void* hip_stream) {
  if (!h) return KV_E_INVAL;
  AttendArgs a{};
  int rc = check_call(h, "kv_paged_attend", pages, batch, &a.c);
  if (rc != KV_OK) return rc;
  if ((rc = check_rows(h, "kv_paged_attend", "q", batch, q, &a.q)) != KV_OK || (rc = check_rows(h, "kv_paged_attend", "out", batch, out, &a.out)) != KV_OK) return rc;
  if (batch->n_tokens > 0 && q->data == out->data) {
    if (weights_out) return fail(h, KV_E_INVAL, "kv_paged_attend: out must not be q where weights are collected");
    if (q->tok_stride != out->tok_stride || q->head_stride != out->head_stride) return fail(h, KV_E_INVAL, "kv_paged_attend: out in the place of q needs its strides");
  }
  if (window < 0) return fail(h, KV_E_INVAL, "kv_paged_attend: window must be >= 0");
  if (weights_out && !a.c.weights) return fail(h, KV_E_INVAL, "kv_paged_attend: weights_out needs pages->weights");
  if ((uintptr_t)lse & 3) return fail(h, KV_E_INVAL, "kv_paged_attend: lse must be 4-byte aligned");
  if ((uintptr_t)weights_out & 15) return fail(h, KV_E_INVAL, "kv_paged_attend: weights_out must be 16-byte aligned");
  // units of keys of all sequences and key heads are counted in 32 bits, and so is the end of the workers' even shares, up to a unit a worker behind them
  if (parts_of(a.c.max_len, kFewKeys) * a.c.n_seqs * a.c.hkv > INT32_MAX - few_workers(h))
    return fail(h, KV_E_RANGE, "kv_paged_attend: n_seqs * max_len * n_kv_heads is too large");
  hipStream_t st = (hipStream_t)hip_stream;
  const kv_paged_config& c = h->cfg;
  const bool e4m3 = c.cache_dtype == KV_E4M3;
  a.lse = lse ? lse : (weights_out ? h->lse : nullptr);
  a.weights_in = a.c.weights;
  a.weights_out = weights_out;
  a.factor = h->factor;
  a.causal = causal != 0;
  a.window = std::min(window, 1 << 28);      // no sequence is longer
  // the whole plan, then the launches
  const bool attends = a.c.n_tokens > 0 && a.c.max_new > 0;
  const int tile_rows = (int64_t)a.c.max_new * h->group <= kFewRows ? kFewRows : kChunkRows;
  bool joins = false;
  if (attends) {
    plan_tiles(h, a, tile_rows);
    if (tile_rows == kFewRows) plan_workers(h, a);
    else plan_splits(h, a);
    joins = a.splits > 1 || a.workers;
    if ((int64_t)a.tiles * a.c.hkv * a.splits > INT32_MAX || !attend_grid(a).fits() || (joins && !merge_grid(a, c.head_dim).fits()))
      return too_large(h, "kv_paged_attend");
    // A kept logit is 4 bytes written and 4 read, a key formed again d elements: up to as many rows as make that the same.
    a.logit_stride = align_up(a.c.max_len, 64);
    if (weights_out && tile_rows == kFewRows && 8ll * a.part_rows <= (int64_t)c.head_dim * h->cache_elt &&
        (int64_t)a.tiles * a.c.hkv * a.part_rows * a.logit_stride <= h->logits_cap)
      a.logits = h->logits;
    a.part_o = (float*)h->work;
    a.part_ml = (float2*)(h->work + h->part_rows_cap * c.head_dim * 4);
  }
  if (weights_out && !a.logits) plan_weights(h, a);
  if (weights_out && !(a.logits ? weights_from_logits_grid(a).fits() : weights_grid(a).fits() && weights_sum_grid(a).fits()))
    return too_large(h, "kv_paged_attend");
  if (attends) launch_attend(a, c.head_dim, c.dtype, e4m3, tile_rows, st);
  if (joins) launch_merge(a, c.head_dim, c.dtype, e4m3, st);
  if (a.logits) launch_weights_from_logits(a, st);
  else if (weights_out) launch_weights(a, c.head_dim, c.dtype, e4m3, st);
  return launched(h, "kv_paged_attend");
}

int kv_paged_evict(kv_paged* h, const kv_pages* pages, const kv_paged_batch* batch, int32_t budget, int32_t sinks, int32_t recent,
                   float* weights_out, int32_t* ids_out, int32_t* lens_out, void* hip_stream) {
  if (!h) return KV_E_INVAL;
  EvictArgs a{};
  int rc = check_call(h, "kv_paged_evict", pages, batch, &a.c);
  if (rc != KV_OK) return rc;
  if (!a.c.weights || !a.c.ids) return fail(h, KV_E_INVAL, "kv_paged_evict: needs pages->weights and pages->ids");
  if (!weights_out || !ids_out || !lens_out) return fail(h, KV_E_INVAL, "kv_paged_evict: weights_out, ids_out or lens_out is NULL");
  if ((uintptr_t)lens_out & 3) return fail(h, KV_E_INVAL, "kv_paged_evict: lens_out must be 4-byte aligned");
  if (((uintptr_t)weights_out | (uintptr_t)ids_out) & 15) return fail(h, KV_E_INVAL, "kv_paged_evict: weights_out and ids_out must be 16-byte aligned");
  if (budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget)
    return fail(h, KV_E_INVAL, "kv_paged_evict: budget must be >= 1, sinks and recent >= 0 and together no more than budget");
  a.max_moves = std::max(1, std::min(budget, a.c.max_len - budget));
  if (a.max_moves > h->cfg.max_evicted)
    return fail(h, KV_E_RANGE, "kv_paged_evict: up to %d tokens of a sequence to move, the handle takes %d (max_evicted)", a.max_moves, h->cfg.max_evicted);
  a.weights_out = weights_out;
  a.ids_out = ids_out;
  a.lens_out = lens_out;
  a.n_moves = (int32_t*)h->work;
  a.moves = (int2*)(h->work + align_up((int64_t)a.c.n_seqs * a.c.hkv * 4, 8));
  a.budget = budget;
  a.sinks = sinks;
  a.recent = recent;
  if (!select_grid(a).fits()) return too_large(h, "kv_paged_evict");
  launch_evict(a, h->cfg.head_dim, h->cfg.cache_dtype == KV_E4M3, h->arrived, (hipStream_t)hip_stream);
  return launched(h, "kv_paged_evict");
}

int kv_paged_status(kv_paged* h, int32_t* flags) {
  if (!h) return KV_E_INVAL;
  if (!flags) return fail(h, KV_E_INVAL, "kv_paged_status: flags is NULL");
  const int rc = check_device(h, "kv_paged_status");      // (another device's work would be waited for)
  if (rc != KV_OK) return rc;
  const int32_t none = 0;
  if (hipDeviceSynchronize() != hipSuccess || hipMemcpy(flags, h->status, 4, hipMemcpyDeviceToHost) != hipSuccess ||
      hipMemcpy(h->status, &none, 4, hipMemcpyHostToDevice) != hipSuccess)
    return fail(h, KV_E_HIP, "kv_paged_status: %s", hipGetErrorString(hipGetLastError()));
  return KV_OK;
}

void kv_paged_destroy(kv_paged* h) {
  if (!h) return;
  if (h->mem) (void)hipFree(h->mem);
  delete h;
}

const char* kv_paged_last_error(kv_paged* h) { return h ? h->err.c_str() : g_paged_error.c_str(); }

}  // extern "C"
