// Driver of the sanitizer build of the paged cache's host code: argument and configuration checks, the workspace and the launch plans.
// The launchers here touch the ends of the workspace that a launch would use, so that a plan that does not fit is an error of the run.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <algorithm>
#include <random>
#include <vector>

#include <hip/hip_runtime.h>

#include "../../include/kvx.h"
#include "paged_dev.h"

#define CHECK(cond)                                                                   \
  do {                                                                                \
    if (!(cond)) {                                                                    \
      std::fprintf(stderr, "paged_host_check: line %d: %s failed\n", __LINE__, #cond); \
      std::exit(1);                                                                   \
    }                                                                                 \
  } while (0)

namespace kvx {
namespace paged {
static int64_t appends, attends, merges, weighings, weight_parts, evictions;
static AttendArgs last;
static AppendArgs last_append;
static int last_rows;
void launch_append(const AppendArgs& a, int, int, bool, bool, hipStream_t) { ++appends; last_append = a; }
void launch_attend(const AttendArgs& a, int d, int, bool, int tile_rows, hipStream_t) {
  ++attends;
  last = a;
  last_rows = tile_rows;
  CHECK(a.tiles >= 1 && a.splits >= 1 && a.split_keys >= 64 && a.split_keys % 64 == 0 && a.part_rows >= 1 && a.part_rows <= tile_rows);
  CHECK(a.tiles_per_seq == 0 || a.tiles == a.tiles_per_seq * a.c.n_seqs);
  // every row has a tile, every key that a tile can read a range
  const int64_t per_seq = ((int64_t)a.c.max_new * a.c.group + tile_rows - 1) / tile_rows;
  CHECK(a.tiles >= std::min<int64_t>(per_seq * a.c.n_seqs, (int64_t)a.c.n_tokens * a.c.group / tile_rows + a.c.n_seqs));
  const int64_t reach = a.window > 0 ? std::min<int64_t>(a.c.max_len, (int64_t)a.window + 63 + (a.causal ? std::min(a.c.max_new, tile_rows) : a.c.max_new)) : a.c.max_len;
  CHECK((int64_t)a.splits * a.split_keys >= reach);
  CHECK(a.workers >= 0 && (!a.workers || (tile_rows == 32 && a.splits == 1)) && (tile_rows != 32 || a.tiles == a.c.n_seqs));
  if (a.splits > 1 || a.workers) {
    const int64_t rows = (a.workers ? 2ll * a.workers : (int64_t)a.tiles * a.c.hkv * a.splits) * a.part_rows;
    a.part_o[0] = a.part_o[rows * d - 1] = 1.f;
    CHECK((void*)(a.part_o + rows * d) <= (void*)a.part_ml);
    a.part_ml[0] = a.part_ml[rows - 1] = float2{1.f, 1.f};
  }
}
void launch_merge(const AttendArgs& a, int, int, bool, hipStream_t) { ++merges; CHECK(a.splits > 1 || a.workers); }
void launch_weights(const AttendArgs& a, int, int, bool, hipStream_t) {
  ++weighings;
  CHECK(a.lse && a.weights_in && a.weights_out);
  if (a.c.n_tokens) a.lse[(int64_t)a.c.n_tokens * a.c.hq - 1] = 1.f;
  CHECK(a.weight_splits >= 1 && a.weight_stride >= a.c.max_len && a.weight_stride % 128 == 0);
  if (a.weight_splits > 1) {
    ++weight_parts;
    a.weight_part[0] = a.weight_part[(int64_t)a.weight_splits * a.c.n_seqs * a.c.hkv * a.weight_stride - 1] = 1.f;
  }
}
void launch_weights_from_logits(const AttendArgs& a, hipStream_t) {
  ++weighings;
  CHECK(last_rows == 32 && a.tiles_per_seq == 1 && a.lse && a.weights_in && a.weights_out && a.logit_stride >= a.c.max_len);
  CHECK(a.logit_stride % 4 == 0 && (int64_t)a.c.max_new * a.c.group <= a.part_rows);
  a.logits[0] = a.logits[(int64_t)a.tiles * a.c.hkv * a.part_rows * a.logit_stride - 1] = 1.f;
}
void launch_evict(const EvictArgs& a, int, bool, int32_t* arrived, hipStream_t) {
  ++evictions;
  const int64_t jobs = (int64_t)a.c.n_seqs * a.c.hkv;
  CHECK(a.max_moves >= std::min(a.budget, a.c.max_len - a.budget));
  a.n_moves[0] = a.n_moves[jobs - 1] = 1;
  a.moves[0] = a.moves[jobs * a.max_moves - 1] = int2{1, 1};
  for (int i = 0; i < a.c.n_seqs; ++i) CHECK(arrived[i] == 0);
}
}  // namespace paged
}  // namespace kvx

using namespace kvx::paged;

namespace {

kv_paged_config config() {
  kv_paged_config c{};
  c.n_q_heads = 8; c.n_kv_heads = 2; c.head_dim = 64; c.page_size = 16; c.dtype = KV_BF16; c.cache_dtype = KV_BF16;
  c.max_seqs = 4; c.max_tokens = 40; c.max_len = 500; c.rotary_dim = 64;
  return c;
}

// One call's worth of arguments; addresses are never followed, so any aligned ones do.
struct Args {
  kv_pages p{};
  kv_paged_batch b{};
  kv_rows q{}, k{}, out{};
  explicit Args(const kv_paged_config& c) {
    auto at = [](uintptr_t x) { return (void*)(x << 12); };
    p.k = at(1); p.v = at(2);
    p.head_stride = c.head_dim; p.slot_stride = (int64_t)c.head_dim * c.n_kv_heads; p.page_stride = p.slot_stride * c.page_size;
    p.n_pages = 100; p.pages_per_seq = (c.max_len + c.page_size - 1) / c.page_size; p.table_stride = p.pages_per_seq;
    p.page_table = (int32_t*)at(3); p.weights = (float*)at(4); p.ids = (int32_t*)at(5);
    b.n_seqs = c.max_seqs; b.n_tokens = c.max_tokens; b.max_new = (c.max_tokens + c.max_seqs - 1) / c.max_seqs; b.max_len = c.max_len;
    b.q_start = (int32_t*)at(6); b.kv_lens = (int32_t*)at(7);
    q.data = at(8); q.head_stride = c.head_dim; q.tok_stride = (int64_t)c.head_dim * c.n_q_heads;
    out = q;
    out.data = at(12);
    k.data = at(9); k.head_stride = c.head_dim; k.tok_stride = (int64_t)c.head_dim * c.n_kv_heads;
  }
};

kv_paged* make(const kv_paged_config& c) {
  kv_paged* h = nullptr;
  CHECK(kv_paged_init(&c, &h) == KV_OK && h);
  return h;
}

void plans() {
  std::mt19937 rng(1);
  auto pick = [&](int64_t lo, int64_t hi) {      // spread over the logarithm
    const double x = std::uniform_real_distribution<double>(std::log((double)lo), std::log((double)hi + 1))(rng);
    return std::min<int64_t>(hi, std::max<int64_t>(lo, (int64_t)std::exp(x)));
  };
  for (int i = 0; i < 3000; ++i) {
    kv_paged_config c = config();
    c.n_kv_heads = (int)pick(1, 16);
    c.n_q_heads = c.n_kv_heads * (int)pick(1, 16);
    c.head_dim = rng() % 2 ? 64 : 128;
    c.max_seqs = (int)pick(1, 300);
    c.max_tokens = (int)pick(1, 5000);
    c.max_len = (int)pick(1, 200000);
    c.max_evicted = (int)pick(1, std::max(1, c.max_len / 4));
    stub_cus = i % 3 ? 256 : 64;
    kv_paged* h = make(c);
    for (int j = 0; j < 6; ++j) {
      Args a(c);
      a.b.n_seqs = (int)pick(1, c.max_seqs);
      a.b.n_tokens = (int)pick(1, c.max_tokens);
      a.b.max_new = (int)pick(1, a.b.n_tokens);
      a.b.max_len = (int)pick(1, c.max_len);
      const int window = rng() % 2 ? 0 : (int)pick(1, 300000);
      CHECK(kv_paged_attend(h, &a.p, &a.b, &a.q, &a.q, nullptr, rng() % 2, window, nullptr, nullptr) == KV_OK);
      const int budget = (int)pick(1, c.max_len);
      const int moves = std::max(1, std::min(budget, a.b.max_len - budget));
      CHECK(kv_paged_evict(h, &a.p, &a.b, budget, 0, 0, a.p.weights, a.p.ids, (int32_t*)a.b.kv_lens, nullptr) == (moves > c.max_evicted ? KV_E_RANGE : KV_OK));
    }
    Args a(c);
    kv_pages p = a.p;
    std::vector<float> w(4);
    p.weights = w.data();
    CHECK(kv_paged_attend(h, &p, &a.b, &a.q, &a.out, nullptr, 1, 0, w.data(), nullptr) == KV_OK);
    a.b.n_tokens = std::min(c.max_tokens, c.max_seqs);
    a.b.n_seqs = c.max_seqs;
    a.b.max_new = 1;
    CHECK(kv_paged_attend(h, &p, &a.b, &a.q, &a.out, nullptr, 1, 0, w.data(), nullptr) == KV_OK);
    kv_paged_destroy(h);
  }
  CHECK(attends > 18000 && merges > 1000 && evictions > 1000 && weighings == 6000 && weight_parts > 100);
}

void frequencies() {
  // pair 0 turns a radian per position; the linear scaling divides, the larger base leaves pair 0 alone
  kv_paged_config c = config();
  for (int scaling = KV_ROPE_PLAIN; scaling <= KV_ROPE_PARTS; ++scaling) {
    c.rope_scaling = scaling;
    c.rope_factor = scaling == KV_ROPE_PLAIN ? 0.0 : 4.0;
    c.rope_original_len = 1000;
    kv_paged* h = make(c);
    Args a(c);
    CHECK(kv_paged_append(h, &a.p, &a.b, nullptr, nullptr, nullptr, &a.k, &a.k, nullptr) == KV_OK);
    const double first = (double)last_append.turns[0] / 18446744073709551616.0 * 6.283185307179586;
    CHECK(std::fabs(first - (scaling == KV_ROPE_LINEAR ? 0.25 : 1.0)) < 1e-12);
    const double end = (double)last_append.turns[31] / 18446744073709551616.0 * 6.283185307179586, w = std::pow(10000.0, -62.0 / 64.0);
    CHECK(std::fabs(end / w - (scaling == KV_ROPE_PLAIN ? 1.0 : 0.25)) < 1e-9);      // (base: 4^(64/62) to the power of 62/64; parts: below a turn)
    kv_paged_destroy(h);
  }
  c.rope_scaling = KV_ROPE_PLAIN;
  std::vector<double> w(32, 0.0);
  w[0] = -6.283185307179586476925286766559 / 4; w[1] = 100.0; w[2] = -1e-300;
  c.rope_freqs = w.data();
  kv_paged* h = make(c);
  Args a(c);
  CHECK(kv_paged_append(h, &a.p, &a.b, nullptr, nullptr, nullptr, &a.k, &a.k, nullptr) == KV_OK);
  CHECK(std::fabs((double)last_append.turns[0] / 18446744073709551616.0 - 0.75) < 1e-15);
  CHECK(std::fabs((double)last_append.turns[1] / 18446744073709551616.0 - (100.0 / 6.283185307179586476925286766559 - 15.0)) < 1e-13);
  kv_paged_destroy(h);
}

// Every refusal leaves its code and a text, and launches nothing.
void refusals() {
  const kv_paged_config c = config();
  kv_paged* h = make(c);
  const int64_t before = appends + attends + weighings + evictions;
  int n = 0;
  enum { kAppend = 1, kAttend = 2, kEvict = 4, kAll = 7 };
  auto refused = [&](int code, int calls, auto&& spoil) {
    Args a(c);
    const int32_t* positions = (const int32_t*)((uintptr_t)10 << 12);
    float *lse = (float*)((uintptr_t)11 << 12), *w = a.p.weights;
    int32_t budget = 300, sinks = 4, recent = 10, window = 0;
    int32_t *ids_out = a.p.ids, *lens_out = (int32_t*)a.b.kv_lens;
    kv_rows q_out = a.q, v = a.k, out = a.out;
    const kv_rows *pq = &a.q, *po = &q_out;
    spoil(a, q_out, v, out, pq, po, positions, lse, w, budget, sinks, recent, window, ids_out, lens_out);
    auto is = [&](int rc) {
      CHECK(rc == code && std::strlen(kv_paged_last_error(h)) > 10);
      ++n;
    };
    if (calls & kAppend) is(kv_paged_append(h, &a.p, &a.b, positions, pq, po, &a.k, &v, nullptr));
    if (calls & kAttend) is(kv_paged_attend(h, &a.p, &a.b, pq, &out, lse, 1, window, w, nullptr));
    if (calls & kEvict) is(kv_paged_evict(h, &a.p, &a.b, budget, sinks, recent, w, ids_out, lens_out, nullptr));
  };
#define SPOIL                                                                                                                                            \
  [&](Args & a, kv_rows & q_out, kv_rows & v, kv_rows & out, const kv_rows*& pq, const kv_rows*& po, const int32_t*& positions, float*& lse, float*& w,   \
      int32_t & budget, int32_t & sinks, int32_t & recent, int32_t & window, int32_t*& ids_out, int32_t*& lens_out)
#define REFUSED(code, calls, what)                                                                                                                       \
  refused(code, calls, SPOIL {                                                                                                                           \
    (void)a; (void)q_out; (void)v; (void)out; (void)pq; (void)po; (void)positions; (void)lse; (void)w; (void)budget; (void)sinks; (void)recent;           \
    (void)window; (void)ids_out; (void)lens_out;                                                                                                         \
    what;                                                                                                                                                \
  })
  REFUSED(KV_E_RANGE, kAll, a.b.n_seqs = 5);
  REFUSED(KV_E_RANGE, kAll, a.b.n_seqs = 0);
  REFUSED(KV_E_RANGE, kAll, a.b.n_tokens = 41);
  REFUSED(KV_E_RANGE, kAll, a.b.n_tokens = -1);
  REFUSED(KV_E_RANGE, kAll, a.b.max_new = 41);
  REFUSED(KV_E_RANGE, kAll, a.b.max_new = -1);
  REFUSED(KV_E_RANGE, kAll, a.b.max_len = 501);
  REFUSED(KV_E_RANGE, kAll, a.b.max_len = 0);
  REFUSED(KV_E_RANGE, kAll, (a.p.pages_per_seq = 31, a.p.table_stride = 31, a.b.max_len = 497));
  REFUSED(KV_E_INVAL, kAll, a.b.q_start = nullptr);
  REFUSED(KV_E_INVAL, kAll, a.b.kv_lens = nullptr);
  REFUSED(KV_E_INVAL, kAll, a.b.seen = (int32_t*)2);
  REFUSED(KV_E_INVAL, kAll, a.p.k = nullptr);
  REFUSED(KV_E_INVAL, kAll, a.p.v = nullptr);
  REFUSED(KV_E_INVAL, kAll, a.p.page_table = nullptr);
  REFUSED(KV_E_INVAL, kAll, a.p.n_pages = 0);
  REFUSED(KV_E_INVAL, kAll, a.p.pages_per_seq = 0);
  REFUSED(KV_E_INVAL, kAll, a.p.table_stride = 2);
  REFUSED(KV_E_INVAL, kAll, a.p.k = (char*)a.p.k + 8);
  REFUSED(KV_E_INVAL, kAll, a.p.slot_stride = 63);
  REFUSED(KV_E_INVAL, kAll, a.p.slot_stride = 132);
  REFUSED(KV_E_INVAL, kAll, a.p.head_stride = 68);
  REFUSED(KV_E_INVAL, kAll, a.p.page_stride = -2048);
  REFUSED(KV_E_INVAL, kAll, a.p.page_stride = 1ll << 41);
  REFUSED(KV_E_INVAL, kAll, a.p.k_scale = (float*)1);
  REFUSED(KV_E_INVAL, kAll, a.p.weights += 1);
  REFUSED(KV_E_INVAL, kAll, a.p.ids += 2);
  REFUSED(KV_E_INVAL, kAttend | kEvict, w += 1);
  REFUSED(KV_E_INVAL, kEvict, ids_out += 1);
  REFUSED(KV_E_INVAL, kAppend, po = nullptr);
  REFUSED(KV_E_INVAL, kAppend, pq = nullptr);
  REFUSED(KV_E_INVAL, kAppend, q_out.tok_stride += 8);
  REFUSED(KV_E_INVAL, kAppend, positions = (int32_t*)6);
  REFUSED(KV_E_INVAL, kAppend, a.k.data = nullptr);
  REFUSED(KV_E_INVAL, kAppend, v.head_stride = 60);
  REFUSED(KV_E_INVAL, kAppend, v.data = (char*)v.data + 2);
  REFUSED(KV_E_INVAL, kAttend, pq = nullptr);
  REFUSED(KV_E_INVAL, kAttend, out.data = nullptr);
  REFUSED(KV_E_INVAL, kAttend, out.tok_stride = 0);
  REFUSED(KV_E_INVAL, kAttend, out.tok_stride = 516);
  REFUSED(KV_E_INVAL, kAttend, out = a.q);
  REFUSED(KV_E_INVAL, kAttend, (w = nullptr, out = a.q, out.tok_stride += 8));
  REFUSED(KV_E_INVAL, kAttend, window = -1);
  REFUSED(KV_E_INVAL, kAttend, a.p.weights = nullptr);
  REFUSED(KV_E_INVAL, kAttend, lse = (float*)2);
  REFUSED(KV_E_INVAL, kEvict, a.p.weights = nullptr);
  REFUSED(KV_E_INVAL, kEvict, a.p.ids = nullptr);
  REFUSED(KV_E_INVAL, kEvict, w = nullptr);
  REFUSED(KV_E_INVAL, kEvict, ids_out = nullptr);
  REFUSED(KV_E_INVAL, kEvict, lens_out = nullptr);
  REFUSED(KV_E_INVAL, kEvict, lens_out = (int32_t*)1);
  REFUSED(KV_E_INVAL, kEvict, budget = 0);
  REFUSED(KV_E_INVAL, kEvict, budget = 13);
  REFUSED(KV_E_INVAL, kEvict, sinks = -1);
  REFUSED(KV_E_INVAL, kEvict, recent = -1);
  REFUSED(KV_E_INVAL, kEvict, (sinks = INT32_MAX, recent = INT32_MAX));
  CHECK(n > 80 && appends + attends + weighings + evictions == before);
  Args a(c);
  CHECK(kv_paged_append(h, nullptr, &a.b, nullptr, nullptr, nullptr, &a.k, &a.k, nullptr) == KV_E_INVAL);
  CHECK(kv_paged_append(h, &a.p, nullptr, nullptr, nullptr, nullptr, &a.k, &a.k, nullptr) == KV_E_INVAL);
  // no rows: their addresses are not looked at
  a.b.n_tokens = a.b.max_new = 0;
  CHECK(kv_paged_append(h, &a.p, &a.b, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == KV_OK);
  CHECK(kv_paged_attend(h, &a.p, &a.b, nullptr, nullptr, nullptr, 1, 0, nullptr, nullptr) == KV_OK);
  CHECK(appends + attends + weighings + evictions == before);
  kv_paged_destroy(h);
}

// Bounds that the kernels' 32-bit counts hold for.
void counts() {
  kv_paged_config c = config();
  c.n_q_heads = c.n_kv_heads = 256;
  c.max_seqs = 65536;
  c.max_len = 1 << 20;
  c.max_evicted = 1;
  c.max_tokens = 1;
  kv_paged* h = make(c);
  Args a(c);
  a.b.n_tokens = a.b.max_new = 1;
  const int64_t before = attends;
  CHECK(kv_paged_attend(h, &a.p, &a.b, &a.q, &a.out, nullptr, 1, 0, nullptr, nullptr) == KV_E_RANGE);
  CHECK(attends == before && std::strlen(kv_paged_last_error(h)) > 10);
  a.b.n_seqs = 1023;
  CHECK(kv_paged_attend(h, &a.p, &a.b, &a.q, &a.out, nullptr, 1, 0, nullptr, nullptr) == KV_OK);
  kv_paged_destroy(h);
}

}  // namespace

int main() {
  plans();
  counts();
  refusals();
  frequencies();
  int32_t flags = 5;
  kv_paged* h = make(config());
  CHECK(kv_paged_status(h, &flags) == KV_OK && flags == 0);
  CHECK(kv_paged_status(h, nullptr) == KV_E_INVAL);
  kv_paged_destroy(h);
  kv_paged_destroy(nullptr);
  std::printf("paged host checks passed\n");
  return 0;
}
