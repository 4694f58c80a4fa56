// Driver of a sanitizer build of the paged cache's host code: every launch that a call makes has fewer than 2^32 threads in a dimension, and a
// call that would need more is refused before its first launch.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include <hip/hip_runtime.h>

#include "../../include/kvx.h"
#include "paged_dev.h"

#define CHECK(cond)                                                                   \
  do {                                                                                \
    if (!(cond)) {                                                                    \
      std::fprintf(stderr, "paged_grid_check: line %d: %s failed\n", __LINE__, #cond); \
      std::exit(1);                                                                   \
    }                                                                                 \
  } while (0)

namespace kvx {
namespace paged {
static int launches, joins, weighings, row_parts;
static void check(const Grid& g) {
  ++launches;
  CHECK(g.x >= 1 && g.y >= 1 && g.threads >= 64 && g.x * g.threads < (1ll << 32) && g.y * 1 <= 65536);
}
void launch_append(const AppendArgs& a, int d, int, bool, bool, hipStream_t) { check(append_grid(a, d)); }
void launch_attend(const AttendArgs& a, int, int, bool, int, hipStream_t) { check(attend_grid(a)); }
void launch_merge(const AttendArgs& a, int d, int, bool, hipStream_t) { check(merge_grid(a, d)); ++joins; }
void launch_weights(const AttendArgs& a, int, int, bool, hipStream_t) {
  check(weights_grid(a));
  if (a.weight_splits > 1) check(weights_sum_grid(a)), ++row_parts;
  ++weighings;
}
void launch_weights_from_logits(const AttendArgs& a, hipStream_t) { check(weights_from_logits_grid(a)); }
void launch_evict(const EvictArgs& a, int, bool, int32_t*, hipStream_t) { check(select_grid(a)); }
}  // namespace paged
}  // namespace kvx

using namespace kvx::paged;

namespace {

struct Calls {
  kv_paged* h = nullptr;
  kv_pages p{};
  kv_paged_batch b{};
  kv_rows q{}, k{}, out{};
  Calls(int hq, int hkv, int d, int seqs, int tokens, int new_tokens, int len) {
    kv_paged_config c{};
    c.n_q_heads = hq; c.n_kv_heads = hkv; c.head_dim = d; c.page_size = 1024; c.dtype = KV_BF16; c.cache_dtype = KV_BF16;
    c.max_seqs = seqs; c.max_tokens = tokens; c.max_len = len; c.max_evicted = 1;
    CHECK(kv_paged_init(&c, &h) == KV_OK);
    auto at = [](uintptr_t x) { return (void*)(x << 12); };      // addresses are never followed
    p.k = at(1); p.v = at(2); p.head_stride = d; p.slot_stride = d * hkv; p.page_stride = p.slot_stride * 1024; p.n_pages = 7;
    p.pages_per_seq = (len + 1023) / 1024; p.table_stride = p.pages_per_seq; p.page_table = (int32_t*)at(3); p.weights = (float*)at(4); p.ids = (int32_t*)at(5);
    b.n_seqs = seqs; b.n_tokens = tokens; b.max_new = new_tokens; b.max_len = len; b.q_start = (int32_t*)at(6); b.kv_lens = (int32_t*)at(7);
    q.data = at(8); q.head_stride = d; q.tok_stride = d * hq;
    k.data = at(9); k.head_stride = d; k.tok_stride = d * hkv;
    out = q;
    out.data = at(10);
  }
  ~Calls() { kv_paged_destroy(h); }
  // the code, having seen that a refusal came before any launch
  int answer(int rc, int before) {
    CHECK(rc == KV_OK || (rc == KV_E_RANGE && launches == before && std::strlen(kv_paged_last_error(h)) > 10));
    return rc;
  }
  int append(bool with_q) { const int n = launches; return answer(kv_paged_append(h, &p, &b, nullptr, with_q ? &q : nullptr, with_q ? &out : nullptr, &k, &k, nullptr), n); }
  int attend(float* w) { const int n = launches; return answer(kv_paged_attend(h, &p, &b, &q, &out, nullptr, 1, 0, w, nullptr), n); }
  int evict() { const int n = launches; return answer(kv_paged_evict(h, &p, &b, b.max_len - 1, 0, 0, p.weights, p.ids, (int32_t*)b.kv_lens, nullptr), n); }
};

}  // namespace

int main() {
  // a generous bound on the length: the launch that forms weights again has 2^24 workgroups, none of which has more than its own check to do
  {
    Calls c(8, 8, 64, 256, 256, 1, 1 << 20);
    CHECK(c.attend(nullptr) == KV_OK && c.attend(c.p.weights) == KV_OK && c.evict() == KV_OK && c.append(true) == KV_OK);
    CHECK(weighings == 1);
  }
  // ... and 2^28 keys x heads in one dimension are too many
  {
    Calls c(16, 16, 64, 2, 2, 1, 1 << 27);
    CHECK(c.attend(nullptr) == KV_OK && c.attend(c.p.weights) == KV_E_RANGE);
  }
  // joins of few rows
  {
    Calls c(1024, 8, 64, 65536, 65536, 1, 2048);      // 128 rows a key head: more than few
    CHECK(c.attend(nullptr) == KV_OK);
  }
  {
    Calls c(1024, 32, 64, 65536, 65536, 1, 2048);
    const int n = joins;
    CHECK(c.attend(nullptr) == KV_E_RANGE && c.attend(c.p.weights) == KV_E_RANGE);      // 2^26 rows
    c.b.n_seqs = c.b.n_tokens = 65535;
    CHECK(c.attend(nullptr) == KV_OK && joins == n + 1);
  }
  // one workgroup of 1024 threads a (sequence, key head)
  {
    Calls c(64, 64, 64, 65536, 1, 1, 1024);
    CHECK(c.evict() == KV_E_RANGE);
    c.b.n_seqs = 65535;
    CHECK(c.evict() == KV_OK);
  }
  // a workgroup a (sequence, key head) of short caches
  {
    Calls c(256, 256, 64, 65536, 65536, 1, 200);
    CHECK(c.attend(nullptr) == KV_E_RANGE);
    c.b.n_seqs = c.b.n_tokens = 65535;
    CHECK(c.attend(nullptr) == KV_OK);
  }
  // rows of 1536 heads
  {
    Calls c(1024, 256, 128, 1, 1 << 21, 1 << 21, 1 << 21);
    CHECK(c.append(true) == KV_E_RANGE && c.append(false) == KV_OK);
    c.b.n_tokens = c.b.max_new = (1 << 21) - 1;
    CHECK(c.append(true) == KV_OK);
  }
  // units of 128 keys: workers' shares are rounded up, and where the last one ends is counted in 32 bits too
  {
    Calls c(1, 1, 64, 65535, 1, 1, 42966 * 128);
    c.b.max_len = 32768 * 128;
    CHECK(c.attend(nullptr) == KV_OK);
    c.b.n_seqs = 49981;
    c.b.max_len = 42966 * 128;                        // 2^31 - 2 of them
    CHECK(c.attend(nullptr) == KV_E_RANGE);
  }
  // parts of the rows
  {
    Calls c(8, 8, 64, 3, 3000, 1000, 1000);
    CHECK(c.attend(c.p.weights) == KV_OK && row_parts == 1);
  }
  std::printf("paged grid checks passed\n");
  return 0;
}
