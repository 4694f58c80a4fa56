// Driver of a sanitizer build of the paged cache's host code: calls while another device than the handle's is current.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include <hip/hip_runtime.h>

#include "../../include/kvx.h"
#include "paged_dev.h"

#define CHECK(cond)                                                                     \
  do {                                                                                  \
    if (!(cond)) {                                                                      \
      std::fprintf(stderr, "paged_device_check: line %d: %s failed\n", __LINE__, #cond); \
      std::exit(1);                                                                     \
    }                                                                                   \
  } while (0)

namespace kvx {
namespace paged {
static int launches;
void launch_append(const AppendArgs&, int, int, bool, bool, hipStream_t) { ++launches; }
void launch_attend(const AttendArgs&, int, int, bool, int, hipStream_t) { ++launches; }
void launch_merge(const AttendArgs&, int, int, bool, hipStream_t) { ++launches; }
void launch_weights(const AttendArgs&, int, int, bool, hipStream_t) { ++launches; }
void launch_weights_from_logits(const AttendArgs&, hipStream_t) { ++launches; }
void launch_evict(const EvictArgs&, int, bool, int32_t*, hipStream_t) { ++launches; }
}  // namespace paged
}  // namespace kvx

int main() {
  kv_paged_config c{};
  c.n_q_heads = 8; c.n_kv_heads = 2; c.head_dim = 64; c.page_size = 16; c.dtype = KV_BF16; c.cache_dtype = KV_BF16;
  c.max_seqs = 4; c.max_tokens = 40; c.max_len = 500;
  stub_device = 1;
  kv_paged* h = nullptr;
  CHECK(kv_paged_init(&c, &h) == KV_OK && h);
  // addresses are never followed
  auto at = [](uintptr_t x) { return (void*)(x << 12); };
  kv_pages p{};
  p.k = at(1); p.v = at(2);
  p.head_stride = 64; p.slot_stride = 128; p.page_stride = 2048; p.n_pages = 100; p.pages_per_seq = p.table_stride = 32;
  p.page_table = (int32_t*)at(3); p.weights = (float*)at(4); p.ids = (int32_t*)at(5);
  kv_paged_batch b{};
  b.n_seqs = 4; b.n_tokens = 40; b.max_new = 10; b.max_len = 500; b.q_start = (int32_t*)at(6); b.kv_lens = (int32_t*)at(7);
  kv_rows q{at(8), 512, 64}, k{at(9), 128, 64}, out{at(10), 512, 64};
  auto all = [&](int code) {
    int32_t flags = 77;
    CHECK(kv_paged_append(h, &p, &b, nullptr, nullptr, nullptr, &k, &k, nullptr) == code);
    CHECK(kv_paged_attend(h, &p, &b, &q, &out, nullptr, 1, 0, nullptr, nullptr) == code);
    CHECK(kv_paged_evict(h, &p, &b, 300, 4, 10, p.weights, p.ids, (int32_t*)b.kv_lens, nullptr) == code);
    CHECK(kv_paged_status(h, &flags) == code);
    CHECK(flags == (code == KV_OK ? 0 : 77));
    CHECK(code == KV_OK || std::strstr(kv_paged_last_error(h), "device"));
  };
  const int devices[] = {1, 0, 1, 2};
  for (int device : devices) {
    stub_device = device;
    const int before = kvx::paged::launches;
    all(device == 1 ? KV_OK : KV_E_STATE);
    CHECK((kvx::paged::launches > before) == (device == 1));
  }
  kv_paged_destroy(h);      // whatever device is current
  std::printf("paged device checks passed\n");
  return 0;
}
