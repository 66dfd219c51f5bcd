"""The list of tokens with many split results that a merge of a pool in 8 bits reads (compiled with gcc under
AddressSanitizer + UndefinedBehaviorSanitizer, with a stand-in for the launcher that checks it).  No GPU."""
from test_host_kv8 import ROOT, _build, _run

SOURCE = """
#include "%s/include/oxy.h"
#include "%s/paper_2603_14371_amd/csrc/oxy_kv8.h"
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>
static int g_long = 0, g_tokens = 0, g_bad = 0;
namespace oxy {
hipError_t launch_append8(const void*, const void*, const int32_t*, int32_t, Layer8, hipStream_t) { return hipSuccess; }
hipError_t launch_attention_work8(const AttnArgs8&, hipStream_t, hipEvent_t, hipEvent_t) { return hipSuccess; }
hipError_t launch_merge8(const AttnArgs8& a, hipStream_t, hipEvent_t, hipEvent_t) {   // "device" memory is host memory here
  std::vector<int32_t> want;
  int32_t most = 0;
  for (int32_t t = 0; t < a.n_q; ++t) {
    if (a.n_parts[t] > kLongParts) want.push_back(t);
    if (a.n_parts[t] > most) most = a.n_parts[t];
  }
  g_bad += (size_t)a.n_long != want.size() || most != a.max_parts;
  for (size_t i = 0; i < want.size() && !g_bad; ++i) g_bad += a.long_toks[i] != want[i];
  g_long += a.n_long, g_tokens += a.n_q;
  return hipSuccess;
}
}  // namespace oxy
#define CHECK(x) do { if (!(x)) { printf("FAILED %%d %%s (%%s)\\n", __LINE__, #x, oxy_last_error()); exit(1); } } while (0)
int main() {
  oxy_pool_config c;
  memset(&c, 0, sizeof(c));
  c.n_layers = 2, c.n_q_heads = 8, c.n_kv_heads = 1, c.head_dim = 256, c.page_size = 16, c.num_blocks = 3000;
  c.max_q_tokens = 64, c.max_append_tokens = 16384, c.stream_split_tokens = 32, c.flags = OXY_POOL_KV_FP8, c.max_partials = 16384;
  c.kv_base = (void*)((uintptr_t)1 << 40), c.kv_bytes = oxy_kv_bytes(&c);
  c.workspace_bytes = oxy_workspace_bytes(&c);
  c.workspace = aligned_alloc(256, (c.workspace_bytes + 255) / 256 * 256);
  oxy_pool* p = nullptr;
  CHECK(oxy_pool_create(&c, &p) == OXY_OK);
  static char rows[1];   // addresses only
  int32_t sid[6];
  const int hist[6] = {5000, 40, 1056, 1000, 9000, 1};
  for (int i = 0; i < 6; ++i) {
    CHECK(oxy_stream_create(p, -1, OXY_KIND_DECODE, &sid[i]) == OXY_OK);
    oxy_item item = {sid[i], hist[i]};
    oxy_batch* b = nullptr;
    CHECK(oxy_batch_build(p, &item, 1, OXY_BATCH_APPEND_ONLY, nullptr, &b) == OXY_OK);
    CHECK(oxy_batch_destroy(b) == OXY_OK);
  }
  // every subset of the requests, one to three new tokens each; as many as the descriptor holds
  for (int set = 1; set < 64; ++set) {
    std::vector<oxy_item> items;
    for (int i = 0; i < 6; ++i)
      if (set >> i & 1) items.push_back({sid[i], set == 16 ? 64 : 1 + (set + i) %% 3});
    oxy_batch* b = nullptr;
    CHECK(oxy_batch_build(p, items.data(), (int32_t)items.size(), 0, nullptr, &b) == OXY_OK);
    CHECK(oxy_mixed_attention(p, b, 0, rows, rows, nullptr, 1.f, nullptr) == OXY_OK);
    CHECK(oxy_step_layers(p, b, 0, 2, rows, rows, 0, rows, rows, 0, nullptr, 0, 1.f, 0, nullptr, nullptr) == OXY_OK);
    for (const oxy_item& it : items) {
      int32_t len = 0;
      CHECK(oxy_stream_info(p, it.stream_id, nullptr, nullptr, &len, nullptr) == OXY_OK);
      CHECK(oxy_stream_rewind(p, it.stream_id, len - it.n_new) == OXY_OK);
    }
    CHECK(oxy_batch_destroy(b) == OXY_OK);
    CHECK(!g_bad);
  }
  CHECK(g_long > 100 && g_tokens > g_long);
  CHECK(oxy_pool_destroy(p) == OXY_OK);
  free(c.workspace);
  printf("OK\\n");
  return 0;
}
"""


def test_the_merge_is_told_which_tokens_have_many_split_results(tmp_path):
    src = tmp_path / "long.cpp"
    src.write_text(SOURCE % (ROOT, ROOT))
    exe = str(tmp_path / "long")
    _build(exe, [str(src)])
    _run(exe)
