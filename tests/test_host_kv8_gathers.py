"""How many launches a read-back list of a pool in 8 bits takes (compiled with gcc under AddressSanitizer +
UndefinedBehaviorSanitizer, with stand-ins for the launchers that count).  No GPU."""
from test_host_kv8 import ROOT, _build, _run

SOURCE = """
#include "%s/include/oxy.h"
#include "%s/paper_2603_14371_amd/csrc/oxy_kv8.h"
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>
static int g_tables = 0, g_runs = 0, g_rows = 0;
namespace oxy {
hipError_t launch_attention_work8(const AttnArgs8&, hipStream_t, hipEvent_t, hipEvent_t) { return hipSuccess; }
hipError_t launch_gather_table8(void*, void*, const Table8&, const int32_t*, int32_t, int32_t n, hipStream_t) {
  ++g_tables, g_rows += n;
  return hipSuccess;
}
hipError_t launch_gather_inline8(Layer8, const GatherRuns& runs, int32_t n, void*, void*, int32_t, size_t, size_t, hipStream_t) {
  ++g_runs;
  for (int32_t i = 0; i < n; ++i) g_rows += (runs.where[i] & 15) + 1;
  return hipSuccess;
}
}  // namespace oxy
int main() {
  oxy_pool_config c;
  memset(&c, 0, sizeof(c));
  c.n_layers = 1, c.n_q_heads = 8, c.n_kv_heads = 1, c.head_dim = 256, c.page_size = 16, c.num_blocks = 4000;
  c.max_q_tokens = c.max_append_tokens = 16, c.flags = OXY_POOL_KV_FP8;
  c.kv_base = (void*)((uintptr_t)1 << 40), c.kv_bytes = oxy_kv_bytes(&c);
  c.workspace_bytes = oxy_workspace_bytes(&c);
  c.workspace = aligned_alloc(256, (c.workspace_bytes + 255) / 256 * 256);
  oxy_pool* p = nullptr;
  if (oxy_pool_create(&c, &p) != OXY_OK) return 1;
  static const int want[][4] = {   // whole blocks, slots elsewhere behind them: launches of tables, of runs
    {1, 0, 1, 0}, {300, 0, 1, 0}, {1, 5, 0, 1}, {64, 5, 0, 1}, {100, 400, 0, 1}, {200, 0, 1, 0}, {255, 5, 0, 1}, {256, 5, 1, 1},
    {1500, 5, 1, 1}, {1920, 0, 1, 0}, {1921, 0, 2, 0}, {1930, 5, 1, 1}};
  for (const auto& w : want) {
    std::vector<int64_t> slots;
    for (int i = 0; i < w[0] * 16; ++i) slots.push_back((int64_t)(3000 - i / 16) * 16 + i %% 16);
    for (int i = 0; i < w[1]; ++i) slots.push_back((int64_t)(3100 + i) * 16 + 3);
    g_tables = g_runs = g_rows = 0;
    if (oxy_gather_kv(p, 0, slots.data(), (int32_t)slots.size(), c.workspace, c.workspace, nullptr) != OXY_OK) return 2;
    if (g_tables != w[2] || g_runs != w[3] || g_rows != (int)slots.size()) {
      printf("FAILED %%d blocks and %%d slots: %%d launches of tables, %%d of runs, %%d rows\\n", w[0], w[1], g_tables, g_runs, g_rows);
      oxy_pool_destroy(p);
      free(c.workspace);
      return 3;
    }
  }
  oxy_pool_destroy(p);
  free(c.workspace);
  printf("OK\\n");
  return 0;
}
"""


def test_a_list_takes_a_table_only_where_that_saves_a_launch(tmp_path):
    """Whole blocks travel as a table where nothing follows them or where they fill a launch of runs."""
    src = tmp_path / "gathers.cpp"
    src.write_text(SOURCE % (ROOT, ROOT))
    exe = str(tmp_path / "gathers")
    _build(exe, [str(src)])
    _run(exe)
