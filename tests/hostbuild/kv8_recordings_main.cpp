// Recorded steps of a pool in 8 bits on the CPU, with sanitizers: batches on both sides of 2048 new tokens, where the
// append becomes another kernel, and of 256, where the merge does; more of them than recordings are held.  The stand-ins
// note the kernels of a recording, and a recording that is updated from one of other kernels is counted.  No GPU.
#include "../../include/oxy.h"
#include "../../paper_2603_14371_amd/csrc/oxy_kv8.h"

#include <cstdio>
#include <cstdlib>
#include <cstring>

extern "C" long oxy_stub_misfits();
extern "C" long oxy_stub_updates();

#define CHECK(x)                                                                    \
  do {                                                                              \
    if (!(x)) {                                                                     \
      printf("FAILED %s:%d %s (%s)\n", __FILE__, __LINE__, #x, oxy_last_error());   \
      exit(1);                                                                      \
    }                                                                               \
  } while (0)

namespace oxy {
// hip_stubs.cpp notes the launchers that it stands in for; these are told apart by what they call of them
hipError_t launch_append8(const void* k, const void* v, const int32_t* slots, int32_t n, Layer8 layer, hipStream_t s) {
  const hipError_t e = launch_append(k, v, slots, n, layer.blocks, s);
  return e == hipSuccess && n > 2048 ? launch_append(k, v, slots, n, layer.blocks, s) : e;
}
hipError_t launch_attention_work8(const AttnArgs8& a, hipStream_t s, hipEvent_t, hipEvent_t) {
  return launch_attention_work(a, s, nullptr, nullptr);
}
hipError_t launch_merge8(const AttnArgs8& a, hipStream_t s, hipEvent_t, hipEvent_t) {
  const hipError_t e = launch_merge_append(a, nullptr, s, nullptr, nullptr);
  return e == hipSuccess && a.max_parts > kLongParts ? launch_merge_append(a, nullptr, s, nullptr, nullptr) : e;
}
}  // namespace oxy

int main() {
  oxy_pool_config c;
  memset(&c, 0, sizeof(c));
  c.n_layers = 2, c.n_q_heads = 8, c.n_kv_heads = 1, c.head_dim = 256, c.page_size = 16, c.num_blocks = 400;
  c.max_q_tokens = c.max_append_tokens = 4096, c.flags = OXY_POOL_KV_FP8;
  c.kv_bytes = oxy_kv_bytes(&c);
  c.workspace_bytes = oxy_workspace_bytes(&c);
  c.kv_base = (void*)((uintptr_t)1 << 40);   // never touched
  c.workspace = aligned_alloc(256, (c.workspace_bytes + 255) / 256 * 256);
  oxy_pool* p = nullptr;
  CHECK(oxy_pool_create(&c, &p) == OXY_OK);
  int32_t sid = 0;
  CHECK(oxy_stream_create(p, -1, OXY_KIND_DECODE, &sid) == OXY_OK);
  static char rows[1];   // addresses only
  for (int i = 0; i < 60; ++i) {
    static const int lens[] = {300, 2049, 257, 2048, 4000, 5, 256};
    oxy_item item = {sid, lens[i % 7] + (i / 7 < 8 && lens[i % 7] != 2048 && lens[i % 7] != 256 ? i / 7 : 0)};
    CHECK(oxy_stream_rewind(p, sid, 0) == OXY_OK);
    oxy_batch* b = nullptr;
    CHECK(oxy_batch_build(p, &item, 1, 0, nullptr, &b) == OXY_OK);
    CHECK(oxy_step_layers(p, b, 0, 2, rows, rows, 0, rows, rows, 0, nullptr, 0, 1.f, OXY_STEP_GRAPH, nullptr, nullptr) == OXY_OK);
    CHECK(oxy_batch_destroy(b) == OXY_OK);
  }
  int32_t made = 0, updated = 0, replayed = 0;
  CHECK(oxy_step_graph_stats(p, &made, &updated, &replayed) == OXY_OK);
  CHECK(oxy_pool_destroy(p) == OXY_OK);
  free(c.workspace);
  if (oxy_stub_misfits()) {
    printf("FAILED %ld of %ld updates from a recording of other kernels\n", oxy_stub_misfits(), oxy_stub_updates());
    return 1;
  }
  CHECK(replayed == 60 && updated > 10 && oxy_stub_updates() == updated);
  printf("OK\n");
  return 0;
}
