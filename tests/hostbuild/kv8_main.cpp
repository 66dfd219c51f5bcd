// Host paths of pools in 8 bits and of the rotating append, compiled with gcc under sanitizers: stand-ins for the
// launchers record what each launch would cover; random calls are checked against that.  No GPU.
#include "../../include/oxy.h"
#include "../../paper_2603_14371_amd/csrc/oxy_kv8.h"

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

extern "C" void oxy_stub_fail_next(int skip, int k);

namespace {
struct Move {   // a row of one layer: slot and row number
  int64_t slot;
  int64_t row;
};
std::vector<Move> g_moves;   // of layer 0 of the launch
int g_launches = 0, g_append8 = 0, g_work8 = 0, g_merge8 = 0, g_rotary = 0;
const char *g_rows_k, *g_rows_v;
int32_t g_layers = 0, g_parts = 0;
oxy::RotaryAppendArgs g_rotary_args;
#define CHECK(x)                                                 \
  do {                                                           \
    if (!(x)) {                                                  \
      printf("FAILED %s:%d %s (%s)\n", __FILE__, __LINE__, #x, oxy_last_error()); \
      exit(1);                                                   \
    }                                                            \
  } while (0)

hipError_t table(const char* k, const char* v, const oxy::Table8& t, const int32_t* blocks, int32_t offset, int32_t n) {
  ++g_launches;
  CHECK(n > 0 && offset >= 0 && offset < 16 && (offset + n + 15) / 16 <= oxy::max_table_blocks(t.small_ids));
  CHECK(k - g_rows_k == v - g_rows_v);
  g_layers = t.n_layers;
  for (int32_t i = 0; i < n; ++i) {
    const int32_t id = blocks[(offset + i) / 16];
    CHECK(id >= 0 && (!t.small_ids || id < 65536));
    g_moves.push_back({(int64_t)id * 16 + (offset + i) % 16, (k - g_rows_k) / 512 + i});
  }
  return hipSuccess;
}
}  // namespace

namespace oxy {
hipError_t launch_append8(const void*, const void*, const int32_t*, int32_t, Layer8, hipStream_t) {
  ++g_append8;
  return hipSuccess;
}
hipError_t launch_append_table8(const void* k, const void* v, const Table8& t, const int32_t* blocks, int32_t offset,
                                int32_t n, hipStream_t) {
  return table((const char*)k, (const char*)v, t, blocks, offset, n);
}
hipError_t launch_gather_table8(void* k, void* v, const Table8& t, const int32_t* blocks, int32_t offset, int32_t n, hipStream_t) {
  return table((const char*)k, (const char*)v, t, blocks, offset, n);
}
hipError_t launch_gather_inline8(Layer8, const GatherRuns& runs, int32_t n_runs, void* k, void* v, int32_t n_layers, size_t,
                                 size_t, hipStream_t) {
  ++g_launches;
  g_layers = n_layers;
  CHECK(n_runs > 0 && n_runs <= kMaxRuns && (char*)k - g_rows_k == (char*)v - g_rows_v);
  for (int32_t i = 0; i < n_runs; ++i) {
    const int32_t len = (runs.where[i] & 15) + 1;
    CHECK(runs.slot[i] % 16 + len <= 16);
    for (int32_t j = 0; j < len; ++j)
      g_moves.push_back({runs.slot[i] + j, ((char*)k - g_rows_k) / 512 + (runs.where[i] >> 4) + j});
  }
  return hipSuccess;
}
hipError_t launch_attention_work8(const AttnArgs8& a, hipStream_t, hipEvent_t, hipEvent_t) {
  ++g_work8;
  CHECK(a.scales && !a.k_new && !a.v_new);
  return hipSuccess;
}
hipError_t launch_merge8(const AttnArgs8& a, hipStream_t, hipEvent_t, hipEvent_t) {
  ++g_merge8;
  g_parts = a.max_parts;
  return hipSuccess;
}
hipError_t launch_rotary_append(const RotaryAppendArgs& a, hipStream_t) {
  ++g_rotary;
  g_rotary_args = a;
  return hipSuccess;
}
}  // namespace oxy

int main() {
  std::mt19937 rng(7);
  auto upto = [&](int n) { return (int)(rng() % (unsigned)n); };
  for (const int32_t blocks : {700, 4200, 66000}) {
    oxy_pool_config c;
    memset(&c, 0, sizeof(c));
    c.n_layers = 2, c.n_q_heads = 8, c.n_kv_heads = 1, c.head_dim = 256, c.page_size = 16, c.num_blocks = blocks;
    c.max_q_tokens = 64, c.max_append_tokens = 64, c.flags = OXY_POOL_KV_FP8;
    std::vector<int32_t> order(blocks);
    for (int i = 0; i < blocks; ++i) order[i] = i;
    for (int i = blocks - 1; i > 0; --i) std::swap(order[i], order[upto(i + 1)]);
    c.free_order = order.data();
    c.kv_bytes = oxy_kv_bytes(&c);
    c.workspace_bytes = oxy_workspace_bytes(&c);
    CHECK(c.kv_bytes == 2 * (((size_t)blocks * 8224 + 255) / 256 * 256));
    c.kv_base = (void*)((uintptr_t)1 << 40);   // never touched
    c.workspace = aligned_alloc(256, (c.workspace_bytes + 255) / 256 * 256);
    oxy_pool* p = nullptr;
    CHECK(oxy_pool_create(&c, &p) == OXY_OK);
    static char rows[1];   // addresses only
    g_rows_k = rows, g_rows_v = rows + ((size_t)1 << 33);
    int32_t pid = 0;
    CHECK(oxy_prefix_create(p, &pid) == OXY_OK);
    int32_t len = 0;
    std::vector<int64_t> slot_of;
    while (len < 16 * blocks / 2 && len < 60000) {
      const int32_t most = upto(4) == 0 ? 40000 : 700, n = std::min(1 + upto(most), 16 * blocks / 2 + 40 - len);
      g_moves.clear(), g_launches = 0;
      CHECK(oxy_prefix_append_layers(p, pid, 0, 2, g_rows_k, g_rows_v, (size_t)n * 512, n, len, nullptr) == OXY_OK);
      std::vector<int32_t> table(blocks);
      CHECK(oxy_prefix_blocks(p, pid, table.data(), blocks) == OXY_OK);
      CHECK((int)g_moves.size() == n && g_layers == 2);
      for (int i = 0; i < n; ++i) {
        const int64_t slot = (int64_t)table[(len + i) / 16] * 16 + (len + i) % 16;
        CHECK(g_moves[i].slot == slot && g_moves[i].row == i);
        slot_of.push_back(slot);
      }
      CHECK(g_launches <= 1 + (n + 31) / (16 * oxy::max_table_blocks(blocks <= 65536)));
      len += n;
    }
    for (int rep = 0; rep < 60; ++rep) {
      std::vector<int64_t> want;
      const int pieces = 1 + upto(5);
      for (int k = 0; k < pieces; ++k) {
        const int from = upto(len), n = 1 + upto(std::min(len - from, upto(3) ? 900 : 50000));
        switch (upto(4)) {
          case 0: for (int i = 0; i < n; ++i) want.push_back(slot_of[upto(len)]); break;
          case 1: for (int i = n - 1; i >= 0; --i) want.push_back(slot_of[from + i]); break;
          default: want.insert(want.end(), slot_of.begin() + from, slot_of.begin() + from + n);
        }
      }
      g_moves.clear(), g_launches = 0;
      CHECK(oxy_gather_kv_layers(p, 0, 2, want.data(), (int32_t)want.size(), (void*)g_rows_k, (void*)g_rows_v,
                                 want.size() * 512, nullptr) == OXY_OK);
      CHECK(g_moves.size() == want.size() && g_layers == 2);
      for (size_t i = 0; i < want.size(); ++i) CHECK(g_moves[i].slot == want[i] && g_moves[i].row == (int64_t)i);
    }
    {   // the whole prefix: as many launches as its ids need
      g_moves.clear(), g_launches = 0;
      CHECK(oxy_gather_kv(p, 1, slot_of.data(), len, (void*)g_rows_k, (void*)g_rows_v, nullptr) == OXY_OK);
      const int most = oxy::max_table_blocks(blocks <= 65536);
      CHECK(g_launches == ((len + 15) / 16 + most - 1) / most && g_layers == 1);
    }
    // a step: three launches a layer, whatever the flags ask for
    int32_t sid = 0;
    CHECK(oxy_stream_create(p, pid, OXY_KIND_DECODE, &sid) == OXY_OK);
    oxy_item item = {sid, 3};
    oxy_batch* b = nullptr;
    int32_t rc = oxy_batch_build(p, &item, 1, 0, nullptr, &b);
    if (rc == OXY_OK) {
      for (int flags : {0, (int)OXY_STEP_FOLD_APPEND, (int)OXY_STEP_FUSE_ACROSS_LAYERS}) {
        g_append8 = g_work8 = g_merge8 = 0;
        CHECK(oxy_step_layers(p, b, 0, 2, rows, rows, 0, rows, rows, 0, nullptr, 0, 1.f, flags, nullptr, nullptr) == OXY_OK);
        CHECK(g_append8 == 2 && g_work8 == 2 && g_merge8 == 2 && g_parts > 0);
      }
      const double* f = (const double*)rows;
      oxy_rotary_config r = {64, OXY_ROTARY_PAIRS, f, 1.0};
      void *a = (void*)((uintptr_t)1 << 30), *out = (char*)a + 65536;
      g_rotary = 0;
      CHECK(oxy_rotary_append(p, b, 1, &r, (const int32_t*)a, a, 5120, out, a, 5120, a, 5120, nullptr) == OXY_OK && g_rotary == 1);
      CHECK(g_rotary_args.n_tokens == 3 && g_rotary_args.scales && g_rotary_args.q_stride == 5120 && g_rotary_args.rotary.pairs);
      CHECK((char*)g_rotary_args.layer_base == (char*)c.kv_base + c.kv_bytes / 2);
      CHECK(oxy_rotary_append(p, b, 1, &r, (const int32_t*)a, a, (size_t)1 << 32, out, a, 5120, a, 5120, nullptr) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_rotary_append(p, b, 1, &r, (const int32_t*)a, a, 5120, a, a, 5120, a, 5120, nullptr) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_rotary_append(p, b, 1, &r, (const int32_t*)a, nullptr, 0, nullptr, a, 512, a, 512, nullptr) == OXY_OK && g_rotary == 2);
      CHECK(oxy_rotary_append(p, b, 1, &r, (const int32_t*)a, a, 4096, a, a, 5120, a, 5120, nullptr) == OXY_OK && g_rotary == 3);
      CHECK(oxy_gather_kv_layers(p, 0, 2, slot_of.data(), 3, rows, rows, 1544, nullptr) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_batch_destroy(b) == OXY_OK);
    }
    CHECK(oxy_pool_destroy(p) == OXY_OK);
    free(c.workspace);
  }
  printf("OK\n");
  return 0;
}
