// Batches of forks on pools that hold exactly the blocks which they need: every page of every record is found, whatever the
// tree of forks; what has no room is refused and changes nothing.
#include "../../include/oxy.h"
#include "../../paper_2603_14371_amd/csrc/oxy_prefill.h"

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#define CHECK(x)                                              \
  do {                                                        \
    if (!(x)) {                                               \
      printf("FAILED %s:%d: %s (%s)\n", __FILE__, __LINE__, #x, oxy_last_error()); \
      exit(1);                                                \
    }                                                         \
  } while (0)

using namespace oxy;
static PrefillArgs g_args;
namespace oxy {
hipError_t launch_prefill(const PrefillArgs& a, hipStream_t) {
  g_args = a;
  return hipSuccess;
}
}  // namespace oxy

static std::mt19937 rng(5);
static int upto(int n) { return (int)(rng() % (unsigned)n); }

// A node: behind its parent's first `at` pages, `more` pages of its own, and new tokens if it is listed.
struct Node {
  int parent, at, more, n_new;
};

// Returns whether the batch was built.
static bool run(const std::vector<Node>& nodes, int work_items, int q_tokens, int spare = 0) {
  int blocks = spare;
  std::vector<int> pages(nodes.size());
  for (size_t i = 0; i < nodes.size(); ++i) {
    pages[i] = (nodes[i].parent < 0 ? 0 : nodes[i].at) + nodes[i].more;
    blocks += nodes[i].more + (nodes[i].n_new + 15) / 16;
  }
  std::vector<int32_t> order(blocks);
  for (int i = 0; i < blocks; ++i) order[i] = i;
  std::shuffle(order.begin(), order.end(), rng);
  char* const rows = (char*)((uintptr_t)1 << 40);   // addresses only
  oxy_pool_config c;
  memset(&c, 0, sizeof(c));
  c.n_layers = 1, c.n_q_heads = 8, c.n_kv_heads = 1, c.head_dim = 256, c.page_size = 16, c.num_blocks = blocks;
  c.max_q_tokens = c.max_append_tokens = q_tokens, c.max_work_items = work_items, c.free_order = order.data();
  c.kv_base = rows, c.kv_bytes = oxy_kv_bytes(&c), c.workspace_bytes = oxy_workspace_bytes(&c);
  c.workspace = aligned_alloc(256, (c.workspace_bytes + 255) / 256 * 256);
  oxy_pool* p = nullptr;
  CHECK(oxy_pool_create(&c, &p) == OXY_OK);
  std::vector<int32_t> ids(nodes.size());
  std::vector<oxy_prefix_item> ask;
  std::vector<int> item;
  for (size_t i = 0; i < nodes.size(); ++i) {
    const Node& n = nodes[i];
    if (n.parent < 0)
      CHECK(oxy_prefix_create(p, &ids[i]) == OXY_OK);
    else
      CHECK(oxy_prefix_fork(p, ids[n.parent], n.at * 16, &ids[i]) == OXY_OK);
    if (n.more) CHECK(oxy_prefix_append(p, ids[i], 0, rows, rows, n.more * 16, (pages[i] - n.more) * 16, nullptr) == OXY_OK);
  }
  for (size_t i = 0; i < nodes.size(); ++i)
    if (nodes[i].n_new) {
      ask.push_back({ids[i], nodes[i].n_new, upto(2) ? 0 : pages[i] * 16 + nodes[i].n_new});
      item.push_back((int)i);
    }
  for (size_t i = ask.size(); i > 1; --i) {
    const int j = upto((int)i);
    std::swap(ask[i - 1], ask[j]), std::swap(item[i - 1], item[j]);
  }
  int32_t free0, free1, x, y;
  CHECK(oxy_pool_stats(p, &free0, &x, &y) == OXY_OK);
  oxy_batch* b = nullptr;
  const int32_t status = oxy_prefix_batch_build(p, ask.data(), (int)ask.size(), 0, nullptr, &b);
  CHECK(status == OXY_OK || (status == OXY_ERR_WORKSPACE && !b));
  if (status != OXY_OK) {
    CHECK(oxy_pool_stats(p, &free1, &x, &y) == OXY_OK && free0 == free1);
    for (size_t k = 0; k < ask.size(); ++k) {
      int32_t len;
      CHECK(oxy_prefix_info(p, ask[k].prefix_id, &len, nullptr, nullptr, nullptr) == OXY_OK && len == pages[item[k]] * 16);
    }
  } else {
    CHECK(oxy_prefix_attention(p, b, 0, rows, 4096, rows, 4096, nullptr, 1.f, nullptr) == OXY_OK);
    std::vector<std::vector<int32_t>> tables(ask.size());
    std::vector<int> item_of;
    for (size_t k = 0; k < ask.size(); ++k) {
      tables[k].resize(pages[item[k]] + (ask[k].n_new + 15) / 16);
      CHECK(oxy_prefix_blocks(p, ask[k].prefix_id, tables[k].data(), (int)tables[k].size()) == OXY_OK);
      item_of.insert(item_of.end(), ask[k].n_new, (int)k);
    }
    std::vector<char> seen(ask.size(), 0);
    for (int w = 0; w < g_args.n_work; ++w) {
      const int32_t* r = g_args.work + (size_t)w * kPrefillWords;
      const std::vector<int32_t>& t = tables[item_of[r[F_TOK0]]];
      seen[item_of[r[F_TOK0]]] = 1;
      const int last = (r[F_LEN] - 1) / 16;
      CHECK(last + 1 == (int)t.size());
      for (int page = r[F_BEGIN] / 16; page <= last; ++page)
        CHECK(g_args.tables[page + (page < r[F_HEAD] ? r[F_SRC] : r[F_OWN])] == t[page]);
      for (int i = 0; i < kPrefillPages; ++i) CHECK(r[F_PAGES + i] == t[std::min(r[F_BEGIN] / 16 + i, last)]);
    }
    for (const char s : seen) CHECK(s);
    CHECK(oxy_batch_destroy(b) == OXY_OK);
  }
  for (const int32_t id : ids) CHECK(oxy_prefix_release(p, id) == OXY_OK);
  CHECK(oxy_pool_stats(p, &free1, &x, &y) == OXY_OK && free1 == blocks);
  CHECK(oxy_pool_destroy(p) == OXY_OK);
  free(c.workspace);
  return status == OXY_OK;
}

int main() {
  // forks of one history: always, with no more work items than there are tiles of tokens
  struct { int forks, pages, n_new; } stars[] = {{4, 36, 256}, {8, 128, 16}, {16, 512, 16}, {64, 300, 1}, {200, 60, 3}, {2, 1, 700}, {5, 7, 200}};
  for (const auto& s : stars)
    for (const bool parent_too : {false, true}) {
      std::vector<Node> n = {{-1, 0, s.pages, parent_too ? 5 : 0}};
      for (int i = 0; i < s.forks; ++i) n.push_back({0, s.pages, 0, s.n_new});
      CHECK(run(n, s.forks * ((s.n_new + 15) / 16) + 1, s.forks * s.n_new + 16));
      for (size_t i = 1; i < n.size(); ++i) n[i].more = upto(9), n[i].n_new = 1 + upto(s.n_new);
      CHECK(run(n, s.forks * ((s.n_new + 15) / 16) + 1, s.forks * s.n_new + 16));
    }
  // a chain, each behind the one before; two histories; a history forked at different places
  for (const int depth : {3, 20, 200}) {
    std::vector<Node> n = {{-1, 0, 30, 1}};
    for (int i = 1; i < depth; ++i) n.push_back({i - 1, 30 + 3 * (i - 1), 3, 1 + upto(20)});
    CHECK(run(n, depth * 2, depth * 20));
  }
  {
    std::vector<Node> n = {{-1, 0, 300, 0}, {-1, 0, 200, 3}};
    for (int i = 0; i < 24; ++i) n.push_back({i & 1, i & 1 ? 200 : 300, upto(3), 1 + upto(30)});
    for (int i = 0; i < 24; ++i) n.push_back({0, 1 + upto(300), upto(2), 1 + upto(30)});
    CHECK(run(n, 4000, 2000));
  }
  // trees of two branches a node, all pages in it
  for (const int levels : {3, 5, 7}) {
    std::vector<Node> n = {{-1, 0, 16, 0}};
    for (int at = 0, l = 1; l <= levels; ++l)
      for (const int end = (int)n.size(); at < end; ++at)
        for (int k = 0; k < 2; ++k) n.push_back({at, 16 * l, 16, l == levels ? 1 + upto(16) : 0});
    CHECK(run(n, 1 << levels, 16 << levels));
  }
  // any tree; few of them have no room
  int built = 0;
  for (int round = 0; round < 90; ++round) {
    std::vector<Node> n = {{-1, 0, 1 + upto(200), upto(2) * upto(50)}};
    std::vector<int> pages = {n[0].more};
    const int count = 2 + upto(40);
    for (int i = 1; i < count; ++i) {
      const int parent = upto(i), at = upto(3) ? pages[parent] : upto(pages[parent] + 1);
      n.push_back({parent, at, upto(30), upto(3) ? 1 + upto(upto(2) ? 2 : 60) : 0});
      pages.push_back(at + n.back().more);
    }
    n.back().n_new += 1;
    built += run(n, upto(2) ? 256 : 4000, 3000, upto(20));
  }
  CHECK(built >= 88);
  // 1024 forks of forks in a descriptor for as many records: refused, or every page is found
  {
    std::vector<Node> n = {{-1, 0, 64, 0}};
    for (int at = 0, l = 1; l <= 10; ++l)
      for (const int end = (int)n.size(); at < end; ++at)
        for (int k = 0; k < 2; ++k) n.push_back({at, 64 * l, 64, l == 10 ? 1 : 0});
    run(n, 1 << 10, 1 << 10);
  }
  printf("OK\n");
  return 0;
}
