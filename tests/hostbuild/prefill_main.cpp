// Host paths of a prefill: the work list of every launch is taken apart, and every (query token, key) pair has to lie in
// exactly one record, every split result in one merge, every page in its table.  Refusals and failing uploads change nothing.
#include "../../include/oxy.h"
#include "../../paper_2603_14371_amd/csrc/oxy_prefill.h"

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <vector>

#define CHECK(x)                                              \
  do {                                                        \
    if (!(x)) {                                               \
      printf("FAILED %s:%d: %s (%s)\n", __FILE__, __LINE__, #x, oxy_last_error()); \
      exit(1);                                                \
    }                                                         \
  } while (0)

extern "C" void oxy_stub_fail_next(int skip, int k);
using namespace oxy;

static PrefillArgs g_args;
static int g_launches = 0;
namespace oxy {
hipError_t launch_prefill(const PrefillArgs& a, hipStream_t) {
  g_args = a;
  ++g_launches;
  return hipSuccess;
}
}  // namespace oxy

struct Item {
  int past, n, full, len;
  std::vector<int32_t> blocks;   // empty: a prompt
};

static void check_work(const std::vector<Item>& items, int n_partials) {
  const PrefillArgs& a = g_args;
  std::vector<int> item_of, first_of;
  int n_tok = 0;
  for (size_t i = 0; i < items.size(); ++i) {
    first_of.push_back(n_tok);
    item_of.insert(item_of.end(), items[i].n, (int)i);
    n_tok += items[i].n;
  }
  std::map<int, std::vector<std::pair<int, int>>> ranges;      // of each token
  std::vector<int> parts(n_partials, -1);
  std::vector<int> n_parts(n_tok, 0);
  for (int w = 0; w < a.n_work; ++w) {
    const int32_t* r = a.work + (size_t)w * kPrefillWords;
    CHECK(r[F_N_TOK] >= 1 && r[F_N_TOK] <= kPrefillTokens && r[F_TOK0] >= 0 && r[F_TOK0] + r[F_N_TOK] <= n_tok);
    const int i = item_of[r[F_TOK0]];
    const Item& it = items[i];
    CHECK(item_of[r[F_TOK0] + r[F_N_TOK] - 1] == i);
    CHECK(r[F_POS] == it.past + r[F_TOK0] - first_of[i] && r[F_LEN] == it.len && r[F_FULL] == std::min(it.full, it.len));
    CHECK(r[F_BEGIN] % 16 == 0 && r[F_BEGIN] < r[F_END] && r[F_END] <= it.len);
    if (it.blocks.empty())
      CHECK(r[F_SRC] == first_of[i]);
    else
      for (size_t k = 0; k < it.blocks.size(); ++k) CHECK(a.tables[r[F_SRC] + k] == it.blocks[k]);
    for (int t = 0; t < r[F_N_TOK]; ++t) {
      ranges[r[F_TOK0] + t].push_back({r[F_BEGIN], r[F_END]});
      if (r[F_PART] < 0) continue;
      const int part = r[F_PART] + t * r[F_N_PARTS];
      CHECK(part >= 0 && part < n_partials && parts[part] == -1);
      parts[part] = r[F_TOK0] + t;
      ++n_parts[r[F_TOK0] + t];
    }
  }
  for (int t = 0; t < n_tok; ++t) {
    const Item& it = items[item_of[t]];
    const int pos = it.past + t - first_of[item_of[t]], sees = std::min(it.len, std::max(pos + 1, it.full));
    auto& v = ranges[t];
    std::sort(v.begin(), v.end());
    CHECK(!v.empty() && v[0].first == 0 && v.back().second >= sees);
    for (size_t k = 1; k < v.size(); ++k) CHECK(v[k].first == v[k - 1].second && v[k].first % 32 == 0);
    CHECK(n_parts[t] == (v.size() > 1 ? (int)v.size() : 0));
  }
  int merged = 0;
  std::vector<char> once(n_tok, 0);
  for (int m = 0; m < a.n_merge; ++m) {
    const int32_t* r = a.merges + (size_t)m * kMergeWords;
    CHECK(r[0] >= 0 && r[0] < n_tok && !once[r[0]] && r[2] == n_parts[r[0]] && r[2] > 1);
    CHECK((m < a.n_long) == (r[2] > kMergeLong));
    once[r[0]] = 1;
    for (int k = 0; k < r[2]; ++k) CHECK(parts[r[1] + k] == r[0]);
    merged += r[2];
  }
  CHECK(merged == n_partials && a.n_long >= 0 && a.n_long <= a.n_merge);
  for (int p : parts) CHECK(p >= 0);
}

static std::vector<int32_t> state(oxy_pool* p, int blocks) {
  int32_t n_free, a, b;
  CHECK(oxy_pool_stats(p, &n_free, &a, &b) == OXY_OK);
  std::vector<int32_t> v(blocks), f(n_free + 1);
  CHECK(oxy_block_refcounts(p, v.data(), blocks) == OXY_OK && oxy_free_blocks(p, f.data(), n_free + 1) == OXY_OK);
  v.insert(v.end(), f.begin(), f.end() - 1);
  return v;
}

int main() {
  std::mt19937 rng(11);
  auto upto = [&](int n) { return (int)(rng() % (unsigned)n); };
  char* const rows = (char*)((uintptr_t)1 << 40);   // addresses only
  for (int round = 0; round < 160; ++round) {
    const bool big = round % 16 == 0;
    const int blocks = big ? 5000 : 400;
    oxy_pool_config c;
    memset(&c, 0, sizeof(c));
    c.n_layers = 2, c.n_q_heads = 8, c.n_kv_heads = 1, c.head_dim = 256, c.page_size = 16, c.num_blocks = blocks;
    c.max_q_tokens = big ? 20000 : 4000, c.max_append_tokens = c.max_q_tokens;
    c.max_partials = upto(3) == 0 ? 1 + upto(500) : 0;
    c.max_work_items = upto(4) == 0 ? 2000 : 0;
    c.kv_bytes = oxy_kv_bytes(&c), c.workspace_bytes = oxy_workspace_bytes(&c);
    const int asked = c.max_partials ? c.max_partials : 32 * c.max_q_tokens;
    int room = std::max(kPrefillPartials, asked);
    if (room > asked && round % 2) {   // a workspace of max_partials split results, with or without bytes that are not enough for more
      const size_t per_batch = (size_t)(room - asked) * 4096 + (room * 128 - (asked * 128 + 255) / 256 * 256);
      c.workspace_bytes -= 2 * per_batch + 1;
      c.workspace = rows;
      oxy_pool* none = nullptr;
      CHECK(oxy_pool_create(&c, &none) == OXY_ERR_INVALID_ARG && !none);
      c.workspace_bytes += round % 4 == 1 ? 1 : 2 * per_batch;
      room = asked;
    }
    c.kv_base = rows;
    c.workspace = aligned_alloc(256, (c.workspace_bytes + 255) / 256 * 256);
    oxy_pool* p = nullptr;
    CHECK(oxy_pool_create(&c, &p) == OXY_OK);
    for (int rep = 0; rep < 6; ++rep) {
      // prefixes of some length, forks among them
      std::vector<oxy_prefix_item> ask;
      std::vector<Item> items;
      const int n_items = 1 + upto(6);
      int left = blocks * 16 / 2;
      for (int i = 0; i < n_items && left > 64; ++i) {
        int32_t pid;
        int past = upto(3) ? upto(std::min(left / 2, big ? 30000 : 900)) : 0;
        if (!ask.empty() && upto(3) == 0) {
          int32_t len;
          CHECK(oxy_prefix_info(p, ask[0].prefix_id, &len, nullptr, nullptr, nullptr) == OXY_OK);
          past = len / 16 * 16;
          CHECK(oxy_prefix_fork(p, ask[0].prefix_id, past, &pid) == OXY_OK);
        } else {
          CHECK(oxy_prefix_create(p, &pid) == OXY_OK);
          if (past) CHECK(oxy_prefix_append(p, pid, 0, rows, rows, past, 0, nullptr) == OXY_OK);
        }
        const int n = 1 + upto(upto(2) ? 40 : std::min(big ? 4000 : 600, left / 2));
        left -= past + n + 32;
        ask.push_back({pid, n, upto(3) ? upto(past + n + 50) : 0});
        items.push_back({past, n, ask.back().n_full, past + n, {}});
      }
      const auto before = state(p, blocks);
      int32_t len0;
      oxy_prefix_info(p, ask[0].prefix_id, &len0, nullptr, nullptr, nullptr);
      oxy_batch* b = nullptr;
      oxy_stub_fail_next(0, 1);
      CHECK(oxy_prefix_batch_build(p, ask.data(), (int)ask.size(), 0, nullptr, &b) == OXY_ERR_DEVICE && !b);
      oxy_stub_fail_next(0, 0);
      int32_t len1;
      oxy_prefix_info(p, ask[0].prefix_id, &len1, nullptr, nullptr, nullptr);
      CHECK(state(p, blocks) == before && len0 == len1);
      CHECK(oxy_prefix_batch_build(p, ask.data(), (int)ask.size(), 0, nullptr, &b) == OXY_OK);
      int32_t n_tok, n_work, n_part;
      CHECK(oxy_batch_info(b, nullptr, &n_tok, &n_work, &n_part) == OXY_OK);
      CHECK(n_part <= room);
      std::vector<int64_t> slots(n_tok);
      CHECK(oxy_batch_slots(b, slots.data(), n_tok) == OXY_OK);
      size_t at = 0;
      for (size_t i = 0; i < items.size(); ++i) {
        int32_t len, nb;
        CHECK(oxy_prefix_info(p, ask[i].prefix_id, &len, &nb, nullptr, nullptr) == OXY_OK && len == items[i].len);
        items[i].blocks.resize(nb);
        CHECK(oxy_prefix_blocks(p, ask[i].prefix_id, items[i].blocks.data(), nb) == OXY_OK && nb == (len + 15) / 16);
        for (int t = items[i].past; t < len; ++t) CHECK(slots[at++] == (int64_t)items[i].blocks[t / 16] * 16 + t % 16);
      }
      g_launches = 0;
      CHECK(oxy_prefix_attention(p, b, 1, rows, 5120, rows, 4096, nullptr, 1.f, nullptr) == OXY_OK && g_launches == 1);
      CHECK(g_args.n_work == n_work && g_args.layer_base == rows + c.kv_bytes / 2 && g_args.q_stride == 5120);
      check_work(items, n_part);
      int32_t out[64];
      CHECK(oxy_mixed_attention(p, b, 0, rows, rows, nullptr, 1.f, nullptr) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_mixed_attention_static(p, b, 0, rows, rows, nullptr, 1.f, nullptr) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_append_attention(p, b, 0, rows, rows, rows, rows, nullptr, 1.f, nullptr) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_step_layers(p, b, 0, 2, rows, rows, 0, rows, rows, 0, nullptr, 0, 1.f, OXY_STEP_GRAPH, nullptr, nullptr) ==
            OXY_ERR_INVALID_ARG);
      CHECK(oxy_batch_work(b, out, 1 << 30) == OXY_ERR_INVALID_ARG && oxy_batch_records(b, nullptr, 0, out) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_prompt_attention(p, b, rows, 4096, rows, 512, rows, 512, rows, 4096, nullptr, 1.f, nullptr) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_stream_append(p, b, 0, rows, rows, nullptr) == OXY_OK);
      CHECK(oxy_batch_destroy(b) == OXY_OK);
      for (auto& x : ask) CHECK(oxy_prefix_release(p, x.prefix_id) == OXY_OK);

      std::vector<oxy_prompt> prompts;
      items.clear();
      int total = 0;
      for (int i = 0, n = 1 + upto(8); i < n; ++i) {
        const int m = std::min(upto(3) ? upto(50) : upto(big ? 9000 : 900), c.max_q_tokens - total);
        total += m;
        prompts.push_back({m, upto(2) ? 0 : upto(m + 20)});
        items.push_back({0, m, prompts.back().n_full, m, {}});
      }
      CHECK(oxy_prompt_batch_build(p, prompts.data(), (int)prompts.size(), nullptr, &b) == OXY_OK);
      CHECK(oxy_batch_info(b, nullptr, &n_tok, &n_work, &n_part) == OXY_OK && n_tok == total && n_part <= room);
      g_launches = 0;
      CHECK(oxy_prompt_attention(p, b, rows, 5120, rows, 512, rows, 640, rows, 4096, nullptr, 1.f, nullptr) == OXY_OK);
      CHECK(g_launches == (total > 0));
      if (total) check_work(items, n_part);
      for (size_t bad : {(size_t)504, (size_t)520, (size_t)1 << 31})
        for (int which = 0; which < 2 && total > 1; ++which)
          CHECK(oxy_prompt_attention(p, b, rows, 4096, rows, which ? 512 : bad, rows, which ? bad : 512, rows, 4096, nullptr, 1.f,
                                     nullptr) == OXY_ERR_INVALID_ARG);
      for (size_t bad : {(size_t)4080, (size_t)4100})
        for (int which = 0; which < 2 && total > 1; ++which)
          CHECK(oxy_prompt_attention(p, b, rows, which ? 4096 : bad, rows, 512, rows, 512, rows, which ? bad : 4096, nullptr, 1.f,
                                     nullptr) == OXY_ERR_INVALID_ARG);
      if (total)
        CHECK(oxy_prompt_attention(p, b, rows + 8, 4096, rows, 512, rows, 512, rows, 4096, nullptr, 1.f, nullptr) == OXY_ERR_INVALID_ARG &&
              oxy_prompt_attention(p, b, nullptr, 4096, rows, 512, rows, 512, rows, 4096, nullptr, 1.f, nullptr) == OXY_ERR_INVALID_ARG &&
              oxy_prompt_attention(p, b, rows, 4096, rows, 512, nullptr, 512, rows, 4096, nullptr, 1.f, nullptr) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_stream_append(p, b, 0, rows, rows, nullptr) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_batch_slots(b, slots.data(), 1 << 30) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_prefix_attention(p, b, 0, rows, 4096, rows, 4096, nullptr, 1.f, nullptr) == OXY_ERR_INVALID_ARG);
      CHECK(oxy_batch_destroy(b) == OXY_OK);
    }
    CHECK(oxy_pool_destroy(p) == OXY_OK);
    free(c.workspace);
  }
  printf("OK\n");
  return 0;
}
