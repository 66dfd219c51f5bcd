// Internal interface between the host pool and the kernels of a prefill (oxy_prefill.hip): attention of a prefix's new
// tokens over its pages, and of whole prompts over the rows that a projection wrote.  The launchers are weak, as those of
// oxy_kv8.h are.
#pragma once
#include "oxy_internal.h"
#include "oxy_kv8.h"

namespace oxy {

// A record of the work list: query tokens of one item that lie side by side, and the keys [begin, end) of that item.
constexpr int kPrefillWords = 32;   // a line of 128 bytes
static_assert(kPrefillWords <= kWorkWords, "a descriptor has room for kWorkWords a record");
enum { F_TOK0 = 0,     // first query token: row of q, out and lse
       F_N_TOK,        // query tokens
       F_POS,          // position of the first one in its item
       F_FULL,         // a query at position p sees keys below max(p + 1, this)
       F_BEGIN, F_END, // keys of this record; F_BEGIN is a multiple of the page size
       F_SRC,          // paged: where page 0 stands in the block tables; a prompt: row of its first token
       F_PART,         // split result of the first query token, -1: the record writes the output
       F_N_PARTS,      // split results of a token: those of token t begin F_N_PARTS * t behind F_PART
       F_LEN,          // tokens of the item
       F_HEAD,         // paged: pages from here on do not stand behind F_SRC, where another item's table is, but
       F_OWN,          // page p at F_OWN + p (0 and F_SRC: a table of the item's own)
       F_PAGES = 16 }; // paged: block ids of the first kPrefillPages pages, the item's last one repeated
constexpr int kPrefillPages = 16;
constexpr int kPrefillTokens = 16;   // query tokens of a record, at most
// Split results that a workspace should have room for: two workgroups on each of 256 CUs (35 MB).
constexpr int32_t kPrefillPartials = 512 * kPrefillTokens;
constexpr int kPrefillCus = 256;
// Words of the merge list for each token that has split results: the token, its first one, how many.
constexpr int kMergeWords = 3;
// Tokens with more split results than this are first in the merge list, and a workgroup joins those of one head.
constexpr int kMergeLong = 16;

struct PrefillArgs {
  const void* q;             // token t, head h at q + t * q_stride + h * 512
  void* out;                 // likewise
  float* lse;                // [n_q][8] or null
  size_t q_stride, out_stride;
  const int32_t* work;       // [n_work][kPrefillWords]
  const int32_t* tables;     // block ids
  const int32_t* merges;     // [n_merge][kMergeWords]
  const char* layer_base;    // a layer of the pool, or the blocks of one in 8 bits; null: a prompt
  const uint8_t* scales;     // in 8 bits: the exponent bytes
  const char *k, *v;         // of a prompt: token t at k + t * k_stride
  size_t k_stride, v_stride;
  uint16_t* part_acc;        // as in AttnArgs
  float* part_ml;
  int32_t n_work, n_merge, n_long;   // n_long: tokens with more than kMergeLong split results
  float scale;
};
OXY_WEAK hipError_t launch_prefill(const PrefillArgs& a, hipStream_t s);

}  // namespace oxy
