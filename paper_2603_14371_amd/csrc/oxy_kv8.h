// Internal interface between the host pool and the kernels of a cache in 8 bits (oxy_kv8.hip) and of rotary positions
// (oxy_rotary.hip).  The launchers are weak: host code that is linked without these kernels refuses the calls that
// need them.
#pragma once
#include "oxy_internal.h"

#define OXY_WEAK __attribute__((weak))

namespace oxy {

constexpr int kPageBytes8 = kPage * kDim;            // one K page or one V page: a byte per element
constexpr int kBlockBytes8 = 2 * kPageBytes8;        // K page + V page of one layer
constexpr int kScaleBytes8 = 2 * kPage;              // per block: exponent bytes of its K rows, then of its V rows

// One layer of a pool in 8 bits: the blocks, then their exponent bytes.
struct Layer8 {
  char* blocks;
  uint8_t* scales;
};
inline Layer8 layer8_of(void* base, int32_t num_blocks) {
  return {(char*)base, (uint8_t*)base + (size_t)num_blocks * kBlockBytes8};
}
inline size_t layer_bytes8(int32_t num_blocks) {
  return ((size_t)num_blocks * (kBlockBytes8 + kScaleBytes8) + 255) / 256 * 256;
}

// Tokens from which on an append is made 16 a workgroup, by a kernel of its own: a recording of one is none of the other.
constexpr int kManyAppend8 = 2049;
constexpr bool many_append8(int32_t n_tokens) { return n_tokens >= kManyAppend8; }
// As launch_append and launch_gather_inline, the latter for n_layers layers that lie pool_layer_stride bytes apart
// (outputs out_layer_stride).
OXY_WEAK hipError_t launch_append8(const void* k_new, const void* v_new, const int32_t* d_slots, int32_t n_tokens,
                                   Layer8 layer, hipStream_t s);
// Consecutive tokens of one table: block i holds tokens 16i - offset .. of rows k, v (or to k_out, v_out), offset =
// the first token's place in blocks[0].  Block ids travel by value, in 16 bits where they fit (ids of up to 1920 blocks
// a launch), else in 32 (960).  n_layers layers; rows of a layer lie rows_layer_stride bytes behind the last one's.
struct Table8 {
  Layer8 layer;            // the first one
  int32_t n_layers;
  size_t pool_layer_stride, rows_layer_stride;
  bool small_ids;          // every id of the pool is below 65536
};
constexpr int32_t max_table_blocks(bool small_ids) { return small_ids ? 1920 : 960; }
OXY_WEAK hipError_t launch_append_table8(const void* k, const void* v, const Table8& t, const int32_t* blocks, int32_t offset,
                                         int32_t n_tokens, hipStream_t s);
OXY_WEAK hipError_t launch_gather_table8(void* k_out, void* v_out, const Table8& t, const int32_t* blocks, int32_t offset,
                                         int32_t n_tokens, hipStream_t s);
OXY_WEAK hipError_t launch_gather_inline8(Layer8 layer, const GatherRuns& runs, int32_t n_runs, void* k_out, void* v_out,
                                          int32_t n_layers, size_t out_layer_stride, size_t pool_layer_stride,
                                          hipStream_t s);
struct AttnArgs8 : AttnArgs {
  const uint8_t* scales;    // layer_base and scales: those of the Layer8
  int32_t max_parts;        // most split results of a token
  const int32_t* long_toks; // [n_long]: the tokens of more than kLongParts
  int32_t n_long;
};
// As launch_attention_work.
OXY_WEAK hipError_t launch_attention_work8(const AttnArgs8& a, hipStream_t s, hipEvent_t start, hipEvent_t stop);
// Merge of a pool in 8 bits: launch_merge_append's where every token has at most kLongParts split results.
constexpr int32_t kLongParts = 32;
OXY_WEAK hipError_t launch_merge8(const AttnArgs8& a, hipStream_t s, hipEvent_t start, hipEvent_t stop);

// ---- rotary positions
struct RotaryArgs {
  const double* freqs;         // [rot_dims / 2]
  const int32_t* positions;    // [n_tokens]
  double amplitude;
  int32_t rot_dims;
  int32_t pairs;               // pairs (2i, 2i + 1), else (i, i + rot_dims / 2)
};
// Rows of n_tokens tokens, n_heads each: x + token * x_stride + head * 512 -> out + token * out_stride + head * 512.
OXY_WEAK hipError_t launch_rotary(const RotaryArgs& r, const void* x, size_t x_stride, void* out, size_t out_stride,
                                  int32_t n_tokens, int32_t n_heads, hipStream_t s);
struct RotaryAppendArgs {
  RotaryArgs rotary;
  const void* q;               // null: no queries
  void* q_out;                 // [n_tokens][8][256]
  const void *k_new, *v_new;
  uint32_t q_stride, k_stride, v_stride;   // bytes from token to token
  const int32_t* d_slots;
  void* layer_base;            // of a bf16 layer, or the blocks of one in 8 bits
  uint8_t* scales;             // null: bf16
  int32_t n_tokens;
};
OXY_WEAK hipError_t launch_rotary_append(const RotaryAppendArgs& a, hipStream_t s);

}  // namespace oxy
