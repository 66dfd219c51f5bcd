// HIP kernels for gfx950 (MI355X) of a cache held in 8 bits: rows quantised as they are written, read back, and the
// mixed-mask paged attention over them.
//
// A row x (the key or the value of a token, 256 bf16) is held as 256 e4m3 codes and one exponent byte b:
//   b = 127 + the smallest e >= -126 with max|x| <= 448 * 2^e,  code_i = e4m3(x_i * 2^-e) to nearest even,
//   value_i = code_i * 2^e.
// A power of two costs a floating-point code nothing (its precision is relative), makes every value exactly a bf16
// number, and is what the conversions of the matrix path take as an operand.  One exponent per row, not one per page:
// rows arrive one at a time, are rewound and written anew (drafts, action chunks), and pages are shared; an exponent over
// several rows would have to grow after rows under it had been rounded, and what a history holds would depend on how it
// was cut into calls.
//
// Attention.  The work items, splits, rounds and split results are those of a bf16 cache (see oxy_kernels.hip, `attend`);
// what differs is what lies in memory: half the bytes, turned into 16-bit operands in registers, bf16 for the logits
// (queries are bf16, a value of the cache is a bf16 number) and fp16 for the sums of values (see `attend8`).  The 8-bit
// matrix instructions round their own sums to about 2^-16 of the products' 2-norm (rms 1.5e-5, up to 5e-5 with
// products of different size, measured on sums of 128), which a log-sum-exp in 32 bits would show, and queries and
// probabilities would have to be split into two and three 8-bit parts.  A conversion of two codes takes about 5 cycles
// of a wavefront: 128 of them a round of 128 keys, beside 32 matrix instructions of 16 cycles per 16 query rows.
#include "oxy_kv8_device.h"
#include "oxy_merge.h"

#include <hip/hip_ext.h>

#include <type_traits>

namespace oxy {

// ------------------------------------------------------------------------------------------
// quantised append
// ------------------------------------------------------------------------------------------
// One wavefront per token: the first half takes the key, the second the value.  Bound by the chain slot - row - largest
// element - codes, and for many tokens by the byte stores of V.
constexpr int kAppendTokens8 = 4;   // wavefronts, and tokens, of a workgroup
// From kManyAppend8 tokens on 16 a workgroup (append_many8_kernel): where the two are equal for tokens of as many requests,
// whose slots do not follow each other; histories gain from about 1300 on.  us a launch, one token a wavefront / 16 a
// workgroup (the same slots again and again, so mostly in caches): 58 tokens 2.4 / 2.85, 1336 of four requests 3.35 / 3.35,
// 1536 of 1536 3.75 / 4.4, 2048 of one 3.65 / 3.05, 2100 of 2100 4.8 / 4.65, 4096 of one 5.3 / 3.3, 16384 15.4 / 5.6, 131072
// 94.7 / 31.3 (6.4 TB/s; 36.6 where they start inside a chunk).
__global__ __launch_bounds__(64 * kAppendTokens8) void append8_kernel(const uint16_t* __restrict__ k_new,
                                                                      const uint16_t* __restrict__ v_new,
                                                                      const int32_t* __restrict__ slots,
                                                                      char* __restrict__ blocks,
                                                                      uint8_t* __restrict__ scales, const int32_t n) {
  const int tok = blockIdx.x * kAppendTokens8 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (tok >= n) return;
  const int lane = threadIdx.x & 63, c = lane & 31;
  const uint16_t* src = (lane < 32 ? k_new : v_new) + (size_t)tok * kDim;
  const Row8 r = quantise_row(*(const u32x4*)(src + 8 * c));
  const int32_t slot = slots[tok];
  char* block = blocks + (size_t)(slot >> 4) * kBlockBytes8;
  uint8_t* sc = scales + (size_t)(slot >> 4) * kScaleBytes8;
  if (lane < 32)
    store_key(r, slot & 15, block, sc, c);
  else
    store_value(r, slot & 15, block, sc, c);
}

// Rows of keys key0..key0+n-1 of one block, by one workgroup: every half wavefront quantises two K rows and two V rows;
// V is turned through LDS and goes out in whole chunks where all four keys of one are among the rows, byte by byte
// elsewhere, so that nothing else in the page is touched.
struct __align__(16) PageLds8 {
  uint8_t v[kPage][kDim + 16];   // +16: rows land in different banks
};
template <bool kWhole>
__device__ __forceinline__ void append_page8(const uint16_t* __restrict__ k_src, const uint16_t* __restrict__ v_src,
                                             const int key0, const int n, char* __restrict__ block,
                                             uint8_t* __restrict__ scales, PageLds8& sm, const int t) {
  u32x4 k[2], v[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int idx = t + 256 * i, c = idx & 31;
    const int row = kWhole ? idx >> 5 : min(max((idx >> 5) - key0, 0), n - 1);
    k[i] = *(const u32x4*)(k_src + (size_t)row * kDim + c * 8);
    v[i] = *(const u32x4*)(v_src + (size_t)row * kDim + c * 8);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int idx = t + 256 * i, key = idx >> 5, c = idx & 31;
    const Row8 rk = quantise_row(k[i]), rv = quantise_row(v[i]);
    if (kWhole || (key >= key0 && key < key0 + n)) {
      store_key(rk, key, block, scales, c);
      if (c == 0) scales[v8_scale_offset(key)] = (uint8_t)rv.exponent;
    }
    *(u32x2*)(&sm.v[key][8 * c]) = (u32x2){rv.codes[0], rv.codes[1]};
  }
  __syncthreads();
  // thread t: chunk t of the V page, four keys of dims d..d+3
  const int key4 = 4 * ((t >> 4) & 3), d = 64 * (t >> 6) + 4 * (t & 15);
  u32x4 rows;
#pragma unroll
  for (int e = 0; e < 4; ++e) rows[e] = *(const uint32_t*)(&sm.v[key4 + e][d]);
  const u32x4 out = transposed4(rows);
  char* vp = block + kPageBytes8 + t * 16;
  if (kWhole || (key0 <= key4 && key0 + n >= key4 + 4)) {
    *(u32x4*)vp = out;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (key4 + e >= key0 && key4 + e < key0 + n) {
#pragma unroll
        for (int c = 0; c < 4; ++c) vp[4 * c + e] = (char)(out[c] >> (8 * e));
      }
  }
}

// 16 tokens of any slots by one workgroup, rows as above.  Tokens that follow each other in their slots over four keys of one
// chunk leave as whole chunks of V, the others byte by byte, a byte per thread.
__global__ __launch_bounds__(256) void append_many8_kernel(const uint16_t* __restrict__ k_new,
                                                           const uint16_t* __restrict__ v_new,
                                                           const int32_t* __restrict__ slots, char* __restrict__ blocks,
                                                           uint8_t* __restrict__ scales, const int32_t n_tokens) {
  __shared__ PageLds8 sm;
  const int tok0 = blockIdx.x * 16, n = min(16, n_tokens - tok0);
  const int t = threadIdx.x, c = t & 31;
  u32x4 k[2], v[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const size_t at = (size_t)(tok0 + min((t >> 5) + 8 * i, n - 1)) * kDim + c * 8;
    k[i] = *(const u32x4*)(k_new + at);
    v[i] = *(const u32x4*)(v_new + at);
  }
  const int j16 = t & 15;
  const int slot = slots[tok0 + min(j16, n - 1)];   // of token j16, in every 16 lanes
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int j = (t >> 5) + 8 * i;
    const Row8 rk = quantise_row(k[i]), rv = quantise_row(v[i]);
    const int mine = __shfl(slot, j);
    if (j < n) {
      uint8_t* sc = scales + (size_t)(mine >> 4) * kScaleBytes8;
      store_key(rk, mine & 15, blocks + (size_t)(mine >> 4) * kBlockBytes8, sc, c);
      if (c == 0) sc[v8_scale_offset(mine & 15)] = (uint8_t)rv.exponent;
    }
    *(u32x2*)(&sm.v[j][8 * c]) = (u32x2){rv.codes[0], rv.codes[1]};
  }
  // bit j: token j + 1 has the next slot; token j starts a chunk whose other three follow it
  const int after = __shfl(slot, (j16 + 1) & 15);   // by all lanes: one that is switched off gives nothing
  const uint32_t next = (uint32_t)__ballot(j16 + 1 < n && after == slot + 1) & 0xffffu;
  const uint32_t starts = (uint32_t)__ballot((slot & 3) == 0) & next & (next >> 1) & (next >> 2);
  uint32_t rest = ((1u << n) - 1u) & ~(starts | starts << 1 | starts << 2 | starts << 3);
  __syncthreads();
  {
    const int wv = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
    uint32_t left = starts;   // the (lane >> 4)-th of at most four
    for (int i = 0; i < (lane >> 4); ++i) left &= left - 1;
    const int j = left ? __builtin_ctz(left) : 0;
    const int first = __shfl(slot, j);
    if (left) {
      u32x4 rows;
#pragma unroll
      for (int e = 0; e < 4; ++e) rows[e] = *(const uint32_t*)(&sm.v[j + e][64 * wv + 4 * (lane & 15)]);
      *(u32x4*)(blocks + (size_t)(first >> 4) * kBlockBytes8 + kPageBytes8 + v8_chunk_offset(wv, (first >> 2) & 3, lane & 15)) =
          transposed4(rows);
    }
  }
  for (; rest; rest &= rest - 1) {
    const int j = __builtin_ctz(rest), mine = __builtin_amdgcn_readlane(slot, j);
    blocks[(size_t)(mine >> 4) * kBlockBytes8 + kPageBytes8 + v8_offset(t, mine & 15)] = (char)sm.v[j][t];
  }
}

// Block ids of a launch over one table (see Table8): 3840 bytes of the 4 KiB of arguments that a launch takes.
template <class Id>
struct TableIds {
  Id v[max_table_blocks(sizeof(Id) == 2)];
};
// The rows of one workgroup: a block's, of those that the launch covers.
struct TableRows {
  int row, key0, n;   // first row, its place in the block, how many
};
__device__ __forceinline__ TableRows rows_of_block(const int i, const int offset, const int n_tokens) {
  const int lo = max(16 * i, offset), hi = min(16 * i + 16, offset + n_tokens);
  return {lo - offset, lo & 15, hi - lo};
}

// Consecutive tokens of one table (a prefix): one workgroup per block, blockIdx.y = layer.  Bound by its bytes (1024 in,
// 514 out a token): 16391 tokens in each of 6 layers 32.0 us, 4.7 TB/s; reading them back 26.0 us, 5.8 TB/s.
template <class Id>
__global__ __launch_bounds__(256) void append_table8_kernel(const char* k, const char* v, char* blocks, uint8_t* scales,
                                                            const size_t rows_layer_stride, const size_t pool_layer_stride,
                                                            const int32_t offset, const int32_t n_tokens,
                                                            const TableIds<Id> ids) {
  __shared__ PageLds8 sm;
  const TableRows r = rows_of_block(blockIdx.x, offset, n_tokens);
  const size_t blk = ids.v[blockIdx.x], at = blockIdx.y * rows_layer_stride + (size_t)r.row * (kDim * 2);
  char* block = blocks + blockIdx.y * pool_layer_stride + blk * kBlockBytes8;
  uint8_t* sc = scales + blockIdx.y * pool_layer_stride + blk * kScaleBytes8;
  if (r.n == kPage)
    append_page8<true>((const uint16_t*)(k + at), (const uint16_t*)(v + at), 0, kPage, block, sc, sm, threadIdx.x);
  else
    append_page8<false>((const uint16_t*)(k + at), (const uint16_t*)(v + at), r.key0, r.n, block, sc, sm, threadIdx.x);
}

// ------------------------------------------------------------------------------------------
// reading back
// ------------------------------------------------------------------------------------------
// two codes -> two bf16: the value has eight significant bits at most, so cutting the float is exact
__device__ __forceinline__ uint32_t values2(uint32_t codes, bool upper, float scale) {
  const f32x2 f = upper ? __builtin_amdgcn_cvt_pk_f32_fp8(codes, true) : __builtin_amdgcn_cvt_pk_f32_fp8(codes, false);
  return (__float_as_uint(f[0] * scale) >> 16) | (__float_as_uint(f[1] * scale) & 0xffff0000u);
}
__device__ __forceinline__ void store_values16(uint16_t* dst, const u32x4 codes, float scale) {
  u32x4 a, b;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    a[2 * i] = values2(codes[i], false, scale), a[2 * i + 1] = values2(codes[i], true, scale);
    b[2 * i] = values2(codes[2 + i], false, scale), b[2 * i + 1] = values2(codes[2 + i], true, scale);
  }
  ((u32x4*)dst)[0] = a;
  ((u32x4*)dst)[1] = b;
}
// len rows from key0 on of one block to rows `at` (elements) of the outputs.  The pages are read as whole chunks; V is
// turned through LDS as codes.
__device__ __forceinline__ void gather_page8(const char* __restrict__ block, const uint8_t* __restrict__ sc, const int key0,
                                             const int len, uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out,
                                             PageLds8& sm, const int t) {
  const int key4 = 4 * ((t >> 4) & 3), d = 64 * (t >> 6) + 4 * (t & 15), end = key0 + len;
  const bool wanted = key0 < key4 + 4 && end > key4;   // a key of the run in the chunk
  // row `key`, dims 16c..16c+15 of this thread
  const int key = t >> 4, c = t & 15;
  const bool mine = key >= key0 && key < end;
  u32x4 v = {0, 0, 0, 0}, k = {0, 0, 0, 0};
  uint32_t ek = 0, ev = 0;
  if (wanted) v = *(const u32x4*)(block + kPageBytes8 + t * 16);
  if (mine) {
    k = *(const u32x4*)(block + k8_chunk_offset(c >> 2, c & 3, key));
    ek = sc[k8_scale_offset(key)];
    ev = sc[v8_scale_offset(key)];
  }
  const u32x4 rows = transposed4(v);
#pragma unroll
  for (int e = 0; e < 4; ++e) *(uint32_t*)(&sm.v[key4 + e][d]) = rows[e];
  __syncthreads();
  if (mine) {
    const size_t at = (size_t)(key - key0) * kDim + 16 * c;
    store_values16(k_out + at, k, scale_of(ek));
    store_values16(v_out + at, *(const u32x4*)(&sm.v[key][16 * c]), scale_of(ev));
  }
}
// Runs of slots anywhere, one workgroup per run, blockIdx.y = layer.  Bound as an append is: 1338 tokens of 4 histories in
// 6 layers 5.2 us (12.3 MB).
__global__ __launch_bounds__(256) void gather8_kernel(const char* __restrict__ blocks, const uint8_t* __restrict__ scales,
                                                      const GatherRuns runs, uint16_t* __restrict__ k_out,
                                                      uint16_t* __restrict__ v_out, size_t out_layer_stride,
                                                      size_t pool_layer_stride) {
  __shared__ PageLds8 sm;
  const int slot = runs.slot[blockIdx.x], where = runs.where[blockIdx.x];
  const size_t at = blockIdx.y * (out_layer_stride / sizeof(uint16_t)) + (size_t)(where >> 4) * kDim;
  gather_page8(blocks + blockIdx.y * pool_layer_stride + (size_t)(slot >> 4) * kBlockBytes8,
               scales + blockIdx.y * pool_layer_stride + (size_t)(slot >> 4) * kScaleBytes8, slot & 15, (where & 15) + 1,
               k_out + at, v_out + at, sm, threadIdx.x);
}
// Consecutive tokens of one table, one workgroup per block, blockIdx.y = layer.
template <class Id>
__global__ __launch_bounds__(256) void gather_table8_kernel(const char* blocks, const uint8_t* scales, char* k_out, char* v_out,
                                                            const size_t rows_layer_stride, const size_t pool_layer_stride,
                                                            const int32_t offset, const int32_t n_tokens,
                                                            const TableIds<Id> ids) {
  __shared__ PageLds8 sm;
  const TableRows r = rows_of_block(blockIdx.x, offset, n_tokens);
  const size_t blk = ids.v[blockIdx.x], at = blockIdx.y * rows_layer_stride + (size_t)r.row * (kDim * 2);
  gather_page8(blocks + blockIdx.y * pool_layer_stride + blk * kBlockBytes8,
               scales + blockIdx.y * pool_layer_stride + blk * kScaleBytes8, r.key0, r.n, (uint16_t*)(k_out + at),
               (uint16_t*)(v_out + at), sm, threadIdx.x);
}

// ------------------------------------------------------------------------------------------
// attention work items
// ------------------------------------------------------------------------------------------
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
// largest of lanes n, n+16, n+32, n+48
__device__ __forceinline__ uint32_t rows4_largest(uint32_t x) {
  x = swap16_max(x);
  const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return larger(b[0], b[1]);
}
__device__ __forceinline__ f32x4 mfma16_f16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// eight codes (two words) times a power of two -> eight bf16, one 16-byte matrix operand
__device__ __forceinline__ u32x4 bf16_operand(const uint32_t lo, const uint32_t hi, const float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  return r;
}
// eight codes -> eight fp16 (every code is an fp16 number)
__device__ __forceinline__ u32x4 f16_operand(const uint32_t lo, const uint32_t hi) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true));
  return r;
}
// Largest of a lane's eight dot products, NaN if one is: four instructions (fmaxf, which passes over a NaN, makes every
// matrix result canonical first: eleven).  No inline assembly: the compiler does not place the wait states between a
// matrix instruction and a reader of its result for what stands in such text.
__device__ __forceinline__ float largest3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}
__device__ __forceinline__ float largest8(const f32x4 s0, const f32x4 s1) {
  return __builtin_elementwise_maximum(largest3(largest3(largest3(s0[0], s0[1], s0[2]), s0[3], s1[0]), s1[1], s1[2]), s1[3]);
}
// first `left` of four bytes
__device__ __forceinline__ uint32_t byte_mask(const int left) {
  return left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
}
constexpr int kSpread = 12;   // see `attend8`
// Exponent bytes of a set of values as one word, the largest in the low half, 255 less the smallest in the high half: 0 is
// the empty set, and the larger half of each is the union.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t span_union(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ uint32_t span_of8(const int (&b)[8]) {
  int top = b[0], low = b[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) top = max(top, b[e]), low = min(low, b[e]);
  return (uint32_t)top | (uint32_t)(255 - low) << 16;
}
__device__ __forceinline__ uint32_t rows4_span(uint32_t s) {   // of lanes n, n+16, n+32, n+48
  const auto a = __builtin_amdgcn_permlane16_swap(s, s, false, false);
  s = span_union(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(s, s, false, false);
  return span_union(b[0], b[1]);
}
__device__ __forceinline__ int span_top(uint32_t s) { return (int)(s & 0xffffu); }
__device__ __forceinline__ int span_low(uint32_t s) { return 255 - (int)(s >> 16); }
// P = 2^(sl2 * s - m) of a lane's eight dot products; what meets the value codes is P times its key's factor, as fp16.
// Returns the sum of P itself.
__device__ __forceinline__ float weights8(const f32x4 s0, const f32x4 s1, const float sl2, const float m,
                                          const float (&factor)[8], u32x4& w) {
  float p[8], sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[e] = fast_exp2(__builtin_fmaf(e < 4 ? s0[e & 3] : s1[e & 3], sl2, -m));
    sum += p[e];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_f16(p[2 * i] * factor[2 * i], p[2 * i + 1] * factor[2 * i + 1]);
  return sum;
}

// The same with a unit of the row's own: P times 2^(its key's exponent byte - unit + 7).
__device__ __forceinline__ float weights8_by_row(const f32x4 s0, const f32x4 s1, const float sl2, const float m,
                                                 const int (&vb)[8], const int unit, u32x4& w) {
  float p[8], sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[e] = fast_exp2(__builtin_fmaf(e < 4 ? s0[e & 3] : s1[e & 3], sl2, -m));
    sum += p[e];
    p[e] = __builtin_amdgcn_ldexpf(p[e], vb[e] + 7 - unit);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_f16(p[2 * i], p[2 * i + 1]);
  return sum;
}

// LDS of a work item: nothing of K and V, only what the four wavefronts exchange.
struct __align__(16) WorkLds8 {
  u32x4 q[kMaxGroups][8][64];      // query fragments, the same for all wavefronts
  u32x4 p[4 * kMaxGroups][64];     // [32-key step][group]: P of a round's keys
  float mx[kMaxGroups][16][4];     // largest logit of a row among each wavefront's keys
  float share[kMaxGroups][16][4];  // largest log2 of a weight times its value's power of two, where units go by the row
  int slot[2 * kMaxGroups];        // split result of each token
  uint32_t span[4];                // exponent bytes of each wavefront's values: see span_of8
  float ls[kMaxGroups][64][4];     // sum of a lane's P over each wavefront's keys
};

// One work item: up to 2*G query tokens against one split of a KV source, in rounds of 128 keys, as `attend` in
// oxy_kernels.hip: wavefront w takes the logits of its 32-key step and contracts all keys of the round for dims
// 64w..64w+63.  A round of 128 keys is 32 + 32 registers of codes (64 + 64 in bf16).  A K operand is converted once
// for all groups, with its rows' exponents as the conversion's scale.  A lane's eight V codes are of eight keys, so
// theirs go into P.
//
// P travels as ONE fp16 number (hi + lo bf16 in a bf16 cache: twice the products, the LDS traffic and the packing).
// A single bf16 would be too coarse (2^-8 of it at most, for queries that see few keys); fp16 has 2^-11, like the split
// results behind it, and e4m3 codes are fp16 numbers.  Its range is short, so the number is P times
// 2^(exponent - unit + 7), acc is in units of 2^(unit - 7), and the unit decides what is left of small ones:
//  - All tokens of the item see all its keys, and their exponents lie within kSpread of each other: the largest exponent so
//    far, the same for all rows.  P is at most 2^8 and at least 1 for some key of a row, so what meets the codes is at most
//    2^15, and at least 2^(7 - kSpread) for the key that adds the most: half a step of the smallest fp16 numbers is 2^-20
//    of that.  acc is rescaled when the unit grows, which a power of two does exactly.
//  - kByRow, otherwise: the row's own, by the largest P times 2^exponent among the keys that it sees.  A token's values then
//    leave no trace in the tokens before it, and a large value that has no weight none in the others.  An item finds out
//    after its first products and starts again: 10 to 33 % slower (one chunk and one request 7.0 us a layer / 8.0, eight
//    chunks on 2048 tokens 19.8 / 23.2, 64 requests and two chunks 15.2 / 20.2, 131072 tokens 15.9 / 17.4).  As a branch
//    of the other form it took the registers of all instances (256, 61 of them spilled: 7.5, 23.2, 18.9 and 16.4 without
//    ever being taken).
//
// A row's arithmetic depends on the split's keys and on whether all tokens of the item see them, not on G or on what the
// other rows hold.  Returns whether the item is done: false, by all wavefronts, where it has to be done by rows.
// kSteps: 32-key steps of a round that are loaded: 4, or 2 for a split of at most 64 keys (eight chunks and eight
// requests on 832 tokens 14.6 us a layer, so 14.3; eight causal chunks of 20 tokens 10.25 / 9.95; eight chunks on 2048
// tokens 18.7 / 18.95).
// kOnce: non-temporal page loads (see kOnceBytes; 64 requests on eight prefixes of 2048 tokens 16.35 us a layer, so 15.4;
// 256 on 32 44.1 / 41.1).
//
// What bounds it.  Small launches: the chain record - pages - logits - P - sums, 2.7 us, and the two launches themselves
// (one chunk and one request 7.0 us a layer, one request 5.8).  Chunks: eight of 50 on 2048 tokens take 19.8 us with the
// merge, of which the items are 16.3 when traced.  A SIMD issues vector instructions for 31 % of those (128 conversions and 300
// others a round) and matrix ones for 17 % (128 a round of eight tokens), which overlap little; the first loads of 512
// workgroups are 2.4 us, 15.2 MB of split results are written, and no phase taken out alone saves more than 1 us.  Seven items
// of a chunk convert the same codes.  Bytes where histories are long: 131072 tokens 15.9 us with the merge, the items alone
// 13.6 when traced, 5.0 TB/s.
// Not kept, for the same launches: a group's softmax beside another's products in program order, raised wave
// priorities, four workgroups per CU (registers spill), rounds of 256 keys.
template <int G, bool kOnce, int kSteps, bool kByRow>
__device__ __forceinline__ bool attend8(const AttnArgs8& early_args, const WorkItem& wi, WorkLds8& sm) {
  constexpr int kLate8 = 5 * 8, kRound = 4;   // steps
  AttnArgs8 a = early_args;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));   // what comes from the thread id stays inside this instance
  const int lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int h = n & 7, sub = n >> 3;
  const float ninf = -__builtin_inff();
  const float sl2 = log2_scale(a);
  const char* __restrict__ base = (const char*)a.layer_base;
  const uint8_t* __restrict__ scales = a.scales;
  const int nsteps = (wi.kv_end - wi.kv_begin + 31) >> 5;
  const int rounds = (nsteps + kRound - 1) / kRound;
  const int npg = ((wi.kv_end + 15) >> 4) - (wi.kv_begin >> 4);

  // A step is two pages, and every load is of one of them: its address is a scalar, and this lane's place in a page.
  u32x4 kr[8];            // kr[2jj+t]: K chunk jj of this lane's key of page t, this wavefront's step
  u32x4 vr[kSteps][2];    // vr[s][t]: V chunk of this wavefront's 64 dims, page t of step s of the round
  uint32_t ke[2];         // exponent of this lane's key of page t
  uint32_t ve[2];         // of the four keys of page t whose logits it receives
  const uint32_t at_k = (g * 16 + n) * 16, at_v = kPageBytes8 + v8_chunk_offset(wv, g, n);
  auto page_load = [](const char* p) {
    if constexpr (kOnce) return __builtin_nontemporal_load((const u32x4*)p);
    return *(const u32x4*)p;
  };
  // A step past the split's end re-reads a page of the split; its logits are masked and its V operands are zeros.
  auto load_k_of = [&](const int t, const int blk) {
    const uint8_t* e = scales + (size_t)(uint32_t)blk * kScaleBytes8;
    ke[t] = e[(uint32_t)n];
    ve[t] = *(const uint32_t*)(e + (uint32_t)(kPage + 4 * g));
    const char* p = base + (size_t)(uint32_t)blk * kBlockBytes8;
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) kr[2 * jj + t] = page_load(p + at_k + jj * 1024);
  };
  auto load_v_of = [&](const int s, const int t, const int blk) {
    vr[s][t] = page_load(base + (size_t)(uint32_t)blk * kBlockBytes8 + at_v);
  };
  // The block ids of the first 16 pages are in the record (no dependent load in front of the first pages), those of
  // later rounds in the block table.
  constexpr int kInlineRounds = kWorkInlinePages / (2 * kRound);
  auto load_k = [&](const int round) {
    if (round < kInlineRounds) {
      const DescPtr id = wi.rec + 16 + 2 * kRound * round + 2 * wv;
      load_k_of(0, id[0]);
      load_k_of(1, id[1]);
    } else {
      const DescPtr ids = (DescPtr)a.tables + wi.tbl_off + (wi.kv_begin >> 4);
      const int at = 2 * kRound * round + 2 * wv;
      load_k_of(0, ids[min(at, npg - 1)]);
      load_k_of(1, ids[min(at + 1, npg - 1)]);
    }
  };
  auto load_v = [&](const int round) {
    if (round < kInlineRounds) {
      const DescPtr8 id = (DescPtr8)(wi.rec + 16 + 2 * kRound * round);
#pragma unroll
      for (int i = 0; i < 2 * kSteps; ++i) load_v_of(i >> 1, i & 1, id[0][i]);
    } else {
      const DescPtr ids = (DescPtr)a.tables + wi.tbl_off + (wi.kv_begin >> 4);
#pragma unroll
      for (int i = 0; i < 2 * kSteps; ++i) load_v_of(i >> 1, i & 1, ids[min(2 * kRound * round + i, npg - 1)]);
    }
  };
  auto load_first_v = [&]() {   // with the ids that came with the record
#pragma unroll
    for (int i = 0; i < 2 * kSteps; ++i) load_v_of(i >> 1, i & 1, wi.pages[i]);
  };

  // The queries first: loads complete in order, so the barrier below waits for them only.  Fragment 2jj+i of a row holds
  // dims 64jj+16g+8i..+7, the half of a K chunk that meets it; wavefront w brings jj = w.
  int slot_req;
  {
    u32x4 qtmp[G][2];
#pragma unroll
    for (int r = 0; r < G; ++r) {
      const char* qrow = (const char*)a.q + ((size_t)token_of(wi, r, sub) * kHeads + h) * (kDim * 2);
#pragma unroll
      for (int i = 0; i < 2; ++i) qtmp[r][i] = *(const u32x4*)(qrow + wv * 128 + g * 32 + i * 16);
    }
    slot_req = request_slot<G>(a, wi, lane);
    __builtin_amdgcn_sched_barrier(0);
    auto store_q = [&]() {
      __builtin_amdgcn_sched_barrier(0);
      take_late<kLate8>(a);
#pragma unroll
      for (int r = 0; r < G; ++r)   // rows past the item's tokens are its last one's again; nothing of them is stored
#pragma unroll
        for (int i = 0; i < 2; ++i) sm.q[r][2 * wv + i][lane] = query_sign(a, qtmp[r][i]);
    };
    if (kSteps == 2 && wv >= 2) {
      ke[0] = ke[1] = ve[0] = ve[1] = 0;
      load_first_v();
      store_q();
    } else {
      load_k(0);
      load_first_v();
      store_q();
    }
  }
  if (tid < 2 * G) sm.slot[tid] = slot_req + wi.part_idx;
  __syncthreads();

  float m[G], l[G];   // reference max (scaled log2 domain) of this lane's row, and the sum of P
  f32x4 acc[G][4];    // over this wavefront's keys; acc[r][c][e] = dim 64w + 16g + 4e + c
  uint32_t span = 1;   // exponent bytes seen
  int unit[G];         // acc's unit, as an exponent byte: that of the largest value seen, or the row's own
#pragma unroll
  for (int r = 0; r < G; ++r) {
    unit[r] = 1;
    m[r] = ninf;
    l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[r][c] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  auto round_body = [&](const int round, auto last) {
    constexpr bool kLast = decltype(last)::value;
    int lane_now = tid & 63;
    asm volatile("" : "+v"(lane_now));
    const int lane = lane_now, n = lane & 15, g = lane >> 4, sub = n >> 3;
    f32x4 s0[G], s1[G];
    int vb[8];   // exponent bytes of this lane's values; of keys that are not there, those of others
    const int pos = wi.kv_begin + 32 * (kRound * round + wv);
    const int left = wi.kv_end - pos;
    const bool need_mask = (kLast && left < 32) || (kByRow && pos + 31 > wi.q0);
    if (kSteps != 2 || wv < 2) {
#pragma unroll
      for (int r = 0; r < G; ++r) s0[r] = s1[r] = (f32x4){0.f, 0.f, 0.f, 0.f};
      const float ks0 = scale_of(ke[0]), ks1 = scale_of(ke[1]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const u32x4 a0 = kr[2 * (j >> 1)], a1 = kr[2 * (j >> 1) + 1];
        const u32x4 k0 = bf16_operand(a0[2 * (j & 1)], a0[2 * (j & 1) + 1], ks0);
        const u32x4 k1 = bf16_operand(a1[2 * (j & 1)], a1[2 * (j & 1) + 1], ks1);
#pragma unroll
        for (int r = 0; r < G; ++r) {
          const u32x4 q = sm.q[r][j][lane];
          s0[r] = mfma16(k0, q, s0[r]);
          s1[r] = mfma16(k1, q, s1[r]);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) vb[e] = (int)((ve[e >> 2] >> (8 * (e & 3))) & 0xffu);
      if (need_mask) {   // wave-uniform: only the end of a split or the causal diagonal
        int k0 = pos + 4 * g;
        asm volatile("" : "+v"(k0));   // a branch: as selects the masks are a quarter of a round's instructions
#pragma unroll
        for (int r = 0; r < G; ++r) {
          const int end = (kByRow ? min(wi.kv_end, wi.q0 + 2 * r + sub + 1) : wi.kv_end) - k0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s0[r][e] = e < end ? s0[r][e] : ninf;
            s1[r][e] = 16 + e < end ? s1[r][e] : ninf;
          }
        }
        // the exponent byte of a slot that was never written may be anything
        const int there = left > 0 ? __builtin_amdgcn_readfirstlane(vb[0]) : 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) vb[e] = (e < 4 ? e : 12 + e) < wi.kv_end - k0 ? vb[e] : there;
      }
    } else {
#pragma unroll
      for (int r = 0; r < G; ++r) s0[r] = s1[r] = (f32x4){ninf, ninf, ninf, ninf};
#pragma unroll
      for (int e = 0; e < 8; ++e) vb[e] = 0;
    }
    {
      float mx[G];
#pragma unroll
      for (int r = 0; r < G; ++r) {
        mx[r] = largest8(s0[r], s1[r]) * sl2;
      }
      const float mine = row_max4_each(mx);
      if (g < G) sm.mx[g][n][wv] = mine;
      if constexpr (kByRow) {   // log2 of the largest share that a key has in its row's sums, up to its codes
#pragma unroll
        for (int r = 0; r < G; ++r) {
          f32x4 c0, c1;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            c0[e] = __builtin_fmaf(s0[r][e], sl2, (float)vb[e]);
            c1[e] = __builtin_fmaf(s1[r][e], sl2, (float)vb[4 + e]);
          }
          mx[r] = largest8(c0, c1);
        }
        const float share = row_max4_each(mx);
        if (g < G) sm.share[g][n][wv] = share;
      } else {
        const uint32_t sp = left > 0 ? rows4_span(span_of8(vb)) : 0;   // the same in all lanes of 16
        if (lane == 0) sm.span[wv] = sp;
      }
    }
    __syncthreads();
    // online softmax with a reference that only moves by more than kGrow: see `attend`
    float mx[G];
    bool grow = false;
#pragma unroll
    for (int r = 0; r < G; ++r) {
      const f32x4 mw = *(const f32x4*)sm.mx[r][n];
      mx[r] = fmaxf(fmaxf(mw[0], mw[1]), fmaxf(mw[2], mw[3]));
      grow |= mx[r] > m[r] + kGrow;
    }
    if constexpr (kByRow) {
#pragma unroll
      for (int r = 0; r < G; ++r) {
        const f32x4 cw = *(const f32x4*)sm.share[r][n];
        const float share = fmaxf(fmaxf(cw[0], cw[1]), fmaxf(cw[2], cw[3]));
        const bool up = mx[r] > m[r] + kGrow;
        const float to = up ? mx[r] : m[r];
        const float alpha = up ? fast_exp2(m[r] - to) : 1.f;
        // the unit that the sums have by the new reference, or that of a larger share
        const float want = fmaxf(share - to, up ? (float)unit[r] + (m[r] - to) : (float)unit[r]);
        const int fits = (int)ceilf(fminf(fmaxf(want, 1.f), 254.f));
        l[r] = rescaled(l[r], alpha);
        if (round > 0) {
          const float down = __builtin_amdgcn_ldexpf(alpha, unit[r] - fits);
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[r][c] *= down;
        }
        m[r] = to;
        unit[r] = fits;
      }
    } else {
      const u32x4 spans = *(const u32x4*)sm.span;
      const uint32_t seen = __builtin_amdgcn_readfirstlane(
          span_union(span, span_union(span_union(spans[0], spans[1]), span_union(spans[2], spans[3]))));
      const int top = span_top(seen);
      if (top - span_low(seen) > kSpread) return false;   // all four wavefronts
      if (top > span_top(span) && round > 0) {   // wave-uniform; acc holds zeros in the first round
        const float down = __builtin_amdgcn_ldexpf(1.f, span_top(span) - top);
#pragma unroll
        for (int r = 0; r < G; ++r)
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[r][c] *= down;
      }
      span = seen;
      if (__any(grow)) {
#pragma unroll
        for (int r = 0; r < G; ++r) {
          const bool up = mx[r] > m[r] + kGrow;
          const float alpha = up ? fast_exp2(m[r] - mx[r]) : 1.f;
          l[r] = rescaled(l[r], alpha);
          if (round > 0) {
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[r][c] *= alpha;
          }
          m[r] = up ? mx[r] : m[r];
        }
      }
    }
    // 2^(exponent - unit + 7); for a key that is not there (P is 0) something finite
    float factor[8];
    if constexpr (!kByRow) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        factor[e] = __uint_as_float((uint32_t)max((vb[e] << 23) + ((127 + 7 - span_top(span)) << 23), 0));
    }
#pragma unroll
    for (int r = 0; r < G; ++r) {
      u32x4 w;
      const float ref = (m[r] == ninf) ? 0.f : m[r];
      l[r] += kByRow ? weights8_by_row(s0[r], s1[r], sl2, ref, vb, unit[r], w) : weights8(s0[r], s1[r], sl2, ref, factor, w);
      sm.p[wv * G + r][lane] = w;
      if constexpr (kLast) sm.ls[r][lane][wv] = l[r];
    }
    __builtin_amdgcn_sched_barrier(0);   // the next K chunks reuse kr[]
    if constexpr (!kLast) load_k(round + 1);
    __builtin_amdgcn_sched_barrier(0);
    // Some rows may not see all keys: P is 0 there, and 0 times NaN is not.  Codes that are NaN become zeros, and the 64
    // dims of the rows that do see one NaN.
    if (kByRow && min(wi.kv_end, wi.kv_begin + 32 * kRound * (round + 1)) - 1 > wi.q0) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        u32x4 nan[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) nan[t] = ((vr[s][t] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;   // bit 7 of a key's byte
        const uint32_t first = nan[0][0] | nan[0][1] | nan[0][2] | nan[0][3];
        const uint32_t second = nan[1][0] | nan[1][1] | nan[1][2] | nan[1][3];
        if (__any(first | second)) {
          const uint32_t key = first    ? 4 * g + (__builtin_ctz(first) >> 3)
                               : second ? 16 + 4 * g + (__builtin_ctz(second) >> 3)
                                        : 63;
          const int lowest = 63 - (int)rows4_largest(lanes16_largest(63 - key));
          const int at = lowest + wi.kv_begin + 32 * (kRound * round + s);
#pragma unroll
          for (int t = 0; t < 2; ++t) vr[s][t] &= ~((nan[t] >> 7) * 0xffu);
#pragma unroll
          for (int r = 0; r < G; ++r)
            if (at < min(wi.kv_end, wi.q0 + 2 * r + sub + 1)) {
#pragma unroll
              for (int c = 0; c < 4; ++c) acc[r][c] *= __builtin_nanf("");
            }
        }
      }
    }
    __syncthreads();
    auto operands = [&](const int s, u32x4 (&v)[4]) {
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = f16_operand(vr[s][0][c], vr[s][1][c]);
    };
    auto contract = [&](const int s, const int r, const u32x4 (&v)[4]) {
      const u32x4 w = sm.p[s * G + r][lane];
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[r][c] = mfma16_f16(v[c], w, acc[r][c]);
    };
    if constexpr (!kLast) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        u32x4 v[4];
        operands(s, v);
#pragma unroll
        for (int r = 0; r < G; ++r) contract(s, r, v);
      }
      __builtin_amdgcn_sched_barrier(0);   // likewise vr[]
      load_v(round + 1);
      __builtin_amdgcn_sched_barrier(0);
    } else {
      const int nv = nsteps - kRound * round;   // steps with keys
      auto clear_past_end = [&](const int s) {   // codes of slots beyond the end may be anything
        const int left_s = wi.kv_end - (wi.kv_begin + 32 * (kRound * round + s));
        if (left_s < 32) {
          const uint32_t m0 = byte_mask(left_s - 4 * g), m1 = byte_mask(left_s - 16 - 4 * g);
          vr[s][0] &= (u32x4){m0, m0, m0, m0};
          vr[s][1] &= (u32x4){m1, m1, m1, m1};
        }
      };
      auto finish_group = [&](const int r) {
        const int slot = sm.slot[2 * r + sub];
        store_part<(G >= 4), true>(a, wi, slot, acc[r], r, wv, lane, (kByRow ? unit[r] : span_top(span)) - 127 - 7);
        if (wv == r) {   // wave-uniform: the sums of the groups are shared out
          const f32x4 lw = *(const f32x4*)sm.ls[r][lane];
          const float total = row_sum4((lw[0] + lw[1]) + (lw[2] + lw[3]));
          if (g == 0 && 2 * r + sub < wi.n_tok)
            // a sum that is not a number has no reference, and would pass for that of a row without visible keys
            *(f32x2*)(a.part_ml + ((size_t)slot * kHeads + (n & 7)) * 4) = (f32x2){total != total ? 0.f : m[r], total};
        }
      };
      if constexpr (G == 1) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
          if (s < nv) {
            u32x4 v[4];
            clear_past_end(s);
            operands(s, v);
            contract(s, 0, v);
          }
        finish_group(0);
      } else {
        // Group by group, so that a group's scaling and stores fall into the products of the next.  Steps without keys
        // are zeros.
        u32x4 v[kSteps][4];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          clear_past_end(s);
          operands(s, v[s]);
        }
#pragma unroll
        for (int r = 0; r < G; ++r) {
#pragma unroll
          for (int s = 0; s < kSteps; ++s) contract(s, r, v[s]);
          finish_group(r);
        }
      }
    }
    return true;
  };
  if constexpr (kSteps != 2)
    for (int round = 0; round + 1 < rounds; ++round)
      if (!round_body(round, std::false_type())) return false;
  return round_body(kSteps != 2 ? rounds - 1 : 0, std::true_type());
}

__global__ __attribute__((aligned(4096))) __launch_bounds__(256, 2) void attn8_kernel(
    const int32_t* work, const void* q, const void* layer_base, const uint8_t* scales, const int32_t part_off,
    const float scale, const LateArgs) {
  __shared__ WorkLds8 sm;
  AttnArgs8 a;
  a.q = q;
  a.layer_base = layer_base;
  a.scales = scales;
  a.part_off = work + part_off;
  a.scale = scale;
  WorkItem wi;
  int path_word;
  auto read_item = [&]() {
    wi.rec = (DescPtr)work + (size_t)blockIdx.x * kWorkWords;
    const i32x8 head = ((DescPtr8)wi.rec)[0];
    wi.toks = ((DescPtr8)wi.rec)[1];
    wi.pages = ((DescPtr8)wi.rec)[2];
    asm volatile("" ::"s"(head), "s"(wi.toks), "s"(wi.pages));
    wi.n_tok = head[W_N_TOK];
    wi.tbl_off = head[W_TBL_OFF];
    wi.kv_begin = head[W_KV_BEGIN];
    wi.kv_end = head[W_KV_END];
    wi.q0 = head[W_CAUSAL_Q0];
    wi.part_idx = head[W_PART_IDX];
    path_word = head[W_PATH];
  };
  read_item();
  if ((path_word & kPathMask) == PATH_NOOP) return;
  const bool few_keys = wi.kv_end - wi.kv_begin <= 64;
  if (wi.kv_end - 1 <= wi.q0) {   // the item's first token sees all keys, and so do the others
    bool done;
    if (wi.n_tok > 4)
      done = few_keys ? attend8<4, false, 2, false>(a, wi, sm) : attend8<4, false, 4, false>(a, wi, sm);
    else if (path_word & kPathAppends)   // one or two tokens on their own pages
      done = path_word & kPathOnce ? attend8<1, true, 4, false>(a, wi, sm) : attend8<1, false, 4, false>(a, wi, sm);
    else if (wi.n_tok <= 2)
      done = few_keys ? attend8<1, false, 2, false>(a, wi, sm) : attend8<1, false, 4, false>(a, wi, sm);
    else
      done = few_keys ? attend8<2, false, 2, false>(a, wi, sm) : attend8<2, false, 4, false>(a, wi, sm);
    if (done) return;
    read_item();   // nothing of it is kept for this
  }
  if (wi.n_tok <= 2)
    attend8<1, false, 4, true>(a, wi, sm);
  else if (wi.n_tok <= 4)
    few_keys ? attend8<2, false, 2, true>(a, wi, sm) : attend8<2, false, 4, true>(a, wi, sm);
  else
    attend8<4, false, 4, true>(a, wi, sm);
}
static_assert(Params<decltype(&attn8_kernel)>::offset_of_last() == 5 * 8, "attend8 reads the last argument there");

// ------------------------------------------------------------------------------------------
// merge of tokens with many split results
// ------------------------------------------------------------------------------------------
// A wavefront per token and head takes 0.9 us for every 16 split results behind the first (29 us for 512: two workgroups
// read 2 MB in turn).  Here a token of more than kLongParts results takes a workgroup for each head and 64 dims: eight
// wavefronts share the results out, 64 at a time with everything in flight at once, each with a maximum of its own, and the
// first one joins the eight (256 results of a history of 131072 tokens 3 us).  These workgroups come first (long_toks); behind
// them every other token is one workgroup, merged by a wavefront for each head as in every other launch, so that a token's bits
// do not depend on what else is in the batch (eight chunks of 50 on 832 tokens beside a history of 9000 15.7 us a layer, of
// 131072 26.6; with 32 workgroups for every token 23.7 and 37.1, with a wavefront a head for every token 18.0 and 46.9).  us
// per layer with a limit of 16 / 32 / 64: one history of 6000 tokens 8.3 / 8.6 / 8.9, 16 of 4000 15.1 / 13.9 / 13.9, one of
// 10000 8.6 / 8.6 / 9.8.
constexpr int kLongWaves = 8, kLongAhead = 16;   // a wavefront's loads: kLongAhead times four results of 128 bytes
__global__ __launch_bounds__(64 * kLongWaves) void merge_long_kernel(const uint16_t* part_acc, const float* part_ml, void* out,
                                                                    float* lse, const int32_t* n_parts,
                                                                    const int32_t* part_off, const int32_t* long_toks,
                                                                    const int32_t n_long) {
  static_assert(kLongWaves == kHeads, "a short token takes a wavefront for each head");
  __shared__ f32x4 os[kLongWaves][16];
  __shared__ float bigs[kLongWaves], totals[kLongWaves];
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n_first = 4 * kHeads * n_long, bid = blockIdx.x;
  const int tok = bid < n_first ? ((DescPtr)long_toks)[bid / (4 * kHeads)] : bid - n_first;
  const int np = ((DescPtr)n_parts)[tok];
  const size_t base = (size_t)((DescPtr)part_off)[tok];
  if (bid >= n_first) {   // the tokens in turn, but those above
    if (np <= kLongParts) merge_any({part_acc, part_ml, out, lse, n_parts, part_off}, base, np, tok, wv, lane);
    return;
  }
  const int h = (bid >> 2) % kHeads, part = bid & 3;
  const int i = lane & 15, p = lane >> 4;   // dims 64 * part + 4i..+3 of every fourth result
  const char* ml = (const char*)(part_ml + (base * kHeads + h) * 4);
  const char* acc = (const char*)(part_acc + (base * kHeads + h) * kDim + 64 * part + 4 * i);
  constexpr size_t kMlStride = kHeads * 4 * sizeof(float), kAccStride = kHeads * kDim * sizeof(uint16_t);
  const float ninf = -__builtin_inff();
  float big = ninf, total = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 4 * kLongAhead * wv; p0 < np; p0 += 4 * kLongAhead * kLongWaves) {
    f32x4 w[kLongAhead];
    u32x2 x[kLongAhead];
#pragma unroll
    for (int u = 0; u < kLongAhead; ++u) {
      const size_t at = min(p0 + 4 * u + p, np - 1);
      w[u] = *(const f32x4*)(ml + at * kMlStride);
      x[u] = __builtin_nontemporal_load((const u32x2*)(acc + at * kAccStride));
    }
    float top = big;
#pragma unroll
    for (int u = 0; u < kLongAhead; ++u) top = fmaxf(top, w[u][0]);
    top = row_max4(top);   // of the wavefront: every lane of 16 has the same results
    const float down = big == ninf ? 0.f : fast_exp2(big - top);
    total *= down;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] *= down;
    big = top;
#pragma unroll
    for (int u = 0; u < kLongAhead; ++u) {
      const bool live = p0 + 4 * u + p < np && w[u][0] != ninf;
      const float wgt = live ? fast_exp2(w[u][0] - big) : 0.f;
      total += wgt * (live ? w[u][1] : 0.f);
      const int ex = (int32_t)(__float_as_uint(w[u][2]) << (24 - 8 * part)) >> 24;   // signed byte `part`
      const float ws = __builtin_amdgcn_ldexpf(wgt, ex - 14);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float lo, hi;
        unpack_f16(x[u][k], lo, hi);
        o[2 * k] = __builtin_fmaf(ws, lo, o[2 * k]);
        o[2 * k + 1] = __builtin_fmaf(ws, hi, o[2 * k + 1]);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = row_sum4(o[k]);
  total = row_sum4(total);
  if (p == 0) os[wv][i] = (f32x4){o[0], o[1], o[2], o[3]};
  if (lane == 0) bigs[wv] = big, totals[wv] = total;
  __syncthreads();
  if (wv != 0) return;
  float top = bigs[0];
#pragma unroll
  for (int w = 1; w < kLongWaves; ++w) top = fmaxf(top, bigs[w]);
  float sum = 0.f;
  f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kLongWaves; ++w) {
    const float wgt = bigs[w] == ninf ? 0.f : fast_exp2(bigs[w] - top);
    sum = __builtin_fmaf(wgt, totals[w], sum);
    const f32x4 theirs = os[w][i];
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = __builtin_fmaf(wgt, theirs[k], r[k]);
  }
  const float inv = 1.f / sum;
  const u32x2 packed = {pack_bf16(r[0] * inv, r[1] * inv), pack_bf16(r[2] * inv, r[3] * inv)};
  if (p == 0) *(u32x2*)((uint16_t*)out + ((size_t)tok * kHeads + h) * kDim + 64 * part + 4 * i) = packed;
  if (lse && part == 0 && lane == 0)
    lse[(size_t)tok * kHeads + h] = (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// ------------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------------
hipError_t launch_append8(const void* k_new, const void* v_new, const int32_t* d_slots, int32_t n_tokens, Layer8 layer,
                          hipStream_t s) {
  if (n_tokens <= 0) return hipSuccess;
  if (many_append8(n_tokens))
    append_many8_kernel<<<(n_tokens + 15) / 16, 256, 0, s>>>((const uint16_t*)k_new, (const uint16_t*)v_new, d_slots,
                                                             layer.blocks, layer.scales, n_tokens);
  else
    append8_kernel<<<(n_tokens + kAppendTokens8 - 1) / kAppendTokens8, 64 * kAppendTokens8, 0, s>>>(
        (const uint16_t*)k_new, (const uint16_t*)v_new, d_slots, layer.blocks, layer.scales, n_tokens);
  return hipGetLastError();
}

namespace {
template <class Id>
TableIds<Id> table_ids(const int32_t* blocks, int32_t n) {
  TableIds<Id> ids;
  for (int32_t i = 0; i < n; ++i) ids.v[i] = (Id)blocks[i];
  return ids;
}
template <class Id>
void append_table(const void* k, const void* v, const Table8& t, const int32_t* blocks, int32_t offset, int32_t n_tokens,
                  int32_t n_blocks, hipStream_t s) {
  append_table8_kernel<Id><<<dim3(n_blocks, t.n_layers), 256, 0, s>>>(
      (const char*)k, (const char*)v, t.layer.blocks, t.layer.scales, t.rows_layer_stride, t.pool_layer_stride, offset,
      n_tokens, table_ids<Id>(blocks, n_blocks));
}
template <class Id>
void gather_table(void* k_out, void* v_out, const Table8& t, const int32_t* blocks, int32_t offset, int32_t n_tokens,
                  int32_t n_blocks, hipStream_t s) {
  gather_table8_kernel<Id><<<dim3(n_blocks, t.n_layers), 256, 0, s>>>(
      t.layer.blocks, t.layer.scales, (char*)k_out, (char*)v_out, t.rows_layer_stride, t.pool_layer_stride, offset, n_tokens,
      table_ids<Id>(blocks, n_blocks));
}
}  // namespace

hipError_t launch_append_table8(const void* k, const void* v, const Table8& t, const int32_t* blocks, int32_t offset,
                                int32_t n_tokens, hipStream_t s) {
  const int32_t n = (offset + n_tokens + kPage - 1) / kPage;
  if (n_tokens <= 0 || offset < 0 || offset >= kPage || t.n_layers <= 0 || n > max_table_blocks(t.small_ids))
    return hipErrorInvalidValue;
  t.small_ids ? append_table<uint16_t>(k, v, t, blocks, offset, n_tokens, n, s)
              : append_table<int32_t>(k, v, t, blocks, offset, n_tokens, n, s);
  return hipGetLastError();
}

hipError_t launch_gather_table8(void* k_out, void* v_out, const Table8& t, const int32_t* blocks, int32_t offset,
                                int32_t n_tokens, hipStream_t s) {
  const int32_t n = (offset + n_tokens + kPage - 1) / kPage;
  if (n_tokens <= 0 || offset < 0 || offset >= kPage || t.n_layers <= 0 || n > max_table_blocks(t.small_ids))
    return hipErrorInvalidValue;
  t.small_ids ? gather_table<uint16_t>(k_out, v_out, t, blocks, offset, n_tokens, n, s)
              : gather_table<int32_t>(k_out, v_out, t, blocks, offset, n_tokens, n, s);
  return hipGetLastError();
}

hipError_t launch_gather_inline8(Layer8 layer, const GatherRuns& runs, int32_t n_runs, void* k_out, void* v_out,
                                 int32_t n_layers, size_t out_layer_stride, size_t pool_layer_stride, hipStream_t s) {
  if (n_runs <= 0 || n_layers <= 0) return hipSuccess;
  gather8_kernel<<<dim3(n_runs, n_layers), 256, 0, s>>>(layer.blocks, layer.scales, runs, (uint16_t*)k_out, (uint16_t*)v_out,
                                                       out_layer_stride, pool_layer_stride);
  return hipGetLastError();
}

hipError_t launch_attention_work8(const AttnArgs8& a, hipStream_t s, hipEvent_t start, hipEvent_t stop) {
  if (a.n_work <= 0 || a.n_q <= 0) return hipErrorInvalidValue;
  const LateArgs late = {a.part_acc, a.part_ml, a.tables, a.write_through};
  const int32_t part_off = (int32_t)(a.part_off - a.work);   // of one descriptor
  if (start || stop)
    hipExtLaunchKernelGGL(attn8_kernel, dim3(a.n_work), dim3(256), 0, s, start, stop, 0, a.work, a.q, a.layer_base, a.scales,
                          part_off, a.scale, late);
  else
    attn8_kernel<<<a.n_work, 256, 0, s>>>(a.work, a.q, a.layer_base, a.scales, part_off, a.scale, late);
  return hipGetLastError();
}

hipError_t launch_merge8(const AttnArgs8& a, hipStream_t s, hipEvent_t start, hipEvent_t stop) {
  if (a.n_long <= 0) return launch_merge_append(a, nullptr, s, start, stop);
  if (a.n_q < a.n_long) return hipErrorInvalidValue;
  const int32_t grid = 4 * kHeads * a.n_long + (a.n_long < a.n_q ? a.n_q : 0);
  if (start || stop)
    hipExtLaunchKernelGGL(merge_long_kernel, dim3(grid), dim3(64 * kLongWaves), 0, s, start, stop, 0, a.part_acc, a.part_ml,
                          a.out, a.lse, a.n_parts, a.part_off, a.long_toks, a.n_long);
  else
    merge_long_kernel<<<grid, 64 * kLongWaves, 0, s>>>(a.part_acc, a.part_ml, a.out, a.lse, a.n_parts, a.part_off, a.long_toks,
                                                       a.n_long);
  return hipGetLastError();
}

}  // namespace oxy
