// Device helpers that the kernels of a bf16 cache (oxy_kernels.hip) and of one in 8 bits (oxy_kv8.hip) share: MFMA and
// packing, lane exchanges, the bf16 page layout, work records, and a work item's way from logits to stored split results.
#pragma once
#include "oxy_internal.h"

#include <tuple>
#include <utility>

namespace oxy {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// two floats -> packed bf16 pair, round to nearest even (inputs are finite here)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
  const f32x2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// two floats -> packed fp16 pair (round to nearest even)
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
  const f32x2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2));
}
__device__ __forceinline__ void unpack_f16(uint32_t u, float& lo, float& hi) {
  typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
  const f16x2 h = __builtin_bit_cast(f16x2, u);
  lo = (float)h[0];
  hi = (float)h[1];
}

// max over the four lanes {n, n+16, n+32, n+48} that hold one query row: two register swaps
// between lane halves (v_permlane16_swap, v_permlane32_swap), no LDS round trip
__device__ __forceinline__ float row_max4(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const uint32_t v = __float_as_uint(y);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// The same of G values at once: lane row g gets the maximum of value g % G.  The first swap leaves two lanes' parts of
// two values in a register, the second one those of all four lanes (of four values: three swaps, not eight).  us per
// layer, one value at a time / so: six chunks on 1500 tokens 17.55 / 17.25, on 2048 18.1 / 17.9, eight on 832 16.6 / 16.5,
// 256 requests 71.6 / 71.4.
template <int G>
__device__ __forceinline__ float row_max4_each(const float (&x)[G]) {
  if constexpr (G == 1) {
    return row_max4(x[0]);
  } else {
    float y[2];
#pragma unroll
    for (int i = 0; i < G / 2; ++i) {
      const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]), false, false);
      y[i] = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    }
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y[0]), __float_as_uint(y[G == 4]), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
  }
}
// sum over the same four lanes, same two swaps: every lane adds its own value and its partner's
__device__ __forceinline__ float row_sum4(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const uint32_t v = __float_as_uint(y);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// x of the lane N places on in the row of 16 lanes
template <int N>
__device__ __forceinline__ float dpp_row_ror(const float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x120 + N, 0xf, 0xf, false));
}
// f(0), f(1), .. f(N - 1) with the index as a constant
template <int N, class F, int... I>
__device__ __forceinline__ void static_for_each(const F& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(const F& f) {
  static_for_each<N>(f, std::make_integer_sequence<int, N>());
}
// ------------------------------------------------------------------------------------------
// page layout (see oxy.h)
// ------------------------------------------------------------------------------------------
// K page: chunk (j, hf, g, k8) holds K[8hf+k8][32j+8g .. +7]
__device__ __forceinline__ int k_chunk_offset(int j, int hf, int g, int k8) {
  return ((((j * 2 + hf) * 4 + g) * 8) + k8) * 16;
}
// V page: chunk (w, c, gp, n) holds V[4gp..4gp+3][d] then V[8+4gp..8+4gp+3][d], d = 64w+4n+c
__device__ __forceinline__ int v_chunk_offset(int w, int c, int gp, int n) {
  return ((((w * 4 + c) * 2 + gp) * 16) + n) * 16;
}
// the chunk of dim d
__device__ __forceinline__ int v_chunk_of_dim(int d, int gp) {
  return v_chunk_offset(d >> 6, d & 3, gp, (d >> 2) & 15);
}
__device__ __forceinline__ int v_slot_of_key(int key) { return ((key >> 3) << 2) | (key & 3); }

// One row of K and V on its way into a page: thread t of 256 carries 16 bytes of K (t < 32)
// and one element of V.  Load and store are separate so that callers can keep several rows in
// flight before the first store.
struct RowPart {
  u32x4 k;
  uint16_t v;
};
__device__ __forceinline__ RowPart load_row(const uint16_t* __restrict__ k_row,
                                            const uint16_t* __restrict__ v_row, int t) {
  RowPart r;
  r.k = *(const u32x4*)(k_row + (t & 31) * 8);
  r.v = v_row[t];
  return r;
}
__device__ __forceinline__ void store_row(const RowPart& r, int32_t slot,
                                          char* __restrict__ layer_base, int t) {
  const int blk = slot >> 4, key = slot & 15;
  char* kp = layer_base + (size_t)blk * kBlockBytes;
  char* vp = kp + kPageBytes;
  if (t < 32) *(u32x4*)(kp + k_chunk_offset(t >> 2, key >> 3, t & 3, key & 7)) = r.k;
  *(uint16_t*)(vp + v_chunk_of_dim(t, (key >> 2) & 1) + v_slot_of_key(key) * 2) = r.v;
}
__device__ __forceinline__ void append_row(const uint16_t* __restrict__ k_row,
                                           const uint16_t* __restrict__ v_row, int32_t slot,
                                           char* __restrict__ layer_base, int t) {
  store_row(load_row(k_row, v_row, t), slot, layer_base, t);
}

// ------------------------------------------------------------------------------------------
// attention work items
// ------------------------------------------------------------------------------------------
constexpr float kGrow = 8.f;  // the reference max only moves when a logit exceeds it by 2^8
constexpr int kMaxGroups = 4; // groups of 16 query rows (two tokens) in one work item

// LDS of a work item: nothing of K and V, only what the four wavefronts exchange.  Every u32x4
// entry is one lane's 16-byte MFMA operand, stored and read back at the lane's own position.
struct __align__(16) WorkLds {
  u32x4 q[kMaxGroups][8][64];      // query fragments (B operand of S^T), the same for all wavefronts
  u32x4 p[4][kMaxGroups][2][64];   // [32-key step of the round][group][hi / lo]: P of all 128 keys
  float mx[kMaxGroups][16][4];     // largest logit of a row among each wavefront's 32 keys
  int slot[2 * kMaxGroups];        // split result of each token
  float ls[kMaxGroups][64][4];     // sum of a lane's P over each wavefront's keys
};

// The descriptor is read with scalar loads: it is not written during a launch and every address
// is wave-uniform, so records, token ids and block ids land in scalar registers, take no part in
// the order in which the vector loads of queries and pages complete, and need no lane reads.
typedef const __attribute__((address_space(4))) int32_t* DescPtr;
typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef const __attribute__((address_space(4))) i32x8* DescPtr8;

// A record: 8 header words, 8 query token ids (the last one repeated), the block ids of the
// split's first 16 pages (the last one repeated).  All but the last eight words are requested
// at once at the start of the kernel.
struct WorkItem {
  DescPtr rec;
  i32x8 toks, pages;
  int n_tok, tbl_off, kv_begin, kv_end, q0, part_idx;
};
// What a work item needs only after its first loads, read from the argument segment there.
struct LateArgs {
  uint16_t* part_acc;
  float* part_ml;
  const int32_t* tables;
  int32_t write_through;
};
template <int kOffset>   // of the argument in the kernel's argument segment: see Params
__device__ __forceinline__ void take_late(AttnArgs& a) {
  auto seg = (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(seg));   // here, and not at the start of the kernel
  const auto* late = (const __attribute__((address_space(4))) LateArgs*)(seg + kOffset);
  a.part_acc = late->part_acc;
  a.part_ml = late->part_ml;
  a.tables = late->tables;
  a.write_through = late->write_through;
}
// query token of this lane's row in group r
__device__ __forceinline__ int token_of(const WorkItem& wi, const int r, const int second) {
  return second ? wi.toks[2 * r + 1] : wi.toks[2 * r];
}
// First split result of token lane % (2*G) of the item.  It is needed at the very end only, but
// requested at the start (a full memory latency in front of the stores otherwise) and kept in LDS
// meanwhile: four groups leave no registers for it.
template <int G>
__device__ __forceinline__ int request_slot(const AttnArgs& a, const WorkItem& wi, const int lane) {
  int tok = wi.toks[0];
#pragma unroll
  for (int i = 1; i < 2 * G; ++i) tok = lane % (2 * G) == i ? wi.toks[i] : tok;
  return a.part_off[tok];
}

// Values of keys at or beyond kv_end may be stale bits (never-written slots, freed blocks):
// they are selected to zero, not multiplied by zero.  `left` = valid keys in this step.
__device__ __forceinline__ u32x4 value_mask(const int left, const int g) {
  const int k0 = 16 * (g >> 1) + 4 * (g & 1);
  u32x4 mask;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    mask[i] = (k0 + 2 * i < left ? 0xffffu : 0u) | (k0 + 2 * i + 1 < left ? 0xffff0000u : 0u);
    mask[2 + i] = (k0 + 8 + 2 * i < left ? 0xffffu : 0u) | (k0 + 8 + 2 * i + 1 < left ? 0xffff0000u : 0u);
  }
  return mask;
}

// Softmax scale in the log2 domain, as a positive factor: the largest logit of a row is then the
// scale times its largest dot product, and one fused multiply-add takes a dot product to its
// exponent.  A negative scale goes into the sign of the queries (see query_sign); a zero one is
// taken as 2^-120, which gives the same uniform weights and keeps -inf (a masked key) what it is.
__device__ __forceinline__ float log2_scale(const AttnArgs& a) {
  const float x = fabsf(a.scale * 1.4426950408889634f);
  return x == 0.f ? 0x1p-120f : x;
}
// flips the signs of eight bf16 query elements where the scale is negative
__device__ __forceinline__ u32x4 query_sign(const AttnArgs& a, const u32x4 q) {
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
  return q ^ (u32x4){flip, flip, flip, flip};
}
// largest of a lane's eight dot products
__device__ __forceinline__ float row_max8(const f32x4 s0, const f32x4 s1) {
  return fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])),
               fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
}
// P = 2^(sl2 * s - m) of a lane's eight dot products as hi + lo bf16 (a single bf16 rounding, 2^-9
// relative, is too coarse for queries that see only a handful of keys); returns their fp32 sum.
__device__ __forceinline__ float softmax_weights(const f32x4 s0, const f32x4 s1, const float sl2,
                                                 const float m, u32x4& hi, u32x4& lo) {
  float p[8], sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[e] = fast_exp2(__builtin_fmaf(e < 4 ? s0[e & 3] : s1[e & 3], sl2, -m));
    sum += p[e];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    hi[i] = pack_bf16(p[2 * i], p[2 * i + 1]);
    lo[i] = pack_bf16(p[2 * i] - __uint_as_float(hi[i] << 16),
                      p[2 * i + 1] - __uint_as_float(hi[i] & 0xffff0000u));
  }
  return sum;
}
// A row's sum times the factor of a moved reference.  Rounded here, never contracted with the addition
// that follows: otherwise `attend`, where the two lie in different branches, and `attend_fresh`, where
// they do not, give different bits.
__device__ __forceinline__ float rescaled(const float l, const float alpha) {
#pragma clang fp contract(off)
  return l * alpha;
}
// Stores a at dst and b 64 bytes on.  A launch leaves its split results dirty in eight L2s, and the
// merge launch starts only when they have been written back: 1.4 us after the last work item of a
// launch with 9 split results, 5.8 us with 15 MB of them.  Written through (sc0 sc1) they reach
// memory while other work items run.  A work item then ends with their acknowledgement, which costs
// a small launch more than it gives, hence a flag (see kWriteThroughParts).  In inline assembly: no
// builtin takes these bits with a 64-bit address.  The wait counts that the compiler places after it are
// only ever stricter than needed, and the two wait states keep the data registers from being
// written in the cycles in which a 128-bit store still reads them.
__device__ __forceinline__ void store_piece_pair(const AttnArgs& args, u32x4* dst, const u32x4 a,
                                                 const u32x4 b) {
  if (args.write_through) {
    asm volatile("global_store_dwordx4 %0, %1, off sc0 sc1\n\t"
                 "global_store_dwordx4 %0, %2, off offset:64 sc0 sc1\n\t"
                 "s_nop 1" ::"v"(dst), "v"(a), "v"(b) : "memory");
  } else {
    dst[0] = a;
    dst[4] = b;
  }
}
// Eight rows' 128 bytes each at (split result, offset), for both tokens of a group: see store_part.  Buffer
// stores take the cache bits of the written-through form as an argument.
__device__ __forceinline__ void store_lines(const AttnArgs& args, const int offset, const int slot_a,
                                            const u32x4 a, const bool live_a, const int slot_b,
                                            const u32x4 b, const bool live_b) {
  constexpr int kPartBytes = kHeads * kDim * (int)sizeof(uint16_t), kFlags = 0x00027000;
  constexpr int kThrough = 1 | 16;   // sc0, sc1
  // a token that is not there has a buffer of no bytes: its rows are dropped
  const auto part_a = __builtin_amdgcn_make_buffer_rsrc((char*)args.part_acc + (size_t)slot_a * kPartBytes, 0,
                                                        live_a ? kPartBytes : 0, kFlags);
  const auto part_b = __builtin_amdgcn_make_buffer_rsrc((char*)args.part_acc + (size_t)slot_b * kPartBytes, 0,
                                                        live_b ? kPartBytes : 0, kFlags);
  if (args.write_through) {
    __builtin_amdgcn_raw_buffer_store_b128(a, part_a, offset, 0, kThrough);
    __builtin_amdgcn_raw_buffer_store_b128(b, part_b, offset, 0, kThrough);
  } else {
    __builtin_amdgcn_raw_buffer_store_b128(a, part_a, offset, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b128(b, part_b, offset, 0, 0);
  }
}
constexpr int kRowRor8 = 0x128;   // DPP: lane n of each 16 gets lane n^8's value
// One wavefront's 64 dims of a group's split result.  A split result leaves as (m, l, four
// exponents) and acc * 2^(14 - exponent) in fp16: half the bytes of fp32, with the exponent of the
// largest value per row and 64 dims, so that the rounding does not depend on the magnitude of the
// values.  kLines: whole lines, for items of eight tokens, whose launches write the most (us per layer, pieces /
// lines: eight chunks on 2048 tokens 24.4 / 23.6, six on 1500 22.1 / 21.6, four and 32 requests on 1024 17.9 / 17.1,
// eight on 832 17.36 / 17.32; narrower items are up to 1 % slower with it).  acc[c][e] = dim 16g + 4e + c of the 64: a lane's sixteen values are consecutive.  slot:
// split result of this lane's token.  kUnit: acc is in units of 2^unit.
template <bool kLines, bool kUnit = false>
__device__ __forceinline__ void store_part(const AttnArgs& a, const WorkItem& wi, const int slot,
                                           const f32x4 (&acc)[4], const int group, const int wv,
                                           const int lane, const int unit = 0) {
  const int n = lane & 15, g = lane >> 4;
  float amax = 0.f;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) amax = fmaxf(amax, fabsf(acc[c][e]));
  amax = row_max4(amax);
  // biased exponent of amax, kept where 2^(14 - exponent) is a normal number
  const int eb = max(24, min(253, (int)(__float_as_uint(amax) >> 23)));
  // an infinite value leaves no exponent for the others: all 64 are NaN then, instead of zeros (looking
  // for the largest finite one in a branch of its own cost 0.5 % of a launch of chunks)
  float up;
  int ex;
  if constexpr (kUnit) {   // the exponent that is stored is that of the values, within its eight bits
    ex = max(-128, min(127, eb - 126 + unit));
    up = __uint_as_float((uint32_t)(127 + 14 - (ex - unit)) << 23) + (amax - amax);
  } else {
    up = __uint_as_float((uint32_t)(127 + 14 + 126 - eb) << 23) + (amax - amax);
    ex = eb - 126;
  }
  u32x4 o[2];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    o[e >> 1][2 * (e & 1)] = pack_f16(acc[0][e] * up, acc[1][e] * up);
    o[e >> 1][2 * (e & 1) + 1] = pack_f16(acc[2][e] * up, acc[3][e] * up);
  }
  if constexpr (kLines) {
    // Lane g of row n holds 16-byte pieces 2g and 2g+1 of the row's eight.  Rows n and n^8 (the group's two
    // tokens) trade one each, so that a store takes whole lines: eight lanes the 128 bytes of one row, a
    // token's eight rows at once.
    u32x4 first = o[0], second = o[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      first[i] = __builtin_amdgcn_update_dpp(o[0][i], o[1][i], kRowRor8, 0xf, 0xc, false);
      second[i] = __builtin_amdgcn_update_dpp(o[1][i], o[0][i], kRowRor8, 0xf, 0x3, false);
    }
    const int offset = (n & 7) * (kDim * 2) + 128 * wv + 32 * g + 16 * (n >> 3);
    store_lines(a, offset, __builtin_amdgcn_readlane(slot, 0), first, 2 * group < wi.n_tok,
                __builtin_amdgcn_readlane(slot, 8), second, 2 * group + 1 < wi.n_tok);
    if (g == 0 && 2 * group + (n >> 3) < wi.n_tok)
      ((int8_t*)(a.part_ml + ((size_t)slot * kHeads + (n & 7)) * 4 + 2))[wv] = (int8_t)ex;
    return;
  }
  // Lane g of a row holds 16-byte pieces 2g and 2g+1 of the row's eight: exchanged so that the
  // four lanes of a row store pieces 0..3 together and then 4..7, 64 contiguous bytes each time.
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto x = __builtin_amdgcn_permlane16_swap(o[0][i], o[1][i], false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(x[0], x[1], false, false);
    o[0][i] = y[0];
    o[1][i] = y[1];
  }
  if (2 * group + (n >> 3) < wi.n_tok) {
    const size_t row = (size_t)slot * kHeads + (n & 7);
    u32x4* dst = (u32x4*)(a.part_acc + row * kDim + 64 * wv + 8 * g);
    store_piece_pair(a, dst, o[0], o[1]);
    if (g == 0) ((int8_t*)(a.part_ml + row * 4 + 2))[wv] = (int8_t)ex;
  }
}

// Where the argument segment holds a kernel's last argument: each lies at the next multiple of its alignment.
template <class Kernel>
struct Params;
template <class... P>
struct Params<void (*)(P...)> {
  using Last = std::tuple_element_t<sizeof...(P) - 1, std::tuple<P...>>;
  static constexpr size_t offset_of_last() {
    constexpr size_t n = sizeof...(P), size[n] = {sizeof(P)...}, align[n] = {alignof(P)...};
    size_t at = 0;
    for (size_t i = 0; i + 1 < n; ++i) at = (at + align[i] - 1) / align[i] * align[i] + size[i];
    return (at + align[n - 1] - 1) / align[n - 1] * align[n - 1];
  }
};

}  // namespace oxy
