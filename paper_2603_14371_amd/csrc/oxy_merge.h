// Merge of a query token's partials by the log-sum-exp rule: device code of every merge launch.
#pragma once
#include "oxy_device.h"

namespace oxy {

constexpr int kMergeAhead = 16;       // partials whose loads are all issued before anything is used
struct MergeArgs {
  const uint16_t* part_acc;
  const float* part_ml;
  void* out;
  float* lse;
  const int32_t *n_parts, *part_off;
};
constexpr int kRowBcast0 = 0x150;     // DPP: all lanes of each 16 get the value of lane 0 (+ u: lane u)

// largest value / sum of a row of 16 lanes, in all of them
__device__ __forceinline__ float lanes16_max(float x) {
  x = fmaxf(x, dpp_row_ror<8>(x));
  x = fmaxf(x, dpp_row_ror<4>(x));
  x = fmaxf(x, dpp_row_ror<2>(x));
  return fmaxf(x, dpp_row_ror<1>(x));
}
__device__ __forceinline__ float lanes16_sum(float x) {
  x += dpp_row_ror<8>(x);
  x += dpp_row_ror<4>(x);
  x += dpp_row_ror<2>(x);
  return x + dpp_row_ror<1>(x);
}

// Bound by the round trip of its loads, by their bytes where tokens are many (400 tokens of 9 split results:
// 14.7 MB).  Lane 16q + i owns dims 64q + 4i..+3 of the output, and, for the weights, split result i of every
// sixteen in the 64 dims q, whose exponent it applies: sixteen weights take one exponential per wavefront, and a
// weight reaches its 16 lanes by a DPP broadcast.  (With a workgroup per token, eight dims per thread and every
// weight computed by every thread, the sums of nine split results alone took 0.7 us of a wavefront.  Layer of
// a decode step 6.80 -> 6.36 us, of 50 queries + one request 8.37 -> 7.88, of three requests 7.37 -> 6.77, of 78 queries
// with up to 15 split results 12.8 -> 11.9, of 64 requests and two chunks on 2048 tokens 23.6 -> 23.1.)
// They are read here and never again, hence the non-temporal hint (50 queries + one request 8.22 -> 8.12 us,
// 64 requests and two chunks 23.2 -> 22.8; on (m, l) too: 2 % slower).
// kAhead: split results whose loads are issued before anything is used, np rounded up to a multiple of four
// or the most: an instance for each, so that the first wait is for (m, l) only (loads under conditions are
// all waited for where the conditions meet; three requests 6.96 us a layer, now 6.77).
template <int kAhead>
__device__ __forceinline__ void merge_head(const MergeArgs& a, const size_t base, const int np, const int tok,
                                           const int h, const int lane) {
  const int i = lane & 15, q = lane >> 4;
  // wave-uniform; a lane adds 32 bits to them
  const char* ml = (const char*)(a.part_ml + (base * kHeads + h) * 4);
  const char* acc = (const char*)(a.part_acc + (base * kHeads + h) * kDim);
  constexpr uint32_t kMlStride = kHeads * 4 * sizeof(float), kAccStride = kHeads * kDim * sizeof(uint16_t);
  const float ninf = -__builtin_inff();
  u32x2 x[kAhead];
  // (m, l, exponents of the 64-dim parts, -) of this lane's split result; past the end the last one's
  auto load_ml = [&](const int p0) {
    return *(const f32x4*)(ml + (uint32_t)min(p0 + i, np - 1) * kMlStride);
  };
  auto load_x = [&](const int p0) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      x[u] = __builtin_nontemporal_load((const u32x2*)(acc + (size_t)min(p0 + u, np - 1) * kAccStride + (uint32_t)lane * 8u));
  };
  f32x4 w = load_ml(0);
  load_x(0);
  float big = w[0];
  if constexpr (kAhead == kMergeAhead)
    for (int p0 = kAhead; p0 < np; p0 += kAhead)
      big = fmaxf(big, load_ml(p0)[0]);
  big = lanes16_max(big);
  float total = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](const int p0) {
    const bool live = p0 + i < np && w[0] != ninf;
    const float wgt = live ? fast_exp2(w[0] - big) : 0.f;
    total += wgt * (live ? w[1] : 0.f);
    const int ex = (int32_t)(__float_as_uint(w[2]) << (24 - 8 * q)) >> 24;   // signed byte q
    const float ws = __builtin_amdgcn_ldexpf(wgt, ex - 14);
    static_for<kAhead>([&](auto u) {
      const float wu = __uint_as_float(
          __builtin_amdgcn_update_dpp(0, __float_as_uint(ws), kRowBcast0 + u.value, 0xf, 0xf, false));
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float lo, hi;
        unpack_f16(x[u.value][k], lo, hi);
        o[2 * k] = __builtin_fmaf(wu, lo, o[2 * k]);
        o[2 * k + 1] = __builtin_fmaf(wu, hi, o[2 * k + 1]);
      }
    });
  };
  add(0);
  if constexpr (kAhead == kMergeAhead)
    for (int p0 = kAhead; p0 < np; p0 += kAhead) {
      w = load_ml(p0);
      load_x(p0);
      add(p0);
    }
  total = lanes16_sum(total);
  const float inv = 1.f / total;
  const u32x2 packed = {pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
  *(u32x2*)((uint16_t*)a.out + ((size_t)tok * kHeads + h) * kDim + 4 * lane) = packed;
  if (a.lse && lane == 0)
    a.lse[(size_t)tok * kHeads + h] = (big + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
}
__device__ __forceinline__ void merge_any(const MergeArgs& a, const size_t base, const int np, const int tok, const int h,
                                          const int lane) {
  if (np <= 4)
    merge_head<4>(a, base, np, tok, h, lane);
  else if (np <= 8)
    merge_head<8>(a, base, np, tok, h, lane);
  else if (np <= 12)
    merge_head<12>(a, base, np, tok, h, lane);
  else
    merge_head<kMergeAhead>(a, base, np, tok, h, lane);
}
template <int kBlockHeads>
__device__ __forceinline__ void merge_block(const MergeArgs& a, const int block) {
  constexpr int kBlocks = kHeads / kBlockHeads;
  const int tok = block / kBlocks, lane = threadIdx.x & 63;
  const int h = kBlockHeads * (block % kBlocks) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int np = ((DescPtr)a.n_parts)[tok];
  const size_t base = (size_t)((DescPtr)a.part_off)[tok];
  merge_any(a, base, np, tok, h, lane);
}

}  // namespace oxy
