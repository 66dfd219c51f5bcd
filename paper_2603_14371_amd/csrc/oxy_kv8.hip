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
// what differs is what lies in memory: half the bytes, turned into bf16 operands in registers.  The products stay in bf16:
// the 8-bit matrix instructions round their own sums to about 2^-16 of the products' 2-norm (rms 1.5e-5, up to 5e-5 with
// products of different size, measured on sums of 128), which a log-sum-exp in 32 bits would show, and queries and
// probabilities would have to be split into two and three 8-bit parts.  A conversion of two codes takes about 5 cycles
// of a wavefront: 128 of them a round beside 48 matrix instructions of 16 cycles per 16 query rows.
#include "oxy_kv8_device.h"
#include "oxy_merge.h"

#include <hip/hip_ext.h>

#include <type_traits>

namespace oxy {

// ------------------------------------------------------------------------------------------
// quantised append
// ------------------------------------------------------------------------------------------
// One wavefront per token: the first half takes the key, the second the value.
constexpr int kAppendTokens8 = 4;   // wavefronts, and tokens, of a workgroup
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
// V is turned through LDS and goes out in whole chunks where all eight keys of one are among the rows, byte by byte
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
  // thread t: chunk t of the V page, eight keys of dims d and d+1
  const int gp = (t >> 4) & 1, d = 64 * (t >> 6) + 4 * (t & 15) + 2 * ((t >> 5) & 1);
  u32x4 out = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t two = *(const uint16_t*)(&sm.v[(e < 4 ? 4 * gp : 4 + 4 * gp) + e][d]);
    out[e >> 2] |= (two & 0xffu) << (8 * (e & 3));
    out[2 + (e >> 2)] |= (two >> 8) << (8 * (e & 3));
  }
  char* vp = block + kPageBytes8 + t * 16;
  if (kWhole || (key0 <= 4 * gp && key0 + n >= 12 + 4 * gp)) {
    *(u32x4*)vp = out;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int key = (e < 4 ? 4 * gp : 4 + 4 * gp) + e;
      if (key >= key0 && key < key0 + n) {
        vp[e] = (char)(out[e >> 2] >> (8 * (e & 3)));
        vp[8 + e] = (char)(out[2 + (e >> 2)] >> (8 * (e & 3)));
      }
    }
  }
}

// A run of consecutive positions of one table (a prefix): one workgroup per block, blockIdx.y = layer.
__global__ __launch_bounds__(256) void append_blocks8_kernel(const uint16_t* __restrict__ k_new,
                                                             const uint16_t* __restrict__ v_new, const InlineIds ids,
                                                             int32_t pos0, int32_t n_tokens, char* __restrict__ blocks,
                                                             uint8_t* __restrict__ scales, size_t src_layer_stride,
                                                             size_t pool_layer_stride) {
  __shared__ PageLds8 sm;
  k_new = (const uint16_t*)((const char*)k_new + blockIdx.y * src_layer_stride);
  v_new = (const uint16_t*)((const char*)v_new + blockIdx.y * src_layer_stride);
  const int page = (pos0 >> 4) + blockIdx.x;
  const int lo = max(pos0, page * kPage), hi = min(pos0 + n_tokens, (page + 1) * kPage);
  const size_t blk = ids.v[blockIdx.x];
  char* block = blocks + blockIdx.y * pool_layer_stride + blk * kBlockBytes8;
  uint8_t* sc = scales + blockIdx.y * pool_layer_stride + blk * kScaleBytes8;
  k_new += (size_t)(lo - pos0) * kDim;
  v_new += (size_t)(lo - pos0) * kDim;
  if (hi - lo == kPage)
    append_page8<true>(k_new, v_new, 0, kPage, block, sc, sm, threadIdx.x);
  else
    append_page8<false>(k_new, v_new, lo & 15, hi - lo, block, sc, sm, threadIdx.x);
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
// Runs of at most the 16 tokens of a block in natural order, one workgroup per run, blockIdx.y = layer.  The pages are
// read as whole chunks; V is turned through LDS as codes.
__global__ __launch_bounds__(256) void gather8_kernel(const char* __restrict__ blocks, const uint8_t* __restrict__ scales,
                                                      const GatherRuns runs, uint16_t* __restrict__ k_out,
                                                      uint16_t* __restrict__ v_out, size_t out_layer_stride,
                                                      size_t pool_layer_stride) {
  __shared__ PageLds8 sm;
  const int t = threadIdx.x;
  const int slot = runs.slot[blockIdx.x], where = runs.where[blockIdx.x];
  const int key0 = slot & 15, len = (where & 15) + 1;
  const char* kp = blocks + blockIdx.y * pool_layer_stride + (size_t)(slot >> 4) * kBlockBytes8;
  const uint8_t* sc = scales + blockIdx.y * pool_layer_stride + (size_t)(slot >> 4) * kScaleBytes8;
  k_out = (uint16_t*)((char*)k_out + blockIdx.y * out_layer_stride);
  v_out = (uint16_t*)((char*)v_out + blockIdx.y * out_layer_stride);
  const int gp = (t >> 4) & 1, d = 64 * (t >> 6) + 4 * (t & 15) + 2 * ((t >> 5) & 1);
  const int lo = 4 * gp, hi = lo + 8, end = key0 + len;
  const bool wanted = (key0 < lo + 4 && end > lo) || (key0 < hi + 4 && end > hi);   // a key of the run in the chunk
  // row `key`, dims 16c..16c+15 of this thread
  const int key = t >> 4, c = t & 15;
  const bool mine = key >= key0 && key < end;
  u32x4 v = {0, 0, 0, 0}, k = {0, 0, 0, 0};
  uint32_t ek = 0, ev = 0;
  if (wanted) v = *(const u32x4*)(kp + kPageBytes8 + t * 16);
  if (mine) {
    k = *(const u32x4*)(kp + k8_chunk_offset(c >> 2, key >> 3, c & 3, key & 7));
    ek = sc[k8_scale_offset(key)];
    ev = sc[v8_scale_offset(key)];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    *(uint16_t*)(&sm.v[(e < 4 ? 4 * gp : 4 + 4 * gp) + e][d]) =
        (uint16_t)(((v[e >> 2] >> (8 * (e & 3))) & 0xffu) | (((v[2 + (e >> 2)] >> (8 * (e & 3))) & 0xffu) << 8));
  __syncthreads();
  if (mine) {
    const size_t at = ((size_t)(where >> 4) + key - key0) * kDim + 16 * c;
    store_values16(k_out + at, k, scale_of(ek));
    store_values16(v_out + at, *(const u32x4*)(&sm.v[key][16 * c]), scale_of(ev));
  }
}

// ------------------------------------------------------------------------------------------
// attention work items
// ------------------------------------------------------------------------------------------
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
// eight codes (two words) times a power of two -> eight bf16, one 16-byte matrix operand
__device__ __forceinline__ u32x4 operand_of(const uint32_t lo, const uint32_t hi, const float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  return r;
}
// first `left` of four bytes
__device__ __forceinline__ uint32_t byte_mask(const int left) {
  return left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
}
// P = 2^(sl2 * s - m) of a lane's eight dot products; what meets the value codes is P times the values' scales, as
// hi + lo bf16 (see softmax_weights).  Returns the sum of P itself.
__device__ __forceinline__ float scaled_weights(const f32x4 s0, const f32x4 s1, const float sl2, const float m,
                                                const float (&vs)[8], u32x4& hi, u32x4& lo) {
  float w[8], sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = fast_exp2(__builtin_fmaf(e < 4 ? s0[e & 3] : s1[e & 3], sl2, -m));
    sum += p;
    w[e] = p * vs[e];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    hi[i] = pack_bf16(w[2 * i], w[2 * i + 1]);
    lo[i] = pack_bf16(w[2 * i] - __uint_as_float(hi[i] << 16), w[2 * i + 1] - __uint_as_float(hi[i] & 0xffff0000u));
  }
  return sum;
}

// One work item: up to 2*G query tokens against one split of a KV source, in rounds of 128 keys, as `attend` in
// oxy_kernels.hip: wavefront w takes the logits of keys 32w..32w+31 and contracts all 128 for dims 64w..64w+63.  A
// round's pages are 32 + 32 registers of codes (64 + 64 in bf16).  A K operand is converted once for all groups, with
// its rows' exponents as the conversion's scale; the V operands with scale 1, since a lane's eight codes are of eight
// keys: their exponents go into P.  A row's arithmetic does not depend on G or on the other rows.
// kSteps: 32-key steps of a round that are loaded, 4, or 2 for a split of at most 64 keys.
// kOnce: non-temporal page loads (see kOnceBytes).
template <int G, bool kOnce, int kSteps>
__device__ __forceinline__ void attend8(const AttnArgs8& early_args, const WorkItem& wi, WorkLds& sm) {
  constexpr int kLate8 = 5 * 8;
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
  const int rounds = (nsteps + 3) >> 2;
  const int npg = ((wi.kv_end + 15) >> 4) - (wi.kv_begin >> 4);

  u32x4 kr[8];            // kr[2jj+hf]: K chunk (jj, hf) of this wavefront's 32 keys
  u32x4 vr[kSteps][2];    // vr[s][cp]: V chunk cp of this wavefront's 64 dims, step s of the round
  uint32_t ke = 0;        // exponents of this lane's keys of the first product (hf = 0, 1)
  u32x2 ve = {0, 0};      // of the eight keys whose logits it receives
  auto page_load = [](const char* p) {
    if constexpr (kOnce) return __builtin_nontemporal_load((const u32x4*)p);
    return *(const u32x4*)p;
  };
  // A step past the split's end re-reads a page of the split; its logits are masked and its V operands are zeros.
  auto load_k_of = [&](const int blk_a, const int blk_b) {
    int off = (g * 8 + (n & 7)) * 16, off_k = 2 * (n & 7), off_v = kPage + 8 * (g & 1);
    asm volatile("" : "+v"(off), "+v"(off_k), "+v"(off_v));
    ke = *(const uint16_t*)(scales + (size_t)((n >> 3) ? blk_b : blk_a) * kScaleBytes8 + off_k);
    ve = *(const u32x2*)(scales + (size_t)((g >> 1) ? blk_b : blk_a) * kScaleBytes8 + off_v);
    const char* p = base + (size_t)((n >> 3) ? blk_b : blk_a) * kBlockBytes8 + off;
#pragma unroll
    for (int i = 0; i < 8; ++i) kr[i] = page_load(p + i * 512);
  };
  auto load_v_of = [&](const i32x8 blks) {
    int off = kPageBytes8 + v8_chunk_offset(wv, 0, g & 1, n);
    asm volatile("" : "+v"(off));
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const char* p = base + (size_t)((g >> 1) ? blks[2 * s + 1] : blks[2 * s]) * kBlockBytes8 + off;
#pragma unroll
      for (int cp = 0; cp < 2; ++cp) vr[s][cp] = page_load(p + cp * 512);
    }
  };
  auto load_k = [&](const int round) {
    if (round < 2) {
      const DescPtr id = wi.rec + 16 + 8 * round + 2 * wv;
      load_k_of(id[0], id[1]);
    } else {
      const DescPtr ids = (DescPtr)a.tables + wi.tbl_off + (wi.kv_begin >> 4);
      const int pi = 8 * round + 2 * wv;
      load_k_of(ids[min(pi, npg - 1)], ids[min(pi + 1, npg - 1)]);
    }
  };
  auto load_v = [&](const int round) {
    if (round < 2) {
      load_v_of(*(DescPtr8)(wi.rec + 16 + 8 * round));
    } else {
      const DescPtr ids = (DescPtr)a.tables + wi.tbl_off + (wi.kv_begin >> 4);
      i32x8 blks;
#pragma unroll
      for (int i = 0; i < 8; ++i) blks[i] = ids[min(8 * round + i, npg - 1)];
      load_v_of(blks);
    }
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
      for (int r = 0; r < G; ++r) {
        const u32x4 z = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 2; ++i)
          sm.q[r][2 * wv + i][lane] = 2 * r + sub < wi.n_tok ? query_sign(a, qtmp[r][i]) : z;
      }
    };
    if (kSteps == 2 && wv >= 2) {
      load_v_of(wi.pages);
      store_q();
    } else {
      load_k_of(wi.rec[16 + 2 * wv], wi.rec[17 + 2 * wv]);
      load_v_of(wi.pages);
      store_q();
    }
  }
  if (tid < 2 * G) sm.slot[tid] = slot_req + wi.part_idx;
  __syncthreads();

  float m[G], l[G];   // reference max (scaled log2 domain) of this lane's row, and the sum of P
  f32x4 acc[G][4];    // over this wavefront's keys; acc[r][c][e] = dim 64w + 16g + 4e + c
#pragma unroll
  for (int r = 0; r < G; ++r) {
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
    const int pos = wi.kv_begin + 32 * (4 * round + wv);
    const int left = wi.kv_end - pos;
    const bool need_mask = (kLast && left < 32) || pos + 31 > wi.q0;
    f32x4 s0[G], s1[G];
    float vs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) vs[e] = 0.f;
    if (kSteps == 4 || wv < 2) {
#pragma unroll
      for (int r = 0; r < G; ++r) s0[r] = s1[r] = (f32x4){0.f, 0.f, 0.f, 0.f};
      const float ks0 = scale_of(ke & 0xffu), ks1 = scale_of(ke >> 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const u32x4 a0 = kr[2 * (j >> 1)], a1 = kr[2 * (j >> 1) + 1];
        const u32x4 k0 = operand_of(a0[2 * (j & 1)], a0[2 * (j & 1) + 1], ks0);
        const u32x4 k1 = operand_of(a1[2 * (j & 1)], a1[2 * (j & 1) + 1], ks1);
#pragma unroll
        for (int r = 0; r < G; ++r) {
          const u32x4 q = sm.q[r][j][lane];
          s0[r] = mfma16(k0, q, s0[r]);
          s1[r] = mfma16(k1, q, s1[r]);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) vs[e] = scale_of((ve[e >> 2] >> (8 * (e & 3))) & 0xffu);
      if (need_mask) {   // wave-uniform: only the end of a split or the causal diagonal
        const int k0 = pos + 16 * (g >> 1) + 4 * (g & 1);
#pragma unroll
        for (int r = 0; r < G; ++r) {
          const int end = min(wi.kv_end, wi.q0 + 2 * r + sub + 1) - k0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s0[r][e] = e < end ? s0[r][e] : ninf;
            s1[r][e] = 8 + e < end ? s1[r][e] : ninf;
          }
        }
        // the exponent byte of a slot that was never written may be anything: 0 * inf would poison a row
#pragma unroll
        for (int e = 0; e < 8; ++e) vs[e] = (e < 4 ? e : 4 + e) < wi.kv_end - k0 ? vs[e] : 0.f;
      }
    } else {
#pragma unroll
      for (int r = 0; r < G; ++r) s0[r] = s1[r] = (f32x4){ninf, ninf, ninf, ninf};
    }
    {
      float mx[G];
#pragma unroll
      for (int r = 0; r < G; ++r) mx[r] = row_max8(s0[r], s1[r]) * sl2;
      const float mine = row_max4_each(mx);
      if (g < G) sm.mx[g][n][wv] = mine;
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
#pragma unroll
    for (int r = 0; r < G; ++r) {
      u32x4 hi, lo;
      l[r] += scaled_weights(s0[r], s1[r], sl2, (m[r] == ninf) ? 0.f : m[r], vs, hi, lo);
      sm.p[wv][r][0][lane] = hi;
      sm.p[wv][r][1][lane] = lo;
      if constexpr (kLast) sm.ls[r][lane][wv] = l[r];
    }
    __builtin_amdgcn_sched_barrier(0);   // the next K chunks reuse kr[]
    if constexpr (!kLast) load_k(round + 1);
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    auto value_operands = [&](const int s, u32x4 (&v)[4]) {
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = operand_of(vr[s][c >> 1][2 * (c & 1)], vr[s][c >> 1][2 * (c & 1) + 1], 1.f);
    };
    auto contract = [&](const u32x4 (&v)[4], const int s, const int r) {
      const u32x4 hi = sm.p[s][r][0][lane], lo = sm.p[s][r][1][lane];
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[r][c] = mfma16(v[c], hi, acc[r][c]);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[r][c] = mfma16(v[c], lo, acc[r][c]);
    };
    if constexpr (!kLast) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        u32x4 v[4];
        value_operands(s, v);
#pragma unroll
        for (int r = 0; r < G; ++r) contract(v, s, r);
      }
      __builtin_amdgcn_sched_barrier(0);   // likewise vr[]
      load_v(round + 1);
      __builtin_amdgcn_sched_barrier(0);
    } else {
      const int nv = nsteps - 4 * round;   // 1..4 steps
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        if (s < nv) {
          const int left_s = wi.kv_end - (wi.kv_begin + 32 * (4 * round + s));
          if (left_s < 32) {   // codes of slots beyond the end may be anything
            const int k0 = 16 * (g >> 1) + 4 * (g & 1);
            const uint32_t m0 = byte_mask(left_s - k0), m1 = byte_mask(left_s - k0 - 8);
#pragma unroll
            for (int cp = 0; cp < 2; ++cp) vr[s][cp] &= (u32x4){m0, m1, m0, m1};
          }
          u32x4 v[4];
          value_operands(s, v);
#pragma unroll
          for (int r = 0; r < G; ++r) contract(v, s, r);
        }
#pragma unroll
      for (int r = 0; r < G; ++r) {
        const int slot = sm.slot[2 * r + sub];
        store_part<(G >= 4)>(a, wi, slot, acc[r], r, wv, lane);
        if (wv == r) {   // wave-uniform: the sums of the groups are shared out
          const f32x4 lw = *(const f32x4*)sm.ls[r][lane];
          const float total = row_sum4((lw[0] + lw[1]) + (lw[2] + lw[3]));
          if (g == 0 && 2 * r + sub < wi.n_tok)
            *(f32x2*)(a.part_ml + ((size_t)slot * kHeads + (n & 7)) * 4) = (f32x2){m[r], total};
        }
      }
    }
  };
  if constexpr (kSteps == 4)
    for (int round = 0; round + 1 < rounds; ++round) round_body(round, std::false_type());
  round_body(kSteps == 4 ? rounds - 1 : 0, std::true_type());
}

__global__ __attribute__((aligned(4096))) __launch_bounds__(256, 2) void attn8_kernel(
    const int32_t* work, const void* q, const void* layer_base, const uint8_t* scales, const int32_t part_off,
    const float scale, const LateArgs) {
  __shared__ WorkLds sm;
  AttnArgs8 a;
  a.q = q;
  a.layer_base = layer_base;
  a.scales = scales;
  a.part_off = work + part_off;
  a.scale = scale;
  WorkItem wi;
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
  const int path_word = head[W_PATH];
  if ((path_word & kPathMask) == PATH_NOOP) return;
  const bool few_keys = wi.kv_end - wi.kv_begin <= 64;
  if (path_word & kPathOnce)
    attend8<1, true, 4>(a, wi, sm);
  else if (wi.n_tok > 4)
    few_keys ? attend8<4, false, 2>(a, wi, sm) : attend8<4, false, 4>(a, wi, sm);
  else if (wi.n_tok > 2)
    few_keys ? attend8<2, false, 2>(a, wi, sm) : attend8<2, false, 4>(a, wi, sm);
  else
    few_keys ? attend8<1, false, 2>(a, wi, sm) : attend8<1, false, 4>(a, wi, sm);
}
static_assert(Params<decltype(&attn8_kernel)>::offset_of_last() == 5 * 8, "attend8 reads the last argument there");

// ------------------------------------------------------------------------------------------
// merge of tokens with many split results
// ------------------------------------------------------------------------------------------
// A wavefront per token and head takes 0.9 us for every 16 split results behind the first (29 us for the 512 of a history
// of 131072 tokens: two workgroups read 2 MB in turn).  Here a workgroup per token and head: a token of more than
// kLongParts results has them shared out among 16 wavefronts, 16 at a time, each with a maximum of its own, and the first
// one joins the sixteen.  Tokens of fewer are merged by one wavefront as in every other launch, so that a token's bits do
// not depend on what else is in the batch.
constexpr int kLongWaves = 16;
__global__ __launch_bounds__(64 * kLongWaves) void merge_long_kernel(const uint16_t* part_acc, const float* part_ml, void* out,
                                                                    float* lse, const int32_t* n_parts,
                                                                    const int32_t* part_off) {
  __shared__ f32x4 os[kLongWaves][64];
  __shared__ float bigs[kLongWaves], totals[kLongWaves];
  const MergeArgs a = {part_acc, part_ml, out, lse, n_parts, part_off};
  const int tok = blockIdx.x / kHeads, h = blockIdx.x % kHeads;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int np = ((DescPtr)n_parts)[tok];
  const size_t base = (size_t)((DescPtr)part_off)[tok];
  if (np <= kLongParts) {
    if (wv == 0) merge_any(a, base, np, tok, h, lane);
    return;
  }
  const int i = lane & 15, q = lane >> 4;
  const char* ml = (const char*)(part_ml + (base * kHeads + h) * 4);
  const char* acc = (const char*)(part_acc + (base * kHeads + h) * kDim);
  constexpr uint32_t kMlStride = kHeads * 4 * sizeof(float), kAccStride = kHeads * kDim * sizeof(uint16_t);
  const float ninf = -__builtin_inff();
  float big = ninf;
  for (int p0 = 16 * wv; p0 < np; p0 += 16 * kLongWaves)
    big = fmaxf(big, *(const float*)(ml + (size_t)min(p0 + i, np - 1) * kMlStride));
  big = lanes16_max(big);
  float total = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 16 * wv; p0 < np; p0 += 16 * kLongWaves) {
    const f32x4 w = *(const f32x4*)(ml + (size_t)min(p0 + i, np - 1) * kMlStride);
    u32x2 x[16];
#pragma unroll
    for (int u = 0; u < 16; ++u)
      x[u] = __builtin_nontemporal_load((const u32x2*)(acc + (size_t)min(p0 + u, np - 1) * kAccStride + (uint32_t)lane * 8u));
    const bool live = p0 + i < np && w[0] != ninf;
    const float wgt = live ? fast_exp2(w[0] - big) : 0.f;
    total += wgt * (live ? w[1] : 0.f);
    const int ex = (int32_t)(__float_as_uint(w[2]) << (24 - 8 * q)) >> 24;
    const float ws = __builtin_amdgcn_ldexpf(wgt, ex - 14);
    static_for<16>([&](auto u) {
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
  }
  os[wv][lane] = (f32x4){o[0], o[1], o[2], o[3]};
  total = lanes16_sum(total);
  if (lane == 0) bigs[wv] = big, totals[wv] = total;
  __syncthreads();
  if (wv != 0) return;
  const float mine = bigs[i];
  const float top = lanes16_max(mine);
  const float wgt = mine == ninf ? 0.f : fast_exp2(mine - top);
  const float sum = lanes16_sum(wgt * totals[i]);
  f32x4 r = {0.f, 0.f, 0.f, 0.f};
  static_for<kLongWaves>([&](auto u) {
    const float wu = __uint_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_uint(wgt), kRowBcast0 + u.value, 0xf, 0xf, false));
    const f32x4 part = os[u.value][lane];
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = __builtin_fmaf(wu, part[k], r[k]);
  });
  const float inv = 1.f / sum;
  const u32x2 packed = {pack_bf16(r[0] * inv, r[1] * inv), pack_bf16(r[2] * inv, r[3] * inv)};
  *(u32x2*)((uint16_t*)out + ((size_t)tok * kHeads + h) * kDim + 4 * lane) = packed;
  if (lse && lane == 0)
    lse[(size_t)tok * kHeads + h] = (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// ------------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------------
hipError_t launch_append8(const void* k_new, const void* v_new, const int32_t* d_slots, int32_t n_tokens, Layer8 layer,
                          hipStream_t s) {
  if (n_tokens <= 0) return hipSuccess;
  append8_kernel<<<(n_tokens + kAppendTokens8 - 1) / kAppendTokens8, 64 * kAppendTokens8, 0, s>>>(
      (const uint16_t*)k_new, (const uint16_t*)v_new, d_slots, layer.blocks, layer.scales, n_tokens);
  return hipGetLastError();
}

hipError_t launch_append_inline8(const void* k_new, const void* v_new, const InlineIds& blocks, int32_t pos0,
                                 int32_t n_tokens, Layer8 layer, int32_t n_layers, size_t src_layer_stride,
                                 size_t pool_layer_stride, hipStream_t s) {
  if (n_tokens <= 0 || n_layers <= 0) return hipSuccess;
  const int32_t n_pages = ((pos0 + n_tokens + kPage - 1) >> 4) - (pos0 >> 4);
  append_blocks8_kernel<<<dim3(n_pages, n_layers), 256, 0, s>>>((const uint16_t*)k_new, (const uint16_t*)v_new, blocks, pos0,
                                                               n_tokens, layer.blocks, layer.scales, src_layer_stride,
                                                               pool_layer_stride);
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
  if (a.max_parts <= kLongParts) return launch_merge_append(a, nullptr, s, start, stop);
  if (a.n_q <= 0) return hipErrorInvalidValue;
  if (start || stop)
    hipExtLaunchKernelGGL(merge_long_kernel, dim3(kHeads * a.n_q), dim3(64 * kLongWaves), 0, s, start, stop, 0, a.part_acc,
                          a.part_ml, a.out, a.lse, a.n_parts, a.part_off);
  else
    merge_long_kernel<<<kHeads * a.n_q, 64 * kLongWaves, 0, s>>>(a.part_acc, a.part_ml, a.out, a.lse, a.n_parts, a.part_off);
  return hipGetLastError();
}

}  // namespace oxy
