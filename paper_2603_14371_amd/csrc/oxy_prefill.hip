// Attention of a prefill for gfx950 (MI355X): many query tokens of an item over its keys, which lie in a paged cache (bf16 or
// 8 bits) or in the rows that a projection wrote.
//
//   o = sum_j softmax_j(scale <q, k_j>) v_j   over   j < min(len, max(p + 1, full)),   p the query's position
//
// One pass over the keys with the running maximum m and sum l of a row: for a tile of keys S = K q, P = 2^(S - m), l += sum P,
// O += V P.  All eight heads of a token share a key, so a token is eight rows of one matrix product.
#include "oxy_merge.h"
#include "oxy_prefill.h"
#include "oxy_kv8_device.h"

namespace oxy {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// largest / sum of the two lanes n and n + 32
__device__ __forceinline__ float pair_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

enum PrefillSource { SRC_PAGES, SRC_PAGES8, SRC_ROWS };

constexpr int kStep = 32;                       // keys of a tile: two pages
constexpr int kTileBytes = 2 * kPageBytes;      // of K, or of V

struct __align__(16) PrefillLds {
  char k[2][kTileBytes];      // in the order of the cache's pages, see oxy.h
  char v[2][kTileBytes];
  float vs[2][kStep];         // in 8 bits: what the tile's values are to be multiplied by
  uint32_t odd[kDim];         // keys of the tile whose value is not finite in a dim
};

typedef const __attribute__((address_space(1))) void* GlobalPtr;
typedef __attribute__((address_space(3))) void* LdsPtr;

// What a thread holds of a tile between its loads and its stores to LDS.
template <int kSrc>
struct Staged {};
template <>
struct Staged<SRC_PAGES8> {
  u32x4 k[2], v[2];
  uint32_t ks[2], vs;
};
template <>
struct Staged<SRC_ROWS> {
  u32x2 v[8];
};

// Tile of keys key0 .. key0 + 31 on its way to LDS buffer b: requested here.
template <int kSrc>
__device__ __forceinline__ void request_tile(const PrefillArgs& a, PrefillLds& lds, Staged<kSrc>& st, const int b, const int key0,
                                             const int src, const int len) {
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int last_page = (len - 1) >> 4, page0 = key0 >> 4;
  if constexpr (kSrc == SRC_PAGES) {
    // wavefronts 0 and 1 bring the first page, 2 and 3 the second one, half of K and half of V each
    const int pg = wave >> 1, part = (wave & 1) * (kPageBytes / 2);
    const int blk = ((DescPtr)a.tables)[src + min(page0 + pg, last_page)];
    const char* from = a.layer_base + (size_t)blk * kBlockBytes + part + lane * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __builtin_amdgcn_global_load_lds((GlobalPtr)(from + i * 1024), (LdsPtr)(lds.k[b] + pg * kPageBytes + part + i * 1024), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((GlobalPtr)(from + kPageBytes + i * 1024),
                                       (LdsPtr)(lds.v[b] + pg * kPageBytes + part + i * 1024), 16, 0, 0);
    }
  } else if constexpr (kSrc == SRC_PAGES8) {
    const int pg = wave >> 1;
    const int blk = ((DescPtr)a.tables)[src + min(page0 + pg, last_page)];
    const char* from = a.layer_base + (size_t)blk * kBlockBytes8;
    const uint8_t* sc = a.scales + (size_t)blk * kScaleBytes8;
    const int u = t & 127;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      st.k[i] = *(const u32x4*)(from + (u + 128 * i) * 16);
      st.ks[i] = sc[k8_scale_offset(u & 15)];
    }
    // chunks (w, gp, n) and (w, gp + 2, n)
    const int n = u & 15, gp = (u >> 4) & 1, w = u >> 5;
    st.v[0] = *(const u32x4*)(from + kPageBytes8 + v8_chunk_offset(w, gp, n));
    st.v[1] = *(const u32x4*)(from + kPageBytes8 + v8_chunk_offset(w, gp + 2, n));
    // stale exponents behind the item's end may be infinite: 0 instead
    st.vs = key0 + pg * 16 + (u & 15) < len ? sc[v8_scale_offset(u & 15)] : 0;
  } else {
    // K: a lane's 16 bytes are one chunk of the page order
    const int pg = wave >> 1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int chunk = (wave & 1) * 256 + i * 64 + lane;
      const int k8 = chunk & 7, g = (chunk >> 3) & 3, hf = (chunk >> 5) & 1, j = chunk >> 6;
      const int key = min(key0 + pg * 16 + hf * 8 + k8, len - 1);
      __builtin_amdgcn_global_load_lds((GlobalPtr)(a.k + (size_t)(src + key) * a.k_stride + (4 * j + g) * 16),
                                       (LdsPtr)(lds.k[b] + pg * kPageBytes + ((wave & 1) * 256 + i * 64) * 16), 16, 0, 0);
    }
    const int u = t & 127, n = u & 15, gp = (u >> 4) & 1, w = u >> 5;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int key = min(key0 + pg * 16 + 4 * gp + (e & 3) + 8 * (e >> 2), len - 1);
      st.v[e] = *(const u32x2*)(a.v + (size_t)(src + key) * a.v_stride + (64 * w + 4 * n) * 2);
    }
  }
}

// four e4m3 codes -> four bf16 of scale times them
__device__ __forceinline__ u32x2 widen4(const uint32_t codes, const float scale) {
  return (u32x2){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))};
}

// What arrived in registers goes to LDS.
template <int kSrc>
__device__ __forceinline__ void store_tile(PrefillLds& lds, const Staged<kSrc>& st, const int b) {
  const int t = threadIdx.x, u = t & 127, pg = t >> 7;
  char* kp = lds.k[b] + pg * kPageBytes;
  char* vp = lds.v[b] + pg * kPageBytes;
  const int n = u & 15, gp = (u >> 4) & 1, w = u >> 5;
  if constexpr (kSrc == SRC_PAGES8) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int chunk = u + 128 * i, key = chunk & 15, ch = 2 * (chunk >> 4);   // 8 dims each: ch and ch + 1
      const float s = scale_of(st.ks[i]);
      const u32x2 x0 = widen4(st.k[i][0], s), x1 = widen4(st.k[i][1], s), x2 = widen4(st.k[i][2], s), x3 = widen4(st.k[i][3], s);
      *(u32x4*)(kp + k_chunk_offset(ch >> 2, key >> 3, ch & 3, key & 7)) = (u32x4){x0[0], x0[1], x1[0], x1[1]};
      *(u32x4*)(kp + k_chunk_offset((ch + 1) >> 2, key >> 3, (ch + 1) & 3, key & 7)) = (u32x4){x2[0], x2[1], x3[0], x3[1]};
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const u32x2 x = widen4(st.v[0][c], 1.f), y = widen4(st.v[1][c], 1.f);
      *(u32x4*)(vp + v_chunk_offset(w, c, gp, n)) = (u32x4){x[0], x[1], y[0], y[1]};
    }
    if (u < 16) lds.vs[b][pg * 16 + u] = scale_of(st.vs);
  } else if constexpr (kSrc == SRC_ROWS) {
    // eight keys of four dims -> four chunks of a dim's eight keys
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t pick = c & 1 ? 0x07060302u : 0x05040100u;
      u32x4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_perm(st.v[2 * i + 1][c >> 1], st.v[2 * i][c >> 1], pick);
      *(u32x4*)(vp + v_chunk_offset(w, c, gp, n)) = x;
    }
  }
}

// A value that a row does not see, or that nothing was written to, must not reach it, and 0 times what is not finite is NaN.
// In tiles that some row sees a part of, such values are therefore taken as 0 and remembered by dim and key: thread t looks
// after dim t.
__device__ __forceinline__ bool set_odd_aside(PrefillLds& lds, const int b) {
  const int t = threadIdx.x;
  uint32_t odd = 0;
#pragma unroll
  for (int pg = 0; pg < 2; ++pg)
#pragma unroll
    for (int gp = 0; gp < 2; ++gp) {
      u32x4* chunk = (u32x4*)(lds.v[b] + pg * kPageBytes + v_chunk_of_dim(t, gp));
      u32x4 x = *chunk;
      uint32_t bits = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t one = e & 1 ? 0x7f800000u : 0x7f80u;
        if ((x[e >> 1] & one) == one) {
          bits |= 1u << (16 * pg + 4 * gp + (e & 3) + 8 * (e >> 2));
          x[e >> 1] &= e & 1 ? 0xffffu : 0xffff0000u;
        }
      }
      if (bits) *chunk = x;
      odd |= bits;
    }
  lds.odd[t] = odd;
  return __syncthreads_or(odd != 0);
}

template <int kSrc>
__global__ __launch_bounds__(256, 2) void prefill_kernel(const PrefillArgs a) {
  __shared__ PrefillLds lds;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int n = lane & 31, h = lane >> 5;
  const DescPtr rec = (DescPtr)a.work + (size_t)blockIdx.x * kPrefillWords;
  const int tok0 = rec[F_TOK0], n_tok = rec[F_N_TOK], pos = rec[F_POS], full = rec[F_FULL];
  const int kv_begin = rec[F_BEGIN], kv_end = rec[F_END], src = rec[F_SRC], part = rec[F_PART], n_parts = rec[F_N_PARTS],
            len = rec[F_LEN];

  Staged<kSrc> st;
  request_tile<kSrc>(a, lds, st, 0, kv_begin, src, len);

  // this lane's row
  const int mine = 4 * wave + (n >> 3), tok = min(mine, n_tok - 1);
  const bool live = mine < n_tok;
  const int sees = min(len, max(pos + tok + 1, full));   // keys below
  u32x4 q[16];
  const char* q_row = (const char*)a.q + (size_t)(tok0 + tok) * a.q_stride + (n & 7) * (kDim * 2) + 16 * h;
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
  for (int s = 0; s < 16; ++s) q[s] = *(const u32x4*)(q_row + 32 * s) ^ (u32x4){flip, flip, flip, flip};
  float sl2 = fabsf(a.scale * 1.4426950408889634f);
  if (sl2 == 0.f) sl2 = 0x1p-120f;

  // keys that all rows of the workgroup see; that all rows of the wavefront see: those of its first token; the last key that any sees: of its last one
  const int first_tok = min(4 * wave, n_tok - 1), last_tok = min(4 * wave + 3, n_tok - 1);
  const int tile_sees = min(len, max(pos + 1, full));
  const int all_see = min(len, max(pos + first_tok + 1, full));
  const int any_sees = 4 * wave < n_tok ? min(len, max(pos + last_tok + 1, full)) : 0;

  f32x16 o[8] = {};
  float m = -__builtin_inff(), l = 0.f;

  store_tile<kSrc>(lds, st, 0);
  __syncthreads();
  int b = 0;
  for (int key0 = kv_begin; key0 < kv_end; key0 += kStep, b ^= 1) {
    const bool more = key0 + kStep < kv_end;
    if (more) request_tile<kSrc>(a, lds, st, b ^ 1, key0 + kStep, src, len);
    const bool odd = key0 + kStep > tile_sees && set_odd_aside(lds, b);
    if (key0 < any_sees) {
      f32x16 s = {};
      const char* kb = lds.k[b] + (n >> 4) * kPageBytes + ((n >> 3) & 1) * 512 + h * 128 + (n & 7) * 16;
#pragma unroll
      for (int i = 0; i < 16; ++i) s = mfma32(*(const u32x4*)(kb + (i >> 1) * 1024 + (i & 1) * 256), q[i], s);
      const bool masked = key0 + kStep > all_see;
      if (masked) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = key0 + 8 * (r >> 2) + 4 * h + (r & 3);
          s[r] = key < sees ? s[r] : -__builtin_inff();
        }
      }
      float top = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
      top = pair_max(top) * sl2;
      if (__ballot(top > m + kGrow)) {
        const float next = top > m + kGrow ? top : m;   // a row's reference does not go by other rows
        const float alpha = next == m ? 1.f : fast_exp2(m - next);
        m = next;
        l *= alpha;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] *= alpha;
      }
      const float ref = m == -__builtin_inff() ? 0.f : m;
      u32x4 p[2];
      float vs[16];
      if constexpr (kSrc == SRC_PAGES8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 x = *(const f32x4*)&lds.vs[b][8 * i + 4 * h];
#pragma unroll
          for (int e = 0; e < 4; ++e) vs[4 * i + e] = x[e];
        }
      }
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        float x = fast_exp2(__builtin_fmaf(s[r], sl2, -ref)), y = fast_exp2(__builtin_fmaf(s[r + 1], sl2, -ref));
        l += x + y;
        if constexpr (kSrc == SRC_PAGES8) x *= vs[r], y *= vs[r + 1];
        p[r >> 3][(r >> 1) & 3] = pack_bf16(x, y);
      }
      const char* vb = lds.v[b] + h * 256 + (n >> 4) * 512 + (n & 15) * 16;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int pg = 0; pg < 2; ++pg)
          o[i] = mfma32(*(const u32x4*)(vb + pg * kPageBytes + i * 1024), p[pg], o[i]);
      if (odd) {
        const uint32_t* odd_at = lds.odd + 16 * h;
        asm volatile("" : "+v"(odd_at));   // addressed here, and not by registers kept through the loop
        const uint32_t mask = sees - key0 >= kStep ? ~0u : (1u << max(sees - key0, 0)) - 1u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int d = 64 * (i >> 1) + 32 * ((r >> 2) & 1) + 4 * (r & 3) + 2 * (i & 1) + (r >> 3);
            if (odd_at[d] & mask) o[i][r] = __builtin_nanf("");
          }
        }
      }
    }
    if (more) store_tile<kSrc>(lds, st, b ^ 1);
    __syncthreads();
  }

  l = pair_sum(l);
  if (part < 0) {
    const float inv = 1.f / l;
    char* out = (char*)a.out + (size_t)(tok0 + tok) * a.out_stride + (n & 7) * (kDim * 2) + 32 * h;
    if (live) {
#pragma unroll
      for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          u32x4 x[2];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = 4 * half + i;
            x[i >> 1][2 * (i & 1)] = pack_bf16(o[2 * w][r] * inv, o[2 * w][8 + r] * inv);
            x[i >> 1][2 * (i & 1) + 1] = pack_bf16(o[2 * w + 1][r] * inv, o[2 * w + 1][8 + r] * inv);
          }
          *(u32x4*)(out + 128 * w + 64 * half) = x[0];
          *(u32x4*)(out + 128 * w + 64 * half + 16) = x[1];
        }
      if (a.lse && h == 0)
        a.lse[(size_t)(tok0 + tok) * kHeads + (n & 7)] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    }
    return;
  }
  const size_t row = ((size_t)part + (size_t)tok * n_parts) * kHeads + (n & 7);
  char* acc = (char*)(a.part_acc + row * kDim) + 32 * h;
  uint32_t exps = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    float amax = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) amax = fmaxf(amax, fmaxf(fabsf(o[2 * w][r]), fabsf(o[2 * w + 1][r])));
    amax = pair_max(amax);
    const int eb = max(24, min(253, (int)(__float_as_uint(amax) >> 23)));   // as in store_part
    const float up = __uint_as_float((uint32_t)(127 + 14 + 126 - eb) << 23) + (amax - amax);
    exps |= (uint32_t)((eb - 126) & 0xff) << (8 * w);
    if (live) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        u32x4 x[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * half + i;
          x[i >> 1][2 * (i & 1)] = pack_f16(o[2 * w][r] * up, o[2 * w][8 + r] * up);
          x[i >> 1][2 * (i & 1) + 1] = pack_f16(o[2 * w + 1][r] * up, o[2 * w + 1][8 + r] * up);
        }
        *(u32x4*)(acc + 128 * w + 64 * half) = x[0];
        *(u32x4*)(acc + 128 * w + 64 * half + 16) = x[1];
      }
    }
  }
  if (live && h == 0) {
    if (l != l && m == -__builtin_inff()) m = 0.f;   // NaN throughout is not a row without keys
    *(f32x4*)(a.part_ml + row * 4) = (f32x4){m, l, __uint_as_float(exps), 0.f};
  }
}

// A wavefront per token and head, four heads a workgroup.
__global__ __launch_bounds__(256) void prefill_merge_kernel(const PrefillArgs a) {
  const DescPtr rec = (DescPtr)a.merges + (size_t)(blockIdx.x >> 1) * kMergeWords;
  const int tok = rec[0], base = rec[1], np = rec[2];
  const int h = 4 * (blockIdx.x & 1) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const MergeArgs m = {a.part_acc, a.part_ml, (char*)a.out + (size_t)tok * a.out_stride,
                       a.lse ? a.lse + (size_t)tok * kHeads : nullptr, nullptr, nullptr};
  merge_any(m, (size_t)base, np, 0, h, threadIdx.x & 63);
}

hipError_t launch_prefill(const PrefillArgs& a, hipStream_t s) {
  if (a.n_work <= 0) return hipSuccess;
  if (!a.layer_base)
    prefill_kernel<SRC_ROWS><<<a.n_work, 256, 0, s>>>(a);
  else if (a.scales)
    prefill_kernel<SRC_PAGES8><<<a.n_work, 256, 0, s>>>(a);
  else
    prefill_kernel<SRC_PAGES><<<a.n_work, 256, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_merge <= 0) return e;
  prefill_merge_kernel<<<2 * a.n_merge, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace oxy
