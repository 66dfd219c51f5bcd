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

constexpr int kMergeWaves = kHeads;   // of a workgroup

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

// Tiles in use and on their way, in rings.  kPipe: one workgroup a CU, see prefill_pipe_kernel; else two.
template <int kSrc, bool kPipe>
struct PrefillLds {
  static constexpr bool kIs8 = kSrc == SRC_PAGES8;
  static constexpr int kKeys = kPipe ? (kIs8 ? 2 : 4) : (kIs8 ? 1 : 2), kRaw = kPipe ? 3 : 1;
  static constexpr int kValues = kPipe ? (kSrc == SRC_PAGES ? 5 : 4) : kKeys;
  char k[kKeys][kTileBytes], v[kValues][kTileBytes];
  float vs[kValues][kStep];   // in 8 bits: scales of the values
  uint32_t odd[kDim];         // keys of a tile whose value is not finite in a dim
  uint32_t found[4];          // [wavefront]: whether it found one
  // In 8 bits: codes and exponents as they lie in the pages, a part for each wavefront, which widens what it requested.
  struct Raw {
    char codes[kRaw][4][4096];   // [wavefront]: two pieces of 1 KiB of a K page, two of a V page
    char exps[kRaw][4][256];     // exponents of a page, then nothing
  };
  struct NoRaw {};
  std::conditional_t<kIs8, Raw, NoRaw> raw;
  uint32_t spare[4][64];      // [wavefront]: what a request in the place of a tile's goes to
};

// `size` bytes a lane to LDS, lane after lane, from offset + more + kImm behind a base that is the same for the wavefront; zeros for
// offset + kImm of `bytes` and above.  kImm counts in LDS too.  A buffer operation, which counts among vector memory operations
// only: behind one with a full address the compiler waits for all reads of LDS at once.
template <int kSize, int kImm = 0>
__device__ __forceinline__ void to_lds(const void* base, const uint32_t bytes, const uint32_t offset, void* to, const int more = 0) {
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, 0x00027000);
  const auto lds = (__attribute__((address_space(3))) void*)to;
  if constexpr (kSize == 16)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, lds, 16, offset, more, kImm, 0);
  else
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, lds, 4, offset, more, kImm, 0);
}
// Waits until at most n of a wavefront's vector memory operations are left.
//
// The compiler waits by itself, for everything, in front of a read of LDS that may be of what is being requested.  It compares a
// read with the kernel's first request only, so that one goes to a place that nothing reads (`spare`), and the reads' indices
// are such that their ranges are seen.
template <int n>
__device__ __forceinline__ void wait_vector() {
  static_assert(n >= 0 && n < 64, "");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (n & 15) | (n >> 4) << 14);
}
// What a workgroup wrote to LDS before is seen behind it; requests stay in flight (a fence of the workgroup's scope would wait
// for those too).
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_s_waitcnt(0xc07f);   // LDS operations only
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// LDS serves sixteen lanes of 16 bytes at a time, from 256 bytes of banks.  Rows lie there as they do in memory, 512 bytes each,
// their 16-byte chunks changing places so that the lanes that are served together find theirs in different banks: sixteen keys of
// one chunk (K), four keys of four chunks (V, read transposed).  Chunks of a page change places within a KiB, so that a product's
// operands lie in the order of the lanes.  (A wavefront's read of K 8.3 -> 7.6 cycles, of V 10.2 -> 7.5.)
__device__ __forceinline__ int k_row_swap(const int key) { return key & 15; }
__device__ __forceinline__ int v_row_swap(const int key) { return (key & 1) * 4 + (key >> 1 & 1); }
__device__ __forceinline__ int k_lds_offset(const int t, const int g, const int key) { return t * 1024 + g * 256 + key * 16; }
__device__ __forceinline__ int v_lds_offset(const int w, const int c, const int gp, const int n) {
  return (2 * w + (c >> 1)) * 1024 + gp * 512 + (c & 1) * 256 + n * 16;
}

// What a wavefront brings of a tile: its share of the keys (kWhat 0; in 8 bits of keys and values) or of the values (1), four
// operations (in 8 bits five) to LDS.  Wavefronts 0 and 1 bring the tile's first 16 keys, 2 and 3 the others.
template <int kSrc>
constexpr int kPartOps = kSrc == SRC_PAGES8 ? 5 : 4;
template <int kSrc>
struct Bring {
  const char* base;
  const char* second;      // in 8 bits: the exponents; of rows: the first row of V
  uint32_t k_stride, v_stride;   // of rows
  int keys;                // of rows: from the wavefront's first one of tile 0 on
  int pg, side, wave;
  uint32_t at[2];          // pages: where a lane's chunk of K, of V comes from; in 8 bits: the lane's 16 bytes
  uint32_t row[2];         // rows: the second of two rows

  __device__ __forceinline__ Bring(const char* from, const void* from2, const size_t ks, const size_t vs, const int src,
                                   const int key0, const int len, const int w, const int lane)
      : base(from), second((const char*)from2), k_stride((uint32_t)ks), v_stride((uint32_t)vs), keys(len - key0 - 8 * w),
        pg(w >> 1), side(w & 1), wave(w) {
    if constexpr (kSrc == SRC_PAGES) {
      at[0] = k_chunk_offset(0, (lane >> 3) & 1, lane >> 4, lane & 7);
      at[1] = v_chunk_offset(0, (lane >> 4) & 1, lane >> 5, lane & 15);
    } else if constexpr (kSrc == SRC_PAGES8) {
      at[0] = lane * 16, at[1] = lane * 4;
    } else {
      base += (size_t)(src + key0 + 8 * w) * ks, second += (size_t)(src + key0 + 8 * w) * vs;
      at[0] = ((lane & 31) ^ (8 * side + (lane >> 5))) * 16, at[1] = ((lane & 31) ^ ((lane >> 5) * 4)) * 16;
      row[0] = (lane >> 5) * k_stride, row[1] = (lane >> 5) * v_stride;
    }
  }
  // Operation i for a tile.  blk: the wavefront's page, of rows: nothing.  there: whether there is such a tile; else the buffer
  // is of no bytes.
  template <int kWhat, int i, class Lds>
  __device__ __forceinline__ void part(Lds& lds, const int tile, const bool there, const int blk) const {
    if constexpr (kSrc == SRC_PAGES) {
      char* to = kWhat ? lds.v[tile % Lds::kValues] : lds.k[tile % Lds::kKeys];
      to_lds<16, i * 1024>(base + (size_t)blk * kBlockBytes, there ? kBlockBytes : 0, at[kWhat],
                           to + pg * kPageBytes + side * (kPageBytes / 2), kWhat * kPageBytes + side * (kPageBytes / 2));
    } else if constexpr (kSrc == SRC_PAGES8) {
      // two K chunks of all keys and half of the dims; two V chunks of all keys of half of the dims
      if constexpr (i < 4)
        to_lds<16>(base + (size_t)blk * kBlockBytes8, there ? kBlockBytes8 : 0, at[0], lds.raw.codes[tile % Lds::kRaw][wave] + i * 1024,
                   i < 2 ? side * 1024 + i * 2048 : kPageBytes8 + side * 2048 + (i - 2) * 1024);
      else   // 8 lanes, then 0
        to_lds<4>(second + (size_t)blk * kScaleBytes8, there ? kScaleBytes8 : 0, at[1], lds.raw.exps[tile % Lds::kRaw][wave]);
    } else {   // two rows; those behind the last one are 0
      const uint32_t stride = kWhat ? v_stride : k_stride;
      const int left = there ? min(keys - tile * kStep, 8) : 0;
      const uint32_t bytes = left > 0 ? (left - 1) * stride + kDim * 2 : 0;
      to_lds<16>((kWhat ? second : base) + (size_t)(tile * kStep) * stride, bytes,
                 (at[kWhat] ^ (kWhat ? (i & 1) * 16 : i * 32)) + (row[kWhat] + 2 * i * stride),
                 (kWhat ? lds.v[tile % Lds::kValues] : lds.k[tile % Lds::kKeys]) + (8 * wave + 2 * i) * 512);
    }
  }
  template <int kWhat, class Lds>
  __device__ __forceinline__ void all(Lds& lds, const int tile, const bool there, const int blk) const {
    static_for<kPartOps<kSrc>>([&](auto i) { part<kWhat, i.value>(lds, tile, there, blk); });
  }
};

// four e4m3 codes -> four bf16 of scale times them
__device__ __forceinline__ u32x2 widen4(const uint32_t codes, const float scale) {
  return (u32x2){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))};
}
// A wavefront's part of a tile in 8 bits, from codes to the page order of bf16, in nine pieces.  Keys with their scale; the scales
// of the values go into the probabilities (see the kernels), since four keys share a word.
struct Widen {
  u32x4 x[4];
  float scale;
  uint32_t v_exp;
  int wave, key, from[2], to[2];   // key of the tile whose scales the lane reads; offsets in its codes, in the tile: of K, of V

  __device__ __forceinline__ Widen(const int w, const int lane) : wave(w), key(16 * (w >> 1) + (lane & 15)) {
    const int side = w & 1, n = lane & 15, gp = (lane >> 4) & 1, half = lane >> 5, ch = 2 * (4 * side + (lane >> 4));
    from[0] = lane * 16, from[1] = 2048 + half * 1024 + (gp * 16 + n) * 16;
    to[0] = (w >> 1) * kPageBytes + k_lds_offset(ch >> 2, ch & 3, n);   // ch: eight dims
    to[1] = (w >> 1) * kPageBytes + v_lds_offset(2 * side + half, 0, gp, n);
  }
  // left: keys of the item from the tile's first on
  template <int i, class Lds>
  __device__ __forceinline__ void piece(Lds& lds, const int tile, const int left) {
    const int r = tile % Lds::kRaw;
    if constexpr (i == 0) {   // all reads before the first write: behind a write the compiler waits for all requests
      const char* codes = lds.raw.codes[r][wave];
      const char* exps = lds.raw.exps[r][wave];
      x[0] = *(const u32x4*)(codes + from[0]), x[1] = *(const u32x4*)(codes + from[0] + 1024);
      x[2] = *(const u32x4*)(codes + from[1]), x[3] = *(const u32x4*)(codes + from[1] + 512);   // keys 4gp.. and 8 + 4gp..
      scale = scale_of((uint8_t)exps[k8_scale_offset(key & 15)]);
      v_exp = (uint8_t)exps[v8_scale_offset(key & 15)];
    } else if constexpr (i < 5) {
      constexpr int half = (i - 1) >> 1, c = (i - 1) & 1;
      if constexpr (i == 1)   // stale exponents behind the item's end may be infinite: 0 instead; by four lanes each
        lds.vs[tile % Lds::kValues][key] = key < left ? scale_of(v_exp) : 0.f;
      const u32x2 a = widen4(x[half][2 * c], scale), b = widen4(x[half][2 * c + 1], scale);
      *(u32x4*)(lds.k[tile % Lds::kKeys] + to[0] + half * 4096 + c * 256) = (u32x4){a[0], a[1], b[0], b[1]};
    } else {
      constexpr int c = i - 5;
      const u32x2 a = widen4(x[2][c], 1.f), b = widen4(x[3][c], 1.f);
      *(u32x4*)(lds.v[tile % Lds::kValues] + to[1] + (c >> 1) * 1024 + (c & 1) * 256) = (u32x4){a[0], a[1], b[0], b[1]};
    }
  }
};

// A value that a row does not see, or that nothing was written to, must not reach it, and 0 times what is not finite is NaN.
// In tiles that some row sees a part of, such values are therefore looked for, which costs a barrier.
__device__ __forceinline__ uint32_t odd_pair(const uint32_t x) {
  return (uint32_t)((x & 0x7f80u) == 0x7f80u) | (uint32_t)((x & 0x7f800000u) == 0x7f800000u);
}
template <class Lds>
__device__ __forceinline__ bool has_odd(Lds& lds, const int b, const int wave) {
  const int t = threadIdx.x & 255;
  uint32_t odd = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32x4 x = *(const u32x4*)(lds.v[b] + (i * 256 + t) * 16);
    odd |= odd_pair(x[0]) | odd_pair(x[1]) | odd_pair(x[2]) | odd_pair(x[3]);
  }
  const bool mine = __ballot(odd != 0) != 0;
  if ((t & 63) == 0) lds.found[wave] = mine;
  lds_barrier();
  const u32x4 all = *(const u32x4*)lds.found;
  return (all[0] | all[1] | all[2] | all[3]) != 0;
}
// Such values are taken as 0 and remembered by dim and key: thread t looks after dim t.
template <int kSrc, class Lds>
__device__ __forceinline__ void set_odd_aside(Lds& lds, const int b) {
  const int t = threadIdx.x & 255;
  uint32_t odd = 0;
#pragma unroll 1
  for (int key = 0; key < kStep; ++key) {
    char* at = lds.v[b];
    if (kSrc == SRC_ROWS)
      at += key * 512 + ((t >> 3) ^ v_row_swap(key)) * 16 + (t & 7) * 2;
    else
      at += (key >> 4) * kPageBytes + v_lds_offset(t >> 6, t & 3, (key >> 2) & 1, (t >> 2) & 15) + v_slot_of_key(key & 15) * 2;
    uint16_t* const x = (uint16_t*)at;
    if ((*x & 0x7f80u) == 0x7f80u) *x = 0, odd |= 1u << key;
  }
  lds.odd[t] = odd;
  lds_barrier();
}

// Four keys of one dim from rows of LDS: within 16 lanes, lane 4a + b names four dims of key a, and lane i receives dim i of
// the sixteen, keys 0 to 3.
__device__ __forceinline__ u32x2 read_turned(const char* at) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at));
}
// The dim, but for 16h, that register r of product j holds: lane half h has 16 dims in a row, of pages in the order of their
// chunks.
template <int kSrc>
constexpr int dim_of(const int j, const int r) {
  return kSrc == SRC_ROWS ? 32 * j + r : 64 * (j >> 1) + 32 * ((r >> 2) & 1) + 4 * (r & 3) + 2 * (j & 1) + (r >> 3);
}
// Register of dim d + 16h, d in [32x, 32x + 16).
template <int kSrc>
__device__ __forceinline__ float of_dim(const f32x16 (&o)[8], const int d) {
  if constexpr (kSrc == SRC_ROWS) return o[d >> 5][d & 15];
  return o[2 * (d >> 6) + ((d >> 1) & 1)][8 * (d & 1) + 4 * ((d >> 5) & 1) + ((d >> 2) & 3)];
}

// Sixteen products whose operands come from LDS: those of the first kAhead are read at once, then each product is followed by
// the read of the one kAhead on.  The order is kept from the compiler, which reads one or two ahead.
template <int kAhead, class Read, class Multiply>
__device__ __forceinline__ void products(const Read& read, const Multiply& multiply) {
  constexpr int kAluPasses = 0x6;
  u32x4 x[kAhead];
  static_for<kAhead>([&](auto j) { x[j.value] = read(j); });
  __builtin_amdgcn_sched_barrier(kAluPasses);
  static_for<16>([&](auto j) {
    multiply(j, x[j.value % kAhead]);
    if constexpr (j.value + kAhead < 16) x[j.value % kAhead] = read(std::integral_constant<int, j.value + kAhead>());
    __builtin_amdgcn_sched_barrier(kAluPasses);
  });
}
// The same with other work in the time that a product takes, between(j) behind product j; the first operands have been read, and
// those of the next sixteen products are (`next`) behind the last ones of these.
template <int kAhead, class Read, class Next, class Multiply, class Between>
__device__ __forceinline__ void products_with(u32x4 (&x)[kAhead], const Read& read, const Next& next, const Multiply& multiply,
                                              const Between& between) {
  static_for<16>([&](auto j) {
    multiply(j, x[j.value % kAhead]);
    if constexpr (j.value + kAhead < 16)
      x[j.value % kAhead] = read(std::integral_constant<int, j.value + kAhead>());
    else
      next(std::integral_constant<int, j.value + kAhead - 16>(), x[j.value % kAhead]);
    between(j);
    __builtin_amdgcn_sched_barrier(0);
  });
}

// A wavefront's rows leave through LDS (8 KiB of its own), as whole lines, half of the dims at a time: outputs, `scale` times
// the sums, in bf16; or split results, see store_part, whose exponents go to exps.  to: the first of its four tokens, of which
// `left` are there.
template <int kSrc, bool kDirect>
__device__ __forceinline__ void store_rows(const f32x16 (&o)[8], const float scale, uint32_t& exps, char* lds, char* to,
                                           const size_t token_stride, const int left, const int lane) {
  const int n = lane & 31, h = lane >> 5;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
#pragma unroll
    for (int w = 2 * half; w < 2 * half + 2; ++w) {
      float up = scale;
      if constexpr (!kDirect) {
        float amax = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) amax = fmaxf(fmaxf(amax, fabsf(o[2 * w][r])), fabsf(o[2 * w + 1][r]));
        amax = pair_max(amax);
        const int eb = max(24, min(253, (int)(__float_as_uint(amax) >> 23)));
        up = __uint_as_float((uint32_t)(127 + 14 + 126 - eb) << 23) + (amax - amax);
        exps |= (uint32_t)((eb - 126) & 0xff) << (8 * w);
      }
#pragma unroll
      for (int d = 64 * w; d < 64 * w + 64; d += 32)
#pragma unroll
        for (int e0 = 0; e0 < 16; e0 += 8) {
          u32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x0 = of_dim<kSrc>(o, d + e0 + 2 * e) * up, x1 = of_dim<kSrc>(o, d + e0 + 2 * e + 1) * up;
            x[e] = kDirect ? pack_bf16(x0, x1) : pack_f16(x0, x1);
          }
          const int chunk = (d & 127) / 8 + e0 / 8 + 2 * h;
          *(u32x4*)(lds + n * 256 + (chunk ^ (n & 15)) * 16) = x;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = 4 * i + (lane >> 4), chunk = (lane & 15) ^ (row & 15);
      const u32x4 x = *(const u32x4*)(lds + row * 256 + (lane & 15) * 16);
      if ((i >> 1) < left) *(u32x4*)(to + (i >> 1) * token_stride + (row & 7) * (kDim * 2) + 256 * half + chunk * 16) = x;
    }
  }
}

// What a workgroup needs behind its first loads.
struct PrefillLate {
  void* out;
  float* lse;
  size_t out_stride;
  const int32_t* tables;
  uint16_t* part_acc;
  float* part_ml;
  float scale;
};

template <int kSrc>
__global__ __launch_bounds__(256, 2) void prefill_kernel(const int32_t* work, const char* q_rows, const size_t q_stride,
                                                         const char* base, const void* second, const size_t k_stride,
                                                         const size_t v_stride, const PrefillLate a) {
  constexpr bool kRaw = kSrc == SRC_PAGES8;
  using Lds = PrefillLds<kSrc, false>;
  __shared__ __align__(16) Lds lds;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6) & 3;
  const int n = lane & 31, h = lane >> 5;
  const DescPtr rec = (DescPtr)work + (size_t)blockIdx.x * kPrefillWords;
  const int tok0 = rec[F_TOK0], n_tok = rec[F_N_TOK], pos = rec[F_POS], full = rec[F_FULL];
  const int kv_begin = rec[F_BEGIN], kv_end = rec[F_END], src = rec[F_SRC], part = rec[F_PART], n_parts = rec[F_N_PARTS],
            len = rec[F_LEN];
  const int n_tiles = (kv_end - kv_begin + kStep - 1) / kStep;

  // the wavefront's page of a tile
  auto page_of = [&](const int tile) {
    if constexpr (kSrc == SRC_ROWS) return 0;
    const int at = 2 * tile + (wave >> 1), page = min((kv_begin >> 4) + at, (len - 1) >> 4);
    return at < kPrefillPages ? rec[F_PAGES + at] : ((DescPtr)a.tables)[src + page];
  };
  auto request = [&](const int tile, const int blk) {
    int at = lane;
    asm volatile("" : "+v"(at));   // addresses are made here, and not kept in registers through the loop
    const Bring<kSrc> bring(base, second, k_stride, v_stride, src, kv_begin, len, wave, at & 63);
    bring.template all<0>(lds, tile, true, blk);
    if constexpr (!kRaw) bring.template all<1>(lds, tile, true, blk);
  };

  // a request that is there to be waited behind
  auto request_spare = [&]() {
    to_lds<4>(work + (size_t)blockIdx.x * kPrefillWords, kPrefillWords * 4, lane * 4, lds.spare[wave]);
  };
  request_spare();   // the first of all, see wait_vector
  request(0, page_of(0));

  // The wavefront's 32 query rows, four tokens' eight heads, come through LDS, as whole lines: a row a lane, as the products
  // take them, would be 64 pieces of 16 bytes each in a line of its own.  Half at a time, into buffers that the first tile does
  // not go to.
  u32x4 q[16];
  char* const q_at = (wave < 2 ? lds.k[Lds::kKeys - 1] : lds.v[Lds::kValues - 1]) + (wave & 1) * 8192;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int two = half * 16 + 2 * i, row = two + (lane >> 5);
      const char* from = q_rows + (size_t)(tok0 + min(4 * wave + (two >> 3), n_tok - 1)) * q_stride;
      to_lds<16>(from, kHeads * kDim * 2, (row & 7) * (kDim * 2) + ((lane & 31) ^ k_row_swap(row)) * 16, q_at + i * 1024);
    }
    request_spare();
    wait_vector<1>();
    if ((n >> 4) == half) {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        q[j] = *(const u32x4*)(q_at + (n & 15) * 512 + ((2 * j + h) ^ k_row_swap(n)) * 16);
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);   // read, before the other half comes there
  }
  if constexpr (kRaw) lds_barrier();   // the first tile is widened into where rows were
  int next_page = page_of(1);

  // this lane's row
  const int mine = 4 * wave + (n >> 3), tok = min(mine, n_tok - 1);
  const int sees = min(len, max(pos + tok + 1, full));   // keys below
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
  for (int s = 0; s < 16; ++s) q[s] ^= (u32x4){flip, flip, flip, flip};
  float sl2 = fabsf(a.scale * 1.4426950408889634f);
  if (sl2 == 0.f) sl2 = 0x1p-120f;

  // keys that all rows of the workgroup see; that all rows of the wavefront see; the last key that any of them sees
  const int first_tok = min(4 * wave, n_tok - 1), last_tok = min(4 * wave + 3, n_tok - 1);
  const int tile_sees = min(len, max(pos + 1, full));
  const int all_see = min(len, max(pos + first_tok + 1, full));
  const int any_sees = 4 * wave < n_tok ? min(len, max(pos + last_tok + 1, full)) : 0;

  f32x16 o[8] = {};
  float m = -__builtin_inff(), l = 0.f;

  for (int i = 0; i < n_tiles; ++i) {
    const int key0 = kv_begin + i * kStep;
    // Tile i has arrived: behind it there is a spare request.  The first one lies in front of the queries.
    if (i > 0) wait_vector<1>();
    if constexpr (kRaw) {
      int at = lane;
      asm volatile("" : "+v"(at));
      at &= 63;
      Widen widen(wave, at);
      static_for<9>([&](auto j) { widen.template piece<j.value>(lds, i, len - key0); });
    }
    lds_barrier();
    // nobody reads the buffers any more that the next requests go to
    if (i + 1 < n_tiles) {
      request(i + 1, next_page);
      next_page = page_of(i + 2);
    }
    request_spare();
    const int bk = i % Lds::kKeys, bv = i % Lds::kValues;
    const bool odd = key0 + kStep > tile_sees && has_odd(lds, bv, wave);
    if (odd) set_odd_aside<kSrc>(lds, bv);
    if (key0 < any_sees) {
      f32x16 s = {};
      constexpr int kReads = kSrc == SRC_PAGES ? 5 : kSrc == SRC_ROWS ? 4 : 3;   // more would not fit the registers
      int turn = h ^ k_row_swap(n);
      if constexpr (kSrc == SRC_ROWS) asm volatile("" : "+v"(turn));   // see request
      const char* kb = lds.k[bk] + (kSrc == SRC_ROWS ? n * 512 : (n >> 4) * kPageBytes + h * 256 + (n & 15) * 16);
      products<kReads>(
          [&](auto at) {
            constexpr int j = at.value;
            if constexpr (kSrc == SRC_ROWS)
              return *(const u32x4*)(kb + ((2 * j) ^ turn) * 16);
            else
              return *(const u32x4*)(kb + j * 512);
          },
          [&](auto at, const u32x4 k) { s = mfma32(k, q[at.value], s); });
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
        for (int j = 0; j < 8; ++j) o[j] *= alpha;
      }
      const float ref = m == -__builtin_inff() ? 0.f : m;
      u32x4 p[2];
      const char* vs_at = (char*)lds.vs[bv] + 16 * h;
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        float x = fast_exp2(__builtin_fmaf(s[r], sl2, -ref)), y = fast_exp2(__builtin_fmaf(s[r + 1], sl2, -ref));
        l += x + y;
        if constexpr (kRaw) {
          const f32x2 vs = *(const f32x2*)(vs_at + 4 * (8 * (r >> 2) + (r & 3)));
          x *= vs[0], y *= vs[1];
        }
        p[r >> 3][(r >> 1) & 3] = pack_bf16(x, y);
      }
      // Rows: lane 16x + i of each half reads keys 4h + i / 4 (and 8 on), group 4x + i % 4 of four dims, see dim_of
      const int g = ((lane >> 4) & 1) * 4 + (lane & 3), key = 4 * h + ((lane >> 2) & 3), c = 2 * (g & 1) + (g >> 2);
      int v_turn = c ^ v_row_swap(key);
      if constexpr (kSrc == SRC_ROWS) asm volatile("" : "+v"(v_turn));
      const char* vb = lds.v[bv] + (kSrc == SRC_ROWS ? key * 512 + (g >> 1 & 1) * 8 : lane * 16);
      products<kReads>(
          [&](auto at) {
            constexpr int pg = at.value >> 3, j = at.value & 7;
            if constexpr (kSrc == SRC_ROWS) {
              const char* from = vb + pg * 8192 + ((4 * j) ^ v_turn) * 16;
              const u32x2 lo = read_turned(from), hi = read_turned(from + 8 * 512);
              return (u32x4){lo[0], lo[1], hi[0], hi[1]};
            } else {
              return *(const u32x4*)(vb + pg * kPageBytes + j * 1024);
            }
          },
          [&](auto at, const u32x4 v) { o[at.value & 7] = mfma32(v, p[at.value >> 3], o[at.value & 7]); });
      if (odd) {
        auto odd_at = (const __attribute__((address_space(3))) uint32_t*)(lds.odd + 16 * h);
        asm volatile("" : "+v"(odd_at));   // addressed here, and not by registers kept through the loop
        const uint32_t mask = sees - key0 >= kStep ? ~0u : (1u << max(sees - key0, 0)) - 1u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float x = odd_at[dim_of<kSrc>(j, r)] & mask ? __builtin_nanf("") : o[j][r];
            asm volatile("" : "+v"(x));   // chosen here, and not where this path meets the other one
            o[j][r] = x;
          }
        }
      }
    }
    if constexpr (kRaw) lds_barrier();   // one buffer: the next tile is widened into it
  }

  l = pair_sum(l);
  lds_barrier();
  if (part < 0) {
    uint32_t exps;
    store_rows<kSrc, true>(o, 1.f / l, exps, (char*)&lds + wave * 8192, (char*)a.out + (size_t)(tok0 + 4 * wave) * a.out_stride,
                           a.out_stride, n_tok - 4 * wave, lane);
    if (a.lse && mine < n_tok && h == 0)
      a.lse[(size_t)(tok0 + mine) * kHeads + (n & 7)] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  } else {
    const size_t part0 = (size_t)part + (size_t)(4 * wave) * n_parts;
    uint32_t exps = 0;
    store_rows<kSrc, false>(o, 0.f, exps, (char*)&lds + wave * 8192, (char*)a.part_acc + part0 * (kHeads * kDim * 2),
                            (size_t)n_parts * (kHeads * kDim * 2), n_tok - 4 * wave, lane);
    if (l != l && m == -__builtin_inff()) m = 0.f;   // NaN throughout is not a row without keys
    if (mine < n_tok && h == 0)
      *(f32x4*)(a.part_ml + ((part0 + (size_t)(n >> 3) * n_parts) * kHeads + (n & 7)) * 4) =
          (f32x4){m, l, __uint_as_float(exps), 0.f};
  }
}

// One workgroup a CU, one wavefront a SIMD: what a wavefront computes by its vector instructions it does while its matrix
// products run.  Around tile i: the products of tile i - 1's values, and meanwhile the maxima of tile i's logits; then the
// products of tile i + 1's keys, and meanwhile the exponentials of tile i.
template <int kSrc>
__global__ __launch_bounds__(256, 1) void prefill_pipe_kernel(const int32_t* work, const char* q_rows, const size_t q_stride,
                                                              const char* base, const void* second, const size_t k_stride,
                                                              const size_t v_stride, const PrefillLate a) {
  constexpr bool kRaw = kSrc == SRC_PAGES8;
  using Lds = PrefillLds<kSrc, true>;
  __shared__ __align__(16) Lds lds;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6) & 3;
  const int n = lane & 31, h = lane >> 5;
  const DescPtr rec = (DescPtr)work + (size_t)blockIdx.x * kPrefillWords;
  const int tok0 = rec[F_TOK0], n_tok = rec[F_N_TOK], pos = rec[F_POS], full = rec[F_FULL];
  const int kv_begin = rec[F_BEGIN], kv_end = rec[F_END], src = rec[F_SRC], part = rec[F_PART], n_parts = rec[F_N_PARTS],
            len = rec[F_LEN];
  const int n_tiles = (kv_end - kv_begin + kStep - 1) / kStep;

  // the wavefront's page of a tile
  auto page_of = [&](const int tile) {
    if constexpr (kSrc == SRC_ROWS) return 0;
    const int at = 2 * tile + (wave >> 1), page = min((kv_begin >> 4) + at, (len - 1) >> 4);
    return at < kPrefillPages ? rec[F_PAGES + at] : ((DescPtr)a.tables)[src + page];
  };
  // Tiles behind the last one are requested too, as buffers of no bytes: every step has as many operations as every other.
  const Bring<kSrc> bring(base, second, k_stride, v_stride, src, kv_begin, len, wave, lane);
  auto request = [&](auto what, const int tile, const int blk) { bring.template all<what.value>(lds, tile, tile < n_tiles, blk); };
  constexpr std::integral_constant<int, 0> kKeys;
  constexpr std::integral_constant<int, 1> kValues;
  to_lds<4>(work + (size_t)blockIdx.x * kPrefillWords, kPrefillWords * 4, lane * 4, lds.spare[wave]);   // see wait_vector
  constexpr int kValuesTo = kSrc == SRC_PAGES ? 3 : 2;   // tiles ahead that values are requested, keys four
  const int page[3] = {page_of(0), page_of(1), page_of(2)};
  request(kKeys, 0, page[0]);

  // The wavefront's 32 query rows, four tokens' eight heads, come through LDS, as whole lines: a row a lane, as the products
  // take them, would be 64 pieces of 16 bytes each in a line of its own.
  u32x4 q[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int row = 2 * i + (lane >> 5);
    const char* from = q_rows + (size_t)(tok0 + min(4 * wave + (i >> 2), n_tok - 1)) * q_stride;
    to_lds<16>(from, kHeads * kDim * 2, (row & 7) * (kDim * 2) + ((lane & 31) ^ k_row_swap(row)) * 16, lds.v[wave] + i * 1024);
  }
  request(kKeys, 1, page[1]);
  if constexpr (kRaw) {
    request(kKeys, 2, page[2]);
    wait_vector<10>();
  } else {
    wait_vector<4>();
  }
#pragma unroll
  for (int j = 0; j < 16; ++j)
    q[j] = *(const u32x4*)(lds.v[wave] + n * 512 + ((2 * j + h) ^ k_row_swap(n)) * 16);
  lds_barrier();   // values go to where rows were
  int next_page = page_of(3), values_page = 0;   // of the tiles whose keys, whose values are requested next
  Widen widen(wave, lane);
  auto widen_piece = [&](const int tile, auto piece) {
    if constexpr (kRaw) {
      widen.template piece<piece.value>(lds, tile, len - kv_begin - tile * kStep);
    }
  };
  auto widen_all = [&](const int tile) { static_for<9>([&](auto i) { widen_piece(tile, i); }); };
  if constexpr (kRaw) {
    widen_all(0);
    request(kKeys, 3, next_page);
    next_page = page_of(4);
    wait_vector<10>();
    widen_all(1);
    request(kKeys, 4, next_page);
    next_page = page_of(5);
    lds_barrier();
  } else {
    // as steps -3 to -1 would
    if constexpr (kValuesTo == 3) request(kValues, 0, page[0]);
    request(kKeys, 2, page[2]);
    request(kValues, kValuesTo - 2, page[kValuesTo - 2]);
    request(kKeys, 3, next_page);
    request(kValues, kValuesTo - 1, page[kValuesTo - 1]);
    values_page = next_page;
    next_page = page_of(4);
  }

  // this lane's row
  const int mine = 4 * wave + (n >> 3), tok = min(mine, n_tok - 1);
  const int sees = min(len, max(pos + tok + 1, full));   // keys below
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
  for (int s = 0; s < 16; ++s) q[s] ^= (u32x4){flip, flip, flip, flip};
  float sl2 = fabsf(a.scale * 1.4426950408889634f);
  if (sl2 == 0.f) sl2 = 0x1p-120f;

  // keys that all rows of the workgroup see; that all rows of the wavefront see
  const int tile_sees = min(len, max(pos + 1, full));
  const int all_see = min(len, max(pos + min(4 * wave, n_tok - 1) + 1, full));

  f32x16 o[8] = {}, s = {};
  float m = -__builtin_inff(), l = 0.f;
  u32x4 p[2] = {};

  constexpr int kReads = 4;
  u32x4 x[kReads];   // operands read ahead
  auto read_key = [&](const int tile, auto at) {
    constexpr int j = at.value;
    const char* from = lds.k[tile % Lds::kKeys];
    if constexpr (kSrc == SRC_ROWS)
      return *(const u32x4*)(from + n * 512 + ((2 * j + h) ^ k_row_swap(n)) * 16);
    else
      return *(const u32x4*)(from + (n >> 4) * kPageBytes + h * 256 + (n & 15) * 16 + j * 512);
  };
  // Rows: lane 16x + i of each half reads keys 4h + i / 4 (and 8 on), group 4x + i % 4 of four dims, see dim_of
  const int g = ((lane >> 4) & 1) * 4 + (lane & 3), key = 4 * h + ((lane >> 2) & 3), c = 2 * (g & 1) + (g >> 2);
  auto read_value = [&](const int tile, auto at) {
    constexpr int pg = at.value >> 3, j = at.value & 7;
    const char* vb = lds.v[tile % Lds::kValues];
    if constexpr (kSrc == SRC_ROWS) {
      const char* from = vb + key * 512 + (g >> 1 & 1) * 8 + pg * 8192 + ((4 * j + c) ^ v_row_swap(key)) * 16;
      const u32x2 lo = read_turned(from), hi = read_turned(from + 8 * 512);
      return (u32x4){lo[0], lo[1], hi[0], hi[1]};
    } else {
      return *(const u32x4*)(vb + lane * 16 + pg * kPageBytes + j * 1024);
    }
  };
  // The first values of a tile are read behind the products of the keys, but for rows: a transposed read waits for all requests.
  constexpr bool kValuesAhead = kSrc != SRC_ROWS;
  auto first_values = [&](const int tile) { static_for<kReads>([&](auto j) { x[j.value] = read_value(tile, j); }); };
  // products of a tile's values, and between them what there is to do
  auto add_values = [&](const int tile, const auto& between) {
    products_with(x, [&](auto at) { return read_value(tile, at); }, [&](auto at, u32x4& y) { y = read_key(tile + 2, at); },
                  [&](auto at, const u32x4 v) { o[at.value & 7] = mfma32(v, p[at.value >> 3], o[at.value & 7]); }, between);
  };
  auto mark_odd = [&](const int tile) {
    const int key0 = kv_begin + tile * kStep;
    auto odd_at = (const __attribute__((address_space(3))) uint32_t*)(lds.odd + 16 * h);
    asm volatile("" : "+v"(odd_at));   // addressed here, and not by registers kept through the loop
    const uint32_t mask = sees - key0 >= kStep ? ~0u : (1u << max(sees - key0, 0)) - 1u;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float x = odd_at[dim_of<kSrc>(j, r)] & mask ? __builtin_nanf("") : o[j][r];
        asm volatile("" : "+v"(x));   // chosen here, and not where this path meets the other one
        o[j][r] = x;
      }
    }
  };
  // by all wavefronts
  auto odd_of_tile = [&](const int tile) {
    if (kv_begin + (tile + 1) * kStep <= tile_sees) return false;
    const bool odd = has_odd(lds, tile % Lds::kValues, wave);
    if (odd) {
      set_odd_aside<kSrc>(lds, tile % Lds::kValues);
      first_values(tile);   // again
    }
    return odd;
  };

  // products of a tile's keys, also of one that is not there, and between them what there is to do
  auto logits = [&](const int tile, const auto& between) {
    f32x16 sum = {};
    products_with(x, [&](auto at) { return read_key(tile, at); },
                  [&](auto at, u32x4& y) {
                    if constexpr (kValuesAhead) y = read_value(max(tile - 1, 0), at);
                  },
                  [&](auto at, const u32x4 k) { sum = mfma32(k, q[at.value], sum); }, between);
    s = sum;
  };
  // What was requested three steps ago (in 8 bits: what the last one requested three steps ago) has arrived, and nobody reads any
  // more what the step before last read.
  auto step = [&]() {
    wait_vector<kRaw ? 10 : 16>();
    lds_barrier();
  };
  auto mask = [&](const int i) {
    const int key0 = kv_begin + i * kStep;
    if (key0 + kStep > all_see) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = key0 + 8 * (r >> 2) + 4 * h + (r & 3) < sees ? s[r] : -__builtin_inff();
    }
  };
  float top;
  auto raise = [&](auto at) {
    if constexpr (at.value & 1) top = fmaxf(fmaxf(top, s[at.value - 1]), s[at.value]);
  };
  // The exponentials of tile i, the logits of the next one, and the requests of step i: of pages and rows keys of tile i + 4 and
  // values of one that has a free place; in 8 bits, where tile i + 2 has been widened, of the one that takes its place.
  auto weigh_and_go_on = [&](const int i) {
    const float ref = m == -__builtin_inff() ? 0.f : m;
    const char* vs_at = (char*)lds.vs[i % Lds::kValues] + 16 * h;
    const f32x16 now = s;
    float x[16];
    logits(i + 1, [&](auto at) {
      constexpr int j = at.value;
      x[j] = fast_exp2(__builtin_fmaf(now[j], sl2, -ref));
      if constexpr (j & 1) {
        float x0 = x[j - 1], x1 = x[j];
        l += x0 + x1;
        if constexpr (kRaw) {
          const f32x2 vs = *(const f32x2*)(vs_at + 4 * (8 * (j >> 2) + (j & 2)));
          x0 *= vs[0], x1 *= vs[1];
        }
        uint32_t two = pack_bf16(x0, x1);
        asm volatile("" : "+v"(two));   // computed here, and not in front of its use in the next step
        p[j >> 3][(j >> 1) & 3] = two;
      }
      if constexpr (kRaw) {
        if constexpr (j % 3 == 1) bring.template part<0, j / 3>(lds, i + 5, i + 5 < n_tiles, next_page);
      } else if constexpr (j < 8) {
        if constexpr (j & 1)
          bring.template part<1, j / 2>(lds, i + kValuesTo, i + kValuesTo < n_tiles, values_page);
        else
          bring.template part<0, j / 2>(lds, i + 4, i + 4 < n_tiles, next_page);
      }
    });
    values_page = next_page;
    next_page = page_of(i + (kRaw ? 6 : 5));
  };

  static_for<kReads>([&](auto j) { x[j.value] = read_key(0, j); });
  logits(0, [](auto) {});
  step();
  widen_all(2);
  mask(0);
  top = -__builtin_inff();
  static_for<16>(raise);
  m = pair_max(top) * sl2;
  static_for<kReads>([&](auto j) { x[j.value] = read_key(1, j); });
  weigh_and_go_on(0);
  for (int i = 1; i < n_tiles; ++i) {
    step();
    if constexpr (!kValuesAhead) first_values(i - 1);
    const bool odd = odd_of_tile(i - 1);
    mask(i);
    top = -__builtin_inff();
    add_values(i - 1, [&](auto j) {
      raise(j);
      if constexpr (j.value == 0 || (j.value >= 4 && j.value < 12)) widen_piece(i + 2, std::integral_constant<int, j.value == 0 ? 0 : j.value - 3>());
    });
    if (odd) mark_odd(i - 1);
    top = pair_max(top) * sl2;
    if (__ballot(top > m + kGrow)) {
      const float next = top > m + kGrow ? top : m;   // a row's reference does not go by other rows
      const float alpha = next == m ? 1.f : fast_exp2(m - next);
      m = next;
      l *= alpha;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] *= alpha;
    }
    weigh_and_go_on(i);
  }
  wait_vector<0>();   // the last tile's values, and requests of no bytes, which write zeros
  lds_barrier();
  if constexpr (!kValuesAhead) first_values(n_tiles - 1);
  const bool odd = odd_of_tile(n_tiles - 1);
  add_values(n_tiles - 1, [](auto) {});
  if (odd) mark_odd(n_tiles - 1);

  l = pair_sum(l);
  lds_barrier();
  if (part < 0) {
    uint32_t exps;
    store_rows<kSrc, true>(o, 1.f / l, exps, (char*)&lds + wave * 8192, (char*)a.out + (size_t)(tok0 + 4 * wave) * a.out_stride,
                           a.out_stride, n_tok - 4 * wave, lane);
    if (a.lse && mine < n_tok && h == 0)
      a.lse[(size_t)(tok0 + mine) * kHeads + (n & 7)] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  } else {
    const size_t part0 = (size_t)part + (size_t)(4 * wave) * n_parts;
    uint32_t exps = 0;
    store_rows<kSrc, false>(o, 0.f, exps, (char*)&lds + wave * 8192, (char*)a.part_acc + part0 * (kHeads * kDim * 2),
                            (size_t)n_parts * (kHeads * kDim * 2), n_tok - 4 * wave, lane);
    if (l != l && m == -__builtin_inff()) m = 0.f;   // NaN throughout is not a row without keys
    if (mine < n_tok && h == 0)
      *(f32x4*)(a.part_ml + ((part0 + (size_t)(n >> 3) * n_parts) * kHeads + (n & 7)) * 4) =
          (f32x4){m, l, __uint_as_float(exps), 0.f};
  }
}

// Joins split results by their (m, l), see merge_head.  A wavefront per token and head, or, where a token has more than sixteen of
// them, a workgroup: a wavefront's sixteen at a time would be a round trip each.
__device__ __forceinline__ void merge_long(const MergeArgs& a, const size_t base, const int np, const int h, const int wave,
                                           const int lane) {
  __shared__ __align__(16) f32x4 sums[kMergeWaves][64];
  __shared__ float ml_of[kMergeWaves][2];
  const int i = lane & 15, q = lane >> 4;
  const char* ml = (const char*)(a.part_ml + (base * kHeads + h) * 4);
  const char* acc = (const char*)(a.part_acc + (base * kHeads + h) * kDim);
  constexpr uint32_t kMlStride = kHeads * 4 * sizeof(float), kAccStride = kHeads * kDim * sizeof(uint16_t);
  const int end = np * (wave + 1) / kMergeWaves;
  float big = -__builtin_inff(), total = 0.f;
  f32x4 o = {};
  for (int p0 = np * wave / kMergeWaves; p0 < end; p0 += 16) {
    const f32x4 w = *(const f32x4*)(ml + (uint32_t)min(p0 + i, end - 1) * kMlStride);
    u32x2 x[16];
#pragma unroll
    for (int u = 0; u < 16; ++u)
      x[u] = __builtin_nontemporal_load((const u32x2*)(acc + (size_t)min(p0 + u, end - 1) * kAccStride + (uint32_t)lane * 8u));
    const float next = fmaxf(big, lanes16_max(w[0]));
    const float alpha = big == next ? 1.f : fast_exp2(big - next);
    big = next;
    const bool live = p0 + i < end && w[0] != -__builtin_inff();
    const float wgt = live ? fast_exp2(w[0] - big) : 0.f;
    total = total * alpha + lanes16_sum(wgt * (live ? w[1] : 0.f));
    o *= alpha;
    const int ex = (int32_t)(__float_as_uint(w[2]) << (24 - 8 * q)) >> 24;   // signed byte q
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
  sums[wave][lane] = o;
  if (lane == 0) ml_of[wave][0] = big, ml_of[wave][1] = total;
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int w = 1; w < kMergeWaves; ++w) big = fmaxf(big, ml_of[w][0]);
  total = 0.f;
  o = (f32x4){};
#pragma unroll
  for (int w = 0; w < kMergeWaves; ++w) {
    const float m = ml_of[w][0], wgt = m == -__builtin_inff() ? 0.f : fast_exp2(m - big);
    total = __builtin_fmaf(wgt, ml_of[w][1], total);
    o += wgt * sums[w][lane];
  }
  const float inv = 1.f / total;
  *(u32x2*)((uint16_t*)a.out + h * kDim + 4 * lane) = (u32x2){pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
  if (a.lse && lane == 0) a.lse[h] = (big + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
}
__global__ __launch_bounds__(64 * kMergeWaves) void prefill_merge_kernel(const PrefillArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, b = blockIdx.x;
  const bool wide = b < kHeads * a.n_long;
  const DescPtr rec = (DescPtr)a.merges + (size_t)(wide ? b / kHeads : b - (kHeads - 1) * a.n_long) * kMergeWords;
  const int tok = rec[0], base = rec[1], np = rec[2];
  const MergeArgs m = {a.part_acc, a.part_ml, (char*)a.out + (size_t)tok * a.out_stride,
                       a.lse ? a.lse + (size_t)tok * kHeads : nullptr, nullptr, nullptr};
  if (wide)
    merge_long(m, (size_t)base, np, b % kHeads, wave, lane);
  else
    merge_any(m, (size_t)base, np, 0, wave, lane);
}

namespace {
template <int kSrc>
void launch_source(const PrefillArgs& a, const char* base, const void* second, hipStream_t s) {
  const PrefillLate late = {a.out, a.lse, a.out_stride, a.tables, a.part_acc, a.part_ml, a.scale};
  const auto launch = [&](auto kernel) {
    kernel<<<a.n_work, 256, 0, s>>>(a.work, (const char*)a.q, a.q_stride, base, second, a.k_stride, a.v_stride, late);
  };
  if (a.n_work <= kPrefillCus)
    launch(prefill_pipe_kernel<kSrc>);
  else
    launch(prefill_kernel<kSrc>);
}
}  // namespace

hipError_t launch_prefill(const PrefillArgs& a, hipStream_t s) {
  if (a.n_work <= 0) return hipSuccess;
  if (!a.layer_base)
    launch_source<SRC_ROWS>(a, a.k, a.v, s);
  else if (a.scales)
    launch_source<SRC_PAGES8>(a, a.layer_base, a.scales, s);
  else
    launch_source<SRC_PAGES>(a, a.layer_base, nullptr, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_merge <= 0) return e;
  prefill_merge_kernel<<<a.n_merge + (kHeads - 1) * a.n_long, 64 * kMergeWaves, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace oxy
