// Attention of a prefill for gfx950 (MI355X): many query tokens of an item over its keys, which lie in a paged cache (bf16 or
// 8 bits) or in the rows that a projection wrote.
//
//   o = sum_j softmax_j(scale <q, k_j>) v_j   over   j < min(len, max(p + 1, full)),   p the query's position
//
// One pass over the keys with the running maximum m and sum l of a row: for a tile of keys S = K q, P = 2^(S - m), l += sum P,
// O += V P.  All eight heads of a token share a key, so a token is eight rows of one matrix product, and 16 tokens, 128 rows, are a
// workgroup's: 32 rows a wavefront, queries (64 registers) and sums (128) in registers, tiles of 32 keys through LDS.  The products
// are taken turned round, keys by rows and dims by rows: a lane then has one row's logits, and with the cache's order of keys
// its probabilities are the next product's operand as they are.
//
// What bounds it: large calls, the products, of which two halves of each weight make half as many again as the formula has: 2048
// new tokens behind 32781 take 680 to 710 us (802 to 837 TFLOP/s of the formula's, 1200 to 1255 of what runs), a causal prompt
// of 16391 tokens 1380 to 1410 (784 to 801, 1180 to 1200), where an 8192^3 product reaches 1247 on this card; the matrix pipes
// are busy 69 % of the cycles.  Middle ones (19 to 29 %), that a workgroup with a CU to itself does a tile's softmax and
// products one after the other, the split results, and the way to the first tile (record - page - rows - the queries' two
// halves: 4 us); small ones, that way and the launches.
//
// A workgroup that has a CU to itself was also built, with tiles requested three and four ahead and a tile's softmax among the
// products of its neighbours (then of weights rounded once): 64 records of 30 tiles 32.2 us instead of 35.6, 208 to 256 records
// of 6 to 10 as here, more of them 1.2 to 1.3 times as slow.
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

// Tiles of keys and values: one in use, one on its way.  Two workgroups share a CU.
template <int kSrc>
struct PrefillLds {
  static constexpr int kTiles = 2;
  char k[kTiles][kTileBytes], v[kTiles][kTileBytes];
};
// In 8 bits what is on its way are codes and exponents as they lie in the pages, a part for each wavefront, which widens what it
// requested.
template <>
struct PrefillLds<SRC_PAGES8> {
  static constexpr int kTiles = 1;
  char k[kTiles][kTileBytes], v[kTiles][kTileBytes];
  char codes[4][4096];     // [wavefront]: two pieces of 1 KiB of a K page, two of a V page
  char exps[4][256];       // exponents of a page, then nothing
  float vs[kStep];         // scales of the values
};
struct PrefillSmall {
  uint32_t odd[kDim];      // keys of a tile whose value is not finite in a dim
  uint32_t found[4];       // [wavefront]: whether it found one
  uint32_t spare[4][64];   // [wavefront]: what a request in the place of a tile's goes to
};
template <int kSrc>
struct PrefillShared : PrefillLds<kSrc>, PrefillSmall {};

// kSize bytes a lane to LDS, lane after lane, from offset + more + kImm behind a base that is the same for the wavefront; zeros
// for offset + kImm of `bytes` and above.  kImm counts in LDS too.  A buffer operation, which counts among vector memory
// operations only: behind one with a full address the compiler waits for all reads of LDS at once.
template <int kSize, int kImm = 0>
__device__ __forceinline__ void to_lds(const void* base, const uint32_t bytes, const uint32_t offset, void* to,
                                       const int more = 0) {
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
// operands lie in the order of the lanes.  (Of an LDS read of K 8.3 -> 7.6
// cycles, of V 10.2 -> 7.5; the counter of conflicts is at zero.)
__device__ __forceinline__ int k_row_swap(const int key) { return key & 15; }
__device__ __forceinline__ int v_row_swap(const int key) { return (key & 3) * 4; }
__device__ __forceinline__ int k_lds_offset(const int t, const int g, const int key) { return t * 1024 + g * 256 + key * 16; }
__device__ __forceinline__ int v_lds_offset(const int w, const int c, const int gp, const int n) {
  return (2 * w + (c >> 1)) * 1024 + gp * 512 + (c & 1) * 256 + n * 16;
}

// A wavefront's part of a tile on its way to LDS, eight operations (in 8 bits five).  blk: the wavefront's page, of rows: nothing.
// Wavefronts 0 and 1 bring the tile's first 16 keys, 2 and 3 the others.
template <int kSrc, class Lds>
__device__ __forceinline__ void request_tile(const char* base, const char* second, const size_t k_stride, const size_t v_stride,
                                             Lds& lds, const int b, const int key0, const int blk, const int src,
                                             const int len, const int wave, const int lane) {
  const int pg = wave >> 1, side = wave & 1, part = side * (kPageBytes / 2);
  if constexpr (kSrc == SRC_PAGES) {
    const char* from = base + (size_t)blk * kBlockBytes;
    const uint32_t k_chunk = k_chunk_offset(0, (lane >> 3) & 1, lane >> 4, lane & 7);
    const uint32_t v_chunk = v_chunk_offset(0, (lane >> 4) & 1, lane >> 5, lane & 15);
    static_for<4>([&](auto i) { to_lds<16, i.value * 1024>(from, kBlockBytes, k_chunk, lds.k[b] + pg * kPageBytes + part, part); });
    static_for<4>([&](auto i) {
      to_lds<16, i.value * 1024>(from, kBlockBytes, v_chunk, lds.v[b] + pg * kPageBytes + part, kPageBytes + part);
    });
  } else if constexpr (kSrc == SRC_PAGES8) {
    // K chunks of all keys and half of the dims; V chunks of all keys of half of the dims
    const char* from = base + (size_t)blk * kBlockBytes8;
    char* to = lds.codes[wave];
    to_lds<16>(from, kBlockBytes8, lane * 16, to, side * 1024);
    to_lds<16>(from, kBlockBytes8, lane * 16, to + 1024, side * 1024 + 2048);
    to_lds<16>(from, kBlockBytes8, lane * 16, to + 2048, kPageBytes8 + side * 2048);
    to_lds<16>(from, kBlockBytes8, lane * 16, to + 3 * 1024, kPageBytes8 + side * 2048 + 1024);
    to_lds<4>(second + (size_t)blk * kScaleBytes8, kScaleBytes8, lane * 4, lds.exps[wave]);   // 8 lanes, then 0
  } else {
    // two rows at a time; those behind the last one are 0.  Strides are below 2^28, so eight of them fit 32 bits.
    const int first = key0 + 8 * wave, left = min(len - first, 8);
    const uint32_t half = lane >> 5, chunk = lane & 31;
    const uint32_t k_chunk = (chunk ^ (8 * side + half)) * 16, v_chunk = (chunk ^ (4 * half)) * 16;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int two = 2 * (i & 3);
      const uint32_t stride = (uint32_t)(i < 4 ? k_stride : v_stride), bytes = left > 0 ? (left - 1) * stride + kDim * 2 : 0;
      to_lds<16>((i < 4 ? base : second) + (size_t)(src + first) * stride, bytes,
                 (i < 4 ? k_chunk ^ two * 16 : v_chunk ^ (two & 2) * 64) + (two + half) * stride,
                 (i < 4 ? lds.k[b] : lds.v[b]) + (8 * wave + two) * 512);
    }
  }
}

// four e4m3 codes -> four bf16 of scale times them
__device__ __forceinline__ u32x2 widen4(const uint32_t codes, const float scale) {
  return (u32x2){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))};
}
// A wavefront's part of a tile in 8 bits, from codes to bf16.  Keys with their scale; the scales of the values go into the
// probabilities (see the kernel), since four keys share a word.  left: keys of the item from the tile's first on.
template <class Lds>
__device__ __forceinline__ void widen_tile(Lds& lds, const int left, const int wave, const int lane) {
  const int pg = wave >> 1, side = wave & 1, n = lane & 15, gp = (lane >> 4) & 1, half = lane >> 5;
  const char* from = lds.codes[wave] + lane * 16;
  const char* v_from = lds.codes[wave] + 2048 + half * 1024 + (gp * 16 + n) * 16;
  // all reads before the first write: behind a write the compiler waits for what is on its way to LDS before it reads
  const u32x4 keys[2] = {*(const u32x4*)from, *(const u32x4*)(from + 1024)};
  const u32x4 lo = *(const u32x4*)v_from, hi = *(const u32x4*)(v_from + 512);   // keys 4gp.. and 8 + 4gp..
  const float s = scale_of((uint8_t)lds.exps[wave][k8_scale_offset(n)]);
  const float vs = scale_of((uint8_t)lds.exps[wave][v8_scale_offset(n)]);
  // stale exponents behind the item's end may be infinite: 0 instead; by eight lanes each
  lds.vs[16 * pg + n] = 16 * pg + n < left ? vs : 0.f;
  const int ch = 2 * (4 * side + (lane >> 4));   // eight dims
  char* const kp = lds.k[0] + pg * kPageBytes + k_lds_offset(ch >> 2, ch & 3, n);
  char* const vp = lds.v[0] + pg * kPageBytes + v_lds_offset(2 * side + half, 0, gp, n);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32x2 x = widen4(keys[i >> 1][2 * (i & 1)], s), y = widen4(keys[i >> 1][2 * (i & 1) + 1], s);
    *(u32x4*)(kp + (i >> 1) * 4096 + (i & 1) * 256) = (u32x4){x[0], x[1], y[0], y[1]};
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const u32x2 x = widen4(lo[c], 1.f), y = widen4(hi[c], 1.f);
    *(u32x4*)(vp + (c >> 1) * 1024 + (c & 1) * 256) = (u32x4){x[0], x[1], y[0], y[1]};
  }
}

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
  using Lds = PrefillShared<kSrc>;
  __shared__ __align__(16) Lds lds;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6) & 3;
  const int n = lane & 31, h = lane >> 5;
  const DescPtr rec = (DescPtr)work + (size_t)blockIdx.x * kPrefillWords;
  const int tok0 = rec[F_TOK0], n_tok = rec[F_N_TOK], pos = rec[F_POS], full = rec[F_FULL];
  const int kv_begin = rec[F_BEGIN], kv_end = rec[F_END], src = rec[F_SRC], part = rec[F_PART], n_parts = rec[F_N_PARTS],
            len = rec[F_LEN], head = rec[F_HEAD], own = rec[F_OWN];
  const int n_tiles = (kv_end - kv_begin + kStep - 1) / kStep;

  // the wavefront's page of a tile
  auto page_of = [&](const int tile) {
    if constexpr (kSrc == SRC_ROWS) return 0;
    const int at = 2 * tile + (wave >> 1), page = min((kv_begin >> 4) + at, (len - 1) >> 4);
    return at < kPrefillPages ? rec[F_PAGES + at] : ((DescPtr)a.tables)[page + (page < head ? src : own)];
  };
  auto request = [&](const int tile, const int blk) {
    int at = lane;
    asm volatile("" : "+v"(at));   // addresses are made here, and not kept in registers through the loop
    request_tile<kSrc>(base, (const char*)second, k_stride, v_stride, lds, tile % Lds::kTiles, kv_begin + tile * kStep, blk, src,
                       len, wave, at & 63);
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
  char* const q_at = (wave < 2 ? lds.k[Lds::kTiles - 1] : lds.v[Lds::kTiles - 1]) + (wave & 1) * 8192;
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
      widen_tile(lds, len - key0, wave, at & 63);
    }
    lds_barrier();
    // nobody reads the buffers any more that the next requests go to
    if (i + 1 < n_tiles) {
      request(i + 1, next_page);
      next_page = page_of(i + 2);
    }
    request_spare();
    const int b = i % Lds::kTiles;
    const bool odd = key0 + kStep > tile_sees && has_odd(lds, b, wave);
    if (odd) set_odd_aside<kSrc>(lds, b);
    if (key0 < any_sees) {
      f32x16 s = {};
      constexpr int kReads = kSrc == SRC_PAGES ? 5 : kSrc == SRC_ROWS ? 4 : 3;   // more would not fit the registers
      int turn = h ^ k_row_swap(n);
      if constexpr (kSrc == SRC_ROWS) asm volatile("" : "+v"(turn));   // see request
      const char* kb = lds.k[b] + (kSrc == SRC_ROWS ? n * 512 : (n >> 4) * kPageBytes + h * 256 + (n & 15) * 16);
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
      // Weights go into the product as two bf16, the second being what the first leaves, so that 2^-16 of each is lost, as in the
      // kernels of a step.  Rounded once (2^-8 of each), they were up to 1.5 times a step's tolerance off where few keys, or a few
      // large weights among thousands, carry a row, and off by as much in all dims where weights round the same way.  Half as
      // many products of the values again, behind the same reads (rounded once / so, us a layer: all of a prompt of 832 22.3 /
      // 23.8, 4 prefixes' 256 tokens behind 576 23.3 / 24.5, a causal prompt of 16391 1085 / 1380 to 1410, 2048 tokens behind
      // 32781 518 / 680 to 710, 48 behind 131071 in 8 bits 76 / 88).  The second product only in tiles with a weight above an eighth
      // of its row's sum so far: 1200 for the long prompt, and roundings that agree still add up.
      const float ref = m == -__builtin_inff() ? 0.f : m;
      u32x4 p[2], rest[2];
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        float x = fast_exp2(__builtin_fmaf(s[r], sl2, -ref)), y = fast_exp2(__builtin_fmaf(s[r + 1], sl2, -ref));
        l += x + y;
        if constexpr (kRaw) {
          const f32x2 vs = *(const f32x2*)&lds.vs[8 * (r >> 2) + 4 * h + (r & 3)];
          x *= vs[0], y *= vs[1];
        }
        const uint32_t w = pack_bf16(x, y);
        p[r >> 3][(r >> 1) & 3] = w;
        rest[r >> 3][(r >> 1) & 3] = pack_bf16(x - __uint_as_float(w << 16), y - __uint_as_float(w & 0xffff0000u));
      }
      // Rows: lane 16x + i of each half reads keys 4h + i / 4 (and 8 on), group 4x + i % 4 of four dims, see dim_of
      const int g = ((lane >> 4) & 1) * 4 + (lane & 3), key = 4 * h + ((lane >> 2) & 3), c = 2 * (g & 1) + (g >> 2);
      int v_turn = c ^ v_row_swap(key);
      if constexpr (kSrc == SRC_ROWS) asm volatile("" : "+v"(v_turn));
      const char* vb = lds.v[b] + (kSrc == SRC_ROWS ? key * 512 + (g >> 1 & 1) * 8 : lane * 16);
      products<2>(   // three ahead would not fit the registers, and with two products a read were no faster
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
          [&](auto at, const u32x4 v) {
            f32x16& sum = o[at.value & 7];
            sum = mfma32(v, p[at.value >> 3], sum);
            sum = mfma32(v, rest[at.value >> 3], sum);
          });
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

hipError_t launch_prefill(const PrefillArgs& a, hipStream_t s) {
  if (a.n_work <= 0) return hipSuccess;
  const PrefillLate late = {a.out, a.lse, a.out_stride, a.tables, a.part_acc, a.part_ml, a.scale};
  const auto launch = [&](auto kernel, const char* base, const void* second) {
    kernel<<<a.n_work, 256, 0, s>>>(a.work, (const char*)a.q, a.q_stride, base, second, a.k_stride, a.v_stride, late);
  };
  if (!a.layer_base)
    launch(prefill_kernel<SRC_ROWS>, a.k, a.v);
  else if (a.scales)
    launch(prefill_kernel<SRC_PAGES8>, a.layer_base, a.scales);
  else
    launch(prefill_kernel<SRC_PAGES>, a.layer_base, nullptr);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_merge <= 0) return e;
  prefill_merge_kernel<<<a.n_merge + (kHeads - 1) * a.n_long, 64 * kMergeWaves, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace oxy
