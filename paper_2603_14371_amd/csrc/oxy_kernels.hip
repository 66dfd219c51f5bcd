// HIP kernels for gfx950 (MI355X): KV append / gather and the mixed-mask paged attention.
//
// What is computed is the attention inside the paper's ActionDenoise and
// BatchedLanguageDecode passes (App. A.1, Eq. 5-6) for queries of several tasks at once,
// all reading one shared prefill cache (Sec. 3.2, cross-task KV sharing) plus their own
// tokens.  Visibility: prefix always; own tokens causally for decode queries, all of the
// chunk for action queries.
//
// Evaluation scheme.  The visible set of a query is cut into (prefix | own) and each part
// into fixed-size splits.  A work item is (query rows that share one KV source, one split of
// that source); it yields an un-normalised partial (reference max m in the log2 domain, sum
// l, accumulator acc[256]).  A second kernel merges a query's partials by the log-sum-exp
// rule.  How many queries share a work item depends on the whole batch; the splits depend on the
// pool and the item only, and a query's arithmetic is the same in a work item of any width, so its
// bits never depend on what else is in the batch.
//
// MFMA mapping (v_mfma_f32_16x16x32_bf16, lane = 16*g + n, keys taken 32 at a time = page A
// and page B of the block table):
//   S^T[key][row]  = sum_d K[key][d] * Q[row][d]      A = K chunks, B = Q rows
//       tile hf (0,1): A-row r is key 8hf + r%8 of page r/8, so lane (n = row, g) receives
//       the logits of keys 8hf + 4(g%2) + e, e < 4, of page g/2
//   O^T[d][row]   += sum_key V[key][d] * P[row][key]  A = V chunk, B = P
//       lane (g) contracts eight keys of one page, the same eight whose logits lane (g) of the
//       first product holds: its V operand is ONE 16-byte chunk of that page, and P goes from
//       wavefront to wavefront without moving between lanes.  A-row m of operand c is dim
//       64w+4m+c -> lane (n = row, g) accumulates dims 64w+16g..64w+16g+15 over four operands
// Both results keep "row = lane % 16", so the softmax state (m, l, rescale factor) is a
// per-lane scalar.  The pool pages are stored in exactly the operand order these products
// want (see oxy.h): every MFMA operand is one aligned 16-byte load.
#include "oxy_merge.h"

#include <hip/hip_ext.h>

#include <mutex>
#include <type_traits>

namespace oxy {

// ------------------------------------------------------------------------------------------
// append / gather
// ------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void append_kernel(const uint16_t* __restrict__ k_new,
                                                     const uint16_t* __restrict__ v_new,
                                                     const int32_t* __restrict__ slots,
                                                     char* __restrict__ layer_base) {
  const int tok = blockIdx.x;
  append_row(k_new + (size_t)tok * kDim, v_new + (size_t)tok * kDim, slots[tok], layer_base,
             threadIdx.x);
}

// Rows of keys key0..key0+n-1 of one block, by one workgroup: all rows are read at once, K goes out as
// 16-byte chunks and V, turned through LDS, as whole chunks where all eight keys of one are among them
// and key by key elsewhere, so that nothing else in the page is touched.  kWhole: all sixteen rows, without
// the other form's clamps and conditions (52 blocks of one layer 2.8 us, with them 3.1; 50 blocks in each of 18
// layers 6.2 / 6.4, kernel trace).
struct __align__(16) PageLds {
  uint16_t v[kPage][kDim + 8];   // +8: rows land in different banks
};
template <bool kWhole>
__device__ __forceinline__ void append_page(const uint16_t* __restrict__ k_src,
                                            const uint16_t* __restrict__ v_src, const int key0,
                                            const int n, char* __restrict__ block, PageLds& sm,
                                            const int t) {
  char* kp = block;
  char* vp = block + kPageBytes;
  u32x4 k[2], v[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int idx = t + 256 * i, cd = idx & 31;
    const int row = kWhole ? idx >> 5 : min(max((idx >> 5) - key0, 0), n - 1);
    k[i] = *(const u32x4*)(k_src + (size_t)row * kDim + cd * 8);
    v[i] = *(const u32x4*)(v_src + (size_t)row * kDim + cd * 8);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int idx = t + 256 * i, key = idx >> 5, cd = idx & 31;
    if (kWhole || (key >= key0 && key < key0 + n))
      *(u32x4*)(kp + k_chunk_offset(cd >> 2, key >> 3, cd & 3, key & 7)) = k[i];
    *(u32x4*)(&sm.v[key][cd * 8]) = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int ci = t + 256 * i, gp = (ci >> 4) & 1, d = 64 * (ci >> 7) + 4 * (ci & 15) + ((ci >> 5) & 3);
    u32x4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k0 = (e < 2 ? 4 * gp : 8 + 4 * gp) + 2 * (e & 1);
      out[e] = (uint32_t)sm.v[k0][d] | ((uint32_t)sm.v[k0 + 1][d] << 16);
    }
    if (kWhole || (key0 <= 4 * gp && key0 + n >= 12 + 4 * gp)) {
      *(u32x4*)(vp + ci * 16) = out;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = (e < 4 ? 4 * gp : 4 + 4 * gp) + e;
        if (key >= key0 && key < key0 + n)
          *(uint16_t*)(vp + ci * 16 + 2 * e) = (uint16_t)(out[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}
__device__ __forceinline__ void append_rows(const uint16_t* __restrict__ k_src,
                                            const uint16_t* __restrict__ v_src, const int key0,
                                            const int n, char* __restrict__ block, PageLds& sm,
                                            const int t) {
  if (n == kPage)
    append_page<true>(k_src, v_src, 0, kPage, block, sm, t);
  else
    append_page<false>(k_src, v_src, key0, n, block, sm, t);
}

// Append of a run of consecutive positions of one table (a prefix): one workgroup per block.
// blockIdx.y = layer relative to the first one: sources advance by src_layer_stride bytes, the
// pool by pool_layer_stride bytes per layer.
__global__ __launch_bounds__(256) void append_blocks_kernel(const uint16_t* __restrict__ k_new,
                                                            const uint16_t* __restrict__ v_new,
                                                            const InlineIds blocks, int32_t pos0,
                                                            int32_t n_tokens,
                                                            char* __restrict__ layer_base,
                                                            size_t src_layer_stride,
                                                            size_t pool_layer_stride) {
  __shared__ PageLds sm;
  k_new = (const uint16_t*)((const char*)k_new + blockIdx.y * src_layer_stride);
  v_new = (const uint16_t*)((const char*)v_new + blockIdx.y * src_layer_stride);
  layer_base += blockIdx.y * pool_layer_stride;
  const int page = (pos0 >> 4) + blockIdx.x;
  const int lo = max(pos0, page * kPage), hi = min(pos0 + n_tokens, (page + 1) * kPage);
  append_rows(k_new + (size_t)(lo - pos0) * kDim, v_new + (size_t)(lo - pos0) * kDim, lo & 15, hi - lo,
              layer_base + (size_t)blocks.v[blockIdx.x] * kBlockBytes, sm, threadIdx.x);
}

// Reads runs of tokens back in natural order, one workgroup per run (at most the 16 tokens of a
// block; see oxy_internal.h for the encoding).  Every V chunk holds one dim of eight keys, so a
// token alone touches all of its V page: the page is read once as whole chunks, turned through
// LDS, and only the run's rows are written; of a page the chunks with a key of the run are read (a
// single token's are half of them).  (One workgroup per token read 256 two-byte pieces per row: the
// 1337 tokens of four histories took three launches of 2.8 us, now one of 3.4 us.  A list of as many
// scattered single slots takes three launches as before; the C call waited for is 23.5 us against 21.7.)
__global__ __launch_bounds__(256) void gather_inline_kernel(const char* __restrict__ layer_base,
                                                            const GatherRuns runs,
                                                            uint16_t* __restrict__ k_out,
                                                            uint16_t* __restrict__ v_out) {
  __shared__ __align__(16) uint16_t v_s[kPage][kDim + 8];   // +8: rows start in different banks
  const int t = threadIdx.x;
  const int slot = runs.slot[blockIdx.x], where = runs.where[blockIdx.x];
  const int key0 = slot & 15, len = (where & 15) + 1;
  const size_t out0 = (size_t)(where >> 4);
  const char* kp = layer_base + (size_t)(slot >> 4) * kBlockBytes;
  const char* vp = kp + kPageBytes;
  // chunks with a key of the run: keys 4gp..4gp+3 and 8+4gp..8+4gp+3 (gp = (t >> 4) & 1 for both)
  const int lo = 4 * ((t >> 4) & 1), hi = lo + 8, end = key0 + len;
  const bool wanted = (key0 < lo + 4 && end > lo) || (key0 < hi + 4 && end > hi);
  u32x4 v[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (wanted) v[i] = *(const u32x4*)(vp + (t + 256 * i) * 16);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int idx = t + 256 * i, key = idx >> 5, cd = idx & 31;
    if (key >= key0 && key < key0 + len)
      *(u32x4*)(k_out + (out0 + key - key0) * kDim + cd * 8) =
          *(const u32x4*)(kp + k_chunk_offset(cd >> 2, key >> 3, cd & 3, key & 7));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int ci = t + 256 * i, gp = (ci >> 4) & 1, d = 64 * (ci >> 7) + 4 * (ci & 15) + ((ci >> 5) & 3);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (wanted) v_s[(e < 4 ? 4 * gp : 4 + 4 * gp) + e][d] = (uint16_t)(v[i][e >> 1] >> (16 * (e & 1)));
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int idx = t + 256 * i, key = idx >> 5, cd = idx & 31;
    if (key >= key0 && key < key0 + len)
      *(u32x4*)(v_out + (out0 + key - key0) * kDim + cd * 8) = *(const u32x4*)(&v_s[key][cd * 8]);
  }
}

// Descriptor upload: pinned host memory -> device memory, read over the bus by the kernel itself.
// A copy of this size (8 to 100 KiB) is bound by its hand-over: hipMemcpyAsync gives one of more
// than 16 KiB to a copy engine, and the two queues then wait for each other's signals (fixed cost of
// a step with a 33 KiB descriptor 30 us, of one with 8 KiB, which is copied by a kernel, 12 us).
__global__ __launch_bounds__(256) void upload_kernel(const int32_t* __restrict__ src,
                                                     int32_t* __restrict__ dst, int32_t n_words) {
  const int i = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (i + 4 <= n_words) {
    *(u32x4*)(dst + i) = __builtin_nontemporal_load((const u32x4*)(src + i));
  } else {
    for (int k = i; k < n_words; ++k) dst[k] = src[k];
  }
}

// The status is the launch's own (hipGetLastError would report, and clear, whatever an earlier call
// of the thread left behind), and the launch completes `done` itself: recording an event behind it
// is one more runtime call and one more packet (one-layer step 19.3 -> 18.5 us, 25.0 -> 24.0 in
// processes where the runtime's calls are slow).
hipError_t launch_upload(const int32_t* pinned, int32_t* device, int32_t n_words, hipStream_t s,
                         hipEvent_t done) {
  if (n_words <= 0) return hipErrorInvalidValue;
  void* args[] = {&pinned, &device, &n_words};
  return hipExtLaunchKernel((const void*)upload_kernel, dim3((n_words + 1023) / 1024), dim3(256),
                            args, 0, s, nullptr, done, 0);
}

hipError_t launch_append(const void* k_new, const void* v_new, const int32_t* d_slots,
                         int32_t n_tokens, void* layer_base, hipStream_t s) {
  if (n_tokens <= 0) return hipSuccess;
  append_kernel<<<n_tokens, 256, 0, s>>>((const uint16_t*)k_new, (const uint16_t*)v_new, d_slots,
                                         (char*)layer_base);
  return hipGetLastError();
}

hipError_t launch_append_inline(const void* k_new, const void* v_new, const InlineIds& blocks,
                                int32_t pos0, int32_t n_tokens, void* layer_base, int32_t n_layers,
                                size_t src_layer_stride, size_t pool_layer_stride, hipStream_t s) {
  if (n_tokens <= 0 || n_layers <= 0) return hipSuccess;
  // blocks.v[i] is the block of page (pos0 / 16 + i)
  const int32_t n_pages = ((pos0 + n_tokens + kPage - 1) >> 4) - (pos0 >> 4);
  append_blocks_kernel<<<dim3(n_pages, n_layers), 256, 0, s>>>(
      (const uint16_t*)k_new, (const uint16_t*)v_new, blocks, pos0, n_tokens, (char*)layer_base,
      src_layer_stride, pool_layer_stride);
  return hipGetLastError();
}

hipError_t launch_gather_inline(const void* layer_base, const GatherRuns& runs, int32_t n_runs,
                                void* k_out, void* v_out, hipStream_t s) {
  if (n_runs <= 0) return hipSuccess;
  gather_inline_kernel<<<n_runs, 256, 0, s>>>((const char*)layer_base, runs, (uint16_t*)k_out,
                                              (uint16_t*)v_out);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// attention work items
// ------------------------------------------------------------------------------------------
constexpr int kLateOffset = 7 * 8;   // behind the preloaded arguments (held against attn_kernel's own list below it)

// Bound by the memory pipeline of the CU where a launch is large (128 KiB of pages per workgroup and
// round, two workgroups per CU), by the length of this chain where it is small.
//
// One work item: up to 2*G query tokens (G groups of 16 rows) against one split of a KV source,
// taken in rounds of 128 keys.  In a round wavefront w
//   1. holds the K operands of keys 32w..32w+31 in registers and computes S^T for all rows,
//   2. publishes each row's largest logit, and after a barrier takes the row's largest of all 128,
//   3. writes its P (hi + lo bf16, relative to the common reference max) to LDS,
//   4. after a second barrier contracts ALL 128 keys for dims 64w..64w+63, whose V operands it
//      loaded itself.
// K and V thus go from memory to registers exactly once per work item and never through LDS; what
// the wavefronts exchange is P (2 KiB per group and step).  The accumulator is 16 registers per
// group, no combination of per-wavefront accumulators follows, and a work item of eight tokens fits
// the registers of two workgroups per CU.  (Before: work items of up to two tokens kept a
// 64-register accumulator per wavefront and combined the four through 66 KiB of LDS, 1.1 us of a
// 4 us work item, now 0.4; larger ones staged K and V in LDS, where each of the four wavefronts
// read all of both.  Work-item launch of one request on 832 tokens 5.44 -> 4.79 us, of eight requests
// and a chunk 7.8 -> 7.05, of eight chunks on 2048 tokens 23.3 -> 20.6, of 64 requests and two
// chunks on 2048-token prefixes 20.55 -> 20.27, kernel trace.)
//
// A row's arithmetic does not depend on G or on the other rows: a query may be evaluated alone or
// beside any others and gives the same bits.
//
// kOwnPages: a decode item's own pages, read by this work item alone, which also writes the item's
// new rows when the append is folded in.  Otherwise the pages are a prefix's or a multi-token item's,
// and other work items read them too.  kOnce: non-temporal page loads, for own pages that will have
// left the Infinity Cache by the next step and are not to push others out (see kOnceBytes).
//
// kSteps: 32-key steps of a round that are loaded, 4, or 2 for a split of at most 64 keys of a prefix or of a
// multi-token item (the last one of an 832-token prefix, a short observation's): wavefronts 2 and 3 load no
// K then, and all of them half of V.  A decode item's own pages always take 4.  (With every step loaded, the
// pages past the end once more, such an item took as long as one of 128 keys and kept the loads of its
// CU's other workgroup waiting: work-item launch of eight requests and a chunk 7.3 us, now 7.0, of six
// requests with 13 new tokens 10.2 / 9.6; others +-0.5 %.)
template <int G, bool kOwnPages, bool kOnce, int kSteps>
__device__ __forceinline__ void attend(const AttnArgs& early_args, const WorkItem& wi, WorkLds& sm) {
  AttnArgs a = early_args;
  int tid = threadIdx.x;
  // keeps what is computed from the thread id inside this instance: shared with the other
  // instances of the kernel it would have to live across all of them, which costs G = 4 spills
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);  // wave-uniform: keep it scalar
  const int n = lane & 15, g = lane >> 4;
  const int h = n & 7, sub = n >> 3;
  const float ninf = -__builtin_inff();
  const float sl2 = log2_scale(a);
  const char* __restrict__ base = (const char*)a.layer_base;
  const int nsteps = (wi.kv_end - wi.kv_begin + 31) >> 5;
  const int rounds = (nsteps + 3) >> 2;
  const int npg = ((wi.kv_end + 15) >> 4) - (wi.kv_begin >> 4);


  u32x4 kr[16];      // kr[2j+hf]: K operand (j, hf) of this wavefront's 32 keys
  u32x4 vr[kSteps][4];    // vr[s][c]: V operand c of this wavefront's 64 dims, step s of the round
  auto page_load = [](const char* p) {
    if constexpr (kOnce) return __builtin_nontemporal_load((const u32x4*)p);
    return *(const u32x4*)p;
  };
  // A step past the split's end re-reads a page of the split; its logits are masked and its V
  // operands are not used.  The block ids of the first two rounds are in the record (no dependent
  // load in front of the first pages), those of later rounds in the block table.
  // Lane offsets are formed anew at every use (the asm statements): hoisted out of the rounds as
  // 64-bit addresses they cost four groups the registers that they do not have.
  auto load_k_of = [&](const int blk_a, const int blk_b) {
    int off = (g * 8 + (n & 7)) * 16;
    asm volatile("" : "+v"(off));
    const char* p = base + (size_t)((n >> 3) ? blk_b : blk_a) * kBlockBytes + off;
#pragma unroll
    for (int i = 0; i < 16; ++i) kr[i] = page_load(p + i * 512);
  };
  auto load_v_of = [&](const i32x8 blks) {
    int off = kPageBytes + v_chunk_offset(wv, 0, g & 1, n);
    asm volatile("" : "+v"(off));
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const char* p = base + (size_t)((g >> 1) ? blks[2 * s + 1] : blks[2 * s]) * kBlockBytes + off;
#pragma unroll
      for (int c = 0; c < 4; ++c) vr[s][c] = page_load(p + c * 512);
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

  // Folded append: the query tokens of an item on its own pages are its new rows.  Those inside
  // this split's key range are written to the pool by this workgroup (no other workgroup reads
  // them in this launch), and a workgroup barrier orders the writes before the page loads that
  // cover them.  The first new row sits in step `first_new`: when that step belongs to a later
  // round, its loads come after the barriers of the first one anyway; otherwise the rows go out,
  // with a barrier of their own, before the first page load.
  RowPart rows[2];
  int32_t row_slot[2] = {0, 0};
  bool row_mine[2] = {false, false};
  bool early = false;
  const bool fold = kOwnPages && a.k_new;
  if (fold) {
    const int pos0 = (wi.q0 == kNoCausal ? 0 : wi.q0);
    const int ta = wi.toks[0], tb = wi.toks[1];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int pos = pos0 + t;
      row_mine[t] = t < wi.n_tok && pos >= wi.kv_begin && pos < wi.kv_end;
      const int tk = t ? tb : ta;
      rows[t] = load_row((const uint16_t*)a.k_new + (size_t)tk * kDim,
                         (const uint16_t*)a.v_new + (size_t)tk * kDim, tid);
    }
    row_slot[0] = ((DescPtr)a.d_slots)[ta];
    row_slot[1] = ((DescPtr)a.d_slots)[tb];
    const int first_new = (max(pos0, wi.kv_begin) - wi.kv_begin) >> 5;
    early = first_new < 4;
    if (early) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (row_mine[t])
          store_row(rows[t], row_slot[t], (char*)a.layer_base, tid);
      __syncthreads();
    }
  }
  // The query loads are issued BEFORE the first pages: loads complete in order per wavefront, so
  // the barrier below waits for the queries only, not for the slowest wavefront's first 32 KiB.
  int slot_req;
  {
    u32x4 qtmp[G][2];
#pragma unroll
    for (int r = 0; r < G; ++r) {
      const char* qrow = (const char*)a.q + ((size_t)token_of(wi, r, sub) * kHeads + h) * (kDim * 2);
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)   // unconditional, zeroed afterwards
        qtmp[r][jj] = *(const u32x4*)(qrow + (2 * wv + jj) * 64 + g * 16);
    }
    slot_req = request_slot<G>(a, wi, lane);
    __builtin_amdgcn_sched_barrier(0);
    auto store_q = [&]() {
      __builtin_amdgcn_sched_barrier(0);
      take_late<kLateOffset>(a);
#pragma unroll
      for (int r = 0; r < G; ++r) {
        const u32x4 z = {0, 0, 0, 0};
#pragma unroll
        for (int jj = 0; jj < 2; ++jj)
          sm.q[r][2 * wv + jj][lane] = 2 * r + sub < wi.n_tok ? query_sign(a, qtmp[r][jj]) : z;
      }
    };
    // on both sides by itself: behind the join the queries would be waited for as if no K were in flight
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
  if (fold && !early) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
      if (row_mine[t])
        store_row(rows[t], row_slot[t], (char*)a.layer_base, tid);
  }
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

  // kLast: the split's last round, the only one with steps past the end or a partial step.  It is
  // a copy of its own so that the loads of the other rounds sit under no condition.
  auto round_body = [&](const int round, auto last) {
    constexpr bool kLast = decltype(last)::value;
    int lane_now = tid & 63;   // likewise, for the mask limits and LDS addresses
    asm volatile("" : "+v"(lane_now));
    const int lane = lane_now, n = lane & 15, g = lane >> 4, sub = n >> 3;
    const int pos = wi.kv_begin + 32 * (4 * round + wv);
    const int left = wi.kv_end - pos;
    const bool need_mask = (kLast && left < 32) || pos + 31 > wi.q0;
    constexpr int kAhead = G == 4 ? 3 : 8;
    f32x4 s0[G], s1[G];
    // with two steps wavefronts 2 and 3 have no keys (and kr[] was never written): nothing is visible
    if (kSteps == 4 || wv < 2) {
#pragma unroll
      for (int r = 0; r < G; ++r) {
        s0[r] = (f32x4){0.f, 0.f, 0.f, 0.f};
        s1[r] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const u32x4 q = sm.q[r][j][lane];
          s0[r] = mfma16(kr[2 * j], q, s0[r]);
          s1[r] = mfma16(kr[2 * j + 1], q, s1[r]);
        }
      }
      // a few query reads ahead of the products: more would cost registers that four groups do
      // not leave, fewer make every pair of products wait a full LDS round trip (four groups with three ahead for
      // two, fewer groups with eight for four, us per layer: five chunks on 1500 tokens 16.6 / 16.4, a chunk of 300
      // 21.2 / 20.85, eight on 832 16.6 / 16.5, six and 48 requests 16.35 / 16.25)
      __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
      for (int i = 0; i < 8 * G - kAhead; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 2 * kAhead, 0);
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
    // Online softmax.  The reference max only moves when a logit exceeds it by more than kGrow,
    // so the rescale of acc is rare; P is then at most 2^kGrow, well inside fp32/bf16 range.  P
    // travels as hi+lo bf16: a single bf16 rounding (2^-9 relative) is too coarse for queries that
    // see only a handful of keys.
    float mx[G];
    bool grow = false;   // true for the first finite logit too (m = -inf)
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
        const float alpha = up ? fast_exp2(m[r] - mx[r]) : 1.f;   // m = -inf gives 0
        l[r] = rescaled(l[r], alpha);
        if (round > 0) {   // acc holds zeros before
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[r][c] *= alpha;
        }
        m[r] = up ? mx[r] : m[r];
      }
    }
#pragma unroll
    for (int r = 0; r < G; ++r) {
      u32x4 hi, lo;
      l[r] += softmax_weights(s0[r], s1[r], sl2, (m[r] == ninf) ? 0.f : m[r], hi, lo);
      sm.p[wv][r][0][lane] = hi;
      sm.p[wv][r][1][lane] = lo;
      if constexpr (kLast) sm.ls[r][lane][wv] = l[r];
    }
    __builtin_amdgcn_sched_barrier(0);   // the next K operands reuse kr[]
    if constexpr (!kLast) load_k(round + 1);
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    // With one group all P operands are requested at once, in front of the branches of a last
    // round; with more the products of one group hide the reads of the next.
    u32x4 ph[kSteps], pl[kSteps];
    if constexpr (G == 1) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        ph[s] = sm.p[s][0][0][lane];
        pl[s] = sm.p[s][0][1][lane];
      }
    }
    auto contract = [&](const int s, const int r) {
      const u32x4 hi = G == 1 ? ph[s] : sm.p[s][r][0][lane];
      const u32x4 lo = G == 1 ? pl[s] : sm.p[s][r][1][lane];
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[r][c] = mfma16(vr[s][c], hi, acc[r][c]);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[r][c] = mfma16(vr[s][c], lo, acc[r][c]);
    };
    if constexpr (!kLast) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int r = 0; r < G; ++r) contract(s, r);
      __builtin_amdgcn_sched_barrier(0);   // likewise vr[]
      load_v(round + 1);
      __builtin_amdgcn_sched_barrier(0);
    } else {
      const int nv = nsteps - 4 * round;   // 1..4 steps
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int left_s = wi.kv_end - (wi.kv_begin + 32 * (4 * round + s));
        if (s < nv && left_s < 32) {
          const u32x4 mask = value_mask(left_s, g);
#pragma unroll
          for (int c = 0; c < 4; ++c) vr[s][c] &= mask;
        }
        if (G == 1 && s < nv) contract(s, 0);
      }
      // Several groups: group by group, so that a group's scaling and stores fall into the
      // products of the next (8 chunks on 2048 tokens 164.1 -> 160.2 us for six layers).
      auto finish = [&](auto full) {
#pragma unroll
        for (int r = 0; r < G; ++r) {
#pragma unroll
          for (int s = 0; s < kSteps; ++s)
            if (G > 1 && (decltype(full)::value || s < nv)) contract(s, r);
          const int slot = sm.slot[2 * r + sub];
          store_part<(G >= 4)>(a, wi, slot, acc[r], r, wv, lane);
          if (wv == r) {   // wave-uniform: the sums of the groups are shared out
            const f32x4 lw = *(const f32x4*)sm.ls[r][lane];
            const float total = row_sum4((lw[0] + lw[1]) + (lw[2] + lw[3]));
            if (g == 0 && 2 * r + sub < wi.n_tok)
              *(f32x2*)(a.part_ml + ((size_t)slot * kHeads + (n & 7)) * 4) = (f32x2){m[r], total};
          }
        }
      };
      if (G > 1 && nv == kSteps)
        finish(std::true_type());
      else
        finish(std::false_type());
    }
  };
  if constexpr (kSteps == 4)
    for (int round = 0; round + 1 < rounds; ++round) round_body(round, std::false_type());
  round_body(kSteps == 4 ? rounds - 1 : 0, std::true_type());
}

// Own phase of an item whose history was empty before the step (an action chunk): up to eight
// tokens whose keys are this step's new rows.  With the append folded in they are read from
// k_new / v_new, and the pool receives them from the merge launch of the same layer.  A split is one 32-key step
// or a few, so the wavefronts share the rows out, not the keys: wavefront w computes the logits
// and P of tokens 2w and 2w+1, with the K operands brought in by all four through LDS, and contracts
// all tokens' P for its 64 dims as in `attend`.  (Each wavefront by itself, all of K, Q and V in its
// own registers and no barrier, waits for four times the loads: 4.3 us until the logits are there
// against 1.8 us for a single wavefront.)
// Every sum is taken in the order of `attend`, rounds of 128 keys included, so that a folded
// append and a separate one give the same bits.  kOneStep: the split is one step, and everything
// it needs is requested at once; otherwise a step's operands are requested when it is their turn.
// kRows: the keys are rows of k_new / v_new (row0 + own position); otherwise (the append went
// before, one step only) they are read from the pages.  kG: groups of two tokens; every wavefront
// scales and stores its 64 dims of all of them, one after the other, which is what a tile ends with.
template <bool kOneStep, bool kRows, int kG>
__device__ __forceinline__ void attend_fresh(const AttnArgs& early_args, const WorkItem& wi, WorkLds& sm,
                                             const int row0) {
  AttnArgs a = early_args;
  static_assert(kOneStep || kRows, "several steps from pages go through attend");
  constexpr int kSteps = kOneStep ? 1 : 4;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4, h = n & 7, sub = n >> 3;
  const float ninf = -__builtin_inff();
  const float sl2 = log2_scale(a);
  const int nsteps = (wi.kv_end - wi.kv_begin + 31) >> 5, last = wi.kv_end - 1;
  const uint16_t* kn = (const uint16_t*)a.k_new + (size_t)row0 * kDim + 64 * wv + 8 * g;
  const uint16_t* vn = (const uint16_t*)a.v_new + (size_t)row0 * kDim + 64 * wv + 4 * n;
  const int blk_a = wi.pages[0], blk_b = wi.pages[1];
  const char* __restrict__ pages = (const char*)a.layer_base;
  u32x4 (*ks)[64] = &sm.q[0][0];   // K operands of the step (the query rows stay in registers)

  u32x4 kr[4], qf[8], vpage[4];
  u32x2 vr[8];   // [key]: dims 64w+4n..+3 of this lane's eight keys, as they lie in the row
  // this wavefront's quarter of the step's K operands: dims 64w..64w+63.  Positions at or beyond
  // the split's end re-read its last row and are masked.
  auto load_k = [&](const int s) {
    if constexpr (!kRows) {
      const char* p = pages + (size_t)(sub ? blk_b : blk_a) * kBlockBytes + (g * 8 + h) * 16;
#pragma unroll
      for (int i = 0; i < 4; ++i) kr[i] = *(const u32x4*)(p + (4 * wv + i) * 512);
      return;
    }
    const int pos = wi.kv_begin + 32 * s + 16 * sub + h;
    const uint16_t* r0 = kn + (size_t)min(pos, last) * kDim;
    const uint16_t* r1 = kn + (size_t)min(pos + 8, last) * kDim;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      kr[2 * j] = *(const u32x4*)(r0 + 32 * j);
      kr[2 * j + 1] = *(const u32x4*)(r1 + 32 * j);
    }
  };
  auto load_v = [&](const int s) {
    if constexpr (!kRows) {
      const char* p = pages + (size_t)((g >> 1) ? blk_b : blk_a) * kBlockBytes + kPageBytes +
                      v_chunk_offset(wv, 0, g & 1, n);
#pragma unroll
      for (int c = 0; c < 4; ++c) vpage[c] = *(const u32x4*)(p + c * 512);
      return;
    }
    const int pos = wi.kv_begin + 32 * s + 16 * (g >> 1) + 4 * (g & 1);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      vr[e] = *(const u32x2*)(vn + (size_t)min(pos + (e < 4 ? e : e + 4), last) * kDim);
  };
  if constexpr (kOneStep) load_k(0);
  {   // wavefronts past the item's tokens hold its last token's rows and store nothing
    const char* qrow = (const char*)a.q + ((size_t)token_of(wi, wv, sub) * kHeads + h) * (kDim * 2);
#pragma unroll
    for (int j = 0; j < 8; ++j) qf[j] = *(const u32x4*)(qrow + j * 64 + g * 16);
  }
  const int slot_req = request_slot<kMaxGroups>(a, wi, lane);
  if constexpr (kOneStep) load_v(0);
  __builtin_amdgcn_sched_barrier(0);
  take_late<kLateOffset>(a);
#pragma unroll
  for (int j = 0; j < 8; ++j) qf[j] = query_sign(a, qf[j]);
  float m_own = ninf, l[4] = {0.f, 0.f, 0.f, 0.f};   // of this wavefront's row n
  f32x4 acc[kG][4];
#pragma unroll
  for (int r = 0; r < kG; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[r][c] = (f32x4){0.f, 0.f, 0.f, 0.f};
  for (int first = 0; first < (kOneStep ? 1 : nsteps); first += 4) {
    f32x4 s0[kSteps], s1[kSteps];
    float mx = ninf;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      if (kOneStep || first + s < nsteps) {
        if constexpr (!kOneStep) {
          __syncthreads();   // the previous step's operands are used up, the previous round's P too
          load_k(first + s);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) ks[4 * wv + i][lane] = kr[i];
        if (kOneStep || s == 0)
          if (threadIdx.x < 8) sm.slot[lane] = slot_req + wi.part_idx;
        __syncthreads();
        s0[s] = s1[s] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          s0[s] = mfma16(ks[2 * j][lane], qf[j], s0[s]);
          s1[s] = mfma16(ks[2 * j + 1][lane], qf[j], s1[s]);
        }
        const int pos = wi.kv_begin + 32 * (first + s);
        const int end = min(wi.kv_end, wi.q0 + 2 * wv + sub + 1) - (pos + 16 * (g >> 1) + 4 * (g & 1));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s0[s][e] = e < end ? s0[s][e] : ninf;
          s1[s][e] = 8 + e < end ? s1[s][e] : ninf;
        }
        mx = fmaxf(mx, row_max4(row_max8(s0[s], s1[s]) * sl2));
      }
    const bool up = mx > m_own + kGrow;
    const float alpha = up ? fast_exp2(m_own - mx) : 1.f;
    m_own = up ? mx : m_own;
    if constexpr (!kOneStep) {
#pragma unroll
      for (int s = 0; s < 4; ++s) l[s] = rescaled(l[s], alpha);
      if (g == 0) sm.mx[wv][n][0] = alpha;
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      if (kOneStep || first + s < nsteps) {
        u32x4 hi, lo;
        l[s] += softmax_weights(s0[s], s1[s], sl2, (m_own == ninf) ? 0.f : m_own, hi, lo);
        sm.p[s][wv][0][lane] = hi;
        sm.p[s][wv][1][lane] = lo;
      }
    __syncthreads();
    if constexpr (!kOneStep) {
#pragma unroll
      for (int r = 0; r < kG; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[r][c] *= sm.mx[r][n][0];
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      if (kOneStep || first + s < nsteps) {
        if constexpr (!kOneStep) load_v(first + s);
        const u32x4 mask = value_mask(wi.kv_end - (wi.kv_begin + 32 * (first + s)), g);
        u32x4 v[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if constexpr (kRows) {   // dim 64w+4n+c: halfword c of every key
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t x = vr[2 * i][c >> 1], y = vr[2 * i + 1][c >> 1];
              v[c][i] = (c & 1) ? ((x >> 16) | (y & 0xffff0000u)) : ((x & 0xffffu) | (y << 16));
            }
          } else {
            v[c] = vpage[c];
          }
          v[c] &= mask;
        }
#pragma unroll
        for (int r = 0; r < kG; ++r) {
          const u32x4 hi = sm.p[s][r][0][lane], lo = sm.p[s][r][1][lane];
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[r][c] = mfma16(v[c], hi, acc[r][c]);
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[r][c] = mfma16(v[c], lo, acc[r][c]);
        }
      }
  }
  const float total = row_sum4((l[0] + l[1]) + (l[2] + l[3]));
  const int own_slot = sm.slot[2 * wv + sub];
  if (g == 0 && 2 * wv + sub < wi.n_tok) {
    *(f32x2*)(a.part_ml + ((size_t)own_slot * kHeads + h) * 4) = (f32x2){m_own, total};
  }
#pragma unroll
  for (int r = 0; r < kG; ++r) store_part<(kG >= 4)>(a, wi, sm.slot[2 * r + sub], acc[r], r, wv, lane);
}

template <bool kRows>
__device__ __forceinline__ void attend_fresh_width(const AttnArgs& a, const WorkItem& wi, WorkLds& sm,
                                                   const int row0) {
  if (wi.n_tok <= 2)
    attend_fresh<true, kRows, 1>(a, wi, sm, row0);
  else if (wi.n_tok <= 4)
    attend_fresh<true, kRows, 2>(a, wi, sm, row0);
  else
    attend_fresh<true, kRows, 4>(a, wi, sm, row0);
}

__device__ __forceinline__ void attend_fresh_any(const AttnArgs& a, const WorkItem& wi, WorkLds& sm,
                                                 const int row0) {
  if (wi.kv_end - wi.kv_begin <= 32)
    attend_fresh_width<true>(a, wi, sm, row0);
  else if (wi.n_tok <= 4)
    attend_fresh<false, true, 2>(a, wi, sm, row0);
  else
    attend_fresh<false, true, 4>(a, wi, sm, row0);
}

// The narrowest is tested last, and with it the four-step instance that every decode step runs: the compiler
// lays the instance that is tested last out first and the widest at the kernel's end.  With the narrowest tested first
// and laid out last a launch whose code has left the caches (other kernels and a read of 512 MB in front of every
// launch) took, one request on 832 tokens 7.3-7.5 us, now 6.9-7.1, three 7.1-7.2 / 7.0, one with a chunk 7.6-7.8 / 7.3-7.5;
// larger launches and launches that follow each other within 1 %.  Where code lies is worth that much for no reason that
// shows in it: the whole kernel 4 KiB further on took 0.2 us more.
__device__ __forceinline__ void attend_shared(const AttnArgs& a, const WorkItem& wi, WorkLds& sm) {
  const bool few_keys = wi.kv_end - wi.kv_begin <= 64;
  if (wi.n_tok > 4)
    attend<4, false, false, 4>(a, wi, sm);   // bound by its products and stores: no faster with half the loads
  else if (wi.n_tok > 2)
    few_keys ? attend<2, false, false, 2>(a, wi, sm) : attend<2, false, false, 4>(a, wi, sm);
  else
    few_keys ? attend<1, false, false, 2>(a, wi, sm) : attend<1, false, false, 4>(a, wi, sm);
}

// What the first loads need is preloaded into scalar registers (all 14 words there are; see build.py).  The rest is
// read from the argument segment once those loads are on their way (take_late): every workgroup of a launch
// reads that segment at the same time, and in front of the first loads it cost, us per layer, 50 queries + one
// request 7.81 / 7.58, a chunk on 100 tokens 7.31 / 7.04, three requests 6.70 / 6.57, four chunks on 832 tokens 11.39 /
// 11.22, one request 6.31 / 6.26, 64 requests and two chunks 22.29 / 22.18, 256 requests 71.6 / 71.8.
// On a page of its own start: 768 bytes further on, because a kernel in front had grown, the same code took
// 7.4-7.6 us instead of 7.0-7.2 in a cold launch of one request, and 19.8-20.1 instead of 19.3-19.5 in
// repeated ones of 64 requests and two chunks.  Multiples of 8, 16 and 32 KiB are no better.
__global__ __attribute__((aligned(4096))) __launch_bounds__(256, 2) void attn_kernel(
    const int32_t* work, const void* q, const void* layer_base, const void* k_new, const void* v_new,
    const int32_t* d_slots, const int32_t part_off, const float scale, const LateArgs) {
  __shared__ WorkLds sm;
  AttnArgs a;
  a.q = q;
  a.layer_base = layer_base;
  a.part_off = work + part_off;
  a.scale = scale;
  a.k_new = k_new;
  a.v_new = v_new;
  a.d_slots = d_slots;
  WorkItem wi;
  wi.rec = (DescPtr)work + (size_t)blockIdx.x * kWorkWords;
  const i32x8 head = ((DescPtr8)wi.rec)[0];
  wi.toks = ((DescPtr8)wi.rec)[1];
  wi.pages = ((DescPtr8)wi.rec)[2];
  // wanted here, in one go, and not one after the other where they are used first
  asm volatile("" ::"s"(head), "s"(wi.toks), "s"(wi.pages));
  wi.n_tok = head[W_N_TOK];
  wi.tbl_off = head[W_TBL_OFF];
  wi.kv_begin = head[W_KV_BEGIN];
  wi.kv_end = head[W_KV_END];
  wi.q0 = head[W_CAUSAL_Q0];
  wi.part_idx = head[W_PART_IDX];
  const int path_word = head[W_PATH];
  if ((path_word & kPathMask) == PATH_NOOP) return;   // padding record
  if (path_word & kPathAppends)                       // one or two tokens on their own pages
    path_word & kPathOnce ? attend<1, true, true, 4>(a, wi, sm) : attend<1, true, false, 4>(a, wi, sm);
  else if (a.k_new && (path_word & kPathFresh))
    attend_fresh_any(a, wi, sm, path_word >> kPathRowShift);
  else if ((path_word & kPathFresh) && wi.kv_end - wi.kv_begin <= 32)
    attend_fresh_width<false>(a, wi, sm, 0);
  else
    attend_shared(a, wi, sm);
}
using AttnParams = Params<decltype(&attn_kernel)>;
static_assert(std::is_same_v<AttnParams::Last, LateArgs> && AttnParams::offset_of_last() == kLateOffset,
              "take_late reads attn_kernel's last argument at kLateOffset");

// ------------------------------------------------------------------------------------------
// merge of a query token's partials (log-sum-exp rule).  One wavefront per token and head, which has
// every load of the first sixteen partials in flight at once.
// (A merge fused into attn_kernel by "last arriver merges" was built twice and measured: with
// device-scope fences every workgroup pays a whole-L2 write-back + invalidate (165 us per
// launch); with scoped write-through stores and no fences it is correct and fence-free, but the
// tile workgroups finish last and then merge their eight tokens serially (53 us).  Hence its own
// kernel.)
// ------------------------------------------------------------------------------------------
// Everything a merge workgroup needs comes preloaded in scalar registers (13 of the 14 there are; see build.py):
// the argument segment is memory that every workgroup of a launch would read at once, in front of its first load.
// us per layer with the segment / preloaded: 50 queries + one request 8.02 / 7.81, eight requests and a chunk 8.92 /
// 8.76, three requests 6.80 / 6.65, eight chunks on 832 tokens 16.82 / 16.61, 64 requests and two chunks 22.66 / 22.40, one
// request (two workgroups) 6.33 / 6.36, eight chunks on 2048 22.44 / 22.49.
#define OXY_MERGE_PARAMS                                                                              \
  const uint16_t *part_acc, const float *part_ml, void *out, float *lse, const int32_t *n_parts, \
      const int32_t *part_off, const int32_t n_q
template <int kBlockHeads>
__global__ __launch_bounds__(64 * kBlockHeads) void merge_kernel(OXY_MERGE_PARAMS) {
  merge_block<kBlockHeads>({part_acc, part_ml, out, lse, n_parts, part_off}, blockIdx.x);
}

// merge of one layer and, in the same launch, an append that touches other memory than the
// merge: the next layer's new rows (cross-layer fusion), or this layer's rows of the items whose
// tiles read their keys from k_new / v_new (nx.runs names them, a block of a table each).  256 threads append.
template <int kBlockHeads>
__global__ __launch_bounds__(64 * kBlockHeads) void merge_append_kernel(OXY_MERGE_PARAMS, const AppendArgs nx) {
  __shared__ PageLds sm;
  const int n_merge = kHeads / kBlockHeads * n_q, i = (int)blockIdx.x - n_merge;
  if (i < 0) {
    merge_block<kBlockHeads>({part_acc, part_ml, out, lse, n_parts, part_off}, blockIdx.x);
    return;
  }
  if (threadIdx.x >= 256) return;   // whole wavefronts: a barrier waits for those of its workgroup that have not ended
  const int run = nx.runs ? nx.runs[i] : i << 4;
  const int tok = run >> 4, slot = nx.d_slots[tok];
  const uint16_t* k_row = (const uint16_t*)nx.k_new + (size_t)tok * kDim;
  const uint16_t* v_row = (const uint16_t*)nx.v_new + (size_t)tok * kDim;
  if (nx.runs)   // a row each: 18 layers of 50 queries + one request 167.2 us instead of 163.6
    append_rows(k_row, v_row, 0, (run & 15) + 1, (char*)nx.layer_base + (size_t)(slot >> 4) * kBlockBytes,
                sm, threadIdx.x);
  else
    append_row(k_row, v_row, slot, (char*)nx.layer_base, threadIdx.x);
}

hipError_t launch_attention_work(const AttnArgs& a, hipStream_t s, hipEvent_t start,
                                 hipEvent_t stop) {
  if (a.n_work <= 0 || a.n_q <= 0) return hipErrorInvalidValue;
  const LateArgs late = {a.part_acc, a.part_ml, a.tables, a.write_through};
  const int32_t part_off = (int32_t)(a.part_off - a.work);   // of one descriptor
  if (start || stop)
    hipExtLaunchKernelGGL(attn_kernel, dim3(a.n_work), dim3(256), 0, s, start, stop, 0, a.work, a.q, a.layer_base,
                          a.k_new, a.v_new, a.d_slots, part_off, a.scale, late);
  else
    attn_kernel<<<a.n_work, 256, 0, s>>>(a.work, a.q, a.layer_base, a.k_new, a.v_new, a.d_slots, part_off, a.scale,
                                         late);
  return hipGetLastError();
}

namespace {
template <int kBlockHeads>
void launch_merge(const AttnArgs& a, const AppendArgs* next, hipStream_t s, hipEvent_t start, hipEvent_t stop) {
  const bool timed = start || stop, appends = next && next->n_blocks > 0;
  const dim3 grid(kHeads / kBlockHeads * a.n_q + (appends ? next->n_blocks : 0)), block(64 * kBlockHeads);
  const auto launch = [&](auto kernel, auto... more) {
    if (timed)
      hipExtLaunchKernelGGL(kernel, grid, block, 0, s, start, stop, 0, a.part_acc, a.part_ml, a.out, a.lse,
                            a.n_parts, a.part_off, a.n_q, more...);
    else
      kernel<<<grid, block, 0, s>>>(a.part_acc, a.part_ml, a.out, a.lse, a.n_parts, a.part_off,
                                    a.n_q, more...);
  };
  if (appends)
    launch(merge_append_kernel<kBlockHeads>, *next);
  else
    launch(merge_kernel<kBlockHeads>);
}
}  // namespace

hipError_t launch_merge_append(const AttnArgs& a, const AppendArgs* next, hipStream_t s,
                               hipEvent_t start, hipEvent_t stop) {
  if (a.n_q <= 0) return hipErrorInvalidValue;
  if (merge_heads(a.n_q) == kHeads)
    launch_merge<kHeads>(a, next, s, start, stop);
  else
    launch_merge<kHeads / 2>(a, next, s, start, stop);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// Split results in static device memory, for callers that cannot allocate (see
// oxy_mixed_attention_static in oxy.h).  Every GPU the library runs on holds its own copy of
// the array, at its own address, until the process ends; that address is looked up once per
// device, with the device current, and is what host code passes on from then.
// ------------------------------------------------------------------------------------------
constexpr size_t kStaticAccBytes = (size_t)kStaticMaxPartials * kHeads * kDim * sizeof(uint16_t);
constexpr size_t kStaticMlBytes = (size_t)kStaticMaxPartials * kHeads * 4 * sizeof(float);
static __device__ __align__(256) unsigned char scratch[kStaticAccBytes + kStaticMlBytes];

hipError_t static_scratch(uint16_t** part_acc, float** part_ml) {
  constexpr int kMaxDevices = 64;
  static std::mutex mu;
  static void* ptr_of_device[kMaxDevices] = {};
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (!ptr_of_device[dev]) {
    void* ptr = nullptr;
    e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
    if (e != hipSuccess) return e;
    if (!ptr) return hipErrorInvalidSymbol;
    ptr_of_device[dev] = ptr;
  }
  *part_acc = (uint16_t*)ptr_of_device[dev];
  *part_ml = (float*)((char*)ptr_of_device[dev] + kStaticAccBytes);
  return hipSuccess;
}

hipError_t launch_attention(const AttnArgs& a, hipStream_t s) {
  hipError_t e = launch_attention_work(a, s);
  if (e != hipSuccess) return e;
  return launch_merge_append(a, nullptr, s);
}

}  // namespace oxy
