// Rotary positions for gfx950 (MI355X): rows of queries and keys turned by their tokens' positions, and the append that
// turns a step's queries and new keys on the way into the pool.
//
// Pair i of a row's first r dims is turned by the angle position * freqs[i]:
//   y1 = x1 c - x2 s,  y2 = x2 c + x1 s,   c, s = amplitude * (cos, sin),
// pairs being (i, i + r/2) or (2i, 2i + 1); the other dims are copied.  Angles are taken in 64 bits, in turns: the
// fraction of a turn of a far position (2^20 radians and more) has no bits left in 32.  Cosine and sine are rounded to 32
// bits, the products are 32-bit ones, each rounded, and the result is rounded once to bf16.
//
// Bound by the bytes of the rows (512 B in, 512 B out) in a prefill, by the length of one workgroup's chain (position,
// frequency, angle, row) in a step.
#include "../../include/oxy.h"
#include "oxy_kv8_device.h"

#include <cmath>
#include <cstdio>

extern "C" __attribute__((visibility("hidden"))) void oxy_internal_set_error(const char* msg);

namespace oxy {

constexpr int kMaxPairs = kDim / 2;

// How a lane finds its dims' partners: pairs lie side by side; halves a whole number of 16-byte chunks apart; or not.
enum RotaryForm { FORM_PAIRS, FORM_HALVES, FORM_HALVES_ANY };

__device__ __forceinline__ void turn_of(const RotaryArgs& r, const int position, const int pair, float& c, float& s) {
  const double turns = (double)position * r.freqs[pair] * 0.15915494309189533577;   // 1 / (2 pi)
  double sd, cd;
  sincospi(2.0 * (turns - rint(turns)), &sd, &cd);
  c = (float)(cd * r.amplitude);
  s = (float)(sd * r.amplitude);
}
__device__ __forceinline__ float element(const u32x4 x, const int e) {
  const uint32_t w = x[e >> 1];
  return __uint_as_float((e & 1) ? w & 0xffff0000u : w << 16);
}
// What lane c of 32 needs of a row: its eight elements, and those they are paired with.
struct RowLoad {
  u32x4 own, other;
};
template <int kForm>
__device__ __forceinline__ RowLoad load_turning(const uint16_t* row, const int rot, const int c) {
  RowLoad x;
  x.own = *(const u32x4*)(row + 8 * c);
  x.other = x.own;
  const int half = rot >> 1;
  if constexpr (kForm == FORM_HALVES) {
    if (8 * c < rot) x.other = *(const u32x4*)(row + (8 * c < half ? 8 * c + half : 8 * c - half));
  } else if constexpr (kForm == FORM_HALVES_ANY) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w = 0;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int d = 8 * c + 2 * i + k;
        const int p = d < half ? d + half : d < rot ? d - half : d;
        w |= (uint32_t)row[p] << (16 * k);
      }
      x.other[i] = w;
    }
  }
  return x;
}
// cs, sn: cosines and sines of this row's token
template <int kForm>
__device__ __forceinline__ u32x4 turned(const RowLoad& x, const float* cs, const float* sn, const int rot, const int c) {
#pragma clang fp contract(off)
  u32x4 out = x.own;
  const int half = rot >> 1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int e = 2 * i + k, d = 8 * c + e;
      int pair;
      float other;
      bool first;
      if constexpr (kForm == FORM_PAIRS) {
        pair = d >> 1;
        other = element(x.own, e ^ 1);
        first = k == 0;
      } else {
        first = d < half;
        pair = first ? d : d - half;
        other = element(x.other, e);
      }
      pair = min(pair, kMaxPairs - 1);   // past the rotated dims: read, and not used
      const float a = element(x.own, e) * cs[pair], b = other * sn[pair];
      y[k] = first ? a - b : a + b;
    }
    const uint32_t w = pack_bf16(y[0], y[1]);
    const int d = 8 * c + 2 * i;
    out[i] = d < rot ? w : x.own[i];   // both or neither: rot is even
  }
  return out;
}

constexpr int kRotaryTokens = 4;   // of a workgroup: their angles are taken once for all heads
template <int kForm>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs r, const char* x, const size_t x_stride, char* out,
                                                     const size_t out_stride, const int32_t n_tokens,
                                                     const int32_t n_heads) {
  __shared__ __align__(16) float cs[kRotaryTokens][kMaxPairs], sn[kRotaryTokens][kMaxPairs];
  const int tok0 = blockIdx.x * kRotaryTokens, here = min(kRotaryTokens, n_tokens - tok0);
  const int t = threadIdx.x, c = t & 31, rows = here * n_heads, half = r.rot_dims >> 1;
  auto row_of = [&](int i) {
    const int tok = i / n_heads;
    return (const uint16_t*)(x + (size_t)(tok0 + tok) * x_stride) + (i - tok * n_heads) * kDim;
  };
  int i = t >> 5;
  RowLoad now = {};
  if (i < rows) now = load_turning<kForm>(row_of(i), r.rot_dims, c);   // on its way while the angles are taken
  for (int k = t; k < here * half; k += 256) {
    const int tok = k / half, pair = k - tok * half;
    turn_of(r, r.positions[tok0 + tok], pair, cs[tok][pair], sn[tok][pair]);
  }
  __syncthreads();
  while (i < rows) {
    const int tok = i / n_heads, next = i + 8;
    RowLoad ahead = {};
    if (next < rows) ahead = load_turning<kForm>(row_of(next), r.rot_dims, c);
    *(u32x4*)(out + (size_t)(tok0 + tok) * out_stride + (size_t)(i - tok * n_heads) * (kDim * 2) + 16 * c) =
        turned<kForm>(now, cs[tok], sn[tok], r.rot_dims, c);
    now = ahead;
    i = next;
  }
}

// One token per workgroup: ten half wavefronts take its eight query rows, its key and its value.
template <int kForm, bool kBits8>
__global__ __launch_bounds__(320) void rotary_append_kernel(const RotaryAppendArgs a) {
  __shared__ __align__(16) float cs[kMaxPairs], sn[kMaxPairs];
  const int tok = blockIdx.x, t = threadIdx.x, c = t & 31, row = t >> 5, rot = a.rotary.rot_dims;
  const bool is_q = row < kHeads, is_v = row == kHeads + 1;
  const char* src = is_q ? (const char*)a.q + tok * a.q_stride + row * (kDim * 2)
                  : is_v ? (const char*)a.v_new + tok * a.v_stride : (const char*)a.k_new + tok * a.k_stride;
  RowLoad x = {};
  const bool live = !is_q || a.q;
  if (live) {
    if (is_v)
      x.own = *(const u32x4*)((const uint16_t*)src + 8 * c);
    else
      x = load_turning<kForm>((const uint16_t*)src, rot, c);
  }
  const int32_t slot = a.d_slots[tok];
  if (t < rot >> 1) turn_of(a.rotary, a.rotary.positions[tok], t, cs[t], sn[t]);
  __syncthreads();
  u32x4 y = x.own;
  if (!is_v) y = turned<kForm>(x, cs, sn, rot, c);
  if (is_q) {   // whole wavefronts: the key and the value are the two halves of the last one
    if (live) *(u32x4*)((uint16_t*)a.q_out + ((size_t)tok * kHeads + row) * kDim + 8 * c) = y;
    return;
  }
  const int key = slot & 15;
  if constexpr (kBits8) {
    char* block = (char*)a.layer_base + (size_t)(slot >> 4) * kBlockBytes8;
    uint8_t* sc = a.scales + (size_t)(slot >> 4) * kScaleBytes8;
    const Row8 r8 = quantise_row(y);
    if (is_v)
      store_value(r8, key, block, sc, c);
    else
      store_key(r8, key, block, sc, c);
  } else {
    char* block = (char*)a.layer_base + (size_t)(slot >> 4) * kBlockBytes;
    if (is_v) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        *(uint16_t*)(block + kPageBytes + v_chunk_of_dim(8 * c + e, (key >> 2) & 1) + v_slot_of_key(key) * 2) =
            (uint16_t)(y[e >> 1] >> (16 * (e & 1)));
    } else {
      *(u32x4*)(block + k_chunk_offset(c >> 2, key >> 3, c & 3, key & 7)) = y;
    }
  }
}

namespace {
int form_of(const RotaryArgs& r) {
  return r.pairs ? FORM_PAIRS : (r.rot_dims >> 1) % 8 == 0 ? FORM_HALVES : FORM_HALVES_ANY;
}
template <int kForm>
void launch_append_form(const RotaryAppendArgs& a, hipStream_t s) {
  if (a.scales)
    rotary_append_kernel<kForm, true><<<a.n_tokens, 320, 0, s>>>(a);
  else
    rotary_append_kernel<kForm, false><<<a.n_tokens, 320, 0, s>>>(a);
}
}  // namespace

hipError_t launch_rotary(const RotaryArgs& r, const void* x, size_t x_stride, void* out, size_t out_stride,
                         int32_t n_tokens, int32_t n_heads, hipStream_t s) {
  if (n_tokens <= 0) return hipSuccess;
  const dim3 grid((n_tokens + kRotaryTokens - 1) / kRotaryTokens);
  const auto launch = [&](auto kernel) {
    kernel<<<grid, 256, 0, s>>>(r, (const char*)x, x_stride, (char*)out, out_stride, n_tokens, n_heads);
  };
  switch (form_of(r)) {
    case FORM_PAIRS: launch(rotary_kernel<FORM_PAIRS>); break;
    case FORM_HALVES: launch(rotary_kernel<FORM_HALVES>); break;
    default: launch(rotary_kernel<FORM_HALVES_ANY>);
  }
  return hipGetLastError();
}

hipError_t launch_rotary_append(const RotaryAppendArgs& a, hipStream_t s) {
  if (a.n_tokens <= 0) return hipSuccess;
  switch (form_of(a.rotary)) {
    case FORM_PAIRS: launch_append_form<FORM_PAIRS>(a, s); break;
    case FORM_HALVES: launch_append_form<FORM_HALVES>(a, s); break;
    default: launch_append_form<FORM_HALVES_ANY>(a, s);
  }
  return hipGetLastError();
}

}  // namespace oxy

namespace {
int32_t refuse(const char* what) {
  oxy_internal_set_error(what);
  return OXY_ERR_INVALID_ARG;
}
}  // namespace

extern "C" {

int32_t oxy_rotary_freqs(const oxy_rotary_scaling* sc, double* freqs, double* amplitude) {
  if (!sc || !freqs) return refuse("rotary_freqs: null argument");
  const int32_t rot = sc->rot_dims;
  if (rot < 2 || rot > oxy::kDim || rot % 2) return refuse("rotary_freqs: rot_dims must be even, 2 to 256");
  if (!(sc->base > 0.0) || !std::isfinite(sc->base)) return refuse("rotary_freqs: base must be positive");
  if (sc->kind < OXY_ROTARY_PLAIN || sc->kind > OXY_ROTARY_RAMP) return refuse("rotary_freqs: unknown kind");
  const double two_pi = 6.283185307179586476925286766559;
  double base = sc->base;
  if (sc->kind != OXY_ROTARY_PLAIN && (!(sc->factor >= 1.0) || !std::isfinite(sc->factor)))
    return refuse("rotary_freqs: factor must be 1 or more");
  if (sc->kind >= OXY_ROTARY_BANDS &&
      (sc->original_len < 1 || !(sc->low > 0.0) || !(sc->high > sc->low) || !std::isfinite(sc->high)))
    return refuse("rotary_freqs: need original_len >= 1 and 0 < low < high");
  if (sc->kind == OXY_ROTARY_RAMP && !(sc->base > 1.0)) return refuse("rotary_freqs: a ramp needs a base above 1");
  if (sc->kind == OXY_ROTARY_BASE && rot > 2) base *= std::pow(sc->factor, rot / (rot - 2.0));
  double lo = 0.0, hi = 0.0;
  if (sc->kind == OXY_ROTARY_RAMP) {
    // the pair that makes `turns` turns in original_len positions
    const auto pair_of = [&](double turns) {
      return rot * std::log(sc->original_len / (two_pi * turns)) / (2.0 * std::log(sc->base));
    };
    lo = std::fmax(0.0, std::floor(pair_of(sc->high)));
    hi = std::fmin(rot - 1.0, std::ceil(pair_of(sc->low)));
  }
  for (int32_t i = 0; i < rot / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot);
    double keep = 1.0;   // how much of the pair stays as it is; the rest is slowed down by the factor
    if (sc->kind == OXY_ROTARY_LINEAR) keep = 0.0;
    if (sc->kind == OXY_ROTARY_BANDS) keep = (sc->original_len * f / two_pi - sc->low) / (sc->high - sc->low);
    if (sc->kind == OXY_ROTARY_RAMP) keep = 1.0 - (i - lo) / std::fmax(hi - lo, 0.001);
    keep = std::fmin(1.0, std::fmax(0.0, keep));
    freqs[i] = keep == 1.0 ? f : f * (keep + (1.0 - keep) / sc->factor);
  }
  if (amplitude) *amplitude = sc->kind == OXY_ROTARY_RAMP ? 1.0 + 0.1 * std::log(sc->factor) : 1.0;
  return OXY_OK;
}

int32_t oxy_rotary(const oxy_rotary_config* c, const int32_t* positions, const void* x, size_t x_stride, void* out,
                   size_t out_stride, int32_t n_tokens, int32_t n_heads, void* hip_stream) {
  if (!c || !c->freqs || !positions || !x || !out) return refuse("rotary: null argument");
  if (c->rot_dims < 2 || c->rot_dims > oxy::kDim || c->rot_dims % 2) return refuse("rotary: rot_dims must be even, 2 to 256");
  if (c->layout != OXY_ROTARY_HALVES && c->layout != OXY_ROTARY_PAIRS) return refuse("rotary: unknown layout");
  if (n_tokens < 0 || n_heads < 1 || n_heads > OXY_ROTARY_MAX_HEADS) return refuse("rotary: n_tokens or n_heads");
  const size_t row = (size_t)n_heads * oxy::kDim * 2;
  if (((uintptr_t)x | (uintptr_t)out | x_stride | out_stride) & 15) return refuse("rotary: rows must be 16-byte aligned");
  if (n_tokens > 1 && (x_stride < row || out_stride < row)) return refuse("rotary: stride below n_heads rows");
  const oxy::RotaryArgs r = {c->freqs, positions, c->amplitude, c->rot_dims, c->layout == OXY_ROTARY_PAIRS};
  const hipError_t e = oxy::launch_rotary(r, x, x_stride, out, out_stride, n_tokens, n_heads, (hipStream_t)hip_stream);
  if (e != hipSuccess) {
    char msg[160];
    snprintf(msg, sizeof(msg), "rotary: launch: %s", hipGetErrorString(e));
    oxy_internal_set_error(msg);
    return OXY_ERR_DEVICE;
  }
  return OXY_OK;
}

}  // extern "C"
