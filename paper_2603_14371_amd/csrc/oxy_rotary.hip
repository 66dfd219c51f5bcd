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

// Cosine and sine of position * freq times the amplitude, rounded to 32 bits once.  The angle is brought to a fraction of a
// turn, then to within an eighth of one around the nearest quarter, where the series of the two functions are cut behind
// x^13 / 13! and x^14 / 14!: the next terms are at most 2e-14 and 1e-15, a millionth of half a unit of the 32-bit result (2^-25
// near one), so the rounding is that of the exact value but for one in a million.  20 instructions in 64 bits, which run at the
// rate of 32 (with the library's sincospi, whose last bits are rounded off here, three times as many: nine heads of 8192
// tokens 20.7 us, with this 17.5).
__device__ __forceinline__ void turn_of(const double freq, const double amplitude, const int position, float& c, float& s) {
  const double turns = (double)position * freq * 0.15915494309189533577;   // 1 / (2 pi)
  const double part = turns - rint(turns), quarter = rint(4.0 * part);
  const double x = (part - 0.25 * quarter) * 6.28318530717958647693, z = x * x;   // |x| <= pi / 4
  double sd = 1.0 / 6227020800.0, cd = -1.0 / 87178291200.0;
  sd = fma(sd, z, -1.0 / 39916800.0), cd = fma(cd, z, 1.0 / 479001600.0);
  sd = fma(sd, z, 1.0 / 362880.0), cd = fma(cd, z, -1.0 / 3628800.0);
  sd = fma(sd, z, -1.0 / 5040.0), cd = fma(cd, z, 1.0 / 40320.0);
  sd = fma(sd, z, 1.0 / 120.0), cd = fma(cd, z, -1.0 / 720.0);
  sd = fma(sd, z, -1.0 / 6.0), cd = fma(cd, z, 1.0 / 24.0);
  sd = fma(sd * z, x, x), cd = fma(fma(cd, z, -0.5), z, 1.0);
  const int k = (int)quarter;   // -2..2 quarters on
  const double cq = (k & 1) ? sd : cd, sq = (k & 1) ? cd : sd;
  c = (float)(((k + 1) & 2) ? -cq * amplitude : cq * amplitude);
  s = (float)((k & 2) ? -sq * amplitude : sq * amplitude);
}
__device__ __forceinline__ float element(const u32x4 x, const int e) {
  const uint32_t w = x[e >> 1];
  return __uint_as_float((e & 1) ? w & 0xffff0000u : w << 16);
}
// What lane c of 32 needs of a row: its eight elements, and those they are paired with.
struct RowLoad {
  u32x4 own, other;
};
// kPartners: partners a whole number of chunks apart are loaded too; otherwise `turned` fetches them from the lanes that
// hold them.
template <int kForm, bool kPartners>
__device__ __forceinline__ RowLoad load_turning(const uint16_t* row, const int rot, const int c) {
  RowLoad x;
  x.own = *(const u32x4*)(row + 8 * c);
  x.other = x.own;
  const int half = rot >> 1;
  if constexpr (kForm == FORM_HALVES && kPartners) {
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
// Cosines and sines of a lane's eight dims, the same for all heads of a token.
struct LaneTurns {
  float c[8], s[8];
};
template <int kForm>
__device__ __forceinline__ LaneTurns turns_of_lane(const float* cs, const float* sn, const int rot, const int c) {
  LaneTurns r;
  const int half = rot >> 1;
  // a - b * s is a + b * -s, bit for bit.  Past the rotated dims: read, and not used
  if constexpr (kForm == FORM_PAIRS) {
    const f32x4 ct = *(const f32x4*)(cs + 4 * c), st = *(const f32x4*)(sn + 4 * c);
#pragma unroll
    for (int e = 0; e < 8; ++e) r.c[e] = ct[e >> 1], r.s[e] = (e & 1) ? st[e >> 1] : -st[e >> 1];
  } else if constexpr (kForm == FORM_HALVES) {
    const bool first = 8 * c < half;
    const int at = first ? 8 * c : min(8 * c - half, kMaxPairs - 8);
    const uint32_t flip = first ? 0x80000000u : 0u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x4 ct = *(const f32x4*)(cs + at + 4 * i), st = *(const f32x4*)(sn + at + 4 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) r.c[4 * i + e] = ct[e], r.s[4 * i + e] = __uint_as_float(__float_as_uint(st[e]) ^ flip);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int d = 8 * c + e, at = min(d < half ? d : d - half, kMaxPairs - 1);
      r.c[e] = cs[at];
      r.s[e] = d < half ? -sn[at] : sn[at];
    }
  }
  return r;
}
// By all lanes of a half wavefront.  In a prefill partners come from other lanes (8192 tokens 19.9 us; loaded a second
// time 21.9); in a step they are loaded, while the angles are taken (58 tokens 2.85 us; from lanes 3.05).
template <int kForm, bool kPartners>
__device__ __forceinline__ u32x4 turned(RowLoad x, const LaneTurns& w, const int rot, const int c) {
#pragma clang fp contract(off)
  u32x4 out = x.own;
  if constexpr (kForm == FORM_HALVES && !kPartners) {
    const int apart = rot >> 4, lane = threadIdx.x & 63;
    const int from = c < apart ? lane + apart : c < 2 * apart ? lane - apart : lane;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.other[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * from, (int)x.own[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int e = 2 * i + k;
      const float other = kForm == FORM_PAIRS ? element(x.own, e ^ 1) : element(x.other, e);
      const float a = element(x.own, e) * w.c[e], b = other * w.s[e];
      y[k] = a + b;
    }
    out[i] = 8 * c + 2 * i < rot ? pack_bf16(y[0], y[1]) : x.own[i];   // both or neither: rot is even
  }
  return out;
}

// kTokens of a workgroup: their angles are taken once for all heads, by all threads, and come to the lanes through LDS.
// With four, two half wavefronts share a token's heads; with one, all eight do.  A half wavefront keeps its cosines and
// sines, and kRows rows in flight.  Nine heads of 8192 tokens (75 MB) 18.0 us in halves, 17.0 in pairs: 4.2 and 4.4 TB/s;
// in halves that are not whole chunks, whose partners are loaded one by one, 29; of 64 tokens 2.6 us.
template <int kForm, int kTokens>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs r, const char* x, const size_t x_stride, char* out,
                                                     const size_t out_stride, const int32_t n_tokens,
                                                     const int32_t n_heads) {
  constexpr int kStep = 8 / kTokens;   // half wavefronts of a token
  constexpr int kRows = kForm == FORM_HALVES_ANY ? 1 : kTokens == 1 ? 2 : 3;   // of each at a time
  __shared__ __align__(16) float cs[kTokens][kMaxPairs], sn[kTokens][kMaxPairs];
  const int tok0 = blockIdx.x * kTokens, here = min(kTokens, n_tokens - tok0);
  const int t = threadIdx.x, c = t & 31, half = r.rot_dims >> 1;
  const int mine = (t >> 5) / kStep, tok = min(mine, here - 1), head0 = (t >> 5) % kStep;
  const char* src = x + (size_t)(tok0 + tok) * x_stride;
  char* dst = out + (size_t)(tok0 + tok) * out_stride + 16 * c;
  RowLoad rows[kRows];
  auto load = [&](const int head) {
#pragma unroll
    for (int k = 0; k < kRows; ++k)   // a row past the last is the last one again
      rows[k] = load_turning<kForm, false>((const uint16_t*)src + min(head + k * kStep, n_heads - 1) * kDim, r.rot_dims, c);
  };
  load(head0);   // on their way while the angles are taken
  for (int k = t; k < here * half; k += 256) {
    const int at = k / half, pair = k - at * half;
    turn_of(r.freqs[pair], r.amplitude, r.positions[tok0 + at], cs[at][pair], sn[at][pair]);
  }
  __syncthreads();
  const LaneTurns w = turns_of_lane<kForm>(cs[tok], sn[tok], r.rot_dims, c);
  for (int head = head0;;) {
    u32x4 y[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) y[k] = turned<kForm, false>(rows[k], w, r.rot_dims, c);
    const int next = head + kRows * kStep;
    if (next - head0 < n_heads) load(next);   // the same for both halves of a wavefront
#pragma unroll
    for (int k = 0; k < kRows; ++k)
      if (head + k * kStep < n_heads && mine < here) *(u32x4*)(dst + (head + k * kStep) * (kDim * 2)) = y[k];
    if (next - head0 >= n_heads) break;
    head = next;
  }
}

// What a workgroup needs behind its first loads.
struct RotaryLate {
  const double* freqs;
  const int32_t* d_slots;
  void* q_out;
  void* layer_base;
  uint8_t* scales;
  double amplitude;
};
// One token per workgroup: ten half wavefronts take its eight query rows, its key and its value (58 tokens 2.8
// us a launch: the chain position - angle - LDS - row).  The addresses of the
// first loads are preloaded into scalar registers (see build.py).
template <int kForm, bool kBits8>
__global__ __launch_bounds__(320) void rotary_append_kernel(const int32_t* positions, const char* q, const char* k_new,
                                                            const char* v_new, const uint32_t q_stride,
                                                            const uint32_t k_stride, const uint32_t v_stride,
                                                            const int32_t rot, const RotaryLate a) {
  __shared__ __align__(16) float cs[kMaxPairs], sn[kMaxPairs];
  const int t = threadIdx.x, c = t & 31, row = t >> 5;
  const size_t tok = blockIdx.x;
  const bool is_q = row < kHeads, is_v = row == kHeads + 1;
  const char* src = is_q ? q + tok * q_stride + row * (kDim * 2) : is_v ? v_new + tok * v_stride : k_new + tok * k_stride;
  RowLoad x = {};
  const bool live = !is_q || q;
  const int32_t position = ((DescPtr)positions)[tok];
  if (live) {
    if (is_v)
      x.own = *(const u32x4*)((const uint16_t*)src + 8 * c);
    else
      x = load_turning<kForm, true>((const uint16_t*)src, rot, c);
  }
  const int32_t slot = ((DescPtr)a.d_slots)[tok];
  if (t < rot >> 1) turn_of(a.freqs[t], a.amplitude, position, cs[t], sn[t]);
  __syncthreads();
  u32x4 y = x.own;
  if (!is_v) y = turned<kForm, true>(x, turns_of_lane<kForm>(cs, sn, rot, c), rot, c);
  if (is_q) {   // whole wavefronts: the key and the value are the two halves of the last one
    if (live) *(u32x4*)((uint16_t*)a.q_out + (tok * kHeads + row) * kDim + 8 * c) = y;
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
// From here on there are four tokens for every CU's two resident workgroups and more, and four share one's start.  One /
// four per workgroup, nine heads in halves: 2048 tokens 5.19 / 5.27 us, 3000 6.77 / 6.64, 8192 18.3 / 17.7; in halves that are
// not whole chunks 2048 tokens 11.9 / 9.7.
constexpr int kManyTokens = 2049;
int form_of(const RotaryArgs& r) {
  return r.pairs ? FORM_PAIRS : (r.rot_dims >> 1) % 8 == 0 ? FORM_HALVES : FORM_HALVES_ANY;
}
template <int kForm>
void launch_append_form(const RotaryAppendArgs& a, hipStream_t s) {
  const RotaryLate late = {a.rotary.freqs, a.d_slots, a.q_out, a.layer_base, a.scales, a.rotary.amplitude};
  const auto launch = [&](auto kernel) {
    kernel<<<a.n_tokens, 320, 0, s>>>(a.rotary.positions, (const char*)a.q, (const char*)a.k_new, (const char*)a.v_new,
                                      a.q_stride, a.k_stride, a.v_stride, a.rotary.rot_dims, late);
  };
  if (a.scales)
    launch(rotary_append_kernel<kForm, true>);
  else
    launch(rotary_append_kernel<kForm, false>);
}
}  // namespace

hipError_t launch_rotary(const RotaryArgs& r, const void* x, size_t x_stride, void* out, size_t out_stride,
                         int32_t n_tokens, int32_t n_heads, hipStream_t s) {
  if (n_tokens <= 0) return hipSuccess;
  const bool many = n_tokens >= kManyTokens;
  const auto launch = [&](auto one, auto four) {
    const dim3 grid(many ? (n_tokens + 3) / 4 : n_tokens);
    (many ? four : one)<<<grid, 256, 0, s>>>(r, (const char*)x, x_stride, (char*)out, out_stride, n_tokens, n_heads);
  };
  switch (form_of(r)) {
    case FORM_PAIRS: launch(rotary_kernel<FORM_PAIRS, 1>, rotary_kernel<FORM_PAIRS, 4>); break;
    case FORM_HALVES: launch(rotary_kernel<FORM_HALVES, 1>, rotary_kernel<FORM_HALVES, 4>); break;
    default: launch(rotary_kernel<FORM_HALVES_ANY, 1>, rotary_kernel<FORM_HALVES_ANY, 4>);
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
  if (!c || !c->freqs || (n_tokens != 0 && (!positions || !x || !out))) return refuse("rotary: null argument");
  if (c->rot_dims < 2 || c->rot_dims > oxy::kDim || c->rot_dims % 2) return refuse("rotary: rot_dims must be even, 2 to 256");
  if (c->layout != OXY_ROTARY_HALVES && c->layout != OXY_ROTARY_PAIRS) return refuse("rotary: unknown layout");
  if (n_tokens < 0 || n_tokens > OXY_ROTARY_MAX_TOKENS || n_heads < 1 || n_heads > OXY_ROTARY_MAX_HEADS)
    return refuse("rotary: n_tokens or n_heads");
  if (n_tokens == 0) return OXY_OK;   // what holds no rows may lie anywhere
  const size_t row = (size_t)n_heads * oxy::kDim * 2;
  if (((uintptr_t)x | (uintptr_t)out | x_stride | out_stride) & 15) return refuse("rotary: rows must be 16-byte aligned");
  if (n_tokens > 1 && (x_stride < row || out_stride < row)) return refuse("rotary: stride below n_heads rows");
  if (n_tokens > 1 && x == out && x_stride != out_stride) return refuse("rotary: in place with two strides");
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
