// The 8-bit cache row (gfx950): d signed bytes and one float32 scale.
//
//   scale = max|x| / 127 (float32, correctly rounded), code = round(x / scale),
//   ties to even, so |code| <= 127 and |x - code * scale| <= scale / 2.
//
// A row whose scale would be subnormal has scale 0 and codes 0; a row with an Inf
// or NaN has scale NaN and codes 0, so it reads back as NaN and never as data.
// A code is exact in bf16 and fp16 (7 bits), so a matrix product over codes is as exact
// as one over bf16 data; the scale of a key multiplies its column of scores, the
// scale of a value its column of probabilities, both in float32.
#pragma once

#include "internal.h"

namespace h2o {
namespace q8 {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kInfBits = 0x7F800000u;

__device__ __forceinline__ float code_f32(uint32_t w, int byte) {
  return (float)(int8_t)(w >> (8 * byte));
}
// Eight codes (two words) as a bf16 matrix operand.
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t lo, uint32_t hi) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = (__bf16)code_f32(lo, i);
    r[4 + i] = (__bf16)code_f32(hi, i);
  }
  return r;
}

// The same in fp16, where 0x6400 + u is 1024 + u.
__device__ __forceinline__ f16x8 codes_f16(uint32_t lo, uint32_t hi) {
  const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
  f16x2 r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u,
                                                           (i < 2 ? lo : hi) ^ 0x80808080u,
                                                           i & 1 ? 0x04030402u : 0x04010400u)) - off;
  return f16x8{r[0][0], r[0][1], r[1][0], r[1][1], r[2][0], r[2][1], r[3][0], r[3][1]};
}

// The weights of values in 8 bits, probability times scale, are rounded to fp16 for
// their product with the codes: by 2^-11 of their size, where bf16's 2^-8 would be as
// large an error as that of the bf16 output itself. They span many more powers of two
// than fp16 has, in any combination (a row of large values that nobody attends, a slot
// that takes nearly all the weight and has no value). So a row's softmax reference goes
// by its weights: it is put where the largest of the first tile with any is 2^aim, and
// moved there again when one exceeds 2^kMost. A weight below 2^-14 is off by 2^-25, which
// for n keys together is n 2^-(25 + aim) of the largest: 2^-11 with the aim of their
// number. Scales are taken relative to `ref`, a power of two above all that the wave has
// seen, and one below 2^kLeast of it counts as that much where the reference is chosen,
// so that probabilities stay below 2^90. Values are lost that are 2^70 or more below the
// largest of their head.
// A lane asks for more only where its largest score and its largest scale would together
// exceed 2^kMost, as different keys' they may (a branch of the wave, rare); before the
// exponentials, which then go out between the products. (Asked of the weights, after the
// exponentials: B1 Hq32 Hkv8 d128 M8192 T1024 202 us.)
constexpr float kMost = 15.f, kTop = 90.f, kLeast = -75.f;
__device__ __forceinline__ float aim_of(int nkeys) {
  const int a = 18 - __builtin_clz(nkeys | 1);   // log2(nkeys) - 13, rounded down
  return (float)(a < 0 ? 0 : a);
}
// log2 of a scale relative to ref, as far as the choice of a reference counts it.
__device__ __forceinline__ float log2_scale(float rel) { return fmaxf(__log2f(rel), kLeast); }
__device__ __forceinline__ float row_max(float y) {   // of a row's four lanes
  y = fmaxf(y, __shfl_xor(y, 16, 64));
  return fmaxf(y, __shfl_xor(y, 32, 64));
}
// How far mu may go down so that a row's probabilities, sofar in a lane, stay below 2^kTop.
__device__ __forceinline__ float least_move(float sofar) {
  return fminf(fmaxf(__log2f(sofar), -30.f) - kTop, 0.f);
}
// A row's reference mu (log2) at a tile that asks for more: fv is what the scales lost by a
// raise of theirs (or 1), and mu goes down by it, so that the weights summed so far keep
// their size; then it moves if the tile's largest weight asks for it. y, yc: log2 of the
// lane's largest, with its scale and as log2_scale counts that; l: its sum of probabilities;
// most: kMost, -inf before the first weight. Returns the factor of the sums of values.
__device__ __forceinline__ float move(float& mu, float& most, float& l, float fv, float y,
                                      float yc, float aim) {
  y = row_max(y);
  yc = row_max(yc);
  float sofar = row_max(l), fo = fv;
  if (most > -INFINITY) {
    const float by = fmaxf(__log2f(fv), least_move(sofar)), f = __builtin_amdgcn_exp2f(-by);
    mu += by;
    y -= by;
    yc -= by;
    l *= f;
    sofar *= f;
    fo *= f;
  }
  if (!(yc > most)) return fo;
  float by = yc - aim;
  if (sofar != 0.f) by = fmaxf(by, least_move(sofar));
  mu += by;
  if (y > -INFINITY) most = kMost;
  if (sofar == 0.f) return fo;
  const float f = __builtin_amdgcn_exp2f(-by);
  l *= f;
  return fo * f;
}
// The reference of a wave's value scales, with room for 16 times what it was taken from
// (a scale is below 2^122).
struct ValueRef {
  float inv = 1.f, limit = 0.f;   // 1 / ref; ref, 0 before the first keys
  // y: the largest |scale| of the wave's keys, above limit; returns what scales and sums
  // taken with the old reference lose
  __device__ __forceinline__ float raise(float y) {
    const uint32_t e = ((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(y)) &
                        0x7F800000u) + 5 * 0x00800000u;   // of 16 times a power of two above y
    const float old = limit;
    limit = __uint_as_float(e);
    inv = __uint_as_float(0x7F000000u - e);
    return old * inv;
  }
  __device__ __forceinline__ float ref() const { return limit == 0.f ? 1.f : limit; }
};

// Scale of a row from the bits of max|x| (as unsigned integers the finite
// magnitudes come before Inf, and Inf before every NaN).
__device__ __forceinline__ float row_scale(uint32_t amax_bits) {
  if (amax_bits >= kInfBits) return __uint_as_float(0x7FC00000u);
  const float s = __uint_as_float(amax_bits) / 127.f;
  return s < 1.17549435e-38f ? 0.f : s;
}

// Codes of N values of a row of that scale. fma(x, 1/scale, 1.5 * 2^23) leaves
// the rounded quotient in its low byte; 1/scale is off by half a unit, so a
// quotient within 127 * 2^-24 of a border can come out one too far: the remainder
// x - r * scale is exact (a multiple of scale's last bit below scale), and where
// it reaches half a scale the code is settled by it. That is rare, so it is
// tested for all N at once.
template <int N>
__device__ __forceinline__ void quantize(const float (&x)[N], float scale,
                                         uint32_t (&codes)[N / 4]) {
  constexpr float kMagic = 12582912.f;   // 1.5 * 2^23
  if (!(scale > 0.f)) {   // zeros, or a row with an Inf or NaN
#pragma unroll
    for (int i = 0; i < N / 4; ++i) codes[i] = 0u;
    return;
  }
  const float inv = 1.f / scale;
  float y[N], worst = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    y[i] = fmaf(x[i], inv, kMagic);
    worst = fmaxf(worst, fabsf(fmaf(kMagic - y[i], scale, x[i])));
  }
  if (worst + worst >= scale) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float r = y[i] - kMagic, t = fmaf(-r, scale, x[i]), t2 = fabsf(t + t);
      const bool odd = ((int)r & 1) != 0;
      if (t2 > scale || (t2 == scale && odd)) y[i] += t > 0.f ? 1.f : -1.f;
    }
  }
#pragma unroll
  for (int i = 0; i < N / 4; ++i)
    codes[i] = (__float_as_uint(y[4 * i]) & 0xFFu) | ((__float_as_uint(y[4 * i + 1]) & 0xFFu) << 8) |
               ((__float_as_uint(y[4 * i + 2]) & 0xFFu) << 16) |
               (__float_as_uint(y[4 * i + 3]) << 24);
}

// N values of a row, 16-byte loads.
template <int N>
__device__ __forceinline__ void load_row(float (&x)[N], const bf16_t* p) {
#pragma unroll
  for (int i = 0; i < N / 8; ++i) {
    const u32x4 v = reinterpret_cast<const u32x4*>(p)[i];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      x[8 * i + 2 * w] = __uint_as_float(v[w] << 16);
      x[8 * i + 2 * w + 1] = __uint_as_float(v[w] & 0xFFFF0000u);
    }
  }
}
template <int N>
__device__ __forceinline__ void load_row(float (&x)[N], const float* p) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const f32x4 v = reinterpret_cast<const f32x4*>(p)[i];
#pragma unroll
    for (int w = 0; w < 4; ++w) x[4 * i + w] = v[w];
  }
}
template <int N>
__device__ __forceinline__ uint32_t amax_bits(const float (&x)[N]) {
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t a = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    m = a > m ? a : m;
  }
  return m;
}
// Maximum over the LANES lanes (a power of two) that share a row.
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t m) {
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) {
    const uint32_t v = __shfl_xor(m, o, 64);
    m = v > m ? v : m;
  }
  return m;
}

// Values of a row that a lane has: 32 bytes.
template <typename E>
__host__ __device__ constexpr int per_lane() { return 32 / (int)sizeof(E); }

// N / 4 words of codes.
template <int N>
__device__ __forceinline__ void store_codes(int8_t* p, const uint32_t (&c)[N / 4]) {
  if constexpr (N == 16) *reinterpret_cast<u32x4*>(p) = u32x4{c[0], c[1], c[2], c[3]};
  else *reinterpret_cast<uint2*>(p) = make_uint2(c[0], c[1]);
}
// A row of K and one of V into slot `dst` (of all heads) of an 8-bit cache, if ok; lane
// `part` of the D / per_lane lanes that share the rows, which are all here.
template <int D, typename E>
__device__ __forceinline__ void put_rows(const CacheQ8& c, const E* k_src, const E* v_src,
                                         size_t dst, bool ok, int part) {
  constexpr int N = per_lane<E>(), LPR = D / N;
  float x[N], y[N];
  load_row<N>(x, k_src + N * part);
  load_row<N>(y, v_src + N * part);
  const float sx = row_scale(lanes_max<LPR>(amax_bits<N>(x)));
  const float sy = row_scale(lanes_max<LPR>(amax_bits<N>(y)));
  if (!ok) return;
  uint32_t cx[N / 4], cy[N / 4];
  quantize<N>(x, sx, cx);
  quantize<N>(y, sy, cy);
  store_codes<N>(c.k + dst * D + N * part, cx);
  store_codes<N>(c.v + dst * D + N * part, cy);
  if (part == 0) {
    c.ks[dst] = sx;
    c.vs[dst] = sy;
  }
}

}  // namespace q8
}  // namespace h2o
