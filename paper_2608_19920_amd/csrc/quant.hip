// The 8-bit cache: rows of K and V quantised into their slots, and read back
// (row format and rounding: q8.h).
//
// Bound by memory: a row of d values is read once (2 d or 4 d bytes) and d + 4
// bytes are written, or the reverse. Lane l of the d / 16 lanes that share a row
// has 16 consecutive values of K and the same of V: 16-byte loads and stores of
// both tensors in flight together, the row's maximum by exchanges between its
// lanes, no LDS and no barrier.
#include "internal.h"
#include "q8.h"

namespace h2o {
namespace {

using namespace q8;

constexpr int kThreads = 256;

// Row i of head bh goes to slot idx[bh][i] (idx null: slot i); slots outside
// [0, M) are skipped. With scores non-null, the insert of an eviction as well:
// the slot's score becomes wsum[bh][M + i] (row pitch M + T) and its position
// pos0 + i.
struct InsertArgs {
  float* scores;
  int32_t* token_pos;
  const float* wsum;
  int T;
  int32_t pos0;
};

template <int D, typename E>
__global__ __launch_bounds__(kThreads) void quantize_rows(
    const E* __restrict__ k_src, const E* __restrict__ v_src, const int32_t* __restrict__ idx,
    int8_t* __restrict__ kc, float* __restrict__ ks, int8_t* __restrict__ vc,
    float* __restrict__ vs, uint32_t nrows, int M, uint32_t k, InsertArgs ins) {
  constexpr int LPR = D / 16;
  const uint32_t row = blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
  if (row >= nrows) return;   // whole rows: the lanes of a row leave together
  const int part = threadIdx.x % LPR;
  const uint32_t bh = row / k, i = row % k;
  const size_t src = (size_t)row * D + 16 * part;
  float x[16], y[16];
  load_row<16>(x, k_src + src);
  load_row<16>(y, v_src + src);
  const int slot = idx ? idx[row] : (int)i;
  const float sx = row_scale(lanes_max<LPR>(amax_bits<16>(x)));
  const float sy = row_scale(lanes_max<LPR>(amax_bits<16>(y)));
  if ((unsigned)slot >= (unsigned)M) return;
  uint32_t cx[4], cy[4];
  quantize<16>(x, sx, cx);
  quantize<16>(y, sy, cy);
  const size_t dst = (size_t)bh * M + slot;
  *reinterpret_cast<u32x4*>(kc + dst * D + 16 * part) = u32x4{cx[0], cx[1], cx[2], cx[3]};
  *reinterpret_cast<u32x4*>(vc + dst * D + 16 * part) = u32x4{cy[0], cy[1], cy[2], cy[3]};
  if (part == 0) {
    ks[dst] = sx;
    vs[dst] = sy;
    if (ins.scores) {
      ins.scores[dst] = ins.wsum[(size_t)bh * (M + ins.T) + M + i];
      if (ins.token_pos) ins.token_pos[dst] = ins.pos0 + (int32_t)i;
    }
  }
}

__device__ __forceinline__ void store_values(float* p, const u32x4& c, float s) {
#pragma unroll
  for (int w = 0; w < 4; ++w)
    reinterpret_cast<f32x4*>(p)[w] =
        f32x4{code_f32(c[w], 0), code_f32(c[w], 1), code_f32(c[w], 2), code_f32(c[w], 3)} * s;
}
__device__ __forceinline__ void store_values(bf16_t* p, const u32x4& c, float s) {
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)(code_f32(c[2 * w + (i >> 2)], i & 3) * s);
    reinterpret_cast<bf16x8*>(p)[w] = r;
  }
}

template <int D, typename E>
__global__ __launch_bounds__(kThreads) void dequantize_rows(
    const int8_t* __restrict__ kc, const float* __restrict__ ks, const int8_t* __restrict__ vc,
    const float* __restrict__ vs, const int32_t* __restrict__ idx, E* __restrict__ k_dst,
    E* __restrict__ v_dst, uint32_t nrows, int M, uint32_t k) {
  constexpr int LPR = D / 16;
  const uint32_t row = blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
  if (row >= nrows) return;
  const int part = threadIdx.x % LPR;
  const int slot = idx ? idx[row] : (int)(row % k);
  if ((unsigned)slot >= (unsigned)M) return;
  const size_t src = (size_t)(row / k) * M + slot, dst = (size_t)row * D + 16 * part;
  const u32x4 a = *reinterpret_cast<const u32x4*>(kc + src * D + 16 * part);
  const u32x4 b = *reinterpret_cast<const u32x4*>(vc + src * D + 16 * part);
  const float sa = ks[src], sb = vs[src];
  store_values(k_dst + dst, a, sa);
  store_values(v_dst + dst, b, sb);
}

template <typename F>
hipError_t with_form(int d, bool f32, F&& f) {
  if (d == 64) return f32 ? f(IntConst<64>{}, float{}) : f(IntConst<64>{}, bf16_t{});
  return f32 ? f(IntConst<128>{}, float{}) : f(IntConst<128>{}, bf16_t{});
}

}  // namespace

hipError_t launch_kv_quantize(const void* k_src, const void* v_src, const int32_t* idx,
                              const CacheQ8& c, int rows, int M, int k, int d, bool f32,
                              hipStream_t st, float* scores, int32_t* token_pos,
                              const float* wsum, int T, int32_t pos0) {
  const uint32_t n = (uint32_t)rows * (uint32_t)k;
  if (n == 0) return hipSuccess;
  const uint32_t per = kThreads / (d / 16);
  return with_form(d, f32, [&](auto D, auto e) {
    typedef decltype(e) E;
    return launch_kernel(K_KV_QUANT, quantize_rows<decltype(D)::value, E>, dim3((n + per - 1) / per),
                         dim3(kThreads), st, (const E*)k_src, (const E*)v_src, idx, c.k, c.ks, c.v,
                         c.vs, n, M, (uint32_t)k, InsertArgs{scores, token_pos, wsum, T, pos0});
  });
}

hipError_t launch_kv_dequantize(const CacheQ8& c, const int32_t* idx, void* k_dst, void* v_dst,
                                int rows, int M, int k, int d, bool f32, hipStream_t st) {
  const uint32_t n = (uint32_t)rows * (uint32_t)k;
  if (n == 0) return hipSuccess;
  const uint32_t per = kThreads / (d / 16);
  return with_form(d, f32, [&](auto D, auto e) {
    typedef decltype(e) E;
    return launch_kernel(K_KV_QUANT, dequantize_rows<decltype(D)::value, E>,
                         dim3((n + per - 1) / per), dim3(kThreads), st, (const int8_t*)c.k,
                         (const float*)c.ks, (const int8_t*)c.v, (const float*)c.vs, idx,
                         (E*)k_dst, (E*)v_dst, n, M, (uint32_t)k);
  });
}

}  // namespace h2o
