// The 8-bit cache: rows of K and V quantised into their slots, and read back
// (row format and rounding: q8.h).
//
// Bound by memory: a row of d values is read once (2 d or 4 d bytes) and d + 4
// bytes are written, or the reverse. A lane has kPer consecutive values of K and the
// same of V, 32 bytes each: loads and stores of both tensors in flight together, the
// row's maximum by exchanges between its lanes, no LDS and no barrier. (Float32 with 16
// values a lane, 64 bytes: B3 Hkv16 d64, 3,001 rows written and read back 49 us, with 8
// 42.) B4 Hkv8 d128 bf16, 32,768 rows: 300 us for both calls, 5.4 TB/s.
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

template <int N>
__device__ __forceinline__ void load_codes(uint32_t (&c)[N / 4], const int8_t* p) {
  if constexpr (N == 16) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = v[i];
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    c[0] = v.x;
    c[1] = v.y;
  }
}

template <int D, typename E>
__global__ __launch_bounds__(kThreads) void quantize_rows(
    const E* __restrict__ k_src, const E* __restrict__ v_src, const int32_t* __restrict__ idx,
    int8_t* __restrict__ kc, float* __restrict__ ks, int8_t* __restrict__ vc,
    float* __restrict__ vs, uint32_t nrows, int M, uint32_t k, InsertArgs ins) {
  constexpr int LPR = D / per_lane<E>();
  const uint32_t row = blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
  if (row >= nrows) return;   // whole rows: the lanes of a row leave together
  const int part = threadIdx.x % LPR;
  const uint32_t bh = row / k, i = row % k;
  const int slot = idx ? idx[row] : (int)i;
  const bool ok = (unsigned)slot < (unsigned)M;
  const size_t dst = (size_t)bh * M + slot;
  put_rows<D, E>(CacheQ8{kc, ks, vc, vs}, k_src + (size_t)row * D, v_src + (size_t)row * D, dst, ok,
                 part);
  if (ok && part == 0 && ins.scores) {
    ins.scores[dst] = ins.wsum[(size_t)bh * (M + ins.T) + M + i];
    if (ins.token_pos) ins.token_pos[dst] = ins.pos0 + (int32_t)i;
  }
}

template <int N>
__device__ __forceinline__ void store_values(float* p, const uint32_t (&c)[N / 4], float s) {
#pragma unroll
  for (int w = 0; w < N / 4; ++w)
    reinterpret_cast<f32x4*>(p)[w] =
        f32x4{code_f32(c[w], 0), code_f32(c[w], 1), code_f32(c[w], 2), code_f32(c[w], 3)} * s;
}
template <int N>
__device__ __forceinline__ void store_values(bf16_t* p, const uint32_t (&c)[N / 4], float s) {
#pragma unroll
  for (int w = 0; w < N / 8; ++w) {
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
  constexpr int N = per_lane<E>(), LPR = D / N;
  const uint32_t row = blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
  if (row >= nrows) return;
  const int part = threadIdx.x % LPR;
  const int slot = idx ? idx[row] : (int)(row % k);
  if ((unsigned)slot >= (unsigned)M) return;
  const size_t src = (size_t)(row / k) * M + slot, dst = (size_t)row * D + N * part;
  uint32_t a[N / 4], b[N / 4];
  load_codes<N>(a, kc + src * D + N * part);
  load_codes<N>(b, vc + src * D + N * part);
  const float sa = ks[src], sb = vs[src];
  store_values<N>(k_dst + dst, a, sa);
  store_values<N>(v_dst + dst, b, sb);
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
  const uint32_t per = kThreads / (d / (f32 ? per_lane<float>() : per_lane<bf16_t>()));
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
  const uint32_t per = kThreads / (d / (f32 ? per_lane<float>() : per_lane<bf16_t>()));
  return with_form(d, f32, [&](auto D, auto e) {
    typedef decltype(e) E;
    return launch_kernel(K_KV_QUANT, dequantize_rows<decltype(D)::value, E>,
                         dim3((n + per - 1) / per), dim3(kThreads), st, (const int8_t*)c.k,
                         (const float*)c.ks, (const int8_t*)c.v, (const float*)c.vs, idx,
                         (E*)k_dst, (E*)v_dst, n, M, (uint32_t)k);
  });
}

}  // namespace h2o
