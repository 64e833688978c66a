// The kernels of flash.hip for float32 data, on the float32 matrix cores (gfx950):
// v_mfma_f32_16x16x4_f32, operands in the order of f32_mfma.hip (lane (i, g) reads
// the 16-byte pieces 16t + 4g of a row; element u of a piece feeds one product).
// 8-bit rows become float32 values on their way into LDS. Bound by the matrix
// cores (32 cycles a product of 16 x 16 x 4) where a chunk has many rows.
//
// A query and a key that do not see each other contribute 0 whatever the values
// are: hidden scores are replaced before the maximum, and a chunk tile whose
// values are not all finite is added key by key, without the hidden pairs.
#include "internal.h"
#include "q8.h"

namespace h2o {
namespace {

using q8::f32x4;
using q8::u32x4;

constexpr int BN = 32;          // keys per tile
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kVmem0 = 0x0F70;  // s_waitcnt vmcnt(0)

__device__ __forceinline__ f32x4 mma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 load4(const float* p) {
  return *reinterpret_cast<const f32x4*>(p);
}
__host__ __device__ constexpr int lds_pitch(int D) { return D + 4; }

struct Args {
  const float* q;
  const void *kc, *vc;
  const float *ks, *vs;
  const float *kn, *vn;
  const int32_t* parents;
  const uint32_t* bits;
  int Hq, Hkv, G, T, M, R, W;
  float c, c_lo;                // scale * log2(e), and what c is short of it
};

// A tile's rows in registers; rows past the tile's end are zeros.
template <int D, bool Q8>
struct Regs {
  static constexpr int N = BN * D / 4 / kThreads;   // 16-byte units of float32 rows
  f32x4 k[N], v[N];
  u32x4 kq, vq;
  float ks, vs;
};
template <int D>
__device__ __forceinline__ void load_rows(f32x4 (&r)[BN * D / 4 / kThreads], const float* base,
                                          int n) {
#pragma unroll
  for (int e = 0; e < BN * D / 4 / kThreads; ++e) {
    const int u = threadIdx.x + e * kThreads, row = u / (D / 4);
    r[e] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (row < n) r[e] = load4(base + (uint32_t)(row * D + 4 * (u % (D / 4))));
  }
}
template <int D, bool Q8>
__device__ __forceinline__ void load_tile(Regs<D, Q8>& g, const Args& a, size_t bh, int t, int tc) {
  if (t < tc) {
    const int j0 = t * BN, n = min(BN, a.M - j0);
    const size_t row = bh * (size_t)a.M + j0;
    if constexpr (Q8) {
      const int u = threadIdx.x, r = u / (D / 16);
      g.kq = g.vq = u32x4{0u, 0u, 0u, 0u};
      g.ks = g.vs = 0.f;
      if (r < n) {   // n <= BN rows: the threads of a whole tile at D = 128, half at 64
        g.kq = reinterpret_cast<const u32x4*>((const int8_t*)a.kc + row * D)[u];
        g.vq = reinterpret_cast<const u32x4*>((const int8_t*)a.vc + row * D)[u];
        g.ks = a.ks[row + r];
        g.vs = a.vs[row + r];
      }
    } else {
      load_rows<D>(g.k, (const float*)a.kc + row * D, n);
      load_rows<D>(g.v, (const float*)a.vc + row * D, n);
    }
  } else {
    const int j0 = (t - tc) * BN, n = min(BN, a.T - j0);
    const size_t row = bh * (size_t)a.T + j0;
    load_rows<D>(g.k, a.kn + row * D, n);
    load_rows<D>(g.v, a.vn + row * D, n);
  }
}
template <int D>
__device__ __forceinline__ void store_codes(float* lds, const u32x4& c, float s) {
  const int u = threadIdx.x, row = u / (D / 16);
  if (row >= BN) return;
#pragma unroll
  for (int w = 0; w < 4; ++w)
    *reinterpret_cast<f32x4*>(lds + row * lds_pitch(D) + 16 * (u % (D / 16)) + 4 * w) =
        f32x4{q8::code_f32(c[w], 0), q8::code_f32(c[w], 1), q8::code_f32(c[w], 2),
              q8::code_f32(c[w], 3)} * s;
}
// Returns whether this thread stored a value that is not finite (chunk tiles).
template <int D, bool Q8>
__device__ __forceinline__ bool store_tile(float* Ks, float* Vs, const Regs<D, Q8>& g, int t,
                                           int tc) {
  if (Q8 && t < tc) {
    store_codes<D>(Ks, g.kq, g.ks);
    store_codes<D>(Vs, g.vq, g.vs);
    return false;
  }
  float z = 0.f;
#pragma unroll
  for (int e = 0; e < Regs<D, Q8>::N; ++e) {
    const int u = threadIdx.x + e * kThreads, o = u / (D / 4) * lds_pitch(D) + 4 * (u % (D / 4));
    *reinterpret_cast<f32x4*>(Ks + o) = g.k[e];
    *reinterpret_cast<f32x4*>(Vs + o) = g.v[e];
#pragma unroll
    for (int i = 0; i < 4; ++i) z = fmaf(g.v[e][i], 0.f, z);
  }
  return z != 0.f;   // 0, or NaN
}

// 64 packed rows per block, 16 per wave.
template <int D, bool Q8, bool TREE>
__global__ __launch_bounds__(kThreads) void flash_f32(Args a, int nsplit, float* __restrict__ out,
                                                      float* __restrict__ lse,
                                                      float2* __restrict__ stats,
                                                      float* __restrict__ opart) {
  constexpr int ROWS = kWaves * 16, P = lds_pitch(D), NK = BN / 16;
  __shared__ __attribute__((aligned(16))) float Ks2[2][BN * P];
  __shared__ __attribute__((aligned(16))) float Vs2[2][BN * P];
  __shared__ int odd[3];            // by tile: it holds a value that is not finite
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nrt = gridDim.x / nsplit, rt = nrt - 1 - (int)blockIdx.x % nrt;
  const int sp = (int)blockIdx.x / nrt;
  const size_t bh = blockIdx.y;
  const int b = (int)bh / a.Hkv, h = (int)bh % a.Hkv;
  const int row0 = rt * ROWS, r = row0 + wave * 16 + l16;
  const bool ok = r < a.R;
  const int i = ok ? r / a.G : 0, gg = ok ? r % a.G : 0;
  const size_t orow = (size_t)(b * a.Hq + h * a.G + gg) * a.T + i;
  const int tc = (a.M + BN - 1) / BN;
  const int i_max = (min(row0 + ROWS, a.R) - 1) / a.G;
  const int ntiles = tc + i_max / BN + 1, per = (ntiles + nsplit - 1) / nsplit;
  const int t0 = min(ntiles, sp * per), t1 = min(ntiles, t0 + per);
  f32x4 qf[D / 16], acc[D / 64][4];
#pragma unroll
  for (int x = 0; x < D / 16; ++x) qf[x] = load4(a.q + orow * D + 16 * x + 4 * g4);
#pragma unroll
  for (int x = 0; x < D / 64; ++x)
#pragma unroll
    for (int u = 0; u < 4; ++u) acc[x][u] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  Regs<D, Q8> g;
  // two LDS buffers, one barrier a tile: tile t + 1 goes from registers to the other
  // buffer, and tile t + 2 is requested, before tile t is used. The flag of a tile is
  // cleared two barriers before it can be set.
  auto put = [&](int t) {
    const bool bad = store_tile<D, Q8>(Ks2[(t - t0) & 1], Vs2[(t - t0) & 1], g, t, tc);
    if (bad && t >= tc) odd[(t - t0) % 3] = 1;
  };
  if (threadIdx.x < 3) odd[threadIdx.x] = 0;
  __syncthreads();
  uint64_t own = 0u;
  if constexpr (TREE)
    if (a.T <= kWaveTree)
      own = __shfl(wave_ancestors(a.parents + (size_t)b * a.T, a.T, lane), i, 64);
  auto word = [&](int t) {   // the chunk keys of tile t that the row's node sees
    if (t < tc) return 0u;
    return a.T <= kWaveTree ? (uint32_t)(own >> (t > tc ? 32 : 0))
                            : a.bits[((size_t)b * a.T + i) * a.W + (t - tc)];
  };
  uint32_t next = 0u;
  if (t0 < t1) {
    if constexpr (TREE) next = word(t0);
    load_tile<D, Q8>(g, a, bh, t0, tc);
    put(t0);
    if (t0 + 1 < t1) load_tile<D, Q8>(g, a, bh, t0 + 1, tc);
  }
  for (int t = t0; t < t1; ++t) {
    const bool cache = t < tc;
    __syncthreads();                // tile t is in LDS, tile t - 1 used up
    // tile t + 1 and the tree's word of tile t are here: a wait for the word where it is
    // used would be one for tile t + 2 as well (B1 Hq32 Hkv8 d128 M8192, 32 nodes: 62 ->
    // 59 us; a chunk, which has no such word, is slower with it, 203 -> 212)
    if constexpr (TREE) __builtin_amdgcn_s_waitcnt(kVmem0);
    if (threadIdx.x == 0) odd[(t - t0 + 2) % 3] = 0;
    const float* Ks = Ks2[(t - t0) & 1];
    const float* Vs = Vs2[(t - t0) & 1];
    const bool finite = !odd[(t - t0) % 3];
    const uint32_t seen = next;
    if (t + 1 < t1) {
      put(t + 1);
      if constexpr (TREE) next = word(t + 1);
      if (t + 2 < t1) load_tile<D, Q8>(g, a, bh, t + 2, tc);
    }
    f32x4 s[NK];
    uint32_t hidden = 0u;
    float mn = m;
#pragma unroll
    for (int kb = 0; kb < NK; ++kb) {
      f32x4 s4[4];                  // shorter sums round less
#pragma unroll
      for (int u = 0; u < 4; ++u) s4[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < D / 16; ++x) {
        const f32x4 kf = load4(&Ks[(16 * kb + l16) * P + 16 * x + 4 * g4]);
#pragma unroll
        for (int u = 0; u < 4; ++u) s4[u] = mma4(kf[u], qf[x][u], s4[u]);
      }
      s[kb] = (s4[0] + s4[1]) + (s4[2] + s4[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = 16 * kb + 4 * g4 + e;
        const bool hid = cache ? t * BN + j >= a.M
                         : TREE ? !((seen >> j) & 1u) : (t - tc) * BN + j > i;
        s[kb][e] = hid ? -INFINITY : s[kb][e] * a.c;
        hidden |= hid ? 1u << (4 * kb + e) : 0u;
        mn = fmaxf(mn, s[kb][e]);
      }
    }
    mn = fmaxf(mn, __shfl_xor(mn, 16, 64));
    mn = fmaxf(mn, __shfl_xor(mn, 32, 64));
    const float mu = mn == -INFINITY ? 0.f : mn;
    if (__builtin_amdgcn_ballot_w64(mn > m)) {
      const float f = __builtin_amdgcn_exp2f(m - mu);
      l *= f;
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[x][u] *= f;
      m = mn;
    }
#pragma unroll
    for (int kb = 0; kb < NK; ++kb)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[kb][e] = __builtin_amdgcn_exp2f(s[kb][e] - mu);
        l += s[kb][e];
      }
    if (finite) {   // block-uniform
#pragma unroll
      for (int kb = 0; kb < NK; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int x = 0; x < D / 64; ++x) {
            const f32x4 v = load4(&Vs[(16 * kb + 4 * g4 + e) * P + 64 * x + 4 * l16]);
#pragma unroll
            for (int u = 0; u < 4; ++u) acc[x][u] = mma4(v[u], s[kb][e], acc[x][u]);
          }
    } else {
#pragma unroll 1
      for (int j = 0; j < BN; ++j) {
        const int from = l16 + 16 * ((j & 15) >> 2), bit = 4 * (j >> 4) + (j & 3);
        float w = 0.f;
#pragma unroll
        for (int e = 0; e < 4 * NK; ++e) w = e == bit ? s[e >> 2][e & 3] : w;
        w = __shfl(w, from, 64);
        const bool hid = (__shfl(hidden, from, 64) >> bit) & 1u;
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const f32x4 v = load4(&Vs[j * P + 64 * x + 16 * g4 + 4 * e]);
#pragma unroll
            for (int u = 0; u < 4; ++u)
              acc[x][u][e] = hid ? acc[x][u][e] : fmaf(w, v[u], acc[x][u][e]);
          }
      }
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (!ok) return;
  const size_t prow = ((size_t)sp * gridDim.y + bh) * a.R + r;
  if (g4 == 0) {
    if (nsplit == 1) lse[orow] = (m + __log2f(l)) * kLn2;
    else stats[prow] = make_float2(m, l);
  }
  float* dst = nsplit == 1 ? out + orow * D : opart + prow * D;
  const float f = nsplit == 1 ? 1.f / l : 1.f;
#pragma unroll
  for (int x = 0; x < D / 64; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<f32x4*>(dst + 64 * x + 16 * g4 + 4 * e) =
          f32x4{acc[x][0][e], acc[x][1][e], acc[x][2][e], acc[x][3][e]} * f;
}

struct ColArgs {
  const float* lse;
  const int32_t* path;
  int A, R;
  float *dst, *k_acc, *v_acc;
  ScoreAcc acc;
};
constexpr int kQRows = 32;

// As column_pass of flash.hip: 16 keys per wave, in registers.
template <int D, bool Q8, bool PATH>
__global__ __launch_bounds__(kThreads) void column_f32(Args a, ColArgs p) {
  constexpr int KB = kWaves * 16, P = lds_pitch(D), NU = kQRows * D / 4 / kThreads;
  __shared__ __attribute__((aligned(16))) float Qs[2][kQRows * P];
  __shared__ float2 lam[2][kQRows];
  __shared__ int pos[2][kQRows];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const size_t bh = blockIdx.y;
  const int b = (int)bh / a.Hkv, h = (int)bh % a.Hkv;
  const int tc = (a.M + KB - 1) / KB, tn = (p.A + KB - 1) / KB;
  const int32_t* path = PATH ? p.path + (size_t)b * p.A : nullptr;
  auto node_of = [&](int i) {
    if (!PATH) return i;
    const int n = path[i];
    return (unsigned)n < (unsigned)a.T ? n : -1;
  };
  if (PATH && (int)blockIdx.x >= tc + tn) {   // the path's rows
    const int e = ((int)blockIdx.x - tc - tn) * kThreads + tid, i = e / (D / 4), c = e % (D / 4);
    if (blockIdx.z || i >= p.A) return;
    const int n = node_of(i);
    f32x4 kv = {0.f, 0.f, 0.f, 0.f}, vv = kv;
    if (n >= 0) {
      kv = load4(a.kn + (bh * a.T + n) * (size_t)D + 4 * c);
      vv = load4(a.vn + (bh * a.T + n) * (size_t)D + 4 * c);
    }
    reinterpret_cast<f32x4*>(p.k_acc + (bh * p.A + i) * (size_t)D)[c] = kv;
    reinterpret_cast<f32x4*>(p.v_acc + (bh * p.A + i) * (size_t)D)[c] = vv;
    return;
  }
  const bool cache = (int)blockIdx.x < tc;
  const int j0 = (cache ? (int)blockIdx.x : (int)blockIdx.x - tc) * KB + wave * 16;
  const int nkeys = cache ? a.M : p.A;
  f32x4 kf[D / 16], cs = {0.f, 0.f, 0.f, 0.f};
  const int j = min(j0 + l16, nkeys - 1);
  if (Q8 && cache) {
    const int8_t* src = (const int8_t*)a.kc + (bh * a.M + j) * (size_t)D;
    const float s = a.ks[bh * a.M + j];
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(src + 16 * x + 4 * g4);
      kf[x] = f32x4{q8::code_f32(w, 0), q8::code_f32(w, 1), q8::code_f32(w, 2),
                    q8::code_f32(w, 3)} * s;
    }
  } else {
    const int n = cache ? j : max(node_of(j), 0);
    const float* src = cache ? (const float*)a.kc + (bh * a.M + n) * (size_t)D
                             : a.kn + (bh * a.T + n) * (size_t)D;
#pragma unroll
    for (int x = 0; x < D / 16; ++x) kf[x] = load4(src + 16 * x + 4 * g4);
  }
  const int first = cache ? 0 : ((int)blockIdx.x - tc) * KB * a.G / kQRows;
  const int steps = (p.R + kQRows - 1) / kQRows;
  const int per = (steps + (int)gridDim.z - 1) / (int)gridDim.z;
  const int s1 = min(steps, ((int)blockIdx.z + 1) * per), s0 = max(first, (int)blockIdx.z * per);
  // rows as in column_pass: stepped without a division, past the last row kept at it
  constexpr int RU = kThreads / (D / 4);
  f32x4 qr[NU];
  float2 lr = {0.f, 0.f};
  int ir = 0, ri[NU], rg[NU], li, lg;
  const int part = 4 * (tid % (D / 4)), di = kQRows / a.G, dg = kQRows % a.G;
#pragma unroll
  for (int e = 0; e < NU; ++e) {
    const int r = s0 * kQRows + tid / (D / 4) + e * RU;
    ri[e] = r / a.G;
    rg[e] = r % a.G;
  }
  li = (s0 * kQRows + tid) / a.G;
  lg = (s0 * kQRows + tid) % a.G;
  const float* qh = a.q + (size_t)(b * a.Hq + h * a.G) * a.T * D + part;
  const float* lh = p.lse + (size_t)(b * a.Hq + h * a.G) * a.T;
  auto advance = [&](int& i, int& g) {
    i += di;
    g += dg;
    if (g >= a.G) { g -= a.G; ++i; }
  };
  auto load = [&]() {   // the rows of the next step
#pragma unroll
    for (int e = 0; e < NU; ++e) {
      const int n = max(node_of(min(ri[e], p.A - 1)), 0);
      qr[e] = load4(qh + (uint32_t)(rg[e] * a.T + n) * (uint32_t)D);
      advance(ri[e], rg[e]);
    }
    if (tid < kQRows) {
      const int n = li < p.A ? node_of(li) : -1;
      lr = n >= 0 ? row_weight(lh[lg * a.T + n]) : make_float2(INFINITY, 0.f);
      ir = li;
      advance(li, lg);
    }
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int e = 0; e < NU; ++e)
      *reinterpret_cast<f32x4*>(&Qs[buf][(tid / (D / 4) + e * RU) * P + part]) = qr[e];
    if (tid < kQRows) {
      lam[buf][tid] = lr;
      pos[buf][tid] = ir;
    }
  };
  if (s0 < s1) {
    load();
    store(0);
    if (s0 + 1 < s1) load();
    __syncthreads();
  }
  for (int s = s0; s < s1; ++s) {
    const int buf = (s - s0) & 1;
    if (s + 1 < s1) {
      store(buf ^ 1);
      if (s + 2 < s1) load();
    }
    f32x4 w[kQRows / 16], w4[kQRows / 16][4];
#pragma unroll
    for (int n = 0; n < kQRows / 16; ++n)
#pragma unroll
      for (int u = 0; u < 4; ++u) w4[n][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
#pragma unroll
      for (int n = 0; n < kQRows / 16; ++n) {
        const f32x4 qf = load4(&Qs[buf][(16 * n + l16) * P + 16 * x + 4 * g4]);
#pragma unroll
        for (int u = 0; u < 4; ++u) w4[n][u] = mma4(kf[x][u], qf[u], w4[n][u]);
      }
#pragma unroll
    for (int n = 0; n < kQRows / 16; ++n) w[n] = (w4[n][0] + w4[n][1]) + (w4[n][2] + w4[n][3]);
#pragma unroll
    for (int n = 0; n < kQRows / 16; ++n) {
      const float2 la = lam[buf][16 * n + l16];
      const int i = pos[buf][16 * n + l16];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = __builtin_amdgcn_exp2f(fmaf(w[n][r], a.c, -la.x) + w[n][r] * a.c_lo);
        const bool hid = la.x == INFINITY || (!cache && j0 + 4 * g4 + r > i);
        cs[r] = fmaf(hid ? 0.f : x, la.y, cs[r]);
      }
    }
    __syncthreads();
  }
  float* dst = p.dst + ((size_t)blockIdx.z * gridDim.y + bh) * (a.M + p.A) + (cache ? 0 : a.M);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float v = cs[r];
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) v += __shfl_xor(v, o, 64);
    const int jj = j0 + 4 * g4 + r;
    if (l16 == 0 && jj < nkeys) {
      dst[jj] = PATH && !cache && node_of(jj) < 0 ? 0.f : v;
      if (cache) p.acc.add(bh * a.M + jj, v);
    }
  }
}

template <typename F>
hipError_t with_cache(int d, bool q8, F&& f) {
  if (d == 64) return q8 ? f(IntConst<64>{}, IntConst<1>{}) : f(IntConst<64>{}, IntConst<0>{});
  return q8 ? f(IntConst<128>{}, IntConst<1>{}) : f(IntConst<128>{}, IntConst<0>{});
}
Args make_args(const FlashShape& s, const FlashIn& in, const char* ws, const FlashPlan& p,
               float scale) {
  const double c = (double)scale * 1.4426950408889634;
  return Args{(const float*)in.q, in.kc, in.vc, in.ks, in.vs, (const float*)in.kn,
              (const float*)in.vn, in.parents, reinterpret_cast<const uint32_t*>(ws + p.off_bits),
              s.Hq, s.Hkv, s.G(), s.T, s.M, s.G() * s.T, (s.T + 31) / 32, (float)c,
              (float)(c - (float)c)};
}

}  // namespace

hipError_t launch_flash_f32(const FlashShape& s, const FlashPlan& p, const FlashIn& in, void* out,
                            float* lse, char* ws, float scale, hipStream_t st) {
  const bool tree = in.parents != nullptr;
  if (tree && s.T > kWaveTree) {
    const hipError_t e = launch_tree_bits(s, p, in.parents, ws, st);
    if (e != hipSuccess) return e;
  }
  const Args a = make_args(s, in, ws, p, scale);
  const dim3 grid((a.R + p.rows - 1) / p.rows * p.nsplit, s.BH());
  float2* stats = reinterpret_cast<float2*>(ws + p.off_stats);
  float* opart = reinterpret_cast<float*>(ws + p.off_opart);
  const hipError_t e = with_cache(s.d, in.q8, [&](auto D, auto q) {
    constexpr int kD = decltype(D)::value;
    constexpr bool kQ = decltype(q)::value;
    auto go = [&](auto kern) {
      return launch_kernel(K_FLASH, kern, grid, dim3(kThreads), st, a, p.nsplit, (float*)out, lse,
                           stats, opart);
    };
    if (tree) return go(flash_f32<kD, kQ, true>);
    if constexpr (kQ) return go(flash_f32<kD, true, false>);
    return hipErrorInvalidValue;
  });
  if (e != hipSuccess || p.nsplit == 1) return e;
  return launch_flash_combine(s, p, out, lse, ws, st);
}

hipError_t launch_columns_f32(const FlashShape& s, const FlashPlan& p, const FlashIn& in,
                              const float* lse, const int32_t* path, int A, void* k_acc,
                              void* v_acc, float* wsum, char* ws, float scale, hipStream_t st,
                              ScoreAcc acc) {
  const Args a = make_args(s, in, ws, p, scale);
  float* parts = reinterpret_cast<float*>(ws + p.off_parts);
  const int ncol = path ? A : s.T, kb = kColumnKeysF32;
  const int tiles = (s.M + kb - 1) / kb + (ncol + kb - 1) / kb;
  const int ncopy = path ? (A * (s.d / 4) + kThreads - 1) / kThreads : 0;
  const ColArgs c{lse, path, ncol, s.G() * ncol, p.nranges > 1 ? parts : wsum, (float*)k_acc,
                  (float*)v_acc, p.nranges > 1 ? ScoreAcc{} : acc};
  const dim3 grid(tiles + ncopy, s.BH(), p.nranges);
  const hipError_t e = with_cache(s.d, in.q8, [&](auto D, auto q) {
    constexpr int kD = decltype(D)::value;
    constexpr bool kQ = decltype(q)::value;
    auto go = [&](auto kern) {
      return launch_kernel(K_COLUMNS, kern, grid, dim3(kThreads), st, a, c);
    };
    if (path) return go(column_f32<kD, kQ, true>);
    if constexpr (kQ) return go(column_f32<kD, true, false>);
    return hipErrorInvalidValue;
  });
  if (e != hipSuccess || p.nranges == 1) return e;
  return launch_column_reduce(parts, wsum, s.BH(), s.M, ncol, p.nranges, acc, st);
}

}  // namespace h2o
