// bf16 attention in one sweep over the keys, and the column sums in a second
// (gfx950): chunks over an 8-bit cache, and the nodes of a drafted token tree over
// either cache.
//
//   flash    out and lse of a tile of packed rows over a range of key tiles, with
//            a running maximum and sum; several ranges leave (m, l, O) partials
//   combine  merges the partials of a row in the order of the ranges
//   columns  wsum_j = sum_rows exp2(c s_rj - lambda_r) with the finished lambda: a
//            wave keeps its keys in registers and goes over the rows, so a key's
//            sum stays in one lane group until the end (no partial sums per tile)
//
// Matrix products are v_mfma_f32_16x16x32_bf16 in the S^T = K Q^T orientation: the
// accumulators of two 16-key blocks are the operand of O^T += V^T P^T. A cache
// tile is whole or ends at slot M, a chunk tile starts at chunk key 0: no tile
// holds both, so the mask is asked of the last cache tile and the chunk tiles
// alone.
//
// 8-bit rows become bf16 codes on their way into LDS (exact); the key's scale
// multiplies the scores, the value's scale the probabilities.
#include "internal.h"
#include "mfma_ops.h"
#include "q8.h"

namespace h2o {
namespace {

using namespace mfma;

constexpr int BN = 64;          // keys per tile
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kXcds = 8;

__host__ __device__ constexpr int lds_pitch(int D) { return D + 16; }   // bf16 per LDS row

struct Args {
  const bf16_t* q;
  const void *kc, *vc;          // [BH][M][D], bf16 or codes
  const float *ks, *vs;         // [BH][M], 8-bit cache
  const bf16_t *kn, *vn;        // [BH][T][D]
  const uint32_t* bits;         // tree: [B][T][W] ancestor bits, a node's own among them
  int Hq, Hkv, G, T, M, R, W;
  float c;                      // scale * log2(e)
};

// Blocks reach the 8 XCDs round-robin: the row tiles of one (head, key range),
// which read the same keys, go to one XCD and share its L2, last rows first.
struct BlockId { int rt, sp, bh; };
__device__ __forceinline__ BlockId block_id(int nsplit) {
  const int nrt = gridDim.x / nsplit, ngroups = nsplit * gridDim.y;
  const int lin = blockIdx.x + blockIdx.y * gridDim.x;
  int grp = lin / nrt, i = lin % nrt;
  if (ngroups % kXcds == 0) {
    const int n = lin / kXcds;
    grp = (n / nrt) * kXcds + lin % kXcds;
    i = n % nrt;
  }
  return BlockId{nrt - 1 - i, grp % nsplit, grp / nsplit};
}

// ------------------------------------------------------------------- staging
// A tile's rows in registers: 16-byte units, 16 codes or 8 bf16 each.
template <int D>
struct Regs {
  static constexpr int N16 = BN * D / 8 / kThreads;
  u32x4 k[N16], v[N16];
  float s;                      // thread t < BN: scale of key t; BN <= t < 2 BN: of value t - BN
};

template <int D>
__device__ __forceinline__ void load_rows16(u32x4 (&r)[Regs<D>::N16], const void* base, int n) {
  const char* p = reinterpret_cast<const char*>(base);
#pragma unroll
  for (int e = 0; e < Regs<D>::N16; ++e) {
    const int u = threadIdx.x + e * kThreads, row = min(u / (D / 8), n - 1);
    r[e] = *reinterpret_cast<const u32x4*>(p + (uint32_t)(row * D + 8 * (u % (D / 8))) * 2u);
  }
}
template <int D>
__device__ __forceinline__ void load_rows8(u32x4 (&r)[Regs<D>::N16], const void* base, int n) {
  const char* p = reinterpret_cast<const char*>(base);
#pragma unroll
  for (int e = 0; e < Regs<D>::N16 / 2; ++e) {
    const int u = threadIdx.x + e * kThreads, row = min(u / (D / 16), n - 1);
    r[e] = *reinterpret_cast<const u32x4*>(p + (uint32_t)(row * D + 16 * (u % (D / 16))));
  }
}
template <int D>
__device__ __forceinline__ void store_rows16(bf16_t* lds, const u32x4 (&r)[Regs<D>::N16]) {
#pragma unroll
  for (int e = 0; e < Regs<D>::N16; ++e) {
    const int u = threadIdx.x + e * kThreads;
    *reinterpret_cast<u32x4*>(lds + u / (D / 8) * lds_pitch(D) + 8 * (u % (D / 8))) = r[e];
  }
}
template <int D>
__device__ __forceinline__ void store_rows8(bf16_t* lds, const u32x4 (&r)[Regs<D>::N16]) {
#pragma unroll
  for (int e = 0; e < Regs<D>::N16 / 2; ++e) {
    const int u = threadIdx.x + e * kThreads;
    bf16x8* dst = reinterpret_cast<bf16x8*>(lds + u / (D / 16) * lds_pitch(D) + 16 * (u % (D / 16)));
    dst[0] = q8::codes_bf16(r[e][0], r[e][1]);
    dst[1] = q8::codes_bf16(r[e][2], r[e][3]);
  }
}

// Rows past the tile's end re-read its last row (in bounds; masked later).
template <int D, bool Q8>
__device__ __forceinline__ void load_tile(Regs<D>& g, const Args& a, size_t bh, int t, int tc) {
  if (t < tc) {
    const int j0 = t * BN, n = min(BN, a.M - j0);
    const size_t row = bh * (size_t)a.M + j0;
    if constexpr (Q8) {
      load_rows8<D>(g.k, (const int8_t*)a.kc + row * D, n);
      load_rows8<D>(g.v, (const int8_t*)a.vc + row * D, n);
      const int r = threadIdx.x % BN;
      if (threadIdx.x < 2 * BN) g.s = (threadIdx.x < BN ? a.ks : a.vs)[row + min(r, n - 1)];
    } else {
      load_rows16<D>(g.k, (const bf16_t*)a.kc + row * D, n);
      load_rows16<D>(g.v, (const bf16_t*)a.vc + row * D, n);
    }
  } else {
    const int j0 = (t - tc) * BN, n = min(BN, a.T - j0);
    const size_t row = bh * (size_t)a.T + j0;
    load_rows16<D>(g.k, a.kn + row * D, n);
    load_rows16<D>(g.v, a.vn + row * D, n);
    if (Q8) g.s = 1.f;
  }
}
template <int D, bool Q8>
__device__ __forceinline__ void store_tile(bf16_t* Ks, bf16_t* Vs, float* sc, const Regs<D>& g,
                                           const Args& a, int t, int tc) {
  if (Q8 && t < tc) {
    store_rows8<D>(Ks, g.k);
    store_rows8<D>(Vs, g.v);
  } else {
    store_rows16<D>(Ks, g.k);
    store_rows16<D>(Vs, g.v);
  }
  if (Q8 && threadIdx.x < 2 * BN) sc[threadIdx.x] = threadIdx.x < BN ? g.s * a.c : g.s;
}

// --------------------------------------------------------------------- flash
// Each wave owns 16 NQB consecutive packed rows r = i*G + g. The reference
// maximum mu of a row (log2 units, common to the 4 lanes that hold it) is raised
// only when a score exceeds it by more than 64, a wave-uniform and rare branch:
// terms stay below 2^64, far inside float32 and bf16.
template <int D, bool Q8, bool TREE, int NQB>
__global__ __launch_bounds__(kThreads) void flash_pass(Args a, int nsplit, bf16_t* __restrict__ out,
                                                       float* __restrict__ lse,
                                                       float2* __restrict__ stats,
                                                       float* __restrict__ opart) {
  constexpr int ROWS = kWaves * NQB * 16, P = lds_pitch(D), NK = BN / 16;
  __shared__ __attribute__((aligned(16))) bf16_t Ks[2][BN * P];
  __shared__ __attribute__((aligned(16))) bf16_t Vs[2][BN * P];
  __shared__ __attribute__((aligned(16))) float sc[2][2 * BN];
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const BlockId id = block_id(nsplit);
  const size_t bh = id.bh;
  const int b = id.bh / a.Hkv, h = id.bh % a.Hkv;
  const int row0 = id.rt * ROWS, wrow0 = row0 + wave * NQB * 16;
  // key tiles of this block: its share of the cache tiles and of the chunk tiles
  // that its last row reaches
  const int tc = (a.M + BN - 1) / BN;
  const int i_max = (min(row0 + ROWS, a.R) - 1) / a.G;
  const int ntiles = tc + i_max / BN + 1;
  const int per = (ntiles + nsplit - 1) / nsplit;
  const int t0 = min(ntiles, id.sp * per), t1 = min(ntiles, t0 + per);
  const int tm = a.M / BN;            // tiles from here on ask for the mask

  bf16x8 qf[NQB][D / 32];
  int qi[NQB];
  float m[NQB], mu[NQB], l[NQB];
  f32x4 oacc[D / 16][NQB];
#pragma unroll
  for (int n = 0; n < NQB; ++n) {
    const int r = wrow0 + 16 * n + l16;
    const bool ok = r < a.R;
    const int i = ok ? r / a.G : 0, gg = ok ? r % a.G : 0;
    const bf16_t* src = a.q + ((size_t)(b * a.Hq + h * a.G + gg) * a.T + i) * D + 8 * g4;
    qi[n] = i;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) qf[n][s] = *reinterpret_cast<const bf16x8*>(src + 32 * s);
    m[n] = -INFINITY;
    mu[n] = 0.f;
    l[n] = 0.f;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) oacc[db][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  auto tile = [&](auto masked, int t, int buf) {
    constexpr bool MASK = decltype(masked)::value;
    f32x4 s[NK][NQB];
#pragma unroll
    for (int kb = 0; kb < NK; ++kb) {
#pragma unroll
      for (int n = 0; n < NQB; ++n) s[kb][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const bf16x8 kf = row_operand(Ks[buf], P, 16 * kb + l16, 32 * x, lane);
#pragma unroll
        for (int n = 0; n < NQB; ++n) s[kb][n] = mma(kf, qf[n][x], s[kb][n]);
      }
    }
    const bool cache = t < tc;
    uint32_t seen[NQB][BN / 32];
    if (MASK && TREE && !cache) {
#pragma unroll
      for (int n = 0; n < NQB; ++n)
#pragma unroll
        for (int w = 0; w < BN / 32; ++w) {
          const int word = (t - tc) * (BN / 32) + w;
          seen[n][w] = word < a.W ? a.bits[((size_t)b * a.T + qi[n]) * a.W + word] : 0u;
        }
    }
    float mx[NQB];
#pragma unroll
    for (int n = 0; n < NQB; ++n) mx[n] = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < NK; ++kb) {
      f32x4 cks;
      if (Q8) cks = *reinterpret_cast<const f32x4*>(&sc[buf][16 * kb + 4 * g4]);
#pragma unroll
      for (int n = 0; n < NQB; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float x = s[kb][n][r] * (Q8 ? cks[r] : a.c);
          if (MASK) {
            const int j = 16 * kb + 4 * g4 + r;
            const bool hid = cache ? t * BN + j >= a.M
                             : TREE ? !((seen[n][kb >> 1] >> (j & 31)) & 1u)
                                    : (t - tc) * BN + j > qi[n];
            if (hid) x = -INFINITY;
          }
          s[kb][n][r] = x;
          mx[n] = fmaxf(mx[n], x);
        }
    }
    bool up = false;
#pragma unroll
    for (int n = 0; n < NQB; ++n) up |= mx[n] > m[n] + 64.f;
    if (__builtin_amdgcn_ballot_w64(up)) {
#pragma unroll
      for (int n = 0; n < NQB; ++n) {
        float x = fmaxf(mx[n], __shfl_xor(mx[n], 16, 64));
        x = fmaxf(x, __shfl_xor(x, 32, 64));
        const bool raise = x > m[n] + 64.f;
        const float f = raise ? __builtin_amdgcn_exp2f(m[n] - x) : 1.f;
        l[n] *= f;
#pragma unroll
        for (int db = 0; db < D / 16; ++db) oacc[db][n] *= f;
        m[n] = raise ? x : m[n];
        mu[n] = raise ? x : mu[n];
      }
    }
#pragma unroll
    for (int kk = 0; kk < BN / 32; ++kk) {
      f32x4 sv[2];
      if (Q8)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          sv[u] = *reinterpret_cast<const f32x4*>(&sc[buf][BN + 32 * kk + 16 * u + 4 * g4]);
      bf16x8 pb[NQB];
#pragma unroll
      for (int n = 0; n < NQB; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = __builtin_amdgcn_exp2f(s[2 * kk + u][n][r] - mu[n]);
            l[n] += p;
            pb[n][4 * u + r] = (__bf16)(Q8 ? p * sv[u][r] : p);
          }
#pragma unroll
      for (int db = 0; db < D / 16; ++db) {
        const bf16x8 vf = tr_operand(Vs[buf] + 32 * kk * P, P, db, lane);
#pragma unroll
        for (int n = 0; n < NQB; ++n) oacc[db][n] = mma(vf, pb[n], oacc[db][n]);
      }
    }
  };

  // two LDS buffers, one barrier a tile: while tile t is used, tile t + 1 goes
  // from registers to the other buffer and the loads of tile t + 2 are in flight
  if (t0 < t1) {
    Regs<D> g;
    load_tile<D, Q8>(g, a, bh, t0, tc);
    store_tile<D, Q8>(Ks[0], Vs[0], sc[0], g, a, t0, tc);
    if (t0 + 1 < t1) load_tile<D, Q8>(g, a, bh, t0 + 1, tc);
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
      const int buf = (t - t0) & 1;
      if (t + 1 < t1) {
        store_tile<D, Q8>(Ks[buf ^ 1], Vs[buf ^ 1], sc[buf ^ 1], g, a, t + 1, tc);
        if (t + 2 < t1) load_tile<D, Q8>(g, a, bh, t + 2, tc);
      }
      if (t < tm) tile(IntConst<0>{}, t, buf);
      else tile(IntConst<1>{}, t, buf);
      __syncthreads();
    }
  }

  const int BH = gridDim.y;
#pragma unroll
  for (int n = 0; n < NQB; ++n) {
    float L = l[n] + __shfl_xor(l[n], 16, 64);
    L += __shfl_xor(L, 32, 64);
    const int r = wrow0 + 16 * n + l16;
    if (r >= a.R) continue;
    const int gg = r % a.G;
    const size_t orow = (size_t)(b * a.Hq + h * a.G + gg) * a.T + qi[n];
    const size_t prow = ((size_t)id.sp * BH + bh) * a.R + r;
    if (g4 == 0) {
      if (nsplit == 1) lse[orow] = (m[n] + __log2f(L)) * kLn2;
      else stats[prow] = make_float2(m[n], L);
    }
    const float inv = 1.f / L;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) {
      const f32x4 o = oacc[db][n];
      if (nsplit == 1) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (__bf16)(o[e] * inv);
        *reinterpret_cast<bf16x4*>(out + orow * D + 16 * db + 4 * g4) = v;
      } else {
        *reinterpret_cast<f32x4*>(opart + prow * D + 16 * db + 4 * g4) = o;
      }
    }
  }
}

// One packed row per D / 4 threads: the ranges' partials in their order.
template <int D, typename E>
__global__ __launch_bounds__(kThreads) void flash_combine(const float2* __restrict__ stats,
                                                          const float* __restrict__ opart,
                                                          E* __restrict__ out,
                                                          float* __restrict__ lse, int BH, int Hq,
                                                          int Hkv, int G, int T, int R,
                                                          int nsplit) {
  constexpr int TPR = D / 4;
  const size_t row = (size_t)blockIdx.x * (kThreads / TPR) + threadIdx.x / TPR;
  if (row >= (size_t)BH * R) return;
  const int c4 = 4 * (threadIdx.x % TPR), bh = (int)(row / R), r = (int)(row % R);
  const size_t plane = (size_t)BH * R;
  float mx = -INFINITY;
  for (int s = 0; s < nsplit; ++s) mx = fmaxf(mx, stats[s * plane + row].x);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float L = 0.f;
  for (int s = 0; s < nsplit; ++s) {
    const float2 st = stats[s * plane + row];
    const f32x4 v = *reinterpret_cast<const f32x4*>(opart + (s * plane + row) * D + c4);
    const float w = st.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.x - mx);
    L = fmaf(w, st.y, L);
    o += w * v;
  }
  const int b = bh / Hkv, h = bh % Hkv;
  const size_t orow = (size_t)(b * Hq + h * G + r % G) * T + r / G;
  if (c4 == 0) lse[orow] = (mx + __log2f(L)) * kLn2;
  const float inv = 1.f / L;
  if constexpr (sizeof(E) == 4) {
    *reinterpret_cast<f32x4*>(out + orow * D + c4) = o * inv;
  } else {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (__bf16)(o[e] * inv);
    *reinterpret_cast<bf16x4*>(out + orow * D + c4) = v;
  }
}

// ------------------------------------------------------------------- columns
// Rows of the sum: all R packed rows of the chunk (path null), or those of the
// path's A nodes, packed row r = a*G + g of node path[b][a]; the chunk's key
// columns are then the path's. Entries outside [0, T) are no rows and no keys.
struct ColArgs {
  const float* lse;             // [B][Hq][T]
  const int32_t* path;          // [B][A] or null
  int A, R;                     // chunk key columns and packed rows
  float* dst;                   // [ranges of rows][BH][M + A]
  bf16_t *k_acc, *v_acc;        // path: [BH][A][D], the path's keys and values
  int ncopy;                    // blocks that copy them
};
constexpr int kQRows = 32;      // rows per step

template <int D, bool Q8, bool PATH, int NKB>
__global__ __launch_bounds__(kThreads) void column_pass(Args a, ColArgs p) {
  constexpr int KB = kWaves * NKB * 16, P = lds_pitch(D), NU = kQRows * D / 8 / kThreads;
  __shared__ __attribute__((aligned(16))) bf16_t Qs[2][kQRows * P];
  __shared__ float lam[2][kQRows];
  __shared__ int pos[2][kQRows];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const size_t bh = blockIdx.y;
  const int b = (int)bh / a.Hkv, h = (int)bh % a.Hkv;
  const int tc = (a.M + KB - 1) / KB, tn = (p.A + KB - 1) / KB;
  const int32_t* path = PATH ? p.path + (size_t)b * p.A : nullptr;
  // node of the chunk's key or row position i, -1 if it is none
  auto node_of = [&](int i) {
    if (!PATH) return i;
    const int n = path[i];
    return (unsigned)n < (unsigned)a.T ? n : -1;
  };
  if (PATH && (int)blockIdx.x >= tc + tn) {   // the path's rows, 16 bytes a thread
    const int e = ((int)blockIdx.x - tc - tn) * kThreads + tid, i = e / (D / 8), c = e % (D / 8);
    if (blockIdx.z || i >= p.A) return;
    const int n = node_of(i);
    u32x4 kv = {0u, 0u, 0u, 0u}, vv = kv;
    if (n >= 0) {
      kv = reinterpret_cast<const u32x4*>(a.kn + (bh * a.T + n) * (size_t)D)[c];
      vv = reinterpret_cast<const u32x4*>(a.vn + (bh * a.T + n) * (size_t)D)[c];
    }
    reinterpret_cast<u32x4*>(p.k_acc + (bh * p.A + i) * (size_t)D)[c] = kv;
    reinterpret_cast<u32x4*>(p.v_acc + (bh * p.A + i) * (size_t)D)[c] = vv;
    return;
  }
  const bool cache = (int)blockIdx.x < tc;
  const int j0 = (cache ? (int)blockIdx.x : (int)blockIdx.x - tc) * KB + wave * NKB * 16;
  const int nkeys = cache ? a.M : p.A;
  // this lane's operand rows: key j0 + 16 kb + l16, elements 64 x + 16 g4 .. +15
  // (an order of d that both operands share; 16 codes are one load)
  bf16x8 kf[NKB][D / 32];
  f32x4 cks[NKB], cs[NKB];
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb) {
    const int j = min(j0 + 16 * kb + l16, nkeys - 1);
    if (Q8 && cache) {
      const int8_t* src = (const int8_t*)a.kc + (bh * a.M + j) * (size_t)D + 16 * g4;
#pragma unroll
      for (int x = 0; x < D / 64; ++x) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(src + 64 * x);
        kf[kb][2 * x] = q8::codes_bf16(v[0], v[1]);
        kf[kb][2 * x + 1] = q8::codes_bf16(v[2], v[3]);
      }
    } else {
      const int n = cache ? j : max(node_of(j), 0);
      const bf16_t* src = (cache ? (const bf16_t*)a.kc + (bh * a.M + n) * (size_t)D
                                 : a.kn + (bh * a.T + n) * (size_t)D) + 16 * g4;
#pragma unroll
      for (int x = 0; x < D / 64; ++x) {
        kf[kb][2 * x] = *reinterpret_cast<const bf16x8*>(src + 64 * x);
        kf[kb][2 * x + 1] = *reinterpret_cast<const bf16x8*>(src + 64 * x + 8);
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int jr = min(j0 + 16 * kb + 4 * g4 + r, nkeys - 1);
      cks[kb][r] = Q8 && cache ? a.ks[bh * a.M + jr] * a.c : a.c;
      cs[kb][r] = 0.f;
    }
  }
  // rows of this block: its share of the steps, in a chunk tile from the first
  // row that sees the block's first key
  const int first = cache ? 0 : ((int)blockIdx.x - tc) * KB * a.G / kQRows;
  const int steps = (p.R + kQRows - 1) / kQRows;
  const int per = (steps + (int)gridDim.z - 1) / (int)gridDim.z;
  const int s1 = min(steps, ((int)blockIdx.z + 1) * per), s0 = max(first, (int)blockIdx.z * per);

  u32x4 qr[NU];
  float lr = 0.f;
  int ir = 0;
  auto load = [&](int s) {
#pragma unroll
    for (int e = 0; e < NU; ++e) {
      const int u = tid + e * kThreads, r = min(s * kQRows + u / (D / 8), p.R - 1);
      const int n = max(node_of(r / a.G), 0);
      qr[e] = *reinterpret_cast<const u32x4*>(
          a.q + ((size_t)(b * a.Hq + h * a.G + r % a.G) * a.T + n) * D + 8 * (u % (D / 8)));
    }
    if (tid < kQRows) {   // a row that is none: lambda +inf, weights 0
      const int r = s * kQRows + tid, n = r < p.R ? node_of(r / a.G) : -1;
      lr = n >= 0 ? p.lse[(size_t)(b * a.Hq + h * a.G + r % a.G) * a.T + n] * kLog2e : INFINITY;
      ir = r / a.G;
    }
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int e = 0; e < NU; ++e) {
      const int u = tid + e * kThreads;
      *reinterpret_cast<u32x4*>(&Qs[buf][u / (D / 8) * P + 8 * (u % (D / 8))]) = qr[e];
    }
    if (tid < kQRows) {
      lam[buf][tid] = lr;
      pos[buf][tid] = ir;
    }
  };
  auto step = [&](auto chunk, int buf) {
#pragma unroll
    for (int n = 0; n < kQRows / 16; ++n) {
      f32x4 s[NKB];
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb) s[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const bf16x8 qf = *reinterpret_cast<const bf16x8*>(
            &Qs[buf][(16 * n + l16) * P + 64 * (x >> 1) + 16 * g4 + 8 * (x & 1)]);
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) s[kb] = mma(kf[kb][x], qf, s[kb]);
      }
      const float la = lam[buf][16 * n + l16];
      const int i = decltype(chunk)::value ? pos[buf][16 * n + l16] : 0;
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float w = __builtin_amdgcn_exp2f(fmaf(s[kb][r], cks[kb][r], -la));
          if (decltype(chunk)::value && j0 + 16 * kb + 4 * g4 + r > i) w = 0.f;
          cs[kb][r] += w;
        }
    }
  };
  if (s0 < s1) {
    load(s0);
    store(0);
    if (s0 + 1 < s1) load(s0 + 1);
    __syncthreads();
    for (int s = s0; s < s1; ++s) {
      const int buf = (s - s0) & 1;
      if (s + 1 < s1) {
        store(buf ^ 1);
        if (s + 2 < s1) load(s + 2);
      }
      if (cache) step(IntConst<0>{}, buf);
      else step(IntConst<1>{}, buf);
      __syncthreads();
    }
  }
  const int nk = a.M + p.A;
  float* dst = p.dst + ((size_t)blockIdx.z * gridDim.y + bh) * nk + (cache ? 0 : a.M);
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float v = cs[kb][r];
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) v += __shfl_xor(v, o, 64);
      const int j = j0 + 16 * kb + 4 * g4 + r;
      if (l16 == 0 && j < nkeys) dst[j] = PATH && !cache && node_of(j) < 0 ? 0.f : v;
    }
}

// wsum = the row ranges' sums, in their order.
__global__ __launch_bounds__(kThreads) void column_reduce(const float* __restrict__ parts,
                                                          float* __restrict__ wsum, size_t n,
                                                          int nranges) {
  const size_t e = (size_t)blockIdx.x * kThreads + threadIdx.x;
  if (e >= n) return;
  float s = parts[e];
  for (int k = 1; k < nranges; ++k) s += parts[k * n + e];
  wsum[e] = s;
}

// ---------------------------------------------------------------------- tree
// bits[b][i] = the nodes on node i's way up, itself among them: a thread walks
// from its node, word by word. A parent that is not in [-1, i) counts as -1, so
// every walk goes down and ends. The parents are in LDS where they fit.
constexpr int kTreeLds = 8192;
template <bool LDS>
__global__ __launch_bounds__(kThreads) void tree_bits(const int32_t* __restrict__ parents, int T,
                                                      int W, uint32_t* __restrict__ bits) {
  __shared__ int32_t up[LDS ? kTreeLds : 1];
  const int32_t* src = parents + (size_t)blockIdx.y * T;
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (LDS) {
    const int n = min(T, (int)(blockIdx.x + 1) * kThreads);   // ancestors come before
    for (int e = threadIdx.x; e < n; e += kThreads) up[e] = src[e];
    __syncthreads();
  }
  if (i >= T) return;
  uint32_t* row = bits + ((size_t)blockIdx.y * T + i) * W;
  for (int w = (i >> 5) + 1; w < W; ++w) row[w] = 0u;
  int n = i, w = i >> 5;
  uint32_t acc = 0u;
  while (n >= 0) {
    while (w > n >> 5) {
      row[w--] = acc;
      acc = 0u;
    }
    acc |= 1u << (n & 31);
    const int p = LDS ? up[n] : src[n];
    n = p < n ? p : -1;
  }
  for (; w >= 0; --w) {
    row[w] = acc;
    acc = 0u;
  }
}

template <typename F>
hipError_t with_cache(int d, bool q8, F&& f) {
  if (d == 64) return q8 ? f(IntConst<64>{}, IntConst<1>{}) : f(IntConst<64>{}, IntConst<0>{});
  return q8 ? f(IntConst<128>{}, IntConst<1>{}) : f(IntConst<128>{}, IntConst<0>{});
}

Args make_args(const FlashShape& s, const FlashIn& in, const char* ws, const FlashPlan& p,
               float scale) {
  return Args{(const bf16_t*)in.q, in.kc, in.vc, in.ks, in.vs, (const bf16_t*)in.kn,
              (const bf16_t*)in.vn, reinterpret_cast<const uint32_t*>(ws + p.off_bits), s.Hq, s.Hkv,
              s.G(), s.T, s.M, s.G() * s.T, (s.T + 31) / 32, scale * kLog2e};
}

}  // namespace

// Rows per block: 128 (32 per wave: every K and V operand read from LDS feeds two
// products) where there are more than 64. Key ranges: enough blocks for two per
// CU, at least two tiles each, at most kMaxFlashSplit (each leaves a float32
// partial of its rows). Row ranges of the column sums: likewise, at least four
// steps each.
FlashPlan flash_plan(const FlashShape& s, bool tree) {
  FlashPlan p{};
  const long long BH = s.BH(), R = (long long)s.G() * s.T, cus = device_cus();
  p.rows = s.f32 || R <= 64 ? 64 : 128;
  const int bn = s.f32 ? 32 : BN;
  const long long nb = (R + p.rows - 1) / p.rows * BH;
  const long long ntiles = (s.M + bn - 1) / bn + (s.T + bn - 1) / bn;
  long long ns = (2 * cus + nb - 1) / nb;
  if (ns > ntiles / 2) ns = ntiles / 2;
  if (ns > kMaxFlashSplit) ns = kMaxFlashSplit;
  p.nsplit = ns < 1 ? 1 : (int)ns;
  p.nranges = column_ranges(s, s.T);
  size_t off = 0;
  p.off_stats = off;
  if (p.nsplit > 1) off = align256_size(off + (size_t)p.nsplit * BH * R * sizeof(float2));
  p.off_opart = off;
  if (p.nsplit > 1) off = align256_size(off + (size_t)p.nsplit * BH * R * s.d * sizeof(float));
  p.off_bits = off;
  if (tree) off = align256_size(off + (size_t)s.B * s.T * ((s.T + 31) / 32) * 4);
  // the tree's column sums are a call of their own, of any path
  p.off_parts = tree ? 0 : off;
  const int nr = tree ? kMaxColumnRanges : p.nranges;
  const size_t parts = nr > 1 ? align256_size((size_t)nr * BH * (s.M + s.T) * sizeof(float)) : 0;
  if (p.off_parts + parts > off) off = p.off_parts + parts;
  p.bytes = off;
  return p;
}

int column_ranges(const FlashShape& s, int ncol) {
  const int kb = s.f32 ? kColumnKeysF32 : kColumnKeys;
  const long long nb = (long long)((s.M + kb - 1) / kb + (ncol + kb - 1) / kb) * s.BH();
  const long long steps = ((long long)s.G() * ncol + kQRows - 1) / kQRows;
  long long n = (2ll * device_cus() + nb - 1) / nb;
  if (n > steps / 4) n = steps / 4;
  if (n > kMaxColumnRanges) n = kMaxColumnRanges;
  return n < 1 ? 1 : (int)n;
}

hipError_t launch_tree_bits(const FlashShape& s, const FlashPlan& p, const int32_t* parents,
                            char* ws, hipStream_t st) {
  uint32_t* bits = reinterpret_cast<uint32_t*>(ws + p.off_bits);
  const int W = (s.T + 31) / 32;
  const dim3 grid((s.T + kThreads - 1) / kThreads, s.B);
  return s.T <= kTreeLds
             ? launch_kernel(K_TREE_BITS, tree_bits<true>, grid, dim3(kThreads), st, parents, s.T, W, bits)
             : launch_kernel(K_TREE_BITS, tree_bits<false>, grid, dim3(kThreads), st, parents, s.T, W, bits);
}

hipError_t launch_flash_combine(const FlashShape& s, const FlashPlan& p, void* out, float* lse,
                                const char* ws, hipStream_t st) {
  const size_t rows = (size_t)s.BH() * s.G() * s.T;
  auto go = [&](auto D, auto e) {
    typedef decltype(e) E;
    constexpr int per = kThreads / (decltype(D)::value / 4);
    return launch_kernel(K_FLASH_COMBINE, flash_combine<decltype(D)::value, E>,
                         dim3((unsigned)((rows + per - 1) / per)), dim3(kThreads), st,
                         reinterpret_cast<const float2*>(ws + p.off_stats),
                         reinterpret_cast<const float*>(ws + p.off_opart), (E*)out, lse, s.BH(),
                         s.Hq, s.Hkv, s.G(), s.T, s.G() * s.T, p.nsplit);
  };
  if (s.f32) return s.d == 64 ? go(IntConst<64>{}, float{}) : go(IntConst<128>{}, float{});
  return s.d == 64 ? go(IntConst<64>{}, bf16_t{}) : go(IntConst<128>{}, bf16_t{});
}

hipError_t launch_column_reduce(const float* parts, float* wsum, size_t n, int nranges,
                                hipStream_t st) {
  return launch_kernel(K_COLUMN_REDUCE, column_reduce,
                       dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), st, parts,
                       wsum, n, nranges);
}

hipError_t launch_flash(const FlashShape& s, const FlashPlan& p, const FlashIn& in, bool tree,
                        void* out, float* lse, char* ws, float scale, hipStream_t st) {
  const Args a = make_args(s, in, ws, p, scale);
  const int nrt = (a.R + p.rows - 1) / p.rows;
  const dim3 grid(nrt * p.nsplit, s.BH());
  float2* stats = reinterpret_cast<float2*>(ws + p.off_stats);
  float* opart = reinterpret_cast<float*>(ws + p.off_opart);
  const hipError_t e = with_cache(s.d, in.q8, [&](auto D, auto q) {
    constexpr int kD = decltype(D)::value;
    constexpr bool kQ = decltype(q)::value;
    auto go = [&](auto kern) {
      return launch_kernel(K_FLASH, kern, grid, dim3(kThreads), st, a, p.nsplit, (bf16_t*)out, lse,
                           stats, opart);
    };
    if (tree)
      return p.rows == 128 ? go(flash_pass<kD, kQ, true, 2>) : go(flash_pass<kD, kQ, true, 1>);
    if constexpr (kQ)
      return p.rows == 128 ? go(flash_pass<kD, true, false, 2>) : go(flash_pass<kD, true, false, 1>);
    return hipErrorInvalidValue;   // the chunk over a bf16 cache has its own kernels
  });
  if (e != hipSuccess || p.nsplit == 1) return e;
  return launch_flash_combine(s, p, out, lse, ws, st);
}

hipError_t launch_columns(const FlashShape& s, const FlashPlan& p, const FlashIn& in,
                          const float* lse, const int32_t* path, int A, void* k_acc, void* v_acc,
                          float* wsum, char* ws, float scale, hipStream_t st) {
  const Args a = make_args(s, in, ws, p, scale);
  float* parts = reinterpret_cast<float*>(ws + p.off_parts);
  const int ncol = path ? A : s.T;
  const int kb = kColumnKeys, tiles = (s.M + kb - 1) / kb + (ncol + kb - 1) / kb;
  const int ncopy = path ? (A * (s.d / 8) + kThreads - 1) / kThreads : 0;
  const ColArgs c{lse, path, ncol, s.G() * ncol, p.nranges > 1 ? parts : wsum, (bf16_t*)k_acc,
                  (bf16_t*)v_acc, ncopy};
  const dim3 grid(tiles + ncopy, s.BH(), p.nranges);
  const hipError_t e = with_cache(s.d, in.q8, [&](auto D, auto q) {
    constexpr int kD = decltype(D)::value;
    constexpr bool kQ = decltype(q)::value;
    constexpr int kN = kColumnKeys / (16 * kWaves);
    auto go = [&](auto kern) {
      return launch_kernel(K_COLUMNS, kern, grid, dim3(kThreads), st, a, c);
    };
    if (path) return go(column_pass<kD, kQ, true, kN>);
    if constexpr (kQ) return go(column_pass<kD, true, false, kN>);
    return hipErrorInvalidValue;
  });
  if (e != hipSuccess || p.nranges == 1) return e;
  return launch_column_reduce(parts, wsum, (size_t)s.BH() * (s.M + ncol), p.nranges, st);
}

}  // namespace h2o
