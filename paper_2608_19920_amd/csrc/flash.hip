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
// 8-bit rows become codes in bf16 (K) and fp16 (V) on their way into LDS, exactly; the
// key's scale multiplies the scores, the value's scale the probabilities. These are
// rounded to fp16 for their product with codes, against a reference that goes by the
// row's weights (q8.h), and with bf16 values split into two bf16 terms, so that next to
// the rounding of the output theirs is small, whatever the values' and the scores' sizes
// (1.7e-3 normwise; with probabilities in bf16 2.3e-3, and 2.8e-3 where there are few
// rows). B1 Hq32 Hkv8 d128 M8192 T1024: 194 us; with probabilities in bf16 172, with a
// reference by the scores and the largest scale, which loses rows beside a larger one that
// nobody attends, 185, with two bf16 terms for codes as well 227.
#include "internal.h"
#include "mfma_ops.h"
#include "q8.h"

#include <cmath>

namespace h2o {
namespace {

using namespace mfma;

constexpr int kThreads = 256;
constexpr int kXcds = 8;
constexpr int kFewSplits = 4;   // key ranges that one thread merges alone
// A lambda over register arrays: a call that is not inlined would put them in memory.
#define H2O_INLINE __attribute__((always_inline))

__host__ __device__ constexpr int lds_pitch(int D) { return D + 16; }   // bf16 per LDS row

// Tiles of a pass: whole ones of the cache, its last, and the chunk's.
enum { kCache, kCacheEnd, kChunk };

struct Args {
  const bf16_t* q;
  const void *kc, *vc;          // [BH][M][D], bf16 or codes
  const float *ks, *vs;         // [BH][M], 8-bit cache
  const bf16_t *kn, *vn;        // [BH][T][D]
  const int32_t* parents;       // tree: [B][T]
  const uint32_t* bits;         // tree of more than 64 nodes: [B][T][W] ancestor bits, a
                                // node's own among them
  int Hq, Hkv, G, T, M, R, W;
  float c;                      // scale * log2(e)
};

// Blocks reach the 8 XCDs round-robin: the row tiles of one (head, key range),
// which read the same keys, go to one XCD and share its L2, last rows first.
struct BlockId { int rt, sp, bh; };
__device__ __forceinline__ void xcd_group(int lin, int per, int ngroups, int& grp, int& i) {
  grp = lin / per;
  i = lin % per;
  if (ngroups % kXcds == 0) {
    const int n = lin / kXcds;
    grp = (n / per) * kXcds + lin % kXcds;
    i = n % per;
  }
}
__device__ __forceinline__ BlockId block_id(int nsplit) {
  const int nrt = gridDim.x / nsplit;
  int grp, i;
  xcd_group(blockIdx.x + blockIdx.y * gridDim.x, nrt, nsplit * gridDim.y, grp, i);
  return BlockId{nrt - 1 - i, grp % nsplit, grp / nsplit};
}

// ------------------------------------------------------------------- staging
// A tile's rows in registers: 16-byte units, 16 codes or 8 bf16 each, unit u of
// thread t being t + u * NT.
template <int D, int NT, int BN>
struct Regs {
  static constexpr int N16 = (BN * D / 8 + NT - 1) / NT;   // (8 waves, D = 64: a part of the
  static constexpr int N8 = (BN * D / 16 + NT - 1) / NT;   // threads; the others load a row again)
  u32x4 k[N16], v[N16];
  float s;                      // thread t < BN: scale of key t; BN <= t < 2 BN: of value t - BN
};

template <int D, int NT, int BN>
__device__ __forceinline__ void load_rows16(u32x4* r, const void* base, int n) {
  const char* p = reinterpret_cast<const char*>(base);
#pragma unroll
  for (int e = 0; e < Regs<D, NT, BN>::N16; ++e) {
    const int u = threadIdx.x + e * NT, row = min(u / (D / 8), n - 1);
    r[e] = *reinterpret_cast<const u32x4*>(p + (uint32_t)(row * D + 8 * (u % (D / 8))) * 2u);
  }
}
template <int D, int NT, int BN>
__device__ __forceinline__ void load_rows8(u32x4* r, const void* base, int n) {
  const char* p = reinterpret_cast<const char*>(base);
#pragma unroll
  for (int e = 0; e < Regs<D, NT, BN>::N8; ++e) {
    const int u = threadIdx.x + e * NT, row = min(u / (D / 16), n - 1);
    r[e] = *reinterpret_cast<const u32x4*>(p + (uint32_t)(row * D + 16 * (u % (D / 16))));
  }
}
template <int D, int NT, int BN>
__device__ __forceinline__ void store_rows16(bf16_t* lds, const u32x4* r) {
#pragma unroll
  for (int e = 0; e < Regs<D, NT, BN>::N16; ++e) {
    const int u = threadIdx.x + e * NT;
    if (BN * D / 8 < NT && u >= BN * D / 8) return;
    *reinterpret_cast<u32x4*>(lds + u / (D / 8) * lds_pitch(D) + 8 * (u % (D / 8))) = r[e];
  }
}
template <int D, int NT, int BN, bool F16>
__device__ __forceinline__ void store_rows8(bf16_t* lds, const u32x4* r) {
#pragma unroll
  for (int e = 0; e < Regs<D, NT, BN>::N8; ++e) {
    const int u = threadIdx.x + e * NT;
    if (BN * D / 16 < NT && u >= BN * D / 16) return;
    bf16_t* dst = lds + u / (D / 16) * lds_pitch(D) + 16 * (u % (D / 16));
    if constexpr (F16) {
      reinterpret_cast<f16x8*>(dst)[0] = q8::codes_f16(r[e][0], r[e][1]);
      reinterpret_cast<f16x8*>(dst)[1] = q8::codes_f16(r[e][2], r[e][3]);
    } else {
      reinterpret_cast<bf16x8*>(dst)[0] = q8::codes_bf16(r[e][0], r[e][1]);
      reinterpret_cast<bf16x8*>(dst)[1] = q8::codes_bf16(r[e][2], r[e][3]);
    }
  }
}

// Rows past the tile's end re-read its last row (in bounds; masked later).
// WHOLE: the caller knows that it is a whole cache tile (no branch).
template <int D, bool Q8, int NT, int BN, bool WHOLE = false>
__device__ __forceinline__ void load_tile(Regs<D, NT, BN>& g, const Args& a, size_t bh, int t,
                                          int tc) {
  if (WHOLE || t < tc) {
    const int j0 = t * BN, n = WHOLE ? BN : min(BN, a.M - j0);
    const size_t row = bh * (size_t)a.M + j0;
    if constexpr (Q8) {
      load_rows8<D, NT, BN>(g.k, (const int8_t*)a.kc + row * D, n);
      load_rows8<D, NT, BN>(g.v, (const int8_t*)a.vc + row * D, n);
      const int r = threadIdx.x % BN;
      if (threadIdx.x < 2 * BN) g.s = (threadIdx.x < BN ? a.ks : a.vs)[row + min(r, n - 1)];
    } else {
      load_rows16<D, NT, BN>(g.k, (const bf16_t*)a.kc + row * D, n);
      load_rows16<D, NT, BN>(g.v, (const bf16_t*)a.vc + row * D, n);
    }
  } else {
    const int j0 = (t - tc) * BN, n = min(BN, a.T - j0);
    const size_t row = bh * (size_t)a.T + j0;
    load_rows16<D, NT, BN>(g.k, a.kn + row * D, n);
    load_rows16<D, NT, BN>(g.v, a.vn + row * D, n);
  }
}
template <int D, bool Q8, int NT, int BN, bool WHOLE = false>
__device__ __forceinline__ void store_tile(bf16_t* Ks, bf16_t* Vs, float* sc,
                                           const Regs<D, NT, BN>& g, const Args& a, int t, int tc) {
  if (Q8 && (WHOLE || t < tc)) {
    store_rows8<D, NT, BN, false>(Ks, g.k);
    store_rows8<D, NT, BN, true>(Vs, g.v);
    if (threadIdx.x < 2 * BN) sc[threadIdx.x] = threadIdx.x < BN ? g.s * a.c : g.s;
  } else {
    store_rows16<D, NT, BN>(Ks, g.k);
    store_rows16<D, NT, BN>(Vs, g.v);
  }
}

// --------------------------------------------------------------------- flash
// Each of NW waves owns 16 NQB consecutive packed rows r = i*G + g. A row's
// probabilities are exp2(x - mu) with x its scores in log2 units and mu a
// reference common to the 4 lanes that hold the row: the maximum of the first
// tile the row sees, raised when a score exceeds it by more than 15 (a
// wave-uniform and rare branch), so terms stay below 2^15, and 2^20 of them times values
// of 2^90 inside float32 (a step of 64 measured the same); over an 8-bit cache's tiles as
// q8.h says.
//
// Tiles have BN keys, 32, or 64 at d = 64 with 128 rows or more, where the registers
// allow them: half the barriers, and more of a wave's own products and exponentials to
// overlap (B1 Hq32 Hkv8 d64 M8192 T1024 128 -> 120 us; at d = 128 they spill, with 64
// rows B4 Hkv8 d64 M8192, a tree of 16, 17.5 -> 23.3).
//
// Tile t + 2 is on its way from memory to registers and tile t + 1 from registers to
// the other LDS buffer while tile t is used; one barrier a tile. (Multiplying the
// scores of tile t + 1 during the exponentials of tile t, a third buffer, requests
// another tile ahead, or an imposed order of products and vector operations, measured
// no faster: B1 Hq32 Hkv8 d128 M8192 T1024 216 us in every form, 4 waves a block.)
//
// Bound by the two pipes of a SIMD together: 32 products (16 cycles each) and some 200
// vector operations, 16 of them exponentials (8 cycles), per 32 keys and 32 rows; 64
// of them (4 waves) or 32 (8 waves) turn codes into bf16 and fp16. The kinds of tiles
// are separate code: one body for the cache's last tile and the chunk's took 254
// registers instead of 212 and 13 % more time.
template <int D, bool Q8, bool TREE, int NQB, int NW, int BN>
__global__ __launch_bounds__(NW * 64, 2) void flash_pass(Args a, int nsplit,
                                                         bf16_t* __restrict__ out,
                                                         float* __restrict__ lse,
                                                         float2* __restrict__ stats,
                                                         float* __restrict__ opart) {
  constexpr int NT = NW * 64, ROWS = NW * NQB * 16, P = lds_pitch(D), NK = BN / 16;
  constexpr float kRaise = 15.f;
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

  bf16x8 qf[NQB][D / 32];
  int qi[NQB];
  float mu[NQB], thr[NQB], l[NQB];
  q8::ValueRef vr;
  float aim = 0.f;
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
    mu[n] = 0.f;
    thr[n] = -INFINITY;               // no tile seen yet
    l[n] = 0.f;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) oacc[db][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  uint64_t own[NQB];   // the ancestors of a tree of at most 64 nodes
  if (TREE && a.T <= kWaveTree) {
    const uint64_t mine = wave_ancestors(a.parents + (size_t)b * a.T, a.T, lane);
#pragma unroll
    for (int n = 0; n < NQB; ++n) own[n] = __shfl(mine, qi[n], 64);
  }

  // Tile t, in LDS at K, V, scl: scores, probabilities, O += P V; then the registers g,
  // with tile t + 1, go to the other buffer, and tile t + 2 is requested into them.
  auto tile = [&](auto kind, auto whole, int t, const bf16_t* K, const bf16_t* V,
                  const float* scl, Regs<D, NT, BN>& g, int t1st, int t2nd, bf16_t* K2, bf16_t* V2,
                  float* scl2) H2O_INLINE {
    constexpr bool CHUNK = decltype(kind)::value == kChunk, MASK = decltype(kind)::value != kCache;
    constexpr bool WHOLE = decltype(whole)::value, CODED = Q8 && !CHUNK;
    f32x4 s[NK][NQB];
#pragma unroll
    for (int kb = 0; kb < NK; ++kb) {
#pragma unroll
      for (int n = 0; n < NQB; ++n) s[kb][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const bf16x8 kf = row_operand(K, P, 16 * kb + l16, 32 * x, lane);
#pragma unroll
        for (int n = 0; n < NQB; ++n) s[kb][n] = mma(kf, qf[n][x], s[kb][n]);
      }
    }
    uint32_t seen[NQB][BN / 32];
    if (TREE && CHUNK)
#pragma unroll
      for (int n = 0; n < NQB; ++n)
#pragma unroll
        for (int w = 0; w < BN / 32; ++w) {
          const int word = (t - tc) * (BN / 32) + w;
          seen[n][w] = word >= a.W ? 0u
                       : a.T <= kWaveTree ? (uint32_t)(own[n] >> (word ? 32 : 0))
                                          : a.bits[((size_t)b * a.T + qi[n]) * a.W + word];
        }
    f32x4 cks[NK], cvs[NK];
    if (CODED)
#pragma unroll
      for (int kb = 0; kb < NK; ++kb) {
        cks[kb] = *reinterpret_cast<const f32x4*>(scl + 16 * kb + 4 * g4);
        cvs[kb] = *reinterpret_cast<const f32x4*>(scl + BN + 16 * kb + 4 * g4);
      }
    auto shifted = [&](int n, float ref, float (&x)[4 * NK]) H2O_INLINE {
#pragma unroll
      for (int kb = 0; kb < NK; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v = fmaf(s[kb][n][r], CODED ? cks[kb][r] : a.c, -ref);
          if (MASK) {
            const int j = 16 * kb + 4 * g4 + r;
            const bool hid = !CHUNK ? t * BN + j >= a.M
                             : TREE ? !((seen[n][kb >> 1] >> (j & 31)) & 1u)
                                    : (t - tc) * BN + j > qi[n];
            if (hid) v = -INFINITY;
          }
          x[4 * kb + r] = v;
        }
    };
    float x[NQB][4 * NK], mx[NQB], vmx = 0.f, lv = 0.f;
    bool up = false;
    if (CODED) {
#pragma unroll
      for (int kb = 0; kb < NK; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) vmx = fmaxf(vmx, fabsf(cvs[kb][r]));
      up = vmx > vr.limit;
      lv = q8::log2_scale(vmx * vr.inv);
    }
#pragma unroll
    for (int n = 0; n < NQB; ++n) {
      shifted(n, mu[n], x[n]);
      mx[n] = x[n][0];
#pragma unroll
      for (int e = 1; e < 4 * NK; ++e) mx[n] = fmaxf(mx[n], x[n][e]);
      up |= (CODED ? mx[n] + lv : mx[n]) > thr[n];
    }
    if (__builtin_amdgcn_ballot_w64(up)) {
      float fv = 1.f;
      if (CODED && __builtin_amdgcn_ballot_w64(vmx > vr.limit)) fv = vr.raise(q8::row_max(vmx));
#pragma unroll
      for (int n = 0; n < NQB; ++n) {
        float f;
        if constexpr (CODED) {
          float y = -INFINITY, yc = -INFINITY;
#pragma unroll
          for (int kb = 0; kb < NK; ++kb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float rel = fabsf(cvs[kb][r]) * vr.inv;
              y = fmaxf(y, x[n][4 * kb + r] + __log2f(rel));
              yc = fmaxf(yc, x[n][4 * kb + r] + q8::log2_scale(rel));
            }
          f = q8::move(mu[n], thr[n], l[n], fv, y, yc, aim);
        } else {
          const float y = q8::row_max(mx[n]);
          const bool raise = y > thr[n];
          f = !raise ? 1.f : thr[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(-y);
          mu[n] = raise ? mu[n] + y : mu[n];
          thr[n] = raise ? kRaise : thr[n];
          l[n] *= f;
        }
#pragma unroll
        for (int db = 0; db < D / 16; ++db) oacc[db][n] *= f;
        shifted(n, mu[n], x[n]);
      }
    }
    if constexpr (CODED) {
#pragma unroll
      for (int kb = 0; kb < NK; ++kb) cvs[kb] *= vr.inv;
#pragma unroll
      for (int kk = 0; kk < BN / 32; ++kk) {
        f16x8 pb[NQB];
#pragma unroll
        for (int n = 0; n < NQB; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float p = __builtin_amdgcn_exp2f(x[n][8 * kk + e]);
            l[n] += p;
            pb[n][e] = (_Float16)(p * cvs[2 * kk + (e >> 2)][e & 3]);
          }
#pragma unroll
        for (int db = 0; db < D / 16; ++db) {
          const f16x8 vf = __builtin_bit_cast(f16x8, tr_operand(V + 32 * kk * P, P, db, lane));
#pragma unroll
          for (int n = 0; n < NQB; ++n) oacc[db][n] = mma(vf, pb[n], oacc[db][n]);
        }
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < BN / 32; ++kk) {
        bf16x8 pb[NQB], rest[NQB];
#pragma unroll
        for (int n = 0; n < NQB; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float p = __builtin_amdgcn_exp2f(x[n][8 * kk + e]);
            l[n] += p;
            const float w = Q8 ? p * vr.inv : p;
            pb[n][e] = (__bf16)w;
            rest[n][e] = (__bf16)(w - (float)pb[n][e]);
          }
#pragma unroll
        for (int db = 0; db < D / 16; ++db) {
          const bf16x8 vf = tr_operand(V + 32 * kk * P, P, db, lane);
#pragma unroll
          for (int n = 0; n < NQB; ++n)
            oacc[db][n] = mma(vf, rest[n], mma(vf, pb[n], oacc[db][n]));
        }
      }
    }
    store_tile<D, Q8, NT, BN, WHOLE>(K2, V2, scl2, g, a, t1st, tc);
    load_tile<D, Q8, NT, BN, WHOLE>(g, a, bh, t2nd, tc);
    __syncthreads();
  };

  if (t0 < t1) {
    Regs<D, NT, BN> g;
    const int last = t1 - 1;
    load_tile<D, Q8, NT, BN>(g, a, bh, t0, tc);
    store_tile<D, Q8, NT, BN>(Ks[0], Vs[0], sc[0], g, a, t0, tc);
    load_tile<D, Q8, NT, BN>(g, a, bh, min(t0 + 1, last), tc);
    __syncthreads();
    auto run = [&](auto kind, auto whole, int ta, int tb) H2O_INLINE {
      for (int t = ta; t < tb; ++t) {
        const int v = (t - t0) & 1;
        tile(kind, whole, t, Ks[v], Vs[v], sc[v], g, min(t + 1, last), min(t + 2, last),
             Ks[v ^ 1], Vs[v ^ 1], sc[v ^ 1]);   // (past the last tile: it again, not used)
      }
    };
    // turns whose tiles t + 1 and t + 2 are whole cache tiles; the other whole ones; the
    // one that ends the cache; the chunk
    aim = q8::aim_of((t1 - t0) * BN);
    const int tm = a.M / BN, te = max(t0, min(t1, tm)), tw = max(t0, min(te, min(t1, tm) - 2));
    const int tk = max(t0, min(t1, tc));
    run(IntConst<kCache>{}, IntConst<1>{}, t0, tw);
    run(IntConst<kCache>{}, IntConst<0>{}, tw, te);
    run(IntConst<kCacheEnd>{}, IntConst<0>{}, te, tk);
    if (Q8)
#pragma unroll
      for (int n = 0; n < NQB; ++n)
        thr[n] = q8::row_max(l[n]) == 0.f ? -INFINITY : kRaise;   // cache keys seen or none
    // the chunk's values are of any size, whatever the cache's: probabilities relative to
    // a far smaller reference would leave float32
    if (Q8 && tk < t1 && vr.limit < 1.f) {
      const float f = vr.raise(0.03125f);   // to 1
#pragma unroll
      for (int n = 0; n < NQB; ++n)
#pragma unroll
        for (int db = 0; db < D / 16; ++db) oacc[db][n] *= f;
    }
    run(IntConst<kChunk>{}, IntConst<0>{}, tk, t1);
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
      if (nsplit == 1) lse[orow] = (mu[n] + __log2f(L)) * kLn2;
      else stats[prow] = make_float2(L == 0.f ? -INFINITY : mu[n], L);
    }
    const float inv = vr.ref() / L;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) {
      const f32x4 o = oacc[db][n];
      if (nsplit == 1) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (__bf16)(o[e] * inv);
        *reinterpret_cast<bf16x4*>(out + orow * D + 16 * db + 4 * g4) = w;
      } else {
        *reinterpret_cast<f32x4*>(opart + prow * D + 16 * db + 4 * g4) = Q8 ? o * vr.ref() : o;
      }
    }
  }
}

// The ranges' partials of a packed row, in a fixed order: D / 4 threads with 4
// columns each and, with SG > 1, SG such groups that take every SG-th range and
// meet in LDS. Few ranges come with many rows (SG = 1); many ranges with few,
// where what counts is that a thread's loads are all in flight at once.
template <int D, typename E, int SG>
__global__ __launch_bounds__(kThreads) void flash_combine(const float2* __restrict__ stats,
                                                          const float* __restrict__ opart,
                                                          E* __restrict__ out,
                                                          float* __restrict__ lse, int BH, int Hq,
                                                          int Hkv, int G, int T, int R,
                                                          int nsplit) {
  constexpr int TPR = D / 4, RPB = kThreads / (TPR * SG);   // rows per block
  constexpr int N = SG > 1 ? kMaxFlashSplit / SG : kFewSplits;
  static_assert(RPB >= 1 && N * SG >= (SG > 1 ? kMaxFlashSplit : 1), "ranges per thread");
  __shared__ __attribute__((aligned(16))) f32x4 os[RPB][SG][SG > 1 ? TPR : 1];
  __shared__ float ls[RPB][SG];
  const int t = threadIdx.x % TPR, sg = threadIdx.x / TPR % SG, rb = threadIdx.x / (TPR * SG);
  const size_t rows = (size_t)BH * R, at = (size_t)blockIdx.x * RPB + rb;
  const size_t row = at < rows ? at : rows - 1;   // (a spare row of threads repeats the last)
  const int c4 = 4 * t, bh = (int)(row / R), r = (int)(row % R);
  float2 st[N];
  f32x4 v[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int s = k * SG + sg;
    st[k] = make_float2(-INFINITY, 0.f);
    v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (s < nsplit) {
      st[k] = stats[s * rows + row];
      v[k] = *reinterpret_cast<const f32x4*>(opart + (s * rows + row) * D + c4);
    }
  }
  float mx = -INFINITY;
#pragma unroll
  for (int k = 0; k < N; ++k) mx = fmaxf(mx, st[k].x);
  if constexpr (SG > 1) {
    __shared__ float ms[RPB][SG];
    if (t == 0) ms[rb][sg] = mx;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SG; ++k) mx = fmaxf(mx, ms[rb][k]);
  }
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float L = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float w = st[k].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[k].x - mx);
    L = fmaf(w, st[k].y, L);
    o += w * v[k];
  }
  if constexpr (SG > 1) {
    os[rb][sg][t] = o;
    if (t == 0) ls[rb][sg] = L;
    __syncthreads();
    if (sg) return;
#pragma unroll
    for (int k = 1; k < SG; ++k) {
      o += os[rb][k][t];
      L += ls[rb][k];
    }
  }
  if (at >= rows) return;
  const int b = bh / Hkv, h = bh % Hkv;
  const size_t orow = (size_t)(b * Hq + h * G + r % G) * T + r / G;
  if (c4 == 0) lse[orow] = (mx + __log2f(L)) * kLn2;
  const float inv = 1.f / L;
  if constexpr (sizeof(E) == 4) {
    *reinterpret_cast<f32x4*>(out + orow * D + c4) = o * inv;
  } else {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (__bf16)(o[e] * inv);
    *reinterpret_cast<bf16x4*>(out + orow * D + c4) = w;
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
  ScoreAcc acc;                 // (one range of rows)
};
constexpr int kQRows = 64;      // rows per step
constexpr int kFewRows = 64;    // rows that a wave keeps (column_few)

// Node of the path's entry (or, path null, chunk position) i, -1 if it is none.
__device__ __forceinline__ int path_node(const int32_t* path, int i, int T) {
  if (!path) return i;
  const int n = path[i];
  return (unsigned)n < (unsigned)T ? n : -1;
}
// Unit e of the path's keys and values, 16 bytes.
template <int D>
__device__ __forceinline__ void copy_path(const Args& a, const ColArgs& p, size_t bh,
                                          const int32_t* path, int e) {
  const int i = e / (D / 8), c = e % (D / 8);
  if (i >= p.A) return;
  const int n = path_node(path, i, a.T);
  u32x4 kv = {0u, 0u, 0u, 0u}, vv = kv;
  if (n >= 0) {
    kv = reinterpret_cast<const u32x4*>(a.kn + (bh * a.T + n) * (size_t)D)[c];
    vv = reinterpret_cast<const u32x4*>(a.vn + (bh * a.T + n) * (size_t)D)[c];
  }
  reinterpret_cast<u32x4*>(p.k_acc + (bh * p.A + i) * (size_t)D)[c] = kv;
  reinterpret_cast<u32x4*>(p.v_acc + (bh * p.A + i) * (size_t)D)[c] = vv;
}

template <int D, bool Q8, bool PATH, int NKB, int NW>
__global__ __launch_bounds__(NW * 64, NW == 8 ? 4 : 1) void column_pass(Args a, ColArgs p) {
  constexpr int NT = NW * 64, KB = NW * NKB * 16, P = lds_pitch(D), NU = kQRows * D / 8 / NT;
  __shared__ __attribute__((aligned(16))) bf16_t Qs[2][kQRows * P];
  // log2(e) lse in one float32: at an lse of 20 a row's weights are off by 2^-20 together,
  // which a sum of 64 rows and more averages (row_weight's factor in every term: 112 -> 130 us)
  __shared__ float lam[2][kQRows];
  __shared__ int pos[2][kQRows];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // a head's blocks, which read the same rows, on one XCD
  int bhi, bx;
  xcd_group(blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z), gridDim.x * gridDim.z,
            gridDim.y, bhi, bx);
  const int bz = bx / gridDim.x;
  bx %= gridDim.x;
  const size_t bh = bhi;
  const int b = bhi / a.Hkv, h = bhi % a.Hkv;
  const int tc = (a.M + KB - 1) / KB, tn = (p.A + KB - 1) / KB;
  const int32_t* path = PATH ? p.path + (size_t)b * p.A : nullptr;
  auto node_of = [&](int i) { return path_node(path, i, a.T); };
  if (PATH && bx >= tc + tn) {   // the path's rows
    if (!bz) copy_path<D>(a, p, bh, path, (bx - tc - tn) * NT + tid);
    return;
  }
  const bool cache = bx < tc;
  const int j0 = (cache ? bx : bx - tc) * KB + wave * NKB * 16;
  const int nkeys = cache ? a.M : p.A;
  // this lane's operand rows: key j0 + 16 kb + l16, elements 32 x + 8 g4 .. +7. All
  // that the block reads first is requested before any of it is used.
  u32x4 kr[NKB][D / 32];
  f32x4 cks[NKB], cs[NKB];
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb) {
    const int j = min(j0 + 16 * kb + l16, nkeys - 1);
    if (Q8 && cache) {
      const int8_t* src = (const int8_t*)a.kc + (bh * a.M + j) * (size_t)D + 8 * g4;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const uint2 v = *reinterpret_cast<const uint2*>(src + 32 * x);
        kr[kb][x] = u32x4{v.x, v.y, 0u, 0u};
      }
    } else {
      const int n = cache ? j : max(node_of(j), 0);
      const bf16_t* src = (cache ? (const bf16_t*)a.kc + (bh * a.M + n) * (size_t)D
                                 : a.kn + (bh * a.T + n) * (size_t)D) + 8 * g4;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) kr[kb][x] = *reinterpret_cast<const u32x4*>(src + 32 * x);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int jr = min(j0 + 16 * kb + 4 * g4 + r, nkeys - 1);
      cks[kb][r] = Q8 && cache ? a.ks[bh * a.M + jr] : 1.f;
      cs[kb][r] = 0.f;
    }
  }
  // rows of this block: its share of the steps, in a chunk tile from the first
  // row that sees the block's first key
  const int first = cache ? 0 : (bx - tc) * KB * a.G / kQRows;
  const int steps = (p.R + kQRows - 1) / kQRows;
  const int per = (steps + (int)gridDim.z - 1) / (int)gridDim.z;
  const int s1 = min(steps, (bz + 1) * per), s0 = max(first, bz * per);

  // A thread's NU units of a step lie NT / (D / 8) rows apart. Its rows, as (position
  // i, head g of the group), advance by kQRows a step without a division; past the
  // last row they stay at it (the weights of such rows are 0).
  constexpr int RU = NT / (D / 8);
  u32x4 qr[NU];
  float lr = 0.f;
  int ir = 0, ri[NU], rg[NU], li, lg;
  const int part = 8 * (tid % (D / 8)), di = kQRows / a.G, dg = kQRows % a.G;
#pragma unroll
  for (int e = 0; e < NU; ++e) {
    const int r = s0 * kQRows + tid / (D / 8) + e * RU;
    ri[e] = r / a.G;
    rg[e] = r % a.G;
  }
  li = (s0 * kQRows + tid) / a.G;
  lg = (s0 * kQRows + tid) % a.G;
  const bf16_t* qh = a.q + (size_t)(b * a.Hq + h * a.G) * a.T * D + part;
  const float* lh = p.lse + (size_t)(b * a.Hq + h * a.G) * a.T;
  auto advance = [&](int& i, int& g) H2O_INLINE {
    i += di;
    g += dg;
    if (g >= a.G) { g -= a.G; ++i; }
  };
  auto load = [&]() H2O_INLINE {   // the rows of the next step
#pragma unroll
    for (int e = 0; e < NU; ++e) {
      const int i = min(ri[e], p.A - 1), n = max(node_of(i), 0);
      qr[e] = *reinterpret_cast<const u32x4*>(qh + (uint32_t)(rg[e] * a.T + n) * (uint32_t)D);
      advance(ri[e], rg[e]);
    }
    if (tid < kQRows) {   // a row that is none: lambda +inf, weights 0 (of a path: not added
                          // at all, whatever query was read in its place)
      const int n = li < p.A ? node_of(li) : -1;
      lr = n >= 0 ? lh[lg * a.T + n] * kLog2e : INFINITY;
      ir = li;
      advance(li, lg);
    }
  };
  auto store = [&](int buf) H2O_INLINE {
#pragma unroll
    for (int e = 0; e < NU; ++e)
      *reinterpret_cast<u32x4*>(&Qs[buf][(tid / (D / 8) + e * RU) * P + part]) = qr[e];
    if (tid < kQRows) {
      lam[buf][tid] = lr;
      pos[buf][tid] = ir;
    }
  };
  if (s0 < s1) load();
  bf16x8 kf[NKB][D / 32];
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb) {
    cks[kb] *= a.c;
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
      kf[kb][x] = Q8 && cache ? q8::codes_bf16(kr[kb][x][0], kr[kb][x][1])
                              : __builtin_bit_cast(bf16x8, kr[kb][x]);
  }
  // the products of the next 16 rows go out before the exponentials of these
  auto step = [&](auto chunk, int buf) H2O_INLINE {
    f32x4 s[2][NKB];
    auto product = [&](f32x4 (&d)[NKB], int n) H2O_INLINE {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb) d[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const bf16x8 qf = row_operand(Qs[buf], P, 16 * n + l16, 32 * x, lane);
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) d[kb] = mma(kf[kb][x], qf, d[kb]);
      }
    };
    product(s[0], 0);
#pragma unroll
    for (int n = 0; n < kQRows / 16; ++n) {
      if (n + 1 < kQRows / 16) product(s[(n + 1) & 1], n + 1);
      const float la = lam[buf][16 * n + l16];
      if (PATH && la == INFINITY) continue;
      const int i = decltype(chunk)::value ? pos[buf][16 * n + l16] : 0;
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float w = __builtin_amdgcn_exp2f(fmaf(s[n & 1][kb][r], cks[kb][r], -la));
          if (decltype(chunk)::value && j0 + 16 * kb + 4 * g4 + r > i) w = 0.f;
          cs[kb][r] += w;
        }
    }
  };
  if (s0 < s1) {
    store(0);
    if (s0 + 1 < s1) load();
    __syncthreads();
    for (int s = s0; s < s1; ++s) {
      const int buf = (s - s0) & 1;
      if (s + 1 < s1) {
        store(buf ^ 1);
        if (s + 2 < s1) load();
      }
      if (cache) step(IntConst<0>{}, buf);
      else step(IntConst<1>{}, buf);
      __syncthreads();
    }
  }
  const int nk = a.M + p.A;
  float* dst = p.dst + ((size_t)bz * gridDim.y + bh) * nk + (cache ? 0 : a.M);
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float v = cs[kb][r];
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) v += __shfl_xor(v, o, 64);
      const int j = j0 + 16 * kb + 4 * g4 + r;
      if (l16 == 0 && j < nkeys) {
        dst[j] = PATH && !cache && node_of(j) < 0 ? 0.f : v;
        if (cache) p.acc.add(bh * a.M + j, v);
      }
    }
}

// The column sums of at most 16 NR packed rows. The rows go into LDS once and the
// keys stream past them, 32 a wave, each group requested before the last one is used,
// without a barrier: bound by the cache's K rows, which are read once, where there are
// many. (B4 Hkv8 G4 d128 M32768, 5 rows a head: 8-bit cache 35 us, bf16 62
// (4.3 TB/s), against 72 and 79 by column_pass.)
template <int D, bool Q8, bool PATH, int NR>
__global__ __launch_bounds__(kThreads) void column_few(Args a, ColArgs p, int nb) {
  constexpr int NX = Q8 ? D / 64 : D / 32;   // 16-byte loads of a key row per lane
  constexpr int P = D + 8, NU = 16 * NR * D / 8 / kThreads;
  __shared__ __attribute__((aligned(16))) bf16_t Qs[16 * NR * P];
  __shared__ float2 lam[16 * NR];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const size_t bh = blockIdx.y;
  const int b = (int)blockIdx.y / a.Hkv, h = (int)blockIdx.y % a.Hkv;
  const int32_t* path = PATH ? p.path + (size_t)b * p.A : nullptr;
  if (PATH && (int)blockIdx.x >= nb) {
    copy_path<D>(a, p, bh, path, ((int)blockIdx.x - nb) * kThreads + tid);
    return;
  }
  const int ngroups = (a.M + 31) / 32, nwaves = 4 * nb, w0 = 4 * (int)blockIdx.x + wave;
  u32x4 kr[2][2][NX];
  float ks[2], old[2][2];       // old: the scores of this lane's columns (lanes l16 < 4)
  // K and the scales of head bh as buffer resources: rows past the cache read as zero
  constexpr uint32_t kRow = Q8 ? D : 2 * D;   // bytes
  const __amdgpu_buffer_rsrc_t krs =
      buffer_rsrc((const char*)a.kc + bh * a.M * (size_t)kRow, (uint32_t)a.M * kRow);
  const __amdgpu_buffer_rsrc_t srs =
      buffer_rsrc(Q8 ? a.ks + bh * (size_t)a.M : nullptr, Q8 ? (uint32_t)a.M * 4u : 0u);
  // (a score asked for behind the keys of a later group would be waited for with them)
  const __amdgpu_buffer_rsrc_t ors =
      buffer_rsrc(p.acc.scores ? p.acc.scores + bh * (size_t)a.M : nullptr,
                  p.acc.scores ? (uint32_t)a.M * 4u : 0u);
  auto issue = [&](int g, int u) H2O_INLINE {
    const uint32_t j0 = 32u * (uint32_t)g;
#pragma unroll
    for (int kb = 0; kb < 2 && !PATH; ++kb)   // (a path's calls add to no scores)
      old[u][kb] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
          ors, (int)(l16 < 4 ? (j0 + 16 * kb + 4 * g4 + l16) * 4u : 0x7FFFFFF0u), 0, 0));
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int x = 0; x < NX; ++x)
        kr[u][kb][x] = __builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       krs, (int)((j0 + 16 * kb + l16) * kRow +
                                  (Q8 ? 16 * g4 + 64 * x
                                      : 2 * (16 * g4 + 64 * (x >> 1) + 8 * (x & 1)))), 0, 0));
    if (Q8)
      ks[u] = __uint_as_float(
          __builtin_amdgcn_raw_buffer_load_b32(srs, (int)((j0 + (lane & 31)) * 4u), 0, 0));
  };
  {
    // rows of this thread's units, then its row's lambda (a row that is none: +inf,
    // weights 0), then the first keys, all before anything is used
    u32x4 qr[NU];
#pragma unroll
    for (int e = 0; e < NU; ++e) {
      const int r = min(tid / (D / 8) + e * (kThreads / (D / 8)), p.R - 1);
      const int node = max(path_node(path, r / a.G, a.T), 0);
      qr[e] = *reinterpret_cast<const u32x4*>(
          a.q + ((size_t)(b * a.Hq + h * a.G + r % a.G) * a.T + node) * D + 8 * (tid % (D / 8)));
    }
    float2 lr = {INFINITY, 0.f};
    if (tid < p.R) {
      const int node = path_node(path, tid / a.G, a.T);
      if (node >= 0)
        lr = row_weight(p.lse[(size_t)(b * a.Hq + h * a.G + tid % a.G) * a.T + node]);
    }
    issue(w0, 0);
#pragma unroll
    for (int e = 0; e < NU; ++e)
      *reinterpret_cast<u32x4*>(&Qs[(tid / (D / 8) + e * (kThreads / (D / 8))) * P +
                                    8 * (tid % (D / 8))]) = qr[e];
    if (tid < 16 * NR) lam[tid] = lr;
    __syncthreads();
  }
  float* dst = p.dst + bh * (size_t)(a.M + p.A);
  // 32 keys from key j0 on, kf their operands, ck their factors; chunk: key columns of
  // the chunk, hidden from the rows before them. keep(j): whether column j is a token.
  auto columns = [&](auto chunk, const bf16x8 (&kf)[2][D / 32], const f32x4 (&ck)[2], int j0,
                     int nkeys, float* to, const float (&prior)[2], auto&& keep) H2O_INLINE {
    f32x4 s[NR][2], cs[2];
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[n][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const bf16x8 qf = *reinterpret_cast<const bf16x8*>(
            &Qs[(16 * n + l16) * P + 64 * (x >> 1) + 16 * g4 + 8 * (x & 1)]);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) s[n][kb] = mma(kf[kb][x], qf, s[n][kb]);
      }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) cs[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const float2 la = lam[16 * n + l16];
      if (PATH && la.x == INFINITY) continue;
      const int i = decltype(chunk)::value ? (16 * n + l16) / a.G : 0;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float w = __builtin_amdgcn_exp2f(fmaf(s[n][kb][r], ck[kb][r], -la.x));
          if (decltype(chunk)::value && j0 + 16 * kb + 4 * g4 + r > i) w = 0.f;
          cs[kb][r] = fmaf(w, la.y, cs[kb][r]);
        }
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float v = cs[kb][r];
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) v += __shfl_xor(v, o, 64);
        const int j = j0 + 16 * kb + 4 * g4 + r;
        if (l16 == r && j < nkeys) {
          to[j] = keep(j) ? v : 0.f;
          if (!PATH && !decltype(chunk)::value && p.acc.scores) {
            const float sum = prior[kb] + v;
            p.acc.scores[bh * a.M + j] = sum;
            if (p.acc.copy) p.acc.copy[bh * a.M + j] = sum;
          }
        }
      }
  };
  auto consume = [&](int g, int u) H2O_INLINE {
    bf16x8 kf[2][D / 32];
    f32x4 ck[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const u32x4 v = kr[u][kb][x];
        if constexpr (Q8) {
          kf[kb][2 * x] = q8::codes_bf16(v[0], v[1]);
          kf[kb][2 * x + 1] = q8::codes_bf16(v[2], v[3]);
        } else {
          kf[kb][x] = __builtin_bit_cast(bf16x8, v);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
        ck[kb][r] = Q8 ? a.c * __shfl(ks[u], 16 * kb + 4 * g4 + r, 64) : a.c;
    }
    columns(IntConst<0>{}, kf, ck, 32 * g, a.M, dst, old[u], [](int) { return true; });
  };
  // whole trips of two groups (one past the cache reads zeros and stores nothing): an
  // exit or a branch between the two makes the compiler wait for the loads in flight
  if (nwaves >= ngroups) {
    if (w0 < ngroups) consume(w0, 0);
  } else {
    for (int g = w0; g < ngroups; g += 2 * nwaves) {
      issue(g + nwaves, 1);
      __builtin_amdgcn_sched_barrier(0);
      consume(g, 0);
      issue(g + 2 * nwaves, 0);
      __builtin_amdgcn_sched_barrier(0);
      consume(g + nwaves, 1);
    }
  }
  for (int j0 = 32 * w0; j0 < p.A; j0 += 32 * nwaves) {
    bf16x8 kf[2][D / 32];
    f32x4 ck[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int i = min(j0 + 16 * kb + l16, p.A - 1);
      const size_t row = bh * (size_t)a.T + max(path_node(path, i, a.T), 0);
      ck[kb] = f32x4{a.c, a.c, a.c, a.c};
#pragma unroll
      for (int x = 0; x < D / 32; ++x)
        kf[kb][x] = *reinterpret_cast<const bf16x8*>(a.kn + row * D + 16 * g4 + 64 * (x >> 1) +
                                                     8 * (x & 1));
    }
    columns(IntConst<1>{}, kf, ck, j0, p.A, dst + a.M, old[0],
            [&](int j) { return path_node(path, j, a.T) >= 0; });
  }
}

// wsum = the row ranges' sums, in their order.
__global__ __launch_bounds__(kThreads) void column_reduce(const float* __restrict__ parts,
                                                          float* __restrict__ wsum, int BH, int M,
                                                          int A, int nranges, ScoreAcc acc) {
  const int j = blockIdx.x * kThreads + threadIdx.x;
  if (j >= M + A) return;
  const size_t bh = blockIdx.y, e = bh * (size_t)(M + A) + j, n = (size_t)BH * (M + A);
  float s = parts[e];
  for (int k = 1; k < nranges; ++k) s += parts[k * n + e];
  wsum[e] = s;
  if (j < M) acc.add(bh * M + j, s);
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
              (const bf16_t*)in.vn, in.parents, reinterpret_cast<const uint32_t*>(ws + p.off_bits),
              s.Hq, s.Hkv, s.G(), s.T, s.M, s.G() * s.T, (s.T + 31) / 32, scale * kLog2e};
}

}  // namespace

// Rows per block and key ranges of the flash pass: those of least estimated time.
// us[k - 1]: microseconds per 32-key tile of a block that shares its CU with k - 1
// others (8-bit cache, Hkv8 G4 M8192; `resident` is what registers allow); a round takes
// every block's tiles at full residency, the last one at what is left, and 5 us to
// start and end; the partials of several ranges are written, read and merged (3 us
// and a byte of them in 1 / 3 TB/s). At B1 Hkv8 G4 T1024 d128 the plan takes 256 rows
// and two ranges, 193 + 8 us; 128 rows 221 + 8, four ranges 206 + 13. At d64 256 rows
// and two ranges 144 + 5, 128 rows and three 141 + 6. At T256 d128 64 rows and four
// ranges 75 + 4 us, two 98 + 4. (All measured with the probabilities in bf16, an
// eighth faster in every form.)
FlashPlan flash_plan(const FlashShape& s, bool tree) {
  FlashPlan p{};
  const long long BH = s.BH(), R = (long long)s.G() * s.T, cus = device_cus();
  const long long ntiles = (s.M + 31) / 32 + (s.T + 31) / 32;
  struct Block { int rows, resident; double us[4]; };
  static const Block k128[] = {{64, 3, {0.75, 1.13, 1.57}}, {128, 2, {1.05, 1.6}}, {256, 1, {1.4}}};
  static const Block k64[] = {{64, 4, {0.62, 0.87, 1.11, 1.41}}, {128, 3, {0.86, 1.21, 1.58}},
                              {256, 1, {1.06}}};
  // float32: 64 rows, two blocks per CU, 16 times the products' time
  static const Block kF32[] = {{64, 2, {4.0, 5.5}}};
  const Block* const blocks = s.f32 ? kF32 : s.d == 64 ? k64 : k128;
  double best = INFINITY;
  for (int v = 0; v < (s.f32 ? 1 : 3); ++v) {
    const Block& k = blocks[v];
    const long long nb = (R + k.rows - 1) / k.rows * BH, round = cus * k.resident;
    for (int n = 1; n <= kMaxFlashSplit && (n == 1 || n <= ntiles / 2); ++n) {
      const long long full = nb * n / round, left = (nb * n % round + cus - 1) / cus;
      const double tiles = (double)((ntiles + n - 1) / n);
      double us = tiles * (full * k.us[k.resident - 1] + (left ? k.us[left - 1] : 0.0)) +
                  5.0 * (double)(full + (left != 0));
      if (n > 1) us += 3.0 + (double)n * (double)BH * (double)R * s.d * 4.0 / 3.0e6;
      if (us < 0.97 * best) {   // a clear gain for more ranges or rows
        best = us;
        p.rows = k.rows;
        p.nsplit = n;
      }
    }
  }
  p.nranges = column_ranges(s, s.T);
  size_t off = 0;
  p.off_stats = off;
  if (p.nsplit > 1) off = align256_size(off + (size_t)p.nsplit * BH * R * sizeof(float2));
  p.off_opart = off;
  if (p.nsplit > 1) off = align256_size(off + (size_t)p.nsplit * BH * R * s.d * sizeof(float));
  p.off_bits = off;
  if (tree && s.T > kWaveTree)
    off = align256_size(off + (size_t)s.B * s.T * ((s.T + 31) / 32) * 4);
  // the tree's column sums are a call of their own, of any path
  p.off_parts = tree ? 0 : off;
  const int nr = tree ? kMaxColumnRanges : p.nranges;
  const size_t parts = nr > 1 ? align256_size((size_t)nr * BH * (s.M + s.T) * sizeof(float)) : 0;
  if (p.off_parts + parts > off) off = p.off_parts + parts;
  p.off_keys = off;
  if (!tree) off = align256_size(off + (size_t)BH * s.M * sizeof(float));
  p.bytes = off;
  return p;
}

// Waves per block of the bf16 column sums (32 keys each): 8, whose blocks read the
// rows half as often, where such blocks give every CU two.
int column_waves(const FlashShape& s, int ncol) {
  const long long nb = (long long)((s.M + 255) / 256 + (ncol + 255) / 256) * s.BH();
  return (long long)s.G() * ncol >= 512 && nb * 4 >= device_cus() ? 8 : 4;
}

// Row ranges of the column sums: blocks for four per CU, at least two steps each, and
// only from eight steps on (a step takes 0.8 us in bf16 and 1.1 in float32, adding the
// ranges 4: B1 Hq16 Hkv4 d64 M2049 T131 in float32 23.8 us in one range, 12.7 + 4 in four).
int column_ranges(const FlashShape& s, int ncol) {
  const int kb = s.f32 ? kColumnKeysF32 : 32 * column_waves(s, ncol), qr = s.f32 ? 32 : kQRows;
  const long long nb = (long long)((s.M + kb - 1) / kb + (ncol + kb - 1) / kb) * s.BH();
  const long long steps = ((long long)s.G() * ncol + qr - 1) / qr;
  long long n = steps < 8 ? 1 : (4ll * device_cus() + nb - 1) / nb;
  if (n > steps / 2) n = steps / 2;
  if (n > kMaxColumnRanges) n = kMaxColumnRanges;
  return n < 1 ? 1 : (int)n;
}

hipError_t launch_tree_bits(const FlashShape& s, const FlashPlan& p, const int32_t* parents,
                            char* ws, hipStream_t st) {
  uint32_t* bits = reinterpret_cast<uint32_t*>(ws + p.off_bits);
  const int W = (s.T + 31) / 32;
  const dim3 grid((s.T + kThreads - 1) / kThreads, s.B);
  return launch_kernel(K_TREE_BITS, s.T <= kTreeLds ? tree_bits<true> : tree_bits<false>, grid,
                       dim3(kThreads), st, parents, s.T, W, bits);
}

hipError_t launch_flash_combine(const FlashShape& s, const FlashPlan& p, void* out, float* lse,
                                const char* ws, hipStream_t st) {
  const size_t rows = (size_t)s.BH() * s.G() * s.T;
  auto go = [&](auto D, auto e) {
    typedef decltype(e) E;
    constexpr int kD = decltype(D)::value;
    const bool few = p.nsplit <= kFewSplits;
    const int per = kThreads / (kD / 4) / (few ? 1 : 8);
    return launch_kernel(K_FLASH_COMBINE, few ? flash_combine<kD, E, 1> : flash_combine<kD, E, 8>,
                         dim3((unsigned)((rows + per - 1) / per)), dim3(kThreads), st,
                         reinterpret_cast<const float2*>(ws + p.off_stats),
                         reinterpret_cast<const float*>(ws + p.off_opart), (E*)out, lse, s.BH(),
                         s.Hq, s.Hkv, s.G(), s.T, s.G() * s.T, p.nsplit);
  };
  if (s.f32) return s.d == 64 ? go(IntConst<64>{}, float{}) : go(IntConst<128>{}, float{});
  return s.d == 64 ? go(IntConst<64>{}, bf16_t{}) : go(IntConst<128>{}, bf16_t{});
}

hipError_t launch_column_reduce(const float* parts, float* wsum, int BH, int M, int A, int nranges,
                                ScoreAcc acc, hipStream_t st) {
  return launch_kernel(K_COLUMN_REDUCE, column_reduce,
                       dim3((unsigned)((M + A + kThreads - 1) / kThreads), BH), dim3(kThreads), st,
                       parts, wsum, BH, M, A, nranges, acc);
}

hipError_t launch_flash(const FlashShape& s, const FlashPlan& p, const FlashIn& in, void* out,
                        float* lse, char* ws, float scale, hipStream_t st) {
  const bool tree = in.parents != nullptr;
  if (tree && s.T > kWaveTree) {
    const hipError_t e = launch_tree_bits(s, p, in.parents, ws, st);
    if (e != hipSuccess) return e;
  }
  const Args a = make_args(s, in, ws, p, scale);
  const int nrt = (a.R + p.rows - 1) / p.rows;
  const dim3 grid(nrt * p.nsplit, s.BH());
  float2* stats = reinterpret_cast<float2*>(ws + p.off_stats);
  float* opart = reinterpret_cast<float*>(ws + p.off_opart);
  const hipError_t e = with_cache(s.d, in.q8, [&](auto D, auto q) {
    constexpr int kD = decltype(D)::value;
    constexpr bool kQ = decltype(q)::value;
    auto go = [&](auto kern) {
      return launch_kernel(K_FLASH, kern, grid, dim3(p.rows == 256 ? 512 : 256), st, a, p.nsplit,
                           (bf16_t*)out, lse, stats, opart);
    };
    auto rows = [&](auto mask) {
      constexpr bool kT = decltype(mask)::value;
      constexpr int kBN = kD == 64 ? 64 : 32;
      return p.rows == 256   ? go(flash_pass<kD, kQ, kT, 2, 8, kBN>)
             : p.rows == 128 ? go(flash_pass<kD, kQ, kT, 2, 4, kBN>)
                             : go(flash_pass<kD, kQ, kT, 1, 4, 32>);
    };
    if (tree) return rows(IntConst<1>{});
    if constexpr (kQ) return rows(IntConst<0>{});
    return hipErrorInvalidValue;   // the chunk over a bf16 cache has its own kernels
  });
  if (e != hipSuccess || p.nsplit == 1) return e;
  return launch_flash_combine(s, p, out, lse, ws, st);
}

hipError_t launch_columns(const FlashShape& s, const FlashPlan& p, const FlashIn& in,
                          const float* lse, const int32_t* path, int A, void* k_acc, void* v_acc,
                          float* wsum, char* ws, float scale, hipStream_t st, ScoreAcc acc) {
  const Args a = make_args(s, in, ws, p, scale);
  float* parts = reinterpret_cast<float*>(ws + p.off_parts);
  const int ncol = path ? A : s.T;
  if (s.G() * ncol <= kFewRows) {
    const ColArgs c{lse, path, ncol, s.G() * ncol, wsum, (bf16_t*)k_acc, (bf16_t*)v_acc, acc};
    // blocks per head: as many as are resident (4 per CU, 3 with 64 rows), then as many
    // as give every wave one group of keys or an even count
    const int groups = (s.M + 31) / 32, most = (c.R <= 32 ? 4 : 3) * device_cus() / s.BH();
    int per = most < 1 ? groups : (groups + 4 * most - 1) / (4 * most);
    if (per > 1) per += per & 1;
    if (per < 1) per = 1;
    const int nb = groups ? (groups + 4 * per - 1) / (4 * per) : 1;
    const dim3 grid(nb + (path ? (A * (s.d / 8) + kThreads - 1) / kThreads : 0), s.BH());
    return with_cache(s.d, in.q8, [&](auto D, auto q) {
      constexpr int kD = decltype(D)::value;
      constexpr bool kQ = decltype(q)::value;
      auto go = [&](auto kern) {
        return launch_kernel(K_COLUMNS, kern, grid, dim3(kThreads), st, a, c, nb);
      };
      const bool two = c.R <= 32;
      if (path) return two ? go(column_few<kD, kQ, true, 2>) : go(column_few<kD, kQ, true, 4>);
      if constexpr (kQ)
        return two ? go(column_few<kD, true, false, 2>) : go(column_few<kD, true, false, 4>);
      return hipErrorInvalidValue;
    });
  }
  const int nw = column_waves(s, ncol);
  const int kb = 32 * nw, nt = 64 * nw, tiles = (s.M + kb - 1) / kb + (ncol + kb - 1) / kb;
  const int ncopy = path ? (A * (s.d / 8) + nt - 1) / nt : 0;
  const ColArgs c{lse, path, ncol, s.G() * ncol, p.nranges > 1 ? parts : wsum, (bf16_t*)k_acc,
                  (bf16_t*)v_acc, p.nranges > 1 ? ScoreAcc{} : acc};
  const dim3 grid(tiles + ncopy, s.BH(), p.nranges);
  const hipError_t e = with_cache(s.d, in.q8, [&](auto D, auto q) {
    constexpr int kD = decltype(D)::value;
    constexpr bool kQ = decltype(q)::value;
    auto go = [&](auto kern) { return launch_kernel(K_COLUMNS, kern, grid, dim3(nt), st, a, c); };
    if (path)
      return nw == 8 ? go(column_pass<kD, kQ, true, 2, 8>) : go(column_pass<kD, kQ, true, 2, 4>);
    if constexpr (kQ)
      return nw == 8 ? go(column_pass<kD, true, false, 2, 8>)
                     : go(column_pass<kD, true, false, 2, 4>);
    return hipErrorInvalidValue;
  });
  if (e != hipSuccess || p.nranges == 1) return e;
  return launch_column_reduce(parts, wsum, s.BH(), s.M, ncol, p.nranges, acc, st);
}

}  // namespace h2o
