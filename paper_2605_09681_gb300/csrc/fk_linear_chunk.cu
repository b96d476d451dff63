// Linear attention with decays, in chunks of 128 tokens on the 5th-generation tensor cores.
//
// With G_i the sum of the decays' logarithms from a chunk's start through token i, and S the state before the chunk,
//   o_i = scale (exp(G_i) q_i S + sum_(j <= i) exp(G_i - G_j) (q_i k_j) v_j),
//   S'  = exp(G_C) S + sum_j exp(G_C - G_j) k_j v_j^T:
// four matrix products of 128 x 128 x D a chunk and head (six: see K'), 1.3 times the time of its 1 KB a token from DRAM if the
// tensor cores run at their measured rate alone.  All exponents are of sums that are <= 0 where decays are.
//
// One CTA takes a segment of one kv head's chunks in turn, for all query heads that share it:
//   warp 0        TMA: K and V of a chunk, Q of a chunk and query head, two stages each, 128-byte swizzle
//   warp 1        tcgen05.mma, one elected lane: A = Q K^T, X = Q S, Y = P V, dS = K'^T V
//   warp 2        the chunk's running sums G (two fp32 numbers, log2 domain) and what follows from them alone
//   warps 4-7     K' = exp(G_C - G_j) k_j, transposed by ldmatrix into tensor memory (the A operand of dS), in three bf16 parts: the
//                 state is kept to fp32 (two parts: 2^-17 of each term).  Half a chunk at a time.  Between the halves
//                 P_ij = exp(G_i - G_j) A_ij for j <= i as bf16, over A's columns.
//   warps 8-11    the state: thread r keeps row r (channel r of k) in registers, S' = exp(G_C) S + dS, and writes it as bf16 to
//                 shared memory, the B operand of X
//   warps 12-15   o: thread i reads row i of X, then of Y (the same columns), and writes its row
// Tensor memory columns: A and P 0-127, X and Y 128.., dS 256.., K' 384-479.
//
// kLocal: the state alone, from zero (what a segment adds), without Q and o.
// Every wait is bounded; when one expires the CTA records it, drains its copies and products, and ends.
#include "fk_linear.h"
#include "fk_tc.h"

namespace fk {
namespace {

constexpr int C = kLinearChunk;
constexpr int kThreads = 512;
constexpr uint32_t kColA = 0, kColX = 128, kColS = 256, kColK = 384;

struct Barriers {
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], q_full[2], q_empty[2];
  uint64_t g_full[2], g_empty[2];
  uint64_t a_full, p_full, kp_full, kp_empty, ds_full, ds_empty;
  uint64_t s_full, s_empty, x_full, x_empty, y_full, y_empty;
  uint64_t fin;
  uint32_t tmem_base;
  volatile int abort;
};

template <int D>
struct Layout {
  static constexpr int kTile = C * D * 2;         // bytes of a tile of Q, K or V: D / 64 panels of 128-byte rows
  static constexpr int kOffK = 0, kOffV = 2 * kTile, kOffQ = 4 * kTile;
  static constexpr int kOffS = 6 * kTile;         // S: D / 64 panels of D 128-byte rows
  static constexpr int kOffG = kOffS + D * D * 2; // [2][C] G (log2), [2][C] exp(G_C - G_j)
  static constexpr int kOffBar = kOffG + 4 * C * 4;
  static constexpr int kUsed = kOffBar + (int)sizeof(Barriers) + 16;   // exp(G_C) of two chunks behind the barriers
  // at least ~116 KB, so that one CTA occupies an SM (its 512 tensor memory columns are then free)
  static constexpr int kSmem = kUsed > 118 * 1024 ? kUsed : 118 * 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory");
};

// 16 lanes x 32 columns of tensor memory from transposed 8 x 8 tiles (ldmatrix): register 2 b + s is lane 8 s + t / 4, column
// 4 b + t % 4 of thread t
__device__ __forceinline__ void tmem_st_tiles(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      :: "r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
      "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t addr, uint32_t* v) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void fence_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// Warp-uniform bounded wait for the phase of parity `parity`; false when the CTA is aborting or the limit expired (which
// starts the abort).  (fk_tc.h's counts in 64 bits; out of line it is a call, which warps of fewer registers cannot make.)
__device__ __forceinline__ bool wait(uint64_t* b, uint32_t parity, Barriers* bar, int* status) {
  if (__all_sync(0xffffffffu, mbar_test(b, parity))) return true;
  uint32_t t0;
  asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(t0));
  while (true) {
#pragma unroll 1
    for (int i = 0; i < 16; ++i)
      if (__all_sync(0xffffffffu, mbar_test(b, parity))) return true;
    uint32_t t;
    asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(t));
    bool stop = bar->abort;
    if (t - t0 > (uint32_t)kWaitLimitNs) {
      bar->abort = 1;
      atomicOr(status, kStatusTimeout);
      stop = true;
    }
    if (__any_sync(0xffffffffu, stop)) return false;
  }
}
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(N)); }
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// a sum kept as two numbers
struct Two {
  float h, l;
};
__device__ __forceinline__ Two add(Two a, Two b) {
  const float s = a.h + b.h, v = s - a.h;
  const float e = (a.h - (s - v)) + (b.h - v) + (a.l + b.l);
  const float h = s + e;
  return {h, e - (h - s)};
}

// Eight columns of a row of sum_(j <= i) P_ij v_j by themselves, in fp32: the product P V multiplies the zeros of P with
// what later tokens of the chunk hold, and gives NaN where that is not finite.
template <int D>
__device__ __noinline__ void row_alone(const LinearChunkArgs& a, const float* g, int64_t tok0, int i, int head, int kvh, int col, float* y) {
  float acc[8] = {};
  const bf16* q = a.Q + (tok0 + i) * a.qstride + (int64_t)head * D;
  for (int j = 0; j <= i; ++j) {
    const bf16* k = a.K + (tok0 + j) * a.kstride + (int64_t)kvh * D;
    float s = 0.0f;
    for (int c = 0; c < D; ++c) s = fmaf(__bfloat162float(q[c]), __bfloat162float(k[c]), s);
    const float p = s * exp2f(g[i] - g[j]);
    const bf16* v = a.V + (tok0 + j) * a.vstride + (int64_t)kvh * D + col;
    for (int c = 0; c < 8; ++c) acc[c] = fmaf(p, __bfloat162float(v[c]), acc[c]);
  }
  for (int c = 0; c < 8; ++c) y[c] = acc[c];
}

template <int D, bool kLocal>
__global__ void __launch_bounds__(kThreads, 1)
linear_chunk_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV, const __grid_constant__ LinearChunkArgs a) {
  using Lay = Layout<D>;
  constexpr int kPanels = D / 64;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* sK = smem + Lay::kOffK;
  uint8_t* sV = smem + Lay::kOffV;
  uint8_t* sQ = smem + Lay::kOffQ;
  uint8_t* sS = smem + Lay::kOffS;
  float* sG = reinterpret_cast<float*>(smem + Lay::kOffG);   // [2][C]
  float* sW = sG + 2 * C;                                    // [2][C]
  Barriers* bar = reinterpret_cast<Barriers*>(smem + Lay::kOffBar);
  volatile float* sE = reinterpret_cast<volatile float*>(smem + Lay::kOffBar + sizeof(Barriers));   // [2]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // ---- this CTA's segment
  int s = 0;
  {
    int hi = a.seqs.n - 1;
    while (s < hi) {
      const int mid = (s + hi + 1) >> 1;
      if (a.seqs.item0[mid] <= (int)blockIdx.x) s = mid;
      else hi = mid - 1;
    }
  }
  const int segs = a.seqs.segs[s], item = (int)blockIdx.x - a.seqs.item0[s];
  const int seg = item / a.Hkv, kvh = item - seg * a.Hkv;
  const int len = a.seqs.len[s], chunks = (len + C - 1) / C;
  const int c0 = (int)((int64_t)chunks * seg / segs), nc = (int)((int64_t)chunks * (seg + 1) / segs) - c0;   // nc >= 1
  const int64_t tok0 = (int64_t)a.seqs.tok0[s] + (int64_t)c0 * C;   // of the segment
  const int tokens = min(len - c0 * C, nc * C);
  const int G = kLocal ? 1 : a.G;
  const int64_t place = (int64_t)a.seqs.place0[s] + kvh * segs + seg;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bar->k_full[i], 1);
      mbar_init(&bar->k_empty[i], kLocal ? 4 : 5);           // the converting warps, and Q K^T
      mbar_init(&bar->v_full[i], 1);
      mbar_init(&bar->v_empty[i], 1);
      mbar_init(&bar->q_full[i], 1);
      mbar_init(&bar->q_empty[i], 1);
      mbar_init(&bar->g_full[i], 1);
      mbar_init(&bar->g_empty[i], kLocal ? 8 : 12);
    }
    mbar_init(&bar->a_full, 1);
    mbar_init(&bar->p_full, 4);
    mbar_init(&bar->kp_full, 4);
    mbar_init(&bar->kp_empty, 1);
    mbar_init(&bar->ds_full, 1);
    mbar_init(&bar->ds_empty, 4);
    mbar_init(&bar->s_full, 4);
    mbar_init(&bar->s_empty, 1);
    mbar_init(&bar->x_full, 1);
    mbar_init(&bar->x_empty, 4);
    mbar_init(&bar->y_full, 1);
    mbar_init(&bar->y_empty, 4);
    mbar_init(&bar->fin, 1);
    bar->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 :: "r"(su32(&bar->tmem_base)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bar->tmem_base;
  const int wq = warp & 3, row = wq * 32 + lane;             // tensor memory lane of a thread of warps 4-15
  const uint32_t lanes = tmem + ((uint32_t)(wq * 32) << 16);
  auto wait_for = [&](uint64_t* b, uint32_t parity) { return wait(b, parity, bar, a.status); };
  auto arrive = [&](uint64_t* b) {                           // of a warp
    __syncwarp();
    if (lane == 0) mbar_arrive(b);
  };

  if (warp < 4) {
    fewer_registers<56>();
    if (warp == 0) {
      // ------------------------------------------------------------------ TMA
      bool ok = true;
      int ik = -1, iv = -1, iq = -1;                         // last tiles issued
      auto load = [&](const CUtensorMap* map, uint8_t* dst, uint64_t* b, int head, int n) {
        if (lane == 0) {
          mbar_expect_tx(b, Lay::kTile);
          for (int p = 0; p < kPanels; ++p) tma_load_2d(dst + p * (C * 128), map, b, head * D + p * 64, (int)(tok0 + n * C));
        }
        __syncwarp();
      };
      for (int n = 0; n < nc && ok; ++n) {
        const int b = n & 1, u = n >> 1;
        if (u > 0 && !(ok = wait_for(&bar->k_empty[b], (u - 1) & 1))) break;
        load(&tmK, sK + b * Lay::kTile, &bar->k_full[b], kvh, n);
        ik = n;
        for (int g = 0; g < G; ++g) {
          if (!kLocal) {
            const int m = n * G + g, qb = m & 1, qu = m >> 1;
            if (qu > 0 && !(ok = wait_for(&bar->q_empty[qb], (qu - 1) & 1))) break;
            load(&tmQ, sQ + qb * Lay::kTile, &bar->q_full[qb], kvh * G + g, n);
            iq = m;
          }
          if (g == 0) {
            if (u > 0 && !(ok = wait_for(&bar->v_empty[b], (u - 1) & 1))) break;
            load(&tmV, sV + b * Lay::kTile, &bar->v_full[b], kvh, n);
            iv = n;
          }
        }
      }
      if (!ok) {                                             // what was issued lands before the CTA ends
        for (int i = max(0, ik - 1); i <= ik; ++i) wait_phase(&bar->k_full[i & 1], (i >> 1) & 1, bar, a.status, false);
        for (int i = max(0, iv - 1); i <= iv; ++i) wait_phase(&bar->v_full[i & 1], (i >> 1) & 1, bar, a.status, false);
        for (int i = max(0, iq - 1); i <= iq; ++i) wait_phase(&bar->q_full[i & 1], (i >> 1) & 1, bar, a.status, false);
      }
      __syncwarp();
    } else if (warp == 1) {
      // ------------------------------------------------------------------ MMA issuer
      // Operations of one thread complete in issue order.
      constexpr uint32_t kIdA = idesc_bf16(C, C, 0), kIdD = idesc_bf16(C, D, 1);
      const uint64_t dQ = sdesc(su32(sQ), 16, 1024), dK = sdesc(su32(sK), 16, 1024);
      const uint64_t dV = sdesc(su32(sV), 16384, 1024), dS = sdesc(su32(sS), D * 128, 1024);
      bool ok = true;
      auto q_k = [&](int m, int n) {                         // A = Q K^T
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = (uint32_t)((kk >> 2) * 1024 + (kk & 3) * 2);
          umma(tmem + kColA, dQ + (uint32_t)((m & 1) * (Lay::kTile >> 4)) + off,
               dK + (uint32_t)((n & 1) * (Lay::kTile >> 4)) + off, kIdA, kk > 0 ? 1u : 0u);
        }
        umma_commit(&bar->a_full);
      };
      auto ds = [&](int n, int half) {                       // dS += K'^T V of 64 tokens
        const uint64_t db = dV + (uint32_t)((n & 1) * (Lay::kTile >> 4)) + (uint32_t)(half * 4 * 128);
#pragma unroll
        for (int part = 0; part < 3; ++part)
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            umma_ts(tmem + kColS, tmem + kColK + part * 32 + kk * 8, db + kk * 128, kIdD, half + part + kk > 0 ? 1u : 0u);
        umma_commit(&bar->kp_empty);
      };
      if (!kLocal) {
        ok = wait_for(&bar->k_full[0], 0) && wait_for(&bar->q_full[0], 0);
        if (ok) {
          tc_fence_after();
          if (elect_one()) {
            q_k(0, 0);
            if (G == 1) umma_commit(&bar->k_empty[0]);
          }
          __syncwarp();
        }
      }
      for (int n = 0; n < nc && ok; ++n) {
        const int b = n & 1, u = n >> 1;
        for (int g = 0; g < G && ok; ++g) {
          const int m = n * G + g;
          if (!kLocal) {                                     // X = Q S
            if (g == 0 && !(ok = wait_for(&bar->s_full, n & 1))) break;
            if (m > 0 && !(ok = wait_for(&bar->y_empty, (m - 1) & 1))) break;
            tc_fence_after();
            if (elect_one()) {
              const uint64_t da = dQ + (uint32_t)((m & 1) * (Lay::kTile >> 4));
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk)
                umma(tmem + kColX, da + (uint32_t)((kk >> 2) * 1024 + (kk & 3) * 2), dS + kk * 128, kIdD, kk > 0 ? 1u : 0u);
              umma_commit(&bar->x_full);
              umma_commit(&bar->q_empty[m & 1]);
              if (g == G - 1) umma_commit(&bar->s_empty);
            }
            __syncwarp();
          }
          if (g == 0) {
            if (!(ok = wait_for(&bar->kp_full, 0) && wait_for(&bar->v_full[b], u & 1))) break;
            if (n > 0 && !(ok = wait_for(&bar->ds_empty, (n - 1) & 1))) break;
            tc_fence_after();
            if (elect_one()) ds(n, 0);
            __syncwarp();
          }
          if (!kLocal) {                                     // Y = P V, and the next A
            if (!(ok = wait_for(&bar->p_full, m & 1) && wait_for(&bar->x_empty, m & 1))) break;
            tc_fence_after();
            if (elect_one()) {
              const uint64_t db = dV + (uint32_t)(b * (Lay::kTile >> 4));
#pragma unroll
              for (int kk = 0; kk < C / 16; ++kk)
                umma_ts(tmem + kColX, tmem + kColA + kk * 8, db + kk * 128, kIdD, kk > 0 ? 1u : 0u);
              umma_commit(&bar->y_full);
              if (G > 1 && g == G - 1) umma_commit(&bar->v_empty[b]);
            }
            __syncwarp();
            if (m + 1 < nc * G) {
              const int n1 = g + 1 < G ? n : n + 1;
              if (n1 > n && !(ok = wait_for(&bar->k_full[n1 & 1], (n1 >> 1) & 1))) break;
              if (!(ok = wait_for(&bar->q_full[(m + 1) & 1], ((m + 1) >> 1) & 1))) break;
              tc_fence_after();
              if (elect_one()) {
                q_k(m + 1, n1);
                if ((m + 1) % G == G - 1) umma_commit(&bar->k_empty[n1 & 1]);
              }
              __syncwarp();
            }
          }
          if (g == 0) {
            if (!(ok = wait_for(&bar->kp_full, 1))) break;
            tc_fence_after();
            if (elect_one()) {
              ds(n, 1);
              umma_commit(&bar->ds_full);
              if (G == 1) umma_commit(&bar->v_empty[b]);
            }
            __syncwarp();
          }
        }
      }
      if (elect_one()) umma_commit(&bar->fin);               // completes once every product above is done
      wait_phase(&bar->fin, 0, bar, a.status, false);
      __syncwarp();
    } else if (warp == 2) {
      // ------------------------------------------------------------------ running sums of a chunk: lane's tokens 4 lane .. + 3
      const float* decay = a.decay + tok0 * a.dstride + kvh;
      float x[4];
      auto fetch = [&](int n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = n * C + 4 * lane + i;
          x[i] = t < tokens ? __ldg(decay + (int64_t)t * a.dstride) : 0.0f;
        }
      };
      fetch(0);
      for (int n = 0; n < nc; ++n) {
        const int b = n & 1, u = n >> 1;
        Two sum[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y = at_least(x[i], kLeastDecay);
          const float h = y * 1.4426950408889634f;           // log2(e) in two numbers
          const Two z{h, fmaf(y, 1.4426950408889634f, -h) + y * 1.925963033500e-8f};
          sum[i] = i == 0 ? z : add(sum[i - 1], z);
        }
        Two all = sum[3];
        for (int o = 1; o < 32; o *= 2) {
          const Two z{__shfl_up_sync(0xffffffffu, all.h, o), __shfl_up_sync(0xffffffffu, all.l, o)};
          if (lane >= o) all = add(z, all);
        }
        const Two before{__shfl_up_sync(0xffffffffu, all.h, 1), __shfl_up_sync(0xffffffffu, all.l, 1)};
        const Two end{__shfl_sync(0xffffffffu, all.h, 31), __shfl_sync(0xffffffffu, all.l, 31)};
        if (n + 1 < nc) fetch(n + 1);
        if (u > 0 && !wait_for(&bar->g_empty[b], (u - 1) & 1)) break;
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (lane > 0) sum[i] = add(before, sum[i]);
          w[i] = n * C + 4 * lane + i < tokens ? exp2f((end.h - sum[i].h) + (end.l - sum[i].l)) : 0.0f;
        }
        *reinterpret_cast<float4*>(sG + b * C + 4 * lane) = make_float4(sum[0].h, sum[1].h, sum[2].h, sum[3].h);
        *reinterpret_cast<float4*>(sW + b * C + 4 * lane) = make_float4(w[0], w[1], w[2], w[3]);
        if (lane == 0) sE[b] = exp2f(end.h + end.l);
        arrive(&bar->g_full[b]);
      }
    }
  } else if (warp < 8) {
    fewer_registers<120>();
    // ------------------------------------------------------------------ K' and P
    // K' of 64 tokens: channels 32 wq .. + 31 of this warp, 16 at a time
    auto convert = [&](int n, int half, int valid) {
      const uint32_t tile = su32(sK) + (uint32_t)((n & 1) * Lay::kTile);
      const float* w = sW + (n & 1) * C + half * 64 + 2 * (lane & 3);
      const int r = lane & 7, mat = lane >> 3;
#pragma unroll 1
      for (int hf = 0; hf < 2; ++hf) {
        const int c = 32 * wq + 16 * hf + (mat & 1) * 8;     // channel of the row that this lane gives ldmatrix
        const uint32_t at = tile + (uint32_t)((c >> 6) * (C * 128) + (half * 64 + (mat >> 1) * 8 + r) * 128 + ((((c & 63) >> 3) ^ r) << 4));
        uint32_t x[16], hi[16], mid[16], lo[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) ldmatrix4t(at + i * (16 * 128), x + 4 * i);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int t = 8 * (i >> 1);                        // token of the pair, less 2 (lane & 3)
          const float2 ww = *reinterpret_cast<const float2*>(w + t);
          uint32_t v = x[i];
          if (valid < C) {                                   // (tokens of others: any values)
            const int j = half * 64 + t + 2 * (lane & 3);
            v = j + 1 < valid ? v : j < valid ? v & 0xFFFFu : 0u;
          }
          float p = low(v) * ww.x, q = high(v) * ww.y;
          hi[i] = pack_bf16(p, q);
          p -= low(hi[i]);
          q -= high(hi[i]);
          mid[i] = pack_bf16(p, q);
          p -= low(mid[i]);
          q -= high(mid[i]);
          lo[i] = pack_bf16(p, q);
        }
        const uint32_t to = lanes + kColK + ((uint32_t)(16 * hf) << 16);
        tmem_st_tiles(to, hi);
        tmem_st_tiles(to + 32, mid);
        tmem_st_tiles(to + 64, lo);
      }
      tmem_wait_st();
      tc_fence_before();
      arrive(&bar->kp_full);
    };
    for (int n = 0; n < nc; ++n) {
      const int b = n & 1, u = n >> 1, valid = min(C, tokens - n * C);
      if (!wait_for(&bar->k_full[b], u & 1) || !wait_for(&bar->g_full[b], u & 1)) break;
      if (n > 0 && !wait_for(&bar->kp_empty, 1)) break;      // the chunk before's second half
      tc_fence_after();
      if (valid < C) {                                       // rows of others: zeros for the products with V
        if (!wait_for(&bar->v_full[b], u & 1)) break;
        if (row >= valid) {
#pragma unroll
          for (int p = 0; p < kPanels; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i)
              *reinterpret_cast<uint4*>(sV + b * Lay::kTile + p * (C * 128) + row * 128 + i * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_to_async();
      }
      const bool mine = 32 * wq < D;                         // D = 64: lanes 64-127 of dS are not used
      if (mine) convert(n, 0, valid);
      else arrive(&bar->kp_full);
      bool ok = true;
      for (int g = 0; g < G && ok; ++g) {
        if (!kLocal) {
          const int m = n * G + g;
          if (!(ok = wait_for(&bar->a_full, m & 1))) break;
          tc_fence_after();
          const float gi = sG[b * C + row];
          const float4* gj = reinterpret_cast<const float4*>(sG + b * C);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t p[16];
            if (q <= wq) {
              uint32_t x[32];
              FK_TMEM_LD32(lanes + kColA + 32 * q, x);
              FK_TMEM_WAIT_LD32(x);
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float4 y = gj[8 * q + i];
                const float yy[4] = {y.x, y.y, y.z, y.w};
                float e[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                  e[c] = __uint_as_float(x[4 * i + c]) * fast_exp2(gi - yy[c]);
                  if (q == wq && 4 * i + c > lane) e[c] = 0.0f;
                }
                p[2 * i] = pack_bf16(e[0], e[1]);
                p[2 * i + 1] = pack_bf16(e[2], e[3]);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) p[i] = 0;
            }
            FK_TMEM_ST16(lanes + kColA + 16 * q, p);
          }
          tmem_wait_st();
          tc_fence_before();
          arrive(&bar->p_full);
        }
        if (g == 0) {
          if (!(ok = wait_for(&bar->kp_empty, 0))) break;
          tc_fence_after();
          if (mine) convert(n, 1, valid);
          else arrive(&bar->kp_full);
          arrive(&bar->k_empty[b]);
        }
      }
      if (!ok) break;
      arrive(&bar->g_empty[b]);
    }
  } else if (warp < 12) {
    more_registers<168>();
    // ------------------------------------------------------------------ the state
    const bool mine = 32 * wq < D;
    float st[D];
    float left = 1.0f;                                       // what the segment leaves of a state
    if (kLocal || !mine) {
#pragma unroll
      for (int i = 0; i < D; ++i) st[i] = 0.0f;
    } else {
      const float* from = (segs > 1 ? a.place + place * (D * D) : a.state + ((int64_t)a.seqs.slot[s] * a.Hkv + kvh) * (D * D)) + row * D;
#pragma unroll
      for (int i = 0; i < D; i += 4) {
        const float4 v = *reinterpret_cast<const float4*>(from + i);
        st[i] = v.x, st[i + 1] = v.y, st[i + 2] = v.z, st[i + 3] = v.w;
      }
    }
    bool ok = true;
    for (int n = 0; n < nc; ++n) {
      const int b = n & 1, u = n >> 1;
      if (!kLocal) {
        if (n > 0 && !(ok = wait_for(&bar->s_empty, (n - 1) & 1))) break;
        if (mine) {
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            const uint4 v = make_uint4(pack_bf16(st[8 * i], st[8 * i + 1]), pack_bf16(st[8 * i + 2], st[8 * i + 3]),
                                       pack_bf16(st[8 * i + 4], st[8 * i + 5]), pack_bf16(st[8 * i + 6], st[8 * i + 7]));
            *reinterpret_cast<uint4*>(sS + (i >> 3) * (D * 128) + row * 128 + (((i & 7) ^ (row & 7)) << 4)) = v;
          }
          fence_to_async();
        }
        arrive(&bar->s_full);
      }
      if (!(ok = wait_for(&bar->g_full[b], u & 1))) break;
      const float e = sE[b];
      arrive(&bar->g_empty[b]);
      left *= e;
      if (!(ok = wait_for(&bar->ds_full, n & 1))) break;
      tc_fence_after();
      if (mine) {
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
          uint32_t x[32];
          FK_TMEM_LD32(lanes + kColS + 32 * q, x);
          FK_TMEM_WAIT_LD32(x);
#pragma unroll
          for (int i = 0; i < 32; ++i) st[32 * q + i] = fmaf(st[32 * q + i], e, __uint_as_float(x[i]));
        }
      }
      tc_fence_before();
      arrive(&bar->ds_empty);
    }
    float* to = nullptr;
    if (kLocal) to = a.place + (place + 1) * (D * D);
    else if (a.state_new && seg == segs - 1)
      to = a.state_new + ((int64_t)(a.to_out ? a.seqs.out[s] : a.seqs.slot[s]) * a.Hkv + kvh) * (D * D);
    if (ok && to && mine) {
#pragma unroll
      for (int i = 0; i < D; i += 4) *reinterpret_cast<float4*>(to + row * D + i) = make_float4(st[i], st[i + 1], st[i + 2], st[i + 3]);
      if (kLocal && row == 0) a.place_decay[place + 1] = left;
    }
  } else {
    more_registers<168>();
    // ------------------------------------------------------------------ o
    bool ok = !kLocal;
    for (int n = 0; n < nc && ok; ++n) {
      const int b = n & 1, u = n >> 1, t = n * C + row;
      if (!(ok = wait_for(&bar->g_full[b], u & 1))) break;
      const float e = a.scale * exp2f(sG[b * C + row]);
      for (int g = 0; g < G; ++g) {
        const int m = n * G + g;
        float o[D];
        if (!(ok = wait_for(&bar->x_full, m & 1))) break;
        tc_fence_after();
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
          uint32_t x[32];
          FK_TMEM_LD32(lanes + kColX + 32 * q, x);
          FK_TMEM_WAIT_LD32(x);
#pragma unroll
          for (int i = 0; i < 32; ++i) o[32 * q + i] = e * __uint_as_float(x[i]);
        }
        tc_fence_before();
        arrive(&bar->x_empty);
        if (!(ok = wait_for(&bar->y_full, m & 1))) break;
        tc_fence_after();
        bf16* to = a.O + (tok0 + t) * a.ostride + (int64_t)(kvh * G + g) * D;
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
          uint32_t y[32];
          FK_TMEM_LD32(lanes + kColX + 32 * q, y);
          FK_TMEM_WAIT_LD32(y);
          if (q == D / 32 - 1) {                             // the last of Y is read
            tc_fence_before();
            arrive(&bar->y_empty);
          }
          float z = 0.0f;                                    // NaN if any of Y is not finite
#pragma unroll
          for (int i = 0; i < 32; ++i) z = fmaf(__uint_as_float(y[i]), 0.0f, z);
          if (z != z && t < tokens) {
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
              float x = 0.0f, f[8];
#pragma unroll
              for (int c = 0; c < 8; ++c) x = fmaf(__uint_as_float(y[i + c]), 0.0f, x);
              if (x == x) continue;
              row_alone<D>(a, sG + b * C, tok0 + n * C, row, kvh * G + g, kvh, 32 * q + i, f);
#pragma unroll
              for (int c = 0; c < 8; ++c) y[i + c] = __float_as_uint(f[c]);
            }
          }
          uint32_t v[16];
#pragma unroll
          for (int i = 0; i < 16; ++i)
            v[i] = pack_bf16(fmaf(a.scale, __uint_as_float(y[2 * i]), o[32 * q + 2 * i]),
                             fmaf(a.scale, __uint_as_float(y[2 * i + 1]), o[32 * q + 2 * i + 1]));
          if (t < tokens) {
            if (a.wide_o) {
#pragma unroll
              for (int i = 0; i < 2; ++i)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                             :: "l"(to + 32 * q + 16 * i), "r"(v[8 * i]), "r"(v[8 * i + 1]), "r"(v[8 * i + 2]), "r"(v[8 * i + 3]),
                             "r"(v[8 * i + 4]), "r"(v[8 * i + 5]), "r"(v[8 * i + 6]), "r"(v[8 * i + 7]) : "memory");
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                *reinterpret_cast<uint4*>(to + 32 * q + 8 * i) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            }
          }
        }
      }
      if (ok) arrive(&bar->g_empty[b]);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(512u) : "memory");
  }
}

// The states before each segment of a head: place i + 1 holds what segment i adds to a zero state.
template <int D>
__global__ void __launch_bounds__(256) linear_join_kernel(const __grid_constant__ LinearChunkArgs a) {
  constexpr int kBlocks = D * D / 4 / 256;        // of a head
  const int k = blockIdx.y, segs = a.seqs.segs[k];
  if (segs < 2) return;
  const int h = blockIdx.x / kBlocks, at = (blockIdx.x % kBlocks) * 256 + threadIdx.x;
  const int64_t place = (int64_t)a.seqs.place0[k] + h * segs;
  float4 s = reinterpret_cast<const float4*>(a.state + ((int64_t)a.seqs.slot[k] * a.Hkv + h) * (D * D))[at];
  float4* p = reinterpret_cast<float4*>(a.place + place * (D * D)) + at;
  p[0] = s;
  p += D * D / 4;
  const float* decay = a.place_decay + place + 1;
  constexpr int kAhead = 8;
  for (int i0 = 1; i0 < segs; i0 += kAhead) {
    float4 x[kAhead];
    float e[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i0 + i < segs) {
        x[i] = p[i * (D * D / 4)];
        e[i] = decay[i];
      }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i0 + i < segs) {
        s.x = fmaf(s.x, e[i], x[i].x);
        s.y = fmaf(s.y, e[i], x[i].y);
        s.z = fmaf(s.z, e[i], x[i].z);
        s.w = fmaf(s.w, e[i], x[i].w);
        p[i * (D * D / 4)] = s;
      }
    p += kAhead * (D * D / 4);
    decay += kAhead;
  }
}

template <int D>
cudaError_t prepare() {
  cudaError_t e = cudaFuncSetAttribute(linear_chunk_kernel<D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<D>::kSmem);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(linear_chunk_kernel<D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<D>::kSmem);
  return e;
}

template <int D>
cudaError_t launch(bool split, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const LinearChunkArgs& a,
                   cudaStream_t s) {
  if (split) {
    LinearChunkArgs b = a;                        // all segments but the last
    int item = 0;
    for (int k = 0; k < a.seqs.n; ++k) {
      b.seqs.item0[k] = item;
      item += (a.seqs.segs[k] - 1) * a.Hkv;
    }
    b.seqs.item0[a.seqs.n] = item;
    linear_chunk_kernel<D, true><<<item, kThreads, Layout<D>::kSmem, s>>>(tmQ, tmK, tmV, b);
    linear_join_kernel<D><<<dim3(a.Hkv * (D * D / 1024), a.seqs.n), 256, 0, s>>>(a);
  }
  linear_chunk_kernel<D, false><<<a.seqs.item0[a.seqs.n], kThreads, Layout<D>::kSmem, s>>>(tmQ, tmK, tmV, a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t linear_chunk_prepare(int D) { return D == 128 ? prepare<128>() : prepare<64>(); }

cudaError_t launch_linear_chunk(int D, bool split, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                                const LinearChunkArgs& a, cudaStream_t s) {
  return D == 128 ? launch<128>(split, tmQ, tmK, tmV, a, s) : launch<64>(split, tmQ, tmK, tmV, a, s);
}

}  // namespace fk
