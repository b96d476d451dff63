// Linear attention with decays, in chunks of 128 tokens on the 5th-generation tensor cores.
//
// With G_i the sum of the decays' logarithms from a chunk's start through token i, and S the state before the chunk,
//   o_i = scale (exp(G_i) q_i S + sum_(j <= i) exp(G_i - G_j) (q_i k_j) v_j),
//   S'  = exp(G_C) S + sum_j exp(G_C - G_j) k_j v_j^T:
// four matrix products of 128 x 128 x D a chunk and head, six with K' in three parts: 2.0 us of an SM's tensor cores at the measured rate of
// large products, for 128 KB of q, k, v and o (D = 128), 2.9 us of an SM's share of the memory.  All exponents are of sums that are <= 0 where
// decays are.
//
// A CTA takes items (segments of one kv head's chunks, with all query heads that share it) one after the other, without a break
// between them:
//   warp 3        TMA: K and V of a chunk, Q of a chunk and query head, two stages each, 128-byte swizzle
//   warp 1        tcgen05.mma, one elected lane: A = Q K^T, X = Q S, Y = exp(G_i) X + P V, dS = K'^T V
//   warp 2        the chunk's running sums G (log2 domain) and what follows from them alone
//   warp 0        whether V holds values that are not finite
//   warps 4-11    two warpgroups.  K' = exp(G_C - G_j) k_j, transposed by ldmatrix into tensor memory (the A operand of dS), in
//                 three bf16 parts, which is exact (two: 2^-17 of each term, and the state is kept to fp32): 32 tokens at a
//                 time, taking turns, each into its own buffer.  Then P_ij = exp(G_i - G_j) A_ij for j <= i as bf16, 32 columns
//                 at a time, taking turns, over the columns of A that it came from.
//   warps 12-15   the state: thread r keeps row r (channel r of k) in registers, S' = exp(G_C) S + dS, and writes it as bf16 to
//                 shared memory, the B operand of X
//   warps 16-19   o: thread i scales row i of X where it is, rounds row i of Y to bf16 over a tile of Q or V that the products are
//                 done with, and a TMA store takes it from there (straight from registers: 16 bytes of 32 lines at a time)
// P and the S of X are rounded to bf16 (half a step, up to 2^-8 of a term): a product's operands have one type, Q's and V's range
// wants bf16, and o is rounded to bf16 itself (0.0017 of it in the 2-norm, 0.0023 so).  Second parts would double two of the products, and
// S's has no room in shared memory at D = 128.
// Tensor memory columns: A and P 0-127, X and Y 128.., dS 256.., K' 384-479 (two buffers; kLocal: four from 0).
//
// kLocal: the state alone, from zero (what a segment adds), without Q and o.
// Every wait is bounded; when one expires the CTA records it, drains its copies and products, and ends.
//
// What bounds it.  A chunk takes 2.8 us of a CTA by itself (2.3 more for each further query head; kLocal 1.8) and 3.2 with all SMs
// loading: 24 chunks of 144 heads of 128 in 85 us, 5.3 TB/s.  By itself it is a chain: S' (and so X of the next chunk) waits for all
// of dS, that for K', P for A and Y for P; the products are in the order that hides most of it, and the tensor pipe is active 31
// to 43% of the time (two chunks at once would want twice the tensor memory at D = 128).  An item costs 3 us besides (its first tiles, its state
// both ways), a launch 4.5.  One sequence of few heads is therefore split (the host's plan): 4680 tokens of 12 heads in 12
// segments 31 us, unsplit 105; what each segment adds is then formed first, which reads K and V twice.
// Loops over columns are rolled where registers are not indexed: the roles' code together has to stay in the instruction
// cache (unrolled, P of a chunk took 2400 cycles, and 4800 with all SMs fetching).  Roles are told apart by a warp number that comes
// from a shuffle, so that the compiler knows branches by it to be uniform.
#include "fk_linear.h"
#include "fk_tc.h"

#include <algorithm>

namespace fk {
namespace {

constexpr int C = kLinearChunk;
constexpr int kThreads = 640;
// Registers of a thread of each warpgroup: together no more than the launch gives them (raising a count waits for registers
// that others gave back: without an end where there are too few).
constexpr int kRegsStart = 65536 / kThreads / 8 * 8;
constexpr int kRegsIssue = 72, kRegsConvert = 80, kRegsState = 176, kRegsOut = 72;
static_assert(kRegsIssue + 2 * kRegsConvert + kRegsState + kRegsOut <= kThreads / 128 * kRegsStart, "registers of the CTA");
static_assert(kRegsIssue <= kRegsStart && kRegsConvert <= kRegsStart && kRegsOut <= kRegsStart && kRegsState >= kRegsStart, "who gives, who takes");
constexpr uint32_t kColA = 0, kColX = 128, kColS = 256, kColK = 384;   // kLocal: K' from 0

// Many of the roles' steps are a few hundred cycles long, and so are a product's way to a barrier and a warp's way from
// one: what can share a barrier does.
struct Barriers {
  uint64_t k_full[3], k_empty[3], v_full[3], v_empty[3], q_full[2], q_empty[2];
  uint64_t g_full[2], g_empty[2];     // the chunk's sums
  uint64_t odd_full[2], odd_empty[2];
  uint64_t kp_full[4], kp_empty[4];   // K' buffers: written, multiplied
  uint64_t ds_full, ds_empty;         // all of dS is there, is read
  uint64_t a_full;                    // A is there
  uint64_t x_ready, x_full;           // S is written, the Y before it read; X is there
  uint64_t y_ready, y_full;           // P is written, X scaled; Y is there
  uint64_t fin;
  uint32_t tmem_base;
  volatile int abort;
  int odd[2];                         // V of the chunk holds values that are not finite
};

// What follows from the decays of a chunk alone, G in the log2 domain.
struct alignas(16) Sums {
  float g[C];                         // G_j
  float u[C];                         // exp(R - G_j), R the sum at the end of j's 32 tokens; `grow`: exp(G_C - G_j)
  __half rest[C];                     // G_j less g[j]: sums run to 2^15 where states start anew (2^22 in a chunk that grows), and
                                      // fp32 has steps of 2^-9 there
  float w[4];                         // exp(G_C - R) of each 32 tokens; `grow`: 1
  float e;                            // exp(G_C)
  float2 left;                        // kLocal: what the segment leaves of a state by the chunk's end, in two parts
  int grow;                           // some g > 0: the factors could overflow where their product does not
};

template <int D>
struct Layout {
  static constexpr int kTile = C * D * 2;         // bytes of a tile of Q, K or V: D / 64 panels of 128-byte rows
  static constexpr int kOffQ = 4 * kTile;
  static constexpr int kOffS = 6 * kTile;         // S: D / 64 panels of D 128-byte rows
  static constexpr int kOffG = kOffS + D * D * 2;
  static constexpr int kOffBar = kOffG + 2 * (int)sizeof(Sums);
  static constexpr int kUsed = kOffBar + (int)sizeof(Barriers);
  // at least ~116 KB, so that one CTA occupies an SM (its 512 tensor memory columns are then free)
  static constexpr int kSmem = kUsed > 118 * 1024 ? kUsed : 118 * 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory");
};

// 16 lanes x 16 columns of tensor memory from transposed 8 x 8 tiles (ldmatrix): register 2 b + s is lane 8 s + t / 4, column
// 4 b + t % 4 of thread t
__device__ __forceinline__ void tmem_st_tiles(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               :: "r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t addr, uint32_t* v) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void fence_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// Warp-uniform bounded wait for the phase of parity `parity`; false when the CTA is aborting or the limit expired (which
// starts the abort; the CTA records it at its end).  As short as it gets: there are thirty of them, and in C++ each took
// 670 bytes of the instruction cache.
__device__ __forceinline__ bool wait(uint64_t* b, uint32_t parity, Barriers* bar) {
  uint32_t done;
  asm volatile(
      "{\n .reg .pred p, q;\n .reg .b32 t0, t;\n"
      " mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      " @p bra DONE%=;\n"
      " mov.u32 t0, %%globaltimer_lo;\n"
      "AGAIN%=:\n"
      " mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 0x4E20;\n"
      " @p bra DONE%=;\n"
      " mov.u32 t, %%globaltimer_lo;\n"
      " sub.u32 t, t, t0;\n"
      " setp.gt.u32 q, t, %4;\n"
      " @q st.volatile.shared.u32 [%3], 1;\n"
      " ld.volatile.shared.u32 t, [%3];\n"
      " setp.eq.u32 q, t, 0;\n"
      " @q bra AGAIN%=;\n"
      "DONE%=:\n"
      " selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(done)
      : "r"(su32(b)), "r"(parity & 1), "r"(su32(const_cast<const int*>(&bar->abort))), "n"((uint32_t)kWaitLimitNs) : "memory");
  return __all_sync(0xffffffffu, done);
}
// The same for what is to be over before the CTA ends, aborting or not.
__device__ __forceinline__ void drain(uint64_t* b, uint32_t parity, Barriers* bar) {
  const uint64_t t0 = now_ns();
#pragma unroll 1
  while (!mbar_test(b, parity))
    if (now_ns() - t0 > kWaitLimitNs) {
      bar->abort = 1;
      break;
    }
}
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(N)); }
__device__ __forceinline__ float2 fmul2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 ra, rb, rd;\n mov.b64 ra, {%2, %3};\n mov.b64 rb, {%4, %5};\n"
      " mul.rn.f32x2 rd, ra, rb;\n mov.b64 {%0, %1}, rd;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// 0 x + z of bf16 pairs
__device__ __forceinline__ uint32_t zero_times(uint32_t x, uint32_t z) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(x), "r"(0u), "r"(z));
  return d;
}
// not 0 where a bf16 pair holds an infinity or NaN: an exponent of ones
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
// x less a bf16 pair (exact where the pair is x rounded)
__device__ __forceinline__ float2 less(float2 x, uint32_t y) {
  float2 d;
  asm("{\n .reg .b16 l, h, m;\n mov.b32 {l, h}, %4;\n mov.b16 m, 0xBF80;\n fma.rn.f32.bf16 %0, l, m, %2;\n fma.rn.f32.bf16 %1, h, m, %3;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(x.x), "f"(x.y), "r"(y));
  return d;
}
__device__ __forceinline__ float2 of_f16(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// a whole number of 2^-40 (to 2^-25), less what fp32 holds of it already
__device__ __forceinline__ float of_fixed(int64_t x, float held = 0.0f) {
  return fmaf((float)(uint32_t)(x >> 8), 0x1p-32f, (float)(int32_t)(x >> 40) - held);
}
// Factors whose error is made up for.  (One by itself is off by up to 2^-23, at every chunk the same way where the decay is the same,
// and slow decays take hundreds of them; what decays faster is forgotten in four.)
__device__ __forceinline__ bool near_one(float e) { return e >= 0.78f && e <= 1.28f; }
// 2^x less such a factor, its fp32 rounding or nearly that.  Of exp(y) - 1, |y| < 1/4; the series' next term is 4^-8 / 8! < 2^-31.
__device__ __forceinline__ float exp_rest(int64_t x, float held) {
  const float y = (float)x * (0.69314718055994531f * 0x1p-40f);
  float t = 1.0f / 5040;
  for (const float c : {1.0f / 720, 1.0f / 120, 1.0f / 24, 1.0f / 6, 0.5f}) t = fmaf(t, y, c);
  return fmaf(y * y, t, y) - (held - 1.0f);
}

// A segment of one kv head of a sequence.
struct Item {
  int s, seg, segs, kvh;
  int nc, tokens;                     // chunks, at least one, and tokens
  int64_t tok0, place;
};
__device__ __forceinline__ Item item_of(const LinearChunkArgs& a, int i) {
  Item t;
  int lo = 0, hi = a.seqs.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.seqs.item0[mid] <= i) lo = mid;
    else hi = mid - 1;
  }
  t.s = lo;
  t.segs = a.seqs.segs[lo];
  i -= a.seqs.item0[lo];
  t.seg = (int)((unsigned)i / (unsigned)a.Hkv);
  t.kvh = i - t.seg * a.Hkv;
  // per chunks to a segment, one more to the first of them
  const int len = a.seqs.len[lo], per = a.seqs.per[lo], more = (int)((unsigned)(len + C - 1) / C) - per * t.segs;
  const int c0 = t.seg * per + min(t.seg, more);
  t.nc = per + (t.seg < more);
  t.tok0 = (int64_t)a.seqs.tok0[lo] + (int64_t)c0 * C;
  t.tokens = min(len - c0 * C, t.nc * C);
  t.place = (int64_t)a.seqs.place0[lo] + t.kvh * t.segs + t.seg;
  return t;
}
// The items of a CTA: one of each round of gridDim.x, forth and back, so that the longest of one round meets the shortest of the
// next (they come longest first).
__device__ __forceinline__ int item_at(int round) {
  const int g = gridDim.x, b = blockIdx.x;
  return round * g + (round & 1 ? g - 1 - b : b);
}

// A warp's 32 rows of D floats, row r of lane r, from and to rows that lie one after the other in memory: 128 bytes of 4 rows
// at a time there, turned through 4 KB of shared memory.  (With each lane at its own row an access touches 32 lines: 4 us for
// both ways of a state of 64 KB.)
template <int D>
__device__ __forceinline__ void turn(float* st, uint8_t* tile, int lane, bool to_rows) {
  float4* v = reinterpret_cast<float4*>(st);
#pragma unroll
  for (int q = 0; q < D / 32; ++q) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = to_rows ? 4 * i + (lane >> 3) : lane, c = to_rows ? lane & 7 : i;
      *reinterpret_cast<float4*>(tile + r * 128 + ((c ^ (r & 7)) << 4)) = v[8 * q + i];
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = to_rows ? lane : 4 * i + (lane >> 3), c = to_rows ? i : lane & 7;
      v[8 * q + i] = *reinterpret_cast<const float4*>(tile + r * 128 + ((c ^ (r & 7)) << 4));
    }
  }
  __syncwarp();
}

template <int D, bool kLocal>
__global__ void __launch_bounds__(kThreads, 1)
linear_chunk_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmO,
                    const __grid_constant__ LinearChunkArgs a) {
  using Lay = Layout<D>;
  constexpr int kStages = kLocal ? 3 : 2;         // of K and V: tiles 2 b and 2 b + 1; Q: tiles 4 and 5 (kLocal: the third stage)
  constexpr int kPanels = D / 64, kBufs = kLocal ? 4 : 2;    // K' buffers, a chunk's quarters in turn
  constexpr uint32_t kColKp = kLocal ? 0 : kColK;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* sK = smem;                             // (2 kTile from stage to stage)
  uint8_t* sV = smem + Lay::kTile;
  uint8_t* sQ = smem + Lay::kOffQ;
  uint8_t* sS = smem + Lay::kOffS;
  Sums* sums = reinterpret_cast<Sums*>(smem + Lay::kOffG);   // of two chunks
  Barriers* bar = reinterpret_cast<Barriers*>(smem + Lay::kOffBar);
  // (the compiler takes what a shuffle or a vote gives for the same in all lanes: branches by it stay plain branches)
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  const int G = kLocal ? 1 : a.G;
  // Every role takes the CTA's items one after the other, and their chunks: chunk c, and c G + g its products with query head g, count
  // on from item to item, and so do the barriers' phases; nothing waits for an item to end.
  const Item first = item_of(a, blockIdx.x);

  // The loading warp makes the barriers and asks for the first tiles before the CTA meets (which takes 1700 cycles: the
  // allocation of tensor memory).
  auto load = [&](const CUtensorMap* map, uint8_t* dst, uint64_t* b, int head, int64_t tok) {   // one lane
    mbar_expect_tx(b, Lay::kTile);
    for (int p = 0; p < kPanels; ++p) tma_load_2d(dst + p * (C * 128), map, b, head * D + p * 64, (int)tok);
  };
  if (warp == 3 && lane == 0) {
    for (const CUtensorMap* map : {&tmK, &tmV, &tmQ, &tmO}) asm volatile("prefetch.tensormap [%0];" :: "l"(map) : "memory");
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bar->q_full[i], 1);
      mbar_init(&bar->q_empty[i], 4);
      mbar_init(&bar->g_full[i], 1);
      mbar_init(&bar->g_empty[i], kLocal ? 12 : 16);
      mbar_init(&bar->odd_full[i], 1);
      mbar_init(&bar->odd_empty[i], 4);
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&bar->k_full[i], 1);
      mbar_init(&bar->k_empty[i], kLocal ? 8 : 9);           // the converting warps, and Q K^T
      mbar_init(&bar->v_full[i], 1);
      mbar_init(&bar->v_empty[i], kLocal ? 1 : 5);           // the products; the check, and O's rows on their way
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&bar->kp_full[i], 4);
      mbar_init(&bar->kp_empty[i], 1);
    }
    mbar_init(&bar->ds_full, 1);
    mbar_init(&bar->ds_empty, 4);
    mbar_init(&bar->a_full, 1);
    mbar_init(&bar->x_ready, 8);
    mbar_init(&bar->x_full, 1);
    mbar_init(&bar->y_ready, 12);
    mbar_init(&bar->y_full, 1);
    mbar_init(&bar->fin, 1);
    bar->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    load(&tmK, sK, &bar->k_full[0], first.kvh, first.tok0);
    if (!kLocal) load(&tmQ, sQ, &bar->q_full[0], first.kvh * G, first.tok0);
    load(&tmV, sV, &bar->v_full[0], first.kvh, first.tok0);
    // (the join's blocks, or those of sequences of few tokens, may take the SMs that this launch leaves idle)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }
  if (warp == 1) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 :: "r"(su32(&bar->tmem_base)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // decays of a chunk (warp 2, lane's tokens 4 lane .. + 3), three chunks ahead: one chunk's time is less than a load takes
  float ahead[3][4];
  auto fetch = [&](const Item& it, int n, float* x) {
    const float* decay = a.decay + it.tok0 * a.dstride + it.kvh;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = n * C + 4 * lane + i;
      x[i] = t < it.tokens ? __ldg(decay + (int64_t)t * a.dstride) : 0.0f;
    }
  };
  if (warp == 2) {
#pragma unroll
    for (int i = 0; i < 3; ++i) fetch(first, i, ahead[i]);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // All of the tensor memory is this CTA's, so that it starts at 0: the products then take constants (with the number read
  // from shared memory an instruction took 130 cycles to issue).
  if (bar->tmem_base != 0) bar->abort = 1;
  constexpr uint32_t tmem = 0;
  const int wq = warp & 3, row = wq * 32 + lane;             // tensor memory lane of a thread of warps 4-19
  const uint32_t lanes = tmem + ((uint32_t)(wq * 32) << 16);
  auto wait_for = [&](uint64_t* b, uint32_t parity) { return wait(b, parity, bar); };
  auto arrive = [&](uint64_t* b) {                           // of a warp
    __syncwarp();
    if (lane == 0) mbar_arrive(b);
  };

  if (warp < 4) {
    fewer_registers<kRegsIssue>();
    if (warp == 3) {
      // ------------------------------------------------------------------ TMA
      bool ok = true;
      int ik = 0, iv = 0, iq = kLocal ? -1 : 0;              // last tiles issued
      int base = 0;                                          // chunks of the items before
#pragma unroll 1
      for (int round = 0; ok && item_at(round) < a.items; ++round) {
        const Item it = item_of(a, item_at(round));
#pragma unroll 1
        for (int n = 0; n < it.nc && ok; ++n) {
          const int c = base + n, b = c % kStages, u = c / kStages;
          const int64_t tok = it.tok0 + n * C;
          if (u > 0 && !(ok = wait_for(&bar->k_empty[b], u - 1))) break;
          if (lane == 0 && c > 0) load(&tmK, sK + b * (2 * Lay::kTile), &bar->k_full[b], it.kvh, tok);
          __syncwarp();
          ik = c;
#pragma unroll 1
          for (int g = 0; g < (kLocal ? 1 : G); ++g) {
            if (!kLocal) {
              const int m = c * G + g, qb = m & 1, qu = m >> 1;
              if (qu > 0 && !(ok = wait_for(&bar->q_empty[qb], qu - 1))) break;
              if (lane == 0 && m > 0) load(&tmQ, sQ + qb * Lay::kTile, &bar->q_full[qb], it.kvh * G + g, tok);
              __syncwarp();
              iq = m;
            }
            if (g > 0) continue;
            if (u > 0 && !(ok = wait_for(&bar->v_empty[b], u - 1))) break;
            if (lane == 0 && c > 0) load(&tmV, sV + b * (2 * Lay::kTile), &bar->v_full[b], it.kvh, tok);
            __syncwarp();
            iv = c;
          }
        }
        base += it.nc;
      }
      if (!ok) {                                             // what was issued lands before the CTA ends
#pragma unroll 1
        for (int i = 0; i < kStages; ++i) {
          if (ik >= i) drain(&bar->k_full[(ik - i) % kStages], ((ik - i) / kStages) & 1, bar);
          if (iv >= i) drain(&bar->v_full[(iv - i) % kStages], ((iv - i) / kStages) & 1, bar);
          if (iq >= i && i < 2) drain(&bar->q_full[(iq - i) & 1], ((iq - i) >> 1) & 1, bar);
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      // ------------------------------------------------------------------ MMA issuer
      // Operations of one thread complete in issue order.  Of a chunk (one query head): the first half of dS, X, the other half,
      // Y, the next chunk's A.  While the last two run, S' is formed from dS and the next K' are made; P and X's scaling
      // are done while the second half of dS runs.  (X, dS, Y, A one after the other in any other order leave the tensor cores
      // waiting for S' or for K'.)
      constexpr uint32_t kIdA = idesc_bf16(C, C, 0), kIdD = idesc_bf16(C, D, 1), kTile16 = Lay::kTile >> 4;
      const uint64_t dQ = sdesc(su32(sQ), 16, 1024), dK = sdesc(su32(sK), 16, 1024);
      const uint64_t dV = sdesc(su32(sV), 16384, 1024), dS = sdesc(su32(sS), 16384, 1024);
      // K = 16 steps of an operand: rows of 128-byte panels (channels along K), or 16 rows of panels (tokens or channels of k)
      auto along = [](int kk) { return (uint32_t)((kk >> 2) * 1024 + (kk & 3) * 2); };
      auto q_k = [&](int m, int n) {                         // A = Q K^T
        const uint64_t x = dQ + (m & 1) * kTile16, y = dK + (n & 1) * (2 * kTile16);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) umma(kColA, x + along(kk), y + along(kk), kIdA, kk > 0 ? 1u : 0u);
        umma_commit(&bar->a_full);
        if (G == 1 || m % G == G - 1) umma_commit(&bar->k_empty[n & 1]);
      };
      auto half_ds = [&](int n, int q0) {                    // dS += K'^T V of 64 tokens
#pragma unroll 1
        for (int q = q0; q < q0 + 2; ++q) {
          if (!wait_for(&bar->kp_full[q % kBufs], n * (4 / kBufs) + q / kBufs)) return false;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t y = dV + (uint32_t)(n % kStages * (2 * kTile16) + q * 256);
            const uint32_t kp = kColKp + (q % kBufs) * 48;
#pragma unroll
            for (int i = 0; i < 6; ++i)                      // part, 16 tokens
              umma_ts(kColS, kp + i * 8, y + (i & 1) * 128, kIdD, q + i > 0 ? 1u : 0u);
            umma_commit(&bar->kp_empty[q % kBufs]);
            if (q == 3) umma_commit(&bar->ds_full);
            if (q == 3 && kLocal) umma_commit(&bar->v_empty[n % kStages]);
          }
          __syncwarp();
        }
        return true;
      };
      int chunks = 0;                                        // of all items
#pragma unroll 1
      for (int round = 0; item_at(round) < a.items; ++round) chunks += item_of(a, item_at(round)).nc;
      bool ok = true;
      if (!kLocal && (ok = wait_for(&bar->k_full[0], 0) && wait_for(&bar->q_full[0], 0))) {
        tc_fence_after();
        if (elect_one()) q_k(0, 0);
        __syncwarp();
      }
#pragma unroll 1
      for (int n = 0; n < chunks && ok; ++n) {
        if (!(ok = wait_for(&bar->v_full[n % kStages], n / kStages))) break;
        if (n > 0 && !(ok = wait_for(&bar->ds_empty, n - 1))) break;
        if (!(ok = half_ds(n, 0))) break;
        if (kLocal) ok = half_ds(n, 2);
#pragma unroll 1
        for (int g = 0; g < G && !kLocal; ++g) {
          const int m = n * G + g;
          if (!(ok = wait_for(&bar->x_ready, m))) break;
          tc_fence_after();
          if (elect_one()) {                                 // X = Q S
            const uint64_t x = dQ + (m & 1) * kTile16;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) umma(kColX, x + along(kk), dS + kk * 128, kIdD, kk > 0 ? 1u : 0u);
            umma_commit(&bar->x_full);
          }
          __syncwarp();
          if (g == 0 && !(ok = half_ds(n, 2))) break;
          if (!(ok = wait_for(&bar->y_ready, m))) break;
          tc_fence_after();
          if (elect_one()) {                                 // Y = exp(G_i) X + P V
            const uint64_t y = dV + (uint32_t)((n & 1) * (2 * kTile16));
#pragma unroll
            for (int kk = 0; kk < C / 16; ++kk) umma_ts(kColX, kColA + (kk >> 1) * 32 + (kk & 1) * 8, y + kk * 128, kIdD, 1u);
            umma_commit(&bar->y_full);
          }
          __syncwarp();
          if (m + 1 < chunks * G) {                          // the next A
            const int n1 = g + 1 < G ? n : n + 1;
            if (n1 > n && !(ok = wait_for(&bar->k_full[n1 & 1], n1 >> 1))) break;
            if (!(ok = wait_for(&bar->q_full[(m + 1) & 1], (m + 1) >> 1))) break;
            tc_fence_after();
            if (elect_one()) q_k(m + 1, n1);
            __syncwarp();
          }
        }
      }
      if (elect_one()) umma_commit(&bar->fin);               // completes once every product above is done
      drain(&bar->fin, 0, bar);
      __syncwarp();
    } else if (warp == 2) {
      // ------------------------------------------------------------------ running sums of a chunk
      int base = 0;
      bool ok = true;
#pragma unroll 1
      for (int round = 0; ok && item_at(round) < a.items; ++round) {
      const Item it = item_of(a, item_at(round));
      if (round > 0) {
#pragma unroll
        for (int i = 0; i < 3; ++i) fetch(it, i, ahead[i]);
      }
      int64_t total = 0;                                     // of the segment's chunks
      bool total_lost = false;
      float owed = 0.0f;                                     // what their factors so far, as rounded, lack of their product
#pragma unroll 1
      for (int n = 0; n < it.nc; ++n) {
        const int c = base + n, b = c & 1, u = c >> 1;
        // whole numbers of 2^-40: sums and their differences are exact however far they run (of g log2 e itself, 2^-41 a token, and its
        // product in fp32 2^-24 of it), and P's from two parts of them to 2^-20 (2^-14 in a
        // chunk that grows); where exp(g) is not a number, nothing is from that token on
        int64_t sum[4];
        bool grows = false;
        int lost = C;                                        // first token whose exp(g) is not a number
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          grows |= !(ahead[0][i] <= 0.0f);
          if (!(ahead[0][i] <= kMostGrowth)) lost = min(lost, 4 * lane + i);
        }
        const bool grow = __any_sync(0xffffffffu, grows);
        const float least = grow ? kLeastAmongGrowth : kLeastDecay;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t z = __float2ll_rn(fminf(fmaxf(ahead[0][i], least), kMostGrowth) * (1.4426950408889634f * 0x1p40f));
          sum[i] = i == 0 ? z : sum[i - 1] + z;
        }
        int64_t all = sum[3];
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
          const int64_t z = __shfl_up_sync(0xffffffffu, all, o);
          if (lane >= o) all += z;
        }
        const int64_t before = all - sum[3], end = __shfl_sync(0xffffffffu, all, 31);
        lost = __reduce_min_sync(0xffffffffu, lost);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ahead[0][i] = ahead[1][i];
          ahead[1][i] = ahead[2][i];
        }
        fetch(it, n + 3, ahead[2]);
        // the sum at the end of this lane's 32 tokens, unless the chunk grows
        const int64_t r = __shfl_sync(0xffffffffu, all, lane | 7), from = grow ? end : r;
        const float nan = __int_as_float(0x7FFFFFFF);
        float gg[4], rest[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t x = before + sum[i];
          gg[i] = of_fixed(x);
          rest[i] = of_fixed(x, gg[i]);
          if (4 * lane + i >= lost) gg[i] = nan;
          v[i] = lost < C ? nan : exp2f(of_fixed(from - x));
        }
        const float w = grow ? 1.0f : exp2f(of_fixed(end - r));
        float e = exp2f(of_fixed(end));
        e = lost < C ? nan : fmaf(e, owed, e);
        float2 left = make_float2(1.0f, 0.0f);
        if (kLocal) {
          // (what passes 2^21 stays there: it is 0 or infinite)
          constexpr int64_t kMost = (int64_t)1 << 61;
          total = min(max(total + end, -kMost), kMost);
          total_lost |= lost < C;
          left.x = total_lost ? nan : exp2f(of_fixed(total));
          if (near_one(left.x)) left.y = exp_rest(total, left.x);
        }
        // (all but the stores is done by now: the chunk may be waited for)
        if (u > 0 && !(ok = wait_for(&bar->g_empty[b], u - 1))) break;
        Sums& out = sums[b];
        *reinterpret_cast<float4*>(out.g + 4 * lane) = make_float4(gg[0], gg[1], gg[2], gg[3]);
        *reinterpret_cast<float4*>(out.u + 4 * lane) = make_float4(v[0], v[1], v[2], v[3]);
        if (!kLocal) *reinterpret_cast<uint2*>(out.rest + 4 * lane) = make_uint2(pack_f16(rest[0], rest[1]), pack_f16(rest[2], rest[3]));
        if ((lane & 7) == 7) out.w[lane >> 3] = w;
        if (lane == 0) {
          out.e = e;
          if (kLocal) out.left = left;
          out.grow = grow;
        }
        arrive(&bar->g_full[b]);
        owed = near_one(e) ? owed + exp_rest(end, e) : 0.0f;
      }
      base += it.nc;
      }
    } else if (!kLocal) {
      // ------------------------------------------------------------------ is V finite
      int base = 0;
      bool ok = true;
#pragma unroll 1
      for (int round = 0; ok && item_at(round) < a.items; ++round) {
      const Item it = item_of(a, item_at(round));
#pragma unroll 1
      for (int n = 0; n < it.nc; ++n) {
        const int c = base + n, b = c & 1, u = c >> 1, valid = min(C, it.tokens - n * C);
        if (!(ok = wait_for(&bar->v_full[b], u))) break;
        // 0 times a value is NaN where it is not finite; 8 runs of 16 bytes to a row of a panel
        uint32_t z[4] = {0, 0, 0, 0};
#pragma unroll 4
        for (int i = lane; i < Lay::kTile / 16; i += 32) {
          uint4 v = *reinterpret_cast<const uint4*>(sV + b * (2 * Lay::kTile) + i * 16);
          if (valid < C && (i >> 3) % C >= valid) v = make_uint4(0, 0, 0, 0);
          z[0] = zero_times(v.x, z[0]);
          z[1] = zero_times(v.y, z[1]);
          z[2] = zero_times(v.z, z[2]);
          z[3] = zero_times(v.w, z[3]);
        }
        if (u > 0 && !(ok = wait_for(&bar->odd_empty[b], u - 1))) break;
        const bool odd = __any_sync(0xffffffffu, ((z[0] | z[1] | z[2] | z[3]) & 0x7FFF7FFFu) != 0);
        if (lane == 0) bar->odd[b] = (int)odd;
        arrive(&bar->odd_full[b]);
        arrive(&bar->v_empty[b]);
      }
      base += it.nc;
      }
    }
  } else if (warp < 12) {
    fewer_registers<kRegsConvert>();
    // ------------------------------------------------------------------ K' and P
    const int w2 = (warp >> 2) - 1;                          // which of the two warpgroups
    const bool mine = 32 * wq < D;                           // D = 64: lanes 64-127 of dS are not used
    bool ok = true;
    int base = 0;
#pragma unroll 1
    for (int round = 0; ok && item_at(round) < a.items; ++round) {
    const Item it = item_of(a, item_at(round));
#pragma unroll 1
    for (int n = 0; n < it.nc && ok; ++n) {
      const int c = base + n, b = c & 1, u = c >> 1, valid = min(C, it.tokens - n * C);
      const Sums& sm = sums[b];
      const int bk = c % kStages;                            // stage of K and V
      if (!(ok = wait_for(&bar->k_full[bk], c / kStages) && wait_for(&bar->g_full[b], u))) break;
      if (valid < C) {                                       // rows of others: zeros for the products with V
        if (!(ok = wait_for(&bar->v_full[bk], c / kStages))) break;
        const int p = wq >> 1, r = 64 * (wq & 1) + 32 * w2 + lane;   // panel, token of this warpgroup's
        if (r >= valid && p < kPanels) {
#pragma unroll 1
          for (int i = 0; i < 8; ++i)
            *reinterpret_cast<uint4*>(sV + bk * (2 * Lay::kTile) + p * (C * 128) + r * 128 + i * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_to_async();
      }
      const float gi = kLocal ? 0.0f : sm.g[row], ri = kLocal ? 0.0f : __half2float(sm.rest[row]) + a.log2_scale;
      const bool grow = !kLocal && __any_sync(0xffffffffu, sm.grow);
      // K' of this warpgroup's first quarter, P of the first query head while that is multiplied, K' of the other quarter, P of
      // further query heads
#pragma unroll 1
      for (int step = 0; step < (kLocal ? 2 : G + 2) && ok; ++step) {
        if (step == 0 || step == (kLocal ? 1 : 2)) {
          const int q = step == 0 ? w2 : w2 + 2, buf = q % kBufs, use = c * (4 / kBufs) + q / kBufs;
          if (use > 0 && !(ok = wait_for(&bar->kp_empty[buf], use - 1))) break;
          tc_fence_after();
          if (mine) {
            // channels 32 wq .. + 31 of this warp, 16 at a time
            const int t0 = 32 * q + 2 * (lane & 3);          // first token of this thread's pairs, 8 apart
            float2 w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = fmul2(*reinterpret_cast<const float2*>(sm.u + t0 + 8 * k), make_float2(sm.w[q], sm.w[q]));
            const int r = lane & 7, mat = lane >> 3;
#pragma unroll 1
            for (int hf = 0; hf < 2; ++hf) {
              const int ch = 32 * wq + 16 * hf + (mat & 1) * 8;  // channel of the row that this lane gives ldmatrix
              const uint32_t at = su32(sK) + (uint32_t)(bk * (2 * Lay::kTile) + (ch >> 6) * (C * 128) + (32 * q + (mat >> 1) * 8 + r) * 128 +
                                                        ((((ch & 63) >> 3) ^ r) << 4));
              uint32_t x[8], hi[8], mid[8], lo[8];
              ldmatrix4t(at, x);
              ldmatrix4t(at + 16 * 128, x + 4);
              if (valid < C) {                               // (tokens of others: any values)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  const int j = t0 + 8 * (k >> 1);
                  x[k] = j + 1 < valid ? x[k] : j < valid ? x[k] & 0xFFFFu : 0u;
                }
              }
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                float2 p = fmul2(make_float2(low(x[k]), high(x[k])), w[k >> 1]);
                hi[k] = pack_bf16(p.x, p.y);
                p = less(p, hi[k]);
                mid[k] = pack_bf16(p.x, p.y);
                p = less(p, mid[k]);
                lo[k] = pack_bf16(p.x, p.y);
              }
              const uint32_t to = lanes + kColKp + buf * 48 + ((uint32_t)(16 * hf) << 16);
              tmem_st_tiles(to, hi);
              tmem_st_tiles(to + 16, mid);
              tmem_st_tiles(to + 32, lo);
            }
            tmem_wait_st();
            tc_fence_before();
          }
          arrive(&bar->kp_full[buf]);
          if (step > 0) arrive(&bar->k_empty[bk]);
          continue;
        }
        if (!(ok = wait_for(&bar->a_full, c * G + (step < 2 ? 0 : step - 2)))) break;
        tc_fence_after();
        // below the diagonal A f u_j with f of the row, on it A exp(G_i - G_j), scaled
#pragma unroll 1
        for (int q = w2; q < 4; q += 2) {
          uint32_t x[32];
          if (q > wq) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = 0;
          } else {
            FK_TMEM_LD32(lanes + kColA + 32 * q, x);
            if (q == wq || grow) {
              const float4* y = reinterpret_cast<const float4*>(sm.g + 32 * q);
              const uint2* z = reinterpret_cast<const uint2*>(sm.rest + 32 * q);
              FK_TMEM_WAIT_LD32(x);
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float4 v = y[i];
                const uint2 w = z[i];
                // (the difference of the fp32 parts is exact where it is small)
                const float2 minus = make_float2(-1.0f, -1.0f), g2 = make_float2(gi, gi), r2 = make_float2(ri, ri);
                const float2 d0 = fadd2(ffma2(make_float2(v.x, v.y), minus, g2), ffma2(of_f16(w.x), minus, r2));
                const float2 d1 = fadd2(ffma2(make_float2(v.z, v.w), minus, g2), ffma2(of_f16(w.y), minus, r2));
                const float vv[4] = {d0.x, d0.y, d1.x, d1.y};
                float e[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                  e[c] = __uint_as_float(x[4 * i + c]) * fast_exp2(vv[c]);
                  if (q == wq && 4 * i + c > lane) e[c] = 0.0f;
                }
                x[2 * i] = pack_bf16(e[0], e[1]);
                x[2 * i + 1] = pack_bf16(e[2], e[3]);
              }
            } else {
              const float4* y = reinterpret_cast<const float4*>(sm.u + 32 * q);
              const float f1 = fast_exp2((gi - sm.g[32 * q + 31]) + (ri - __half2float(sm.rest[32 * q + 31])));
              const float2 f = make_float2(f1, f1);
              FK_TMEM_WAIT_LD32(x);
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float4 v = y[i];
                const float2 s0 = fmul2(fmul2(make_float2(__uint_as_float(x[4 * i]), __uint_as_float(x[4 * i + 1])), make_float2(v.x, v.y)), f);
                const float2 s1 = fmul2(fmul2(make_float2(__uint_as_float(x[4 * i + 2]), __uint_as_float(x[4 * i + 3])), make_float2(v.z, v.w)), f);
                x[2 * i] = pack_bf16(s0.x, s0.y);
                x[2 * i + 1] = pack_bf16(s1.x, s1.y);
              }
            }
          }
          FK_TMEM_ST16(lanes + kColA + 32 * q, x);
        }
        tmem_wait_st();
        tc_fence_before();
        arrive(&bar->y_ready);
      }
      if (ok) arrive(&bar->g_empty[b]);
    }
    base += it.nc;
    }
  } else if (warp < 16) {
    more_registers<kRegsState>();
    // ------------------------------------------------------------------ the state
    const bool mine = 32 * wq < D;
    const int at = (32 * wq + (lane >> 3)) * D + (lane & 7) * 4;   // of a state, in memory: rows 4 i + lane / 8 of the warp's
    // Where segments are joined, this kernel starts while the join still runs: its states alone come from there.
    if (!kLocal) asm volatile("griddepcontrol.wait;" ::: "memory");
    bool ok = true;
    int base = 0;
#pragma unroll 1
    for (int round = 0; ok && item_at(round) < a.items; ++round) {
      const Item it = item_of(a, item_at(round));
      auto from = [&](const Item& t) {
        return (t.segs > 1 ? a.place + t.place * (D * D) : a.state + ((int64_t)a.seqs.slot[t.s] * a.Hkv + t.kvh) * (D * D)) + at;
      };
      alignas(16) float st[D];
      float2 left = make_float2(1.0f, 0.0f);                 // what the segment leaves of a state
      if (kLocal || !mine) {
#pragma unroll
        for (int i = 0; i < D; ++i) st[i] = 0.0f;
      } else {
        const float* x = from(it);
#pragma unroll
        for (int i = 0; i < D / 4; ++i) {                    // 4 rows of 32 columns at a time
          const float4 v = *reinterpret_cast<const float4*>(x + (i >> 3) * 32 + (i & 7) * (4 * D));
          st[4 * i] = v.x, st[4 * i + 1] = v.y, st[4 * i + 2] = v.z, st[4 * i + 3] = v.w;
        }
        turn<D>(st, sS + wq * 4096, lane, true);             // (S's place: no X is on its way)
        if (item_at(round + 1) < a.items) {                  // the next item's state on its way to L2
          const float* y = from(item_of(a, item_at(round + 1)));
#pragma unroll
          for (int i = 0; i < D / 4; ++i)
            if ((lane & 7) == 0) asm volatile("prefetch.global.L2 [%0];" :: "l"(y + (i >> 3) * 32 + (i & 7) * (4 * D)));
        }
      }
      // State n is formed from dS of chunk n - 1 and written, 32 columns at a time.
#pragma unroll 1
      for (int n = 0; n <= it.nc; ++n) {
        const int c = base + n - 1;
        float e = 1.0f;
        if (n > 0) {
          if (!(ok = wait_for(&bar->g_full[c & 1], c >> 1))) break;
          e = sums[c & 1].e;
          if (kLocal && n == it.nc) left = sums[c & 1].left;
          arrive(&bar->g_empty[c & 1]);
          // every X of the chunk (each phase is seen): S's place is free, and further query heads' X may follow
#pragma unroll 1
          for (int g = 0; g < G && !kLocal && ok; ++g) {
            if (g > 0) arrive(&bar->x_ready);
            ok = wait_for(&bar->x_full, c * G + g);
          }
          if (!ok || !(ok = wait_for(&bar->ds_full, c))) break;
          tc_fence_after();
        }
        if (mine) {
#pragma unroll
          for (int q = 0; q < D / 32; ++q) {
            if (n > 0) {
              uint32_t x[32];
              FK_TMEM_LD32(lanes + kColS + 32 * q, x);
              FK_TMEM_WAIT_LD32(x);
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const float2 y = ffma2(make_float2(st[32 * q + i], st[32 * q + i + 1]), make_float2(e, e),
                                       make_float2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])));
                st[32 * q + i] = y.x;
                st[32 * q + i + 1] = y.y;
              }
            }
            if (!kLocal && n < it.nc) {
#pragma unroll
              for (int i = 4 * q; i < 4 * q + 4; ++i) {
                const uint4 v = make_uint4(pack_bf16(st[8 * i], st[8 * i + 1]), pack_bf16(st[8 * i + 2], st[8 * i + 3]),
                                           pack_bf16(st[8 * i + 4], st[8 * i + 5]), pack_bf16(st[8 * i + 6], st[8 * i + 7]));
                *reinterpret_cast<uint4*>(sS + (i >> 3) * (D * 128) + row * 128 + (((i & 7) ^ (row & 7)) << 4)) = v;
              }
            }
          }
        }
        if (n > 0) {
          tc_fence_before();
          arrive(&bar->ds_empty);
        }
        if (!kLocal && n < it.nc) {
          fence_to_async();
          arrive(&bar->x_ready);
        }
      }
      float* to = nullptr;
      if (kLocal) to = a.place + (it.place + 1) * (D * D);
      else if (a.state_new && it.seg == it.segs - 1)
        to = a.state_new + ((int64_t)(a.to_out ? a.seqs.out[it.s] : a.seqs.slot[it.s]) * a.Hkv + it.kvh) * (D * D);
      if (ok && to && mine) {
        turn<D>(st, sS + wq * 4096, lane, false);
#pragma unroll
        for (int i = 0; i < D / 4; ++i)
          *reinterpret_cast<float4*>(to + at + (i >> 3) * 32 + (i & 7) * (4 * D)) = make_float4(st[4 * i], st[4 * i + 1], st[4 * i + 2], st[4 * i + 3]);
        if (kLocal && row == 0) a.place_decay[it.place + 1] = left;
      }
      base += it.nc;
    }
  } else {
    fewer_registers<kRegsOut>();
    // ------------------------------------------------------------------ o
    bool ok = !kLocal, any_odd = false;
    if (!kLocal) arrive(&bar->x_ready);                      // no Y before the first X
    int base = 0;
#pragma unroll 1
    for (int round = 0; ok && item_at(round) < a.items; ++round) {
    const Item it = item_of(a, item_at(round));
#pragma unroll 1
    for (int n = 0; n < it.nc && ok; ++n) {
      const int c = base + n, b = c & 1, u = c >> 1, t = n * C + row;
      if (!(ok = wait_for(&bar->g_full[b], u) && wait_for(&bar->odd_full[b], u))) break;
      const float e = exp2f(sums[b].g[row] + (__half2float(sums[b].rest[row]) + a.log2_scale));
      const bool odd = __any_sync(0xffffffffu, bar->odd[b]);
      for (int g = 0; g < G; ++g) {
        const int m = c * G + g, head = it.kvh * G + g;
        bf16* to = a.O + (it.tok0 + t) * a.ostride + (int64_t)head * D;
        if (!(ok = wait_for(&bar->x_full, m))) break;
        tc_fence_after();
        // O goes out from the place of a tile that all products are done with: Q of this query head, or V after the last one (Q can
        // then be loaded anew by now: the next but one is wanted soon)
        const bool last = g == G - 1;
        if (last) arrive(&bar->q_empty[m & 1]);
        if (!odd) {
#pragma unroll 1
          for (int q = 0; q < D / 32; ++q) {
            uint32_t x[32];
            FK_TMEM_LD32(lanes + kColX + 32 * q, x);
            FK_TMEM_WAIT_LD32(x);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const float2 y = fmul2(make_float2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), make_float2(e, e));
              x[i] = __float_as_uint(y.x);
              x[i + 1] = __float_as_uint(y.y);
            }
            FK_TMEM_ST32(lanes + kColX + 32 * q, x);
          }
          tmem_wait_st();
        } else {
          // P V multiplies the zeros of P with what later tokens hold, and gives NaN where that is not finite: X alone is
          // written, and the rest of o added to it at the end, token by token.
          any_odd = true;
#pragma unroll 1
          for (int q = 0; q < D / 8; ++q) {
            float x[8];
            asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                         : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                         : "r"(lanes + kColX + 8 * q));
            asm volatile("tcgen05.wait::ld.sync.aligned;"
                         : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]) :: "memory");
            if (t < it.tokens)
              *reinterpret_cast<uint4*>(to + 8 * q) = make_uint4(pack_bf16(e * x[0], e * x[1]), pack_bf16(e * x[2], e * x[3]),
                                                                 pack_bf16(e * x[4], e * x[5]), pack_bf16(e * x[6], e * x[7]));
          }
          __syncwarp();
        }
        tc_fence_before();
        arrive(&bar->y_ready);
        if (!(ok = wait_for(&bar->y_full, m))) break;
        tc_fence_after();
        const bool whole = n * C + 32 * wq + 32 <= it.tokens;   // all rows of this warp
        uint8_t* tile = last ? sV + b * (2 * Lay::kTile) : sQ + (m & 1) * Lay::kTile;
#pragma unroll 1
        for (int q = 0; q < D / 32 && !odd; ++q) {
          uint32_t y[32];
          FK_TMEM_LD32(lanes + kColX + 32 * q, y);
          FK_TMEM_WAIT_LD32(y);
#pragma unroll
          for (int i = 0; i < 16; ++i) y[i] = pack_bf16(__uint_as_float(y[2 * i]), __uint_as_float(y[2 * i + 1]));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = 4 * q + i;                         // run of 16 bytes
            *reinterpret_cast<uint4*>(tile + (k >> 3) * (C * 128) + row * 128 + (((k & 7) ^ (row & 7)) << 4)) =
                make_uint4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
          }
        }
        tc_fence_before();
        arrive(&bar->x_ready);
        if (whole && !odd) {
          fence_to_async();
          __syncwarp();
          if (lane == 0) {
#pragma unroll
            for (int p = 0; p < kPanels; ++p)
              asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];"
                           :: "l"(&tmO), "r"(su32(tile + p * (C * 128) + wq * (32 * 128))), "r"(head * D + p * 64),
                           "r"((int)(it.tok0 + n * C) + 32 * wq) : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          }
        }
        if (!whole && !odd && t < it.tokens) {               // (the last chunk's last rows)
#pragma unroll 1
          for (int k = 0; k < D / 8; ++k)
            *reinterpret_cast<uint4*>(to + 8 * k) =
                *reinterpret_cast<const uint4*>(tile + (k >> 3) * (C * 128) + row * 128 + (((k & 7) ^ (row & 7)) << 4));
        }
        arrive(last ? &bar->v_empty[b] : &bar->q_empty[m & 1]);
      }
      if (!ok) break;
      arrive(&bar->odd_empty[b]);
      arrive(&bar->g_empty[b]);
    }
    base += it.nc;
    }
    // Each thread's factors of a chunk's values go to shared memory, over the tiles: these are done with once O's warps have
    // let go of the last two of V.
    if (!kLocal && any_odd && ok) ok = wait_for(&bar->v_empty[(base - 1) & 1], (base - 1) >> 1);
    if (!kLocal && any_odd && ok && base > 1) ok = wait_for(&bar->v_empty[base & 1], (base - 2) >> 1);
    if (!kLocal && any_odd && ok) {
      // o's terms of a chunk's own tokens, where V of the chunk is not all finite, in fp32 (0.5 ms a chunk and query head of 128: this
      // is for inputs that went wrong)
      float* factor = reinterpret_cast<float*>(smem) + row;  // [token][row]
      static_assert(4 * Lay::kTile >= C * C * 4, "the factors' place");
#pragma unroll 1
      for (int round = 0; item_at(round) < a.items; ++round) {
        const Item it = item_of(a, item_at(round));
#pragma unroll 1
        for (int n = 0; n < it.nc; ++n) {
          const int valid = min(C, it.tokens - n * C), own = min(row, valid - 1);   // (rows behind the last one: not written)
          const int64_t tok = it.tok0 + n * C;
          const int newest = __reduce_max_sync(0xffffffffu, own);
          bool odd = false;
          for (int i = lane; i < valid * (D / 8); i += 32) {
            const uint4 v = *reinterpret_cast<const uint4*>(a.V + (tok + i / (D / 8)) * a.vstride + (int64_t)it.kvh * D + i % (D / 8) * 8);
            odd |= not_finite(v.x) || not_finite(v.y) || not_finite(v.z) || not_finite(v.w);
          }
          if (!__any_sync(0xffffffffu, odd)) continue;
#pragma unroll 1
          for (int g = 0; g < G; ++g) {
            const uint4* q = reinterpret_cast<const uint4*>(a.Q + (tok + own) * a.qstride + (int64_t)(it.kvh * G + g) * D);
            float d = 0.0f;
#pragma unroll 1
            for (int j = newest; j >= 0; --j) {
              const uint4* k = reinterpret_cast<const uint4*>(a.K + (tok + j) * a.kstride + (int64_t)it.kvh * D);
              float p = 0.0f;
#pragma unroll 4
              for (int i = 0; i < D / 8; ++i) {
                const uint4 x = q[i], y = k[i];
                const uint32_t xx[4] = {x.x, x.y, x.z, x.w}, yy[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) p = fmaf(high(xx[e]), high(yy[e]), fmaf(low(xx[e]), low(yy[e]), p));
              }
              factor[j * C] = p * a.scale * expf(d);
              if (j <= own) d += at_least(__ldg(a.decay + (tok + j) * a.dstride + it.kvh), kLeastAmongGrowth);
            }
            bf16* to = a.O + (tok + own) * a.ostride + (int64_t)(it.kvh * G + g) * D;
#pragma unroll 1
            for (int k0 = 0; k0 < D; k0 += 8) {
              uint4 x = *reinterpret_cast<const uint4*>(to + k0);
              float o[8] = {low(x.x), high(x.x), low(x.y), high(x.y), low(x.z), high(x.z), low(x.w), high(x.w)};
#pragma unroll 2
              for (int j = newest; j >= 0; --j) {
                x = *reinterpret_cast<const uint4*>(a.V + (tok + j) * a.vstride + (int64_t)it.kvh * D + k0);
                const float v[8] = {low(x.x), high(x.x), low(x.y), high(x.y), low(x.z), high(x.z), low(x.w), high(x.w)};
                if (j > own) continue;
                const float p = factor[j * C];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = fmaf(p, v[i], o[i]);
              }
              if (row < valid)
                *reinterpret_cast<uint4*>(to + k0) = make_uint4(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]), pack_bf16(o[4], o[5]), pack_bf16(o[6], o[7]));
            }
          }
          __syncwarp();
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && bar->abort) atomicOr(a.status, kStatusTimeout);
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(bar->tmem_base), "r"(512u) : "memory");
  }
}

// The states before each segment of a head: place i + 1 holds what segment i adds to a zero state.
template <int D>
__global__ void __launch_bounds__(256) linear_join_kernel(const __grid_constant__ LinearChunkArgs a) {
  constexpr int kBlocks = D * D / 4 / 256;        // of a head
  // (launched while the kernel before still runs, and lets the next one start)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int k = blockIdx.y, segs = a.seqs.segs[k];
  const int h = blockIdx.x / kBlocks, at = (blockIdx.x % kBlocks) * 256 + threadIdx.x;
  const int64_t place = (int64_t)a.seqs.place0[k] + h * segs;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f), *p = reinterpret_cast<float4*>(a.place + place * (D * D)) + at;
  if (segs > 1) p[0] = s = reinterpret_cast<const float4*>(a.state + ((int64_t)a.seqs.slot[k] * a.Hkv + h) * (D * D))[at];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  p += D * D / 4;
  const float2* decay = a.place_decay + place + 1;
  constexpr int kAhead = 8;
  for (int i0 = 1; i0 < segs; i0 += kAhead) {
    float4 x[kAhead];
    float2 e[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i0 + i < segs) {
        x[i] = p[i * (D * D / 4)];
        e[i] = decay[i];
      }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i0 + i < segs) {
        s.x = fmaf(s.x, e[i].x, fmaf(s.x, e[i].y, x[i].x));
        s.y = fmaf(s.y, e[i].x, fmaf(s.y, e[i].y, x[i].y));
        s.z = fmaf(s.z, e[i].x, fmaf(s.z, e[i].y, x[i].z));
        s.w = fmaf(s.w, e[i].x, fmaf(s.w, e[i].y, x[i].w));
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
cudaError_t launch(bool split, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                   const CUtensorMap& tmO, const LinearChunkArgs& a,
                   cudaStream_t s) {
  if (split) {
    LinearChunkArgs b = a;                        // all segments but the last
    int item = 0;
    for (int k = 0; k < a.seqs.n; ++k) {
      b.seqs.item0[k] = item;
      item += (a.seqs.segs[k] - 1) * a.Hkv;
    }
    b.seqs.item0[a.seqs.n] = b.items = item;
    linear_chunk_kernel<D, true><<<std::min(item, a.ctas), kThreads, Layout<D>::kSmem, s>>>(tmQ, tmK, tmV, tmO, b);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) e = launch_early(linear_join_kernel<D>, dim3(a.Hkv * (D * D / 1024), a.seqs.n), 256, 0, s, a);
    if (e == cudaSuccess)
      e = launch_early(linear_chunk_kernel<D, false>, dim3(std::min(a.items, a.ctas)), kThreads, Layout<D>::kSmem, s, tmQ, tmK, tmV, tmO, a);
    return e;
  }
  linear_chunk_kernel<D, false><<<std::min(a.items, a.ctas), kThreads, Layout<D>::kSmem, s>>>(tmQ, tmK, tmV, tmO, a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t linear_chunk_prepare(int D) { return D == 128 ? prepare<128>() : prepare<64>(); }

cudaError_t launch_linear_chunk(int D, bool split, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                                const CUtensorMap& tmO, const LinearChunkArgs& a, cudaStream_t s) {
  return D == 128 ? launch<128>(split, tmQ, tmK, tmV, tmO, a, s) : launch<64>(split, tmQ, tmK, tmV, tmO, a, s);
}

}  // namespace fk
