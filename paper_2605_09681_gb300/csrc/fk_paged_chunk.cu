// Attention of many queries over the paged 8-bit cache (chunks, prompts): 5th-generation tensor cores.
//   S = q k^T 2^(e_q + e_k) log2(e) scale,  p = 2^(S - m),  l = sum p,  O = 2^r sum p 2^(e_v - r) v / l
// with v the codes' values.
// CTA = (sequence, kv head, two tiles of 128 query rows, key split); a query row is (query, head of the group), so
// that a group's heads share every key tile.  Small grids: one tile of 128 rows per CTA over two sets of key
// tiles (kOne).  Keys come in tiles of 128, from 1 to 4 pages each:
//   warps 0-3 / 4-7    softmax of query tile 0 / 1 (kOne: of key tiles 0, 2, .. / 1, 3, ..), thread = row;
//   warp 8             page numbers, exponents, and TMA of K and V codes into rings of three and two stages;
//   warp 9             tcgen05.mma, in the order PV_0(j), S_0(j+1), PV_1(j), S_1(j+1);
//   warps 10-11        V codes -> f16 values (exact), two stages.
// Q K^T needs no conversion of the keys: with q 2^-e_q = hi + lo, both E4M3 (a bf16 element of at least 2^-9 of its
// row's largest is the sum exactly, smaller ones to 2^-17 of the largest), S = hi K^T + lo K^T is two E4M3 products
// at twice the bf16 rate, on the codes as the cache holds them.  P V needs P in more than 4 bits, and P split the
// same way would cost each of the 256 x 128 numerators of a key tile five more instructions; the tile's 128 x D values
// cost twelve instructions per 16 instead, in warps of their own, and P goes as f16 (11 bits).  The block exponents come
// for free: e_k and e_v - r of each 32 keys in the factor and the summand of the softmax's fused multiply-add.
// The loading warp says which r (see kRefWindow) a key tile asks for, and each row goes there as far as what it holds allows (follow).  A
// tile whose own pages differ by more than the window allows, or has one of zeros ("wild"), is handed over 32 keys at a time,
// which ask for their own, O rescaled in between.
// Key splits leave (m, l, r, O) in a workspace; join_kernel joins them.
// What bounds it: 4680 queries over 32760 keys, 12 heads of 128, take 626-641 us, 1470-1505 TFLOP/s.  A key tile takes the two query tiles
// 2950 cycles, 2048 of them products at their nominal rate: a query tile's softmax (1600) and the wait for its next S take turns, since
// P lies over S and tensor memory is full (S, O of two tiles), and Q K^T wants 128 bytes of shared memory a cycle, all there is, beside
// the conversion's.  A CTA starts and ends in ~15000 cycles (queries copied 3300, their codes 3500, first S 1450, first tile
// 2000 more than the others, rows out 3000), which is what causal prompts (6 of 63 to 4001 tokens, 32 heads of 128: 220-228 us)
// and windows (2048 queries, window 1024: 29.0 us) pay for.  kOne (8 sequences of 16000 keys, 12 kv heads, 30 rows: 100 us, the
// codes' bytes 58) is bound by its products' operands.
// Measured and left: an MMA warp for each query tile (their products then interleave: 821 us), looking for the next hand-over
// between products (712), four converting warps at 88 registers (677; kOne 105.8), keys handed over as 112 + 16 (701), the
// two-pass path for masked tiles (prompts 244, window 33.8), a thread's query row from global memory into registers (64 channels and kOne
// 2-3% faster, 128 channels 3-4% slower: the instruction cache again, which every wait's polling inline also overran: 705 us).
// The pipeline, its barriers and the lazily raised running maximum are those of the chunk attention over packed views.
#include "fk_paged_rows.h"

namespace fk {
namespace {

constexpr float kRescaleThreshold = 1.0f;          // log2 units by which a part must exceed m to raise it
constexpr float kNoMax = -3.402823466e38f;         // m before any key: finite, so that 2^(-inf - m) is 0
constexpr int kWarpTma = 8, kWarpMma = 9, kWarpConv = 10;
constexpr int kChunkThreads = 384;
constexpr int kKStages = 3;
constexpr int kBM = kAttnBM, kBN = kAttnBN;
constexpr float kShiftP = 7.0f;                    // P is stored times 2^7: at most 2^15 in f16
constexpr int kInfo = 64;                          // key tiles whose pages and exponents are at hand

struct ChunkInfo {                                 // of a key tile
  int y[4];                                        // row of each box in the layer's pages
  uint32_t ve;                                     // e_v of each 32 keys, one byte each
  int r;                                           // reference that the tile asks for (a wild one's 32 keys ask for their own)
  int wild;
  int key0;                                        // first key
  // of each 32 keys: 2^e_k, and where the tile is not wild the exponent's summand e_v - r + 7, and 2^(r - e_v) for the
  // row sum
  float fk[4], add[4], mul[4];
};
struct ChunkBarriers {
  uint64_t q_ready;                 // the queries' codes written
  uint64_t info_ready;              // the first 32 tiles' numbers
  uint64_t tmem_ready;              // the tensor memory's address
  uint64_t k_full[kKStages], k_empty[kKStages];
  uint64_t v8_full[2], v8_empty[2]; // V codes
  uint64_t vf_full[2], vf_empty[2]; // f16 values
  uint64_t s_full[2], p_full[2], pa_full[2], pva_done[2];
  uint64_t o_done[2], fin;
  volatile uint32_t tmem_base;
  int n_info;                       // key tiles whose ChunkInfo has been written
  volatile int abort;
  // what the epilogue needs of the CTA's place (kept here and not in registers across the key tiles)
  volatile int seq, kvh, row0, rows, split, n_splits, slot0;
};

template <int D>
struct ChunkLayout {
  static constexpr int kQ = kBM * D;              // one E4M3 query tile (hi or lo)
  static constexpr int kK = kBN * D;              // one tile of codes
  static constexpr int kV = kBN * D * 2;          // one tile of f16 values
  static constexpr int kOffQ = 0;                 // hi, lo of tile 0, hi, lo of tile 1
  static constexpr int kOffK = kOffQ + 4 * kQ;
  static constexpr int kOffV8 = kOffK + kKStages * kK;
  static constexpr int kOffV = kOffV8 + 2 * kK;
  static constexpr int kOffInfo = kOffV + 2 * kV;
  static constexpr int kOffBar = kOffInfo + kInfo * (int)sizeof(ChunkInfo);
  static constexpr int kOffHeld = kOffBar + 384;
  static constexpr int kUsed = kOffHeld + 256 * 4;
  static_assert(sizeof(ChunkBarriers) <= 384, "barriers");
  // the epilogue's rows of O in fp32 (256) and their (m, l, r)
  static_assert(2 * kBM * D * 4 + 2 * kBM * 16 <= kOffInfo, "O over the operand tiles");
  // at least ~116 KB so that one CTA occupies an SM (its 512 TMEM columns are then free)
  static constexpr int kSmem = (kUsed + 1024) > 118 * 1024 ? (kUsed + 1024) : 118 * 1024;
};

// exponent of chunk c (32 keys) of four packed ones
__device__ __forceinline__ int chunk_exp(uint32_t packed, int c) { return (int)(int8_t)(packed >> (8 * c)); }

// Two bf16 query elements times `scale` (at most 448) as f16, x = hi + lo: E4M3 codes of both parts.  hi has the leading
// four bits of each element and lo the rest (a bf16 has eight).
__device__ __forceinline__ uint16_t e4m3x2_of_f16x2(uint32_t x) {
  uint16_t c;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(c) : "r"(x));
  return c;
}
__device__ __forceinline__ void split2(uint32_t w, float scale, uint16_t& hi, uint16_t& lo) {
  const uint32_t x = pack_f16(__uint_as_float(w << 16) * scale, __uint_as_float(w & 0xFFFF0000u) * scale);
  hi = e4m3x2_of_f16x2(x);
  const uint32_t h = f16x2_of_e4m3x2(hi);
  const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&h));
  lo = e4m3x2_of_f16x2(*reinterpret_cast<const uint32_t*>(&d));
}
// 32 bytes to global memory at once (32-byte aligned)
__device__ __forceinline__ void store32(void* dst, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               :: "l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
// byte offset of 16-byte run c of row `row` in a tile of D-byte rows (the TMA's and the MMA's swizzle)
template <int D>
__device__ __forceinline__ int code_run(int row, int c) {
  return D == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
}
// warp_wait whose polling is out of line (a copy of it for each of the kernel's waits outgrows the instruction cache).
__device__ __noinline__ bool poll(uint64_t* b, uint32_t parity, ChunkBarriers* bar, int* status) { return warp_wait(b, parity, bar, status); }
__device__ __forceinline__ bool tile_wait(uint64_t* b, uint32_t parity, ChunkBarriers* bar, int* status) {
  return __all_sync(0xffffffffu, mbar_test(b, parity)) || poll(b, parity, bar, status);
}
// 16 columns of tensor memory, awaited
#define FK_TMEM_LD16(taddr, v)                                                              \
  asm volatile(                                                                             \
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,"  \
      "%13,%14,%15}, [%16];"                                                                \
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),  \
        "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]),           \
        "=r"(v[13]), "=r"(v[14]), "=r"(v[15])                                               \
      : "r"(taddr));                                                                        \
  asm volatile("tcgen05.wait::ld.sync.aligned;"                                             \
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]),    \
                 "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]),  \
                 "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]) :: "memory")
template <int D, bool kOne>
__global__ void __launch_bounds__(kChunkThreads, 1)
chunk_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
             const __grid_constant__ PagedAttnArgs a) {
  using Lay = ChunkLayout<D>;
  constexpr int kAhead = kOne ? 2 : 1;            // S_t(j + kAhead) follows P_t V_j
  constexpr int kTiles = kOne ? 1 : 2;            // query tiles
  constexpr uint32_t kTmemCols = 512;
  constexpr uint32_t kColO = 2 * kBN;             // S0 = cols 0..127, S1 = 128..255, O0, O1 after
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem + Lay::kOffQ;
  uint8_t* sK = smem + Lay::kOffK;
  uint8_t* sV8 = smem + Lay::kOffV8;
  uint8_t* sV = smem + Lay::kOffV;
  ChunkInfo* info = reinterpret_cast<ChunkInfo*>(smem + Lay::kOffInfo);
  ChunkBarriers* bar = reinterpret_cast<ChunkBarriers*>(smem + Lay::kOffBar);
  float* held = reinterpret_cast<float*>(smem + Lay::kOffHeld);   // of a softmax thread's row: see less
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // ---- this CTA's rows and key tiles
  int s = 0;
  {
    int hi = a.seqs.n - 1;
    while (s < hi) {
      const int mid = (s + hi + 1) >> 1;
      if (a.seqs.item0[mid] <= (int)blockIdx.x) s = mid;
      else hi = mid - 1;
    }
  }
  const int n_keys = a.seqs.n_keys[s], n_q = a.seqs.n_q[s], n_rows = n_q * a.G;
  // items: (rows, kv head) pairs, the longest rows first; the first `whole` of them unsplit
  const int groups = (n_rows + kTiles * kBM - 1) / (kTiles * kBM), whole = a.seqs.whole[s];
  const int item = (int)blockIdx.x - a.seqs.item0[s];
  const int n_splits = item < whole ? 1 : a.seqs.splits[s];
  const int split = item < whole ? 0 : (item - whole) % n_splits;
  const int pair = item < whole ? item : whole + (item - whole) / n_splits;
  const int kvh = pair % a.Hkv, row0 = (groups - 1 - pair / a.Hkv) * (kTiles * kBM);
  const int rows = min(kTiles * kBM, n_rows - row0);
  const int p_first = n_keys - n_q;
  const TileRange tr = paged_tiles(n_keys, p_first + a.by_g.div(row0), p_first + a.by_g.div(row0 + rows - 1), a.mask, kBN);
  const int n_tiles = tr.count();
  const int i0 = (int)((int64_t)n_tiles * split / n_splits);
  const int nt = (int)((int64_t)n_tiles * (split + 1) / n_splits) - i0;        // may be 0

  const int box = min(a.P, kPagedFewTile), boxes = kBN / box;   // rows of a TMA box, boxes of a tile
  auto load = [&](const CUtensorMap* map, uint8_t* dst, int j, uint64_t* b) {   // lanes < boxes
    if (lane < boxes) tma_load_2d(dst + lane * box * D, map, b, 0, info[j & (kInfo - 1)].y[lane]);
  };
  auto load_k = [&](int j) {
    const int st = j % kKStages;
    if (lane == 0) mbar_expect_tx(&bar->k_full[st], Lay::kK);
    __syncwarp();
    load(&tmK, sK + st * Lay::kK, j, &bar->k_full[st]);
  };
  // Key tiles j0 + lane (a warp): their pages, and then, which the loads need not wait for, exponents and references.
  int pages[4] = {0, 0, 0, 0};                      // of each 32 keys
  auto fetch_pages = [&](int j0) {
    const int j = j0 + lane;
    if (j < nt) {
      const int* table = a.table + (int64_t)a.seqs.slot[s] * a.max_pages;
      const int last_page = max(n_keys - 1, 0) / a.P, key0 = tr.at(i0 + j) * kBN;
      ChunkInfo& x = info[j & (kInfo - 1)];
#pragma unroll
      for (int c = 0; c < 4; ++c) pages[c] = __ldg(table + min((key0 + 32 * c) / a.P, last_page));
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int y = (pages[c] * a.Hkv + kvh) * a.P + (key0 + 32 * c) % a.P;
        if (boxes == 4) x.y[c] = y;
        else if ((c & 1) == 0) x.y[c >> 1] = y;
      }
    }
    __syncwarp();
  };
  int ref[2] = {kNoRef, kNoRef};                    // of the last tile (kOne: of each key set)
  auto fetch_exps = [&](int j0) {
    const int j = j0 + lane;
    int lo = 127, hi = -127, last = kNoRef, ev[4];  // of the tile's blocks that are not zeros
    float fk[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    bool wild = false, zeros = false;
#pragma unroll
    for (int c = 0; c < 4; ++c) ev[c] = kZeroExp;
    if (j < nt) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int64_t block = (int64_t)pages[c] * a.Hkv + kvh;
        fk[c] = pow2f(a.ke[block]);
        ev[c] = a.ve[block];
      }
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (ev[c] != kZeroExp) {
          lo = min(lo, ev[c]);
          hi = max(hi, ev[c]);
          last = ev[c];
        } else {
          zeros = true;
        }
      wild = zeros || hi - lo > kRefWindow - kRefRoom;
    }
    int mine = kNoRef;
    for (int i = 0; i < min(32, nt - j0); ++i) {    // the references, tile by tile
      int r = kOne && (i & 1) ? ref[1] : ref[0];
      const int thi = __shfl_sync(0xffffffffu, hi, i), tlo = __shfl_sync(0xffffffffu, lo, i);
      const int tlast = __shfl_sync(0xffffffffu, last, i), tw = __shfl_sync(0xffffffffu, (int)wild, i);
      if (tlast != kNoRef && (tw || thi > r || tlo < r - kRefWindow)) r = (tw ? tlast : thi) + kRefRoom;
      (kOne && (i & 1) ? ref[1] : ref[0]) = r;
      if (lane == i) mine = r;
    }
    if (j < nt) {
      ChunkInfo& x = info[j & (kInfo - 1)];
      x.r = mine;
      x.wild = wild;
      x.key0 = tr.at(i0 + j) * kBN;
      uint32_t ve = 0;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int below = wild ? 0 : mine - ev[c];
        ve |= (uint32_t)(uint8_t)ev[c] << (8 * c);
        x.fk[c] = fk[c];
        x.add[c] = kShiftP - (float)below;
        x.mul[c] = pow2_any(below);
      }
      x.ve = ve;
    }
    __syncwarp();
    if (lane == 0) asm volatile("st.release.cta.shared::cta.b32 [%0], %1;" :: "r"(su32(&bar->n_info)), "r"(j0 + 32) : "memory");
  };

  if (warp == kWarpTma) {
    if (lane == 0) {
      mbar_init(&bar->q_ready, 8);
      mbar_init(&bar->info_ready, 1);
      mbar_init(&bar->tmem_ready, 1);
      for (int i = 0; i < kKStages; ++i) {
        mbar_init(&bar->k_full[i], 1);
        mbar_init(&bar->k_empty[i], 1);
      }
      for (int i = 0; i < 2; ++i) {
        mbar_init(&bar->v8_full[i], 1);
        mbar_init(&bar->v8_empty[i], 2);            // both converting warps
        mbar_init(&bar->vf_full[i], 2);
        mbar_init(&bar->vf_empty[i], 1);
        mbar_init(&bar->s_full[i], 1);
        mbar_init(&bar->p_full[i], 4);
        mbar_init(&bar->pa_full[i], 4);
        mbar_init(&bar->pva_done[i], 1);
      }
      mbar_init(&bar->o_done[0], 1);
      mbar_init(&bar->o_done[1], 1);
      mbar_init(&bar->fin, 1);
      bar->abort = 0;
      bar->n_info = 0;
      bar->seq = s;
      bar->kvh = kvh;
      bar->row0 = row0;
      bar->rows = rows;
      bar->split = split;
      bar->n_splits = n_splits;
      bar->slot0 = a.seqs.part0[s] + (item - whole) * kTiles;   // workspace tiles of this CTA
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
  }
  const int t = warp >> 2;                          // query tile (kOne: key set) of a softmax warpgroup
  const int wq = warp & 3, row = wq * 32 + lane;
  if (warp < 8 && nt > 0) {
    // a softmax warp's query rows, bf16, on their way to where the values go later
    constexpr int kRuns = D / 8;                    // 16-byte runs of a row
    const int q0 = a.seqs.q0[s];
#pragma unroll 4
    for (int i = lane / kRuns; i < 32; i += 32 / kRuns) {
      const int rr = wq * 32 + i, at = row0 + (kOne ? 0 : t * kBM) + rr, tok = a.by_g.div(at), c = lane % kRuns;
      if (at < row0 + rows)
        cp_async16(sV + (t * kBM + rr) * (D * 2) + c * 16,
                   a.Q + ((int64_t)q0 + tok) * a.qstride + (int64_t)(kvh * a.G + at - tok * a.G) * D + c * 8);
    }
  }
  // The loading warp, which has set the barriers up, goes on at once; the others come when the copies are on their way.
  if (warp == kWarpTma) {
    __syncwarp();
    asm volatile("bar.arrive 2, %0;" :: "n"(kChunkThreads) : "memory");
  } else {
    asm volatile("bar.sync 2, %0;" :: "n"(kChunkThreads) : "memory");
  }

  // softmax state (warps 0-7)
  float m = kNoMax, l = 0.0f;
  int r = kNoRef;                                   // reference of O
  if (warp < 8) held[threadIdx.x] = 0.0f;
  uint32_t n_pa = 0;                                // parts handed over on pa_full
  bool ok = true;

  if (warp == kWarpTma) {
    // ------------------------------------------------------------------ TMA producer
    // V_j, then K_{j+2} (K_0 and K_1 are under way)
    fetch_pages(0);
    for (int j = 0; j < min(2, nt); ++j) load_k(j);
    int jv = -1, jk = min(2, nt) - 1;               // last tiles issued
    for (int j = 0; j < nt; ++j) {
      const int b = j & 1;
      if (j >= 2 && !tile_wait(&bar->v8_empty[b], ((j >> 1) - 1) & 1, bar, a.status)) { ok = false; break; }
      if (lane == 0) mbar_expect_tx(&bar->v8_full[b], Lay::kK);
      __syncwarp();
      load(&tmV, sV8 + b * Lay::kK, j, &bar->v8_full[b]);
      jv = j;
      if (j == 0) {
        fetch_exps(0);
        if (lane == 0) mbar_arrive(&bar->info_ready);
      }
      if (j + 2 >= nt) continue;
      if (((j + 2) & 31) == 0) {
        fetch_pages(j + 2);
        fetch_exps(j + 2);
      }
      if (j + 2 >= kKStages && !tile_wait(&bar->k_empty[(j + 2) % kKStages], ((j + 2) / kKStages - 1) & 1, bar, a.status)) { ok = false; break; }
      load_k(j + 2);
      jk = j + 2;
    }
    if constexpr (kOne) allow_join();               // (16 x 2000 keys, 48 rows: 21.7 -> 18.5 us; two tiles, whose join is short: slower)
    if (!ok) {                                      // what was issued lands before the CTA ends
      for (int j = max(0, jk - kKStages + 1); j <= jk; ++j) wait_phase(&bar->k_full[j % kKStages], (j / kKStages) & 1, bar, a.status, false);
      for (int j = max(0, jv - 1); j <= jv; ++j) wait_phase(&bar->v8_full[j & 1], (j >> 1) & 1, bar, a.status, false);
    }
    __syncwarp();
  } else if (warp == kWarpMma) {
    // ------------------------------------------------------------------ MMA issuer
    // Tensor-core operations of one thread complete in issue order: when S_t(j+1) is complete, so is PV_t(j).
    // (The allocation takes ~1000 cycles: nobody waits for it at the start.)
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 :: "r"(su32(const_cast<uint32_t*>(&bar->tmem_base))), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    if (lane == 0) mbar_arrive(&bar->tmem_ready);
    const uint32_t tmem = bar->tmem_base;
    constexpr uint32_t kIdQK = idesc_e4m3(kBM, kBN), kIdPV = idesc_f16(kBM, D, 1);
    constexpr uint32_t kLayout = D == 128 ? 2 : 4, kSbo = 8 * D;
    const uint64_t dQ = sdesc(su32(sQ), 16, kSbo, kLayout), dK = sdesc(su32(sK), 16, kSbo, kLayout);
    const uint64_t dV = sdesc(su32(sV), 16384, 1024);
    auto qk = [&](int j, int tt) {
      const uint64_t da = dQ + (uint32_t)((kOne ? 0 : tt) * (2 * Lay::kQ >> 4)), db = dK + (uint32_t)((j % kKStages) * (Lay::kK >> 4));
      const uint32_t d = tmem + (uint32_t)(tt * kBN);
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) umma_f8(d, da + kk * 2, db + kk * 2, kIdQK, kk > 0 ? 1u : 0u);
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) umma_f8(d, da + (Lay::kQ >> 4) + kk * 2, db + kk * 2, kIdQK, 1u);
      umma_commit(&bar->s_full[tt]);
    };
    // PV of a tile's keys 32 c0 .. 32 c1 - 1
    auto pv = [&](int j, int tt, int c0, int c1) {
      const uint64_t db = dV + (uint32_t)((j & 1) * (Lay::kV >> 4));
      const uint32_t d = tmem + kColO + (uint32_t)(tt * D), p = tmem + (uint32_t)(tt * kBN);
#pragma unroll
      for (int kk = 2 * c0; kk < 2 * c1; ++kk)
        umma_ts(d, p + kk * 8, db + kk * 128, kIdPV, (j >= kAhead || kk > 0) ? 1u : 0u);
    };
    auto pv1 = [&](int j, int tt, int c) {          // 32 keys
      const uint64_t db = dV + (uint32_t)((j & 1) * (Lay::kV >> 4) + c * 256);
      const uint32_t d = tmem + kColO + (uint32_t)(tt * D), p = tmem + (uint32_t)(tt * kBN + c * 16);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        umma_ts(d, p + kk * 8, db + kk * 128, kIdPV, (j >= kAhead || c > 0 || kk > 0) ? 1u : 0u);
    };
    auto wait = [&](uint64_t* b, uint32_t parity) { return tile_wait(b, parity, bar, a.status); };
    uint32_t n_pa[2] = {0, 0};                      // parts of P taken on pa_full
    auto k_ready = [&](int j) { return wait(&bar->k_full[j % kKStages], (j / kKStages) & 1); };
    if (nt > 0) {
      ok = wait(&bar->q_ready, 0) && k_ready(0);
      if (ok) {
        tc_fence_after();
        if (elect_one()) {
          qk(0, 0);
          if (!kOne) qk(0, 1);
          umma_commit(&bar->k_empty[0]);
        }
      }
      ok = ok && wait(&bar->info_ready, 0) && wait(&bar->vf_full[0], 0);
      if (kOne && nt > 1 && ok) {
        ok = k_ready(1);
        if (ok && elect_one()) {
          qk(1, 1);
          umma_commit(&bar->k_empty[1]);
        }
      }
    }
    for (int j = 0; j < nt && ok; ++j) {
      const int b = j & 1;
      const bool more = j + kAhead < nt;
      const uint32_t ph = kOne ? (j >> 1) & 1 : j & 1;   // of a query tile's (kOne: key set's) barriers
      const bool wild = info[j & (kInfo - 1)].wild != 0;
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        const int tt = kOne ? b : i;
        uint32_t& np = tt ? n_pa[1] : n_pa[0];
        if (kOne && j > 0 && !wait(&bar->vf_full[b], (j >> 1) & 1)) { ok = false; break; }
        if (!wild) {
          if (!wait(&bar->pa_full[tt], np++ & 1)) { ok = false; break; }
          tc_fence_after();
          if (elect_one()) {
            pv(j, tt, 0, 3);
            umma_commit(&bar->pva_done[tt]);
          }
        } else {
#pragma unroll 1
          for (int c = 0; c < 4 && ok; ++c) {
            ok = wait(&bar->pa_full[tt], np++ & 1);
            tc_fence_after();
            if (ok && elect_one()) {
              pv1(j, tt, c);
              umma_commit(&bar->pva_done[tt]);
            }
          }
          if (!ok) break;
        }
        // K for the tile's S before the second part, the next V before the last one: neither has anything left to
        // hide behind between a tile's S and the next tile's P (a wait takes ~100 cycles when there is nothing to wait for)
        if (i == 0 && more && !k_ready(j + kAhead)) { ok = false; break; }
        // (kOne: its values are not there yet, and cannot be while this tile's products wait: it is looked for later.)
        if (!kOne && i == kTiles - 1 && j + 1 < nt && !wait(&bar->vf_full[b ^ 1], ((j + 1) >> 1) & 1)) { ok = false; break; }
        if (!wait(&bar->p_full[tt], ph)) { ok = false; break; }
        tc_fence_after();
        if (elect_one()) {
          if (!wild) pv(j, tt, 3, 4);
          if (more) qk(j + kAhead, tt);
          else umma_commit(&bar->o_done[tt]);
          if (i == kTiles - 1) {
            umma_commit(&bar->vf_empty[b]);
            if (more) umma_commit(&bar->k_empty[(j + kAhead) % kKStages]);
          }
        }
      }
    }
    if (elect_one()) {
      if (nt == 0) umma_commit(&bar->o_done[0]);
      if (nt <= (kOne ? 1 : 0)) umma_commit(&bar->o_done[1]);
      umma_commit(&bar->fin);                       // completes once every MMA above is done
    }
    wait_phase(&bar->fin, 0, bar, a.status, false);
    __syncwarp();
  } else if (warp >= kWarpConv) {
    // ------------------------------------------------------------------ V codes -> f16 values
    // A thread takes 8 codes of a row at a time: half a 16-byte run, one 16-byte unit of the f16 row.
    constexpr int kOct = D / 8, kStepRows = 64 / kOct, kFly = 16;   // units of a row; rows per pass; loads in flight
    ok = nt == 0 || tile_wait(&bar->q_ready, 0, bar, a.status);   // (the query rows were staged where the values go)
    const int x = threadIdx.x - kWarpConv * 32, prow = x / kOct, unit = x % kOct;
    for (int j = 0; j < nt && ok; ++j) {
      const int b = j & 1, u = j >> 1;
      if (!tile_wait(&bar->v8_full[b], u & 1, bar, a.status) ||
          (j >= 2 && !tile_wait(&bar->vf_empty[b], (u - 1) & 1, bar, a.status))) { ok = false; break; }
      const uint8_t* src = sV8 + b * Lay::kK;
      uint8_t* dst = sV + b * Lay::kV;
#pragma unroll
      for (int k0 = 0; k0 < kBN / kStepRows; k0 += kFly) {   // (loads would not pass the stores by themselves)
        uint2 v[kFly];
#pragma unroll
        for (int k = 0; k < kFly; ++k) {
          const int r = prow + (k0 + k) * kStepRows;
          v[k] = *reinterpret_cast<const uint2*>(src + code_run<D>(r, unit >> 1) + (unit & 1) * 8);
        }
#pragma unroll
        for (int k = 0; k < kFly; ++k) {
          const int r = prow + (k0 + k) * kStepRows;
          *reinterpret_cast<uint4*>(dst + (unit >> 3) * 16384 + r * 128 + (((unit & 7) ^ (r & 7)) << 4)) =
              make_uint4(f16x2_of_e4m3x2((uint16_t)v[k].x), f16x2_of_e4m3x2((uint16_t)(v[k].x >> 16)),
                         f16x2_of_e4m3x2((uint16_t)v[k].y), f16x2_of_e4m3x2((uint16_t)(v[k].y >> 16)));
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the tensor core reads them through it
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&bar->vf_full[b]);
        mbar_arrive(&bar->v8_empty[b]);
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ softmax warpgroups
    const int crow = (kOne ? 0 : t * kBM) + row;    // row of the CTA
    const bool in = crow < rows;
    const int pos = p_first + a.by_g.div(row0 + (in ? crow : 0));
    float sl2 = a.scale_log2;
    // The thread's row of Q from the staged rows: scaled to E4M3's range, hi and lo in the MMA's layout.  16-byte chunks in
    // an order of the row's own (j ^ row), so that the rows of a warp meet few banks.  (kOne: both key sets
    // want the scale.)  Loading rows from global memory a warp at a time, with the maximum by shuffles, took
    // 12000-58000 cycles: the shuffles waited for the loads in flight.
    if (nt > 0) {
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
      const uint8_t* src = sV + (t * kBM + row) * (D * 2);
      uint32_t top = 0;
#pragma unroll 8
      for (int j = 0; j < D / 8; ++j) {
        const uint4 v = *reinterpret_cast<const uint4*>(src + ((j ^ (row & 7)) << 4));
        top = __vmaxu2(top, __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu)));
      }
      top = in ? max(top & 0xFFFFu, top >> 16) : 0;        // as bf16 bits; rows past the end were not loaded
      const bool fine = top < 0x7F80u;
      const int e = fine ? e4m3_row_exponent(__uint_as_float(top << 16)) : 0;
      if (!kOne || t == 0) {
        const float scale = in ? pow2f(-e) : 0.0f;
        uint8_t* dst = sQ + (kOne ? 0 : t) * (2 * Lay::kQ);
        constexpr int kFly = 4;                      // (loads would not pass the stores by themselves)
#pragma unroll 1
        for (int j0 = 0; j0 < D / 8; j0 += kFly) {
          uint4 v[kFly];
          uint2 hi[kFly], lo[kFly];
#pragma unroll
          for (int k = 0; k < kFly; ++k)
            v[k] = in ? *reinterpret_cast<const uint4*>(src + (((j0 + k) ^ (row & 7)) << 4)) : make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int k = 0; k < kFly; ++k) {
            uint16_t h[4], g[4];
            split2(v[k].x, scale, h[0], g[0]);
            split2(v[k].y, scale, h[1], g[1]);
            split2(v[k].z, scale, h[2], g[2]);
            split2(v[k].w, scale, h[3], g[3]);
            hi[k] = make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
            lo[k] = make_uint2(g[0] | (uint32_t)g[1] << 16, g[2] | (uint32_t)g[3] << 16);
          }
#pragma unroll
          for (int k = 0; k < kFly; ++k) {
            const int c = (j0 + k) ^ (row & 7);
            uint8_t* to = dst + code_run<D>(row, c >> 1) + (c & 1) * 8;
            *reinterpret_cast<uint2*>(to) = hi[k];
            *reinterpret_cast<uint2*>(to + Lay::kQ) = lo[k];
          }
        }
      }
      if (fine) sl2 *= pow2f(e);
      else l = NAN;                                 // infinities or NaN: the row's O is NaN
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar->q_ready);
    }
    // visible keys: [lower, limit) and those below the sinks; tiles without a masked key for any of the tile's rows
    const int limit = a.mask.causal ? min(pos + 1, n_keys) : n_keys;
    const int lower = a.mask.window > 0 ? pos - a.mask.window + 1 : 0;
    const int trow1 = min(kOne ? rows : rows - t * kBM, kBM) - 1;   // last row of this query tile
    const int trow0 = row0 + (kOne ? 0 : t * kBM), pa = p_first + a.by_g.div(trow0), pb = p_first + a.by_g.div(trow0 + max(trow1, 0));
    const int full_hi = a.mask.causal ? min(pa + 1, n_keys) : n_keys;
    const int full_lo = a.mask.window > 0 ? pb - a.mask.window + 1 : 0;

    ok = tile_wait(&bar->tmem_ready, 0, bar, a.status) && ok;
    const uint32_t lanes = bar->tmem_base + ((uint32_t)(wq * 32) << 16);
    const uint32_t tS = lanes + (uint32_t)(t * kBN), tO = lanes + kColO + (uint32_t)(t * D);
    auto known = [&] {
      int n;
      asm volatile("ld.acquire.cta.shared::cta.b32 %0, [%1];" : "=r"(n) : "r"(su32(&bar->n_info)) : "memory");
      return n;
    };
    int n_info = 0;                                 // tiles whose numbers are known to be there
    if (nt > 0) ok = tile_wait(&bar->info_ready, 0, bar, a.status) && ok;
    for (int it = 0; ok; ++it) {
      const int j = kOne ? 2 * it + t : it;         // kOne: this warpgroup's key set is every other tile
      if (j >= nt) break;
      // The tile's numbers, before its S is complete: they are mostly written many tiles ahead, at the latest before its K is
      // loaded (the first 32 tiles': info_ready).
      if (j >= n_info) {
        n_info = known();
        if (j >= n_info) {
          if (!tile_wait(&bar->s_full[t], it & 1, bar, a.status)) { ok = false; break; }
          n_info = known();
        }
      }
      const ChunkInfo& ti = info[j & (kInfo - 1)];
      const bool wild = ti.wild != 0;
      if (it == 0 && !wild) r = ti.r;
      // of 32 keys: factor and summand of the exponent S + e_v - r + 7 - m, and what the row sum takes of theirs
      float fc[4];
#pragma unroll
      for (int c = 0; c < 4; ++c)                   // neither 0 nor infinite: masked logits are -inf, codes may all be 0
        fc[c] = fminf(fmaxf(sl2 * ti.fk[c], 1e-37f), 3e38f);
      auto factor = [&](int c) { return make_float2(fc[c], fc[c]); };
      auto factor_at = [&](int c) { return fminf(fmaxf(sl2 * ti.fk[c], 1e-37f), 3e38f); };   // (c not a constant)
      auto summand = [&](int c) {
        const float x = ti.add[c] - m;
        return make_float2(x, x);
      };
      auto weighted = [&](const float2* ah, int c, float& plain) {   // 32 numerators' sum, and its share of l
        const float2 x = fadd2(fadd2(ah[0], ah[1]), fadd2(ah[2], ah[3]));
        plain += x.x + x.y;
        return (x.x + x.y) * ti.mul[c];
      };
      const int key0 = ti.key0;
      const bool full = trow1 < 0 || (key0 + kBN <= full_hi && (key0 >= full_lo || key0 + kBN <= a.mask.sinks));
      bool direct = !wild && __all_sync(0xffffffffu, r == ti.r);   // the rows go together, at the tile's reference
      if (!tile_wait(&bar->s_full[t], it & 1, bar, a.status)) { ok = false; break; }
      tc_fence_after();
      uint32_t ca[32], cb[32], ov = 0;
      if (!full) {                                  // masked keys' logits become -inf, in place
        auto below = [](int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; };
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          const int k0 = key0 + 32 * c;
          const uint32_t seen = below(limit - k0) & (~below(lower - k0) | below(a.mask.sinks - k0));
          if (__all_sync(0xffffffffu, seen == ~0u)) continue;
          FK_TMEM_LD32(tS + c * 32, ca);
          FK_TMEM_WAIT_LD32(ca);
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (!(seen >> i & 1u)) ca[i] = __float_as_uint(-INFINITY);
          FK_TMEM_ST32(tS + c * 32, ca);
        }
        tmem_wait_st();
      }
      if (it == 0 && !wild) {                       // the first tile: m from 32 of its keys, at its end where a window begins in it
        const int c = key0 >= full_lo || key0 < a.mask.sinks ? 0 : 3;
        FK_TMEM_LD32(tS + c * 32, ca);
        FK_TMEM_WAIT_LD32(ca);
        float mxa[4] = {kNoMax, kNoMax, kNoMax, kNoMax};
#pragma unroll
        for (int i = 0; i < 32; ++i) mxa[i & 3] = fmaxf(mxa[i & 3], __uint_as_float(ca[i]));
        m = fmaxf(fmaxf(fmaxf(mxa[0], mxa[1]), fmaxf(mxa[2], mxa[3])) * factor_at(c), kNoMax);
      }
      // A tile goes in two parts, keys 0-95 and 96-127 (a wild one 32 keys at a time).  P is
      // computed with the running max m straight away; a part with a weight beyond 2^8 (2^15 as stored) is
      // done again after a max pass, which raises m and moves the rows' references.  Rows that do not go together afterwards take
      // the loop at its end.  (Few instructions beside those: the kernel's loops are at the size of the instruction cache,
      // and some hundred more of them cost a tenth.)
      const int parts = wild ? 4 : 2;
#pragma unroll 1
      for (int part = 0; part < parts; ++part) {
#pragma unroll 1
        for (bool again = false;; again = true) {
          if (direct) {
            float plain = 0.0f, dl = 0.0f;
            bool fits;
            auto chunk = [&](const uint32_t* x, int c, uint32_t* pk) {
              float2 ah[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) ah[i] = make_float2(0.0f, 0.0f);
              exp_chunk<PFormat::kF16>(x, factor(c), summand(c), ah, pk, ov);
              dl += weighted(ah, c, plain);
            };
            if (part == 0) {
              uint32_t pk[48];
              FK_TMEM_LD32(tS, ca);
              FK_TMEM_WAIT_LD32(ca);
              FK_TMEM_LD32(tS + 32, cb);
              chunk(ca, 0, pk);
              FK_TMEM_WAIT_LD32(cb);
              FK_TMEM_LD32(tS + 64, ca);
              chunk(cb, 1, pk + 16);
              FK_TMEM_WAIT_LD32(ca);
              FK_TMEM_LD32(tS + 96, cb);
              chunk(ca, 2, pk + 32);
              FK_TMEM_WAIT_LD32(cb);
              fits = again || !__any_sync(0xffffffffu, plain > 32768.0f);   // (no numerator exceeds the sum) warp-uniform
              if (fits) {
                FK_TMEM_ST32(tS, pk);
                FK_TMEM_ST16(tS + 32, (pk + 32));
              }
            } else {
              uint32_t pk[16];
              if (again) {                           // (not kept across what follows)
                FK_TMEM_LD32(tS + 96, cb);
                FK_TMEM_WAIT_LD32(cb);
              }
              chunk(cb, 3, pk);
              fits = again || !__any_sync(0xffffffffu, plain > 32768.0f);
              if (fits) FK_TMEM_ST16(tS + 48, pk);
            }
            if (fits) {
              l += dl;
              break;
            }
          }
          const int c0 = wild ? part : 3 * part, c1 = wild ? part + 1 : 3 + part;   // chunks of 32 keys
          const int e0 = chunk_exp(ti.ve, part);
          const int to = !wild ? ti.r : e0 != kZeroExp ? e0 + kRefRoom : l == 0.0f ? kNoRef : r;   // reference asked for
          float mx = -INFINITY;
#pragma unroll 1
          for (int c = c0; c < c1; ++c) {
            FK_TMEM_LD32(tS + c * 32, ca);
            FK_TMEM_WAIT_LD32(ca);
            float mxa[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < 32; ++i) mxa[i & 3] = fmaxf(mxa[i & 3], __uint_as_float(ca[i]));
            mx = fmaxf(mx, fmaxf(fmaxf(mxa[0], mxa[1]), fmaxf(mxa[2], mxa[3])) * factor_at(c));
          }
          const float m_new = fmaxf(m, mx);
          float rs = 1.0f, less = held[threadIdx.x]; // what O has to be scaled by: rs 2^d; |O| <= 2^9 l + less
          int d = 0;
          if (__any_sync(0xffffffffu, m_new > m + kRescaleThreshold)) {   // warp-uniform
            rs = fast_exp2(m - m_new);               // 0 when m = kNoMax
            l *= rs;
            less *= rs;
            m = m_new;
          }
          // The row's reference.  One that holds nothing takes any, one that does not see the part keeps its own.
          if (__any_sync(0xffffffffu, to != r)) {
            const bool none = l == 0.0f || r == kNoRef;
            float most = none ? 0.0f : fmaxf(fmaf(512.0f, l, less), 1e-37f);   // |O|, at most
            int want = none ? to : r;
            if (want != to && mx > -INFINITY) want = follow(r, to, mx - m, above2(most));
            d = r - want;
            less = fmaf(-512.0f, l, most * pow2_any(max(d, -100)) * pow2_any(min(d + 100, 0)));
            r = want;
          }
          const bool rescale = __any_sync(0xffffffffu, rs != 1.0f || d != 0) && (it > 0 || c0 > 0);   // O holds every key before chunk c0 ...
          // ... once pva_done says so.  (A wild tile's parts all go over pa_full: no warp hands one over before all four have
          // handed over the one before, or a fast warp's arrival would stand for a slow one's.)
          if (c0 > 0 && (rescale || wild)) {
            if (!tile_wait(&bar->pva_done[t], (n_pa - 1) & 1, bar, a.status)) { ok = false; break; }
            tc_fence_after();
          }
          // (in turns where a factor by itself would be too small for fp32, and what O holds in the end is not)
#pragma unroll 1
          for (bool more = rescale, first = true; more; first = false) {
            const int step = first && d < -20 ? 0 : max(d, -100);
            rs *= pow2_any(step);
            d -= step;
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
              FK_TMEM_LD32(tO + c * 32, ca);
              FK_TMEM_WAIT_LD32(ca);
#pragma unroll
              for (int e = 0; e < 32; ++e) ca[e] = __float_as_uint(__uint_as_float(ca[e]) * rs);
              FK_TMEM_ST32(tO + c * 32, ca);
            }
            rs = 1.0f;
            more = __any_sync(0xffffffffu, d != 0);
            if (more) tmem_wait_st();
          }
          held[threadIdx.x] = less;
          direct = !wild && __all_sync(0xffffffffu, r == ti.r);
          if (direct) continue;
          // numerators, and then the block's size relative to the row's reference, which l does not know
#pragma unroll 1
          for (int x = 2 * c0; x < 2 * c1; ++x) {    // 16 keys (P's columns lie over logits already read)
            const int c = x >> 1, e = chunk_exp(ti.ve, c);
            const float f = factor_at(c), below = kShiftP - m, size = e == kZeroExp ? 0.0f : pow2_any(e - r);
            float sum = 0.0f;
            uint32_t v[16], pk[8];
            FK_TMEM_LD16(tS + x * 16, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float y0 = fast_exp2(fmaf(__uint_as_float(v[2 * i]), f, below));
              const float y1 = fast_exp2(fmaf(__uint_as_float(v[2 * i + 1]), f, below));
              sum += y0 + y1;
              pk[i] = pack_f16(y0 * size, y1 * size);
            }
            FK_TMEM_ST8(tS + x * 8, pk);
            l += sum;
            less = fmaf(512.0f * sum, size - 1.0f, less);
          }
          held[threadIdx.x] = less;
          break;
        }
        if (!ok) break;
        // P in TMEM -> the MMA warp
        const bool more = wild || part == 0;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(more ? &bar->pa_full[t] : &bar->p_full[t]);
        n_pa += more;
      }
      if (!ok) break;
      if (wild) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar->p_full[t]);
      }
    }
    // ---------------------------------------------------------------- epilogue
    // This accumulator's last MMA is done, and with it every MMA that reads Q: that shared memory is free.
    ok = ok && tile_wait(&bar->o_done[t], 0, bar, a.status);
    tc_fence_after();
    const bool has = kOne ? t < nt : nt > 0;        // this accumulator was written
    const int row0 = bar->row0, rows = bar->rows, kvh = bar->kvh, n_splits = bar->n_splits;
    const int64_t q0 = a.seqs.q0[bar->seq];
    auto out_row = [&](int r) {                      // row r of the CTA
      const int q = row0 + r, tok = a.by_g.div(q);
      return a.O + (q0 + tok) * a.ostride + (int64_t)(kvh * a.G + q - tok * a.G) * D;
    };
    if (!kOne && n_splits == 1) {
      // normalise; a thread writes its row, a whole 32-byte sector at a time where rows are aligned to that (through shared
      // memory to coalesced rows, side by side: 228.7 us for the prompts; 16 bytes at a time 228.3; 32: 221.4)
      const Normal to(l, max(r, -60));
      const float inv = to.by_l * to.size, low = pow2_any(min(r + 60, 0));
      const bool tiny = __any_sync(0xffffffffu, r < -60);                // (inv by itself would lose bits)
      const int cr = (kOne ? 0 : t * kBM) + row;
      if (ok) {
        bf16* dst = out_row(min(cr, rows - 1));
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32], v[16];
          FK_TMEM_LD32(tO + c * 32, o);
          FK_TMEM_WAIT_LD32(o);
          if (tiny) {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * low);
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = has ? pack_bf16(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv) : 0u;
          if (cr >= rows) continue;
          if (a.wide_o) {
            store32(dst + c * 32, v);
            store32(dst + c * 32 + 16, v + 8);
          } else {
#pragma unroll
            for (int e = 0; e < 16; e += 4) *reinterpret_cast<uint4*>(dst + c * 32 + 2 * e) = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
          }
        }
      }
    } else {
      ok = ok && tile_wait(&bar->o_done[t ^ 1], 0, bar, a.status);   // all operand tiles are free
      // both accumulators to shared memory, [t][row][D] with 16-byte run c of a row at c ^ (row & 7), and their (m, l, r)
      float* so = reinterpret_cast<float*>(smem) + (t * kBM + row) * D;
      float4* ml = reinterpret_cast<float4*>(smem + 2 * kBM * D * 4);
      // a part goes out at the reference of what it holds (O may have been lifted), or the joins' factors could not hold it
      const int lift = max(above2(fmaxf(fmaf(512.0f, l, held[threadIdx.x]), 1e-37f)) - 24, 0);
      const float down = pow2_any(-lift);
      r += lift;
      if (ok) {
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          FK_TMEM_LD32(tO + c * 32, o);
          FK_TMEM_WAIT_LD32(o);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * down);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<uint4*>(so + (((c * 8 + e) ^ (row & 7)) << 2)) =
                has ? make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]) : make_uint4(0, 0, 0, 0);
        }
      }
      ml[t * kBM + row] = make_float4(m, l, (float)r, 0.0f);
      asm volatile("bar.sync 1, 256;" ::: "memory");
      constexpr int kRuns = D / 4;
      const float* base = reinterpret_cast<const float*>(smem);
      const int slot0 = bar->slot0, split = bar->split;
      float4* part = reinterpret_cast<float4*>(a.part);
      float4* mls = part + (int64_t)a.part_tiles * kBM * kRuns;
      for (int i = threadIdx.x; i < rows * kRuns; i += 256) {
        const int r = i / kRuns, c = i % kRuns;
        float4 x = *reinterpret_cast<const float4*>(base + r * D + ((c ^ (r & 7)) << 2));
        float M = ml[r].x, L = ml[r].y, R = ml[r].z;
        if constexpr (kOne) {                        // the two key sets
          const float4 o = ml[kBM + r];
          const float4 y = *reinterpret_cast<const float4*>(base + (kBM + r) * D + ((c ^ (r & 7)) << 2));
          const float M2 = fmaxf(M, o.x), R2 = floorf(fmaxf((M - M2) + R, (o.x - M2) + o.z));   // (as join_ref)
          const float w0 = fast_exp2(M - M2), w1 = fast_exp2(o.x - M2);
          const float v0 = fast_exp2((M - M2) + (R - R2)), v1 = fast_exp2((o.x - M2) + (o.z - R2));
          x = make_float4(fmaf(x.x, v0, y.x * v1), fmaf(x.y, v0, y.y * v1), fmaf(x.z, v0, y.z * v1), fmaf(x.w, v0, y.w * v1));
          L = fmaf(L, w0, o.y * w1);
          M = M2;
          R = R2;
        }
        if (n_splits == 1) {
          *reinterpret_cast<uint2*>(out_row(r) + 4 * c) = Normal(L, (int)R).bf16x4(x);
        } else {
          part[((int64_t)slot0 * kBM + r) * kRuns + c] = x;
          if (c == 0) mls[(int64_t)slot0 * kBM + r] = make_float4(M, L, R, 0.0f);
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kWarpMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(bar->tmem_base), "r"(kTmemCols) : "memory");
  }
}

// Joins the key splits of the chunk kernel: a warp for a row.  (A kernel of its own: the last of 18 splits took 27 us to join
// 128 rows by itself.)  With M = max m, R from join_ref: O = 2^R sum 2^(m - M) 2^(r - R) O_s / sum 2^(m - M) l_s.
template <int D>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ PagedAttnArgs a, int tiles) {
  constexpr int kRuns = D / 4, kFly = 4;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int place = (int)blockIdx.x * 8 + warp, shift = tiles == 2 ? 8 : 7;   // row of the split items' rows; tiles 128 = 2^shift
  static_assert(kBM == 128, "shift");
  int s = 0;
  for (int hi = a.seqs.n - 1; s < hi;) {
    const int mid = (s + hi + 1) >> 1;
    if (a.seqs.join0[mid] <= place >> shift) s = mid;
    else hi = mid - 1;
  }
  // `pair` counts the (rows, kv head) pairs of the sequence as the chunk kernel does, unsplit ones first
  const int n_splits = a.seqs.splits[s], whole = a.seqs.whole[s], n_rows = a.seqs.n_q[s] * a.G;
  const int groups = (n_rows + tiles * kBM - 1) >> shift;
  const int split_pair = (place >> shift) - a.seqs.join0[s], r = place & (tiles * kBM - 1);
  const int pair = whole + split_pair, kvh = pair % a.Hkv, row = (groups - 1 - pair / a.Hkv) * (tiles * kBM) + r;
  if (s >= a.seqs.n || pair >= groups * a.Hkv || row >= n_rows) return;
  const float4* part = reinterpret_cast<const float4*>(a.part);
  const float4* mls = part + (int64_t)a.part_tiles * kBM * kRuns;
  const int64_t first = ((int64_t)a.seqs.part0[s] + (int64_t)split_pair * n_splits * tiles) * kBM + r;   // split 0's row
  const int64_t next = (int64_t)tiles * kBM;
  wait_for_parts();
  // (m, l, r) of the first 32 splits are asked for once
  const float4 e0 = lane < n_splits ? __ldcg(mls + first + lane * next) : make_float4(kNoMax, 0.0f, (float)kNoRef, 0.0f);
  float M = e0.x, R = e0.z, L = 0.0f;
  for (int sp = lane + 32; sp < n_splits; sp += 32) {
    const float4 e = __ldcg(mls + first + sp * next);
    M = fmaxf(M, e.x);
    R = fmaxf(R, e.z);
  }
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) {
    M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
    R = fmaxf(R, __shfl_xor_sync(0xffffffffu, R, off));
  }
  R = join_ref(M, R, e0, n_splits, [&](int sp) { return __ldcg(mls + first + sp * next); });
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int s0 = 0; s0 < n_splits; s0 += 32) {        // weights of 32 splits, a lane each
    float w = 0.0f;
    if (s0 + lane < n_splits) {
      const float4 e = s0 == 0 ? e0 : __ldcg(mls + first + (s0 + lane) * next);
      L = fmaf(fast_exp2(e.x - M), e.y, L);
      w = fast_exp2((e.x - M) + (e.z - R));
    }
    const int n = min(32, n_splits - s0);
    for (int k0 = 0; k0 < n; k0 += kFly) {
      float4 x[kFly];
#pragma unroll
      for (int k = 0; k < kFly; ++k)
        x[k] = k0 + k < n && lane < kRuns ? __ldcg(part + (first + (s0 + k0 + k) * next) * kRuns + lane) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < kFly; ++k) {
        const float f = __shfl_sync(0xffffffffu, w, (k0 + k) & 31);
        acc = make_float4(fmaf(f, x[k].x, acc.x), fmaf(f, x[k].y, acc.y), fmaf(f, x[k].z, acc.z), fmaf(f, x[k].w, acc.w));
      }
    }
  }
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) L += __shfl_xor_sync(0xffffffffu, L, off);
  const int tok = a.by_g.div(row);
  bf16* o = a.O + ((int64_t)a.seqs.q0[s] + tok) * a.ostride + (int64_t)(kvh * a.G + row - tok * a.G) * D;
  if (lane < kRuns)
    *reinterpret_cast<uint2*>(o + 4 * lane) = Normal(L, (int)R).bf16x4(acc);
}

}  // namespace

cudaError_t paged_chunk_prepare(int D) {
  cudaError_t e = cudaSuccess;
  for (int one = 0; one < 2 && e == cudaSuccess; ++one) {
    if (D == 128)
      e = cudaFuncSetAttribute(one ? chunk_kernel<128, true> : chunk_kernel<128, false>,
                               cudaFuncAttributeMaxDynamicSharedMemorySize, ChunkLayout<128>::kSmem);
    else
      e = cudaFuncSetAttribute(one ? chunk_kernel<64, true> : chunk_kernel<64, false>,
                               cudaFuncAttributeMaxDynamicSharedMemorySize, ChunkLayout<64>::kSmem);
  }
  return e;
}

cudaError_t launch_paged_chunk(int D, bool one_tile, const CUtensorMap& tmK, const CUtensorMap& tmV,
                               const PagedAttnArgs& a, cudaStream_t s) {
  const unsigned grid = (unsigned)a.seqs.item0[a.seqs.n];
  if (grid == 0) return cudaSuccess;
  if (D == 128) {
    if (one_tile) chunk_kernel<128, true><<<grid, kChunkThreads, ChunkLayout<128>::kSmem, s>>>(tmK, tmV, a);
    else chunk_kernel<128, false><<<grid, kChunkThreads, ChunkLayout<128>::kSmem, s>>>(tmK, tmV, a);
  } else {
    if (one_tile) chunk_kernel<64, true><<<grid, kChunkThreads, ChunkLayout<64>::kSmem, s>>>(tmK, tmV, a);
    else chunk_kernel<64, false><<<grid, kChunkThreads, ChunkLayout<64>::kSmem, s>>>(tmK, tmV, a);
  }
  const int tiles = one_tile ? 1 : 2;
  if (const unsigned pairs = (unsigned)a.seqs.join0[a.seqs.n]) {       // 8 rows to a CTA
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_join(D == 128 ? join_kernel<128> : join_kernel<64>, dim3(pairs * (tiles * kBM / 8)), 256, s, a, tiles);
  }
  return cudaGetLastError();
}

}  // namespace fk
