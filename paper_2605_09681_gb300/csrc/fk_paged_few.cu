// Attention of a few queries over the paged 8-bit cache (single tokens, drafted tokens): the bytes of the cache
// bound it, so the keys are split over as many CTAs as the device holds and every byte is loaded once.
//   S = q k^T 2^(e_q + e_k) log2(e) scale,  p = 2^(S - m),  l = sum p,  O = 2^r sum p 2^(e_v - r) v / l
// with v the codes' values.
// CTA = (sequence, up to 8 kN query rows of one kv head's group, key split): warp 4 streams tiles of 64 keys and
// values into a ring (TMA, 2 boxes of a page's rows where pages are smaller); warps 0-3 take 16 keys of
// each tile by themselves, with their own running maximum m, sum l and O, and meet only at the end.
//   products  mma.m16n8k16 in f16, keys and values as the 16-row operand (S^T = K Q^T, O^T = V^T P^T), so that 8 query rows
//             fill an instruction and half the accumulators do (16 query rows as the 16-row operand: 168 registers, two
//             CTAs to an SM).  E4M3 codes are f16 values exactly, and a query row scaled by 2^-e_q (bf16 has fewer bits
//             than f16) is too, so that S is exact up to fp32 sums; p 2^(e_v - r) is rounded to f16 (11 bits) and
//             turned into the other operand's layout by movmatrix.  The tensor-memory path would need 128 query rows
//             to be worth its hand-overs.
//   layout    an MMA's inner index and its rows may be permuted at will, so that each lane reads whole 16-byte
//             runs of a row from shared memory and converts them in place: row n of a 16-key group is key
//             tok(n) = n (n even) or ((n - 1) ^ 4) + 1 (n odd), and with the 128-byte swizzle no two lanes of a
//             quarter warp then meet in a bank, neither for keys (4 lanes on a row) nor for values (2 runs of 4 rows).
//   scales    e_k is in the factor of the exponent and e_v - r in its summand (r: see kRefWindow), so no key or value
//             is scaled.  m is raised only when a row outgrows it by 2^4: a vote finds that no row does, without a maximum
//             over lanes, and O is seldom rescaled.  r is one for a warp's rows: it goes with a block outside its window if all rows hold
//             nothing yet, or see large p there, or it is near, and if O has room.  Where that does not hold (blocks of values that
//             differ by 2^74 and more, or by less with rows that give the larger next to nothing) the CTA does its rows again by
//             exact_rows, 30 times as slowly (131072 keys in pages 10^50 apart: 1.6 ms).  (References of the rows' own, held in
//             shared memory, cost every call 4-7%.)
// What bounds it: the cache's bytes.  One token of 32 heads over 131072 keys of 8 kv heads (268 MB of codes) 51 us, 5.2 TB/s, where
// reading those bytes and nothing else takes 42.8; 64 streams of 500 to 7000 keys (489 MB) 83 us, 5.9 TB/s (76.4).  With
// little to read the launch and the join do: one token of 12 heads over 1561 keys 6.5-6.9 us.  At 16 rows its products and
// conversions bound it (16 sequences of up to 96 rows of 64 channels, 200 to 4000 keys: 14.5 us).
// Splits leave (m, l, r, O) in a workspace; the last one to arrive (8 rows) or a kernel of its own (16) joins them in the order of
// the splits (no atomics on values: results do not change from run to run).
#include "fk_paged_rows.h"

namespace fk {
namespace {

constexpr int kWarps = 4;                             // consumer warps; one more loads
constexpr int kFewThreads = (kWarps + 1) * 32;
constexpr int kStages = 4;
constexpr float kLowest = -3.402823466e38f;           // m before any key: finite, so that 2^(-inf - m) is 0
constexpr float kRaise = 4.0f;                        // log2 units by which a row may outgrow m
// A warp whose rows did not go together; how far the warps' references may lie apart; how far moves down may lift O in all (log2: at most
// 2^(9 + kRaised) l), and one move up press it
constexpr int kApart = 1 << 20, kCloseRefs = 100, kRaised = 74, kFall = 100;
constexpr float kShiftP = 8.0f;                       // p is stored times 2^8: at most 2^12 in f16

template <int D>
struct FewLayout {
  static constexpr int kTile = kPagedFewTile * D;     // bytes of a key (or value) tile
  static constexpr int kOffK = 0;
  static constexpr int kOffV = kOffK + kStages * kTile;
  static constexpr int kOffBar = kOffV + kStages * kTile;
  static constexpr int kSmem = kOffBar + 256 + 1024;
  static_assert(kWarps * kPagedFewRows * D * 4 <= kOffBar, "the warps' O over the stages");
  static_assert(kMaxFewSplits * kPagedFewRows * 4 + kFewThreads * 16 <= 8 * kPagedFewTile * D, "the join's numbers over the stages");
};

struct FewBarriers {
  uint64_t full[kStages], empty[kStages];
  int last;
  volatile int abort;
};

// D += A B, A 16 x 16 (row), B 16 x 8 (column), f16 in, f32 out
__device__ __forceinline__ void mma16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the transpose of an 8 x 8 matrix of 16-bit elements, two of a row to a lane
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// 2^k in 64 bits, k in [-1022, 1023]
__device__ __forceinline__ double pow2_double(int k) { return __hiloint2double((1023 + k) << 20, 0); }
// byte offset of 16-byte run c of row `row` in a tile (TMA swizzle of the row length)
template <int D>
__device__ __forceinline__ int run_at(int row, int c) {
  return D == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
}

// A CTA's rows over its key tiles once more, O in 64 bits and without references: where the blocks of values of its keys differ by more
// than the rows can go through together.  A warp to a row, 32 keys (of one block) at a time.  Writes what the tensor-core path would: O, or O and (m, l, r) to part and mls.
template <int D>
__device__ __forceinline__ void exact_rows(const PagedAttnArgs& a, int s, int kvh, int row0, int rows, TileRange tr, int i0, int i1,
                                        float* part, float4* mls, uint8_t* smem) {
  constexpr int kC = D / 32;                            // channels of a lane
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n_keys = a.seqs.n_keys[s], p_first = n_keys - a.seqs.n_q[s], last_page = max(n_keys - 1, 0) / a.P;
  const int* table = a.table + (int64_t)a.seqs.slot[s] * a.max_pages;
  float* q = reinterpret_cast<float*>(smem) + warp * D;
#pragma unroll 1
  for (int row = warp; row < rows; row += kWarps + 1) {
    const int rr = row0 + row, tok = a.by_g.div(rr), pos = p_first + tok;
    const int64_t at = (int64_t)(kvh * a.G + rr - tok * a.G) * D + kC * lane;
    const bf16* src = a.Q + ((int64_t)a.seqs.q0[s] + tok) * a.qstride + at;
    const int limit = a.mask.causal ? min(pos + 1, n_keys) : n_keys, lower = a.mask.window > 0 ? pos - a.mask.window + 1 : 0;
    float top = 0.0f;
    bool fine = true;
    for (int c = 0; c < kC; ++c) {
      const float x = __bfloat162float(src[c]);
      fine = fine && fabsf(x) <= 3.402823466e38f;
      top = fmaxf(top, fabsf(x));
    }
    for (int off = 16; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    fine = __all_sync(0xffffffffu, fine);
    const int eq = fine ? e4m3_row_exponent(top) : 0;
    __syncwarp();
    for (int c = 0; c < kC; ++c) q[kC * lane + c] = fine ? __bfloat162float(src[c]) * pow2f(-eq) : 0.0f;
    __syncwarp();
    double o[kC] = {}, l = 0.0;
    float m = kLowest;
#pragma unroll 1
    for (int i = 2 * i0; i < 2 * i1; ++i) {
      const int key = tr.at(i >> 1) * kPagedFewTile + (i & 1) * 32 + lane;
      const int64_t block = (int64_t)__ldg(table + min(key / a.P, last_page)) * a.Hkv + kvh, place = (block * a.P + key % a.P) * D;
      const bool seen = key < limit && (key >= lower || key < a.mask.sinks);
      float x = -INFINITY;
      if (seen) {
        float dot = 0.0f;
#pragma unroll 1
        for (int c = 0; c < D; c += 4) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(a.k + place + c);
          const uint32_t h0 = f16x2_of_e4m3x2((uint16_t)w), h1 = f16x2_of_e4m3x2((uint16_t)(w >> 16));
          const float2 k0 = __half22float2(*reinterpret_cast<const __half2*>(&h0)), k1 = __half22float2(*reinterpret_cast<const __half2*>(&h1));
          dot = fmaf(q[c], k0.x, fmaf(q[c + 1], k0.y, fmaf(q[c + 2], k1.x, fmaf(q[c + 3], k1.y, dot))));
        }
        x = (float)fmin(fmax((double)dot * a.scale_log2 * pow2_double(eq + a.ke[block]), -3e38), 3e38);
      }
      float mx = x;
      for (int off = 16; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
      if (!(mx > -INFINITY)) continue;
      if (mx > m) {
        const double al = exp2((double)m - mx);
        m = mx;
        l *= al;
        for (int c = 0; c < kC; ++c) o[c] *= al;
      }
      const float p = seen ? exp2f(x - m) : 0.0f;
      l += p;
      float sum[kC] = {};
#pragma unroll 1
      for (int k = 0; k < 32; ++k) {
        const float w = __shfl_sync(0xffffffffu, p, k);
        const int64_t pk = __shfl_sync(0xffffffffu, place, k);
        for (int c = 0; c < kC; c += 2) {
          const uint32_t h = f16x2_of_e4m3x2(*reinterpret_cast<const uint16_t*>(a.v + pk + kC * lane + c));
          const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
          sum[c] = fmaf(w, v.x, sum[c]);
          sum[c + 1] = fmaf(w, v.y, sum[c + 1]);
        }
      }
      const double size = pow2_double(a.ve[block]);       // (of one block)
      for (int c = 0; c < kC; ++c) o[c] = fma((double)sum[c], size, o[c]);
    }
    for (int off = 16; off >= 1; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
    if (!part) {                                        // no visible key: 0; infinities or NaN in the query: NaN
      bf16* out = a.O + ((int64_t)a.seqs.q0[s] + tok) * a.ostride + at;
      for (int c = 0; c < kC; ++c) out[c] = __float2bfloat16_rn(!fine ? NAN : l > 0.0 ? (float)(o[c] / l) : 0.0f);
      continue;
    }
    double most = 0.0;                                  // r: the exponent of the largest |O|
    for (int c = 0; c < kC; ++c) most = fmax(most, fabs(o[c]));
    for (int off = 16; off >= 1; off >>= 1) most = fmax(most, __shfl_xor_sync(0xffffffffu, most, off));
    const int r = most > 0.0 ? min(max(ilogb(most), -110), 110) : kNoRef;
    for (int c = 0; c < kC; ++c) part[(int64_t)row * D + kC * lane + c] = r == kNoRef ? 0.0f : (float)(o[c] * pow2_double(-r)) * (1 << (int)kShiftP);
    if (lane == 0) mls[row] = make_float4(m, fine ? (float)(l * (1 << (int)kShiftP)) : NAN, (float)r, 0.0f);
  }
}

template <int D, int kN>
__global__ void __launch_bounds__(kFewThreads, kN == 1 ? 3 : 2)
few_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
           const __grid_constant__ PagedAttnArgs a) {
  using Lay = FewLayout<D>;
  constexpr int kRows = 8 * kN, kT = kPagedFewTile;
  constexpr int kSteps = D / 16;                      // inner steps of S^T
  constexpr int kRowTiles = D / 16;                   // row tiles of O^T
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sK = smem + Lay::kOffK;
  uint8_t* sV = smem + Lay::kOffV;
  FewBarriers* bar = reinterpret_cast<FewBarriers*>(smem + Lay::kOffBar);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int kvh = blockIdx.y;

  // ---- this CTA's rows and key tiles
  int s = 0;
  for (int hi = a.seqs.n - 1; s < hi;) {              // the last one whose items begin at or before this one
    const int mid = (s + hi + 1) >> 1;
    if (a.seqs.item0[mid] <= (int)blockIdx.x) s = mid;
    else hi = mid - 1;
  }
  const int n_keys = a.seqs.n_keys[s], n_q = a.seqs.n_q[s], n_splits = a.seqs.splits[s];
  const int n_rows = n_q * a.G;
  const int item = blockIdx.x - a.seqs.item0[s];
  const int split = item % n_splits, row0 = (item / n_splits) * kRows;
  const int rows = min(kRows, n_rows - row0);
  const int p_first = n_keys - n_q;                    // position of query 0
  const int pos0 = p_first + a.by_g.div(row0), pos1 = p_first + a.by_g.div(row0 + rows - 1);
  const TileRange tr = paged_tiles(n_keys, pos0, pos1, a.mask, kT);
  const int n_tiles = tr.count();
  const int i0 = (int)((int64_t)n_tiles * split / n_splits), i1 = (int)((int64_t)n_tiles * (split + 1) / n_splits);
  const int* table = a.table + (int64_t)a.seqs.slot[s] * a.max_pages;
  const int last_page = max(n_keys - 1, 0) / a.P;

  if (threadIdx.x == kWarps * 32) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&bar->full[i], 1);
      mbar_init(&bar->empty[i], kWarps);
    }
    bar->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();

  float m[kN][2], l[kN][2];                             // of rows 8 j + 2 t, + 1 (l: this lane's keys only)
  float o[kN][kRowTiles][4];
#pragma unroll
  for (int j = 0; j < kN; ++j) {
#pragma unroll
    for (int c = 0; c < kRowTiles; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[j][c][i] = 0.0f;
    m[j][0] = m[j][1] = kLowest;
    l[j][0] = l[j][1] = 0.0f;
  }
  int r = kNoRef, raised = 0;                           // reference of the warp's O, and by how much moves down have lifted O
  bool zeros = false, edge = false, apart = false;      // see below
  const int g = lane >> 2, t = lane & 3;

  if (warp == kWarps) {
    // ------------------------------------------------------------------ loads
    const int box = min(a.P, kT), boxes = kT / box;     // rows of a page in a tile
    int y0 = 0, y1 = 0;                                 // lane: rows of the boxes of tile i0 + 32 n + lane
    bool ok = true;
    int i = i0;
    for (; i < i1; ++i) {
      const int k = i - i0;
      if ((k & 31) == 0) {
        const int key = tr.at(min(i + lane, i1 - 1)) * kT;
        y0 = (__ldg(table + min(key / a.P, last_page)) * a.Hkv + kvh) * a.P + key % a.P;
        if (boxes == 2) y1 = (__ldg(table + min((key + box) / a.P, last_page)) * a.Hkv + kvh) * a.P;
      }
      const int st = k % kStages, u = k / kStages;
      if (u > 0 && !warp_wait(&bar->empty[st], (u - 1) & 1, bar, a.status)) { ok = false; break; }
      const int ya = __shfl_sync(0xffffffffu, y0, k & 31), yb = __shfl_sync(0xffffffffu, y1, k & 31);
      if (elect_one()) {
        mbar_expect_tx(&bar->full[st], 2 * Lay::kTile);
        tma_load_2d(sK + st * Lay::kTile, &tmK, &bar->full[st], 0, ya);
        tma_load_2d(sV + st * Lay::kTile, &tmV, &bar->full[st], 0, ya);
        if (boxes == 2) {
          tma_load_2d(sK + st * Lay::kTile + box * D, &tmK, &bar->full[st], 0, yb);
          tma_load_2d(sV + st * Lay::kTile + box * D, &tmV, &bar->full[st], 0, yb);
        }
      }
      __syncwarp();
    }
    if (!ok)                                            // loads in flight land before the CTA ends
      for (int k = max(0, i - i0 - kStages); k < i - i0; ++k)
        wait_phase(&bar->full[k % kStages], (k / kStages) & 1, bar, a.status, false);
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ this lane's part of the queries
    // B fragment: row 8 j + g, inner step st: channels base + 4 w + {0, 1} and + {2, 3}, base and w as the lane's runs
    // of a key row: run t (16 t ..) for the first four steps, run t + 4 (64 + 16 t ..) for the others
    uint32_t q[kN][kSteps][2];
    float sc[kN][2];                                    // of rows 8 j + 2 t, + 1
    int limit[kN][2], lower[kN][2];                     // visible keys: [lower, limit) and those below `sinks`
    const bf16* qbase = a.Q + (int64_t)a.seqs.q0[s] * a.qstride + (int64_t)kvh * a.G * D;
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const int row = 8 * j + g, rr = row0 + min(row, rows - 1), tok = a.by_g.div(rr);
      const bf16* src = qbase + (int64_t)tok * a.qstride + (int64_t)(rr - tok * a.G) * D + 16 * t;
      uint4 v[D / 32];
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        v[2 * c] = __ldg(reinterpret_cast<const uint4*>(src + 64 * c));
        v[2 * c + 1] = __ldg(reinterpret_cast<const uint4*>(src + 64 * c) + 1);
      }
      uint32_t top = 0;                                 // largest magnitude as bf16 bits
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
        top = __vmaxu2(top, __vmaxu2(__vmaxu2(v[c].x & 0x7FFF7FFFu, v[c].y & 0x7FFF7FFFu), __vmaxu2(v[c].z & 0x7FFF7FFFu, v[c].w & 0x7FFF7FFFu)));
      top = max(top & 0xFFFFu, top >> 16);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const bool fine = top < 0x7F80u;
      const int e = fine ? e4m3_row_exponent(__uint_as_float(top << 16)) : 0;
      const float inv = pow2f(-e);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        const uint32_t w[4] = {v[c].x, v[c].y, v[c].z, v[c].w};
#pragma unroll
        for (int i = 0; i < 4; ++i)                     // channels 8 c' + 2 i, + 1
          q[j][2 * c + (i >> 1)][i & 1] = pack_f16(__uint_as_float(w[i] << 16) * inv, __uint_as_float(w[i] & 0xFFFF0000u) * inv);
      }
      // what belongs to row 8 j + g, to the lanes that hold its sums
      const float scale = fine ? a.scale_log2 * pow2f(e) : NAN;
      const int pos = p_first + tok, lim = row >= rows ? 0 : a.mask.causal ? min(pos + 1, n_keys) : n_keys;
      const int low = a.mask.window > 0 ? pos - a.mask.window + 1 : 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int from = (2 * t + h) * 4;
        sc[j][h] = __shfl_sync(0xffffffffu, scale, from);
        limit[j][h] = __shfl_sync(0xffffffffu, lim, from);
        lower[j][h] = __shfl_sync(0xffffffffu, low, from);
        if (sc[j][h] != sc[j][h]) {                     // infinities or NaN: the row's O is NaN
          l[j][h] = NAN;
          sc[j][h] = 0.0f;
        }
      }
    }
    // a tile without a masked key for any row of the CTA: [full_lo, full_hi), or all below the sinks
    const int full_hi = a.mask.causal ? min(pos0 + 1, n_keys) : n_keys;
    const int full_lo = a.mask.window > 0 ? pos1 - a.mask.window + 1 : 0;
    const int krow = warp * 16 + ((g & 1) ? ((g ^ 1) ^ 4) + 1 : g);   // key row of MMA row g
    const int va = warp * 16 + 2 * t, vb = warp * 16 + ((2 * t) ^ 4) + 1;

    int packed = 0;                                     // lane: exponents of this warp's block of tile i0 + 32 n + lane
    for (int i = i0; i < i1; ++i) {
      const int k = i - i0, st = k % kStages;
      if ((k & 31) == 0) {
        const int key = tr.at(min(i + lane, i1 - 1)) * kT + warp * 16;
        const int64_t block = (int64_t)__ldg(table + min(key / a.P, last_page)) * a.Hkv + kvh;
        packed = (int)(uint8_t)a.ke[block] | (int)a.ve[block] << 8;
      }
      const int both = __shfl_sync(0xffffffffu, packed, k & 31), ek = (int)(int8_t)both, ev = both >> 8;
      if (!warp_wait(&bar->full[st], (k / kStages) & 1, bar, a.status)) break;
      const uint8_t* kt = sK + st * Lay::kTile;
      const uint8_t* vt = sV + st * Lay::kTile;
      // S^T of the warp's 16 keys (rows g and g + 8), in two chains
      float sv[kN][4];
      {
        uint4 ka[D / 64], kb[D / 64];
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          ka[c] = *reinterpret_cast<const uint4*>(kt + run_at<D>(krow, t + 4 * c));
          kb[c] = *reinterpret_cast<const uint4*>(kt + run_at<D>(krow + 8, t + 4 * c));
        }
        float s2[kN][4];
#pragma unroll
        for (int j = 0; j < kN; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) sv[j][x] = s2[j][x] = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          const uint32_t wa[4] = {ka[c].x, ka[c].y, ka[c].z, ka[c].w}, wb[4] = {kb[c].x, kb[c].y, kb[c].z, kb[c].w};
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint32_t a0 = f16x2_of_e4m3x2((uint16_t)wa[x]), a2 = f16x2_of_e4m3x2((uint16_t)(wa[x] >> 16));
            const uint32_t a1 = f16x2_of_e4m3x2((uint16_t)wb[x]), a3 = f16x2_of_e4m3x2((uint16_t)(wb[x] >> 16));
#pragma unroll
            for (int j = 0; j < kN; ++j)
              mma16816(x & 1 ? s2[j] : sv[j], a0, a1, a2, a3, q[j][4 * c + x][0], q[j][4 * c + x][1]);
          }
        }
#pragma unroll
        for (int j = 0; j < kN; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) sv[j][x] += s2[j][x];
      }
      // the values' loads are under way meanwhile
      uint4 w[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int row = (x & 1 ? vb : va) + (x >> 1) * 8;
        if constexpr (D == 128) {
          w[x] = *reinterpret_cast<const uint4*>(vt + run_at<D>(row, g));
        } else {
          const uint2 y = *reinterpret_cast<const uint2*>(vt + run_at<D>(row, g >> 1) + (g & 1) * 8);
          w[x] = make_uint4(y.x, y.y, 0, 0);
        }
      }
      // scale and mask: keys krow (x = 0, 1) and krow + 8 (2, 3), rows 2 t (0, 2) and 2 t + 1 (1, 3)
      const float ske = pow2f(ek);
      const int j0 = tr.at(i) * kT;
      const bool full = j0 + kT <= full_hi && (j0 >= full_lo || j0 + kT <= a.mask.sinks);
      bool grows = false;
#pragma unroll
      for (int j = 0; j < kN; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float c = fminf(sc[j][h] * ske, 3e38f);  // (codes may all be 0)
          sv[j][h] *= c;
          sv[j][2 + h] *= c;
          if (!full) {
            const int x = j0 + krow, y = x + 8;
            if (x >= limit[j][h] || (x < lower[j][h] && x >= a.mask.sinks)) sv[j][h] = -INFINITY;
            if (y >= limit[j][h] || (y < lower[j][h] && y >= a.mask.sinks)) sv[j][2 + h] = -INFINITY;
          }
          grows |= fmaxf(sv[j][h], sv[j][2 + h]) > m[j][h] + kRaise;
        }
      const bool move = ev != kZeroExp && (ev > r || ev < r - kRefWindow);   // warp-uniform
      zeros |= ev == kZeroExp;
      edge |= move && !full;
      if (__any_sync(0xffffffffu, grows || move)) {
        const int to = ev + kRefRoom;
        bool seen = false, go = raised + r - to <= kRaised && (to - r <= kFall || r == kNoRef);
#pragma unroll
        for (int j = 0; j < kN; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float mx = fmaxf(sv[j][h], sv[j][2 + h]);    // over the 16 keys
#pragma unroll
            for (int off = 4; off <= 16; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            const float mn = fmaxf(m[j][h], mx);
            seen |= mx > -INFINITY;
            go &= r == kNoRef || m[j][h] == kLowest || 8 * j + 2 * t + h >= rows || to <= r + kAbove || mx - mn >= kAskPast;
            const float al = fast_exp2(m[j][h] - mn);
            m[j][h] = mn;
            l[j][h] *= al;
#pragma unroll
            for (int c = 0; c < kRowTiles; ++c) {
              o[j][c][h] *= al;
              o[j][c][2 + h] *= al;
            }
          }
        if (move && __any_sync(0xffffffffu, seen)) {     // the rows go together, or not at all
          apart |= !__all_sync(0xffffffffu, go);
          const float f = pow2_any(r - to);
          raised = r == kNoRef ? 0 : max(0, raised + r - to);
          r = to;
#pragma unroll
          for (int j = 0; j < kN; ++j)
#pragma unroll
            for (int c = 0; c < kRowTiles; ++c)
#pragma unroll
              for (int x = 0; x < 4; ++x) o[j][c][x] *= f;
        }
      }
      // (a block of which no row sees a key may still be far from r: its numerators are 0)
      const int d = ev == kZeroExp ? 0 : min(max(ev - r, -kRefWindow), 0);
      const float we = kShiftP + (float)d, fl = pow2f(-d);
      uint32_t p0[kN], p1[kN];
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        const float za = we - m[j][0], zb = we - m[j][1];
        const float x0 = fast_exp2(sv[j][0] + za), x1 = fast_exp2(sv[j][1] + zb);
        const float x2 = fast_exp2(sv[j][2] + za), x3 = fast_exp2(sv[j][3] + zb);
        l[j][0] = fmaf(x0 + x2, fl, l[j][0]);
        l[j][1] = fmaf(x1 + x3, fl, l[j][1]);
        p0[j] = transpose8(pack_f16(x0, x1));            // lane: row g, keys of MMA rows 2 t, 2 t + 1
        p1[j] = transpose8(pack_f16(x2, x3));            // and 2 t + 8, 2 t + 9
      }
      // O^T += V^T P^T: row tile 2 x + y: channels of the lane's run, 4 x + 2 y (rows g) and + 1 (rows g + 8)
#pragma unroll
      for (int x = 0; x < kRowTiles / 2; ++x) {
        const uint32_t wa[2] = {x == 0 ? w[0].x : x == 1 ? w[0].y : x == 2 ? w[0].z : w[0].w,
                                x == 0 ? w[2].x : x == 1 ? w[2].y : x == 2 ? w[2].z : w[2].w};
        const uint32_t wb[2] = {x == 0 ? w[1].x : x == 1 ? w[1].y : x == 2 ? w[1].z : w[1].w,
                                x == 0 ? w[3].x : x == 1 ? w[3].y : x == 2 ? w[3].z : w[3].w};
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t lo = __byte_perm(wa[0], wb[0], y ? 0x7362 : 0x5140), hi = __byte_perm(wa[1], wb[1], y ? 0x7362 : 0x5140);
          const uint32_t a0 = f16x2_of_e4m3x2((uint16_t)lo), a1 = f16x2_of_e4m3x2((uint16_t)(lo >> 16));
          const uint32_t a2 = f16x2_of_e4m3x2((uint16_t)hi), a3 = f16x2_of_e4m3x2((uint16_t)(hi >> 16));
#pragma unroll
          for (int j = 0; j < kN; ++j) mma16816(o[j][2 * x + y], a0, a1, a2, a3, p0[j], p1[j]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar->empty[st]);
    }
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int off = 4; off <= 16; off <<= 1) l[j][h] += __shfl_xor_sync(0xffffffffu, l[j][h], off);
  }
  if constexpr (kN == 2) allow_join();
  __syncthreads();                                      // every tile has been read: the stages are free

  // ---- the warps' (m, l, r) and O
  float* sO = reinterpret_cast<float*>(smem);           // [warp][row][D], 16-byte run c of row at c ^ (row & 7)
  __shared__ float sm[kWarps][kRows], sl[kWarps][kRows];
  __shared__ int sr[kWarps];                            // reference (kApart: what the warp holds is of no use)
  if (warp < kWarps) {
    if (raised > 0) {                                   // back to the reference of what O holds
      const float f = pow2_any(-raised);
#pragma unroll
      for (int j = 0; j < kN; ++j)
#pragma unroll
        for (int c = 0; c < kRowTiles; ++c)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[j][c][x] *= f;
      r += raised;
    }
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = 8 * j + 2 * t + h;
        float* dst = sO + (warp * kRows + row) * D;
        // channels D/8 g .. + D/8 - 1
#pragma unroll
        for (int c = 0; c < kRowTiles; c += 2) {
          const int run = D / 32 * g + c / 2;
          *reinterpret_cast<float4*>(dst + ((run ^ (row & 7)) << 2)) = make_float4(o[j][c][h], o[j][c][2 + h], o[j][c + 1][h], o[j][c + 1][2 + h]);
        }
        if (g == 0) {
          sm[warp][row] = m[j][h];
          sl[warp][row] = l[j][h];
        }
      }
    // (A row that took a block's reference without seeing it, and then saw blocks of zeros, holds nothing of that size.)
    apart |= zeros && edge;
    if (lane == 0) {
      sr[warp] = apart ? kApart : r;
    }
  }
  __syncthreads();
  // O of the CTA relative to (M, 2^R): weights 2^(m_w - M) 2^(r_w - R)
  int r_low = INT_MAX, R = kNoRef;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    R = max(R, sr[w]);
    if (sr[w] != kNoRef) r_low = min(r_low, sr[w]);
  }
  const int cta = a.seqs.part0[s] + kvh * (a.seqs.item0[s + 1] - a.seqs.item0[s]) + item;   // workspace slot
  constexpr int kRuns = D / 4;
  auto out_row = [&](int row) {
    const int rr = row0 + row, tok = a.by_g.div(rr);
    return a.O + ((int64_t)a.seqs.q0[s] + tok) * a.ostride + (int64_t)(kvh * a.G + rr - tok * a.G) * D;
  };
  float4* part = reinterpret_cast<float4*>(a.part);                     // [slot][row][run]
  float4* mls = part + (int64_t)kPartSlots * kPagedFewRows * kRuns;     // [slot][row]: m, l, r
  const bool together = R < kApart && R - r_low <= kCloseRefs;
  if (!together) {
    __syncthreads();                                    // (the numbers above have been read)
    exact_rows<D>(a, s, kvh, row0, rows, tr, i0, i1, n_splits > 1 ? a.part + (int64_t)cta * kPagedFewRows * D : nullptr,
                  mls + cta * kPagedFewRows, smem);
  }
#pragma unroll 1
  for (int i = threadIdx.x; together && i < rows * kRuns; i += kFewThreads) {
    const int row = i / kRuns, c = i % kRuns;
    float M = kLowest, L = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm[w][row]);
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = fast_exp2(sm[w][row] - M), fo = f * pow2_any(sr[w] - R);
      const float4 x = *reinterpret_cast<const float4*>(sO + (w * kRows + row) * D + ((c ^ (row & 7)) << 2));
      L = fmaf(f, sl[w][row], L);
      acc.x = fmaf(fo, x.x, acc.x);
      acc.y = fmaf(fo, x.y, acc.y);
      acc.z = fmaf(fo, x.z, acc.z);
      acc.w = fmaf(fo, x.w, acc.w);
    }
    if (n_splits == 1) {
      *reinterpret_cast<uint2*>(out_row(row) + 4 * c) = Normal(L, R).bf16x4(acc);
    } else {
      part[((int64_t)cta * kPagedFewRows + row) * kRuns + c] = acc;
      if (c == 0) mls[cta * kPagedFewRows + row] = make_float4(M, L, (float)R, 0.0f);
    }
  }
  if (n_splits == 1 || kN == 2) return;

  // ---- the last split of the group joins them all.  The CTA's writes come before thread 0's release (barrier, then
  // an atomic of acquire and release at device scope), the others' before its acquire.
  __syncthreads();
  const int first = cta - split;                        // slot of split 0
  if (threadIdx.x == 0) {
    unsigned before;
    asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;"
                 : "=r"(before) : "l"(a.arrived + first), "r"((unsigned)(n_splits - 1)) : "memory");
    bar->last = before == (unsigned)(n_splits - 1);
  }
  __syncthreads();
  if (!bar->last) return;
  // each row's weights (join_ref), first (row by row, a warp each), then the sums.  What both need of the workspace
  // is asked for at once: its numbers of the first 32 splits, and the first twelve runs of a thread's sum.
  float* wts = reinterpret_cast<float*>(smem);          // [row][split]
  constexpr int kRowsEach = (kRows + kWarps) / (kWarps + 1), kFly = 12;
  float4 e0[kRowsEach];
#pragma unroll
  for (int k = 0; k < kRowsEach; ++k) {
    const int row = warp + k * (kWarps + 1);
    e0[k] = row < rows && lane < n_splits ? __ldcg(mls + (first + lane) * kPagedFewRows + row) : make_float4(kLowest, 0.0f, (float)kNoRef, 0.0f);
  }
  // A place (row, run) is summed by `sets` threads, each over every sets-th split, twelve loads in flight.
  const int places = rows * kRuns, sets = max(1, kFewThreads / places);
  const int set = sets > 1 ? (int)threadIdx.x / places : 0, i_first = sets > 1 ? (int)threadIdx.x % places : (int)threadIdx.x;
  float4 x[kFly];
  auto ask = [&](int i, int sp0) {
    const float4* src = part + ((int64_t)first * kPagedFewRows + i / kRuns) * kRuns + i % kRuns;
#pragma unroll
    for (int k = 0; k < kFly; ++k) {
      const int sp = sp0 + k * sets;
      if (sp < n_splits) x[k] = __ldcg(src + (int64_t)sp * kPagedFewRows * kRuns);
    }
  };
  if (i_first < places && set < sets) ask(i_first, set);
#pragma unroll
  for (int k = 0; k < kRowsEach; ++k) {
    const int row = warp + k * (kWarps + 1);
    if (row >= rows) break;
    float M = e0[k].x, RR = e0[k].z, L = 0.0f;
    for (int sp = lane + 32; sp < n_splits; sp += 32) {
      const float4 e = __ldcg(mls + (first + sp) * kPagedFewRows + row);
      M = fmaxf(M, e.x);
      RR = fmaxf(RR, e.z);
    }
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) {
      M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
      RR = fmaxf(RR, __shfl_xor_sync(0xffffffffu, RR, off));
    }
    RR = join_ref(M, RR, e0[k], n_splits, [&](int sp) { return __ldcg(mls + (first + sp) * kPagedFewRows + row); });
    for (int sp = lane; sp < n_splits; sp += 32) {
      const float4 e = sp == lane ? e0[k] : __ldcg(mls + (first + sp) * kPagedFewRows + row);
      L = fmaf(fast_exp2(e.x - M), e.y, L);
      wts[row * n_splits + sp] = fast_exp2((e.x - M) + (e.z - RR));
    }
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) L += __shfl_xor_sync(0xffffffffu, L, off);
    if (lane == 0) {
      sl[0][row] = L;
      sm[0][row] = RR;
    }
  }
  __syncthreads();
  float4* sums = reinterpret_cast<float4*>(smem + kMaxFewSplits * kPagedFewRows * 4);     // [set][place]
#pragma unroll 1
  for (int i0 = 0; i0 < places; i0 += kFewThreads) {
    const int i = i0 + i_first;
    const bool mine = i < places && set < sets;
    const int row = i / kRuns, c = i % kRuns;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (mine) {
#pragma unroll 1
      for (int sp = set; sp < n_splits; sp += kFly * sets) {
        if (i0 > 0 || sp > set) ask(i, sp);
#pragma unroll
        for (int k = 0; k < kFly; ++k)
          if (sp + k * sets < n_splits) {
            const float f = wts[row * n_splits + sp + k * sets];
            acc.x = fmaf(f, x[k].x, acc.x);
            acc.y = fmaf(f, x[k].y, acc.y);
            acc.z = fmaf(f, x[k].z, acc.z);
            acc.w = fmaf(f, x[k].w, acc.w);
          }
      }
    }
    if (sets > 1) {
      if (mine) sums[threadIdx.x] = acc;
      __syncthreads();
      if (mine && set == 0)
        for (int k = 1; k < sets; ++k) {
          const float4 y = sums[k * places + i];
          acc = make_float4(acc.x + y.x, acc.y + y.y, acc.z + y.z, acc.w + y.w);
        }
    }
    if (mine && set == 0) {
      *reinterpret_cast<uint2*>(out_row(row) + 4 * c) = Normal(sl[0][row], (int)sm[0][row]).bf16x4(acc);
    }
  }
}

// The same join by a kernel of its own, a warp for a row, for 16-row CTAs: one CTA would take long over the rows of many splits
// (two queries of 64 heads over 20000 keys of 8, one call after the other: 30.3 us, this 22.9; 16 streams' drafts 17.1, 16.5;
// without the early launch 24.6 and 18.6).  For 8 rows or fewer the last
// CTA is as good or better (two rows: 9.9 us, a kernel of its own 15.1).
template <int D>
__global__ void __launch_bounds__(512) few_join_kernel(const __grid_constant__ PagedAttnArgs a) {
  constexpr int kRuns = D / 4, kFly = 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, kvh = blockIdx.y;
  int s = 0;
  for (int hi = a.seqs.n - 1; s < hi;) {
    const int mid = (s + hi + 1) >> 1;
    if (a.seqs.item0[mid] <= (int)blockIdx.x) s = mid;
    else hi = mid - 1;
  }
  const int n_splits = a.seqs.splits[s], item = blockIdx.x - a.seqs.item0[s];
  wait_for_parts();
  const int row = item / n_splits * kPagedFewRows + warp;   // of the sequence's rows of this kv head
  if (n_splits == 1 || item % n_splits != 0 || row >= a.seqs.n_q[s] * a.G) return;
  const int first = a.seqs.part0[s] + kvh * (a.seqs.item0[s + 1] - a.seqs.item0[s]) + item;
  const float4* part = reinterpret_cast<const float4*>(a.part);
  const float4* mls = part + (int64_t)kPartSlots * kPagedFewRows * kRuns + (int64_t)first * kPagedFewRows + warp;
  part += ((int64_t)first * kPagedFewRows + warp) * kRuns + lane;
  const float4 none = make_float4(kLowest, 0.0f, (float)kNoRef, 0.0f);
  const float4 e0 = lane < n_splits ? __ldcg(mls + lane * kPagedFewRows) : none;
  float M = e0.x, R = e0.z, L = 0.0f;
  for (int sp = lane + 32; sp < n_splits; sp += 32) {
    const float4 e = __ldcg(mls + sp * kPagedFewRows);
    M = fmaxf(M, e.x);
    R = fmaxf(R, e.z);
  }
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) {
    M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
    R = fmaxf(R, __shfl_xor_sync(0xffffffffu, R, off));
  }
  R = join_ref(M, R, e0, n_splits, [&](int sp) { return __ldcg(mls + sp * kPagedFewRows); });
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int s0 = 0; s0 < n_splits; s0 += 32) {           // weights of 32 splits, a lane each
    const float4 e = s0 == 0 ? e0 : s0 + lane < n_splits ? __ldcg(mls + (s0 + lane) * kPagedFewRows) : none;
    const float w = s0 + lane < n_splits ? fast_exp2((e.x - M) + (e.z - R)) : 0.0f;
    L = fmaf(s0 + lane < n_splits ? fast_exp2(e.x - M) : 0.0f, e.y, L);
    const int n = min(32, n_splits - s0);
    for (int k0 = 0; k0 < n; k0 += kFly) {
      float4 x[kFly];
#pragma unroll
      for (int k = 0; k < kFly; ++k)
        x[k] = k0 + k < n && lane < kRuns ? __ldcg(part + (int64_t)(s0 + k0 + k) * kPagedFewRows * kRuns) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < kFly; ++k) {
        const float g = __shfl_sync(0xffffffffu, w, (k0 + k) & 31);
        acc = make_float4(fmaf(g, x[k].x, acc.x), fmaf(g, x[k].y, acc.y), fmaf(g, x[k].z, acc.z), fmaf(g, x[k].w, acc.w));
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

using FewKern = void (*)(const CUtensorMap, const CUtensorMap, const PagedAttnArgs);
FewKern few_of(int D, int row_tiles) {
  if (D == 128) return row_tiles == 1 ? few_kernel<128, 1> : few_kernel<128, 2>;
  return row_tiles == 1 ? few_kernel<64, 1> : few_kernel<64, 2>;
}

}  // namespace

cudaError_t paged_few_prepare(int D) {
  cudaError_t e = cudaSuccess;
  for (int n = 1; n <= 2 && e == cudaSuccess; ++n)
    e = cudaFuncSetAttribute(few_of(D, n), cudaFuncAttributeMaxDynamicSharedMemorySize, D == 128 ? FewLayout<128>::kSmem : FewLayout<64>::kSmem);
  return e;
}

cudaError_t launch_paged_few(int D, int row_tiles, const CUtensorMap& tmK, const CUtensorMap& tmV, const PagedAttnArgs& a,
                             cudaStream_t s) {
  const dim3 grid((unsigned)a.seqs.item0[a.seqs.n], (unsigned)a.Hkv);
  if (grid.x == 0) return cudaSuccess;
  few_of(D, row_tiles)<<<grid, kFewThreads, D == 128 ? FewLayout<128>::kSmem : FewLayout<64>::kSmem, s>>>(tmK, tmV, a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || !a.join) return e;
  return launch_join(D == 128 ? few_join_kernel<128> : few_join_kernel<64>, grid, 32 * kPagedFewRows, s, a);
}

}  // namespace fk
