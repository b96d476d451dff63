// Attention of a few queries over the paged 8-bit cache (single tokens, drafted tokens): the bytes of the cache
// bound it, so the keys are split over as many CTAs as the device holds and every byte is loaded once.
//   S = q k^T 2^(e_q + e_k) log2(e) scale,  p = 2^(S - m),  l = sum p,  O = 2^r sum p 2^(e_v - r) v / l
// with v the codes' values.
// CTA = (sequence, up to 16 query rows of one kv head's group, key split): warp 4 streams tiles of 64 keys and
// values into a ring (TMA, 2 boxes of a page's rows where pages are smaller); warps 0-3 take 16 keys of
// each tile by themselves, with their own running maximum m, sum l and O, and meet only at the end.
//   products  mma.m16n8k16 in f16: E4M3 codes are f16 values exactly, and a query row scaled by 2^-e_q (bf16 has
//             fewer bits than f16) is too, so that S is exact up to fp32 sums; p 2^(e_v - r) is rounded to f16 (11 bits).  The
//             tensor memory path would need 128 query rows to be worth its hand-overs.
//   layout    an MMA's inner index and its columns may be permuted at will, so that each lane reads whole 16-byte
//             runs of a row from shared memory and converts them in place: key column n of a 16-key group is key
//             tok(n) = n (n even) or ((n - 1) ^ 4) + 1 (n odd), and with the 128-byte swizzle no two lanes of a
//             quarter warp then meet in a bank, neither for keys (4 lanes on a row) nor for values (2 runs of 4 rows).
//   scales    e_k is in the factor of the exponent and e_v - r in its summand (r: see kRefWindow), so no key or value
//             is scaled.  m is raised only when a row outgrows it by 2^4, so that O is seldom rescaled.
// Splits leave (m, l, r, O) in a workspace; the last one to arrive joins them in the order of the splits (no atomics on
// values: results do not change from run to run).
#include "fk_paged.h"
#include "fk_tc.h"

namespace fk {
namespace {

constexpr int kWarps = 4;                             // consumer warps; one more loads
constexpr int kFewThreads = (kWarps + 1) * 32;
constexpr int kStages = 4;
constexpr float kLowest = -3.402823466e38f;           // m before any key: finite, so that 2^(-inf - m) is 0
constexpr float kRaise = 4.0f;                        // log2 units by which a row may outgrow m
constexpr float kShiftP = 8.0f;                       // p is stored times 2^8: at most 2^12 in f16

template <int D>
struct FewLayout {
  static constexpr int kTile = kPagedFewTile * D;     // bytes of a key (or value) tile
  static constexpr int kOffK = 0;
  static constexpr int kOffV = kOffK + kStages * kTile;
  static constexpr int kOffBar = kOffV + kStages * kTile;
  static constexpr int kSmem = kOffBar + 256 + 1024;
  static_assert(kWarps * kPagedFewRows * D * 4 <= kOffBar, "the warps' O over the stages");
};

struct FewBarriers {
  uint64_t full[kStages], empty[kStages];
  int8_t ke[kStages][2], ve[kStages][2];              // exponents of the tile's halves (pages)
  int last;
  volatile int abort;
};

// D += A B, A 16 x 16 (row), B 16 x 8 (column), f16 in, f32 out
__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// byte offset of 16-byte run c of row `row` in a tile (TMA swizzle of the row length)
template <int D>
__device__ __forceinline__ int run_at(int row, int c) {
  return D == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
}
// Sequence of work item b: the last s with first[s] <= b.
__device__ __forceinline__ int find_item(const int* first, int n, int b) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= b) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

template <int D>
__global__ void __launch_bounds__(kFewThreads, 2)
few_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
           const __grid_constant__ PagedAttnArgs a) {
  using Lay = FewLayout<D>;
  constexpr int kRows = kPagedFewRows, kT = kPagedFewTile;
  constexpr int kSteps = D / 16;                      // inner steps of S
  constexpr int kCols = D / 8;                        // column tiles of O
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sK = smem + Lay::kOffK;
  uint8_t* sV = smem + Lay::kOffV;
  FewBarriers* bar = reinterpret_cast<FewBarriers*>(smem + Lay::kOffBar);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int kvh = blockIdx.y;

  // ---- this CTA's rows and key tiles
  const int s = find_item(a.seqs.item0, a.seqs.n, blockIdx.x);
  const int n_keys = a.seqs.n_keys[s], n_q = a.seqs.n_q[s];
  const int n_rows = n_q * a.G;
  const int n_splits = a.seqs.splits[s];
  const int item = blockIdx.x - a.seqs.item0[s];
  const int split = item % n_splits, row0 = (item / n_splits) * kRows;
  const int rows = min(kRows, n_rows - row0);
  const int p_first = n_keys - n_q;                    // position of query 0
  const int pos0 = p_first + a.by_g.div(row0), pos1 = p_first + a.by_g.div(row0 + rows - 1);
  const TileRange tr = paged_tiles(n_keys, pos0, pos1, a.mask, kT);
  const int n_tiles = tr.count();
  const int i0 = (int)((int64_t)n_tiles * split / n_splits), i1 = (int)((int64_t)n_tiles * (split + 1) / n_splits);

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&bar->full[i], 1);
      mbar_init(&bar->empty[i], kWarps);
    }
    bar->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();

  float m[2] = {kLowest, kLowest}, l[2] = {0.0f, 0.0f};
  float o[kCols][4];
#pragma unroll
  for (int c = 0; c < kCols; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[c][i] = 0.0f;
  int r = -1000;                                        // reference of O (none yet)
  const int g = lane >> 2, t = lane & 3;

  if (warp == kWarps) {
    // ------------------------------------------------------------------ loads
    const int box = min(a.P, kT), boxes = kT / box;     // rows of a page in a tile
    const int* table = a.table + (int64_t)a.seqs.slot[s] * a.max_pages;
    const int last_page = max(n_keys - 1, 0) / a.P;
    int pg[2] = {0, 0}, ek[2] = {0, 0}, ev[2] = {0, 0}, tile = 0;
    bool ok = true;
    int lastU[kStages];
#pragma unroll
    for (int i = 0; i < kStages; ++i) lastU[i] = -1;
    for (int i = i0; i < i1 && ok; ++i) {
      const int k = i - i0;
      if ((k & 31) == 0) {                              // lane: pages and exponents of tile i + lane
        if (i + lane < i1) {
          tile = tr.at(i + lane);
          for (int b = 0; b < boxes; ++b) {
            pg[b] = __ldg(table + min((tile * kT + b * box) / a.P, last_page));
            ek[b] = a.ke[(int64_t)pg[b] * a.Hkv + kvh];
            ev[b] = a.ve[(int64_t)pg[b] * a.Hkv + kvh];
          }
        }
        __syncwarp();
      }
      const int st = k % kStages, u = k / kStages;
      if (u > 0 && !warp_wait(&bar->empty[st], (u - 1) & 1, bar, a.status)) { ok = false; break; }
      const int from = k & 31;
      const int tl = __shfl_sync(0xffffffffu, tile, from);
      if (lane == from) {
        for (int b = 0; b < 2; ++b) {
          bar->ke[st][b] = (int8_t)ek[boxes == 2 ? b : 0];
          bar->ve[st][b] = (int8_t)ev[boxes == 2 ? b : 0];
        }
        mbar_expect_tx(&bar->full[st], 2 * Lay::kTile);
        for (int b = 0; b < boxes; ++b) {
          const int y = (pg[b] * a.Hkv + kvh) * a.P + (boxes == 1 ? (tl * kT) % a.P : 0);
          tma_load_2d(sK + st * Lay::kTile + b * box * D, &tmK, &bar->full[st], 0, y);
          tma_load_2d(sV + st * Lay::kTile + b * box * D, &tmV, &bar->full[st], 0, y);
        }
      }
      __syncwarp();
#pragma unroll
      for (int q = 0; q < kStages; ++q)
        if (q == st) lastU[q] = u;
    }
    if (!ok)                                            // loads in flight land before the CTA ends
#pragma unroll
      for (int q = 0; q < kStages; ++q)
        if (lastU[q] >= 0) wait_phase(&bar->full[q], lastU[q] & 1, bar, a.status, false);
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ this lane's part of the queries
    // A fragment: rows g and g + 8, inner step st: channels base + 4 w + {0, 1} and + {2, 3}, base and w as the
    // lane's runs of a key row: run t (16 t ..) for the first four steps, run t + 4 (64 + 16 t ..) for the others
    uint32_t q[kSteps][4];
    float sc[2];
    int limit[2], lower[2];                             // visible keys: [lower, limit) and those below `sinks`
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = g + 8 * h;
      const bool in = row < rows;
      const int rr = row0 + (in ? row : 0), tok = a.by_g.div(rr), pos = p_first + tok;
      limit[h] = !in ? 0 : a.mask.causal ? min(pos + 1, n_keys) : n_keys;
      lower[h] = a.mask.window > 0 ? pos - a.mask.window + 1 : 0;
      const bf16* src = a.Q + ((int64_t)a.seqs.q0[s] + tok) * a.qstride + (int64_t)(kvh * a.G + rr - tok * a.G) * D;
      uint4 v[D / 32];
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        v[2 * c] = __ldg(reinterpret_cast<const uint4*>(src + 64 * c + 16 * t));
        v[2 * c + 1] = __ldg(reinterpret_cast<const uint4*>(src + 64 * c + 16 * t) + 1);
      }
      float amax = 0.0f;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) amax = fmaxf(amax, absmax8(v[c]));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      if (!(amax <= 3.402823466e38f)) l[h] = NAN;       // infinities (NaN makes its own way)
      const int e = e4m3_row_exponent(amax);
      const float inv = pow2f(-e);
      sc[h] = a.scale_log2 * pow2f(e);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        const uint32_t w[4] = {v[c].x, v[c].y, v[c].z, v[c].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {                   // channels 8 c' + 2 i, + 1
          const uint32_t p = pack_f16(__uint_as_float(w[i] << 16) * inv, __uint_as_float(w[i] & 0xFFFF0000u) * inv);
          q[2 * c + (i >> 1)][(i & 1) * 2 + h] = p;
        }
      }
    }
    // a tile without a masked key for any row of the CTA: [full_lo, full_hi), or all below the sinks
    const int full_hi = a.mask.causal ? min(pos0 + 1, n_keys) : n_keys;
    const int full_lo = a.mask.window > 0 ? pos1 - a.mask.window + 1 : 0;
    const int krow = warp * 16 + ((g & 1) ? ((g ^ 1) ^ 4) + 1 : g);   // key row of column g, first 8 columns
    const int va = warp * 16 + 2 * t, vb = warp * 16 + ((2 * t) ^ 4) + 1;

    bool ok = true;
    for (int i = i0; i < i1; ++i) {
      const int k = i - i0, st = k % kStages;
      if (!warp_wait(&bar->full[st], (k / kStages) & 1, bar, a.status)) { ok = false; break; }
      const uint8_t* kt = sK + st * Lay::kTile;
      const uint8_t* vt = sV + st * Lay::kTile;
      const int ek = bar->ke[st][warp >> 1], ev = bar->ve[st][warp >> 1];
      // S of the warp's 16 keys
      float sv[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
#pragma unroll
        for (int c = 0; c < 4; ++c) sv[n][c] = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          const uint4 kv = *reinterpret_cast<const uint4*>(kt + run_at<D>(krow + 8 * n, t + 4 * c));
          const uint32_t w[4] = {kv.x, kv.y, kv.z, kv.w};
#pragma unroll
          for (int x = 0; x < 4; ++x)
            mma16816(sv[n], q[4 * c + x], f16x2_of_e4m3x2((uint16_t)w[x]), f16x2_of_e4m3x2((uint16_t)(w[x] >> 16)));
        }
      }
      // scale and mask
      const float ske = pow2f(ek);
      const int j0 = tr.at(i) * kT;
      const bool full = j0 + kT <= full_hi && (j0 >= full_lo || j0 + kT <= a.mask.sinks);
      const int ja = j0 + va, jb = j0 + vb;             // keys of columns 2 t and 2 t + 1
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float c = fminf(sc[h] * ske, 3e38f);      // (codes may all be 0)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          sv[n][2 * h] *= c;
          sv[n][2 * h + 1] *= c;
          if (!full) {
            const int x = ja + 8 * n, y = jb + 8 * n;
            if (x >= limit[h] || (x < lower[h] && x >= a.mask.sinks)) sv[n][2 * h] = -INFINITY;
            if (y >= limit[h] || (y < lower[h] && y >= a.mask.sinks)) sv[n][2 * h + 1] = -INFINITY;
          }
        }
      }
      // running maximum and reference
      float mx[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        mx[h] = fmaxf(fmaxf(sv[0][2 * h], sv[0][2 * h + 1]), fmaxf(sv[1][2 * h], sv[1][2 * h + 1]));
        mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
        mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
      }
      const bool move = ev != kZeroExp && (ev > r || ev < r - kRefWindow);   // warp-uniform
      if (__any_sync(0xffffffffu, move || mx[0] > m[0] + kRaise || mx[1] > m[1] + kRaise)) {
        const float fr = move ? pow2_any(r - (ev + kRefRoom)) : 1.0f;
        if (move) r = ev + kRefRoom;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float mn = fmaxf(m[h], mx[h]), al = fast_exp2(m[h] - mn);
          m[h] = mn;
          l[h] *= al;
#pragma unroll
          for (int c = 0; c < kCols; ++c) {
            o[c][2 * h] *= al * fr;
            o[c][2 * h + 1] *= al * fr;
          }
        }
      }
      const float we = ev == kZeroExp ? 0.0f : (float)(ev - r), fl = ev == kZeroExp ? 1.0f : pow2f(r - ev);
      uint32_t p[4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float z = we + kShiftP - m[h], x = fast_exp2(sv[n][2 * h] + z), y = fast_exp2(sv[n][2 * h + 1] + z);
          l[h] = fmaf(x + y, fl, l[h]);
          p[2 * n + h] = pack_f16(x, y);
        }
      // O += P V
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
#pragma unroll
      for (int x = 0; x < kCols / 4; ++x) {
        const uint32_t wa[2] = {x == 0 ? w[0].x : x == 1 ? w[0].y : x == 2 ? w[0].z : w[0].w,
                                x == 0 ? w[2].x : x == 1 ? w[2].y : x == 2 ? w[2].z : w[2].w};
        const uint32_t wb[2] = {x == 0 ? w[1].x : x == 1 ? w[1].y : x == 2 ? w[1].z : w[1].w,
                                x == 0 ? w[3].x : x == 1 ? w[3].y : x == 2 ? w[3].z : w[3].w};
        const uint32_t lo0 = __byte_perm(wa[0], wb[0], 0x5140), hi0 = __byte_perm(wa[0], wb[0], 0x7362);
        const uint32_t lo1 = __byte_perm(wa[1], wb[1], 0x5140), hi1 = __byte_perm(wa[1], wb[1], 0x7362);
        mma16816(o[4 * x], p, f16x2_of_e4m3x2((uint16_t)lo0), f16x2_of_e4m3x2((uint16_t)lo1));
        mma16816(o[4 * x + 1], p, f16x2_of_e4m3x2((uint16_t)(lo0 >> 16)), f16x2_of_e4m3x2((uint16_t)(lo1 >> 16)));
        mma16816(o[4 * x + 2], p, f16x2_of_e4m3x2((uint16_t)hi0), f16x2_of_e4m3x2((uint16_t)hi1));
        mma16816(o[4 * x + 3], p, f16x2_of_e4m3x2((uint16_t)(hi0 >> 16)), f16x2_of_e4m3x2((uint16_t)(hi1 >> 16)));
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar->empty[st]);
    }
    (void)ok;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    }
  }
  __syncthreads();                                      // every tile has been read: the stages are free

  // ---- the warps' (m, l, r) and O
  float* sO = reinterpret_cast<float*>(smem);           // [warp][row][D], 16-byte run c of row at c ^ (row & 7)
  __shared__ float sm[kWarps][kRows], sl[kWarps][kRows];
  __shared__ int sr[kWarps];
  if (warp < kWarps) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = g + 8 * h;
      float* dst = sO + (warp * kRows + row) * D;
      // lane t holds channels 2 kCols t + c (even columns) and 2 kCols t + kCols + c (odd columns)
#pragma unroll
      for (int c = 0; c < kCols; c += 4) {
        const int ca = (2 * kCols * t + c) / 4, cb = ca + kCols / 4;
        *reinterpret_cast<float4*>(dst + ((ca ^ (row & 7)) << 2)) = make_float4(o[c][2 * h], o[c + 1][2 * h], o[c + 2][2 * h], o[c + 3][2 * h]);
        *reinterpret_cast<float4*>(dst + ((cb ^ (row & 7)) << 2)) = make_float4(o[c][2 * h + 1], o[c + 1][2 * h + 1], o[c + 2][2 * h + 1], o[c + 3][2 * h + 1]);
      }
      if (t == 0) {
        sm[warp][row] = m[h];
        sl[warp][row] = l[h];
      }
    }
    if (lane == 0) sr[warp] = r;
  }
  __syncthreads();
  // O of the CTA relative to (M, 2^R): weights 2^(m_w - M) 2^(r_w - R)
  const int R = max(max(sr[0], sr[1]), max(sr[2], sr[3]));
  const int cta = a.seqs.part0[s] + kvh * (a.seqs.item0[s + 1] - a.seqs.item0[s]) + item;   // workspace slot
  constexpr int kRuns = D / 4;
  auto out_row = [&](int row) {
    const int rr = row0 + row, tok = a.by_g.div(rr);
    return a.O + ((int64_t)a.seqs.q0[s] + tok) * a.ostride + (int64_t)(kvh * a.G + rr - tok * a.G) * D;
  };
  float* part = a.part + (int64_t)cta * kRows * D;
  float4* mls = reinterpret_cast<float4*>(a.part + (int64_t)kPartSlots * kRows * D);   // m, l, r
  for (int i = threadIdx.x; i < rows * kRuns; i += kFewThreads) {
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
      const float inv = L > 0.0f || L != L ? pow2_any(R) / L : 0.0f;   // no visible key: 0
      *reinterpret_cast<uint2*>(out_row(row) + 4 * c) =
          make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    } else {
      *reinterpret_cast<float4*>(part + row * D + 4 * c) = acc;
      if (c == 0) mls[cta * kRows + row] = make_float4(M, L, (float)R, 0.0f);
    }
  }
  if (n_splits == 1) return;

  // ---- the last split of the group joins them all
  __threadfence();
  __syncthreads();
  const int first = cta - split;                        // slot of split 0
  if (threadIdx.x == 0) bar->last = atomicInc(reinterpret_cast<unsigned*>(a.arrived + first), n_splits - 1) == (unsigned)(n_splits - 1);
  __syncthreads();
  if (!bar->last) return;
  __threadfence();
  const float* parts = a.part + (int64_t)first * kRows * D;
  for (int i = threadIdx.x; i < rows * kRuns; i += kFewThreads) {
    const int row = i / kRuns, c = i % kRuns;
    float M = kLowest, RR = -1000.0f, L = 0.0f;
    for (int sp = 0; sp < n_splits; ++sp) {
      const float4 e = __ldcg(mls + (first + sp) * kRows + row);
      M = fmaxf(M, e.x);
      RR = fmaxf(RR, e.z);
    }
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int sp = 0; sp < n_splits; ++sp) {
      const float4 e = __ldcg(mls + (first + sp) * kRows + row);
      const float4 x = __ldcg(reinterpret_cast<const float4*>(parts + ((int64_t)sp * kRows + row) * D + 4 * c));
      const float f = fast_exp2(e.x - M), fo = f * pow2_any((int)(e.z - RR));
      L = fmaf(f, e.y, L);
      acc.x = fmaf(fo, x.x, acc.x);
      acc.y = fmaf(fo, x.y, acc.y);
      acc.z = fmaf(fo, x.z, acc.z);
      acc.w = fmaf(fo, x.w, acc.w);
    }
    const float inv = L > 0.0f || L != L ? pow2_any((int)RR) / L : 0.0f;
    *reinterpret_cast<uint2*>(out_row(row) + 4 * c) =
        make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
  }
}

}  // namespace

cudaError_t paged_few_prepare(int D) {
  return D == 128 ? cudaFuncSetAttribute(few_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewLayout<128>::kSmem)
                  : cudaFuncSetAttribute(few_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewLayout<64>::kSmem);
}

cudaError_t launch_paged_few(int D, const CUtensorMap& tmK, const CUtensorMap& tmV, const PagedAttnArgs& a,
                             cudaStream_t s) {
  const dim3 grid((unsigned)a.seqs.item0[a.seqs.n], (unsigned)a.Hkv);
  if (grid.x == 0) return cudaSuccess;
  if (D == 128) few_kernel<128><<<grid, kFewThreads, FewLayout<128>::kSmem, s>>>(tmK, tmV, a);
  else few_kernel<64><<<grid, kFewThreads, FewLayout<64>::kSmem, s>>>(tmK, tmV, a);
  return cudaGetLastError();
}

}  // namespace fk
