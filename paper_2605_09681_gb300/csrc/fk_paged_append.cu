// Appending to the paged 8-bit cache, reading it back, and its page table.
//
// Append, one launch for a step: every (page written, kv head) is one block of the cache with one exponent for its
// keys and one for its values; a CTA takes a block's keys, its values, or the queries of its tokens.
//   rotation  y_i = x_i c_i - x_j s_i, y_j = x_j c_i + x_i s_i on channel pairs (i, j) of the first R channels,
//             (i, i + R/2) or (2i, 2i + 1), in fp32 with every product and sum rounded by itself;
//   block     a = largest finite |y| of the page's tokens so far (those of this step and those already there),
//             e = smallest integer >= -120 with a <= 448 2^e (kZeroExp for zeros), code = E4M3(y 2^-e) (exact scaling, one rounding
//             to nearest even).  Infinities saturate, NaN becomes 0: the cache holds finite values only, so that a
//             masked key or value can never reach a row that does not see it; the status word tells.
// A block's codes depend on its tokens only and not on how they came in steps: the open page's tokens are kept as they
// were before the rounding (rotated keys in fp32, values in bf16: both exact) with each token's largest magnitude, and
// where e moves, its older tokens are rounded again from there.  Most steps leave e alone, and then only the new
// tokens are touched.  A step's append may be repeated with other keys and values: nothing it reads is what it wrote.
// Threads: P D / 32, in rows of D / 16; a thread holds 16 channels (two runs of 8, the two halves of its pairs) of
// 2 tokens, so that a page is loaded at once and never read again.  Steps of a few tokens: append_few_kernel.
// What bounds it: latency.  Bytes move at half the copy rate: a CTA loads, reduces and stores once, two of 512 threads fit an SM, its rotation
// factors are asked for when its rows are there, and nothing is in flight from one page to the next (issue slots 51% busy, loads
// the first reason to wait).  4680 tokens of 12 + 12 + 12 heads of 128, pages of 128: 21.0 us (75 MB, 3.6 TB/s);
// reading the 37 pages back as bf16 9.3 us (43 MB, 4.6 TB/s).  Keys, values and queries in CTAs of their own, so that registers hold one tensor's
// rows (all three in one CTA: 25.6 us).
#include "fk_paged.h"
#include "fk_tc.h"

#include <algorithm>

namespace fk {
namespace {

// exponent of a block whose largest finite magnitude is `amax`
__device__ __forceinline__ int block_exponent(float amax) { return amax == 0.0f ? kZeroExp : e4m3_row_exponent(amax); }

__device__ __forceinline__ void unpack8(uint4 v, float* x) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float* x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&p);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// eight floats times `scale` -> eight codes
__device__ __forceinline__ uint2 codes8(const float* x, float scale) {
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = e4m3x2(x[2 * i] * scale, x[2 * i + 1] * scale);
  return make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410));
}

// Sequence of page (or item) b: the last s with first[s] <= b.
__device__ __forceinline__ int find_seq(const int* first, int n, int b) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= b) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// The two runs of 8 channels of thread column j (of D / 16) and whether they are rotated.
struct Cols {
  int c0, c1;                         // first channels
  bool rot;
};
__device__ __forceinline__ Cols cols_of(int j, int R, int interleaved) {
  const int half = R / 16;            // runs in half of the rotated channels
  if (interleaved) return {16 * j, 16 * j + 8, j < half};
  if (j < half) return {8 * j, 8 * (j + half), true};
  return {8 * (2 * half + 2 * (j - half)), 8 * (2 * half + 2 * (j - half) + 1), false};
}

// Rotate the 16 channels x (two runs); cs, sn: 8 factors each.  (Packed products and sums would be contracted.)
__device__ __forceinline__ void rotate16(float* x, const float* cs, const float* sn, int interleaved) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = __fsub_rn(__fmul_rn(a, cs[i]), __fmul_rn(b, sn[i]));
      x[2 * i + 1] = __fadd_rn(__fmul_rn(b, cs[i]), __fmul_rn(a, sn[i]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = x[i], b = x[8 + i];
      x[i] = __fsub_rn(__fmul_rn(a, cs[i]), __fmul_rn(b, sn[i]));
      x[8 + i] = __fadd_rn(__fmul_rn(b, cs[i]), __fmul_rn(a, sn[i]));
    }
  }
}

__device__ __forceinline__ void load8(const float* p, float* x) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// What an append CTA or warp knows of its page.
struct PageOf {
  int slot, pi, base, lo, hi;         // sequence's slot, page of the sequence, its first token, this step's rows of it
  int64_t tok;                        // caller's token of row 0
  int64_t tail_old, tail_new;         // tail rows of row 0
};
__device__ __forceinline__ PageOf page_of(const AppendArgs& a, int b, int h) {
  const int s = find_seq(a.seqs.page0, a.seqs.n, b), P = a.P, shift = 31 - __clz(P);   // (a power of two)
  const int old_len = a.seqs.old_len[s], new_len = a.seqs.new_len[s], buf = a.seqs.buf[s];
  PageOf g;
  g.slot = a.seqs.slot[s];
  g.pi = (old_len >> shift) + (b - a.seqs.page0[s]);
  g.base = g.pi << shift;
  g.lo = max(old_len - g.base, 0);
  g.hi = min(new_len - g.base, P);
  g.tok = (int64_t)a.seqs.tok0[s] + (g.base - old_len);
  g.tail_old = (((int64_t)g.slot * 2 + (buf & 1)) * a.Hkv + h) * P;
  g.tail_new = (((int64_t)g.slot * 2 + (buf >> 1)) * a.Hkv + h) * P;
  return g;
}

// Table row of caller's token t, row `row` of the page (asked for early: the factors' address hangs on it).
__device__ __forceinline__ int position_of(const AppendArgs& a, const PageOf& g, int64_t t, int row) {
  return a.positions ? __ldg(a.positions + t) : g.base + row;
}
// Rotate 16 channels x by table row `pos`.
__device__ __forceinline__ void rotate_row(const AppendArgs& a, int pos, int j, float* x) {
  if ((unsigned)pos >= (unsigned)a.rope_rows) {
    atomicOr(a.status, kStatusPosition);
    return;
  }
  float cs[8], sn[8];
  const int64_t at = (int64_t)pos * (a.R / 2) + 8 * j;
  load8(a.cos + at, cs);
  load8(a.sin + at, sn);
  rotate16(x, cs, sn, a.interleaved);
}

// Largest finite magnitude of 16 values; `bad` when one is not finite.  (Beside an infinity at least the smallest number, which has the
// exponent of zeros, -120, but is not one: a block of zeros and infinities holds 448 2^-120, and kZeroExp says that it holds nothing.)
__device__ __forceinline__ float largest16(const float* x, bool& bad) {
  float m = 0.0f;
  float2 z = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int c = 0; c < 16; ++c) m = fmaxf(m, fabsf(x[c]));
#pragma unroll
  for (int c = 0; c < 16; c += 2) z = ffma2(make_float2(x[c], x[c + 1]), make_float2(0.0f, 0.0f), z);   // NaN from infinities and NaN
  if (z.x + z.y != 0.0f) {
    bad = true;
    m = 0.0f;
#pragma unroll
    for (int c = 0; c < 16; ++c)
      if (x[c] == x[c]) m = fmaxf(m, fabsf(x[c]) <= 3.402823466e38f ? fabsf(x[c]) : __uint_as_float(1u));
  }
  return m;
}
__device__ __forceinline__ void no_nan16(float* x) {
#pragma unroll
  for (int c = 0; c < 16; ++c)
    if (x[c] != x[c]) x[c] = 0.0f;
}

// Largest of a warp's non-negative floats (their bits are ordered as they are).
__device__ __forceinline__ float warp_max(float m) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m))); }

// Codes of a row's 16 channels, and their unrounded copy in the tail (`keep`: the row's place there, -1: none).
template <int D>
__device__ __forceinline__ void put16(const AppendArgs& a, bool is_v, uint8_t* dst, int row, const Cols& cl, const float* x, float inv,
                                      int64_t keep) {
  *reinterpret_cast<uint2*>(dst + row * D + cl.c0) = codes8(x, inv);
  *reinterpret_cast<uint2*>(dst + row * D + cl.c1) = codes8(x + 8, inv);
  if (keep < 0) return;
  if (is_v) {
    bf16* p = a.pool.tail_v + keep * D;
    *reinterpret_cast<uint4*>(p + cl.c0) = pack8(x);
    *reinterpret_cast<uint4*>(p + cl.c1) = pack8(x + 8);
  } else {
    float* p = a.pool.tail_k + keep * D;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      *reinterpret_cast<float4*>(p + cl.c0 + 4 * q) = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
      *reinterpret_cast<float4*>(p + cl.c1 + 4 * q) = make_float4(x[8 + 4 * q], x[9 + 4 * q], x[10 + 4 * q], x[11 + 4 * q]);
    }
  }
}
// A tail row's 16 channels.
template <int D>
__device__ __forceinline__ void tail16(const AppendArgs& a, bool is_v, int64_t row, const Cols& cl, float* x) {
  if (is_v) {
    const bf16* p = a.pool.tail_v + row * D;
    unpack8(*reinterpret_cast<const uint4*>(p + cl.c0), x);
    unpack8(*reinterpret_cast<const uint4*>(p + cl.c1), x + 8);
  } else {
    const float* p = a.pool.tail_k + row * D;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      x[c] = p[cl.c0 + c];
      x[8 + c] = p[cl.c1 + c];
    }
  }
}

// Queries of the page's new tokens, heads of group h: rows (token, head) first, first + step, ..
template <int D>
__device__ __forceinline__ void rotate_queries(const AppendArgs& a, const PageOf& g, int h, int first, int step, int j, const Cols& cl) {
  const int n = (g.hi - g.lo) * a.G;
#pragma unroll 2
  for (int i = first; i < n; i += step) {
    const int row = g.lo + a.by_g.div(i);
    const int64_t t = g.tok + row, hd = h * a.G + i - (row - g.lo) * a.G;
    const int pos = cl.rot ? position_of(a, g, t, row) : 0;
    float x[16];
    const bf16* q = a.Q + t * a.qstride + hd * D;
    unpack8(__ldg(reinterpret_cast<const uint4*>(q + cl.c0)), x);
    unpack8(__ldg(reinterpret_cast<const uint4*>(q + cl.c1)), x + 8);
    if (cl.rot) rotate_row(a, pos, j, x);
    bf16* o = a.Qr + t * a.qrstride + hd * D;
    *reinterpret_cast<uint4*>(o + cl.c0) = pack8(x);
    *reinterpret_cast<uint4*>(o + cl.c1) = pack8(x + 8);
  }
}

// (64 registers for either head dimension: at 64, 86 without the bound took 13.6 us for 7.9 k tokens of 16 + 4 + 4 heads, this 11.0.)
template <int D>
__global__ void __launch_bounds__(4 * D, 256 / D) append_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int kCols = D / 16;       // threads of one token
  __shared__ float red[16];
  const int h = blockIdx.y, P = a.P;
  const PageOf g = page_of(a, blockIdx.x, h);
  const int j = threadIdx.x % kCols, r0 = threadIdx.x / kCols, step = P / 2;
  const Cols cl = cols_of(j, a.cos ? a.R : 0, a.interleaved);
  // z: keys, values, then the heads of the group's queries
  const bool is_q = blockIdx.z >= 2, is_v = blockIdx.z == 1, turn = !is_v && cl.rot;
  const bf16* src = is_q ? a.Q + (int64_t)(h * a.G + (int)blockIdx.z - 2) * D : (is_v ? a.V : a.K) + h * D;
  const int64_t stride = is_q ? a.qstride : is_v ? a.vstride : a.kstride;
  uint4 v[2][2];
  int pos[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = r0 + i * step;
    v[i][0] = v[i][1] = make_uint4(0, 0, 0, 0);
    if (row >= g.lo && row < g.hi) {
      if (turn) pos[i] = position_of(a, g, g.tok + row, row);
      const bf16* p = src + (g.tok + row) * stride;
      v[i][0] = __ldg(reinterpret_cast<const uint4*>(p + cl.c0));
      v[i][1] = __ldg(reinterpret_cast<const uint4*>(p + cl.c1));
    }
  }
  if (is_q) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = r0 + i * step;
      if (row < g.lo || row >= g.hi) continue;
      float x[16];
      unpack8(v[i][0], x);
      unpack8(v[i][1], x + 8);
      if (turn) rotate_row(a, pos[i], j, x);
      bf16* o = a.Qr + (g.tok + row) * a.qrstride + (int64_t)(h * a.G + (int)blockIdx.z - 2) * D;
      *reinterpret_cast<uint4*>(o + cl.c0) = pack8(x);
      *reinterpret_cast<uint4*>(o + cl.c1) = pack8(x + 8);
    }
    return;
  }
  const int64_t block = (int64_t)__ldg(a.table + (int64_t)g.slot * a.max_pages + g.pi) * a.Hkv + h;
  uint8_t* dst = (is_v ? a.pool.v : a.pool.k) + block * P * D;
  int8_t* exps = is_v ? a.pool.ve : a.pool.ke;
  float* tmax = is_v ? a.pool.tail_vmax : a.pool.tail_kmax;
  const int e_old = g.lo > 0 ? (int)exps[block] : 0;
  const bool open = g.hi < P;                  // the page stays open: its new tokens are kept unrounded
  float m = 0.0f, x[2][16];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = r0 + i * step;
    unpack8(v[i][0], x[i]);
    unpack8(v[i][1], x[i] + 8);
    if (turn && row >= g.lo && row < g.hi) rotate_row(a, pos[i], j, x[i]);
    float rmax = largest16(x[i], bad);
    m = fmaxf(m, rmax);
    if (open) {
#pragma unroll
      for (int off = kCols / 2; off >= 1; off >>= 1) rmax = fmaxf(rmax, __shfl_xor_sync(0xffffffffu, rmax, off));
      if (j == 0 && row >= g.lo && row < g.hi) tmax[g.tail_new + row] = rmax;
    }
  }
  if (bad) atomicOr(a.status, kStatusNonFinite);
  for (int r = threadIdx.x; r < g.lo; r += blockDim.x) m = fmaxf(m, tmax[g.tail_old + r]);
  m = warp_max(m);
  const int lane = threadIdx.x & 31;
  if (lane == 0) red[threadIdx.x >> 5] = m;
  __syncthreads();
  m = warp_max(lane < (int)(blockDim.x >> 5) ? red[lane] : 0.0f);
  const int e = block_exponent(m);
  const float inv = pow2f(-e);                 // (2^126 for zeros)
  if (threadIdx.x == 0) exps[block] = (int8_t)e;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = r0 + i * step;
    if (row < g.lo || row >= g.hi) continue;
    if (bad) no_nan16(x[i]);
    put16<D>(a, is_v, dst, row, cl, x[i], inv, open ? g.tail_new + row : -1);
  }
  if (g.lo > 0 && e != e_old)                  // the older tokens' codes have another exponent
    for (int row = r0; row < g.lo; row += step) {
      float x[16];
      tail16<D>(a, is_v, g.tail_old + row, cl, x);
      put16<D>(a, is_v, dst, row, cl, x, inv, -1);
    }
}

// A few new tokens to a page (decoding): a warp each for a page's keys, values and queries, so that nothing waits for a CTA;
// up to kPass passes of 32 / (D / 16) rows.
template <int D>
__global__ void __launch_bounds__(96) append_few_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int kCols = D / 16, kRows = 32 / kCols, kPass = kAppendFewRows / kRows;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = blockIdx.y, P = a.P;
  const PageOf g = page_of(a, blockIdx.x, h);
  const int j = lane % kCols, r0 = lane / kCols;
  const Cols cl = cols_of(j, a.cos ? a.R : 0, a.interleaved);
  if (warp == 2) {
    rotate_queries<D>(a, g, h, r0, kRows, j, cl);
    return;
  }
  const bool is_v = warp == 1, turn = !is_v && cl.rot;
  const bf16* src = is_v ? a.V : a.K;
  const int64_t stride = is_v ? a.vstride : a.kstride;
  uint4 v[kPass][2];
  int pos[kPass];
#pragma unroll
  for (int i = 0; i < kPass; ++i) {
    const int row = g.lo + r0 + i * kRows;
    v[i][0] = v[i][1] = make_uint4(0, 0, 0, 0);
    pos[i] = 0;
    if (row < g.hi) {
      if (turn) pos[i] = position_of(a, g, g.tok + row, row);
      const bf16* p = src + (g.tok + row) * stride + h * D;
      v[i][0] = __ldg(reinterpret_cast<const uint4*>(p + cl.c0));
      v[i][1] = __ldg(reinterpret_cast<const uint4*>(p + cl.c1));
    }
  }
  const int64_t block = (int64_t)__ldg(a.table + (int64_t)g.slot * a.max_pages + g.pi) * a.Hkv + h;
  uint8_t* dst = (is_v ? a.pool.v : a.pool.k) + block * P * D;
  int8_t* exps = is_v ? a.pool.ve : a.pool.ke;
  float* tmax = is_v ? a.pool.tail_vmax : a.pool.tail_kmax;
  float m = 0.0f;                              // of the older tokens, under way while the new ones load
  for (int r = lane; r < g.lo; r += 32) m = fmaxf(m, tmax[g.tail_old + r]);
  const int e_old = g.lo > 0 ? (int)exps[block] : 0;
  const bool open = g.hi < P;
  bool bad = false;
  float x[kPass][16];
#pragma unroll
  for (int i = 0; i < kPass; ++i) {
    const int row = g.lo + r0 + i * kRows;
    unpack8(v[i][0], x[i]);
    unpack8(v[i][1], x[i] + 8);
    if (turn && row < g.hi) rotate_row(a, pos[i], j, x[i]);
    float rmax = largest16(x[i], bad);
    m = fmaxf(m, rmax);
    if (open) {
#pragma unroll
      for (int off = kCols / 2; off >= 1; off >>= 1) rmax = fmaxf(rmax, __shfl_xor_sync(0xffffffffu, rmax, off));
      if (j == 0 && row < g.hi) tmax[g.tail_new + row] = rmax;
    }
  }
  if (bad) atomicOr(a.status, kStatusNonFinite);
  m = warp_max(m);
  const int e = block_exponent(m);
  const float inv = pow2f(-e);
  if (lane == 0) exps[block] = (int8_t)e;
#pragma unroll
  for (int i = 0; i < kPass; ++i) {
    const int row = g.lo + r0 + i * kRows;
    if (row >= g.hi) continue;
    if (bad) no_nan16(x[i]);
    put16<D>(a, is_v, dst, row, cl, x[i], inv, open ? g.tail_new + row : -1);
  }
  if (g.lo > 0 && e != e_old)
    for (int row = r0; row < g.lo; row += kRows) {
      float y[16];
      tail16<D>(a, is_v, g.tail_old + row, cl, y);
      put16<D>(a, is_v, dst, row, cl, y, inv, -1);
    }
}

// eight codes -> eight values times 2^e as bf16 (exact; beyond bf16's range the largest finite value)
__device__ __forceinline__ uint4 values8(uint2 c, float scale) {
  float x[8];
  const uint16_t p[4] = {(uint16_t)c.x, (uint16_t)(c.x >> 16), (uint16_t)c.y, (uint16_t)(c.y >> 16)};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(p[i]));
    const __half2 v = *reinterpret_cast<const __half2*>(&h);
    const float top = 3.3895313892515355e38f;
    x[2 * i] = fminf(fmaxf(__low2float(v) * scale, -top), top);
    x[2 * i + 1] = fminf(fmaxf(__high2float(v) * scale, -top), top);
  }
  return pack8(x);
}

template <int D>
__global__ void __launch_bounds__(256) read_kernel(const __grid_constant__ ReadArgs a) {
  const int s = find_seq(a.seqs.page0, a.seqs.n, blockIdx.x);
  const int P = a.P, h = blockIdx.y;
  const int first = a.whole ? 0 : a.seqs.old_len[s] / P;
  const int pi = first + (blockIdx.x - a.seqs.page0[s]);
  const int rows = min(a.seqs.new_len[s] - pi * P, P);
  const int page = __ldg(a.table + (int64_t)a.seqs.slot[s] * a.max_pages + pi);
  const int64_t block = (int64_t)page * a.Hkv + h;
  const uint8_t* src = (blockIdx.z ? a.pool.v : a.pool.k) + block * P * D;
  bf16* dst = (blockIdx.z ? a.V : a.K) + ((int64_t)a.seqs.tok0[s] + (int64_t)(pi - first) * P) * a.Hkv * D + h * D;
  const float scale = pow2f(blockIdx.z ? a.pool.ve[block] : a.pool.ke[block]);
  constexpr int kCols = D / 8, kFly = 4;            // (a run at a time: 11.1 us for the 37 pages above)
  for (int i0 = threadIdx.x; i0 < rows * kCols; i0 += blockDim.x * kFly) {
    uint2 v[kFly];
#pragma unroll
    for (int k = 0; k < kFly; ++k) {
      const int i = i0 + k * blockDim.x;
      if (i < rows * kCols) v[k] = *reinterpret_cast<const uint2*>(src + i * 8);
    }
#pragma unroll
    for (int k = 0; k < kFly; ++k) {
      const int i = i0 + k * blockDim.x;
      if (i < rows * kCols) *reinterpret_cast<uint4*>(dst + (int64_t)(i / kCols) * a.Hkv * D + (i % kCols) * 8) = values8(v[k], scale);
    }
  }
}

__global__ void table_kernel(const __grid_constant__ TableArgs a) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < a.n) a.table[a.index[i]] = a.page[i];
}

// The status word's report: a timeout by itself, else all there is; only what is reported is cleared.
__global__ void status_kernel(int* status, int* report) {
  const int word = atomicOr(status, 0), told = word & kStatusTimeout ? kStatusTimeout : word;
  atomicAnd(status, ~told);
  *report = told;
}

}  // namespace

cudaError_t launch_paged_append(int D, const AppendArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)a.seqs.page0[a.seqs.n], (unsigned)a.Hkv, a.Q ? 2 + a.G : 2);
  if (grid.x == 0) return cudaSuccess;
  // at most kAppendFewRows new tokens on any page: a warp takes a page's (64 streams, a token each, 32 + 8 + 8 heads of 128: 3.6 us, a
  // CTA for a page 8.3)
  if (a.most <= kAppendFewRows) {
    const dim3 few(grid.x, grid.y, 1);
    const int threads = a.Q ? 96 : 64;
    if (D == 128) append_few_kernel<128><<<few, threads, 0, s>>>(a);
    else append_few_kernel<64><<<few, threads, 0, s>>>(a);
    return cudaGetLastError();
  }
  if (D == 128) append_kernel<128><<<grid, a.P * 4, 0, s>>>(a);
  else append_kernel<64><<<grid, a.P * 2, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_paged_read(int D, const ReadArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)a.seqs.page0[a.seqs.n], (unsigned)a.Hkv, 2);
  if (grid.x == 0) return cudaSuccess;
  const int threads = std::min(256, a.P * D / 32);
  if (D == 128) read_kernel<128><<<grid, threads, 0, s>>>(a);
  else read_kernel<64><<<grid, threads, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_paged_table(const TableArgs& a, cudaStream_t s) {
  if (a.n == 0) return cudaSuccess;
  table_kernel<<<(a.n + 127) / 128, 128, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_paged_status(int* status, int* report, cudaStream_t s) {
  status_kernel<<<1, 1, 0, s>>>(status, report);
  return cudaGetLastError();
}

}  // namespace fk
