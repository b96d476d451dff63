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
// Threads: P D / 64, in rows of D / 16; a thread holds 16 channels (two runs of 8, the two halves of its pairs) of
// 4 tokens, so that a page is loaded at once and never read again.
#include "fk_paged.h"

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
  return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
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

// Rotate the 16 channels x (two runs) by table row `pos`; c, s: 8 factors each.
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

template <int D>
__global__ void __launch_bounds__(2 * D) append_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int kCols = D / 16;       // threads of one token
  __shared__ float red[8];
  const int s = find_seq(a.seqs.page0, a.seqs.n, blockIdx.x);
  const int h = blockIdx.y, P = a.P;
  const int slot = a.seqs.slot[s], old_len = a.seqs.old_len[s], new_len = a.seqs.new_len[s];
  const int pi = old_len / P + (blockIdx.x - a.seqs.page0[s]);     // page of the sequence
  const int base = pi * P;                                           // its first token
  const int lo = max(old_len - base, 0), hi = min(new_len - base, P);   // this step's rows of the page
  const int64_t tok = (int64_t)a.seqs.tok0[s] + (base - old_len);    // caller's token of row 0
  const int j = threadIdx.x % kCols, r0 = threadIdx.x / kCols, step = P / 4;
  const Cols cl = cols_of(j, a.cos ? a.R : 0, a.interleaved);

  auto factors = [&](int64_t t, int row, float* cs, float* sn) -> bool {   // of caller's token t, row of the page
    const int pos = a.positions ? __ldg(a.positions + t) : base + row;
    if ((unsigned)pos >= (unsigned)a.rope_rows) {
      atomicOr(a.status, kStatusPosition);
      return false;
    }
    const int64_t at = (int64_t)pos * (a.R / 2) + 8 * j;
    load8(a.cos + at, cs);
    load8(a.sin + at, sn);
    return true;
  };

  if (blockIdx.z == 2) {              // queries of the page's new tokens, heads of the group
    const int n = (hi - lo) * a.G;
#pragma unroll 2
    for (int i = r0; i < n; i += step) {
      const int row = lo + i / a.G;
      const int64_t t = tok + row, hd = h * a.G + i % a.G;
      float x[16], cs[8], sn[8];
      const bf16* q = a.Q + t * a.qstride + hd * D;
      unpack8(__ldg(reinterpret_cast<const uint4*>(q + cl.c0)), x);
      unpack8(__ldg(reinterpret_cast<const uint4*>(q + cl.c1)), x + 8);
      if (cl.rot && factors(t, row, cs, sn)) rotate16(x, cs, sn, a.interleaved);
      bf16* o = a.Qr + t * a.qrstride + hd * D;
      *reinterpret_cast<uint4*>(o + cl.c0) = pack8(x);
      *reinterpret_cast<uint4*>(o + cl.c1) = pack8(x + 8);
    }
    return;
  }

  const bool is_v = blockIdx.z == 1;
  const bf16* src = is_v ? a.V : a.K;
  const int64_t stride = is_v ? a.vstride : a.kstride;
  const int page = __ldg(a.table + (int64_t)slot * a.max_pages + pi);
  const int64_t block = (int64_t)page * a.Hkv + h;
  uint8_t* dst = (is_v ? a.pool.v : a.pool.k) + block * P * D;
  int8_t* exps = is_v ? a.pool.ve : a.pool.ke;
  const int64_t tail_old = (((int64_t)slot * 2 + (a.seqs.buf[s] & 1)) * a.Hkv + h) * P;      // rows
  const int64_t tail_new = (((int64_t)slot * 2 + (a.seqs.buf[s] >> 1)) * a.Hkv + h) * P;
  float* tmax = is_v ? a.pool.tail_vmax : a.pool.tail_kmax;
  const int e_old = lo > 0 ? (int)exps[block] : 0;

  // the new tokens, rotated, and the largest finite magnitude
  float x[4][16], rmax[4];
  bool bad = false;
  {
    uint4 v[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = r0 + i * step;
      v[i][0] = v[i][1] = make_uint4(0, 0, 0, 0);
      if (row >= lo && row < hi) {
        const bf16* p = src + (tok + row) * stride + h * D;
        v[i][0] = __ldg(reinterpret_cast<const uint4*>(p + cl.c0));
        v[i][1] = __ldg(reinterpret_cast<const uint4*>(p + cl.c1));
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = r0 + i * step;
      unpack8(v[i][0], x[i]);
      unpack8(v[i][1], x[i] + 8);
      if (!is_v && cl.rot && row >= lo && row < hi) {
        float cs[8], sn[8];
        if (factors(tok + row, row, cs, sn)) rotate16(x[i], cs, sn, a.interleaved);
      }
      rmax[i] = 0.0f;
#pragma unroll
      for (int c = 0; c < 16; ++c) {
        const float m = fabsf(x[i][c]);
        const bool fine = m <= 3.402823466e38f;
        bad |= !fine;
        if (fine) rmax[i] = fmaxf(rmax[i], m);
        if (x[i][c] != x[i][c]) x[i][c] = 0.0f;
      }
    }
  }
  if (bad) atomicOr(a.status, kStatusNonFinite);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int off = kCols / 2; off >= 1; off >>= 1) rmax[i] = fmaxf(rmax[i], __shfl_xor_sync(0xffffffffu, rmax[i], off));
  float m = fmaxf(fmaxf(rmax[0], rmax[1]), fmaxf(rmax[2], rmax[3]));
  for (int r = threadIdx.x; r < lo; r += blockDim.x) m = fmaxf(m, tmax[tail_old + r]);
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
  __syncthreads();
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) m = fmaxf(m, red[w]);
  const int e = block_exponent(m);
  const float inv = pow2f(-e);                 // (2^126 for zeros)
  if (threadIdx.x == 0) exps[block] = (int8_t)e;
  const bool again = lo > 0 && e != e_old;     // the older tokens' codes have another exponent
  const bool open = hi < P;                    // the page stays open: keep its new tokens unrounded
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = r0 + i * step;
    if (row < lo && again) {
      if (is_v) {
        const bf16* p = a.pool.tail_v + (tail_old + row) * D;
        unpack8(*reinterpret_cast<const uint4*>(p + cl.c0), x[i]);
        unpack8(*reinterpret_cast<const uint4*>(p + cl.c1), x[i] + 8);
      } else {
        const float* p = a.pool.tail_k + (tail_old + row) * D;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          x[i][c] = p[cl.c0 + c];
          x[i][8 + c] = p[cl.c1 + c];
        }
      }
    }
    if (row < hi && (row >= lo || again)) {
      *reinterpret_cast<uint2*>(dst + row * D + cl.c0) = codes8(x[i], inv);
      *reinterpret_cast<uint2*>(dst + row * D + cl.c1) = codes8(x[i] + 8, inv);
    }
    if (open && row >= lo && row < hi) {
      if (is_v) {
        bf16* p = a.pool.tail_v + (tail_new + row) * D;
        *reinterpret_cast<uint4*>(p + cl.c0) = pack8(x[i]);
        *reinterpret_cast<uint4*>(p + cl.c1) = pack8(x[i] + 8);
      } else {
        float* p = a.pool.tail_k + (tail_new + row) * D;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          *reinterpret_cast<float4*>(p + cl.c0 + 4 * q) = make_float4(x[i][4 * q], x[i][4 * q + 1], x[i][4 * q + 2], x[i][4 * q + 3]);
          *reinterpret_cast<float4*>(p + cl.c1 + 4 * q) = make_float4(x[i][8 + 4 * q], x[i][9 + 4 * q], x[i][10 + 4 * q], x[i][11 + 4 * q]);
        }
      }
      if (j == 0) tmax[tail_new + row] = rmax[i];
    }
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
  constexpr int kCols = D / 8;
  for (int i = threadIdx.x; i < rows * kCols; i += blockDim.x) {
    const int row = i / kCols, c = (i % kCols) * 8;
    *reinterpret_cast<uint4*>(dst + (int64_t)row * a.Hkv * D + c) =
        values8(*reinterpret_cast<const uint2*>(src + row * D + c), scale);
  }
}

__global__ void table_kernel(const __grid_constant__ TableArgs a) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < a.n) a.table[a.index[i]] = a.page[i];
}

}  // namespace

cudaError_t launch_paged_append(int D, const AppendArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)a.seqs.page0[a.seqs.n], (unsigned)a.Hkv, a.Q ? 3 : 2);
  if (grid.x == 0) return cudaSuccess;
  if (D == 128) append_kernel<128><<<grid, a.P * 2, 0, s>>>(a);
  else append_kernel<64><<<grid, a.P, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_paged_read(int D, const ReadArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)a.seqs.page0[a.seqs.n], (unsigned)a.Hkv, 2);
  if (grid.x == 0) return cudaSuccess;
  if (D == 128) read_kernel<128><<<grid, 256, 0, s>>>(a);
  else read_kernel<64><<<grid, 256, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_paged_table(const TableArgs& a, cudaStream_t s) {
  if (a.n == 0) return cudaSuccess;
  table_kernel<<<(a.n + 127) / 128, 128, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace fk
