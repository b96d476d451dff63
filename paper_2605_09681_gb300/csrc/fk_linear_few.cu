// Linear attention with decays, token by token: S = exp(g) S + k v^T, o = scale q^T S in fp32.
//
// For single tokens and drafts.  A CTA holds 32 columns (channels of v) of one head's state in its registers: D^2 floats of
// each head are read and written once, whatever the number of tokens.
//
// linear_one_kernel: single tokens, bound by the states' bytes (64 streams of 16 heads of 128: 21.3 us, 94% of the measured
// copy rate), and groups of more than 8 query heads.  Thread (r, c): rows r D/16 .. and columns 4c .. 4c + 3, 16 bytes at a time.  A
// token's k and q come straight from global memory (the same 16 or 8 bytes for the 8 threads of a row group), the next
// token's while this one is computed; o is a sum over the 16 row groups: by shuffles in a warp, then over the 4 warps through
// shared memory.
//
// linear_few_kernel: drafts, bound by arithmetic and latency.  Warp w: rows w D/4 .., lane: a column, so that a token's k
// and q are the same for a warp (fp32 pairs in shared memory, blocks of tokens, the next block's on their way) and o needs no
// shuffles.  64 streams of 16 heads of 128, 8 tokens each: 35 us (54.5 through the other kernel; the states' bytes take 20); 16
// streams' drafts of 1 to 8 tokens, 32 over 8 heads of 64: 5.6 us.  One sequence takes 0.28 us a token, all SMs together 3.1 ns a
// token and head (D = 128; by a third more for each further query head).
#include "fk_linear.h"

namespace fk {
namespace {

constexpr int kThreads = 128;
constexpr int kCols = 32;             // of a CTA
constexpr int kSums = 32;             // rows of o that are collected before the warps' parts are added

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n .reg .b64 ra, rb, rc, rd;\n mov.b64 ra, {%2, %3};\n mov.b64 rb, {%4, %5};\n mov.b64 rc, {%6, %7};\n"
      " fma.rn.f32x2 rd, ra, rb, rc;\n mov.b64 {%0, %1}, rd;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

template <int N>
struct Row {                          // N bf16 in registers
  uint32_t w[N / 2];
  __device__ __forceinline__ void load(const bf16* p) {
    if constexpr (N == 8) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {
      const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
      w[0] = v.x, w[1] = v.y;
    }
  }
  __device__ __forceinline__ float get(int i) const {
    return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
  }
};

// This launch ends no earlier than the one before it in the stream, beside which it may run: one block, the last to start, stays.
__device__ __forceinline__ void end_behind() {
  if (blockIdx.x == gridDim.x - 1) asm volatile("griddepcontrol.wait;" ::: "memory");
}

template <int D>
__global__ void __launch_bounds__(kThreads, 8) linear_one_kernel(const __grid_constant__ LinearArgs a) {
  constexpr int kRows = D / 16;       // of a thread
  constexpr int kSlices = D / kCols;
  __shared__ __align__(16) float sums[kSums][4][kCols];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c = tid & 7, r = tid >> 3;
  const int slice = blockIdx.x % kSlices, rest = blockIdx.x / kSlices;
  const int h = rest % a.Hkv, k = rest / a.Hkv;
  const int n = a.seqs.len[k];
  const int64_t tok0 = a.seqs.tok0[k];
  const int64_t at = (int64_t)(r * kRows) * D + slice * kCols + c * 4;
  const float* s0 = a.state + ((int64_t)a.seqs.slot[k] * a.Hkv + h) * (D * D) + at;
  float4 s[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) s[i] = *reinterpret_cast<const float4*>(s0 + i * D);

  const bf16* K = a.K + tok0 * a.kstride + h * D + r * kRows;
  const bf16* V = a.V + tok0 * a.vstride + h * D + slice * kCols + c * 4;
  const bf16* Q = a.Q + tok0 * a.qstride + (int64_t)h * a.G * D + r * kRows;
  const float* decay = a.decay + tok0 * a.dstride + h;
  Row<kRows> kk, qq;
  Row<4> vv;
  float g = 0.0f;
  auto load = [&](int t) {
    kk.load(K + t * a.kstride);
    vv.load(V + t * a.vstride);
    qq.load(Q + t * a.qstride);
    g = __ldg(decay + t * a.dstride);
  };
  // rows [first, first + m) of o, numbered token by token and query head by query head
  auto flush = [&](int64_t first, int m) {
    __syncthreads();
    for (int i = tid; i < m * (kCols / 2); i += kThreads) {
      const int p = i / (kCols / 2), x = 2 * (i % (kCols / 2));
      float2 o = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float2 y = *reinterpret_cast<const float2*>(&sums[p][w][x]);
        o.x += y.x;
        o.y += y.y;
      }
      const int64_t row = first + p, t = row / a.G;
      *reinterpret_cast<__nv_bfloat162*>(a.O + (tok0 + t) * a.ostride + ((int64_t)h * a.G + (row - t * a.G)) * D +
                                         slice * kCols + x) = __floats2bfloat162_rn(o.x * a.scale, o.y * a.scale);
    }
    __syncthreads();
  };
  if (n > 0) load(0);
  int64_t row = 0;
  int held = 0;
  for (int t = 0; t < n; ++t) {
    const Row<kRows> kt = kk;
    const Row<4> vt = vv;
    Row<kRows> q = qq;
    const float e = expf(g), less = expm1f(g);
    if (t + 1 < n) load(t + 1);
    // exp(g) rounded is off by up to 2^-24 at every token alike, and a slow decay takes thousands of them: there what the
    // state loses, S (exp(g) - 1), is added
    if (e > 0.5f) {
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const float x = kt.get(i);
        s[i].x = fmaf(less, s[i].x, fmaf(x, vt.get(0), s[i].x));
        s[i].y = fmaf(less, s[i].y, fmaf(x, vt.get(1), s[i].y));
        s[i].z = fmaf(less, s[i].z, fmaf(x, vt.get(2), s[i].z));
        s[i].w = fmaf(less, s[i].w, fmaf(x, vt.get(3), s[i].w));
      }
    } else {
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const float x = kt.get(i);
        s[i].x = fmaf(e, s[i].x, x * vt.get(0));
        s[i].y = fmaf(e, s[i].y, x * vt.get(1));
        s[i].z = fmaf(e, s[i].z, x * vt.get(2));
        s[i].w = fmaf(e, s[i].w, x * vt.get(3));
      }
    }
    for (int j = 0; j < a.G; ++j) {
      Row<kRows> next = q;
      if (j + 1 < a.G) next.load(Q + t * a.qstride + (j + 1) * D);
      float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const float x = q.get(i);
        o.x = fmaf(x, s[i].x, o.x);
        o.y = fmaf(x, s[i].y, o.y);
        o.z = fmaf(x, s[i].z, o.z);
        o.w = fmaf(x, s[i].w, o.w);
      }
#pragma unroll
      for (int m = 8; m < 32; m *= 2) {
        o.x += __shfl_xor_sync(0xffffffffu, o.x, m);
        o.y += __shfl_xor_sync(0xffffffffu, o.y, m);
        o.z += __shfl_xor_sync(0xffffffffu, o.z, m);
        o.w += __shfl_xor_sync(0xffffffffu, o.w, m);
      }
      if (lane < 8) *reinterpret_cast<float4*>(&sums[held][warp][4 * lane]) = o;
      if (++held == kSums) {
        flush(row, held);
        row += held;
        held = 0;
      }
      q = next;
    }
  }
  if (a.state_new) {
    float* s1 = a.state_new + ((int64_t)(a.to_out ? a.seqs.out[k] : a.seqs.slot[k]) * a.Hkv + h) * (D * D) + at;
#pragma unroll
    for (int i = 0; i < kRows; ++i) *reinterpret_cast<float4*>(s1 + i * D) = s[i];
  }
  if (held > 0) flush(row, held);
  end_behind();
}

constexpr int kMostHeads = 8;         // query heads of a group
constexpr int kBlockRows = 16;        // tokens times query heads of a block

template <int D>
__global__ void __launch_bounds__(kThreads) linear_few_kernel(const __grid_constant__ LinearArgs a) {
  constexpr int kRows = D / 4, kSlices = D / kCols;
  __shared__ __align__(16) float sk[8][D];
  __shared__ __align__(16) float sq[kBlockRows][D];
  __shared__ __align__(16) float sv[8][kCols];
  __shared__ float2 se[8];            // exp(g), exp(g) - 1
  __shared__ __align__(16) float sums[kBlockRows][4][kCols];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int slice = blockIdx.x % kSlices, rest = blockIdx.x / kSlices;
  const int h = rest % a.Hkv, k = rest / a.Hkv, G = a.G;
  const int n = a.seqs.len[k];
  const int64_t tok0 = a.seqs.tok0[k];
  const int tb = G <= 2 ? 8 : G <= 4 ? 4 : 2;                // tokens of a block
  const int64_t at = (int64_t)(warp * kRows) * D + slice * kCols + lane;
  const float* s0 = a.state + ((int64_t)a.seqs.slot[k] * a.Hkv + h) * (D * D) + at;

  // a block's values: 16 bytes of k and of v, and up to two of q
  constexpr int kRuns = D / 8;
  uint4 rk, rv, rq[2];
  float rg = 0.0f;
  auto load = [&](int t0) {
    const int m = min(tb, n - t0);
    if (tid / kRuns < m) rk = __ldg(reinterpret_cast<const uint4*>(a.K + (tok0 + t0 + tid / kRuns) * a.kstride + h * D + tid % kRuns * 8));
    if (tid / 4 < m) rv = __ldg(reinterpret_cast<const uint4*>(a.V + (tok0 + t0 + tid / 4) * a.vstride + h * D + slice * kCols + tid % 4 * 8));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = (tid + i * kThreads) / kRuns, t = r / G;   // row: token, query head
      if (t < m)
        rq[i] = __ldg(reinterpret_cast<const uint4*>(a.Q + (tok0 + t0 + t) * a.qstride + ((int64_t)h * G + r - t * G) * D + tid % kRuns * 8));
    }
    if (tid < m) rg = __ldg(a.decay + (tok0 + t0 + tid) * a.dstride + h);
  };
  auto put = [](float* to, uint4 v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    reinterpret_cast<float4*>(to)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(to)[1] = make_float4(x[4], x[5], x[6], x[7]);
  };
  load(0);
  float2 s[kRows / 2];                // rows 2 i, 2 i + 1
#pragma unroll
  for (int i = 0; i < kRows / 2; ++i) s[i] = make_float2(s0[(2 * i) * D], s0[(2 * i + 1) * D]);

  for (int t0 = 0; t0 < n; t0 += tb) {
    const int m = min(tb, n - t0);
    __syncthreads();
    if (tid / kRuns < m) put(&sk[tid / kRuns][tid % kRuns * 8], rk);
    if (tid / 4 < m) put(&sv[tid / 4][tid % 4 * 8], rv);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = (tid + i * kThreads) / kRuns;
      if (r < m * G) put(&sq[r][tid % kRuns * 8], rq[i]);
    }
    if (tid < m) se[tid] = make_float2(expf(rg), expm1f(rg));
    __syncthreads();
    if (t0 + tb < n) load(t0 + tb);
    for (int t = 0; t < m; ++t) {
      const float4* kk = reinterpret_cast<const float4*>(&sk[t][warp * kRows]);
      const float v1 = sv[t][lane];
      const float2 v = make_float2(v1, v1), e = se[t];
      // (exp(g) rounded is off by up to 2^-24 at every token alike, and a slow decay takes thousands of them: there what the
      // state loses, S (exp(g) - 1), is added)
      if (e.x > 0.5f) {
        const float2 less = make_float2(e.y, e.y);
#pragma unroll
        for (int i = 0; i < kRows / 4; ++i) {
          const float4 x = kk[i];
          s[2 * i] = fma2(less, s[2 * i], fma2(make_float2(x.x, x.y), v, s[2 * i]));
          s[2 * i + 1] = fma2(less, s[2 * i + 1], fma2(make_float2(x.z, x.w), v, s[2 * i + 1]));
        }
      } else {
        const float2 keep = make_float2(e.x, e.x);
#pragma unroll
        for (int i = 0; i < kRows / 4; ++i) {
          const float4 x = kk[i];
          s[2 * i] = fma2(keep, s[2 * i], make_float2(x.x * v1, x.y * v1));
          s[2 * i + 1] = fma2(keep, s[2 * i + 1], make_float2(x.z * v1, x.w * v1));
        }
      }
      for (int g = 0; g < G; ++g) {
        const float4* qq = reinterpret_cast<const float4*>(&sq[t * G + g][warp * kRows]);
        float2 o0 = make_float2(0.0f, 0.0f), o1 = o0;
#pragma unroll
        for (int i = 0; i < kRows / 4; ++i) {
          const float4 x = qq[i];
          o0 = fma2(make_float2(x.x, x.y), s[2 * i], o0);
          o1 = fma2(make_float2(x.z, x.w), s[2 * i + 1], o1);
        }
        sums[t * G + g][warp][lane] = (o0.x + o0.y) + (o1.x + o1.y);
      }
    }
    __syncthreads();
    for (int i = tid; i < m * G * (kCols / 2); i += kThreads) {
      const int r = i / (kCols / 2), x = 2 * (i % (kCols / 2)), t = r / G;
      float2 o = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float2 y = *reinterpret_cast<const float2*>(&sums[r][w][x]);
        o.x += y.x;
        o.y += y.y;
      }
      *reinterpret_cast<__nv_bfloat162*>(a.O + (tok0 + t0 + t) * a.ostride + ((int64_t)h * G + r - t * G) * D + slice * kCols + x) =
          __floats2bfloat162_rn(o.x * a.scale, o.y * a.scale);
    }
  }
  if (a.state_new) {
    float* s1 = a.state_new + ((int64_t)(a.to_out ? a.seqs.out[k] : a.seqs.slot[k]) * a.Hkv + h) * (D * D) + at;
#pragma unroll
    for (int i = 0; i < kRows / 2; ++i) {
      s1[(2 * i) * D] = s[i].x;
      s1[(2 * i + 1) * D] = s[i].y;
    }
  }
  end_behind();
}

__global__ void linear_status_kernel(int* status, int* report) { *report = atomicExch(status, 0); }

}  // namespace

cudaError_t launch_linear_few(int D, const LinearArgs& a, bool beside, cudaStream_t s) {
  const unsigned grid = (unsigned)a.seqs.n * a.Hkv * (D / kCols);
  int most = 0;
  for (int k = 0; k < a.seqs.n; ++k) most = most > a.seqs.len[k] ? most : a.seqs.len[k];
  const bool one = most <= 1 || a.G > kMostHeads;
  const auto kernel = D == 128 ? (one ? linear_one_kernel<128> : linear_few_kernel<128>) : (one ? linear_one_kernel<64> : linear_few_kernel<64>);
  if (beside) return launch_early(kernel, dim3(grid), kThreads, 0, s, a);
  kernel<<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_linear_status(int* status, int* report, cudaStream_t s) {
  linear_status_kernel<<<1, 1, 0, s>>>(status, report);
  return cudaGetLastError();
}

}  // namespace fk
