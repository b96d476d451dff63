// Rotary positions: queries and keys turned by their positions, and tables of the angles.
//
// A pair's angle is position * f modulo a turn.  f is kept as a 64-bit fraction of a turn, so that the 64-bit product
// with the position, taken modulo 2^64, is the angle modulo whole turns without any error: an fp32 product of
// a position and a frequency is off by a radian and more at position 10^7.  It is then rounded to fp32 (three roundings of at
// most a quarter turn: under 2^-24 of a turn).
//
// Both kernels move each byte once.  The angles are the expensive part (a sine and a cosine of a pair take as long as the
// rotation of three heads), so a thread turns the same 8 pairs of several heads, and the rotation is bound by DRAM: 40003
// tokens of 40 heads of 64 in fp16 in 65.6 us, 92% of the measured copy rate, in fp32 in 126 us, 96%; a video chunk (4680 tokens of 24
// heads of 128, 57 MB, where loads wait for the angles and there is one round of blocks) in 13.6 us, 63%.  The tables are bound by the
// angles' arithmetic: 131072 x 64 in 15.3 us (14.6 where they stay in L2), 10 us of which their writes would take.
#include "fk_internal.h"
#include "fk_rows.h"

#include <cuda_fp16.h>

#include <cmath>

namespace fk {
namespace {

constexpr int kMaxPairs = 128;
constexpr int kThreads = 256;
constexpr int kBlocksPerSm = 4;       // of rotate_kernel (64 registers)
constexpr int kSms = 152;

struct Angles {
  uint64_t turns[kMaxPairs];
  const int* positions;               // [tokens][axes]
  int axes;
  int first[4];                       // first pair of each axis
  float magnitude;
};

struct RotateArgs {
  Angles a;
  int64_t tokens;
  int dim, units, rotated;            // units of a head: 8 pairs each, then 8 channels each that are copied
  int per_block, per_group;           // tokens of a block, heads of a thread
  int heads1, heads;                  // of the first tensor, of both
  int head_dim;
  const char* x[2];
  char* y[2];
  int64_t xs[2], ys[2];               // bytes from token to token
  int inverse;
};

struct TableArgs {
  Angles a;
  int64_t tokens;
  int pairs, per_block, rounds;       // tokens of a block at once, and how often
  float* cos;
  float* sin;
};

// The fractions in shared memory: every thread reads others, which one warp's read of the arguments takes one after the
// other (half of the tables' time when all did).
__device__ __forceinline__ void stage(const Angles& a, int pairs, uint64_t* s) {
  for (int i = threadIdx.x; i < pairs; i += blockDim.x) s[i] = a.turns[i];
  __syncthreads();
}

// cos and sin of the angle `pos * turns` (times m, sin with the sign of `dir`).  The fraction of a turn is taken to the nearest
// half and a rest a of at most pi / 2 either way, whose sine and cosine are the first seven terms of their series:
// the next ones are a^15 / 15! < 2^-30 and a^14 / 14! < 2^-27; with the roundings 2^-23.  (The device is busier with integers and signs
// than with products: to the nearest quarter, five terms and more to choose from, a whole context's tables took 19.7 us, so 18.1, 17.3 with
// positions of several axes taken by address and not by choice, 16.8 with two pairs' products in one; with sincospif 40.)
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n .reg .b64 ra, rb, rc, rd;\n mov.b64 ra, {%2, %3};\n mov.b64 rb, {%4, %5};\n mov.b64 rc, {%6, %7};\n"
      " fma.rn.f32x2 rd, ra, rb, rc;\n mov.b64 {%0, %1}, rd;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 two(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return fma2(a, b, two(-0.0f)); }

// the rest of an angle in radians, and its odd half turn in the highest bit
__device__ __forceinline__ float rest(uint64_t turns, int pos, uint32_t* odd) {
  const uint64_t t = turns * (uint64_t)(int64_t)pos + (1ull << 62);   // + 1/4: the half is rounded, not cut off
  const uint32_t top = (uint32_t)(t >> 32);
  *odd = top & 0x80000000u;
  return fmaf((float)(uint32_t)t, 0x1p-32f, (float)((int32_t)(top & 0x7FFFFFFFu) - 0x40000000)) * (6.2831853071795865f * 0x1p-32f);
}
// of two pairs
__device__ __forceinline__ void angles(const uint64_t* turns, int pos0, int pos1, float m, float dir, float* c, float* s) {
  uint32_t odd[2];
  const float2 a = make_float2(rest(turns[0], pos0, &odd[0]), rest(turns[1], pos1, &odd[1])), z = mul2(a, a);
  float2 sn = fma2(z, two(1.0f / 6227020800), two(-1.0f / 39916800)), cs = fma2(z, two(1.0f / 479001600), two(-1.0f / 3628800));
  for (const float x : {1.0f / 362880, -1.0f / 5040, 1.0f / 120, -1.0f / 6}) sn = fma2(z, sn, two(x));
  for (const float x : {1.0f / 40320, -1.0f / 720, 1.0f / 24, -0.5f, 1.0f}) cs = fma2(z, cs, two(x));
  sn = fma2(mul2(a, z), sn, a);
  c[0] = cs.x * __uint_as_float(__float_as_uint(m) ^ odd[0]);
  c[1] = cs.y * __uint_as_float(__float_as_uint(m) ^ odd[1]);
  s[0] = sn.x * __uint_as_float(__float_as_uint(dir) ^ odd[0]);
  s[1] = sn.y * __uint_as_float(__float_as_uint(dir) ^ odd[1]);
}

// a token's positions, and a pair's of them
struct Places {
  int at[4];
  __device__ __forceinline__ Places(const Angles& a, int64_t t) {
    const int* p = a.positions + t * a.axes;
    at[0] = __ldg(p);
#pragma unroll
    for (int i = 1; i < 4; ++i) at[i] = i < a.axes ? __ldg(p + i) : 0;
  }
  __device__ __forceinline__ int of(const Angles& a, int pair) const {   // (behind the last axis, `first` is past all pairs)
    return pair < a.first[1] ? at[0] : pair < a.first[2] ? at[1] : pair < a.first[3] ? at[2] : at[3];
  }
};

// eight channels in memory <-> fp32
template <class T>
struct Eight;
template <>
struct Eight<float> {
  float4 v[2];
  __device__ __forceinline__ void load(const char* p) {
    v[0] = reinterpret_cast<const float4*>(p)[0];
    v[1] = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void store(char* p) const {
    reinterpret_cast<float4*>(p)[0] = v[0];
    reinterpret_cast<float4*>(p)[1] = v[1];
  }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = v[0].x, x[1] = v[0].y, x[2] = v[0].z, x[3] = v[0].w;
    x[4] = v[1].x, x[5] = v[1].y, x[6] = v[1].z, x[7] = v[1].w;
  }
  __device__ __forceinline__ void set(const float* x) {
    v[0] = make_float4(x[0], x[1], x[2], x[3]);
    v[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
};
template <class T, class T2>
struct EightHalves {
  uint4 v;
  __device__ __forceinline__ void load(const char* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(char* p) const { *reinterpret_cast<uint4*>(p) = v; }
};
template <>
struct Eight<bf16> : EightHalves<bf16, __nv_bfloat162> {
  __device__ __forceinline__ void get(float* x) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
  __device__ __forceinline__ void set(const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Eight<__half> : EightHalves<__half, __half2> {
  __device__ __forceinline__ void get(float* x) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      x[2 * i] = f.x, x[2 * i + 1] = f.y;
    }
  }
  __device__ __forceinline__ void set(const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 p = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// One thread: a unit of a token, in the heads of one group.  kHalf: pairs (i, i + dim / 2).
template <class T, bool kHalf>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const __grid_constant__ RotateArgs a) {
  __shared__ uint64_t turns[kMaxPairs];
  stage(a.a, a.dim / 2, turns);
  const int tb = threadIdx.x / a.units, u = threadIdx.x - tb * a.units;
  const int64_t t = (int64_t)blockIdx.x * a.per_block + tb;
  if (tb >= a.per_block || t >= a.tokens) return;
  const int h0 = blockIdx.y * a.per_group, h1 = min(h0 + a.per_group, a.heads);
  const bool turn = u < a.rotated;
  // byte offsets in a head of the unit's two blocks of 8 channels (one block where channels are copied)
  const int c0 = turn ? (kHalf ? 8 * u : 16 * u) : a.dim + 8 * (u - a.rotated);
  const int c1 = kHalf ? c0 + a.dim / 2 : c0 + 8;
  float cs[8], sn[8];
  if (turn) {
    const Places pos(a.a, t);
    const float dir = a.inverse ? -a.a.magnitude : a.a.magnitude;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const int p = 8 * u + i;
      angles(turns + p, pos.of(a.a, p), pos.of(a.a, p + 1), a.a.magnitude, dir, cs + i, sn + i);
    }
  }
  // several heads' loads before the first is turned: a thread's own are few bytes
  constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;
#pragma unroll 1
  for (int hb = h0; hb < h1; hb += kAhead) {
    Eight<T> p[kAhead], q[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int h = hb + j, k = h >= a.heads1, hh = k ? h - a.heads1 : h;
      const char* x = a.x[k] + t * a.xs[k] + (int64_t)hh * a.head_dim * sizeof(T);
      if (h < h1) {
        p[j].load(x + c0 * sizeof(T));
        if (turn) q[j].load(x + c1 * sizeof(T));
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int h = hb + j, k = h >= a.heads1, hh = k ? h - a.heads1 : h;
      char* y = a.y[k] + t * a.ys[k] + (int64_t)hh * a.head_dim * sizeof(T);
      if (h >= h1) break;
      if (turn) {
        float f[16];
        p[j].get(f);
        q[j].get(f + 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float& u0 = kHalf ? f[i] : f[2 * i];
          float& u1 = kHalf ? f[8 + i] : f[2 * i + 1];
          const float v0 = fmaf(u0, cs[i], -(u1 * sn[i])), v1 = fmaf(u1, cs[i], u0 * sn[i]);
          u0 = v0;
          u1 = v1;
        }
        p[j].set(f);
        q[j].set(f + 8);
        q[j].store(y + c1 * sizeof(T));
      }
      p[j].store(y + c0 * sizeof(T));
    }
  }
}

// One thread: 4 pairs of several tokens, per_block apart.
__global__ void __launch_bounds__(kThreads) tables_kernel(const __grid_constant__ TableArgs a) {
  __shared__ uint64_t all[kMaxPairs];
  stage(a.a, a.pairs, all);
  const int quads = a.pairs / 4, tb = threadIdx.x / quads, p = 4 * (threadIdx.x - tb * quads);
  if (tb >= a.per_block) return;
  uint64_t turns[4];
  int axis[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    turns[i] = all[p + i];
    axis[i] = (p + i >= a.a.first[1]) + (p + i >= a.a.first[2]) + (p + i >= a.a.first[3]);
  }
  const int64_t t0 = (int64_t)blockIdx.x * a.per_block * a.rounds + tb;
  for (int r = 0; r < a.rounds; ++r) {
    const int64_t t = t0 + (int64_t)r * a.per_block;
    if (t >= a.tokens) return;
    const int* pos = a.a.positions + t * a.a.axes;
    float c[4], s[4];
#pragma unroll
    for (int i = 0; i < 4; i += 2)
      angles(turns + i, __ldg(pos + axis[i]), __ldg(pos + axis[i + 1]), a.a.magnitude, a.a.magnitude, c + i, s + i);
    *reinterpret_cast<float4*>(a.cos + t * a.pairs + p) = make_float4(c[0], c[1], c[2], c[3]);
    *reinterpret_cast<float4*>(a.sin + t * a.pairs + p) = make_float4(s[0], s[1], s[2], s[3]);
  }
}

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int current_device() {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) cudaGetLastError();
  return dev;
}

bool on_device(const void* p, int dev) {
  cudaPointerAttributes at{};
  if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  return at.type == cudaMemoryTypeManaged || (at.type == cudaMemoryTypeDevice && at.device == dev);
}

// what fk_rotary_make makes
bool made(const fk_rotary& r) {
  if (r.head_dim < 16 || r.head_dim > 256 || r.head_dim % 8 || r.dim < 16 || r.dim > r.head_dim || r.dim % 16) return false;
  if (r.style != FK_ROPE_HALF && r.style != FK_ROPE_INTERLEAVED) return false;
  if (r.n_axes < 1 || r.n_axes > 4 || r.first[0] != 0) return false;
  for (int i = 1; i < 4; ++i)
    if (i < r.n_axes ? r.first[i] <= r.first[i - 1] || r.first[i] >= r.dim / 2 : r.first[i] != r.dim / 2) return false;
  return std::isfinite(r.magnitude);
}

void fill(const fk_rotary& r, const int32_t* positions, Angles* a) {
  for (int i = 0; i < kMaxPairs; ++i) a->turns[i] = r.turns[i];
  a->positions = positions;
  a->axes = r.n_axes;
  for (int i = 0; i < 4; ++i) a->first[i] = r.first[i];
  a->magnitude = r.magnitude;
}

// A frequency in radians a position -> the fraction of a turn in 2^-64 (its sign goes into the two's complement).  f / 2 pi as two
// doubles: one alone is off by up to 2^-54 of a turn, which 2^31 positions make 2^-23.
uint64_t turns_of(double f) {
  constexpr double kInverse = 0.15915494309189535, kRest = -9.839338337591243e-18;   // of 2 pi
  const double x = std::fabs(f), t = x * kInverse, rest = std::fma(x, kInverse, -t) + x * kRest;   // t below 1/2
  const double hi = std::floor(std::ldexp(t, 32)), lo = std::ldexp(std::ldexp(t, 32) - hi, 32);
  const uint64_t u = ((uint64_t)hi << 32) + (uint64_t)(int64_t)std::floor(lo + std::ldexp(rest, 64));
  return f < 0 ? 0 - u : u;
}

template <class T>
cudaError_t launch_rotate(const RotateArgs& a, int style, dim3 grid, cudaStream_t s) {
  if (style == FK_ROPE_HALF) rotate_kernel<T, true><<<grid, kThreads, 0, s>>>(a);
  else rotate_kernel<T, false><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace
}  // namespace fk

using namespace fk;

extern "C" {

fk_status fk_rotary_make(const fk_rotary_config* c, fk_rotary* out) {
  if (!c || !out) return FK_ERR_ARG;
  fk_rotary r{};
  r.head_dim = c->head_dim;
  r.dim = c->dim;
  r.style = c->style;
  r.n_axes = c->n_axes;
  if (c->n_axes < 1 || c->n_axes > 4) return FK_ERR_CONFIG;
  if (c->scaling < FK_ROPE_SCALE_NONE || c->scaling > FK_ROPE_SCALE_RAMP) return FK_ERR_CONFIG;
  if (!std::isfinite(c->magnitude) || c->magnitude < 0.0) return FK_ERR_CONFIG;
  int n = 0;
  for (int a = 0; a < 4; ++a) {
    r.first[a] = n;
    if (a >= c->n_axes) continue;
    if (c->pairs[a] < 1 || c->pairs[a] > kMaxPairs) return FK_ERR_CONFIG;
    n += c->pairs[a];
  }
  r.magnitude = c->magnitude > 0.0 ? (float)c->magnitude : 1.0f;
  if (2 * n != c->dim || !made(r)) return FK_ERR_CONFIG;
  if (c->frequencies) {
    for (int i = 0; i < n; ++i) {
      if (!(std::fabs(c->frequencies[i]) < 3.14159265358979)) return FK_ERR_CONFIG;
      r.turns[i] = turns_of(c->frequencies[i]);
    }
    *out = r;
    return FK_OK;
  }
  if (!(c->base > 1.0) || std::isinf(c->base)) return FK_ERR_CONFIG;
  if (c->scaling != FK_ROPE_SCALE_NONE && (!(c->factor >= 1.0) || std::isinf(c->factor))) return FK_ERR_CONFIG;
  if (c->scaling == FK_ROPE_SCALE_RAMP) {
    if (c->original_tokens < 1 || !(c->slow_turns >= 0.0) || !(c->fast_turns > c->slow_turns) || std::isinf(c->fast_turns))
      return FK_ERR_CONFIG;
    if (!(c->magnitude > 0.0)) r.magnitude = (float)(0.1 * std::log(c->factor) + 1.0);
  }
  for (int a = 0; a < c->n_axes; ++a) {
    const double d = 2.0 * c->pairs[a];
    if (c->scaling == FK_ROPE_SCALE_BASE && c->pairs[a] < 2) return FK_ERR_CONFIG;
    const double base = c->scaling == FK_ROPE_SCALE_BASE ? c->base * std::pow(c->factor, d / (d - 2.0)) : c->base;
    for (int i = 0; i < c->pairs[a]; ++i) {
      double f = std::pow(base, -2.0 * i / d);
      if (c->scaling == FK_ROPE_SCALE_LINEAR) f /= c->factor;
      if (c->scaling == FK_ROPE_SCALE_RAMP) {
        const double t = c->original_tokens * f / 6.283185307179586476925286766559;
        const double keep = std::fmin(1.0, std::fmax(0.0, (t - c->slow_turns) / (c->fast_turns - c->slow_turns)));
        f = f * keep + f / c->factor * (1.0 - keep);
      }
      r.turns[r.first[a] + i] = turns_of(f);
    }
  }
  *out = r;
  return FK_OK;
}

fk_status fk_rotate(const fk_rotary* r, int64_t tokens, const int32_t* positions, int inverse, int type, const void* X,
                    int64_t x_stride, int x_heads, void* Y, int64_t y_stride, const void* X2, int64_t x2_stride, int x2_heads,
                    void* Y2, int64_t y2_stride, void* stream) {
  if (!r) return FK_ERR_ARG;
  if (!made(*r) || (inverse != 0 && inverse != 1) || type < FK_TYPE_BF16 || type > FK_TYPE_F32) return FK_ERR_CONFIG;
  if (tokens < 0 || tokens >= ((int64_t)1 << 31)) return FK_ERR_CONFIG;
  if (x_heads < 1 || x_heads > 1024 || x2_heads < 0 || x2_heads > 1024) return FK_ERR_CONFIG;
  if (tokens == 0) return FK_OK;        // (tensors of no tokens may have no address)
  if (!X2 != !Y2 || !X2 != (x2_heads == 0)) return FK_ERR_ARG;
  const int size = type == FK_TYPE_F32 ? 4 : 2;
  const int dev = current_device();
  auto rows_ok = [&](const void* p, int64_t stride, int heads) {
    return p && aligned(p, 16) && stride >= (int64_t)heads * r->head_dim && stride * size % 16 == 0 && on_device(p, dev);
  };
  if (!positions || !aligned(positions, 4) || !on_device(positions, dev)) return FK_ERR_ARG;
  if (!rows_ok(X, x_stride, x_heads) || !rows_ok(Y, y_stride, x_heads)) return FK_ERR_ARG;
  if (X2 && (!rows_ok(X2, x2_stride, x2_heads) || !rows_ok(Y2, y2_stride, x2_heads))) return FK_ERR_ARG;
  // outputs meet nothing but their own input, row for row
  auto rows = [&](const void* p, int64_t stride, int heads) {
    return Rows{reinterpret_cast<uintptr_t>(p), stride * size, (int64_t)heads * r->head_dim * size};
  };
  const Rows at{reinterpret_cast<uintptr_t>(positions), r->n_axes * 4, r->n_axes * 4};
  const Rows x = rows(X, x_stride, x_heads), y = rows(Y, y_stride, x_heads);
  auto apart = [&](const Rows& in, const Rows& out) { return in.p == out.p ? in.stride == out.stride : !meet(in, out, tokens); };
  if (!apart(x, y) || meet(at, y, tokens)) return FK_ERR_ARG;
  if (X2) {
    const Rows x2 = rows(X2, x2_stride, x2_heads), y2 = rows(Y2, y2_stride, x2_heads);
    if (!apart(x2, y2) || meet(at, y2, tokens) || meet(x, y2, tokens) || meet(x2, y, tokens) || meet(y, y2, tokens)) return FK_ERR_ARG;
  }
  RotateArgs a;
  fill(*r, positions, &a.a);
  a.tokens = tokens;
  a.dim = r->dim;
  a.rotated = r->dim / 16;
  a.units = a.rotated + (r->head_dim - r->dim) / 8;
  a.heads1 = x_heads;
  a.heads = x_heads + x2_heads;
  a.head_dim = r->head_dim;
  a.inverse = inverse;
  a.x[0] = static_cast<const char*>(X);
  a.x[1] = static_cast<const char*>(X2);
  a.y[0] = static_cast<char*>(Y);
  a.y[1] = static_cast<char*>(Y2);
  a.xs[0] = x_stride * size;
  a.xs[1] = x2_stride * size;
  a.ys[0] = y_stride * size;
  a.ys[1] = y2_stride * size;
  // Heads of a thread: its angles take as long as three of them, and the last of a few rounds of blocks as long as a full one
  // (4680 tokens of 24 heads: 6 heads in one round 13.4 us, 4 in one and a half 14.5).
  a.per_block = kThreads / a.units;
  const int64_t columns = (tokens + a.per_block - 1) / a.per_block;
  a.per_group = 1;
  double least = 1e30;
  for (int p = 1; p <= 8 && p <= a.heads; ++p) {
    double rounds = (double)(columns * ((a.heads + p - 1) / p)) / (kSms * kBlocksPerSm);
    if (rounds < 4.0) rounds = std::ceil(rounds);
    if (rounds * (3 + p) < least) {
      least = rounds * (3 + p);
      a.per_group = p;
    }
  }
  const dim3 grid((unsigned)columns, (unsigned)((a.heads + a.per_group - 1) / a.per_group));
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (type == FK_TYPE_BF16) e = launch_rotate<bf16>(a, r->style, grid, s);
  else if (type == FK_TYPE_F16) e = launch_rotate<__half>(a, r->style, grid, s);
  else e = launch_rotate<float>(a, r->style, grid, s);
  return e == cudaSuccess ? FK_OK : FK_ERR_CUDA;
}

fk_status fk_rotary_tables(const fk_rotary* r, int64_t tokens, const int32_t* positions, float* cos, float* sin, void* stream) {
  if (!r) return FK_ERR_ARG;
  if (!made(*r) || tokens < 0 || tokens >= ((int64_t)1 << 31)) return FK_ERR_CONFIG;
  if (tokens == 0) return FK_OK;
  const int dev = current_device();
  if (!positions || !aligned(positions, 4) || !on_device(positions, dev)) return FK_ERR_ARG;
  for (const float* p : {cos, sin})
    if (!p || !aligned(p, 16) || !on_device(p, dev)) return FK_ERR_ARG;
  auto all = [&](const void* p, int64_t width) { return Rows{reinterpret_cast<uintptr_t>(p), width, tokens * width}; };
  const Rows at = all(positions, r->n_axes * 4), c = all(cos, r->dim * 2), n = all(sin, r->dim * 2);
  if (meet(at, c, 1) || meet(at, n, 1) || meet(c, n, 1)) return FK_ERR_ARG;
  TableArgs a;
  fill(*r, positions, &a.a);
  a.tokens = tokens;
  a.pairs = r->dim / 2;
  a.cos = cos;
  a.sin = sin;
  a.per_block = kThreads / (a.pairs / 4);
  // (a thread's frequencies are for many tokens, but the device wants threads first)
  a.rounds = 1;
  while (a.rounds < 16 && tokens * (a.pairs / 4) / (2 * a.rounds) >= (int64_t)kSms * 2048) a.rounds *= 2;
  const int64_t block = (int64_t)a.per_block * a.rounds;
  tables_kernel<<<(unsigned)((tokens + block - 1) / block), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
  return cudaGetLastError() == cudaSuccess ? FK_OK : FK_ERR_CUDA;
}

}  // extern "C"
