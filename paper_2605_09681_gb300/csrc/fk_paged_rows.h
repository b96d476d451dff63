// Device code that the attention kernels of the paged 8-bit cache share: a row's reference (see kRefWindow), its parts joined, its O
// written.
#pragma once

#include "fk_paged.h"
#include "fk_tc.h"

namespace fk {
namespace {

// Where a row's reference r goes when a block that it sees asks for `to`.  p: log2 of the row's largest numerator in the block; 2^top > |O|
// relative to r (a numerator of 1 in a block of reference r is 2^kRowTop there at most).  Not lower than leaves O room, which then grows, and
// no higher above what the row holds or the block adds than leaves the bits of both.
constexpr int kRowTop = 16, kRoom = 110, kAbove = 8;
__device__ __forceinline__ int follow(int r, int to, float p, int top) {
  const int most = max(r + top - kRowTop, to + (int)fmaxf(p, -1000.0f));
  return max(max(min(to, most + kAbove), -120), max(r + top - kRoom, r - 127));
}

// O = 2^r x / l by two factors (their product need not be a number of fp32).  No visible key (l = 0): 0.
struct Normal {
  float by_l, size;
  __device__ __forceinline__ Normal(float l, int r) : by_l(l > 0.0f || l != l ? 1.0f / l : 0.0f), size(pow2_any(r)) {}
  __device__ __forceinline__ uint2 bf16x4(const float4& x) const {
    return make_uint2(pack_bf16(x.x * by_l * size, x.y * by_l * size), pack_bf16(x.z * by_l * size, x.w * by_l * size));
  }
};

// Parts of a row's keys, each with its maximum m, its l and its reference r, joined by a warp: weights 2^(m - M) of l, M = max m, and
// 2^((m - M) + (r - R)) of O.  R: the largest r, unless no part holds nearly 2^R (then that of what they hold).  e0: part `lane`.
template <class Part>
__device__ __forceinline__ float join_ref(float M, float R, const float4& e0, int n, Part part) {
  float most = (e0.x - M) + e0.z;
  if (__any_sync(0xffffffffu, most >= R - 40.0f)) return R;
  for (int i = (threadIdx.x & 31) + 32; i < n; i += 32) {
    const float4 e = part(i);
    most = fmaxf(most, (e.x - M) + e.z);
  }
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
  return floorf(most);
}

}  // namespace
}  // namespace fk
