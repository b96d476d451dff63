// Internal declarations of linear attention with decays: argument blocks and launchers of its kernels.
#pragma once

#include "fk_internal.h"

namespace fk {

constexpr int kLinearSeqs = 256;      // sequences of one launch (their numbers travel by value)
// g below this is taken as this: exp of it is 0 in fp32, and differences of sums stay numbers when a state starts anew
constexpr float kLeastDecay = -110.0f;

struct LinearSeqs {
  int n;
  int slot[kLinearSeqs];
  int out[kLinearSeqs];               // place in state_out
  int tok0[kLinearSeqs];              // first token in the caller's tensors
  int len[kLinearSeqs];
};

struct LinearArgs {
  const bf16* Q;                      // [T][Hkv G][D], rows of a token contiguous
  const bf16* K;                      // [T][Hkv][D]
  const bf16* V;
  bf16* O;
  int64_t qstride, kstride, vstride, ostride;
  const float* decay;                 // [T][Hkv], dstride from token to token (0: [Hkv])
  int64_t dstride;
  float scale;
  int Hkv, G;
  const float* state;                 // [slots][Hkv][D][D], of k and of v
  float* state_new;                   // the same memory (slots), state_out (out), or nullptr
  int to_out;
  int* status;
  LinearSeqs seqs;
};

// The recurrence, token by token.
cudaError_t launch_linear_few(int D, const LinearArgs& a, cudaStream_t s);

// *report = *status, which is cleared
cudaError_t launch_linear_status(int* status, int* report, cudaStream_t s);

#ifdef __CUDACC__
__device__ __forceinline__ float at_least(float g, float least) { return g < least ? least : g; }   // (NaN stays)
#endif

}  // namespace fk
