// Internal declarations of linear attention with decays: argument blocks and launchers of its kernels.
#pragma once

#include "fk_internal.h"

#include <utility>

namespace fk {

constexpr int kLinearSeqs = 256;      // sequences of one launch (their numbers travel by value)
// g below this is taken as this: exp of it is 0 in fp32 (the least positive number is exp(-103.3)), and differences of sums stay
// numbers when a state starts anew.  Among tokens that grow the least is lower, since 127 of them may multiply by exp(11268).
constexpr float kLeastDecay = -110.0f, kLeastAmongGrowth = -12000.0f;
// exp of more is no fp32 number: nothing is from there on
constexpr float kMostGrowth = 88.72283f;

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

// Chunks of kLinearChunk tokens on the tensor cores; a work item is a segment (a run of chunks) of one kv head of a sequence.
constexpr int kLinearChunk = 128;
struct LinearChunkSeqs {
  int n;
  int slot[kLinearSeqs];
  int out[kLinearSeqs];
  int tok0[kLinearSeqs];
  int len[kLinearSeqs];               // at least 1
  int segs[kLinearSeqs];              // segments of a head
  int per[kLinearSeqs];               // chunks of a segment, rounded down
  int place0[kLinearSeqs];            // its states' places in the workspace, where segs > 1: place0 + head * segs + segment
  int item0[kLinearSeqs + 1];         // items before the sequence's first one
};
struct LinearChunkArgs {
  bf16* O;
  const bf16* Q;                      // (the tiles come by tensor maps: for values that are not finite)
  const bf16* K;
  const bf16* V;
  int64_t ostride, qstride, kstride, vstride;
  float log2_scale;
  const float* decay;
  int64_t dstride;
  float scale;
  int Hkv, G;
  const float* state;
  float* state_new;
  int to_out;
  float* place;                       // [places][D][D]: the state before a segment
  float2* place_decay;                // [places]: what the segment before it leaves of a state, in two parts
  int* status;
  int items, ctas;                    // work items, CTAs that take them in turn
  LinearChunkSeqs seqs;
};
cudaError_t linear_chunk_prepare(int D);
// With segments: first what each adds to a state that starts at zero (all but the last), then the states before each.
cudaError_t launch_linear_chunk(int D, bool split, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                                const CUtensorMap& tmO, const LinearChunkArgs& a, cudaStream_t s);

// [rows][cols] bf16, `stride` elements from row to row: tiles of box_rows rows of 64 columns, 128-byte swizzle.
bool encode_bf16_rows(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t stride, int box_rows);

// The recurrence, token by token.  beside: it may run beside the chunks' launch before it (of other sequences).
cudaError_t launch_linear_few(int D, const LinearArgs& a, bool beside, cudaStream_t s);

// *report = *status, which is cleared
cudaError_t launch_linear_status(int* status, int* report, cudaStream_t s);

#ifdef __CUDACC__
// A launch that may come before the end of the kernel before it in the stream.  It, or what it waits for, waits for that one's end
// before it ends itself, so that the stream's order holds behind it.
template <class... Params, class... Args>
inline cudaError_t launch_early(void (*kernel)(Params...), dim3 grid, unsigned threads, size_t smem, cudaStream_t s, Args&&... args) {
  cudaLaunchAttribute early{};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

__device__ __forceinline__ float at_least(float g, float least) { return g < least ? least : g; }   // (NaN stays)
#endif

}  // namespace fk
