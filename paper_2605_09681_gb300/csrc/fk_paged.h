// Internal declarations of the paged 8-bit cache: argument blocks and launchers of its kernels.
#pragma once

#include "fk_internal.h"

#include <utility>

namespace fk {

constexpr int kStepSeqs = 256;        // sequences of one launch (their numbers travel by value)
constexpr int kPagedFewRows = 16;     // query rows of a CTA of the few-row kernel, at most
constexpr int kPagedFewTile = 64;     // keys per tile of the few-row kernel

constexpr int kMaxFewSplits = 460;    // key splits of a row of the few-row kernel
constexpr int kPartSlots = 4096;      // CTAs of a launch that share their rows with other key splits, at most

// Stored exponent of a block of zeros (others are at least -120).
constexpr int kZeroExp = -126;
// The attention folds a value block's 2^e into the softmax numerators, w = p 2^(e - r), as f16, relative to a
// reference r that O (fp32) is kept to: e - r stays in [-kRefWindow, 0] where the rows go together, and a block outside asks for
// r = e + kRefRoom: O moves by a power of two, as far as what it holds allows.  f16 has 2^-24 and up, so that p = 2^-24 is the
// smallest that counts at the window's end, and 2^-13 the smallest that keeps all 11 bits (a window of 16 lost all p below 2^-17 there, which
// l counts: thousands of keys of small weight gave 0).
constexpr int kRefWindow = 8, kRefRoom = 2;
constexpr int kNoRef = -1000;         // r before any block but zeros
constexpr int kAskPast = -8;          // log2 of a block's largest p from which on a row simply takes a larger block's reference

constexpr int kAppendFewRows = 8;     // new tokens on a page that one warp takes

constexpr int kStatusNonFinite = 4;   // device status: an appended key or value was not finite
constexpr int kStatusPosition = 8;    // device status: a position outside the rotation tables

// One layer's pages.  A page of P tokens of kv head h is one block: P rows of D codes, contiguous, and
// one exponent e (held value = E4M3 code * 2^e) for keys and one for values.
struct PagedPool {
  uint8_t* k;                         // [n_pages][Hkv][P][D]
  uint8_t* v;
  int8_t* ke;                         // [n_pages][Hkv]
  int8_t* ve;
  // the open (last, unfilled) page of each sequence as it was before the rounding, in two slots that
  // take turns (a step reads the old open page's while it writes the new one's)
  float* tail_k;                      // [max_seqs][2][Hkv][P][D], rotated
  bf16* tail_v;
  float* tail_kmax;                   // [max_seqs][2][Hkv][P]: a token's largest finite magnitude
  float* tail_vmax;
};

// Division of 0 .. 2^31 - 1 by a number that the host knows: q = (umulhi(n, mul) + n) >> shift.
struct FastDiv {
  uint32_t d, mul, shift;
  explicit FastDiv(uint32_t div = 1) : d(div), mul(0), shift(0) {
    while (((uint64_t)1 << shift) < d) ++shift;
    mul = (uint32_t)(((((uint64_t)1 << shift) - d) << 32) / d + 1);
  }
#ifdef __CUDACC__
  __device__ __forceinline__ int div(int n) const { return (int)((__umulhi((uint32_t)n, mul) + (uint32_t)n) >> shift); }
#endif
};

// Sequences of one append or read-back launch.
struct PagedSeqs {
  int n;
  int slot[kStepSeqs];
  int old_len[kStepSeqs];
  int new_len[kStepSeqs];
  int tok0[kStepSeqs];                // first token of the sequence in the caller's tensors
  int page0[kStepSeqs + 1];           // pages before the sequence's first one in this launch
  uint8_t buf[kStepSeqs];             // bit 0: tail slot read, bit 1: tail slot written
};

struct AppendArgs {
  PagedPool pool;
  const int* table;                   // [max_seqs][max_pages]
  int max_pages, Hkv, G, P;
  int most;                           // new tokens on a page, at most
  FastDiv by_g;                       // row of a page's queries -> token
  const bf16* K;                      // [T][Hkv][D], rows of a token contiguous, kstride from token to token
  const bf16* V;
  const bf16* Q;                      // [T][Hkv G][D] or nullptr
  bf16* Qr;                           // [T][Hkv G][D]
  int64_t kstride, vstride, qstride, qrstride;
  const float* cos;                   // [rope_rows][R / 2] or nullptr: no rotation
  const float* sin;
  const int* positions;               // table row of each token (nullptr: its place in the sequence)
  int rope_rows, R, interleaved;
  int* status;
  PagedSeqs seqs;
};
cudaError_t launch_paged_append(int D, const AppendArgs& a, cudaStream_t s);

// Held keys and values of tokens first(s) .. new_len - 1 of each sequence as bf16, first(s) = the first token of
// the first page that the step writes (or 0): page0 counts from that page, tok0 its place in the output.
struct ReadArgs {
  PagedPool pool;
  const int* table;
  int max_pages, Hkv, P;
  int whole;                          // 1: from token 0
  bf16* K;                            // [tokens][Hkv][D]
  bf16* V;
  PagedSeqs seqs;
};
cudaError_t launch_paged_read(int D, const ReadArgs& a, cudaStream_t s);

constexpr int kTableEntries = 480;
struct TableArgs {                    // table[index[i]] = page[i]
  int* table;
  int n;
  int index[kTableEntries];
  int page[kTableEntries];
};
cudaError_t launch_paged_table(const TableArgs& a, cudaStream_t s);

// *report = what is to be reported of *status, which is cleared of it
cudaError_t launch_paged_status(int* status, int* report, cudaStream_t s);

// Visible keys of the query at position p of a sequence of n keys: j < (causal ? p + 1 : n), and under a window W
// also j > p - W or j < sinks.
struct PagedMask {
  int causal, window, sinks;
};
// Key tiles of `tile` keys that hold a visible key of some query at positions p0 .. p1: tiles
// [0, n_sink) and [first, last).
struct TileRange {
  int n_sink, first, last;
  __host__ __device__ int count() const { return n_sink + (last > first ? last - first : 0); }
  // the i-th of them
  __host__ __device__ int at(int i) const { return i < n_sink ? i : first + (i - n_sink); }
};
__host__ __device__ inline TileRange paged_tiles(int n_keys, int p0, int p1, const PagedMask& m, int tile) {
  int end = m.causal ? (p1 + 1 < n_keys ? p1 + 1 : n_keys) : n_keys;
  if (end < 0) end = 0;               // queries before the first key
  TileRange r{0, 0, end > 0 ? (end + tile - 1) / tile : 0};
  if (m.window > 0) {
    const int lo = p0 - m.window + 1;
    r.first = lo > 0 ? lo / tile : 0;
    if (r.first > r.last) r.first = r.last;
    const int s = ((m.sinks < end ? m.sinks : end) + tile - 1) / tile;
    r.n_sink = s < r.first ? s : r.first;
  }
  return r;
}

struct PagedAttnSeqs {
  int n;
  int slot[kStepSeqs];
  int n_keys[kStepSeqs];
  int q0[kStepSeqs];                  // first query of the sequence in Q and O
  int n_q[kStepSeqs];
  int item0[kStepSeqs + 1];           // work items before the sequence's first one
  int part0[kStepSeqs];               // workspace slots before the sequence's first one (key splits)
  int splits[kStepSeqs];              // key splits of an item
  int whole[kStepSeqs];               // chunk kernel: (rows, kv head) pairs that are not split, the first ones
  int join0[kStepSeqs + 1];           // chunk kernel: split pairs before the sequence's first one
};

struct PagedAttnArgs {
  const int* table;
  const uint8_t* k;                   // as in PagedPool
  const uint8_t* v;
  const int8_t* ke;
  const int8_t* ve;
  int max_pages, Hkv, G, P;
  FastDiv by_g;                       // query row -> query (row = query * G + head of the group)
  const bf16* Q;                      // [T][Hkv G][D]
  bf16* O;
  int64_t qstride, ostride;
  int wide_o;                         // rows of O are 32-byte aligned
  int join;                           // 16-row CTAs: there are splits to join
  float scale_log2;                   // log2(e) * scale
  PagedMask mask;
  // partial O of the key splits and then (m, l, r, -) of their rows: [kPartSlots][16][D] and [..][16][4] (few
  // rows), [part_tiles][128][D] and [..][128][4] (chunks)
  float* part;
  int part_tiles;
  int* arrived;                       // [kPartSlots]: splits of a group that are done (0 between launches)
  int* status;
  PagedAttnSeqs seqs;
};
// 8 row_tiles (1 or 2) query rows (query, head of the group) per CTA, any number of keys.
cudaError_t launch_paged_few(int D, int row_tiles, const CUtensorMap& tmK, const CUtensorMap& tmV, const PagedAttnArgs& a,
                             cudaStream_t s);
cudaError_t paged_few_prepare(int D);
// Any number of query rows, 256 per CTA (one_tile: 128).
cudaError_t launch_paged_chunk(int D, bool one_tile, const CUtensorMap& tmK, const CUtensorMap& tmV,
                               const PagedAttnArgs& a, cudaStream_t s);
cudaError_t paged_chunk_prepare(int D);

#ifdef __CUDACC__
// exponent e of x > 0, 2^e > x (below 2^-126: -126)
__device__ __forceinline__ int above2(float x) { return (int)(__float_as_uint(x) >> 23) - 126; }

// A join's launch may come while the kernel before it in the stream still runs (that one allows it, once all its CTAs have
// started): the join waits for its end, and its writes, before it reads anything.
__device__ __forceinline__ void allow_join() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_parts() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <class... Params, class... Args>
cudaError_t launch_join(void (*kernel)(Params...), dim3 grid, unsigned threads, cudaStream_t s, Args&&... args) {
  cudaLaunchAttribute early{};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}
#endif

}  // namespace fk
