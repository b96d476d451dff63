// Host side of the paged 8-bit cache: sequences, pages and steps, and the C ABI (fk_paged_*).
//
// The host knows every length, so it hands the kernels their sequences by value (kStepSeqs to a launch) and only the
// page table lives on the device; it changes by a small kernel when a step takes pages.  Nothing is allocated,
// copied or waited for after fk_paged_create, so that a step's appends and attentions can be captured in a graph.
#include "fk_paged.h"

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

using namespace fk;

namespace {

struct Seq {
  int len = 0;                        // tokens held before the current step
  int buf = 0;                        // tail slot of the open page
  std::vector<int> pages;
};

struct StepSeq {
  int seq, n_new, n_query, old_pages;
};

// the caller's current device comes back when a call ends
struct DeviceGuard {
  int before = -1;
  cudaError_t err;
  explicit DeviceGuard(int dev) {
    err = cudaGetDevice(&before);
    if (err == cudaSuccess && before != dev) err = cudaSetDevice(dev);
    else if (err == cudaSuccess) before = -1;
  }
  ~DeviceGuard() {
    if (before >= 0) cudaSetDevice(before);
  }
};

}  // namespace

struct fk_paged {
  fk_paged_config cfg{};
  int max_pages = 0;                  // table entries of a sequence
  std::vector<Seq> seqs;
  std::vector<int> free_pages;        // the next one to be taken last
  std::vector<StepSeq> step;
  bool in_step = false;
  int64_t step_new = 0;               // tokens of the step, all sequences
  std::vector<uint8_t> appended;      // per layer: this step's append was made
  std::vector<PagedPool> pools;
  std::vector<CUtensorMap> tmK, tmV;
  int* table = nullptr;
  float* part_few = nullptr;          // key splits' partial results
  float* part_chunk = nullptr;
  int part_tiles = 0;                 // query tiles that part_chunk holds
  int* arrived = nullptr;
  int* status = nullptr;
  int sms = 0;
  std::vector<void*> allocs;
  size_t reserved = 0;
  int64_t launches = 0;
  ~fk_paged() {
    for (void* p : allocs) cudaFree(p);
    cudaGetLastError();
  }
};

namespace {

// No C++ exception leaves a C entry: the only ones here are failed host allocations.
template <class F>
fk_status guarded(F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return FK_ERR_NOMEM;
  } catch (...) {
    return FK_ERR_STATE;
  }
}

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bool on_device(const void* p, int dev) {
  cudaPointerAttributes at{};
  if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  return at.type == cudaMemoryTypeManaged || (at.type == cudaMemoryTypeDevice && at.device == dev);
}

// a [tokens][heads][D] bf16 tensor whose tokens lie `stride` elements apart
bool rows_ok(const fk_paged* h, const void* p, int64_t stride, int heads) {
  return p && aligned(p, 16) && stride >= (int64_t)heads * h->cfg.head_dim && stride % 8 == 0 && on_device(p, h->cfg.device);
}

fk_status done(fk_paged* h, cudaError_t e) {
  h->launches++;
  return e == cudaSuccess ? FK_OK : FK_ERR_CUDA;
}

fk_status alloc(fk_paged* h, size_t bytes, void** out) {
  void* p = nullptr;
  cudaError_t e = cudaMalloc(&p, bytes);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return e == cudaErrorMemoryAllocation ? FK_ERR_NOMEM : FK_ERR_CUDA;
  }
  h->allocs.push_back(p);
  h->reserved += bytes;
  *out = p;
  return cudaMemset(p, 0, bytes) == cudaSuccess ? FK_OK : FK_ERR_CUDA;
}

int pages_of(const fk_paged* h, int tokens) {
  return (tokens + h->cfg.page_tokens - 1) / h->cfg.page_tokens;
}

// The current step ends: its tokens join their sequences.  A step that no layer was appended to is withdrawn (its
// pages go back); one that some layers were not appended to cannot end.
enum class StepEnd { kJoin, kWithdraw, kRefused };
StepEnd step_end(const fk_paged* h) {
  const int64_t n = std::count(h->appended.begin(), h->appended.end(), (uint8_t)1);
  if (n == (int64_t)h->appended.size() || h->step_new == 0) return StepEnd::kJoin;
  return n == 0 ? StepEnd::kWithdraw : StepEnd::kRefused;
}

fk_status end_step(fk_paged* h) {
  if (!h->in_step) return FK_OK;
  const StepEnd how = step_end(h);
  if (how == StepEnd::kRefused) return FK_ERR_STATE;
  const bool all = how == StepEnd::kJoin;
  for (auto it = h->step.rbegin(); it != h->step.rend(); ++it) {
    Seq& q = h->seqs[it->seq];
    if (all) {
      const int len = q.len + it->n_new, P = h->cfg.page_tokens;
      if (it->n_new > 0 && (len - 1) / P != q.len / P) q.buf ^= 1;
      q.len = len;
    } else {
      for (; (int)q.pages.size() > it->old_pages; q.pages.pop_back()) h->free_pages.push_back(q.pages.back());
    }
  }
  h->in_step = false;
  h->step.clear();
  h->step_new = 0;
  return FK_OK;
}

// Sequences [i0, i1) of the step as an append or read-back launch takes them; the tokens' places start at *tok.
void fill_seqs(const fk_paged* h, size_t i0, size_t i1, bool whole, bool read, int64_t* tok, PagedSeqs* out) {
  const int P = h->cfg.page_tokens;
  out->n = 0;
  int page0 = 0;
  for (size_t i = i0; i < i1; ++i) {
    const StepSeq& st = h->step[i];
    const Seq& q = h->seqs[st.seq];
    const int len = q.len + st.n_new;
    const int first = whole ? 0 : q.len / P;               // first page
    const int tokens = read ? len - first * P : st.n_new;
    const int n_pages = (read ? tokens > 0 : st.n_new > 0) ? pages_of(h, len) - first : 0;
    if (n_pages > 0) {
      const int k = out->n++;
      out->slot[k] = st.seq;
      out->old_len[k] = q.len;
      out->new_len[k] = len;
      out->tok0[k] = (int)*tok;
      out->page0[k] = page0;
      const int buf = (len - 1) / P != q.len / P ? q.buf ^ 1 : q.buf;
      out->buf[k] = (uint8_t)(q.buf | (buf << 1));
      page0 += n_pages;
    }
    *tok += tokens;
  }
  out->page0[out->n] = page0;
}

// Sequences in the order of `key`, the largest first (their items then start first).
void sort_seqs(PagedAttnSeqs& s, const int* key) {
  int order[kStepSeqs], old[kStepSeqs];
  for (int k = 0; k < s.n; ++k) order[k] = k;
  std::stable_sort(order, order + s.n, [&](int x, int y) { return key[x] > key[y]; });
  for (int* v : {s.slot, s.n_keys, s.q0, s.n_q}) {
    std::copy(v, v + s.n, old);
    for (int k = 0; k < s.n; ++k) v[k] = old[order[k]];
  }
}

// Work items of the few-row kernel: 8 or 16 rows to a CTA (returned, in eights), and key splits where they do not fill
// the device.
int plan_few(const fk_paged* h, PagedAttnArgs* a) {
  PagedAttnSeqs& s = a->seqs;
  int tiles[kStepSeqs], row_tiles[kStepSeqs], eights = 1;
  for (int k = 0; k < s.n; ++k)
    if (s.n_q[k] * a->G > 8) eights = 2;
  auto count = [&](int k) { return paged_tiles(s.n_keys[k], s.n_keys[k] - s.n_q[k], s.n_keys[k] - 1, a->mask, kPagedFewTile).count(); };
  for (int k = 0; k < s.n; ++k) tiles[k] = count(k);
  sort_seqs(s, tiles);
  int64_t work = 0;                   // key tiles of all CTAs, unsplit
  for (int k = 0; k < s.n; ++k) {
    row_tiles[k] = (s.n_q[k] * a->G + 8 * eights - 1) / (8 * eights);
    tiles[k] = count(k);
    work += (int64_t)tiles[k] * row_tiles[k] * a->Hkv;
  }
  // Three CTAs fit an SM (two of 16 rows); a split takes at least 4 tiles.  Where whole sequences already make many
  // CTAs, of lengths of their own, pieces of half a CTA's share even out the end (64 ragged streams: 92 us with
  // pieces of a share, 84 half, 86 a third, 87 a quarter); where the keys of a few are split, each further split costs
  // the one that joins them (one stream of 131072 keys: 51 us, halves 62).
  int64_t base = 0;
  for (int k = 0; k < s.n; ++k) base += (int64_t)row_tiles[k] * a->Hkv;
  const int64_t slots = (eights == 1 ? 3 : 2) * h->sms, pieces = 2 * base > slots ? 2 * slots : slots;
  const int64_t per = std::max<int64_t>(4, (work + pieces - 1) / pieces);
  int item = 0, part = 0;
  for (int k = 0; k < s.n; ++k) {
    int splits = (int)std::min<int64_t>(kMaxFewSplits, std::max<int64_t>(1, (tiles[k] + per - 1) / per));
    if (splits > 1 && part + (int64_t)splits * row_tiles[k] * a->Hkv > kPartSlots) splits = 1;
    s.item0[k] = item;
    s.part0[k] = part;
    s.splits[k] = splits;
    s.whole[k] = 0;
    item += row_tiles[k] * splits;
    if (splits > 1) part += splits * row_tiles[k] * a->Hkv;
  }
  s.item0[s.n] = item;
  return eights;
}

// Work items of the chunk kernel; true: one query tile per CTA.
bool plan_chunk(const fk_paged* h, PagedAttnArgs* a) {
  PagedAttnSeqs& s = a->seqs;
  int64_t pairs = 0;
  for (int k = 0; k < s.n; ++k) pairs += ((int64_t)s.n_q[k] * a->G + 2 * kAttnBM - 1) / (2 * kAttnBM) * a->Hkv;
  const bool one = pairs < h->sms;
  const int rows = (one ? 1 : 2) * kAttnBM;
  int tiles[kStepSeqs], items[kStepSeqs];
  int64_t work = 0, total = 0;
  for (int k = 0; k < s.n; ++k) {
    items[k] = (int)(((int64_t)s.n_q[k] * a->G + rows - 1) / rows * a->Hkv);
    tiles[k] = paged_tiles(s.n_keys[k], s.n_keys[k] - s.n_q[k], s.n_keys[k] - 1, a->mask, kAttnBN).count();
    work += (int64_t)tiles[k] * items[k];
    total += items[k];
  }
  // Key splits, one CTA to an SM: of everything where the items do not fill the device; else, with one sequence
  // whose items take about as long, of those left over after the last whole wave.
  int64_t per = INT32_MAX;
  if (total < h->sms) {
    per = std::max<int64_t>(2, (work + h->sms - 1) / h->sms);
  } else if (s.n == 1 && !a->mask.causal && total % h->sms && total < 8 * h->sms) {
    const int rest = (int)(total % h->sms), splits = std::min<int>(tiles[0] / 2, std::max(1, h->sms / rest));
    if (splits > 1 && (int64_t)splits * rest * (rows / kAttnBM) <= h->part_tiles) {
      s.item0[0] = s.part0[0] = 0;
      s.splits[0] = splits;
      s.whole[0] = items[0] - rest;
      s.item0[1] = s.whole[0] + rest * splits;
      return one;
    }
  }
  int item = 0, part = 0;
  for (int k = 0; k < s.n; ++k) {
    int splits = (int)std::max<int64_t>(1, (tiles[k] + per - 1) / per);
    const int64_t slots = (int64_t)splits * items[k] * (rows / kAttnBM);
    if (splits > 1 && part + slots > h->part_tiles) splits = 1;
    s.item0[k] = item;
    s.part0[k] = part;
    s.splits[k] = splits;
    s.whole[k] = splits > 1 ? 0 : items[k];
    item += items[k] * splits;
    if (splits > 1) part += (int)slots;
  }
  s.item0[s.n] = item;
  return one;
}

int64_t read_tokens(const fk_paged* h, bool whole) {
  int64_t n = 0;
  const int P = h->cfg.page_tokens;
  for (const StepSeq& st : h->step) {
    const int old_len = h->seqs[st.seq].len;
    n += old_len + st.n_new - (whole ? 0 : old_len / P * P);
  }
  return n;
}

}  // namespace

extern "C" {

fk_status fk_paged_validate_config(const fk_paged_config* c) {
  if (!c) return FK_ERR_ARG;
  if (c->n_layers < 1 || c->n_layers > kMaxLayers) return FK_ERR_CONFIG;
  if (c->n_kv_heads < 1 || c->n_kv_heads > kMaxHeads || c->n_q_heads < c->n_kv_heads || c->n_q_heads > 1024 ||
      c->n_q_heads % c->n_kv_heads)
    return FK_ERR_CONFIG;
  if (c->head_dim != 64 && c->head_dim != 128) return FK_ERR_CONFIG;
  if (c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return FK_ERR_CONFIG;
  if (c->n_pages < 1 || c->max_seqs < 1 || c->max_seqs > 65536) return FK_ERR_CONFIG;
  if (c->max_seq_tokens < 1 || c->max_seq_tokens > (1 << 30)) return FK_ERR_CONFIG;
  if (c->rope_style != FK_ROPE_HALF && c->rope_style != FK_ROPE_INTERLEAVED) return FK_ERR_CONFIG;
  // rows of a layer's pages are TMA coordinates, entries of the page table 32-bit places
  if ((int64_t)c->n_pages * c->n_kv_heads * c->page_tokens >= ((int64_t)1 << 31)) return FK_ERR_CONFIG;
  const int64_t per_seq = ((int64_t)c->max_seq_tokens + c->page_tokens - 1) / c->page_tokens;
  if (per_seq * c->max_seqs >= ((int64_t)1 << 30)) return FK_ERR_CONFIG;
  return FK_OK;
}

fk_status fk_paged_create(const fk_paged_config* cfg, fk_paged** out) {
  if (!out) return FK_ERR_ARG;
  *out = nullptr;
  fk_status st = fk_paged_validate_config(cfg);
  if (st != FK_OK) return st;
  return guarded([&]() -> fk_status {
    int n_dev = 0;
    if (cudaGetDeviceCount(&n_dev) != cudaSuccess || cfg->device < 0 || cfg->device >= n_dev) {
      cudaGetLastError();
      return FK_ERR_CUDA;
    }
    DeviceGuard dev(cfg->device);
    if (dev.err != cudaSuccess) return FK_ERR_CUDA;
    std::unique_ptr<fk_paged> h(new fk_paged());
    h->cfg = *cfg;
    const size_t P = cfg->page_tokens, D = cfg->head_dim, H = cfg->n_kv_heads, N = cfg->n_pages, S = cfg->max_seqs;
    h->max_pages = (int)((cfg->max_seq_tokens + P - 1) / P);
    h->seqs.resize(S);
    h->free_pages.resize(N);
    for (size_t i = 0; i < N; ++i) h->free_pages[i] = (int)(N - 1 - i);
    h->appended.assign(cfg->n_layers, 0);
    h->pools.resize(cfg->n_layers);
    h->tmK.resize(cfg->n_layers);
    h->tmV.resize(cfg->n_layers);
    if (cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, cfg->device) != cudaSuccess) return FK_ERR_CUDA;
    fk_status e = FK_OK;
    auto get = [&](size_t bytes, auto** p) {
      void* q = nullptr;
      if (e == FK_OK) e = alloc(h.get(), bytes, &q);
      *p = static_cast<std::remove_reference_t<decltype(**p)>*>(q);
    };
    // The pages start as zeros: what a tile reads beyond a sequence's end is finite whatever was there before.
    for (int l = 0; l < cfg->n_layers && e == FK_OK; ++l) {
      PagedPool& p = h->pools[l];
      get(N * H * P * D, &p.k);
      get(N * H * P * D, &p.v);
      get(N * H, &p.ke);
      get(N * H, &p.ve);
      get(S * 2 * H * P * D * sizeof(float), &p.tail_k);
      get(S * 2 * H * P * D * sizeof(bf16), &p.tail_v);
      get(S * 2 * H * P * sizeof(float), &p.tail_kmax);
      get(S * 2 * H * P * sizeof(float), &p.tail_vmax);
      const int box = (int)std::min<size_t>(P, kPagedFewTile);
      if (e == FK_OK && (!encode_byte_rows(&h->tmK[l], p.k, (int64_t)(N * H * P), (int)D, box) ||
                         !encode_byte_rows(&h->tmV[l], p.v, (int64_t)(N * H * P), (int)D, box)))
        e = FK_ERR_CUDA;
    }
    get(S * h->max_pages * sizeof(int), &h->table);
    get((size_t)kPartSlots * kPagedFewRows * (D + 4) * sizeof(float), &h->part_few);
    h->part_tiles = std::min(4 * h->sms, kPartSlots);
    get((size_t)h->part_tiles * kAttnBM * (D + 4) * sizeof(float), &h->part_chunk);
    get(kPartSlots * sizeof(int), &h->arrived);
    get(sizeof(int), &h->status);
    if (e != FK_OK) return e;
    if (paged_few_prepare((int)D) != cudaSuccess || paged_chunk_prepare((int)D) != cudaSuccess) return FK_ERR_CUDA;
    if (cudaDeviceSynchronize() != cudaSuccess) return FK_ERR_CUDA;
    *out = h.release();
    return FK_OK;
  });
}

void fk_paged_destroy(fk_paged* h) {
  if (!h) return;
  DeviceGuard dev(h->cfg.device);
  cudaDeviceSynchronize();
  delete h;
}

fk_status fk_paged_step(fk_paged* h, int n_seqs, const int32_t* seqs, const int32_t* n_new, const int32_t* n_query,
                        void* stream) {
  if (!h || n_seqs < 0 || (n_seqs > 0 && (!seqs || !n_new))) return FK_ERR_ARG;
  if (n_seqs > h->cfg.max_seqs) return FK_ERR_ARG;
  return guarded([&]() -> fk_status {
    std::vector<uint8_t> seen(h->cfg.max_seqs, 0);
    int64_t total = 0, queries = 0;
    for (int i = 0; i < n_seqs; ++i) {
      if (seqs[i] < 0 || seqs[i] >= h->cfg.max_seqs || seen[seqs[i]] || n_new[i] < 0 || (n_query && n_query[i] < 0))
        return FK_ERR_ARG;
      seen[seqs[i]] = 1;
      total += n_new[i];
      queries += n_query ? n_query[i] : n_new[i];
    }
    if (total >= ((int64_t)1 << 31) || queries * h->cfg.n_q_heads >= ((int64_t)1 << 31)) return FK_ERR_ARG;
    DeviceGuard dev(h->cfg.device);
    if (dev.err != cudaSuccess) return FK_ERR_CUDA;
    // lengths and pages as they are once the current step has ended: a refusal leaves it as it is
    const StepEnd how = h->in_step ? step_end(h) : StepEnd::kJoin;
    if (how == StepEnd::kRefused) return FK_ERR_STATE;
    std::vector<int> ended(h->cfg.max_seqs, 0);     // tokens that the current step adds
    int64_t pages = 0, free_pages = (int64_t)h->free_pages.size();
    for (const StepSeq& s : h->step) {
      if (how == StepEnd::kJoin) ended[s.seq] = s.n_new;
      else free_pages += (int64_t)h->seqs[s.seq].pages.size() - s.old_pages;
    }
    for (int i = 0; i < n_seqs; ++i) {
      const int64_t len = (int64_t)h->seqs[seqs[i]].len + ended[seqs[i]];
      if (len + n_new[i] > h->cfg.max_seq_tokens) return FK_ERR_FULL;
      pages += pages_of(h, (int)len + n_new[i]) - pages_of(h, (int)len);
    }
    if (pages > free_pages) return FK_ERR_FULL;
    fk_status st = end_step(h);
    if (st != FK_OK) return st;
    // the table first: if its launch fails, no page has been taken
    std::vector<StepSeq> step(n_seqs);
    auto a = std::make_unique<TableArgs>();
    a->table = h->table;
    a->n = 0;
    size_t next = h->free_pages.size();
    for (int i = 0; i < n_seqs; ++i) {
      Seq& q = h->seqs[seqs[i]];
      const int old_pages = (int)q.pages.size(), need = pages_of(h, q.len + n_new[i]);
      step[i] = {seqs[i], n_new[i], n_query ? n_query[i] : n_new[i], old_pages};
      q.pages.reserve(need);
      for (int p = old_pages; p < need; ++p) {
        a->index[a->n] = seqs[i] * h->max_pages + p;
        a->page[a->n] = h->free_pages[--next];
        if (++a->n == kTableEntries) {
          if ((st = done(h, launch_paged_table(*a, static_cast<cudaStream_t>(stream)))) != FK_OK) return st;
          a->n = 0;
        }
      }
    }
    if (a->n > 0 && (st = done(h, launch_paged_table(*a, static_cast<cudaStream_t>(stream)))) != FK_OK) return st;
    for (int i = 0; i < n_seqs; ++i) {
      Seq& q = h->seqs[seqs[i]];
      for (const int need = pages_of(h, q.len + n_new[i]); (int)q.pages.size() < need; h->free_pages.pop_back())
        q.pages.push_back(h->free_pages.back());
    }
    h->step.swap(step);
    h->step_new = total;
    std::fill(h->appended.begin(), h->appended.end(), (uint8_t)0);
    h->in_step = true;
    return FK_OK;
  });
}

fk_status fk_paged_append(fk_paged* h, int layer, const void* K, int64_t k_stride, const void* V, int64_t v_stride,
                          const fk_rope* rope, const void* Q, int64_t q_stride, void* Q_out, int64_t q_out_stride,
                          void* stream) {
  if (!h || layer < 0 || layer >= h->cfg.n_layers) return FK_ERR_ARG;
  if (!h->in_step) return FK_ERR_STATE;
  const fk_paged_config& c = h->cfg;
  if ((Q == nullptr) != (Q_out == nullptr) || (Q && !rope)) return FK_ERR_ARG;
  if (rope) {
    if (rope->dim < 16 || rope->dim > c.head_dim || rope->dim % 16 || rope->rows < 1) return FK_ERR_CONFIG;
    if (!rope->cos || !rope->sin || !aligned(rope->cos, 16) || !aligned(rope->sin, 16)) return FK_ERR_ARG;
    if (rope->positions && !aligned(rope->positions, 4)) return FK_ERR_ARG;
  }
  if (h->step_new == 0) return FK_OK;
  return guarded([&]() -> fk_status {
    DeviceGuard dev(c.device);
    if (dev.err != cudaSuccess) return FK_ERR_CUDA;
    if (!rows_ok(h, K, k_stride, c.n_kv_heads) || !rows_ok(h, V, v_stride, c.n_kv_heads)) return FK_ERR_ARG;
    if (Q && (!rows_ok(h, Q, q_stride, c.n_q_heads) || !rows_ok(h, Q_out, q_out_stride, c.n_q_heads))) return FK_ERR_ARG;
    if (rope) {
      if (!on_device(rope->cos, c.device) || !on_device(rope->sin, c.device) ||
          (rope->positions && !on_device(rope->positions, c.device)))
        return FK_ERR_ARG;
      if (!rope->positions)           // the tokens' own places: known here
        for (const StepSeq& s : h->step)
          if (s.n_new > 0 && h->seqs[s.seq].len + s.n_new > rope->rows) return FK_ERR_ARG;
    }
    auto a = std::make_unique<AppendArgs>();
    a->pool = h->pools[layer];
    a->table = h->table;
    a->max_pages = h->max_pages;
    a->Hkv = c.n_kv_heads;
    a->G = c.n_q_heads / c.n_kv_heads;
    a->P = c.page_tokens;
    a->by_g = FastDiv((uint32_t)a->G);
    a->K = static_cast<const bf16*>(K);
    a->V = static_cast<const bf16*>(V);
    a->Q = static_cast<const bf16*>(Q);
    a->Qr = static_cast<bf16*>(Q_out);
    a->kstride = k_stride;
    a->vstride = v_stride;
    a->qstride = q_stride;
    a->qrstride = q_out_stride;
    if (rope) {
      a->cos = rope->cos;
      a->sin = rope->sin;
      a->positions = rope->positions;
      a->rope_rows = rope->rows;
      a->R = rope->dim;
      a->interleaved = c.rope_style == FK_ROPE_INTERLEAVED;
    }
    a->status = h->status;
    int64_t tok = 0;
    for (size_t i = 0; i < h->step.size(); i += kStepSeqs) {
      fill_seqs(h, i, std::min(h->step.size(), i + kStepSeqs), false, false, &tok, &a->seqs);
      if (a->seqs.n == 0) continue;
      a->most = 0;
      for (int k = 0; k < a->seqs.n; ++k) a->most = std::max(a->most, a->seqs.new_len[k] - a->seqs.old_len[k]);
      const fk_status st = done(h, launch_paged_append(c.head_dim, *a, static_cast<cudaStream_t>(stream)));
      if (st != FK_OK) return st;
    }
    h->appended[layer] = 1;
    return FK_OK;
  });
}

fk_status fk_paged_attend(fk_paged* h, int layer, const void* Q, int64_t q_stride, void* O, int64_t o_stride,
                          int causal, int window, int sinks, float scale, void* stream) {
  if (!h || layer < 0 || layer >= h->cfg.n_layers) return FK_ERR_ARG;
  if ((causal != 0 && causal != 1) || window < 0 || sinks < 0 || !(scale >= 0.0f) || std::isinf(scale)) return FK_ERR_CONFIG;
  if (!h->in_step || (h->step_new > 0 && !h->appended[layer])) return FK_ERR_STATE;
  const fk_paged_config& c = h->cfg;
  int64_t queries = 0;
  for (const StepSeq& s : h->step) queries += s.n_query;
  if (queries == 0) return FK_OK;
  return guarded([&]() -> fk_status {
    DeviceGuard dev(c.device);
    if (dev.err != cudaSuccess) return FK_ERR_CUDA;
    if (!rows_ok(h, Q, q_stride, c.n_q_heads) || !rows_ok(h, O, o_stride, c.n_q_heads)) return FK_ERR_ARG;
    auto a = std::make_unique<PagedAttnArgs>();
    a->table = h->table;
    a->ke = h->pools[layer].ke;
    a->ve = h->pools[layer].ve;
    a->max_pages = h->max_pages;
    a->Hkv = c.n_kv_heads;
    a->G = c.n_q_heads / c.n_kv_heads;
    a->P = c.page_tokens;
    a->by_g = FastDiv((uint32_t)a->G);
    a->Q = static_cast<const bf16*>(Q);
    a->O = static_cast<bf16*>(O);
    a->qstride = q_stride;
    a->ostride = o_stride;
    a->scale_log2 = (float)(1.4426950408889634 * (scale > 0.0f ? (double)scale : 1.0 / std::sqrt((double)c.head_dim)));
    a->mask = {causal, window, window > 0 ? sinks : 0};
    a->part_tiles = h->part_tiles;
    a->arrived = h->arrived;
    a->status = h->status;
    int64_t q0 = 0;
    for (size_t i = 0; i < h->step.size(); i += kStepSeqs) {
      const size_t i1 = std::min(h->step.size(), i + kStepSeqs);
      for (const bool chunk : {false, true}) {
        int64_t q = q0;
        a->seqs.n = 0;
        for (size_t j = i; j < i1; ++j) {
          const StepSeq& st = h->step[j];
          if (st.n_query > 0 && ((int64_t)st.n_query * a->G > kPagedFewRows) == chunk) {
            const int k = a->seqs.n++;
            a->seqs.slot[k] = st.seq;
            a->seqs.n_keys[k] = h->seqs[st.seq].len + st.n_new;
            a->seqs.q0[k] = (int)q;
            a->seqs.n_q[k] = st.n_query;
          }
          q += st.n_query;
        }
        if (chunk) q0 = q;
        if (a->seqs.n == 0) continue;
        const int shape = chunk ? (plan_chunk(h, a.get()) ? 1 : 2) : plan_few(h, a.get());
        a->part = chunk ? h->part_chunk : h->part_few;
        const cudaStream_t s = static_cast<cudaStream_t>(stream);
        const fk_status st = done(h, chunk ? launch_paged_chunk(c.head_dim, shape == 1, h->tmK[layer], h->tmV[layer], *a, s)
                                           : launch_paged_few(c.head_dim, shape, h->tmK[layer], h->tmV[layer], *a, s));
        if (st != FK_OK) return st;
      }
    }
    return FK_OK;
  });
}

fk_status fk_paged_read(fk_paged* h, int layer, int whole, void* K, void* V, int64_t capacity, int64_t* n_tokens,
                        void* stream) {
  if (!h || layer < 0 || layer >= h->cfg.n_layers || !n_tokens || (whole != 0 && whole != 1)) return FK_ERR_ARG;
  if (!h->in_step || (h->step_new > 0 && !h->appended[layer])) return FK_ERR_STATE;
  const fk_paged_config& c = h->cfg;
  *n_tokens = read_tokens(h, whole != 0);
  if (*n_tokens >= ((int64_t)1 << 31)) return FK_ERR_CONFIG;
  if (*n_tokens > capacity) return FK_ERR_ARG;
  if (*n_tokens == 0) return FK_OK;
  return guarded([&]() -> fk_status {
    DeviceGuard dev(c.device);
    if (dev.err != cudaSuccess) return FK_ERR_CUDA;
    const int64_t row = (int64_t)c.n_kv_heads * c.head_dim;
    if (!rows_ok(h, K, row, c.n_kv_heads) || !rows_ok(h, V, row, c.n_kv_heads)) return FK_ERR_ARG;
    auto a = std::make_unique<ReadArgs>();
    a->pool = h->pools[layer];
    a->table = h->table;
    a->max_pages = h->max_pages;
    a->Hkv = c.n_kv_heads;
    a->P = c.page_tokens;
    a->whole = whole;
    a->K = static_cast<bf16*>(K);
    a->V = static_cast<bf16*>(V);
    int64_t tok = 0;
    for (size_t i = 0; i < h->step.size(); i += kStepSeqs) {
      fill_seqs(h, i, std::min(h->step.size(), i + kStepSeqs), whole != 0, true, &tok, &a->seqs);
      if (a->seqs.n == 0) continue;
      const fk_status st = done(h, launch_paged_read(c.head_dim, *a, static_cast<cudaStream_t>(stream)));
      if (st != FK_OK) return st;
    }
    return FK_OK;
  });
}

fk_status fk_paged_drop(fk_paged* h, int seq) {
  if (!h || seq < 0 || seq >= h->cfg.max_seqs) return FK_ERR_ARG;
  return guarded([&]() -> fk_status {
    const fk_status st = end_step(h);
    if (st != FK_OK) return st;
    Seq& q = h->seqs[seq];
    for (; !q.pages.empty(); q.pages.pop_back()) h->free_pages.push_back(q.pages.back());
    q.len = 0;
    return FK_OK;
  });
}

int64_t fk_paged_length(const fk_paged* h, int seq) {
  if (!h || seq < 0 || seq >= h->cfg.max_seqs) return -1;
  int64_t n = h->seqs[seq].len;
  for (const StepSeq& s : h->step)
    if (s.seq == seq) n += s.n_new;
  return n;
}

int64_t fk_paged_free_pages(const fk_paged* h) { return h ? (int64_t)h->free_pages.size() : -1; }

size_t fk_paged_reserved_bytes(const fk_paged* h) { return h ? h->reserved : 0; }

int64_t fk_paged_launch_count(const fk_paged* h) { return h ? h->launches : 0; }

fk_status fk_paged_sync_status(fk_paged* h, void* stream) {
  if (!h) return FK_ERR_ARG;
  DeviceGuard dev(h->cfg.device);
  if (dev.err != cudaSuccess) return FK_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int word = 0;
  if (cudaMemcpyAsync(&word, h->status, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess)
    return FK_ERR_CUDA;
  if (word && cudaMemset(h->status, 0, sizeof(int)) != cudaSuccess) return FK_ERR_CUDA;
  if (word & kStatusTimeout) return FK_ERR_TIMEOUT;
  if (word & (kStatusNonFinite | kStatusPosition)) return FK_ERR_RANGE;
  return FK_OK;
}

}  // extern "C"
