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

// One launch of an attention: rows of a CTA in eights (few) or tiles of 128 (chunk).
struct AttnLaunch {
  bool chunk;
  int shape;
  bool join;                          // a second kernel joins the splits
  PagedAttnSeqs seqs;
};
struct AttnPlan {
  PagedMask mask;
  std::vector<AttnLaunch> launches;
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
  std::vector<AttnPlan> plans;        // of the step
  std::vector<uint8_t> appended;      // per layer: this step's append was made
  std::vector<PagedPool> pools;
  std::vector<CUtensorMap> tmK, tmV;
  int* table = nullptr;
  float* part_few = nullptr;          // key splits' partial results
  float* part_chunk = nullptr;
  int part_tiles = 0;                 // query tiles that part_chunk holds
  int* arrived = nullptr;
  int* status = nullptr;              // the status word, and a report of it
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
  h->plans.clear();
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

// ---- plans of an attention
// Estimated times, in us, of what a CTA takes for a key tile (D = 128) with the device full of such CTAs, and of its start and end;
// `slots` such CTAs fit an SM.  Measured back to back with 16 to 256 rows, 1000 to 16000 keys, 1 to 64 sequences and 2 to 8 kv heads;
// the plans barely depend on them (`fixed` of the chunks a sixth or a third lower: one of 36 drawn steps changed by more than 5%,
// for the worse).
struct Shape {
  int rows, tile, slots;
  double per_tile, fixed;
};
constexpr Shape kFew8{8, kPagedFewTile, 3, 1.2, 4.0}, kFew16{16, kPagedFewTile, 2, 1.0, 5.0};
constexpr Shape kChunk1{kAttnBM, kAttnBN, 1, 1.1, 9.0}, kChunk2{2 * kAttnBM, kAttnBN, 1, 1.55, 10.0};

struct Candidate {
  double us = 1e30;
  int per = INT32_MAX;                // key tiles of a split, at most
};

// Sequences of one launch: key tiles and items (row tiles times kv heads) under a shape.
struct Load {
  int n = 0;
  int tiles[kStepSeqs];
  int64_t items[kStepSeqs];
};
Load load_of(const PagedAttnArgs& a, const PagedAttnSeqs& s, const Shape& sh) {
  Load w;
  w.n = s.n;
  for (int k = 0; k < s.n; ++k) {
    w.tiles[k] = paged_tiles(s.n_keys[k], s.n_keys[k] - s.n_q[k], s.n_keys[k] - 1, a.mask, sh.tile).count();
    w.items[k] = ((int64_t)s.n_q[k] * a.G + sh.rows - 1) / sh.rows * a.Hkv;
  }
  return w;
}
int splits_of(int tiles, int per) { return per >= tiles ? 1 : (int)(((int64_t)tiles + per - 1) / per); }

// How the keys are best split: the time of the device's slots filled with the pieces, longest first, and what a join adds.
Candidate best_split(const fk_paged* h, const Load& w, const Shape& sh, int min_tiles, int max_splits, int64_t max_slots, double join) {
  const double per_tile = sh.per_tile * (sh.slots == 1 ? (h->cfg.head_dim == 128 ? 1.0 : 0.75) : h->cfg.head_dim == 128 ? 1.0 : 0.7);
  const int slots = sh.slots * h->sms;
  int most = 0;
  for (int k = 0; k < w.n; ++k) most = std::max(most, w.tiles[k]);
  Candidate best;
  std::pair<float, int64_t> piece[kStepSeqs];
  std::vector<float> room(2 * (size_t)slots);
  float *busy = room.data(), *other = busy + slots;
  for (int s = 1; s <= max_splits; s += std::max(1, s / 6)) {
    const int per = std::max(min_tiles, (most + s - 1) / s);
    double total = 0, longest = 0, shortest = 1e30;
    int64_t ctas = 0, split = 0;
    for (int k = 0; k < w.n; ++k) {
      const int n = splits_of(w.tiles[k], per);
      piece[k] = {(float)((w.tiles[k] + n - 1) / n * per_tile + sh.fixed), w.items[k] * n};
      total += (double)piece[k].first * (double)piece[k].second;
      longest = std::max(longest, (double)piece[k].first);
      shortest = std::min(shortest, (double)piece[k].first);
      ctas += piece[k].second;
      if (n > 1) split += piece[k].second;
    }
    if (split > max_slots || (s > 1 && ctas > 6 * slots)) break;
    // Pieces of one length come in whole waves; of several, the longest first, each goes to the slot that is free first.
    double us;
    if (longest <= 1.2 * shortest) {
      us = (double)((ctas + slots - 1) / slots) * longest;
    } else if (ctas > 6 * slots) {
      us = std::max(longest, total / slots + 0.5 * shortest);
    } else {
      std::sort(piece, piece + w.n, [](const auto& x, const auto& y) { return x.first > y.first; });
      const int q = std::min(8, h->cfg.n_kv_heads & -h->cfg.n_kv_heads), m = slots / q;   // pieces come q at a time
      std::fill(busy, busy + m, 0.0f);                     // ascending
      for (int k = 0; k < w.n; ++k)
        for (int64_t left = piece[k].second / q; left > 0;) {
          const int n = (int)std::min<int64_t>(left, m);
          for (int i = 0; i < n; ++i) busy[i] += piece[k].first;
          std::merge(busy, busy + n, busy + n, busy + m, other);
          std::swap(busy, other);
          left -= n;
        }
      us = busy[m - 1];
    }
    if (split > 0) us += join + 0.02 * splits_of(most, per);
    if (us < best.us - 0.2) best = {us, per};
    if (per <= min_tiles) break;
  }
  return best;
}

// Sequences in the order of their pieces' lengths, the longest first (their items then start first).
void sort_seqs(PagedAttnSeqs& s, const Load& w, int per) {
  int order[kStepSeqs], old[kStepSeqs];
  auto len = [&](int k) { return (w.tiles[k] + splits_of(w.tiles[k], per) - 1) / splits_of(w.tiles[k], per); };
  for (int k = 0; k < s.n; ++k) order[k] = k;
  std::stable_sort(order, order + s.n, [&](int x, int y) { return len(x) > len(y); });
  for (int* v : {s.slot, s.n_keys, s.q0, s.n_q}) {
    std::copy(v, v + s.n, old);
    for (int k = 0; k < s.n; ++k) v[k] = old[order[k]];
  }
}

// The launch of a plan: work items, workspace places and joins.
void lay_out(const PagedAttnArgs& a, PagedAttnSeqs& s, const Shape& sh, int per) {
  sort_seqs(s, load_of(a, s, sh), per);
  const Load w = load_of(a, s, sh);
  const bool few = sh.tile == kPagedFewTile;
  const int tiles = std::max(1, sh.rows / kAttnBM);        // workspace places of a CTA
  int item = 0, part = 0, pair = 0;
  for (int k = 0; k < s.n; ++k) {
    const int n = splits_of(w.tiles[k], per);
    s.item0[k] = item;
    s.part0[k] = part;
    s.splits[k] = n;
    s.join0[k] = pair;
    s.whole[k] = n > 1 ? 0 : (int)w.items[k];
    item += (int)(few ? w.items[k] / a.Hkv : w.items[k]) * n;
    if (n > 1) {
      part += (int)w.items[k] * n * tiles;
      if (!few) pair += (int)w.items[k];
    }
  }
  s.item0[s.n] = item;
  s.join0[s.n] = pair;
}

// One sequence of equally long items that fill the device more than once: only those left over after the last whole wave are split.
bool split_the_rest(const fk_paged* h, const PagedAttnArgs& a, PagedAttnSeqs& s, const Shape& sh) {
  if (s.n != 1 || a.mask.causal) return false;
  const Load w = load_of(a, s, sh);
  const int64_t items = w.items[0], rest = items % h->sms;
  const int tiles = sh.rows / kAttnBM, n = rest ? (int)std::min<int64_t>(w.tiles[0] / 2, h->sms / rest) : 0;
  if (items < h->sms || n < 2 || rest * n * tiles > h->part_tiles) return false;
  s.item0[0] = s.part0[0] = s.join0[0] = 0;
  s.splits[0] = n;
  s.whole[0] = (int)(items - rest);
  s.item0[1] = (int)(items - rest + rest * n);
  s.join0[1] = (int)rest;
  return true;
}

// The launches of an attention over the step's sequences i .. i1 - 1 (at most kStepSeqs): those of few rows and the others.  Up to
// which row count the few-row kernel is the better one depends on how much there is to fill the device with (it takes a
// sequence's keys once for every 16 rows): the estimates decide.
void plan_group(const fk_paged* h, const PagedAttnArgs& a, size_t i, size_t i1, int64_t* q0, std::vector<AttnLaunch>* out) {
  PagedAttnSeqs all;
  all.n = 0;
  int most = 0;
  for (size_t j = i; j < i1; ++j) {
    const StepSeq& st = h->step[j];
    if (st.n_query > 0) {
      const int k = all.n++;
      all.slot[k] = st.seq;
      all.n_keys[k] = h->seqs[st.seq].len + st.n_new;
      all.q0[k] = (int)*q0;
      all.n_q[k] = st.n_query;
      most = std::max(most, st.n_query * a.G);
    }
    *q0 += st.n_query;
  }
  if (all.n == 0) return;
  auto take = [&](int above, int upto, PagedAttnSeqs& s) {     // sequences of above + 1 .. upto rows
    s.n = 0;
    for (int k = 0; k < all.n; ++k) {
      const int rows = all.n_q[k] * a.G;
      if (rows <= above || rows > upto) continue;
      s.slot[s.n] = all.slot[k];
      s.n_keys[s.n] = all.n_keys[k];
      s.q0[s.n] = all.q0[k];
      s.n_q[s.n++] = all.n_q[k];
    }
  };
  auto few_of = [&](const PagedAttnSeqs& s) {
    for (int k = 0; k < s.n; ++k)
      if (s.n_q[k] * a.G > kFew8.rows) return kFew16;
    return kFew8;
  };
  auto few_plan = [&](const PagedAttnSeqs& s) {
    const Shape sh = few_of(s);
    return best_split(h, load_of(a, s, sh), sh, 1, kMaxFewSplits, kPartSlots, 2.0);
  };
  auto chunk_plan = [&](const PagedAttnSeqs& s, Shape* sh) {
    Candidate best;
    for (const Shape& x : {kChunk2, kChunk1}) {
      const Candidate c = best_split(h, load_of(a, s, x), x, 2, 64, h->part_tiles / (x.rows / kAttnBM), 4.0);
      if (c.us < best.us) {
        best = c;
        *sh = x;
      }
    }
    return best;
  };
  PagedAttnSeqs part[2];
  struct {
    int upto = 0;
    Candidate few, chunk;
    Shape shape = kChunk2;
  } best;
  double us = 1e30;
  for (int t : {16, 32, 64, 128}) {                           // the few-row kernel's (16 rows it always takes)
    Shape sh = kChunk2;
    Candidate few, chunk;
    take(0, t, part[0]);
    take(t, INT32_MAX, part[1]);
    if (part[0].n) few = few_plan(part[0]);
    if (part[1].n) chunk = chunk_plan(part[1], &sh);
    const double x = (part[0].n ? few.us : 0.0) + (part[1].n ? chunk.us : 0.0);
    if (x < us) {
      us = x;
      best.upto = t;
      best.few = few;
      best.chunk = chunk;
      best.shape = sh;
    }
    if (t >= most) break;
  }
  take(0, best.upto, part[0]);
  take(best.upto, INT32_MAX, part[1]);
  if (part[0].n) {
    const Shape sh = few_of(part[0]);
    lay_out(a, part[0], sh, best.few.per);
    const bool split = std::any_of(part[0].splits, part[0].splits + part[0].n, [](int n) { return n > 1; });
    out->push_back({false, sh.rows / 8, split && sh.rows == kPagedFewRows, part[0]});
  }
  if (part[1].n) {
    if (!split_the_rest(h, a, part[1], best.shape)) lay_out(a, part[1], best.shape, best.chunk.per);
    out->push_back({true, best.shape.rows / kAttnBM, part[1].join0[part[1].n] > 0, part[1]});
  }
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
    get(2 * sizeof(int), &h->status);
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
    // (rows and positions are 32-bit numbers in the kernels, where a tile and a window go beside them)
    if (total >= ((int64_t)1 << 31) || queries * h->cfg.n_q_heads >= ((int64_t)1 << 30)) return FK_ERR_ARG;
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
    std::unique_ptr<PagedAttnArgs> a(new PagedAttnArgs);
    a->table = h->table;
    a->k = h->pools[layer].k;
    a->v = h->pools[layer].v;
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
    a->wide_o = aligned(O, 32) && o_stride % 16 == 0;
    a->scale_log2 = (float)(1.4426950408889634 * (scale > 0.0f ? (double)scale : 1.0 / std::sqrt((double)c.head_dim)));
    // (no sequence is longer than 2^30, and a position before the first key less a wider window would not fit)
    a->mask = {causal, std::min(window, 1 << 30), window > 0 ? sinks : 0};
    a->part_tiles = h->part_tiles;
    a->arrived = h->arrived;
    a->status = h->status;
    // The launches are planned once for a step and mask: every layer of a model takes the same ones.
    AttnPlan* plan = nullptr;
    for (AttnPlan& p : h->plans)
      if (p.mask.causal == a->mask.causal && p.mask.window == a->mask.window && p.mask.sinks == a->mask.sinks) plan = &p;
    if (!plan) {
      AttnPlan p;
      p.mask = a->mask;
      int64_t q0 = 0;
      for (size_t i = 0; i < h->step.size(); i += kStepSeqs)
        plan_group(h, *a, i, std::min(h->step.size(), i + kStepSeqs), &q0, &p.launches);
      if (h->plans.size() >= 8) h->plans.clear();
      h->plans.push_back(std::move(p));
      plan = &h->plans.back();
    }
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    for (const AttnLaunch& l : plan->launches) {
      a->seqs = l.seqs;
      a->part = l.chunk ? h->part_chunk : h->part_few;
      a->join = !l.chunk && l.join;
      h->launches += l.join;
      const fk_status st = done(h, l.chunk ? launch_paged_chunk(c.head_dim, l.shape == 1, h->tmK[layer], h->tmV[layer], *a, s)
                                           : launch_paged_few(c.head_dim, l.shape, h->tmK[layer], h->tmV[layer], *a, s));
      if (st != FK_OK) return st;
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
  // (cleared by a kernel of the same stream: a memset of the legacy one would come whenever that has time, and take later reports with it)
  if (done(h, launch_paged_status(h->status, h->status + 1, s)) != FK_OK ||
      cudaMemcpyAsync(&word, h->status + 1, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess)
    return FK_ERR_CUDA;
  if (word & kStatusTimeout) return FK_ERR_TIMEOUT;
  if (word & (kStatusNonFinite | kStatusPosition)) return FK_ERR_RANGE;
  return FK_OK;
}

}  // extern "C"
