// Host side of linear attention with decays: states, steps, and the C ABI (fk_linear_*).
//
// The host knows every length, so it hands the kernels their sequences by value (kLinearSeqs to a launch).  Nothing is
// allocated or waited for after fk_linear_create, so that a step's attentions can be captured in a graph; which states
// a launch reads depends on the step alone, so that a graph's replays go on from one another.
#include "fk_linear.h"
#include "fk_rows.h"

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

using namespace fk;

namespace {

struct StepSeq {
  int seq, n_new;
};

constexpr int kPlaces = 512;          // states of segments that the workspace holds

// One launch of a step's plan (the same for every layer): sequences of few tokens, or in chunks.
struct Launch {
  bool chunk, split;
  LinearSeqs few;
  LinearChunkSeqs seqs;
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

struct fk_linear {
  fk_linear_config cfg{};
  std::vector<StepSeq> step;
  bool in_step = false;
  int64_t tokens = 0;                 // of the step
  std::vector<Launch> plan;           // of the step's sequences that have tokens
  int force_few = 0, force_segments = 0;
  float* place = nullptr;             // [kPlaces][D][D], and what segments leave of a state
  float2* place_decay = nullptr;
  int sms = 0;
  float* states = nullptr;            // [layers][max_seqs][Hkv][D][D]
  size_t per_seq = 0, per_layer = 0;  // floats
  int* status = nullptr;              // the status word, and a report of it
  std::vector<void*> allocs;
  size_t reserved = 0;
  int64_t launches = 0;
  ~fk_linear() {
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

fk_status done(fk_linear* h, cudaError_t e) {
  h->launches++;
  return e == cudaSuccess ? FK_OK : FK_ERR_CUDA;
}

fk_status alloc(fk_linear* h, size_t bytes, void** out) {
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

// ---- plan of a step
// Estimated times in us, measured back to back on a GB300: a launch's start and end; an item, and its chunks and each
// further query head of them, of the kernel that computes o and of the one that forms segments' states; the join of those; of the
// recurrence, a launch, a token of one sequence, and what all SMs together take for a token of one head.
struct Times {
  double start, item, chunk, head, item_local, chunk_local, join, few, few_token, few_share;
};
constexpr Times kTimes128{4.5, 3.0, 2.8, 2.3, 2.0, 1.8, 1.0, 2.2, 0.28, 0.0031}, kTimes64{3.0, 2.5, 2.0, 1.3, 1.5, 1.3, 1.0, 2.0, 0.22, 0.00105};

// Time of `groups` of equally long items (length, count), longest first, on the SMs: each goes to the one that is free first.
double fill_sms(const fk_linear* h, std::vector<std::pair<double, int64_t>>& groups) {
  std::sort(groups.begin(), groups.end(), [](const auto& x, const auto& y) { return x.first > y.first; });
  size_t kinds = 0;
  for (size_t i = 0; i < groups.size(); ++i) {       // those of one length as one group
    if (kinds > 0 && groups[kinds - 1].first == groups[i].first) groups[kinds - 1].second += groups[i].second;
    else groups[kinds++] = groups[i];
  }
  groups.resize(kinds);
  std::vector<double> busy(h->sms, 0.0), other(h->sms);
  for (const auto& g : groups) {
    int64_t left = g.second;
    const int64_t whole = left / h->sms > 8 ? left / h->sms - 8 : 0;   // (many rounds: as much for everyone)
    for (double& t : busy) t += (double)whole * g.first;
    left -= whole * h->sms;
    while (left > 0) {
      const auto again = std::lower_bound(busy.begin() + 1, busy.end(), busy[0] + g.first);   // (the first SM is free before it)
      const int n = (int)std::min<int64_t>(left, again - busy.begin());
      for (int i = 0; i < n; ++i) busy[i] += g.first;
      std::merge(busy.begin(), busy.begin() + n, busy.begin() + n, busy.end(), other.begin());
      busy.swap(other);
      left -= n;
    }
  }
  return busy.back();
}

int chunks_of(int tokens) { return (tokens + kLinearChunk - 1) / kLinearChunk; }

// ... of at most `per` each.
int segments_of(int chunks, int per) { return (chunks + per - 1) / per; }

// Estimated time of the sequences of more than `upto` tokens, sequence i split into segs[i]; huge where the workspace is too small.
double time_split(const fk_linear* h, const std::vector<StepSeq>& step, int upto, const std::vector<int>& segs) {
  const Times& t = h->cfg.head_dim == 128 ? kTimes128 : kTimes64;
  const int H = h->cfg.n_kv_heads;
  const double chunk = t.chunk + (h->cfg.n_q_heads / H - 1) * t.head;
  std::vector<std::pair<double, int64_t>> full, local;
  int64_t places = 0;
  for (size_t i = 0; i < step.size(); ++i) {
    if (step[i].n_new <= upto) continue;
    const int c = chunks_of(step[i].n_new), n = segs[i], per = c / n, more = c % n;
    if (more) full.push_back({t.item + (per + 1) * chunk, (int64_t)more * H});
    full.push_back({t.item + per * chunk, (int64_t)(n - more) * H});
    if (n > 1) {
      if (more) local.push_back({t.item_local + (per + 1) * t.chunk_local, (int64_t)more * H});
      if (n - 1 > more) local.push_back({t.item_local + per * t.chunk_local, (int64_t)(n - 1 - more) * H});
      places += (int64_t)n * H;
    }
  }
  if (places > kPlaces) return 1e30;
  return t.start + fill_sms(h, full) + (local.empty() ? 0.0 : t.start + fill_sms(h, local) + t.join);
}

// Into how many segments each sequence of more than `upto` tokens is split.  Splitting a sequence reads its keys and values twice and
// takes two launches more, and pays where long sequences would leave SMs idle.  First segments of the same length for all, then
// one more or less for single sequences, as long as it helps: the last round of items is what it evens out (prompts of
// 4001, 2500, 1777 and five shorter of 16 heads: 92.7 us with equal lengths alone, 89.8 so).
double best_split(const fk_linear* h, const std::vector<StepSeq>& step, int upto, std::vector<int>* segs) {
  int most = 0;
  segs->assign(step.size(), 1);
  std::vector<int> longest;
  for (size_t i = 0; i < step.size(); ++i)
    if (step[i].n_new > upto) {
      most = std::max(most, chunks_of(step[i].n_new));
      if (step[i].n_new > kLinearChunk) longest.push_back((int)i);
    }
  if (most == 0) return 0.0;
  // where all SMs are busy for longer than the longest sequence takes, there is nothing to gain
  int64_t chunks = 0;
  for (const StepSeq& s : step) chunks += s.n_new > upto ? chunks_of(s.n_new) : 0;
  if (chunks * h->cfg.n_kv_heads >= 2 * (int64_t)most * h->sms) return time_split(h, step, upto, *segs);
  double least = 1e30;
  std::vector<int> n(step.size(), 1);
  for (int parts = 1; parts <= most; parts += std::max(1, parts / 8)) {
    const int per = (most + parts - 1) / parts;
    for (const int i : longest) n[i] = segments_of(chunks_of(step[i].n_new), per);
    const double us = time_split(h, step, upto, n);
    if (us > 1e29) break;
    if (us < least - 0.5) {
      least = us;
      *segs = n;
    }
    if (per <= 1) break;
  }
  if (longest.size() < 2) return least;
  std::stable_sort(longest.begin(), longest.end(), [&](int x, int y) { return step[x].n_new > step[y].n_new; });
  if (longest.size() > 8) longest.resize(8);
  bool better = true;
  for (int pass = 0; pass < 3 && better; ++pass) {
    better = false;
    for (const int i : longest)
      for (const int d : {1, -1}) {
        n = *segs;
        n[i] += d;
        if (n[i] < 1 || n[i] > chunks_of(step[i].n_new)) continue;
        const double us = time_split(h, step, upto, n);
        if (us < least - 0.3) {
          least = us;
          *segs = n;
          better = true;
          break;
        }
      }
  }
  return least;
}

// Sequences of up to how many tokens go through the recurrence: it takes longer for each token, but a chunk takes as long
// for one as for 128.
int best_few(const fk_linear* h, const std::vector<StepSeq>& step, std::vector<int>* segs) {
  const Times& t = h->cfg.head_dim == 128 ? kTimes128 : kTimes64;
  const int G = h->cfg.n_q_heads / h->cfg.n_kv_heads;
  int best = 0;
  double least = 1e30;
  int64_t before = -1;
  std::vector<int> n;
  for (int upto : {1, 2, 4, 8, 16, 32}) {
    int longest = 0;
    int64_t tokens = 0, seqs = 0, beyond = 0, items = 0;
    for (const StepSeq& s : step) {
      if (s.n_new > upto) {
        ++beyond;
      } else {
        longest = std::max(longest, s.n_new);
        tokens += s.n_new;
        seqs += s.n_new > 0;
      }
    }
    if (beyond == before) continue;     // the same sequences as with the number before
    before = beyond;
    const double chunks_us = best_split(h, step, upto, &n);
    double few_us = 0.0;
    if (tokens > 0)
      few_us = t.few + (double)seqs * h->per_seq * 8 / 6.3e6 +   // (the states' bytes, and the tokens)
               (0.65 + 0.36 * G) * std::max(t.few_token * longest, t.few_share * (double)tokens * h->cfg.n_kv_heads);
    // they run beside one another where there are SMs for both: of the recurrence, four blocks of 32 columns keep an SM busy
    for (size_t i = 0; i < step.size(); ++i) items += step[i].n_new > upto ? (int64_t)n[i] * h->cfg.n_kv_heads : 0;
    const double blocks = (double)seqs * h->cfg.n_kv_heads * h->cfg.head_dim / 32;
    const double both = std::min(1.0, (double)items / h->sms) + std::min(1.0, blocks / (4.0 * h->sms)) - 1.0;
    const double us = std::max(few_us, chunks_us) + (0.2 + 0.8 * std::max(0.0, both)) * std::min(few_us, chunks_us);
    if (us < least) {
      least = us;
      best = upto;
      segs->swap(n);
    }
    if (beyond == 0) break;
  }
  return best;
}

// The launches of a step: sequences in chunks, the longest segments first, then those of few tokens, which fill the SMs that the
// chunks leave idle; kLinearSeqs to a launch.
void make_plan(const fk_linear* h, const std::vector<StepSeq>& step, std::vector<Launch>* plan) {
  const int H = h->cfg.n_kv_heads;
  int upto = 1;
  std::vector<int> segs_of(step.size(), 1);
  if (std::all_of(step.begin(), step.end(), [](const StepSeq& s) { return s.n_new <= 1; }) && h->force_few == 0) {
    upto = 1;                           // (a decoding step: nothing to estimate)
  } else if (h->force_few > 0) {
    upto = h->force_few;
    best_split(h, step, upto, &segs_of);
  } else {
    upto = best_few(h, step, &segs_of);
  }
  std::vector<int> order(step.size());
  std::vector<int64_t> tok0(step.size());
  int64_t tok = 0;
  for (size_t i = 0; i < step.size(); tok += step[i++].n_new) {
    order[i] = (int)i;
    tok0[i] = tok;
  }
  auto segments = [&](int i) { return h->force_segments > 0 ? std::min(h->force_segments, chunks_of(step[i].n_new)) : segs_of[i]; };
  auto length = [&](int i) { return segments_of(chunks_of(step[i].n_new), std::max(1, segments(i))); };
  for (const bool chunk : {true, false}) {
    Launch l{};
    int places = 0;
    auto push = [&] {
      if (chunk ? l.seqs.n : l.few.n) plan->push_back(l);
      l = Launch{};
      l.chunk = chunk;
      places = 0;
    };
    l.chunk = chunk;
    if (chunk) std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return length(x) > length(y); });
    for (const int i : order) {
      const StepSeq& s = step[i];
      if (s.n_new == 0 || (s.n_new > upto) != chunk) continue;
      if ((chunk ? l.seqs.n : l.few.n) == kLinearSeqs) push();
      if (!chunk) {
        const int k = l.few.n++;
        l.few.slot[k] = s.seq;
        l.few.out[k] = i;
        l.few.tok0[k] = (int)tok0[i];
        l.few.len[k] = s.n_new;
        continue;
      }
      const int k = l.seqs.n++;
      int segs = std::min(segments(i), (kPlaces - places) / H);
      if (segs < 2) segs = 1;
      l.seqs.slot[k] = s.seq;
      l.seqs.out[k] = i;
      l.seqs.tok0[k] = (int)tok0[i];
      l.seqs.len[k] = s.n_new;
      l.seqs.segs[k] = segs;
      l.seqs.per[k] = chunks_of(s.n_new) / segs;
      l.seqs.place0[k] = places;
      l.seqs.item0[k + 1] = l.seqs.item0[k] + segs * H;
      if (segs > 1) {
        places += segs * H;
        l.split = true;
      }
    }
    push();
  }
}

}  // namespace

extern "C" {

fk_status fk_linear_validate_config(const fk_linear_config* c) {
  if (!c) return FK_ERR_ARG;
  if (c->n_layers < 1 || c->n_layers > kMaxLayers) return FK_ERR_CONFIG;
  if (c->n_kv_heads < 1 || c->n_kv_heads > kMaxHeads || c->n_q_heads < c->n_kv_heads || c->n_q_heads > 1024 ||
      c->n_q_heads % c->n_kv_heads)
    return FK_ERR_CONFIG;
  if (c->head_dim != 64 && c->head_dim != 128) return FK_ERR_CONFIG;
  if (c->max_seqs < 1 || c->max_seqs > 65536) return FK_ERR_CONFIG;
  return FK_OK;
}

fk_status fk_linear_create(const fk_linear_config* cfg, fk_linear** out) {
  if (!out) return FK_ERR_ARG;
  *out = nullptr;
  fk_status st = fk_linear_validate_config(cfg);
  if (st != FK_OK) return st;
  return guarded([&]() -> fk_status {
    int n_dev = 0;
    if (cudaGetDeviceCount(&n_dev) != cudaSuccess || cfg->device < 0 || cfg->device >= n_dev) {
      cudaGetLastError();
      return FK_ERR_CUDA;
    }
    DeviceGuard dev(cfg->device);
    if (dev.err != cudaSuccess) return FK_ERR_CUDA;
    std::unique_ptr<fk_linear> h(new fk_linear());
    h->cfg = *cfg;
    h->per_seq = (size_t)cfg->n_kv_heads * cfg->head_dim * cfg->head_dim;
    h->per_layer = h->per_seq * cfg->max_seqs;
    void* p = nullptr;
    if ((st = alloc(h.get(), h->per_layer * cfg->n_layers * sizeof(float), &p)) != FK_OK) return st;
    h->states = static_cast<float*>(p);
    if ((st = alloc(h.get(), 2 * sizeof(int), &p)) != FK_OK) return st;
    h->status = static_cast<int*>(p);
    if ((st = alloc(h.get(), (size_t)kPlaces * cfg->head_dim * cfg->head_dim * sizeof(float), &p)) != FK_OK) return st;
    h->place = static_cast<float*>(p);
    if ((st = alloc(h.get(), kPlaces * sizeof(float2), &p)) != FK_OK) return st;
    h->place_decay = static_cast<float2*>(p);
    if (cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, cfg->device) != cudaSuccess) return FK_ERR_CUDA;
    if (linear_chunk_prepare(cfg->head_dim) != cudaSuccess) return FK_ERR_CUDA;
    if (cudaDeviceSynchronize() != cudaSuccess) return FK_ERR_CUDA;
    *out = h.release();
    return FK_OK;
  });
}

void fk_linear_destroy(fk_linear* h) {
  if (!h) return;
  DeviceGuard dev(h->cfg.device);
  cudaDeviceSynchronize();
  delete h;
}

fk_status fk_linear_step(fk_linear* h, int n_seqs, const int32_t* seqs, const int32_t* n_new) {
  if (!h || n_seqs < 0 || (n_seqs > 0 && (!seqs || !n_new))) return FK_ERR_ARG;
  if (n_seqs > h->cfg.max_seqs) return FK_ERR_ARG;
  return guarded([&]() -> fk_status {
    std::vector<uint8_t> seen(h->cfg.max_seqs, 0);
    std::vector<StepSeq> step(n_seqs);
    int64_t total = 0;
    for (int i = 0; i < n_seqs; ++i) {
      if (seqs[i] < 0 || seqs[i] >= h->cfg.max_seqs || seen[seqs[i]] || n_new[i] < 0) return FK_ERR_ARG;
      seen[seqs[i]] = 1;
      step[i] = {seqs[i], n_new[i]};
      total += n_new[i];
    }
    if (total * h->cfg.n_q_heads >= ((int64_t)1 << 31)) return FK_ERR_ARG;
    std::vector<Launch> plan;
    make_plan(h, step, &plan);
    h->plan.swap(plan);
    h->step.swap(step);
    h->tokens = total;
    h->in_step = true;
    return FK_OK;
  });
}

fk_status fk_linear_attend(fk_linear* h, int layer, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                           const void* V, int64_t v_stride, const float* decay, int64_t decay_stride, void* O, int64_t o_stride,
                           float scale, int mode, float* state_out, void* stream) {
  if (!h || layer < 0 || layer >= h->cfg.n_layers) return FK_ERR_ARG;
  if ((mode != FK_LINEAR_ADVANCE && mode != FK_LINEAR_STAY) || !(scale >= 0.0f) || std::isinf(scale)) return FK_ERR_CONFIG;
  if (mode == FK_LINEAR_ADVANCE && state_out) return FK_ERR_ARG;
  if (!h->in_step) return FK_ERR_STATE;
  const fk_linear_config& c = h->cfg;
  if (h->step.empty() || (h->tokens == 0 && !state_out)) return FK_OK;
  return guarded([&]() -> fk_status {
    DeviceGuard dev(c.device);
    if (dev.err != cudaSuccess) return FK_ERR_CUDA;
    Rows taken{};                       // state_out
    if (state_out) {
      const size_t bytes = h->step.size() * h->per_seq * sizeof(float);
      const uintptr_t p = reinterpret_cast<uintptr_t>(state_out), own = reinterpret_cast<uintptr_t>(h->states);
      if (!aligned(state_out, 16) || !on_device(state_out, c.device)) return FK_ERR_ARG;
      if (p < own + h->per_layer * c.n_layers * sizeof(float) && own < p + bytes) return FK_ERR_ARG;
      taken = Rows{p, (int64_t)bytes, (int64_t)bytes};
    }
    if (h->tokens > 0) {
      const int64_t wq = (int64_t)c.n_q_heads * c.head_dim, wk = (int64_t)c.n_kv_heads * c.head_dim;
      auto rows_ok = [&](const void* p, int64_t stride, int64_t width) {
        return p && aligned(p, 16) && stride >= width && stride % 8 == 0 && on_device(p, c.device);
      };
      if (!rows_ok(Q, q_stride, wq) || !rows_ok(O, o_stride, wq) || !rows_ok(K, k_stride, wk) || !rows_ok(V, v_stride, wk))
        return FK_ERR_ARG;
      if (!decay || !aligned(decay, 4) || (decay_stride != 0 && decay_stride < c.n_kv_heads) || !on_device(decay, c.device))
        return FK_ERR_ARG;
      auto rows = [](const void* p, int64_t stride, int64_t width) {
        return Rows{reinterpret_cast<uintptr_t>(p), stride * 2, width * 2};
      };
      const int64_t T = h->tokens;
      const Rows o = rows(O, o_stride, wq), own = whole(Rows{reinterpret_cast<uintptr_t>(h->states), (int64_t)(h->per_layer * 4), (int64_t)(h->per_layer * 4)}, c.n_layers);
      const Rows g{reinterpret_cast<uintptr_t>(decay), decay_stride * 4, (int64_t)c.n_kv_heads * 4};
      for (const Rows& in : {rows(Q, q_stride, wq), rows(K, k_stride, wk), rows(V, v_stride, wk), g}) {
        if (in.stride ? meet(o, in, T) : meet(whole(o, T), in, 1)) return FK_ERR_ARG;
        if (state_out && meet(taken, whole(in, T), 1)) return FK_ERR_ARG;
      }
      if (meet(whole(o, T), own, 1) || (state_out && meet(taken, whole(o, T), 1))) return FK_ERR_ARG;
    }
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const float sc = scale > 0.0f ? scale : (float)(1.0 / std::sqrt((double)c.head_dim));
    const float* held = h->states + h->per_layer * layer;
    float* state_new = mode == FK_LINEAR_ADVANCE ? h->states + h->per_layer * layer : state_out;
    auto fill = [&](auto& a) {
      a.Q = static_cast<const bf16*>(Q);
      a.K = static_cast<const bf16*>(K);
      a.V = static_cast<const bf16*>(V);
      a.O = static_cast<bf16*>(O);
      a.qstride = q_stride;
      a.kstride = k_stride;
      a.vstride = v_stride;
      a.ostride = o_stride;
      a.decay = decay;
      a.dstride = decay_stride;
      a.scale = sc;
      a.Hkv = c.n_kv_heads;
      a.G = c.n_q_heads / c.n_kv_heads;
      a.state = held;
      a.state_new = state_new;
      a.to_out = mode != FK_LINEAR_ADVANCE;
      a.status = h->status;
    };
    LinearArgs f;
    fill(f);
    bool beside = false;
    for (const Launch& l : h->plan) {
      if (!l.chunk) {
        f.seqs = l.few;
        const fk_status e = done(h, launch_linear_few(c.head_dim, f, beside, st));
        beside = false;
        if (e != FK_OK) return e;
        continue;
      }
      LinearChunkArgs a;
      fill(a);
      a.log2_scale = (float)std::log2((double)sc);
      a.place = h->place;
      a.place_decay = h->place_decay;
      a.seqs = l.seqs;
      a.items = l.seqs.item0[l.seqs.n];
      a.ctas = h->sms;
      CUtensorMap tmQ, tmK, tmV, tmO;
      if (!encode_bf16_rows(&tmQ, Q, h->tokens, (int64_t)c.n_q_heads * c.head_dim, q_stride, kLinearChunk) ||
          !encode_bf16_rows(&tmK, K, h->tokens, (int64_t)c.n_kv_heads * c.head_dim, k_stride, kLinearChunk) ||
          !encode_bf16_rows(&tmV, V, h->tokens, (int64_t)c.n_kv_heads * c.head_dim, v_stride, kLinearChunk) ||
          !encode_bf16_rows(&tmO, O, h->tokens, (int64_t)c.n_q_heads * c.head_dim, o_stride, 32))
        return FK_ERR_CUDA;
      h->launches += l.split ? 2 : 0;
      beside = true;
      const fk_status e = done(h, launch_linear_chunk(c.head_dim, l.split, tmQ, tmK, tmV, tmO, a, st));
      if (e != FK_OK) return e;
    }
    if (!state_out || !std::any_of(h->step.begin(), h->step.end(), [](const StepSeq& s) { return s.n_new == 0; })) return FK_OK;
    // sequences without tokens: their states as they are
    f.seqs.n = 0;
    for (size_t i = 0; i < h->step.size(); ++i) {
      if (h->step[i].n_new == 0) {
        const int k = f.seqs.n++;
        f.seqs.slot[k] = h->step[i].seq;
        f.seqs.out[k] = (int)i;
        f.seqs.tok0[k] = f.seqs.len[k] = 0;
      }
      if (f.seqs.n == kLinearSeqs || (i + 1 == h->step.size() && f.seqs.n > 0)) {
        const fk_status e = done(h, launch_linear_few(c.head_dim, f, false, st));
        if (e != FK_OK) return e;
        f.seqs.n = 0;
      }
    }
    return FK_OK;
  });
}

fk_status fk_linear_force_plan(fk_linear* h, int few, int segments) {
  if (!h) return FK_ERR_ARG;
  if (few < 0 || segments < 0) return FK_ERR_CONFIG;
  h->force_few = few;
  h->force_segments = segments;
  return FK_OK;
}

fk_status fk_linear_states(const fk_linear* h, int layer, float** states) {
  if (!h || layer < 0 || layer >= h->cfg.n_layers || !states) return FK_ERR_ARG;
  *states = h->states + h->per_layer * layer;
  return FK_OK;
}

fk_status fk_linear_drop(fk_linear* h, int seq, void* stream) {
  if (!h || seq < 0 || seq >= h->cfg.max_seqs) return FK_ERR_ARG;
  DeviceGuard dev(h->cfg.device);
  if (dev.err != cudaSuccess) return FK_ERR_CUDA;
  for (int l = 0; l < h->cfg.n_layers; ++l)
    if (cudaMemsetAsync(h->states + h->per_layer * l + h->per_seq * seq, 0, h->per_seq * sizeof(float),
                        static_cast<cudaStream_t>(stream)) != cudaSuccess)
      return FK_ERR_CUDA;
  return FK_OK;
}

fk_status fk_linear_fork(fk_linear* h, int dst, int src, void* stream) {
  if (!h || dst < 0 || dst >= h->cfg.max_seqs || src < 0 || src >= h->cfg.max_seqs) return FK_ERR_ARG;
  if (dst == src) return FK_OK;
  DeviceGuard dev(h->cfg.device);
  if (dev.err != cudaSuccess) return FK_ERR_CUDA;
  for (int l = 0; l < h->cfg.n_layers; ++l) {
    float* s = h->states + h->per_layer * l;
    if (cudaMemcpyAsync(s + h->per_seq * dst, s + h->per_seq * src, h->per_seq * sizeof(float), cudaMemcpyDeviceToDevice,
                        static_cast<cudaStream_t>(stream)) != cudaSuccess)
      return FK_ERR_CUDA;
  }
  return FK_OK;
}

size_t fk_linear_reserved_bytes(const fk_linear* h) { return h ? h->reserved : 0; }

int64_t fk_linear_launch_count(const fk_linear* h) { return h ? h->launches : 0; }

fk_status fk_linear_sync_status(fk_linear* h, void* stream) {
  if (!h) return FK_ERR_ARG;
  DeviceGuard dev(h->cfg.device);
  if (dev.err != cudaSuccess) return FK_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int word = 0;
  if (done(h, launch_linear_status(h->status, h->status + 1, s)) != FK_OK ||
      cudaMemcpyAsync(&word, h->status + 1, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess)
    return FK_ERR_CUDA;
  return word & kStatusTimeout ? FK_ERR_TIMEOUT : FK_OK;
}

}  // extern "C"
