// C-ABI entry points of the vocabulary ends: argument checks, upload of the token tables, dispatch.  See include/dta.h.
#include <atomic>
#include <cstdio>
#include <new>

#include "dta_vocab.h"

namespace {

inline bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

// The tables' copy on the current device, made if it is not there (waits for the copy only).  Under tokens->mu.
int tables_on(dta_tokens* t, int dev, dta::TokenTables* out) {
  const int32_t* base = nullptr;
  for (const auto& c : t->copies)
    if (c.device == dev) base = (const int32_t*)c.block;
  if (!base) {
    void* block = nullptr;
    size_t cap = 0;
    t->copies.reserve(t->copies.size() + 1);
    const int st = dta::upload_block(dev, t->table.data(), t->table.size() * sizeof(int32_t), &block, &cap);
    if (st != DTA_OK) return st;
    t->copies.push_back({dev, block, cap});
    base = (const int32_t*)block;
  }
  out->id = base + t->at.id;
  out->slot = base + t->at.slot;
  out->before = base + t->at.before;
  out->row = base + t->at.row;
  out->edge_ptr = base + t->at.edge_ptr;
  out->only = base + t->at.only;
  out->edge_token = base + t->at.edge_token;
  out->edge_id = base + t->at.edge_id;
  out->order = base + t->at.order;
  out->part = (const dta::EmbedPart*)(base + t->at.part);
  out->merge = (const dta::EmbedMerge*)(base + t->at.merge);
  out->present = (const uint32_t*)(base + t->at.present);
  return DTA_OK;
}

// The calling thread's number, from 1 on; no other thread of the process has had it.
uint64_t thread_number() {
  static std::atomic<uint64_t> last{0};
  static thread_local const uint64_t mine = ++last;
  return mine;
}

// The event of the latest call on (stream, device).  Streams that are no longer used leave theirs behind;
// completed ones are taken out when there are many.
hipEvent_t use_event(dta_tokens* t, void* stream, int dev) {
  const uint64_t thread = stream == (void*)hipStreamPerThread ? thread_number() : 0;
  for (const auto& u : t->uses)
    if (u.stream == stream && u.thread == thread && u.device == dev) return (hipEvent_t)u.event;
  if (t->uses.size() >= 64) {
    size_t kept = 0;
    for (const auto& u : t->uses) {
      if (hipEventQuery((hipEvent_t)u.event) == hipSuccess) {
        (void)hipEventDestroy((hipEvent_t)u.event);
      } else {
        (void)hipGetLastError();
        t->uses[kept++] = u;
      }
    }
    t->uses.resize(kept);
  }
  hipEvent_t ev;
  t->uses.reserve(t->uses.size() + 1);
  // (without the system-scope fence: it orders uses of tables that kernels only read)
  if (hipEventCreateWithFlags(&ev, hipEventDisableTiming | hipEventDisableSystemFence) != hipSuccess) {
    (void)hipGetLastError();
    return nullptr;
  }
  t->uses.push_back({stream, thread, dev, ev});
  return ev;
}

// Runs a call's launches on the current device, and has the event of its stream complete after them.  A call under
// capture leaves no event: the tables outlive the graph.
int run(dta_tokens* t, dta::VocabArgs& a, int (*launcher)(const dta::VocabArgs&)) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) {
    fprintf(stderr, "dta: hipGetDevice failed (no usable GPU?)\n");
    (void)hipGetLastError();
    return DTA_ERR_HIP;
  }
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(a.stream, &capture) != hipSuccess) {
    (void)hipGetLastError();
    capture = hipStreamCaptureStatusNone;
  }
  try {
    std::lock_guard<std::mutex> lock(t->mu);
    if (capture != hipStreamCaptureStatusNone) {
      bool resident = false;
      for (const auto& c : t->copies) resident |= c.device == dev;
      if (!resident) return DTA_ERR_INVALID_ARG;
    }
    const int st = tables_on(t, dev, &a.tab);
    if (st != DTA_OK) return st;
    a.tokens = t;
    bool recorded = false, failed = false;
    a.done_recorded = &recorded;
    a.failed = &failed;
    if (capture != hipStreamCaptureStatusNone) return launcher(a);
    const hipEvent_t ev = use_event(t, (void*)a.stream, dev);
    if (!ev) return DTA_ERR_HIP;
    a.done_event = ev;
    const int launched = launcher(a);
    // (also after a launch that failed, which the event may have been attached to: those before it may be running)
    if ((!recorded || launched != DTA_OK) && hipEventRecord(ev, a.stream) != hipSuccess) {
      (void)hipGetLastError();
      return launched != DTA_OK ? launched : DTA_ERR_HIP;
    }
    return launched;
  } catch (const std::bad_alloc&) {
    return DTA_ERR_ALLOC;
  }
}

// Parameters, and sizes whose launches would have 2^32 threads: a thread of the narrowest kernel has 4 elements of a row (of
// which the last block of a row may leave half empty), a block of 256 threads a row.
int check_params(const dta_tokens* t, const dta_vocab_params_t* p, bool logprob) {
  const int st = dta::validate_vocab_params(p);
  if (st != DTA_OK) return st;
  const int64_t most = t->n_tokens > t->vocab ? t->n_tokens : t->vocab;
  return most * p->width >= (int64_t)1 << 33 || (logprob && most >= 1 << 24) ? DTA_ERR_UNSUPPORTED : DTA_OK;
}

int check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (need == 0) return DTA_OK;
  return workspace && bytes >= need && ((uintptr_t)workspace & 255u) == 0 ? DTA_OK : DTA_ERR_WORKSPACE;
}

}  // namespace

extern "C" {

int dta_tokens_prepare(dta_tokens_t* tokens) {
  if (!tokens) return DTA_ERR_INVALID_ARG;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) {
    fprintf(stderr, "dta: hipGetDevice failed (no usable GPU?)\n");
    (void)hipGetLastError();
    return DTA_ERR_HIP;
  }
  try {
    std::lock_guard<std::mutex> lock(tokens->mu);
    dta::TokenTables tab;
    return tables_on(tokens, dev, &tab);
  } catch (const std::bad_alloc&) {
    return DTA_ERR_ALLOC;
  }
}

void dta_tokens_destroy(dta_tokens_t* tokens) {
  if (!tokens) return;
  try {
    // the copies go back to the pool together with the events after the last launches that read them
    std::vector<dta::DeviceBlock> blocks;
    std::vector<void*> events;
    for (const auto& c : tokens->copies) blocks.push_back({c.device, c.block, c.cap});
    for (const auto& u : tokens->uses) events.push_back(u.event);
    dta::release_blocks(blocks.data(), blocks.size(), events.data(), events.size());
  } catch (const std::bad_alloc&) {   // (no memory to note them down: the blocks stay as they are)
  }
  delete tokens;
}

size_t dta_vocab_workspace_bytes(const dta_tokens_t* tokens, const dta_vocab_params_t* params, int call) {
  if (!tokens || check_params(tokens, params, call != DTA_VOCAB_EMBED_BWD) != DTA_OK) return 0;
  switch (call) {
    case DTA_VOCAB_EMBED_BWD: return dta::embed_bwd_workspace(tokens, params);
    case DTA_VOCAB_LOGPROB_FWD: return dta::logprob_fwd_workspace(tokens, params);
    case DTA_VOCAB_LOGPROB_BWD: return dta::logprob_bwd_workspace(tokens, params);
  }
  return 0;
}

int dta_tree_embed_fwd(dta_tokens_t* tokens, const dta_vocab_params_t* params, const void* table, void* x,
                       void* hip_stream) {
  if (!tokens || !params) return DTA_ERR_INVALID_ARG;
  const int st = check_params(tokens, params, false);
  if (st != DTA_OK) return st;
  if (!table || !x || misaligned(table) || misaligned(x)) return DTA_ERR_INVALID_ARG;
  dta::VocabArgs a{};
  a.p = *params;
  a.table = table;
  a.x = x;
  a.stream = (hipStream_t)hip_stream;
  return run(tokens, a, dta::launch_embed_fwd);
}

int dta_tree_embed_bwd(dta_tokens_t* tokens, const dta_vocab_params_t* params, const void* d_x, void* d_table,
                       uint32_t flags, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!tokens || !params) return DTA_ERR_INVALID_ARG;
  int st = check_params(tokens, params, false);
  if (st != DTA_OK) return st;
  if (flags & ~(uint32_t)DTA_GRAD_ADD) return DTA_ERR_INVALID_ARG;
  if (!d_x || !d_table || misaligned(d_x) || misaligned(d_table)) return DTA_ERR_INVALID_ARG;
  if ((st = check_workspace(workspace, workspace_bytes, dta::embed_bwd_workspace(tokens, params))) != DTA_OK) return st;
  dta::VocabArgs a{};
  a.p = *params;
  a.d_x = d_x;
  a.d_table = d_table;
  a.add = flags & DTA_GRAD_ADD;
  a.workspace = (char*)workspace;
  a.stream = (hipStream_t)hip_stream;
  return run(tokens, a, dta::launch_embed_bwd);
}

int dta_tree_logprob_fwd(dta_tokens_t* tokens, const dta_vocab_params_t* params, const void* hidden,
                         const void* weight, float* logp, float* lse, void* workspace, size_t workspace_bytes,
                         void* hip_stream) {
  if (!tokens || !params) return DTA_ERR_INVALID_ARG;
  int st = check_params(tokens, params, true);
  if (st != DTA_OK) return st;
  if (!hidden || !weight || !logp || !lse) return DTA_ERR_INVALID_ARG;
  if (misaligned(hidden) || misaligned(weight) || misaligned(logp) || misaligned(lse)) return DTA_ERR_INVALID_ARG;
  if ((st = check_workspace(workspace, workspace_bytes, dta::logprob_fwd_workspace(tokens, params))) != DTA_OK)
    return st;
  dta::VocabArgs a{};
  a.p = *params;
  a.hidden = hidden;
  a.weight = weight;
  a.logp = logp;
  a.lse = lse;
  a.workspace = (char*)workspace;
  a.stream = (hipStream_t)hip_stream;
  return run(tokens, a, dta::launch_logprob_fwd);
}

int dta_tree_logprob_bwd(dta_tokens_t* tokens, const dta_vocab_params_t* params, const void* hidden,
                         const void* weight, const float* lse, const float* d_logp, void* d_hidden,
                         void* d_weight, uint32_t flags, void* workspace, size_t workspace_bytes,
                         void* hip_stream) {
  if (!tokens || !params) return DTA_ERR_INVALID_ARG;
  int st = check_params(tokens, params, true);
  if (st != DTA_OK) return st;
  if (flags & ~(uint32_t)DTA_GRAD_ADD) return DTA_ERR_INVALID_ARG;
  if (!hidden || !weight || !lse || !d_logp || (!d_hidden && !d_weight)) return DTA_ERR_INVALID_ARG;
  if (misaligned(hidden) || misaligned(weight) || misaligned(lse) || misaligned(d_logp) || misaligned(d_hidden) ||
      misaligned(d_weight))
    return DTA_ERR_INVALID_ARG;
  if ((st = check_workspace(workspace, workspace_bytes, dta::logprob_bwd_workspace(tokens, params))) != DTA_OK)
    return st;
  dta::VocabArgs a{};
  a.p = *params;
  a.hidden = hidden;
  a.weight = weight;
  a.lse_in = lse;
  a.d_logp = d_logp;
  a.d_hidden = d_hidden;
  a.d_weight = d_weight;
  a.add = flags & DTA_GRAD_ADD;
  a.workspace = (char*)workspace;
  a.stream = (hipStream_t)hip_stream;
  return run(tokens, a, dta::launch_logprob_bwd);
}

}  // extern "C"
