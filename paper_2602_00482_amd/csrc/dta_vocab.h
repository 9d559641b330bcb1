// The vocabulary ends of a tree pass: what the entry points hand to the launchers.  Not part of the public interface.
#pragma once

#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include "dta_internal.h"
#include "dta_tokens.h"

namespace dta {

struct VocabArgs {
  const dta_tokens* tokens;
  TokenTables tab;
  dta_vocab_params_t p;
  // embedding: table / x, or d_x / d_table
  const void *table, *d_x;
  void *x, *d_table;
  // log-probabilities
  const void *hidden, *weight;
  const float *lse_in, *d_logp;
  float *logp, *lse;
  void *d_hidden, *d_weight;
  bool add;   // d_table / d_weight is an fp32 accumulator
  char* workspace;
  hipStream_t stream;
  // event the call's last launch may attach to itself, and whether it has; null: recorded afterwards
  hipEvent_t done_event;
  bool* done_recorded;
  bool* failed;   // a launch of the call was refused: the rest of them are left out
};

// Launches a kernel on the call's stream; `last`: no launch of the call follows.  Nothing behind one that failed: it would read
// what that one did not write.
template <typename... P, typename... A>
inline void launch(const VocabArgs& a, bool last, void (*kernel)(P...), size_t grid, unsigned block, A... args) {
  if (*a.failed) return;
  if (last && a.done_event != nullptr) {
    hipExtLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(block), 0, a.stream, nullptr, a.done_event, 0,
                          static_cast<P>(args)...);
    *a.done_recorded = true;
  } else {
    kernel<<<(unsigned)grid, block, 0, a.stream>>>(static_cast<P>(args)...);
  }
  *a.failed = hipPeekAtLastError() != hipSuccess;
}

inline size_t elem_size(const dta_vocab_params_t& p) { return p.dtype == DTA_F32 ? 4 : 2; }

size_t embed_bwd_workspace(const dta_tokens* t, const dta_vocab_params_t* p);
size_t logprob_fwd_workspace(const dta_tokens* t, const dta_vocab_params_t* p);
size_t logprob_bwd_workspace(const dta_tokens* t, const dta_vocab_params_t* p);
int launch_embed_fwd(const VocabArgs& a);
int launch_embed_bwd(const VocabArgs& a);
int launch_logprob_fwd(const VocabArgs& a);
int launch_logprob_bwd(const VocabArgs& a);

}  // namespace dta
