// The host handle of a cache, shared by the files that implement the C ABI.
#pragma once
#include "mixkvq_internal.h"

struct SeqState {
  int64_t n_quant;   // quantized tokens
  int32_t n_res;     // tokens in the residual window
  int32_t n_sink;    // tokens in the sink
  bool operator==(const SeqState& o) const { return n_quant == o.n_quant && n_res == o.n_res && n_sink == o.n_sink; }
};

struct mixkvq_cache {
  mixkvq::CacheView v;   // v.cfg.R is the number of tokens per RECORD (what the kernels work on): rec_tokens()
  int32_t Rw;            // the residual length R of the configuration: window size and flush unit, Rw / v.cfg.R records per block
  SeqState* seq;         // [B]: every sequence has its own counts (they are equal while the batch runs in lock-step)
  hipEvent_t ev_start = nullptr, ev_stop = nullptr;   // optional timing of the split kernel
  int last_path = MIXKVQ_PATH_NONE;                   // kernel of the last attention launch
  int last_chunk = 0;                                 // query rows of a workgroup in the last launch of several new tokens
  bool tickets_clear = false;                         // the ticket words were set to 0 once
};

namespace mixkvq {

int hip_fail(hipError_t e);                  // keeps HIP's message for mixkvq_strerror; MIXKVQ_EHIP
#define MIXKVQ_TRY_HIP(expr)                          \
  do {                                                \
    hipError_t e__ = (expr);                          \
    if (e__ != hipSuccess) return hip_fail(e__);      \
  } while (0)

bool lock_step(const mixkvq_cache* c);       // do all sequences hold the same numbers of tokens?

}  // namespace mixkvq
