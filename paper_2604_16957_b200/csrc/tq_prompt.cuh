// A packed sequence's rows and the keys that a query sees (tq_sdpa_prompt).
#pragma once
#include "tq_internal.cuh"

namespace tq {

struct PromptSeq {
  int q0, lq, k0, lk;  // first query row and count, first key row and count
};

// Rows of sequence b, inside the buffers whatever the offsets say.  `report`: this thread sets the status bits.
__device__ __forceinline__ PromptSeq prompt_seq(const PromptArgs& a, int b, bool report) {
  const int q0 = a.q_offsets[b], q1 = a.q_offsets[b + 1], k0 = a.kv_offsets[b], k1 = a.kv_offsets[b + 1];
  PromptSeq s;
  s.q0 = min(max(q0, 0), a.n_q);
  s.lq = max(min(max(q1, 0), a.n_q) - s.q0, 0);
  s.k0 = min(max(k0, 0), a.n_kv);
  s.lk = max(min(max(k1, 0), a.n_kv) - s.k0, 0);
  if (report && a.status) {
    int bits = 0;
    if (q0 < 0 || q1 < q0 || q1 > a.n_q || k0 < 0 || k1 < k0 || k1 > a.n_kv) bits |= TQ_STATUS_BAD_LEN;
    if (s.lq > 0 && s.lk == 0) bits |= TQ_STATUS_EMPTY_SEQ;
    if (bits) atomicOr(a.status, bits);
  }
  return s;
}

// Keys [lo, up) of the sequence that its query i sees.
__device__ __forceinline__ void prompt_keys(const PromptArgs& a, const PromptSeq& s, int i, int& lo, int& up) {
  lo = 0;
  up = s.lk;
  if (a.causal) {
    up = i + s.lk - s.lq + 1;
    up = up < 0 ? 0 : up;
    if (a.window > 0 && up > a.window) lo = up - a.window;
  }
}

}  // namespace tq
