// prompt_common.cuh -- what the kernels over packed prompts share: where a sequence lies and what its
// queries look at.
#pragma once

#include "hill_internal.h"

namespace hill {
namespace {

// Sequence b: its query rows [q0, q0 + n) and key rows [k0, k0 + m); query i is at position i + m - n.
struct Seq {
  int q0, n, k0, m;
  __device__ __forceinline__ int shift() const { return m - n; }
};

__device__ __forceinline__ Seq seq_at(const PromptArgs& a, int b) {
  const int q0 = a.q_start[b], q1 = a.q_start[b + 1], k0 = a.k_start[b], k1 = a.k_start[b + 1];
  Seq s;
  s.q0 = min(max(q0, 0), a.q_rows);
  s.n = max(min(q1, a.q_rows) - s.q0, 0);
  s.k0 = min(max(k0, 0), a.k_rows);
  s.m = max(min(k1, a.k_rows) - s.k0, 0);
  if (q0 < 0 || q1 < q0 || q1 > a.q_rows || k0 < 0 || k1 < k0 || k1 > a.k_rows) raise_error(a.err, kErrDevArg);
  return s;
}

// Bits 0 to x.
__device__ __forceinline__ uint32_t bits_to(int x) { return x < 0 ? 0u : (x >= 31 ? ~0u : (2u << x) - 1u); }

}  // namespace
}  // namespace hill
