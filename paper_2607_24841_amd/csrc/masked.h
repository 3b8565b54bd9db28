// Internal declarations of the masked attention and of drawing tokens (not installed).
#pragma once

#include "common.h"

namespace nmdlm {

struct MaskedAttnCall {
  const uint64_t* q;
  const uint64_t* k_cache;
  const uint64_t* vt_cache;
  int64_t cap;
  int T, M, n_keys, H, dh;
  const uint8_t* lut;
  nmdlm_mask mask;
  const int8_t* bias;  // or null
  int32_t* a_out;      // or null
  int32_t theta;
  uint64_t* s_out;     // or null
  uint64_t* u_out;     // or null: per-row union over t
  void* ws;
};
// Rows of a workgroup (1: the row kernel; 16 or 32: tiles), waves a timestep, most
// splits; heads: workgroups of several heads, whose sums a second kernel joins.
struct MaskedRoute {
  int tile, parts, splits;
  bool heads;
};
MaskedRoute masked_route(int T, int M, int n_keys, int H);
size_t masked_attn_ws(int T, int M, int n_keys, int H, int dh);
nmdlm_status launch_masked_attn(const MaskedAttnCall& c, hipStream_t st);

// A block step whose rows see the keys of a mask.
struct MaskedStep {
  const nmdlm_mask* mask;
  const int8_t* const* bias;  // host array [n_layers], or null
};

struct VerifyCall {
  const float* logits;
  const float* draft_logits;  // or null
  const int32_t* draft;       // null: every row is drawn from its logits
  const float* u;             // [M][2], or [M] without drafts
  int M, V;
  double tau, draft_tau;
  const int32_t* cu;          // or null
  int n_seq;
  bool each;
  int32_t* tokens;
  uint8_t* accepted;
  int32_t* n_accepted;
  double* conf;
  void* ws;
};
size_t verify_ws(int M, int V, bool drafts);
// The logits to read for row m's draft.  A row without one has none: the caller's may end
// before it (the row that follows a request's drafts), so the target's are read instead.
__host__ __device__ inline const float* draft_logits_at(const float* logits, const float* draft_logits, int m,
                                                        int V, int32_t draft) {
  return ((uint32_t)draft < (uint32_t)V ? draft_logits : logits) + (size_t)m * V;
}
nmdlm_status launch_verify(const VerifyCall& c, hipStream_t st);

}  // namespace nmdlm
