// Tokens drawn from logits and verification of drafted tokens: weights in
// float64, running sums in the order of the ids (the definitions: nmdlm.h).
#include <math.h>

#include "masked.h"

namespace nmdlm {

struct VerifyArgs {
  const float* logits;
  const float* draft_logits;
  const int32_t* draft;
  const float* u;
  const int32_t* cu;
  int M, V, n_seq;
  double tau, draft_tau;
  int32_t* tokens;
  uint8_t* accepted;
  int32_t* n_accepted;
  double* conf;
  bool chain;
};

constexpr int kRowThreads = 256;
constexpr double kExpFloor = -700.0;  // exponents below weigh nothing

// A row of logits at a temperature: its largest value, that value's first id and
// the sum of the weights.
struct Row {
  const float* l;
  float top;
  int first;
  double inv, sum;
  bool some, sharp;  // any weight; temperature 0
  __device__ __forceinline__ double weight(int v) const {
    const float x = l[v];
    if (!some || x != x) return 0.0;
    if (x == top) return 1.0;
    const double e = ((double)x - (double)top) * inv;
    return e >= kExpFloor ? exp(e) : 0.0;
  }
  // probability in the draw (temperature 0: all on the first)
  __device__ __forceinline__ double prob(int v) const {
    if (!some) return 0.0;
    return sharp ? (v == first ? 1.0 : 0.0) : weight(v) / sum;
  }
};

struct Shared {
  double sum[kRowThreads];
  float top[kRowThreads];
  int id[kRowThreads];
};

// Thread i's ids are [i n / 256, (i + 1) n / 256).
__device__ __forceinline__ int part_of(int V, int i) { return (int)((long long)V * i / kRowThreads); }

__device__ Row read_row(const float* l, int V, double tau, Shared& s) {
  const int tid = threadIdx.x, v0 = part_of(V, tid), v1 = part_of(V, tid + 1);
  Row r{l, -INFINITY, 0, tau > 0.0 ? 1.0 / tau : 1.0, 0.0, false, tau == 0.0};
  for (int v = v0; v < v1; ++v)
    if (l[v] > r.top) {
      r.top = l[v];
      r.first = v;
    }
  __syncthreads();
  s.top[tid] = r.top;
  s.id[tid] = r.first;
  __syncthreads();
  for (int i = 0; i < kRowThreads; ++i)  // in the order of the ids
    if (i == 0 || s.top[i] > r.top) {
      r.top = s.top[i];
      r.first = s.id[i];
    }
  r.some = r.top > -INFINITY;
  double sum = 0.0;
  for (int v = v0; v < v1; ++v) sum += r.weight(v);
  s.sum[tid] = sum;
  __syncthreads();
  for (int i = 0; i < kRowThreads; ++i) r.sum += s.sum[i];
  return r;
}

// First id whose running sum of w exceeds u times the sum of all (the last of
// positive weight when none does); -1 when the sum is 0.
template <typename W>
__device__ int pick(int V, float u, Shared& s, W w) {
  const int tid = threadIdx.x, v0 = part_of(V, tid), v1 = part_of(V, tid + 1);
  double sum = 0.0;
  for (int v = v0; v < v1; ++v) sum += w(v);
  __syncthreads();
  s.sum[tid] = sum;
  __syncthreads();
  double total = 0.0;
  for (int i = 0; i < kRowThreads; ++i) total += s.sum[i];
  if (!(total > 0.0)) return -1;
  const double target = u < 1.0f ? (double)u * total : INFINITY;  // 1 and beyond: no sum exceeds it
  double before = 0.0;
  int at = -1, last = -1;  // the thread whose ids hold the token
  for (int i = 0; i < kRowThreads; ++i) {
    if (s.sum[i] > 0.0) last = i;
    if (before + s.sum[i] > target) {
      at = i;
      break;
    }
    before += s.sum[i];
  }
  if (at < 0) at = last;
  if (tid == at) {
    int id = v0;
    for (int v = v0; v < v1; ++v) {
      const double x = w(v);
      if (x > 0.0) id = v;
      before += x;
      if (x > 0.0 && before > target) break;
    }
    s.id[0] = id;
  }
  __syncthreads();
  return s.id[0];
}

// k_verify_rows: a workgroup a row: the draft is taken or a token is drawn.
__global__ __launch_bounds__(kRowThreads) void k_verify_rows(VerifyArgs a) {
  __shared__ Shared s;
  const int m = blockIdx.x, V = a.V;
  if (a.cu && (m < a.cu[0] || m >= a.cu[a.n_seq])) return;  // uniform
  const Row p = read_row(a.logits + (size_t)m * V, V, a.tau, s);
  const int x = a.draft ? a.draft[m] : -1;
  const bool real = x >= 0 && x < V;
  int tok = -1;
  bool take = false;
  if (real) {
    const bool certain = a.draft_logits == nullptr;
    const Row q = certain ? Row{} : read_row(a.draft_logits + (size_t)m * V, V, a.draft_tau, s);
    auto q_of = [&](int v) { return certain ? (v == x ? 1.0 : 0.0) : q.prob(v); };
    take = (double)a.u[2 * m] * q_of(x) < p.prob(x);
    if (take) tok = x;
    else if (p.some) tok = pick(V, a.u[2 * m + 1], s, [&](int v) { return fmax(p.prob(v) - q_of(v), 0.0); });
  }
  if (tok < 0 && p.some)
    tok = p.sharp ? p.first : pick(V, a.draft ? a.u[2 * m + 1] : a.u[m], s, [&](int v) { return p.weight(v); });
  if (threadIdx.x == 0) {
    a.tokens[m] = tok;
    if (a.accepted) a.accepted[m] = take ? 1 : 0;
    if (a.conf) a.conf[m] = tok >= 0 ? p.weight(tok) / p.sum : 0.0;
  }
}

// k_verify_join: a wave a request: the drafts taken, and in a chain the rows after
// the first that takes none.
__global__ __launch_bounds__(64) void k_verify_join(VerifyArgs a) {
  const int s = blockIdx.x, lane = threadIdx.x;
  const int r0 = a.cu ? min(max(a.cu[s], 0), a.M) : 0, r1 = a.cu ? min(a.cu[s + 1], a.M) : a.M;
  int n = 0;
  bool ended = false;
  for (int b = r0; b < r1; b += 64) {
    const int m = b + lane;
    const bool in = m < r1, took = in && a.accepted[m];
    const uint64_t no = __builtin_amdgcn_ballot_w64(in && !took);
    const uint64_t yes = __builtin_amdgcn_ballot_w64(took);
    if (!a.chain) {
      n += (int)__popcll(yes);
      continue;
    }
    const int stop = no ? (int)__builtin_ctzll(no) : 64;  // the first row that takes none
    if (in && (ended || lane > stop)) {
      a.tokens[m] = -1;
      a.accepted[m] = 0;
      if (a.conf) a.conf[m] = 0.0;
    }
    if (!ended) n += stop;
    ended = ended || no;
  }
  if (a.chain && !ended) n = max(r1 - r0, 0);
  if (a.n_accepted && lane == 0) a.n_accepted[s] = n;
}

nmdlm_status launch_verify(const VerifyCall& c, hipStream_t st) {
  const VerifyArgs a{c.logits, c.draft_logits, c.draft, c.u, c.cu, c.M, c.V, c.n_seq, c.tau, c.draft_tau,
                     c.tokens, c.accepted, c.n_accepted, c.conf, !c.each};
  hipLaunchKernelGGL(k_verify_rows, dim3((unsigned)c.M), dim3(kRowThreads), 0, st, a);
  const nmdlm_status rc = hip_status();
  if (rc != NMDLM_OK || !c.draft || (c.each && !c.n_accepted)) return rc;
  hipLaunchKernelGGL(k_verify_join, dim3((unsigned)c.n_seq), dim3(64), 0, st, a);
  return hip_status();
}

}  // namespace nmdlm
