// Tokens drawn from logits and verification of drafted tokens: weights in
// float64, running sums in the order of the ids (the definitions: nmdlm.h).
//
// A row's ids go in parts of kPartIds, a wave each, so that one row fills many CUs
// and many rows stream through small workgroups without a barrier:
//   k_logit_parts  the largest logit of a part and the sum of its weights against it,
//                  of the target's rows and of the draft's: the logits' one full read
//   k_verify_left  (with drafts) whether a row's draft is taken; where not, the parts'
//                  sums of max(p - q, 0)
//   k_draw         the part in which the running sum passes the drawn number, then the
//                  id in it; and a request's count and end
// Every sum that decides is made in the same way by all waves that need it.
#include <math.h>

#include <algorithm>

#include "masked.h"

namespace nmdlm {

struct PartStat {
  float top;     // -inf: no weight
  int32_t first; // id of the largest
  double sum;    // of exp((l - top) / tau)
};

// A temperature's constants, from the host: a float64 division costs a wave more than the
// weights of its ids.
struct Temper {
  double inv, scale;  // 1 / tau (finite, so that 0 * inv is 0); 32 / (tau ln 2)
  bool sharp;         // temperature 0: weights at 1
};
static Temper temper(double tau) {
  // each rounded to 53 bits once: what the scale is off counts for an exponent of 700 that often
  const long double inv = tau == 0.0 ? 1.0L : std::min(1.0L / tau, 1e300L);
  return Temper{(double)inv, (double)(inv * 46.166241308446829035517589792L), tau == 0.0};
}

struct VerifyArgs {
  const float* logits;
  const float* draft_logits;
  const int32_t* draft;
  const float* u;
  const int32_t* cu;
  int M, V, n_seq, parts;
  Temper tau, draft_tau;
  int32_t* tokens;
  uint8_t* accepted;
  int32_t* n_accepted;
  double* conf;
  PartStat* p_stat;  // [M][parts]
  PartStat* q_stat;
  double* left;      // [M][parts]
  bool chain;
};

constexpr int kQuads = 4;                   // groups of four consecutive ids of a lane
constexpr int kPartIds = 64 * 4 * kQuads;
constexpr int kPartWaves = 4;               // of a workgroup
constexpr double kExpFloor = -700.0;        // exponents below weigh nothing

// 2^(j/32), correctly rounded
__device__ const double kPow[32] = {
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0,
    0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0,
    0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0,
    0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0,
    0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0,
    0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0,
};
__device__ __forceinline__ void fill_pow(double* pow) {
  if (threadIdx.x < 32) pow[threadIdx.x] = kPow[threadIdx.x];
}

// A row and where a lane's ids of it lie: group k of lane i of part w begins at id 1024 w +
// 4 (64 k + i) - shift, the target's groups 16-byte aligned; a wave reads runs of 1 KB.
struct RowAt {
  const float* l;
  int V, shift;
  bool vec;  // the groups are aligned
  __device__ __forceinline__ static int shift_of(const float* row) {
    return (int)((reinterpret_cast<uintptr_t>(row) >> 2) & 3);
  }
  __device__ __forceinline__ RowAt(const float* row, int V_, int shift_)
      : l(row), V(V_), shift(shift_), vec(shift_of(row) == shift_) {}
  __device__ __forceinline__ int id(int part, int k) const {
    return part * kPartIds + 4 * (64 * k + (int)(threadIdx.x & 63)) - shift;
  }
  // ids outside the row become -inf
  __device__ __forceinline__ void load(float (&x)[kQuads][4], int part) const {
    if (vec && part * kPartIds >= shift && (part + 1) * kPartIds - shift <= V) {  // uniform
#pragma unroll
      for (int k = 0; k < kQuads; ++k) {
        const float4 f = *reinterpret_cast<const float4*>(l + id(part, k));
        x[k][0] = f.x;
        x[k][1] = f.y;
        x[k][2] = f.z;
        x[k][3] = f.w;
      }
    } else {  // the row's first or last part, or a draft's row at another address
#pragma unroll
      for (int k = 0; k < kQuads; ++k) {
        const int v = id(part, k);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[k][e] = -INFINITY;
        if (vec && v >= 0 && v + 3 < V) {
          const float4 f = *reinterpret_cast<const float4*>(l + v);
          x[k][0] = f.x;
          x[k][1] = f.y;
          x[k][2] = f.z;
          x[k][3] = f.w;
        } else if (v + 3 >= 0 && v < V) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v + e >= 0 && v + e < V) x[k][e] = l[v + e];
        }
      }
    }
  }
  __device__ __forceinline__ float at(int v) const { return fmaxf(l[v], -INFINITY); }
};
__device__ __forceinline__ RowAt target_row(const VerifyArgs& a, int m) {
  const float* l = a.logits + (size_t)m * a.V;
  return RowAt(l, a.V, RowAt::shift_of(l));
}
// The draft's row (x: its draft) at the target's ids.
__device__ __forceinline__ RowAt draft_row(const VerifyArgs& a, int m, int x) {
  return RowAt(draft_logits_at(a.logits, a.draft_logits, m, a.V, x), a.V,
               RowAt::shift_of(a.logits + (size_t)m * a.V));
}
__device__ __forceinline__ bool row_counts(const VerifyArgs& a, int m) {
  return !a.cu || (m >= a.cu[0] && m < a.cu[a.n_seq]);
}

// The weights of a row.  exp(e), e = (x - top) / tau in [-700, 0], with t = 32 e / ln 2, n =
// round(t) and r = t - n: 2^(n/32) from a table of 32 powers, whose entries fill each
// LDS bank once (no conflicts), times exp(r ln 2 / 32) as 1 + r g(r), g the polynomial of
// degree 4 that meets (exp(r ln 2 / 32) - 1) / r at the five Chebyshev points of [-1/2, 1/2]
// (so exp(0) is 1).  Relative errors: the polynomial's 1.4e-16, its own rounding 0.9e-16, those
// of the power and of the product 2.3e-16, and the scale's rounding, 1.2e-16 |e|: together
// 4.6e-16 + 1.2e-16 |e|, of which the division of the definition has the second part too.
// With a degree less it was 7.9e-14 and one instruction fewer (1000 rows x 32000 drawn in
// 43.2 us, now 44.2).
// Float64 runs at the rate of float32 here, so it is the instructions that count, 18
// a weight.
struct Dist {
  float top;  // the largest
  double inv, scale;
  double sum;
  bool some, sharp, lift;  // any weight; temperature 0; the largest is +inf
  int first;               // id of the largest
  __device__ __forceinline__ explicit Dist(const Temper& t)
      : inv(t.inv), scale(t.scale), sum(0.0), sharp(t.sharp), first(0) {
    set_top(-INFINITY);
  }
  // with a largest of +inf these logits count as 0, the others as -inf
  __device__ __forceinline__ void set_top(float t) {
    some = t > -INFINITY;
    lift = t == INFINITY;
    top = lift ? 0.0f : t;
  }
  __device__ __forceinline__ float seen(float x) const {
    return !lift ? x : x == INFINITY ? 0.0f : -INFINITY;
  }
  template <bool CLEAN>  // CLEAN: the exponent is not below the floor
  __device__ __forceinline__ double weight_of(float x, const double* pow) const {
    constexpr double kMagic = 6755399441055744.0;  // 1.5 * 2^52: the sum's low bits are the integer
    const double y = (double)x - (double)top;
    const double big = __builtin_fma(y, scale, kMagic);
    const int n = (int)__double_as_longlong(big);
    const double r = __builtin_fma(y, scale, kMagic - big);
    double p = __builtin_fma(r, 0x1.5d884e708e6aap-35, 0x1.3b2b1bee88b09p-27);
    p = __builtin_fma(p, r, 0x1.c6b08d70400d0p-20);
    p = __builtin_fma(p, r, 0x1.ebfbdff8131c3p-13);
    p = __builtin_fma(p, r, 0x1.62e42fefa39efp-6);
    p = __builtin_fma(p, r, 1.0);
    p *= pow[n & 31];
    const long long b = __double_as_longlong(p);
    const double w = __longlong_as_double((long long)((int)(b >> 32) + ((n & ~31) << 15)) << 32 | (uint32_t)b);
    return CLEAN || y * inv >= kExpFloor ? w : 0.0;
  }
  __device__ __forceinline__ double weight(float x, const double* pow) const {
    return weight_of<false>(seen(x), pow);
  }
  // use(k, the weights of group k) for a lane's ids, four chains at a time: more would
  // take the registers of other waves
  template <bool CLEAN, typename U>
  __device__ __forceinline__ void each_group(const float (&x)[kQuads][4], const double* pow, U use) const {
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      double w[4] = {0.0, 0.0, 0.0, 0.0};
      // a group of ids past the row's end, or all ruled out, weighs nothing
      if (CLEAN || __builtin_amdgcn_ballot_w64(fmaxf(fmaxf(x[k][0], x[k][1]), fmaxf(x[k][2], x[k][3])) > -INFINITY)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = weight_of<CLEAN>(x[k][e], pow);
      }
      use(k, w);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  template <typename U>
  __device__ __forceinline__ void groups(float (&x)[kQuads][4], const double* pow, U use) const {
    float least = INFINITY;  // NaN where a logit is
    if (lift) {  // uniform
#pragma unroll
      for (int k = 0; k < kQuads; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[k][e] = seen(x[k][e]);
    }
#pragma unroll
    for (int k = 0; k < kQuads; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) least = __builtin_elementwise_minimum(least, x[k][e]);
    // the floor's own comparison, made for the least logit: in float64, since a float beside a
    // large logit may lie many exponents beside what it stands for
    const double e = ((double)least - (double)top) * inv;
    if (__builtin_amdgcn_ballot_w64(e >= kExpFloor) == ~0ull) each_group<true>(x, pow, use);
    else each_group<false>(x, pow, use);
  }
  __device__ __forceinline__ void weights(float (&x)[kQuads][4], double (&w)[kQuads][4], const double* pow) const {
    groups(x, pow, [&](int k, const double (&g)[4]) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[k][e] = g[e];
    });
  }
  __device__ __forceinline__ double weight_sum(float (&x)[kQuads][4], const double* pow) const {
    double sum = 0.0;
    groups(x, pow, [&](int, const double (&g)[4]) __attribute__((always_inline)) { sum += (g[0] + g[1]) + (g[2] + g[3]); });
    return sum;
  }
};

// Sums over the lanes, inclusive from the first.
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double x) {
  const long long b = __double_as_longlong(x);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, false);
  return x + __longlong_as_double((long long)hi << 32 | (uint32_t)lo);
}
__device__ __forceinline__ double lane_scan(double x) {
  x = dpp_add<0x111, 0xf>(x);  // row_shr 1, 2, 4, 8
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);     // row_bcast 15
  return dpp_add<0x143, 0xc>(x);  // row_bcast 31
}
__device__ __forceinline__ double read_lane(double x, int lane) {
  const long long b = __double_as_longlong(x);
  return __longlong_as_double((long long)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32 |
                              (uint32_t)__builtin_amdgcn_readlane((int)b, lane));
}
__device__ __forceinline__ double wave_total(double x) { return read_lane(lane_scan(x), 63); }
template <int CTRL>
__device__ __forceinline__ float dpp_max(float x) {
  return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), CTRL, 0xf, 0xf, false)));
}
__device__ __forceinline__ float wave_top(float x) {
  x = dpp_max<0x111>(x);
  x = dpp_max<0x112>(x);
  x = dpp_max<0x114>(x);
  x = dpp_max<0x118>(x);
  x = dpp_max<0x142>(x);
  x = dpp_max<0x143>(x);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ int wave_min(int x) {
  for (int o = 32; o > 0; o >>= 1) x = min(x, __shfl_xor(x, o));
  return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ double sum4(const double (&w)[4]) { return (w[0] + w[1]) + (w[2] + w[3]); }

// ---------------------------------------------------------------------------
// k_logit_parts: the parts of all rows, the target's and then the draft's, in runs to the
// waves; a wave's next part is on its way while it weighs one.  (With the parts in turn to
// the waves a wave met the same part of every row, and those of a row's last, partial one
// took 42 us where half of the others were through in 21: 1000 rows x 32000.)
//
// Bound by the float64 instructions, 18 a weight and 480 a part in all, beside the read:
// 1000 rows x 32000 39 us, 3.3 TB/s (the read without the weights 27 us).  Five waves a SIMD
// hold what they need in registers; with eight some was spilled (52 us).
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(64 * kPartWaves, 5) void k_logit_parts(VerifyArgs a) {
  __shared__ double pow[32];
  const int lane = threadIdx.x & 63, rows = a.draft_logits ? 2 * a.M : a.M;
  const int wave = blockIdx.x * kPartWaves + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int nwaves = gridDim.x * kPartWaves;
  const long long units = (long long)rows * a.parts;
  const int first_unit = (int)(units * wave / nwaves);  // fewer than 2^31 units
  int left = (int)(units * (wave + 1) / nwaves) - first_unit;
  int m = first_unit / a.parts, part = first_unit - m * a.parts;  // rows past M: the draft's
  // whether the row's parts are needed
  auto wanted = [&](int r) {
    const bool of_draft = r >= a.M;
    const int row = of_draft ? r - a.M : r;
    return row_counts(a, row) && !(of_draft && (uint32_t)a.draft[row] >= (uint32_t)a.V);
  };
  auto row_at = [&](int r) { return r >= a.M ? draft_row(a, r - a.M, a.draft[r - a.M]) : target_row(a, r); };
  float next[kQuads][4], x[kQuads][4];
  if (left > 0) row_at(m).load(next, part);  // whether it counts or not: asking takes as long
  bool here = left > 0 && wanted(m);
  fill_pow(pow);
  __syncthreads();
  for (; left > 0; --left) {  // wave-uniform
#pragma unroll
    for (int k = 0; k < kQuads; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[k][e] = next[k][e];
    const int at_m = m, at_part = part;
    const bool at_here = here;
    if (++part == a.parts) {
      part = 0;
      ++m;
    }
    here = left > 1 && wanted(m);
    if (here) row_at(m).load(next, part);
    if (!at_here) continue;
    float t = -INFINITY;  // NaN where a logit is
#pragma unroll
    for (int k = 0; k < kQuads; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) t = __builtin_elementwise_maximum(t, x[k][e]);
    if (__builtin_amdgcn_ballot_w64(t != t)) {  // wave-uniform, rare
      t = -INFINITY;
#pragma unroll
      for (int k = 0; k < kQuads; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) t = fmaxf(t, x[k][e]);
    }
    t = wave_top(t);
    Dist d(at_m >= a.M ? a.draft_tau : a.tau);
    d.set_top(t);
    int first = a.V;
    if (d.sharp) {  // uniform
      const RowAt row = row_at(at_m);
#pragma unroll
      for (int k = 0; k < kQuads; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (x[k][e] == t && d.some) first = min(first, row.id(at_part, k) + e);
      first = wave_min(first);
    }
    double sum = 0.0;
    if (d.some) {  // wave-uniform
      sum = d.weight_sum(x, pow);
      sum = lane_scan(sum);
    }
    if (lane == 63)
      (at_m >= a.M ? a.q_stat : a.p_stat)[(size_t)(at_m >= a.M ? at_m - a.M : at_m) * a.parts + at_part] =
          PartStat{t, first, sum};
  }
}

// A lane's part of the first 64 of a row: loaded early, before what it is for is known.
__device__ __forceinline__ PartStat lane_stat(const PartStat* st, int parts) {
  return st[min((int)(threadIdx.x & 63), parts - 1)];
}
// The row's distribution from its parts (mine: this lane's of the first 64); every lane
// gets it.
__device__ __forceinline__ Dist row_dist(const PartStat* st, PartStat mine, int parts, const Temper& tau,
                                         const double* pow) {
  const int lane = threadIdx.x & 63;
  Dist d(tau);
  if (lane >= parts) mine = PartStat{-INFINITY, INT32_MAX, 0.0};
  float top = mine.top;
  for (int i = lane + 64; i < parts; i += 64) top = fmaxf(top, st[i].top);
  top = wave_top(top);
  d.set_top(top);
  double sum = mine.sum * d.weight(mine.top, pow);
  int first = mine.top == top ? mine.first : INT32_MAX;
  for (int i = lane + 64; i < parts; i += 64) {
    const PartStat s = st[i];
    sum += s.sum * d.weight(s.top, pow);
    if (s.top == top) first = min(first, s.first);
  }
  d.sum = wave_total(sum);
  if (d.sharp) d.first = wave_min(first);
  return d;
}

// The logits of a part of a row, the target's and the draft's.
struct Logits {
  float p[kQuads][4], q[kQuads][4];
  __device__ __forceinline__ void load(const VerifyArgs& a, int m, int x, int part) {
    target_row(a, m).load(p, part);
    if (a.draft_logits) draft_row(a, m, x).load(q, part);
  }
};

// The target's and the draft's distribution of a row with a draft x.
struct Pair {
  Dist p, q;
  int x;
  bool certain;  // q is 1 at x
  __device__ __forceinline__ Pair(const VerifyArgs& a, int m, int x_, const Dist& p_, PartStat mine_q, const double* pow)
      : p(p_), q(a.draft_tau), x(x_), certain(!a.draft_logits) {
    if (!certain) q = row_dist(a.q_stat + (size_t)m * a.parts, mine_q, a.parts, a.draft_tau, pow);
  }
  // max(p - q, 0) of a part's ids
  __device__ __forceinline__ void left(const RowAt& row, int part, Logits& l, double (&w)[kQuads][4],
                                       const double* pow) const {
    // each product rounded by itself: of equal distributions nothing is left, and the part's sum
    // and its weights come out alike in both kernels
#pragma clang fp contract(off)
    auto &lp = l.p, &lq = l.q;
    double y[kQuads][4];
    if (p.sharp) {
#pragma unroll
      for (int k = 0; k < kQuads; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) w[k][e] = row.id(part, k) + e == p.first ? 1.0 : 0.0;
    } else {
      const double ip = 1.0 / p.sum;
      p.weights(lp, w, pow);
#pragma unroll
      for (int k = 0; k < kQuads; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) w[k][e] *= ip;
    }
    if (certain || q.sharp || !q.some) {
      const int at = certain ? x : q.some ? q.first : INT32_MIN;
#pragma unroll
      for (int k = 0; k < kQuads; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[k][e] = row.id(part, k) + e == at ? 1.0 : 0.0;
    } else {
      const double iq = 1.0 / q.sum;
      q.weights(lq, y, pow);
#pragma unroll
      for (int k = 0; k < kQuads; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[k][e] *= iq;
    }
#pragma unroll
    for (int k = 0; k < kQuads; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) w[k][e] = fmax(w[k][e] - y[k][e], 0.0);
  }
};

// ---------------------------------------------------------------------------
// k_verify_left: grid (waves of a row / 4, rows).  Each wave decides on its row's draft for
// itself; the first writes what was decided.  (With the logits of the wave's first part on
// their way meanwhile, 372 rows took 62 us against 58: most rows do not need them.)  372
// rows x 32000: 17 us; few rows, 6 us, are a chain of trips to memory.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(64 * kPartWaves) void k_verify_left(VerifyArgs a) {
  __shared__ double pow[32];
  const int m = blockIdx.y, lane = threadIdx.x & 63, step = gridDim.x * kPartWaves;
  int part = blockIdx.x * kPartWaves + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  // the loads leave before what they are for is known: each wait is a trip to memory, since
  // another die wrote the sums
  const PartStat* const p_stat = a.p_stat + (size_t)m * a.parts;
  const PartStat mine_p = lane_stat(p_stat, a.parts);
  const PartStat mine_q = a.draft_logits ? lane_stat(a.q_stat + (size_t)m * a.parts, a.parts) : mine_p;
  const int x = a.draft[m], at = min(max(x, 0), a.V - 1);
  const float u = a.u[2 * m];
  const RowAt row = target_row(a, m);
  const float px = row.at(at), qx = a.draft_logits ? draft_row(a, m, x).at(at) : 0.0f;
  fill_pow(pow);
  if (!row_counts(a, m)) return;  // uniform
  if ((uint32_t)x >= (uint32_t)a.V) {
    if (part == 0 && lane == 0) a.accepted[m] = 0;
    return;
  }
  __syncthreads();
  if (part >= a.parts) return;
  const Pair d(a, m, x, row_dist(p_stat, mine_p, a.parts, a.tau, pow), mine_q, pow);
  const Dist &p = d.p, &q = d.q;
  bool take = false;
  double prob = 0.0;
  if (p.some) {
    prob = p.weight(px, pow) / p.sum;
    const double pr = p.sharp ? (x == p.first ? 1.0 : 0.0) : prob;
    double qr = 1.0;
    if (!d.certain) qr = !q.some ? 0.0 : q.sharp ? (x == q.first ? 1.0 : 0.0) : q.weight(qx, pow) / q.sum;
    take = (double)u * qr < pr;
  }
  if (part == 0 && lane == 0) {
    a.accepted[m] = take ? 1 : 0;
    if (take) {
      a.tokens[m] = x;
      if (a.conf) a.conf[m] = prob;
    }
  }
  if (take || !p.some) return;
  for (; part < a.parts; part += step) {
    Logits l;
    l.load(a, m, x, part);
    double w[kQuads][4], sum = 0.0;
    d.left(row, part, l, w, pow);
#pragma unroll
    for (int k = 0; k < kQuads; ++k) sum += sum4(w[k]);
    sum = lane_scan(sum);
    if (lane == 63) a.left[(size_t)m * a.parts + part] = sum;
  }
}

// First part whose running sum exceeds u times the sum of all (the last of positive sum
// when none does), and the running sum before it.  of(i): part i's sum.
struct Spot {
  int part;
  double before, target, total;
};
template <typename F>
__device__ __forceinline__ Spot find_part(int parts, float u, F of) {
  const int lane = threadIdx.x & 63;
  double x = lane < parts ? of(lane) : 0.0, in = lane_scan(x);
  Spot s{-1, 0.0, 0.0, read_lane(in, 63)};
  for (int b = 64; b < parts; b += 64) s.total += wave_total(b + lane < parts ? of(b + lane) : 0.0);
  // 1 and beyond: no sum exceeds it
  s.target = u < 1.0f ? (double)u * s.total : INFINITY;
  double run = 0.0;
  for (int b = 0; b < parts; b += 64) {  // uniform
    if (b > 0) {
      x = b + lane < parts ? of(b + lane) : 0.0;
      in = lane_scan(x);
    }
    const uint64_t some = __builtin_amdgcn_ballot_w64(x > 0.0);
    const uint64_t over = __builtin_amdgcn_ballot_w64(x > 0.0 && run + in > s.target);
    if (some) {
      const int L = over ? (int)__builtin_ctzll(over) : 63 - (int)__builtin_clzll(some);
      s.part = b + L;
      s.before = run + (read_lane(in, L) - read_lane(x, L));
      if (over) break;
    }
    run += read_lane(in, 63);
  }
  return s;
}
// The id in the spot's part, from the weights of its ids, and the target's logit there;
// every lane gets them.
struct Token {
  int id;
  float logit;  // as Dist::seen has it
};
__device__ __forceinline__ Token find_id(const Spot& s, const double (&w)[kQuads][4], const float (&l)[kQuads][4],
                                         const RowAt& row) {
  Token t{-1, -INFINITY};
  double run = s.before;
#pragma unroll
  for (int k = 0; k < kQuads; ++k) {
    const double x = sum4(w[k]), in = lane_scan(x);
    const uint64_t some = __builtin_amdgcn_ballot_w64(x > 0.0);
    const uint64_t over = __builtin_amdgcn_ballot_w64(x > 0.0 && run + in > s.target);
    if (some) {  // uniform
      const int L = over ? (int)__builtin_ctzll(over) : 63 - (int)__builtin_clzll(some);
      double r = run + (in - x);
      Token mine{-1, -INFINITY};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool past = mine.id >= 0 && r > s.target;
        if (!past && w[k][e] > 0.0) mine = Token{row.id(s.part, k) + e, l[k][e]};
        r += past ? 0.0 : w[k][e];
      }
      t.id = __builtin_amdgcn_readlane(mine.id, L);
      t.logit = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine.logit), L));
      if (over) return t;
    }
    run += read_lane(in, 63);
  }
  return t;
}

// ---------------------------------------------------------------------------
// k_draw: a wave a row that has no token yet, then one a request for its count.  In a
// chain a row that follows one without an accepted draft is void.  (A void row's flag
// is cleared while later rows look: they are void by the earlier row's, which stays.)
// 5 to 8.4 us: a chain of trips to memory, stats, the part's logits, a token.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(64) void k_draw(VerifyArgs a) {
  __shared__ double pow[32];
  const int lane = threadIdx.x;
  if ((int)blockIdx.x >= a.M) {  // a request's count
    const int s = blockIdx.x - a.M;
    const int r0 = a.cu ? min(max(a.cu[s], 0), a.M) : 0, r1 = a.cu ? min(a.cu[s + 1], a.M) : a.M;
    int n = 0;
    for (int b = r0; b < r1; b += 64) {
      const uint64_t there = r1 - b >= 64 ? ~0ull : (1ull << (r1 - b)) - 1;
      const uint64_t yes = __builtin_amdgcn_ballot_w64(b + lane < r1 && a.accepted[b + lane]), no = there & ~yes;
      if (a.chain && no) {
        n += (int)__builtin_ctzll(no);
        break;
      }
      n += (int)__popcll(yes);
    }
    if (lane == 0) a.n_accepted[s] = n;
    return;
  }
  const int m = blockIdx.x;
  // the loads leave before what they are for is known
  const PartStat* const st = a.p_stat + (size_t)m * a.parts;
  const double* const left = a.draft ? a.left + (size_t)m * a.parts : nullptr;
  const PartStat mine_p = lane_stat(st, a.parts);
  const PartStat mine_q = a.draft_logits ? lane_stat(a.q_stat + (size_t)m * a.parts, a.parts) : mine_p;
  const double mine_left = left ? left[min(lane, a.parts - 1)] : 0.0;
  const int x = a.draft ? a.draft[m] : -1;
  const float u = a.draft ? a.u[2 * m + 1] : a.tau.sharp ? 0.0f : a.u[m];
  const bool taken = a.accepted && a.accepted[m];
  fill_pow(pow);
  if (!row_counts(a, m)) return;
  if (a.chain) {
    int r0 = 0;
    if (a.cu) {  // where the last request begins that begins at or before the row: 64 probes at once
      for (int lo = 0, n = a.n_seq; n > 0;) {  // among cu[lo], ..., cu[lo + n - 1]; cu[0] is one
        const int gap = (n + 63) / 64, i = lo + lane * gap;
        const int c = a.cu[min(i, lo + n - 1)];
        const uint64_t at = __builtin_amdgcn_ballot_w64(i < lo + n && c <= m);
        const int L = at ? 63 - (int)__builtin_clzll(at) : 0;
        r0 = max(__builtin_amdgcn_readlane(c, L), 0);
        n = min(gap - 1, lo + n - 1 - (lo + L * gap));
        lo += L * gap + 1;
        if (n > 0 && a.cu[lo] > m) break;  // none of the rest
      }
    }
    bool ended = false;
    for (int b = r0; b < m && !ended; b += 64)
      ended = __builtin_amdgcn_ballot_w64(b + lane < m && !a.accepted[b + lane]) != 0;
    if (ended) {
      if (lane == 0) {
        a.tokens[m] = -1;
        a.accepted[m] = 0;
        if (a.conf) a.conf[m] = 0.0;
      }
      return;
    }
  }
  if (taken) return;
  __syncthreads();
  const bool real = (uint32_t)x < (uint32_t)a.V;
  const RowAt row = target_row(a, m);
  const Dist p = row_dist(st, mine_p, a.parts, a.tau, pow);
  Token tok{-1, 0.0f};
  if (p.some) {
    double w[kQuads][4];
    if (real) {
      const Spot s = find_part(a.parts, u, [&](int i) { return i < 64 ? mine_left : left[i]; });
      if (s.total > 0.0) {
        Logits l;
        l.load(a, m, x, s.part);
        const Pair d(a, m, x, p, mine_q, pow);
        d.left(row, s.part, l, w, pow);
        tok = find_id(s, w, l.p, row);
        if (p.sharp) tok.logit = p.seen(tok.logit);  // else weighing has made it so
      }
    }
    if (tok.id < 0 && p.sharp) tok = Token{p.first, p.seen(row.at(p.first))};
    if (tok.id < 0) {
      const Spot s = find_part(a.parts, u, [&](int i) {
        const PartStat t = i < 64 ? mine_p : st[i];
        return t.sum * p.weight(t.top, pow);
      });
      float l[kQuads][4];
      row.load(l, s.part);
      p.weights(l, w, pow);
      tok = find_id(s, w, l, row);
    }
  }
  if (lane == 0) {
    a.tokens[m] = tok.id;
    if (a.conf) a.conf[m] = tok.id >= 0 ? p.weight_of<false>(tok.logit, pow) / p.sum : 0.0;
  }
}

constexpr int kPartWgs = 1280;     // five waves a SIMD
constexpr int kLeftWaves = 4096;
static int parts_of(int V) { return (V + 3 + kPartIds - 1) / kPartIds; }  // with up to 3 ids before the row

size_t verify_ws(int M, int V, bool drafts) {
  const size_t n = (size_t)M * parts_of(V);
  return align_up(n * sizeof(PartStat), 256) * (drafts ? 2 : 1) + (drafts ? align_up(n * sizeof(double), 256) : 0);
}

nmdlm_status launch_verify(const VerifyCall& c, hipStream_t st) {
  const int parts = parts_of(c.V);
  const size_t n = (size_t)c.M * parts;
  Carver cv{static_cast<char*>(c.ws), 0, (size_t)-1, true};
  PartStat* const p_stat = cv.take<PartStat>(n);
  PartStat* const q_stat = c.draft ? cv.take<PartStat>(n) : nullptr;
  double* const left = c.draft ? cv.take<double>(n) : nullptr;
  const VerifyArgs a{c.logits, c.draft_logits, c.draft, c.u, c.cu, c.M, c.V, c.n_seq, parts, temper(c.tau), temper(c.draft_tau),
                     c.tokens, c.accepted, c.n_accepted, c.conf, p_stat, q_stat, left, c.draft && !c.each};
  // waves to fill the chip once, a few parts each where there are more
  const long long units = (long long)n * (c.draft_logits ? 2 : 1);
  if (units > INT32_MAX) return NMDLM_ERR_UNSUPPORTED;
  const unsigned wgs = (unsigned)std::min<long long>((units + kPartWaves - 1) / kPartWaves, kPartWgs);
  hipLaunchKernelGGL(k_logit_parts, dim3(wgs), dim3(64 * kPartWaves), 0, st, a);
  nmdlm_status rc = hip_status();
  if (rc != NMDLM_OK) return rc;
  if (c.draft) {
    const int each = (int)std::min<long long>(std::max<long long>(n / kLeftWaves, 1), parts);
    const unsigned row_wgs = (parts + each * kPartWaves - 1) / (each * kPartWaves);
    hipLaunchKernelGGL(k_verify_left, dim3(row_wgs, c.M), dim3(64 * kPartWaves), 0, st, a);
    if ((rc = hip_status()) != NMDLM_OK) return rc;
  }
  hipLaunchKernelGGL(k_draw, dim3((unsigned)c.M + (c.n_accepted ? c.n_seq : 0)), dim3(64), 0, st, a);
  return hip_status();
}

}  // namespace nmdlm
