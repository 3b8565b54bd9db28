// Tokens drawn from logits and verification of drafted tokens: weights in
// float64, running sums in the order of the ids (the definitions: nmdlm.h).
#include <float.h>
#include <math.h>

#include <type_traits>

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

// ---------------------------------------------------------------------------
// A workgroup takes a row (of the target, and of the draft): a thread holds
// kQuads groups of four consecutive logits in registers, group k of thread i being
// ids 4 (k nth + i) on, less the row's offset from a 16-byte address, so that a
// wave reads 1 KB runs.  Up to kQuads * 4 * 1024 ids the row is read once; longer rows go
// in tiles of that size and are read again for each step.
// ---------------------------------------------------------------------------
constexpr int kQuads = 8;
constexpr int kMaxThreads = 1024;
constexpr int kSegs = kQuads * kMaxThreads / 16;  // of 64 ids: the sums of 16 lanes
constexpr int kMaxTiles = NMDLM_MAX_SAMPLE_V / (kQuads * 4 * kMaxThreads) + 1;
constexpr double kExpFloor = -700.0;  // exponents below weigh nothing

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

struct Quads {
  float x[kQuads][4];
};

struct RowShared {
  double seg[kSegs];
  double tile[kMaxTiles];
  double part[2][kMaxThreads / 16];
  double pow[32];  // 2^(j/32)
  float top[2][kMaxThreads / 64];
  int first[kMaxThreads / 64];
};

// A row and where a thread's groups of it lie: the target's from the 16-byte address
// at or before the row on, the draft's the same ids.
struct RowAt {
  const float* l;
  int V, shift;  // ids before the row's first
  bool vec;      // the groups are 16-byte aligned
  __device__ __forceinline__ static int shift_of(const float* row) {
    return (int)((reinterpret_cast<uintptr_t>(row) >> 2) & 3);
  }
  __device__ __forceinline__ RowAt(const float* row, int V_, int shift_)
      : l(row), V(V_), shift(shift_), vec(shift_of(row) == shift_) {}
  __device__ __forceinline__ int tile_ids() const { return kQuads * 4 * blockDim.x; }
  __device__ __forceinline__ int tiles() const { return (V + shift + tile_ids() - 1) / tile_ids(); }
  __device__ __forceinline__ int id(int tile, int k) const {
    return tile * tile_ids() + 4 * (int)(k * blockDim.x + threadIdx.x) - shift;
  }
  // any id of the workgroup in group k
  __device__ __forceinline__ bool has(int tile, int k) const {
    return tile * tile_ids() + 4 * (int)(k * blockDim.x) - shift < V;
  }
  // NaN and ids outside the row become -inf
  __device__ __forceinline__ void load(Quads& q, int tile) const {
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      const int v = id(tile, k);
      if (vec && v >= 0 && v + 3 < V) {
        const float4 f = *reinterpret_cast<const float4*>(l + v);
        q.x[k][0] = f.x;
        q.x[k][1] = f.y;
        q.x[k][2] = f.z;
        q.x[k][3] = f.w;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) q.x[k][e] = v + e >= 0 && v + e < V ? l[v + e] : -INFINITY;
      }
    }
#pragma unroll
    for (int k = 0; k < kQuads; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) q.x[k][e] = fmaxf(q.x[k][e], -INFINITY);
  }
};

// The weights of a row.  exp(e), e = (x - top) / tau in [-700, 0], with t = 32 e / ln 2, n =
// round(t) and r = t - n: 2^(n/32) from a table of 32 powers, whose entries fill each
// LDS bank once (no conflicts), times exp(r ln 2 / 32) by the polynomial of degree 4
// that meets it at the five Chebyshev points of [-1/2, 1/2] (0 is one: exp(0) is 1).  Its
// relative error, 7.9e-14, is 2^-43: a running sum errs by less than what decides
// between two ids in one draw of 10^9.  Float64 runs at the rate of float32 here, so
// it is the instructions that count, 17 a weight.
struct Dist {
  float top, cut;    // the largest; below cut an exponent may be below -700
  double inv, scale;  // 1 / tau; 32 / (tau ln 2)
  double sum;
  bool some, sharp, lift;  // any weight; temperature 0; the largest is +inf
  int first;               // id of the largest (temperature 0 only)
  __device__ __forceinline__ void init(double tau) {
    sharp = tau == 0.0;
    inv = sharp ? 1.0 : fmin(1.0 / tau, 1e300);  // finite, so that 0 * inv is 0
    scale = inv * 46.16624130844683;
    top = -INFINITY;
    sum = 0.0;
    first = 0;
  }
  // top is known: with a largest of +inf these logits count as 0, the others as -inf
  __device__ __forceinline__ void set_top() {
    some = top > -INFINITY;
    lift = top == INFINITY;
    if (lift) top = 0.0f;
    cut = fmaxf((float)((double)top - 690.0 / inv), -FLT_MAX);
  }
  __device__ __forceinline__ float lifted(float x) const { return x == INFINITY ? 0.0f : -INFINITY; }
  // CLEAN: none below cut
  template <bool CLEAN>
  __device__ __forceinline__ double weight(float x, const double* pow) const {
    constexpr double kMagic = 6755399441055744.0;  // 1.5 * 2^52: the sum's low bits are the integer
    const double y = (double)x - (double)top;
    const double big = __builtin_fma(y, scale, kMagic);
    const int n = (int)__double_as_longlong(big);
    const double r = __builtin_fma(y, scale, kMagic - big);
    double p = __builtin_fma(r, 0x1.3b2b1bee88b09p-27, 0x1.c6b167e571135p-20);
    p = __builtin_fma(p, r, 0x1.ebfbdff8131c3p-13);
    p = __builtin_fma(p, r, 0x1.62e42fef6d01ap-6);
    p = __builtin_fma(p, r, 1.0);
    p *= pow[n & 31];
    const long long b = __double_as_longlong(p);
    const double w = __longlong_as_double((long long)((int)(b >> 32) + ((n & ~31) << 15)) << 32 | (uint32_t)b);
    return CLEAN || y * inv >= kExpFloor ? w : 0.0;
  }
  template <bool CLEAN>
  __device__ __forceinline__ void weights(const float (&x)[4], double (&w)[4], const double* pow) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = weight<CLEAN>(x[e], pow);
  }
};

// Sums over the 16 lanes of a row of lanes, inclusive from its first lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double x) {
  const long long b = __double_as_longlong(x);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, false);
  return x + __longlong_as_double((long long)hi << 32 | (uint32_t)lo);
}
__device__ __forceinline__ double row_scan(double x) {
  x = dpp_add<0x111, 0xf>(x);  // row_shr 1, 2, 4, 8
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  return dpp_add<0x118, 0xf>(x);
}
__device__ __forceinline__ double lane_scan(double x) {
  x = row_scan(x);
  x = dpp_add<0x142, 0xa>(x);    // row_bcast 15
  return dpp_add<0x143, 0xc>(x);  // row_bcast 31
}
__device__ __forceinline__ double read_lane(double x, int lane) {
  const long long b = __double_as_longlong(x);
  return __longlong_as_double((long long)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32 |
                              (uint32_t)__builtin_amdgcn_readlane((int)b, lane));
}

__device__ __forceinline__ float thread_top(const Quads& q) {
  float t = -INFINITY;
#pragma unroll
  for (int k = 0; k < kQuads; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) t = fmaxf(t, q.x[k][e]);
  return t;
}
// none of the wave's logits is below the cut
__device__ __forceinline__ bool wave_clean(const Quads& q, float cut) {
  float t = INFINITY;
#pragma unroll
  for (int k = 0; k < kQuads; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) t = fminf(t, q.x[k][e]);
  return __builtin_amdgcn_ballot_w64(t >= cut) == ~0ull;
}
__device__ __forceinline__ void lift_all(Quads& q, const Dist& d) {
#pragma unroll
  for (int k = 0; k < kQuads; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) q.x[k][e] = d.lifted(q.x[k][e]);
}
// Keeps the compiler from carrying what it made of the logits in one pass into the next:
// the weights of a row would take 128 registers.
__device__ __forceinline__ void renew(Quads& q) {
#pragma unroll
  for (int k = 0; k < kQuads; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) asm("" : "+v"(q.x[k][e]));
}
__device__ __forceinline__ float wave_top(float t) {
  for (int o = 32; o > 0; o >>= 1) t = fmaxf(t, __shfl_xor(t, o));
  return t;
}

// Where the running sum of a tile passes a target: a segment of 64 ids (16 lanes of
// wave `wave`, group k), the sum before it, found by every wave alike.
struct Spot {
  int k, wave, lanes;
  double before;
};

// A tile's segments: the sums of 16 lanes' groups of four ids, by group, wave and
// lanes, which is the order of the ids.  w4(k, out) gives the weights of the thread's
// group k.  All threads; two barriers.  The sums then lie in LDS such that lane i of
// a wave reads segments i n .. i n + n - 1 (n = a 64th of them) without conflicts.
template <typename W>
__device__ __forceinline__ void fill_segments(RowShared& s, const RowAt& at, int tile, W w4) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rows = blockDim.x / 16;
  const int per = kQuads * rows / 64;
  __syncthreads();  // the segments before are read
#pragma unroll
  for (int k = 0; k < kQuads; ++k) {
    double x = 0.0;
    if (at.has(tile, k)) {  // uniform
      double w[4];
      w4(k, w);
      x = row_scan((w[0] + w[1]) + (w[2] + w[3]));
      __builtin_amdgcn_sched_barrier(0);
    }
    const int seg = k * rows + wave * 4 + (lane >> 4);
    if ((lane & 15) == 15) s.seg[(seg % per) * 64 + seg / per] = x;
  }
  __syncthreads();
}
// The sum of the tile's segments; pre: that of the lanes before.
__device__ __forceinline__ double segment_sum(const RowShared& s, double& pre) {
  const int lane = threadIdx.x & 63, per = kQuads * (blockDim.x / 16) / 64;
  double x = 0.0;
  for (int i = 0; i < per; ++i) x += s.seg[i * 64 + lane];
  const double in = lane_scan(x);
  pre = in - x;
  return read_lane(in, 63);
}
// First segment whose running sum, from `before` on, exceeds the target; the last of
// positive sum when none does.
__device__ __forceinline__ Spot find_segment(const RowShared& s, double before, double target) {
  const int lane = threadIdx.x & 63, rows = blockDim.x / 16, per = kQuads * rows / 64;
  double x = 0.0;
  for (int i = 0; i < per; ++i) x += s.seg[i * 64 + lane];
  const double in = lane_scan(x);
  double run = before + __shfl_up(in, 1);
  if (lane == 0) run = before;
  int over = -1, last = -1;
  double run_over = 0.0, run_last = 0.0;
  for (int i = 0; i < per; ++i) {
    const double y = s.seg[i * 64 + lane];
    if (y > 0.0) {
      last = i;
      run_last = run;
      if (over < 0 && run + y > target) {
        over = i;
        run_over = run;
      }
    }
    run += y;
  }
  const uint64_t has_over = __builtin_amdgcn_ballot_w64(over >= 0), has_last = __builtin_amdgcn_ballot_w64(last >= 0);
  const int L = has_over ? (int)__builtin_ctzll(has_over) : 63 - (int)__builtin_clzll(has_last | 1ull);
  const int i = __builtin_amdgcn_readlane(has_over ? over : max(last, 0), L);
  const int seg = L * per + i;
  return Spot{seg / rows, (seg % rows) / 4, seg % 4, read_lane(has_over ? run_over : run_last, L)};
}
// In the spot's wave: the lane that holds the token returns its id, the others -1.
template <typename W>
__device__ __forceinline__ int find_id(const Spot& sp, double target, const RowAt& at, int tile, W w4) {
  const int lane = threadIdx.x & 63;
  double w[4];
  w4(sp.k, w);
  const double x = (w[0] + w[1]) + (w[2] + w[3]);
  const double in = row_scan(x);
  const bool mine = (lane >> 4) == sp.lanes;
  const uint64_t over = __builtin_amdgcn_ballot_w64(mine && x > 0.0 && sp.before + in > target);
  const uint64_t some = __builtin_amdgcn_ballot_w64(mine && x > 0.0);
  const int L = over ? (int)__builtin_ctzll(over) : 63 - (int)__builtin_clzll(some | 1ull);
  if (lane != L) return -1;
  double run = sp.before + (in - x);
  int id = -1;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool past = id >= 0 && run > target;
    if (!past && w[e] > 0.0) id = at.id(tile, sp.k) + e;
    run += past ? 0.0 : w[e];
  }
  return id;
}

// Group k of the registers, k uniform.
__device__ __forceinline__ void take_group(const Quads& q, int k, float (&x)[4]) {
#pragma unroll
  for (int j = 0; j < kQuads; ++j)
    if (j == k) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = q.x[j][e];
    }
}

__device__ __forceinline__ double weight_at(const Dist& d, const RowAt& at, int id, const double* pow) {
  const float x = fmaxf(at.l[id], -INFINITY);
  return d.weight<false>(d.lift ? d.lifted(x) : x, pow);
}

// ---------------------------------------------------------------------------
// k_verify_rows: a workgroup a row: its draft is taken or a token is drawn.  DRAFT:
// with drafts; ONE: the row fits the registers.
// ---------------------------------------------------------------------------
template <bool DRAFT, bool ONE>
__global__ __launch_bounds__(kMaxThreads) void k_verify_rows(VerifyArgs a) {
  __shared__ RowShared s;
  const int m = blockIdx.x, V = a.V, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int nwaves = blockDim.x / 64;
  if (a.cu && (m < a.cu[0] || m >= a.cu[a.n_seq])) return;  // uniform
  const float* const row = a.logits + (size_t)m * V;
  const RowAt pa(row, V, RowAt::shift_of(row));
  const int x = DRAFT ? a.draft[m] : -1;
  const bool real = x >= 0 && x < V, has_q = DRAFT && real && a.draft_logits;
  const RowAt qa(has_q ? a.draft_logits + (size_t)m * V : row, V, pa.shift);
  const int tiles = ONE ? 1 : pa.tiles();
  Quads P, Q = {};
  const double* pow = s.pow;
  if (tid < 32) s.pow[tid] = kPow[tid];

  // the largest
  Dist p, q;
  p.init(a.tau);
  q.init(a.draft_tau);
  for (int t = 0; t < tiles; ++t) {
    pa.load(P, t);
    if (has_q) qa.load(Q, t);
    p.top = fmaxf(p.top, thread_top(P));
    if (has_q) q.top = fmaxf(q.top, thread_top(Q));
  }
  p.top = wave_top(p.top);
  if (DRAFT) q.top = wave_top(q.top);
  if (lane == 0) {
    s.top[0][wave] = p.top;
    s.top[1][wave] = q.top;
  }
  __syncthreads();
  for (int i = 0; i < nwaves; ++i) {
    p.top = fmaxf(p.top, s.top[0][i]);
    q.top = fmaxf(q.top, s.top[1][i]);
  }
  p.set_top();
  q.set_top();
  // a tile of the row (and its draft's) into registers; with ONE it is there
  bool clean_p = false, clean_q = false;  // of the wave
  auto lift_tile = [&]() __attribute__((always_inline)) {
    if (p.lift) lift_all(P, p);
    if (has_q && q.lift) lift_all(Q, q);
    clean_p = wave_clean(P, p.cut);
    if (has_q) clean_q = wave_clean(Q, q.cut);
  };
  auto tile = [&](int t) __attribute__((always_inline)) {
    if (ONE) {
      renew(P);
      if (DRAFT) renew(Q);
      return;
    }
    pa.load(P, t);
    if (has_q) qa.load(Q, t);
    lift_tile();
  };
  if (ONE) lift_tile();

  // at temperature 0, the first of the largest
  auto first_id = [&](Dist& d, const Quads& r) __attribute__((always_inline)) {
    int id = V;
    for (int t = 0; t < tiles; ++t) {
      tile(t);
#pragma unroll
      for (int k = 0; k < kQuads; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (r.x[k][e] == d.top && d.some) id = min(id, pa.id(t, k) + e);
    }
    for (int o = 32; o > 0; o >>= 1) id = min(id, __shfl_xor(id, o));
    __syncthreads();
    if (lane == 0) s.first[wave] = id;
    __syncthreads();
    for (int i = 0; i < nwaves; ++i) id = min(id, s.first[i]);
    d.first = id;
  };
  if (p.sharp) first_id(p, P);
  if (has_q && q.sharp) first_id(q, Q);

  // the sums of the weights
  auto thread_sum = [&](auto clean, const Dist& d, const Quads& r, int t) __attribute__((always_inline)) {
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kQuads; ++k)
      if (pa.has(t, k)) {  // uniform
        double w[4];
        d.template weights<decltype(clean)::value>(r.x[k], w, pow);
        sum += (w[0] + w[1]) + (w[2] + w[3]);
        __builtin_amdgcn_sched_barrier(0);  // four chains at a time: more would spill the rows
      }
    return sum;
  };
  auto tile_sum = [&](bool clean, const Dist& d, const Quads& r, int t) __attribute__((always_inline)) {
    return clean ? thread_sum(std::true_type{}, d, r, t) : thread_sum(std::false_type{}, d, r, t);
  };
  int tok = -1;
  bool take = false, mine = tid == 0;  // the thread that writes
  if (real && p.some) {
    double wp = 0.0, wq = 0.0;
    for (int t = 0; t < tiles; ++t) {
      tile(t);
      wp += tile_sum(clean_p, p, P, t);
      if (has_q && q.some) wq += tile_sum(clean_q, q, Q, t);
    }
    wp = row_scan(wp);
    wq = row_scan(wq);
    if ((lane & 15) == 15) {
      s.part[0][tid >> 4] = wp;
      s.part[1][tid >> 4] = wq;
    }
    __syncthreads();
    p.sum = read_lane(lane_scan(lane < nwaves * 4 ? s.part[0][lane] : 0.0), 63);
    q.sum = read_lane(lane_scan(lane < nwaves * 4 ? s.part[1][lane] : 0.0), 63);
    const double pr = p.sharp ? (x == p.first ? 1.0 : 0.0) : weight_at(p, pa, x, pow) / p.sum;
    double qr = 1.0;
    if (has_q) qr = !q.some ? 0.0 : q.sharp ? (x == q.first ? 1.0 : 0.0) : weight_at(q, qa, x, pow) / q.sum;
    take = (double)a.u[2 * m] * qr < pr;
    if (take) tok = x;
  }

  // a token: from max(p - q, 0) where a draft was refused, else from p
  if (!take && p.some) {
    const float u = DRAFT ? a.u[2 * m + 1] : (p.sharp ? 0.0f : a.u[m]);
    // draws from the weights w4(k, tile, out) of all tiles: false when they sum to 0
    auto draw = [&](auto w4, double& total) __attribute__((always_inline)) {
      int at = 0;
      double before = 0.0, pre;
      if (ONE) {
        tile(0);
        fill_segments(s, pa, 0, [&](int k, double (&w)[4]) __attribute__((always_inline)) { w4(k, 0, w); });
        total = segment_sum(s, pre);
      } else {
        total = 0.0;
        int last = 0;
        for (int t = 0; t < tiles; ++t) {
          tile(t);
          fill_segments(s, pa, t, [&](int k, double (&w)[4]) __attribute__((always_inline)) { w4(k, t, w); });
          const double sum = segment_sum(s, pre);
          if (tid == 0) s.tile[t] = sum;
          total += sum;
          if (sum > 0.0) last = t;
        }
        __syncthreads();
        const double target = u < 1.0f ? (double)u * total : INFINITY;
        for (at = 0; at < last && !(before + s.tile[at] > target); ++at) before += s.tile[at];
      }
      if (!(total > 0.0)) return false;
      const double target = u < 1.0f ? (double)u * total : INFINITY;  // 1 and beyond: no sum exceeds it
      if (!ONE) {
        tile(at);
        fill_segments(s, pa, at, [&](int k, double (&w)[4]) __attribute__((always_inline)) { w4(k, at, w); });
      }
      const Spot sp = find_segment(s, before, target);
      mine = false;
      if (wave == sp.wave) {  // wave-uniform
        if (ONE) tile(0);
        tok = find_id(sp, target, pa, at, [&](int k, double (&w)[4]) __attribute__((always_inline)) { w4(k, at, w); });
        mine = tok >= 0;
      }
      return true;
    };
    double total;
    bool drawn = false;
    if constexpr (DRAFT) {
      if (real) {
        const double ip = 1.0 / p.sum, iq = 1.0 / q.sum;
        drawn = draw([&](int k, int t, double (&w)[4]) __attribute__((always_inline)) {
          float v[4];
          double y[4] = {};
          const int id = pa.id(t, k);
          take_group(P, k, v);
          if (p.sharp) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = id + e == p.first ? 1.0 : 0.0;
          } else {
            p.template weights<false>(v, w, pow);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] *= ip;
          }
          if (!has_q || (q.some && q.sharp)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = id + e == (has_q ? q.first : x) ? 1.0 : 0.0;
          } else if (q.some) {
            take_group(Q, k, v);
            q.template weights<false>(v, y, pow);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] *= iq;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = fmax(w[e] - y[e], 0.0);
        }, total);
      }
    }
    if (!drawn) {
      auto from_p = [&](auto clean, int k, double (&w)[4]) __attribute__((always_inline)) {
        float v[4];
        take_group(P, k, v);
        p.template weights<decltype(clean)::value>(v, w, pow);
      };
      draw([&](int k, int, double (&w)[4]) __attribute__((always_inline)) { clean_p ? from_p(std::true_type{}, k, w) : from_p(std::false_type{}, k, w); },
           p.sum);
      if (p.sharp) {
        tok = p.first;
        mine = tid == 0;
      }
    }
  }
  if (!mine) return;
  a.tokens[m] = tok;
  if (a.accepted) a.accepted[m] = take ? 1 : 0;
  if (a.conf) a.conf[m] = tok >= 0 ? weight_at(p, pa, tok, pow) / p.sum : 0.0;
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
  // the fewest threads whose registers hold the row, with up to 3 ids before it
  int threads = 256;
  while (threads < kMaxThreads && threads * kQuads * 4 < c.V + 3) threads *= 2;
  const bool one = threads * kQuads * 4 >= c.V + 3;
  const auto fn = c.draft ? (one ? k_verify_rows<true, true> : k_verify_rows<true, false>)
                          : (one ? k_verify_rows<false, true> : k_verify_rows<false, false>);
  hipLaunchKernelGGL(fn, dim3((unsigned)c.M), dim3(threads), 0, st, a);
  const nmdlm_status rc = hip_status();
  if (rc != NMDLM_OK || !c.draft || (c.each && !c.n_accepted)) return rc;
  hipLaunchKernelGGL(k_verify_join, dim3((unsigned)c.n_seq), dim3(64), 0, st, a);
  return hip_status();
}

}  // namespace nmdlm
