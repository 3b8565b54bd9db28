// Attention on spike operands whose rows see the keys of two ranges each, with a
// bias of the scores by distance (the formulas: attn_device.h and nmdlm.h).
#include <algorithm>

#include "attn_device.h"
#include "masked.h"

namespace nmdlm {

struct MaskedArgs {
  const uint64_t* q;
  const uint64_t* kc;
  const uint64_t* vt;
  int64_t cap;
  const int4* ranges;
  const int32_t* q_pos;
  const int32_t* k_pos;
  const int8_t* bias;
  const uint8_t* lut;
  int32_t* a_out;
  uint64_t* s_out;
  uint64_t* u_out;
  int32_t* part;  // sums of the splits [row][head][split][T][64 DHW + kMaskedDen]
  int n_keys, max_rows, T, H, parts, splits, max_dist;
  int32_t theta;
};
constexpr int kMaskedDen = 4;    // the weights' sum behind the channels' sums, and padding
constexpr int kSplitChunks = 8;  // a split has at least this many chunks

// The keys of two ranges [lo, hi) within [0, n_keys), the empty ones at 0.
struct KeyRanges {
  int a0, a1, b0, b1;
};
__device__ __forceinline__ KeyRanges key_ranges(int4 r, int n_keys) {
  KeyRanges k{max(r.x, 0), min(r.y, n_keys), max(r.z, 0), min(r.w, n_keys)};
  if (k.a1 <= k.a0) k.a0 = k.a1 = 0;
  if (k.b1 <= k.b0) k.b0 = k.b1 = 0;
  return k;
}

// The 64-key chunks of both ranges, each once: n of them, the first na from a on,
// the others from b on.
struct ChunkList {
  int a, na, b, n;
  __device__ __forceinline__ int at(int i) const { return i < na ? a + i : b + (i - na); }
};
__device__ __forceinline__ ChunkList chunk_list(const KeyRanges& k) {
  int a = k.a0 >> 6, a1 = (k.a1 + 63) >> 6, b = k.b0 >> 6, b1 = (k.b1 + 63) >> 6;
  if (a1 <= a) {  // the first is empty
    a = b;
    a1 = b1;
    b = b1 = 0;
  } else if (b1 > b && b <= a1 && a <= b1) {  // they meet: one
    a = min(a, b);
    a1 = max(a1, b1);
    b = b1 = 0;
  }
  return ChunkList{a, a1 - a, b, a1 - a + b1 - b};
}
// Splits of a list of n chunks, and the part of split z.
__device__ __forceinline__ int split_count(const MaskedArgs& a, int n) {
  return min(a.splits, max(n / kSplitChunks, 1));
}
__device__ __forceinline__ int split_at(int n, int z, int splits) { return (int)((long long)n * z / splits); }

template <int DHW>
__device__ __forceinline__ int32_t* split_sums(const MaskedArgs& a, int row, int h, int z) {
  return a.part + (((size_t)row * a.H + h) * a.splits + z) * a.T * (64 * DHW + kMaskedDen);
}

// ---------------------------------------------------------------------------
// k_masked_rows: one row, head and split; wave = (timestep, part).  Bit by bit:
// lane = key for the scores (popcount of the key's row and the query, the same
// for all lanes), the weight's eight bits become eight 64-key masks by ballots,
// and with lane = channel
//     sum_j p_j V[j,c] = sum_b 2^b popcount(mask_b AND word of channel c).
// A key that the row does not see weighs 0.
// ---------------------------------------------------------------------------
constexpr int kRowWaves = 12;  // of a workgroup at most

template <int DHW>
__global__ __launch_bounds__(64 * kRowWaves) void k_masked_rows(MaskedArgs a) {
  constexpr int DH = 64 * DHW;
  __shared__ uint8_t sLut[256];
  __shared__ int8_t sBias[2 * NMDLM_MAX_DIST + 1];
  __shared__ int sNum[NMDLM_MAX_T][DH];
  __shared__ int sDen[NMDLM_MAX_T];
  const int nth = blockDim.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nwaves = nth >> 6;
  // neighbouring heads share key lines: consecutive logical ids, head fastest
  const int lid = xcd_order(blockIdx.x, gridDim.x);
  const int h = lid % a.H, z = (lid / a.H) % a.splits, row = lid / (a.H * a.splits);
  const KeyRanges kr = key_ranges(a.ranges[row], a.n_keys);
  const ChunkList cl = chunk_list(kr);
  const int splits = split_count(a, cl.n);
  if (z >= splits) return;  // uniform
  const int i0 = split_at(cl.n, z, splits), i1 = split_at(cl.n, z + 1, splits);
  const int np = a.parts, t = wave / np, part = wave - t * np;
  const int d = a.H * DH, dw = d / 64;
  const uint64_t* kb = a.kc + (size_t)t * a.cap * dw + h * DHW;
  const uint64_t* vb = a.vt + (size_t)t * (a.cap / 64) * d + h * DH;
  const uint64_t* qp = a.q + ((size_t)t * a.max_rows + row) * dw + h * DHW;
  uint64_t q[DHW];
#pragma unroll
  for (int w = 0; w < DHW; ++w) q[w] = qp[w];
  const int D = a.max_dist, q_pos = a.bias ? a.q_pos[row] : 0;
  for (int i = tid; i < 256; i += nth) sLut[i] = a.lut[i];
  if (a.bias)
    for (int i = tid; i < 2 * D + 1; i += nth) sBias[i] = a.bias[(size_t)h * (2 * D + 1) + i];
  for (int i = tid; i < a.T * DH; i += nth) (&sNum[0][0])[i] = 0;
  if (tid < a.T) sDen[tid] = 0;
  __syncthreads();

  int acc[8][DHW], den = 0;
#pragma unroll
  for (int b = 0; b < 8; ++b)
#pragma unroll
    for (int w = 0; w < DHW; ++w) acc[b][w] = 0;
  for (int i = i0 + part; i < i1; i += np) {  // wave-uniform
    const int jc = cl.at(i), j = 64 * jc + lane;
    int s = 0;
    uint64_t v[DHW];
#pragma unroll
    for (int w = 0; w < DHW; ++w) {
      s += (int)__popcll(kb[(size_t)j * dw + w] & q[w]);
      v[w] = vb[(size_t)jc * d + w * 64 + lane];
    }
    const bool seen = (j >= kr.a0 && j < kr.a1) || (j >= kr.b0 && j < kr.b1);
    if (a.bias) {
      const int off = __builtin_elementwise_sub_sat(q_pos, a.k_pos[min(j, a.n_keys - 1)]);
      s = min(max(s + sBias[min(max(off, -D), D) + D], 0), 255);
    }
    const int p = seen ? sLut[s] : 0;
    den += p;
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const uint64_t mask = __builtin_amdgcn_ballot_w64((p >> b) & 1);
#pragma unroll
      for (int w = 0; w < DHW; ++w) acc[b][w] += (int)__popcll(v[w] & mask);
    }
  }
  for (int o = 32; o > 0; o >>= 1) den += __shfl_xor(den, o);
  if (lane == 0) atomicAdd(&sDen[t], den);
#pragma unroll
  for (int w = 0; w < DHW; ++w) {
    int x = 0;
#pragma unroll
    for (int b = 7; b >= 0; --b) x = 2 * x + acc[b][w];
    atomicAdd(&sNum[t][64 * w + lane], x);
  }
  __syncthreads();
  if (splits > 1) {  // uniform
    int32_t* o = split_sums<DHW>(a, row, h, z);
    for (int i = tid; i < a.T * DH; i += nth) o[(i / DH) * (DH + kMaskedDen) + i % DH] = (&sNum[0][0])[i];
    if (tid < a.T) o[tid * (DH + kMaskedDen) + DH] = sDen[tid];
    return;
  }
  for (int w = wave; w < DHW; w += nwaves)
    fire_row<DHW>(a, row, h, w, lane, a.n_keys < 65536, [&](int tt) { return sNum[tt][w * 64 + lane]; },
                  [&](int tt) { return sDen[tt]; });
}

// k_masked_join: the sums of a row's splits (integers: any order gives the same)
// and the neuron.  A workgroup per row and head, a wave per timestep and 64
// channels.
template <int DHW>
__global__ __launch_bounds__(64 * NMDLM_MAX_T * DHW) void k_masked_join(MaskedArgs a) {
  constexpr int LD = 64 * DHW + kMaskedDen;
  __shared__ int sNum[NMDLM_MAX_T][64 * DHW];
  __shared__ int sDen[NMDLM_MAX_T];
  const int h = blockIdx.x % a.H, row = blockIdx.x / a.H;
  const int n = split_count(a, chunk_list(key_ranges(a.ranges[row], a.n_keys)).n);
  if (n == 1) return;  // uniform; a single split fired by itself
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int t = wave / DHW, w = wave - t * DHW;
  const int32_t* base = split_sums<DHW>(a, row, h, 0) + (size_t)t * LD;
  const size_t ld = (size_t)a.T * LD;
  int x = 0, den = 0;
  for (int z = 0; z < n; ++z) {
    x += base[z * ld + w * 64 + lane];
    den += base[z * ld + 64 * DHW];
  }
  sNum[t][w * 64 + lane] = x;
  if (w == 0 && lane == 0) sDen[t] = den;
  __syncthreads();
  if (wave < DHW)
    fire_row<DHW>(a, row, h, wave, lane, a.n_keys < 65536,
                  [&](int tt) { return sNum[tt][wave * 64 + lane]; }, [&](int tt) { return sDen[tt]; });
}

MaskedRoute masked_route(int T, int M, int n_keys, int H) {
  MaskedRoute r{std::max(std::min(kRowWaves / T, 4), 1), 1};
  r.splits = (int)std::max(1LL, std::min<long long>({512 / ((long long)M * H), 64, n_keys / (64 * kSplitChunks)}));
  return r;
}

size_t masked_attn_ws(int T, int M, int n_keys, int H, int dh) {
  const MaskedRoute r = masked_route(T, M, n_keys, H);
  if (r.splits == 1) return 0;
  return align_up((size_t)M * H * r.splits * T * (dh + kMaskedDen) * sizeof(int32_t), 256);
}

template <int DHW>
static nmdlm_status launch_masked_dh(const MaskedAttnCall& c, hipStream_t st) {
  const MaskedRoute r = masked_route(c.T, c.M, c.n_keys, c.H);
  const MaskedArgs a{c.q, c.k_cache, c.vt_cache, c.cap, reinterpret_cast<const int4*>(c.mask.ranges),
                     c.mask.q_pos, c.mask.k_pos, c.bias, c.lut, c.a_out, c.s_out, c.u_out,
                     static_cast<int32_t*>(c.ws), c.n_keys, c.M, c.T, c.H, r.parts, r.splits,
                     c.bias ? c.mask.max_dist : 0, c.theta};
  hipLaunchKernelGGL(k_masked_rows<DHW>, dim3((unsigned)c.M * c.H * r.splits), dim3(64 * c.T * r.parts), 0, st, a);
  const nmdlm_status rc = hip_status();
  if (rc != NMDLM_OK || r.splits == 1) return rc;
  hipLaunchKernelGGL(k_masked_join<DHW>, dim3((unsigned)c.M * c.H), dim3(64 * c.T * DHW), 0, st, a);
  return hip_status();
}

nmdlm_status launch_masked_attn(const MaskedAttnCall& c, hipStream_t st) {
  return c.dh == 64 ? launch_masked_dh<1>(c, st) : launch_masked_dh<2>(c, st);
}

}  // namespace nmdlm
