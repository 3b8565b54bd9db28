// Attention on spike operands over a contiguous cache: binary-binary scores
// (popcount of AND), table weights, integer-normalised weighted sum of binary
// values (the sums of a wave: attn_device.h).
#include <algorithm>

#include "attn_device.h"

namespace nmdlm {

// ---------------------------------------------------------------------------
// k_attn: scores and weighted sums of one (head, 16 queries, timestep), the
// chunks shared by NW waves whose sums meet in LDS; the IF of the output
// follows in its own kernel.  For grids too small for one wave per 16 queries
// (the denoising step's): every load of a short context is in flight at once.
//
// grid (H, n_seq * ceil(M/16), T), M queries per sequence, rows of q and
// a_out sequence-major (n_seq * M per timestep), the caches of sequence s at
// s * seq_words words past kc / vt.
//
// dh = 128 takes 129 registers, one too many for two workgroups on a CU.  WPE = 4
// (waves per SIMD) holds it to 128, an address pair of the chunk loop spilled: for
// grids of more workgroups than CUs (T = 8, 133 x 773 keys, 12 heads 28.0 -> 23.2 us; 101 x
// 899, 16 heads 28.2 -> 23.2); smaller ones lose 4% by the spill.  The
// entries stand at 1 KB, as the products' do: at 256 bytes the same code took 0.2 us more.
// ---------------------------------------------------------------------------
template <int DHW, int NW, int WPE>
__global__ __launch_bounds__(NW * 64, WPE) __attribute__((aligned(1024)))
void k_attn(const uint64_t* __restrict__ q,
            const uint64_t* __restrict__ kc,
            const uint64_t* __restrict__ vt, int64_t cap,
            int T, int M, int C, int H,
            const uint8_t* __restrict__ lut,
            int32_t* __restrict__ a_out, int n_seq,
            int64_t seq_words) {
  constexpr int DH = DHW * 64;
  constexpr int NT = DH / 16;
  constexpr int NTH = NW * 64;
  __shared__ AttnLut sLut;
  __shared__ v4i sNum[NT * 64];  // [tile n][lane]: query c, channels 16n + 4g + e
  __shared__ int sDen[16];
  __shared__ AttnStage<DHW> sStage[kAttnStages * NW];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = lane >> 4, c = lane & 15;
  // neighbouring heads share key lines: consecutive logical ids, head fastest
  const int nwg = gridDim.x * gridDim.y * gridDim.z;
  const int lid = xcd_order(blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z), nwg);
  const int h = lid % gridDim.x, qbg = (lid / gridDim.x) % gridDim.y,
            t = lid / (gridDim.x * gridDim.y);
  const int qbps = gridDim.y / n_seq;               // query blocks per sequence
  const int sq = qbg / qbps, qb = qbg - sq * qbps;  // sequence, block within it
  const int Mt = n_seq * M, r0 = sq * M;            // rows per timestep, first row of sq
  const int d = H * DH, dw = d / 64;
  const int J = C + M;
  const int nch = (J + 63) / 64;
  const uint64_t* kb = kc + sq * seq_words + (size_t)t * cap * dw + h * DHW;
  const uint64_t* vb = vt + sq * seq_words + (size_t)t * (cap / 64) * d + h * DH;

  AttnChunk<DHW> first, next;
  // every load of the prologue leaves before the first is waited for
  const LutRegs lr = load_lut(lut, tid, NTH);
  uint32_t qraw[1];
  AttnWave<DHW, 1>::load_queries(qraw, q + ((size_t)t * Mt + r0) * dw + h * DHW, dw, qb * 16, M - 1, g, c);
  AttnWave<DHW, 1>::load(first, kb, vb, dw, d, min(wave, nch - 1), lane);
  AttnWave<DHW, 1>::load(next, kb, vb, dw, d, min(wave + NW, nch - 1), lane);
  __builtin_amdgcn_sched_barrier(0);
  AttnWave<DHW, 1> w;
  w.init(qraw);
  fill_lut(sLut, lr, tid, NTH);
  for (int i = tid; i < NT * 64; i += NTH) sNum[i] = v4i{0, 0, 0, 0};
  if (tid < 16) sDen[tid] = 0;
  __syncthreads();
  if (wave < nch) {  // wave-uniform
    w.run(kb, vb, dw, d, J, nch, wave, NW, sLut, &sStage[kAttnStages * wave], lane, g, c, first, next);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const v4i x = w.acc[0][n];
#pragma unroll
      for (int e = 0; e < 4; ++e) atomicAdd(reinterpret_cast<int*>(&sNum[n * 64 + lane]) + e, x[e]);
    }
    if (g == 0) atomicAdd(&sDen[c], w.den[0] + 128 * keys_of(wave, NW, nch, J));
  }
  __syncthreads();

  const bool small = J < 65536;
  for (int i = tid; i < NT * 64; i += NTH) {
    const int n = i >> 6, lc = i & 15, lg = (i >> 4) & 3;
    const int iq = qb * 16 + lc;
    if (iq >= M) continue;
    const v4i x = sNum[i];
    const int den = sDen[lc];
    v4i a;
    if (small) {
      a = attn_norm4(x, den);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = attn_norm(x[e], den);
    }
    int32_t* o = a_out + ((size_t)t * Mt + r0 + iq) * d + h * DH + n * 16 + 4 * lg;
    if ((reinterpret_cast<uintptr_t>(a_out) & 15) == 0) {  // uniform
      *reinterpret_cast<v4i*>(o) = a;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = a[e];
    }
  }
}

// ---------------------------------------------------------------------------
// k_attn_if: attention followed by the IF neuron of its output, in one kernel.
// Workgroup = one head and 16*QG queries, wave = (timestep, part): the parts of
// a timestep (PARTS, QG = 1: grids that leave SIMDs idle) take its chunks in
// turn and add their sums in LDS; without parts a wave takes all chunks of its
// timestep and normalises its sums itself.  The sums or currents meet in LDS
// (16 queries at a time, over the chunks' stages) and the waves share the
// tiles of 16 channels for the IF recurrence over t, the spike words and the
// token's union over t.  a_out (the currents) and s_out are each optional.
// No currents go through memory (64 MB written and read at the 2048-token
// prompt below) and there is no launch between the two.
// ---------------------------------------------------------------------------
struct AttnIfArgs {
  const uint64_t* q;
  const uint64_t* kc;
  const uint64_t* vt;
  int64_t cap;
  int T, M, C, H, n_seq, parts;
  int64_t seq_words;
  const uint8_t* lut;
  int32_t theta;
  int32_t* a_out;
  uint64_t* s_out;
  uint64_t* u_out;
};

template <int DHW, int QG, bool PARTS>
__global__ __launch_bounds__(64 * NMDLM_MAX_T) void k_attn_if(AttnIfArgs a) {
  constexpr int DH = DHW * 64;
  constexpr int NT = DHW * 4;
  static_assert(!PARTS || QG == 1, "parts: one query group");
  __shared__ AttnLut sLut;
  __shared__ int sDen[PARTS ? NMDLM_MAX_T : 1][16];
  __shared__ uint32_t sWord[NMDLM_MAX_T][16][2 * DHW];  // halves of the spike words
  // the waves' stages, then (chunks done) the sums [T][NT][64]
  extern __shared__ v4i sNum[];
  AttnStage<DHW>* sStage = reinterpret_cast<AttnStage<DHW>*>(sNum);

  const int nth = blockDim.x;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nwaves = nth >> 6;
  const int g = lane >> 4, c = lane & 15;
  const int nwg = gridDim.x * gridDim.y;
  const int lid = xcd_order(blockIdx.x + gridDim.x * blockIdx.y, nwg);
  const int h = lid % gridDim.x, qbg = lid / gridDim.x;
  const int qbps = gridDim.y / a.n_seq;
  const int sq = qbg / qbps, qb = qbg - sq * qbps;
  const int Mt = a.n_seq * a.M, r0 = sq * a.M;
  const int d = a.H * DH, dw = d / 64;
  const int J = a.C + a.M, nch = (J + 63) / 64;
  const int np = PARTS ? a.parts : 1;
  const int t = PARTS ? wave / np : wave, part = wave - t * np;
  const uint64_t* kb = a.kc + sq * a.seq_words + (size_t)t * a.cap * dw + h * DHW;
  const uint64_t* vb = a.vt + sq * a.seq_words + (size_t)t * (a.cap / 64) * d + h * DH;

  AttnChunk<DHW> first, next;
  // every load of the prologue leaves before the first is waited for
  const LutRegs lr = load_lut(a.lut, tid, nth);
  uint32_t qraw[QG];
  AttnWave<DHW, QG>::load_queries(qraw, a.q + ((size_t)t * Mt + r0) * dw + h * DHW, dw, qb * 16 * QG,
                                  a.M - 1, g, c);
  AttnWave<DHW, QG>::load(first, kb, vb, dw, d, min(part, nch - 1), lane);
  AttnWave<DHW, QG>::load(next, kb, vb, dw, d, min(part + np, nch - 1), lane);
  __builtin_amdgcn_sched_barrier(0);
  AttnWave<DHW, QG> w;
  w.init(qraw);
  fill_lut(sLut, lr, tid, nth);
  __syncthreads();
  if (!PARTS || part < nch)  // wave-uniform
    w.run(kb, vb, dw, d, J, nch, part, np, sLut, &sStage[kAttnStages * wave], lane, g, c, first, next);
  __syncthreads();  // the stages are read
  if constexpr (PARTS) {
    for (int i = tid; i < a.T * NT * 64; i += nth) sNum[i] = v4i{0, 0, 0, 0};
    for (int i = tid; i < a.T * 16; i += nth) (&sDen[0][0])[i] = 0;
    __syncthreads();
  }
  const bool small = J < 65536;
  const bool vec = (reinterpret_cast<uintptr_t>(a.a_out) & 15) == 0;

#pragma unroll
  for (int u = 0; u < QG; ++u) {
    if (u > 0) __syncthreads();  // the previous group's currents and words are read
    const int iq0 = (qb * QG + u) * 16, iq = iq0 + c;
    for (int i = tid; i < a.T * 32 * DHW; i += nth) (&sWord[0][0][0])[i] = 0u;
    if constexpr (PARTS) {
      if (part < nch) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            atomicAdd(reinterpret_cast<int*>(&sNum[(t * NT + n) * 64 + lane]) + e, w.acc[u][n][e]);
        if (g == 0) atomicAdd(&sDen[t][c], w.den[u] + 128 * keys_of(part, np, nch, J));
      }
    } else {
      const int den = w.den[u] + 128 * J;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        v4i x;
        if (small) {
          x = attn_norm4(w.acc[u][n], den);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = attn_norm(w.acc[u][n][e], den);
        }
        sNum[(t * NT + n) * 64 + lane] = x;
      }
    }
    __syncthreads();
    for (int n = wave; n < NT; n += nwaves) {
      v4i V = v4i{0, 0, 0, 0};  // at most 256 T
      for (int t0 = 0; t0 < a.T; t0 += 4) {
        v4i cur[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int tt = min(t0 + k, a.T - 1);
          cur[k] = sNum[(tt * NT + n) * 64 + lane];
          if constexpr (PARTS) {
            const int den = sDen[tt][c];
            if (small) {
              cur[k] = attn_norm4(cur[k], den);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) cur[k][e] = attn_norm(cur[k][e], den);
            }
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int tt = t0 + k;
          if (tt >= a.T) break;  // uniform
          if (a.a_out && iq < a.M) {
            int32_t* o = a.a_out + ((size_t)tt * Mt + r0 + iq) * d + h * DH + n * 16 + 4 * g;
            if (vec) {
              *reinterpret_cast<v4i*>(o) = cur[k];
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) o[e] = cur[k][e];
            }
          }
          uint32_t bits = 0u;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            V[e] += cur[k][e];
            const bool s = V[e] >= a.theta;
            if (s) V[e] -= a.theta;
            bits |= (uint32_t)s << e;
          }
          // tile n's 16 bits of the query's word, four from each lane group
          atomicOr(&sWord[tt][c][n >> 1], bits << (16 * (n & 1) + 4 * g));
        }
      }
    }
    if (!a.s_out) continue;  // uniform
    __syncthreads();
    for (int i = tid; i < 16 * DHW * a.T; i += nth) {
      const int k = i % DHW, m = (i / DHW) % 16, tt = i / (16 * DHW);
      if (iq0 + m < a.M)
        a.s_out[((size_t)tt * Mt + r0 + iq0 + m) * dw + h * DHW + k] =
            sWord[tt][m][2 * k] | (uint64_t)sWord[tt][m][2 * k + 1] << 32;
    }
    if (a.u_out)
      for (int i = tid; i < 16 * DHW; i += nth) {
        const int k = i % DHW, m = i / DHW;
        uint64_t uor = 0ull;
        for (int tt = 0; tt < a.T; ++tt) uor |=
            sWord[tt][m][2 * k] | (uint64_t)sWord[tt][m][2 * k + 1] << 32;
        if (iq0 + m < a.M) a.u_out[(size_t)(r0 + iq0 + m) * dw + h * DHW + k] = uor;
      }
  }
}

template <int DHW, int QG, bool PARTS = false>
static nmdlm_status attn_if_launch(const AttnIfArgs& a, hipStream_t st) {
  const dim3 grid(a.H, a.n_seq * ((a.M + 16 * QG - 1) / (16 * QG)));
  const size_t dyn = std::max((size_t)a.T * DHW * 4 * 64 * sizeof(v4i),
                              a.T * a.parts * kAttnStages * sizeof(AttnStage<DHW>));
  if (dyn > 57344 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(&k_attn_if<DHW, QG, PARTS>),
                          hipFuncAttributeMaxDynamicSharedMemorySize, (int)dyn) != hipSuccess)
    return NMDLM_ERR_HIP;
  hipLaunchKernelGGL((k_attn_if<DHW, QG, PARTS>), grid, dim3(64 * a.T * a.parts), (uint32_t)dyn, st, a);
  return hip_status();
}

// Which kernel, all measured with spikes out, H = 16 unless said, dh = 64 / 128:
//  * 32 queries a wave (QG = 2) halve the expansions and the staging per
//    query but need two such waves per SIMD: T = 4, 2048 x 2048 keys 45.8 / 75.3
//    us against 80.3 / 93.6 with 16; 600 x 1200 keys 20.2 / 29.0 against
//    19.5 / 27.4.
//  * Parts: where the waves of 16 queries leave SIMDs idle.  T = 1 (four; the
//    parts also share the epilogue of what would be a workgroup of one wave):
//    H = 8, 32 x 700 keys, dh = 128 7.4 us against 10.7; 1000 x 2000 9.5 / 13.7
//    against 14.5 / 22.6; 4 x 480, dh = 64 4.8 against 6.3.  T = 2 (four) from 7 / 4
//    chunks on: 7 chunks 6.0 / 7.8 against 6.1 / 8.8, 4 chunks of 64: 5.7 against
//    5.4.  Below 12 chunks only while the parts run at once: T = 1, 300 workgroups, 10
//    chunks, dh = 128 9.7 against 11.1, 672 workgroups, 6 chunks, dh = 64 7.9 against 7.4.
//    T = 3, 4 (two) from 12: 256 x 1256 11.7 / 15.6 against 11.2 / 15.8; 9 chunks 8.8
//    against 7.5.
//  * k_attn and the IF kernel, a second launch and the currents through
//    memory, where few workgroups would each walk a long context.  From 128
//    workgroups on never (256 x 1256 keys 17.2 / 31.0 against 11.2 / 15.8); below,
//    from 12 chunks on, when a wave walks more than 6: T = 4, 32 x 1056 keys,
//    dh = 128 11.5 us against 13.7 (8032 keys: 20 against 63).  With few of them (up
//    to one workgroup of k_attn per CU) also for shorter walks, by the chunk's
//    cost (kWalk): inside a step, graph time, T = 4, dh = 128, 6 chunks 7.5 against
//    8.3, 11 chunks 8.4 against 11.0; T = 8, dh = 64 5 chunks 7.5 against 7.7, 8 chunks
//    7.5 against 8.8; T = 8, dh = 128 3 chunks 7.6 against 8.4, 8 chunks 8.5 against 11.7.
//    A call by itself pays the host's pace for the second launch (11.3 us a call
//    against 8.3): T = 4, dh = 128, 11 chunks 11.2 against 10.7; T = 8, 7 chunks 11.1 against
//    11.4, 11 chunks 10.5 against 14.2.
constexpr int kAttnNW = 8;           // waves per workgroup of k_attn
constexpr int kPartsMinChunks = 12;
constexpr int kFusedMaxWalk = 6;     // chunks per wave of few workgroups with parts
constexpr long long kFusedMinWgs = 128;
constexpr long long kFullWaves = 2048;  // two waves per SIMD
// longest walk in one kernel with at most kOneRound workgroups of k_attn:
// [step][dh / 64 - 1][T = 1, 2 | 3, 4 | 5, 6 | 7, 8] (T = 1, 2: as with parts)
constexpr long long kOneRound = 256;  // one workgroup of k_attn per CU
constexpr int kWalk[2][2][4] = {{{11, 11, 11, 11}, {11, 11, 6, 6}}, {{11, 11, 5, 5}, {11, 5, 2, 1}}};

AttnRoute attn_route(const AttnCall& c) {
  const long long heads = (long long)c.H * c.n_seq;
  const long long wgs = heads * ((c.M + 15) / 16);
  const int nch = (c.C + c.M + 63) / 64, w = c.dh / 64 - 1;
  AttnRoute r{1, 1, false};
  if (c.M >= 32 && heads * ((c.M + 31) / 32) * c.T >= kFullWaves) {
    r.groups = 2;
    return r;
  }
  if (nch >= kPartsMinChunks) {
    if (wgs * c.T < kFullWaves) r.parts = c.T <= 2 ? 4 : (c.T <= 4 ? 2 : 1);
  } else if (wgs * c.T <= kFullWaves / 4 && (c.T == 1 || (c.T == 2 && nch >= (w ? 4 : 7)))) {
    r.parts = 4;
  }
  if (c.fused || wgs >= kFusedMinWgs) return r;
  const int walk = (nch + r.parts - 1) / r.parts;
  r.split = (nch >= kPartsMinChunks && walk > kFusedMaxWalk) ||
            (wgs * c.T <= kOneRound && walk > kWalk[c.step][w][(c.T - 1) / 2]);
  return r;
}

template <int DHW>
static nmdlm_status launch_attention_dh(const AttnCall& c, hipStream_t st) {
  const AttnRoute r = attn_route(c);
  const AttnIfArgs a{c.q, c.k_cache, c.vt_cache, c.cap, c.T, c.M, c.C, c.H, c.n_seq, r.parts,
                     c.seq_words, c.lut, c.theta, c.a_out, c.s_out, c.u_out};
  if (r.groups == 2) return attn_if_launch<DHW, 2>(a, st);
  if (!r.split) return r.parts > 1 ? attn_if_launch<DHW, 1, true>(a, st) : attn_if_launch<DHW, 1>(a, st);
  int32_t* const cur = c.a_out ? c.a_out : c.a_scratch;
  const dim3 grid(c.H, c.n_seq * ((c.M + 15) / 16), c.T);
  const auto fn = (long long)grid.x * grid.y * grid.z > kOneRound ? k_attn<DHW, kAttnNW, DHW == 2 ? 4 : 1>
                                                                  : k_attn<DHW, kAttnNW, 1>;
  hipLaunchKernelGGL(fn, grid, dim3(kAttnNW * 64), 0, st, c.q, c.k_cache, c.vt_cache, c.cap, c.T, c.M, c.C,
                     c.H, c.lut, cur, c.n_seq, c.seq_words);
  const nmdlm_status rc = hip_status();
  if (rc != NMDLM_OK || !c.s_out) return rc;
  return launch_if(cur, c.T, c.n_seq * c.M, c.H * c.dh, c.theta, nullptr, nullptr, nullptr, c.s_out,
                   st, c.u_out);
}

nmdlm_status launch_attention(const AttnCall& c, hipStream_t st) {
  if (c.n_seq < 1) return NMDLM_ERR_INVALID_ARG;
  if (c.dh == 64) return launch_attention_dh<1>(c, st);
  if (c.dh == 128) return launch_attention_dh<2>(c, st);
  return NMDLM_ERR_UNSUPPORTED;
}

}  // namespace nmdlm
