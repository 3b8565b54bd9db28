// Device code of the spike attentions: the sums' normalisation and one wave's
// share of the scores and weighted sums.
//
//   s = popcount(Q_i AND K_j) per head;  p = lut[s] in [0, 255]
//   num[i,c] = sum_j p_ij V[j,c];  den[i] = sum_j p_ij
//   a[i,c] = floor(256 * num / den)   (0 if den = 0)
//
// Both products run on v_mfma_i32_16x16x64_i8, exact in int32: the scores as
// a 0/1-byte product of key and query bits over the head's channels, the
// weighted sum with p - 128 (signed byte) against the value bits expanded to
// bytes, to which 128 * (number of ones of V[.,c]) is added back.  A sum is at
// most 255 per key: below 2^31 up to NMDLM_MAX_KEYS keys.
#pragma once

#include "common.h"

namespace nmdlm {

static_assert(255LL * NMDLM_MAX_KEYS < 1LL << 31, "sums of table weights fit int32");

// floor(256 * num / den) for 0 <= num <= den (0 when den = 0): from 65536 keys
// on, in 64 bits.  (num and den themselves stay below 2^31 up to
// NMDLM_MAX_KEYS keys of weight 255.)
__device__ __forceinline__ int32_t attn_norm(int num, int den) {
  return den <= 0 ? 0 : (int32_t)((256LL * num) / den);
}

// The same for four numerators over one denominator and fewer than 65536 keys
// (num and den below 2^24, exact as floats): k = 256 / den, lowered by 2^-20 of
// itself, more than the rounding errors of the reciprocal and the two products
// (4 units of 2^-24), so the truncated estimate is the floor or one below it; the
// remainder 256 num - q den, one rounding of an exact value, decides which.
// An empty denominator (num = 0) counts as one.
__device__ __forceinline__ v4i attn_norm4(v4i num, int den_i) {
  const float den = (float)max(den_i, 1);
  const float k = __builtin_amdgcn_rcpf(den) * (256.0f - 0x1p-12f);
  v4i a;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float n = (float)num[e];
    const float q = __builtin_truncf(n * k);
    a[e] = (int)q + (__builtin_fmaf(-q, den, 256.0f * n) >= den ? 1 : 0);
  }
  return a;
}

// attn_norm4 in two: the factor k of a denominator and four numerators.
__device__ __forceinline__ float attn_factor(float den) {
  return __builtin_amdgcn_rcpf(den) * (256.0f - 0x1p-12f);
}
__device__ __forceinline__ v4i attn_norm4(v4i num, float den, float k) {
  v4i a;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float n = (float)num[e];
    const float q = __builtin_truncf(n * k);
    a[e] = (int)q + (__builtin_fmaf(-q, den, 256.0f * n) >= den ? 1 : 0);
  }
  return a;
}

// One numerator, as attn_norm4 for fewer than 65536 keys and else as attn_norm.
__device__ __forceinline__ int32_t attn_norm1(int num, int den_i, bool small) {
  if (!small) return attn_norm(num, den_i);
  const float den = (float)max(den_i, 1), n = (float)num;
  const float q = __builtin_truncf(n * (__builtin_amdgcn_rcpf(den) * (256.0f - 0x1p-12f)));
  return (int)q + (__builtin_fmaf(-q, den, 256.0f * n) >= den ? 1 : 0);
}

// ---------------------------------------------------------------------------
// One wave's share of the attention of 16*QG queries of one head and
// timestep: 64-key chunks, each lane (g = lane/16, c = lane%16).
//
// Scores: the A operand of tile u (u = 0..3) holds 16 keys, row r = key
// 16*(r/4) + 4u + r%4 of the chunk, the B operand the 16 queries; the result
// of lane (g, c) is then the scores of query c with keys 16g + 4u + e, so over
// the four tiles a lane owns the 16 consecutive keys 16g .. 16g+15 of its
// query: the operand the weighted sum wants, with no exchange.  A lane's key
// bits (dh = 128: dword g of the row, two k-steps; dh = 64: 16-bit piece g)
// become bytes in place as bits & (0x01010101 << i), of value 2^i; the query's
// byte is 2^(3-i), so a score arrives times 8, the byte offset into the table.
// The order of the channels differs from the memory order, the same way for
// keys and queries.
//
// Weights: the table sits in LDS four times, the entry p - 128 shifted to byte
// 0..3 of a dword, so a P operand dword is four reads and two ORs; scores less
// than 32 apart fall in different banks, equal scores broadcast.
//
// Weighted sum: A = the value bits of 16 channels (rows), B = P (columns =
// queries): lane (g, c) accumulates query c, channels 16n + 4g + e.  Value
// bits h (16 keys of a channel) become bytes as (x >> i) & 0x01010101 of
// x = h | h << 12: byte b of dword i is key i + {0, 8, 4, 12}[b], and P is
// packed to match.
//
// Per 32 queries and chunk (QG = 2, dh = 128) that is 125 vector instructions
// and 32 MFMAs, where scoring by popcounts took 350 vector instructions per 16
// queries; the key and value expansions (100 of the 125) are shared by the QG
// query groups.  Bound by LDS, whose indexed path is busy 51% of the cycles (a third of
// that conflicts of the table reads, 32 of them a chunk), and by instruction issue;
// the matrix cores are busy 37% (counters of the call below).
// T = 4, 16 heads of 128, 2048 queries x 2048 keys: 213 -> 76 us (1.8 POP/s).
// ---------------------------------------------------------------------------
typedef uint32_t __attribute__((may_alias)) u32_alias;
typedef uint16_t __attribute__((may_alias)) u16_alias;
typedef int __attribute__((may_alias)) i32_alias;
typedef v4i __attribute__((may_alias)) v4i_alias;
constexpr uint32_t kByteOnes = 0x01010101u;
constexpr int kAttnStages = 3;    // chunks of a wave in LDS
constexpr int kLutEntries = 132;  // scores 0..128, padded to a multiple of four

// Entry s of the table, 8 bytes (a score arrives times 8, as a byte offset):
// the byte lut[s] - 128 at byte positions 2h and 2h + 1 of two dwords, h = 0, 1
// the half of the table.
struct AttnLut {
  int e[2][kLutEntries][2];
};
constexpr int kLutLoads = (kLutEntries + 63) / 64;  // for a workgroup of one wave
struct LutRegs {
  uint8_t v[kLutLoads];
};
// loads at clamped places, without a condition, to leave with the others
__device__ __forceinline__ LutRegs load_lut(const uint8_t* __restrict__ lut, int tid, int nth) {
  LutRegs r;
#pragma unroll
  for (int k = 0; k < kLutLoads; ++k) r.v[k] = lut[min(tid + k * nth, kLutEntries - 1)];
  return r;
}
__device__ __forceinline__ void fill_lut(AttnLut& sLut, const LutRegs& r, int tid, int nth) {
#pragma unroll
  for (int k = 0; k < kLutLoads; ++k) {
    const int i = tid + k * nth;
    if (i < kLutEntries) {
      const uint32_t v = (uint32_t)r.v[k] ^ 0x80u;
#pragma unroll
      for (int b = 0; b < 4; ++b) sLut.e[b >> 1][i][b & 1] = (int)(v << (8 * b));
    }
  }
}

__device__ __forceinline__ v4i bytes16(uint32_t x) {  // (x >> i) & ones, i = 0..3
  return v4i{(int)(x & kByteOnes), (int)((x >> 1) & kByteOnes), (int)((x >> 2) & kByteOnes),
             (int)((x >> 3) & kByteOnes)};
}
// key bits in place (values 2^i) and the query bits that make every product 8
__device__ __forceinline__ v4i key_bytes(uint32_t x) {
  return v4i{(int)(x & kByteOnes), (int)(x & (kByteOnes << 1)), (int)(x & (kByteOnes << 2)),
             (int)(x & (kByteOnes << 3))};
}
__device__ __forceinline__ v4i query_bytes(uint32_t x) {
  const v4i b = bytes16(x);
  return v4i{b[0] << 3, b[1] << 2, b[2] << 1, b[3]};
}

// A wave's LDS buffer for the chunk being scored: its 64 key rows, in the
// order the tiles take them, and one value word per channel.
template <int DHW>
struct AttnStage {
  uint64_t k[64 * DHW];
  uint64_t v[DHW * 64];
};

// What a lane loads of a chunk: key row `lane`, the value words of channels
// lane and lane + 64 (whole rows and words: adjacent lanes at adjacent
// addresses, where fetching the operand pieces directly cost 400 cache
// accesses per chunk and set the kernel's time).
template <int DHW>
struct AttnChunk {
  uint64_t k[DHW], v[DHW];
};

// FUSED: the value bits' shift and OR in one instruction, where the compiler
// takes two and shares the shift; 3% of the paged kernels' time, but two registers
// too many for the contiguous ones' occupancy.
template <int DHW, int QG, bool FUSED = false>
struct AttnWave {
  static constexpr int NT = DHW * 4;
  v4i q[QG][DHW];
  v4i acc[QG][NT];
  int den[QG];  // sum of p - 128 of query c over this lane's keys
  int cnt[NT];  // ones of channel 16n + c over this lane's keys

  // query rows iq0 + 16u + c (clamped to the last valid row), channels of head h
  __device__ __forceinline__ static void load_queries(uint32_t (&raw)[QG],
                                                      const uint64_t* __restrict__ qrow, int dw,
                                                      int iq0, int mlast, int g, int c) {
#pragma unroll
    for (int u = 0; u < QG; ++u) {
      const uint64_t* p = qrow + (size_t)min(iq0 + 16 * u + c, mlast) * dw;
      if constexpr (DHW == 2) raw[u] = reinterpret_cast<const u32_alias*>(p)[g];
      else raw[u] = reinterpret_cast<const u16_alias*>(p)[g];
    }
  }
  __device__ __forceinline__ void init(const uint32_t (&raw)[QG]) {
#pragma unroll
    for (int u = 0; u < QG; ++u) {
      const uint32_t w = raw[u];
      if constexpr (DHW == 2) {
        q[u][0] = query_bytes(w);
        q[u][1] = query_bytes(w >> 4);
      } else {
        q[u][0] = query_bytes(w | (w << 12));
      }
      den[u] = 0;
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[u][n] = v4i{0, 0, 0, 0};
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) cnt[n] = 0;
  }

  // kb: key row 0 of the timestep at this head's words; vb: value word 0 of
  // the timestep at this head's channels.  The cache capacity is a multiple
  // of 64, so every row of a chunk holds memory (rows past C+M are masked).
  __device__ __forceinline__ static void load(AttnChunk<DHW>& ch, const uint64_t* __restrict__ kb,
                                              const uint64_t* __restrict__ vb, int dw, int d, int jc,
                                              int lane) {
    const uint64_t* kr = kb + (size_t)jc * 64 * dw;
    const uint64_t* vr = vb + (size_t)jc * d;
#pragma unroll
    for (int w = 0; w < DHW; ++w) {
      ch.k[w] = kr[(uint32_t)(lane * dw + w)];
      ch.v[w] = vr[(uint32_t)(w * 64 + lane)];
    }
  }

  // the chunk into LDS
  __device__ __forceinline__ static void put(const AttnChunk<DHW>& ch, AttnStage<DHW>& st, int lane) {
    const int slot = ((lane >> 2) & 3) * 16 + (lane >> 4) * 4 + (lane & 3);
#pragma unroll
    for (int w = 0; w < DHW; ++w) {
      st.k[slot * DHW + w] = ch.k[w];
      st.v[w * 64 + lane] = ch.v[w];
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }

  // tile u's key is row c of the tile, its bits dword g of the row (dh = 128)
  // or 16-bit piece g (dh = 64)
  __device__ __forceinline__ static void key_pieces(const AttnStage<DHW>& st, uint32_t (&k)[4], int g,
                                                    int c) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if constexpr (DHW == 2) k[u] = reinterpret_cast<const u32_alias*>(st.k)[(u * 16 + c) * 4 + g];
      else k[u] = reinterpret_cast<const u16_alias*>(st.k)[(u * 16 + c) * 4 + g];
    }
  }
  // the bits of channel 16n + c over keys 16g .. 16g+15
  __device__ __forceinline__ static void value_pieces(const AttnStage<DHW>& st, uint32_t (&v)[NT], int g,
                                                      int c) {
#pragma unroll
    for (int n = 0; n < NT; ++n) v[n] = reinterpret_cast<const u16_alias*>(st.v)[(n * 16 + c) * 4 + g];
  }

  // 8 * scores of the chunk's keys
  __device__ __forceinline__ void scores(const uint32_t (&k)[4], v4i (&s)[QG][4]) const {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      v4i k0, k1;
      if constexpr (DHW == 2) {
        k0 = key_bytes(k[u]);
        k1 = key_bytes(k[u] >> 4);
      } else {
        k0 = key_bytes(k[u] | (k[u] << 12));
      }
#pragma unroll
      for (int w = 0; w < QG; ++w)
        s[w][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k0, q[w][0], v4i{0, 0, 0, 0}, 0, 0, 0);
      if constexpr (DHW == 2) {
#pragma unroll
        for (int w = 0; w < QG; ++w)
          s[w][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k1, q[w][1], s[w][u], 0, 0, 0);
      }
    }
  }

  // table bytes in place of the scores (tile u's at byte {0, 2, 1, 3}[u])
  __device__ __forceinline__ static void lookup(v4i (&s)[QG][4], const char* lb) {
#pragma unroll
    for (int w = 0; w < QG; ++w)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int b = u == 1 ? 2 : (u == 2 ? 1 : u);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s[w][u][e] = *reinterpret_cast<const int*>(lb + kLutEntries * 8 * (b >> 1) + 4 * (b & 1) + s[w][u][e]);
      }
  }

  __device__ __forceinline__ static void pack(const v4i (&s)[QG][4], v4i (&p)[QG]) {
#pragma unroll
    for (int w = 0; w < QG; ++w) p[w] = s[w][0] | s[w][1] | s[w][2] | s[w][3];
  }

  __device__ __forceinline__ void weigh(const uint32_t (&v)[NT], const v4i (&p)[QG]) {
#pragma unroll
    for (int w = 0; w < QG; ++w)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        den[w] = __builtin_amdgcn_sdot4(p[w][i], (int)kByteOnes, den[w], false);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint32_t h = v[n];
      cnt[n] += __popc(h);
      uint32_t x = h | (h << 12);
      if constexpr (FUSED) asm("v_lshl_or_b32 %0, %1, 12, %1" : "=v"(x) : "v"(h));
      const v4i va = bytes16(x);
#pragma unroll
      for (int w = 0; w < QG; ++w)
        acc[w][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(va, p[w], acc[w][n], 0, 0, 0);
    }
  }

  // the chunks jc0, jc0 + step, ... < nch (jc0 < nch).  Two chunks are in
  // work: while the weighted sum of one runs, the table reads of the next are
  // in flight, and the loads of the one after that.  Only the last chunk of
  // the context can be partial.
  __device__ __forceinline__ void run(const uint64_t* __restrict__ kb, const uint64_t* __restrict__ vb,
                                      int dw, int d, int J, int nch, int jc0, int step,
                                      const AttnLut& sLut, AttnStage<DHW>* st, int lane,
                                      int g, int c, const AttnChunk<DHW>& first,
                                      AttnChunk<DHW> nxt) {
    const char* lb = reinterpret_cast<const char*>(&sLut);
    int jc = jc0;
    AttnStage<DHW>*s0 = st, *s1 = st + 1, *s2 = st + 2;  // chunks j - 1, j, j + 1
    v4i s[QG][4], p[QG];
    uint32_t k[4], v[NT];
    put(first, *s0, lane);
    key_pieces(*s0, k, g, c);
    put(nxt, *s1, lane);
    load(nxt, kb, vb, dw, d, min(jc + 2 * step, nch - 1), lane);
    scores(k, s);
    lookup(s, lb);
    key_pieces(*s1, k, g, c);
    pack(s, p);
    for (jc += step; jc < nch; jc += step) {
      value_pieces(*s0, v, g, c);
      scores(k, s);
      __builtin_amdgcn_sched_barrier(0);
      lookup(s, lb);
      put(nxt, *s2, lane);
      load(nxt, kb, vb, dw, d, min(jc + 2 * step, nch - 1), lane);
      key_pieces(*s2, k, g, c);
      weigh(v, p);
      __builtin_amdgcn_sched_barrier(0);
      pack(s, p);
      AttnStage<DHW>* const t = s0;
      s0 = s1;
      s1 = s2;
      s2 = t;
    }
    value_pieces(*s0, v, g, c);
    const int jl = jc - step;
    if (jl * 64 + 64 > J) {  // wave-uniform
      const int nvalid = J - (jl * 64 + 16 * g);  // of this lane's 16 keys
      const uint32_t vm = nvalid >= 16 ? 0xFFFFu : (nvalid <= 0 ? 0u : ((1u << nvalid) - 1u));
      const v4i m = bytes16(vm | (vm << 12)) * 0xFF;
#pragma unroll
      for (int w = 0; w < QG; ++w) p[w] &= m;
#pragma unroll
      for (int n = 0; n < NT; ++n) v[n] &= vm;
    }
    weigh(v, p);
    finish(reinterpret_cast<char*>(st), lane, g, c);
  }

  // The wave's sums over its lane groups; sc: LDS of the wave, 64 bytes a tile.
  __device__ __forceinline__ void finish(char* sc, int lane, int g, int c) {
#pragma unroll
    for (int w = 0; w < QG; ++w) {  // over the four lane groups
      den[w] += __shfl_xor(den[w], 16);
      den[w] += __shfl_xor(den[w], 32);
    }
    // 128 * the ones of each channel over the wave's keys, added to the sums
    // of channels 16n + 4g + e (the counts change lanes through the stage)
#pragma unroll
    for (int n = 0; n < NT; ++n) cnt[n] += __shfl_xor(cnt[n], 16);
#pragma unroll
    for (int n = 0; n < NT; ++n) cnt[n] += __shfl_xor(cnt[n], 32);
#pragma unroll
    for (int n = 0; n < NT; ++n)  // the four lane groups store the same values
      *reinterpret_cast<i32_alias*>(sc + 64 * n + 4 * c) = 128 * cnt[n];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const v4i x = *reinterpret_cast<const v4i_alias*>(sc + 64 * n + 16 * g);
#pragma unroll
      for (int w = 0; w < QG; ++w) acc[w][n] += x;
    }
  }
};

// valid keys of the chunks jc0, jc0 + step, ... < nch
__device__ __forceinline__ int keys_of(int jc0, int step, int nch, int J) {
  if (jc0 >= nch) return 0;
  const int n = (nch - 1 - jc0) / step + 1;
  return n * 64 - (((nch - 1 - jc0) % step == 0) ? nch * 64 - J : 0);
}

// The neuron of 16 rows over their sums: sNum [part][t][tile][lane] (row lane%16,
// channels 16n + 4(lane/16) + e) and sDen [part][t][row].  Waves share the NT
// tiles of 16 channels; a timestep's weights are summed and inverted once for
// all tiles of a wave.  All threads of the workgroup call it.
template <int DHW, typename Args>
__device__ __forceinline__ void fire_rows(const Args& a, const v4i* sNum, const int (*sDen)[16],
                                          uint32_t (*sWord)[16][2 * DHW], int row0, int nr, int h, bool small,
                                          int tid, int nth) {
  constexpr int NT = DHW * 4, DH = DHW * 64;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), nwaves = nth >> 6;
  const int g = lane >> 4, c = lane & 15;
  const int d = a.H * DH, dw = d / 64;
  const bool vec = (reinterpret_cast<uintptr_t>(a.a_out) & 15) == 0;
  for (int i = tid; i < a.T * 32 * DHW; i += nth) (&sWord[0][0][0])[i] = 0u;
  __syncthreads();
  v4i V[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) V[j] = v4i{0, 0, 0, 0};
  for (int t = 0; t < a.T; ++t) {
    int den = 0;
    for (int p = 0; p < a.parts; ++p) den += sDen[p * a.T + t][c];
    const float den_f = (float)max(den, 1), k = attn_factor(den_f);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int n = wave + j * nwaves;
      if (n >= NT) break;  // wave-uniform
      v4i x = sNum[(t * NT + n) * 64 + lane];
      for (int p = 1; p < a.parts; ++p) x += sNum[((p * a.T + t) * NT + n) * 64 + lane];
      if (small) {  // uniform
        x = attn_norm4(x, den_f, k);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = attn_norm(x[e], den);
      }
      if (a.a_out && c < nr) {
        int32_t* o = a.a_out + ((size_t)t * a.max_rows + row0 + c) * d + h * DH + n * 16 + 4 * g;
        if (vec) {
          *reinterpret_cast<v4i*>(o) = x;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = x[e];
        }
      }
      uint32_t bits = 0u;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        V[j][e] += x[e];
        const bool s = V[j][e] >= a.theta;
        if (s) V[j][e] -= a.theta;
        bits |= (uint32_t)s << e;
      }
      atomicOr(&sWord[t][c][n >> 1], bits << (16 * (n & 1) + 4 * g));
    }
  }
  if (!a.s_out) return;  // uniform
  __syncthreads();
  for (int i = tid; i < 16 * DHW * a.T; i += nth) {
    const int k = i % DHW, m = (i / DHW) % 16, t = i / (16 * DHW);
    if (m < nr)
      a.s_out[((size_t)t * a.max_rows + row0 + m) * dw + h * DHW + k] =
          sWord[t][m][2 * k] | (uint64_t)sWord[t][m][2 * k + 1] << 32;
  }
  if (a.u_out)
    for (int i = tid; i < 16 * DHW; i += nth) {
      const int k = i % DHW, m = i / DHW;
      uint64_t uor = 0ull;
      for (int t = 0; t < a.T; ++t) uor |= sWord[t][m][2 * k] | (uint64_t)sWord[t][m][2 * k + 1] << 32;
      if (m < nr) a.u_out[(size_t)(row0 + m) * dw + h * DHW + k] = uor;
    }
}

// ---------------------------------------------------------------------------
// The neuron of one row and head: num(t) is the channel's sum, den(t) the
// weights' sum; one wave per 64 channels.  Rows of the outputs are max_rows a timestep.
// ---------------------------------------------------------------------------
template <int DHW, typename Args, typename N, typename D>
__device__ __forceinline__ void fire_row(const Args& a, int row, int h, int w, int lane, bool small, N num,
                                         D den) {
  const int dw = a.H * DHW;
  int V = 0;
  uint64_t uor = 0;
  for (int t = 0; t < a.T; ++t) {
    const int x = attn_norm1(num(t), den(t), small);
    const size_t at = ((size_t)t * a.max_rows + row) * dw + h * DHW + w;
    if (a.a_out) a.a_out[at * 64 + lane] = x;
    V += x;
    const bool s = V >= a.theta;
    if (s) V -= a.theta;
    const uint64_t word = __builtin_amdgcn_ballot_w64(s);
    uor |= word;
    if (a.s_out && lane == 0) a.s_out[at] = word;
  }
  if (a.u_out && lane == 0) a.u_out[(size_t)row * dw + h * DHW + w] = uor;
}

}  // namespace nmdlm
