// Attention on spike operands whose rows see the keys of two ranges each, with a
// bias of the scores by distance (the formulas: attn_device.h and nmdlm.h).
#include <limits.h>

#include <algorithm>

#include "attn_device.h"
#include "masked.h"
#include "pages.h"

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
  int tile;       // rows that a workgroup takes: 1, 16 or 32
  bool vec;       // the caches are 16-byte aligned
  bool spread;    // see Place
  int32_t theta;
};
constexpr int kMaskedDen = 4;    // the weights' sum behind the channels' sums, and padding
constexpr int kSplitChunks = 2;  // a split has at least this many chunks

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
// The rows of a tile together: the hulls of their two ranges, and the keys that all
// of them see by the first or by the second.  Every lane of the wave gets the same.
struct TileKeys {
  KeyRanges hull, all;
};
__device__ __forceinline__ int wave_min(int x) { return ~wave_max(~x); }
__device__ __forceinline__ TileKeys tile_keys(const MaskedArgs& a, int row0, int lane) {
  const int row = row0 + lane % a.tile;
  KeyRanges k = key_ranges(a.ranges[min(row, a.max_rows - 1)], a.n_keys);
  const bool there = row < a.max_rows, in_a = there && k.a1 > 0, in_b = there && k.b1 > 0;
  TileKeys t;
  t.hull = KeyRanges{wave_min(in_a ? k.a0 : INT_MAX), wave_max(in_a ? k.a1 : 0),
                     wave_min(in_b ? k.b0 : INT_MAX), wave_max(in_b ? k.b1 : 0)};
  if (t.hull.a1 == 0) t.hull.a0 = 0;
  if (t.hull.b1 == 0) t.hull.b0 = 0;
  // a row that is not there asks for nothing; one whose range is empty sees nothing by it
  t.all = KeyRanges{wave_max(there ? k.a0 : 0), wave_min(there ? k.a1 : INT_MAX),
                    wave_max(there ? k.b0 : 0), wave_min(there ? k.b1 : INT_MAX)};
  return t;
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

// What a wave of a workgroup takes.  HEADS: up to kHeadWaves heads of one timestep, split
// and tile, a wave each: their key rows lie in the same 128-byte lines, which the first
// wave brings into the CU's cache for all (with a head a workgroup the reads of L2, eight
// times the keys' bytes, set the pace).  Else a head and tile, wave = (timestep, part).
// Logical ids go head fastest, and the last tiles first, which see most keys where
// rows see what is before them.  In grids that fill the chip (spread) groups of up to eight
// heads of a tile go to the dies in turn: a range of tiles a die, as xcd_order has it,
// gave the first die the longest ones (2048 causal rows with a bias 94 us against 66, 2 x
// 1024 rows in blocks 51 against 45).
constexpr int kHeadWaves = 8;
struct Place {
  int h, h0, t, z, tile, part, np;  // h0: the workgroup's first head
  bool there;                       // the wave has a head
};
template <bool HEADS>
__device__ __forceinline__ Place place(const MaskedArgs& a, int wave, int nwaves) {
  const int lid = xcd_order(blockIdx.x, gridDim.x), n_tiles = (a.max_rows + a.tile - 1) / a.tile;
  if constexpr (HEADS) {
    const int hg = (a.H + nwaves - 1) / nwaves;
    const int h0 = (lid % hg) * nwaves, h = h0 + wave, r = lid / hg, tz = r % (a.T * a.splits);
    return Place{min(h, a.H - 1), h0, tz % a.T, tz / a.T, n_tiles - 1 - r / (a.T * a.splits), 0, 1, h < a.H};
  } else {
    const int t = wave / a.parts;
    if (a.spread) {  // uniform
      const int groups = (a.H + kHeadWaves - 1) / kHeadWaves, gs = (a.H + groups - 1) / groups;
      const int slot = (int)blockIdx.x / kXcds, u = slot / gs * kXcds + (int)blockIdx.x % kXcds;
      const int h = u % groups * gs + slot % gs, tile = n_tiles - 1 - u / groups;
      return Place{h, h, t, 0, tile, wave - t * a.parts, a.parts, tile >= 0 && h < a.H};
    }
    return Place{lid % a.H, lid % a.H, t, 0, n_tiles - 1 - lid / a.H, wave - t * a.parts, a.parts, true};
  }
}

// ---------------------------------------------------------------------------
// k_masked_rows: single rows.  HEADS: a workgroup takes one timestep and one of the
// row's splits, wave = head, and leaves the sums to k_masked_join; else one head, wave =
// (timestep, part), and the neuron.  Bit by bit:
// lane = key for the scores (popcount of the key's row and the query, the same
// for all lanes), the weight's eight bits become eight 64-key masks by ballots,
// and with lane = channel
//     sum_j p_j V[j,c] = sum_b 2^b popcount(mask_b AND word of channel c).
// A key that the row does not see weighs 0.
//
// HEADS: the waves bring a chunk's key rows into LDS together, 8 rows of all their heads
// each, one barrier a chunk, two buffers.  (Each wave reading its own pieces counted
// on the CU's cache to keep the lines for the others: 80 us a call of 130 thousand keys, 16
// heads of 128, T = 4, where 92 with four chunks of loads on their way in place of two: they
// no longer fitted.)  That call takes 57 to 66 us of the kernel and 8 of the join: 268 MB at
// 4.1 to 4.7 TB/s, where a plain read has 6.3; what is missing is at the chunk's barrier,
// where all waves wait for the slowest load.  One row of 300 keys, 5.5 us, is a chain
// of trips to memory: arguments, ranges, query, keys, values.
// ---------------------------------------------------------------------------
constexpr int kRowWaves = 12;  // of a workgroup at most

template <int DHW>
struct RowValues {
  uint64_t v[DHW];  // channels DHW * lane (and + 1)
  int pos;          // the position of key `lane` (with a bias)
};
// DHW words from 8-byte aligned memory, at once where vec says that it is 16-byte aligned
template <int DHW>
__device__ __forceinline__ void load_words(uint64_t (&r)[DHW], const uint64_t* p, bool vec) {
  typedef const ulonglong2 __attribute__((may_alias)) pair;
  if (DHW == 2 && vec) {  // uniform
    const ulonglong2 x = *reinterpret_cast<pair*>(p);
    r[0] = x.x;
    r[DHW - 1] = x.y;
  } else {
#pragma unroll
    for (int w = 0; w < DHW; ++w) r[w] = p[w];
  }
}

template <int DHW, bool HEADS>
__global__ __launch_bounds__(64 * kRowWaves) void k_masked_rows(MaskedArgs a) {
  constexpr int DH = 64 * DHW;
  constexpr int kKeyLd = DHW * (kHeadWaves + 1);  // words of a key in LDS, a head of padding
  __shared__ uint8_t sLut[256];
  __shared__ int8_t sBiasAll[HEADS ? kHeadWaves : 1][2 * NMDLM_MAX_DIST + 4];
  __shared__ int sNum[HEADS ? 1 : NMDLM_MAX_T][DH];
  __shared__ int sDen[NMDLM_MAX_T];
  __shared__ __attribute__((aligned(16))) uint64_t sKeys[HEADS ? 2 : 1][HEADS ? 64 * kKeyLd : 1];
  const int nth = blockDim.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nwaves = nth >> 6;
  const Place pl = place<HEADS>(a, wave, nwaves);
  const int h = pl.h, t = pl.t, part = pl.part, np = pl.np, row = pl.tile;
  const KeyRanges kr = key_ranges(a.ranges[row], a.n_keys);
  const ChunkList cl = chunk_list(kr);
  const int splits = HEADS ? split_count(a, cl.n) : 1;
  if (pl.z >= splits) return;  // uniform
  const int i0 = split_at(cl.n, pl.z, splits), i1 = split_at(cl.n, pl.z + 1, splits);
  const int d = a.H * DH, dw = d / 64;
  const uint64_t* kt = a.kc + (size_t)t * a.cap * dw;
  const uint64_t* vb = a.vt + (size_t)t * (a.cap / 64) * d + h * DH;
  const uint64_t* qp = a.q + ((size_t)t * a.max_rows + row) * dw + h * DHW;
  // HEADS: key row `wave * 8 + lane / 8` (of eight waves) of head `lane % 8` of the group, for
  // all of the workgroup's waves; else the wave's own, row `lane`
  const int my_head = HEADS ? min(pl.h0 + lane % kHeadWaves, a.H - 1) : h;
  auto load_keys = [&](uint64_t (&k)[DHW], int i, int row8) __attribute__((always_inline)) {
    const int jc = cl.at(min(i, i1 - 1));
    load_words<DHW>(k, kt + (size_t)jc * 64 * dw + (uint32_t)(row8 * dw + my_head * DHW), a.vec);
  };
  auto load = [&](int i) __attribute__((always_inline)) {
    RowValues<DHW> r;
    const int jc = cl.at(min(i, i1 - 1));
    load_words<DHW>(r.v, vb + (size_t)jc * d + (uint32_t)(lane * DHW), a.vec);
    r.pos = a.bias ? a.k_pos[min(64 * jc + lane, a.n_keys - 1)] : 0;
    return r;
  };
  // rows of a chunk that this wave brings: all 64 over the waves there are
  constexpr int kPieces = HEADS ? 8 : 1;  // at most (one wave: eight times 8 rows)
  uint64_t keys[2][HEADS ? 1 : DHW];      // without HEADS: two chunks on their way
  uint64_t piece[kPieces][DHW];
  RowValues<DHW> val[2];
  auto load_pieces = [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < kPieces; ++n) {
      const int r = (n * nwaves + wave) * 8 + lane / kHeadWaves;
      if (n * nwaves * 8 < 64) load_keys(piece[n], i, min(r, 63));  // uniform
    }
  };
  auto put_pieces = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < kPieces; ++n) {
      const int r = (n * nwaves + wave) * 8 + lane / kHeadWaves;
      if (n * nwaves * 8 < 64 && r < 64) {
#pragma unroll
        for (int w = 0; w < DHW; ++w) sKeys[HEADS ? buf : 0][HEADS ? r * kKeyLd + (lane % kHeadWaves) * DHW + w : 0] = piece[n][w];
      }
    }
  };
  if (i0 < i1) {  // uniform
    if constexpr (HEADS) load_pieces(i0);
    else {
      load_keys(keys[0], i0 + part, lane);
      load_keys(keys[1], i0 + part + np, lane);
    }
    val[0] = load(i0 + part);
    val[1] = load(i0 + part + np);
  }
  uint64_t q[DHW];
#pragma unroll
  for (int w = 0; w < DHW; ++w) q[w] = qp[w];
  const int D = a.max_dist, q_pos = a.bias ? a.q_pos[row] : 0;
  int8_t* const sBias = sBiasAll[HEADS ? wave : 0];
  for (int i = tid; i < 256; i += nth) sLut[i] = a.lut[i];
  if (a.bias)
    for (int i = HEADS ? lane : tid; i < 2 * D + 1; i += HEADS ? 64 : nth)
      sBias[i] = a.bias[(size_t)h * (2 * D + 1) + i];
  if constexpr (!HEADS) {
    for (int i = tid; i < a.T * DH; i += nth) (&sNum[0][0])[i] = 0;
    if (tid < a.T) sDen[tid] = 0;
  } else if (i0 < i1) {
    put_pieces(0);
    load_pieces(i0 + 1);
  }
  __syncthreads();

  int acc[8][DHW], den = 0;
#pragma unroll
  for (int b = 0; b < 8; ++b)
#pragma unroll
    for (int w = 0; w < DHW; ++w) acc[b][w] = 0;
  auto weigh = [&](const uint64_t (&k)[DHW], const RowValues<DHW>& r, int jc) __attribute__((always_inline)) {
    const int j = 64 * jc + lane;
    int s = 0;
#pragma unroll
    for (int w = 0; w < DHW; ++w) s += (int)__popcll(k[w] & q[w]);
    const bool seen = (j >= kr.a0 && j < kr.a1) || (j >= kr.b0 && j < kr.b1);
    if (a.bias) {
      const int off = __builtin_elementwise_sub_sat(q_pos, r.pos);
      s = min(max(s + sBias[min(max(off, -D), D) + D], 0), 255);
    }
    const int p = seen ? sLut[s] : 0;
    den += p;
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const uint64_t mask = __builtin_amdgcn_ballot_w64((p >> b) & 1);
#pragma unroll
      for (int w = 0; w < DHW; ++w) acc[b][w] += (int)__popcll(r.v[w] & mask);
    }
  };
  for (int i = i0 + part; i < i1; i += 2 * np) {  // wave-uniform; HEADS: uniform
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int e = i + n * np;
      if (e < i1) {
        if constexpr (HEADS) {
          put_pieces((e - i0 + 1) & 1);  // the next chunk's, whose readers of two chunks ago are through
          load_pieces(e + 2);
          uint64_t k[DHW];
#pragma unroll
          for (int w = 0; w < DHW; ++w) k[w] = sKeys[(e - i0) & 1][lane * kKeyLd + wave * DHW + w];
          weigh(k, val[n], cl.at(e));
          val[n] = load(e + 2);
          __syncthreads();
        } else {
          uint64_t k[DHW];
#pragma unroll
          for (int w = 0; w < DHW; ++w) k[w] = keys[n][HEADS ? 0 : w];
          weigh(k, val[n], cl.at(e));
          if constexpr (!HEADS) load_keys(keys[n], e + 2 * np, lane);
          val[n] = load(e + 2 * np);
        }
      }
    }
  }
  den = wave_sum(den);
  int num[DHW];
#pragma unroll
  for (int w = 0; w < DHW; ++w) {
    num[w] = 0;
#pragma unroll
    for (int b = 7; b >= 0; --b) num[w] = 2 * num[w] + acc[b][w];
  }
  if constexpr (HEADS) {
    if (!pl.there) return;  // wave-uniform
    int32_t* o = split_sums<DHW>(a, row, h, pl.z) + (size_t)t * (DH + kMaskedDen);
#pragma unroll
    for (int w = 0; w < DHW; ++w) o[DHW * lane + w] = num[w];
    if (lane == 0) o[DH] = den;
    return;
  }
  if (lane == 0) atomicAdd(&sDen[t], den);
#pragma unroll
  for (int w = 0; w < DHW; ++w) atomicAdd(&sNum[HEADS ? 0 : t][DHW * lane + w], num[w]);
  __syncthreads();
  for (int w = wave; w < DHW; w += nwaves)
    fire_row<DHW>(a, row, h, w, lane, a.n_keys < 65536, [&](int tt) { return sNum[HEADS ? 0 : tt][w * 64 + lane]; },
                  [&](int tt) { return sDen[tt]; });
}

// ---------------------------------------------------------------------------
// k_masked_tiles: a tile of 16*QG rows, the sums and the pipeline of attn_device.h over the
// chunks that any row of the tile sees.  HEADS: wave = head of one timestep and split,
// the sums go to k_masked_join; else wave = (timestep, part) of one head, and the neuron.
// A chunk that not all of them see whole is masked: a lane (one row, 16 keys) makes
// the bits of its keys from the row's ranges, and the weights of the others become 0
// (byte -128).  The values of the keys past n_keys in the last chunk then count with
// weight 0 too.
//
// Bias: the scores' sums begin with 8 * bias, so it costs no instruction behind the
// products; the table is extended by 128 entries below and above, which clamps.  A
// chunk whose keys are all at least max_dist before (or behind) all rows of the tile
// has one bias for all pairs.  Where a chunk's positions are consecutive a lane's 16
// keys take 16 consecutive entries of the bias, reversed and extended by 16 on each
// side: one clamped index for all of them.
//
// Bound by the instructions issued at two waves a SIMD: 266 vector instructions a chunk of
// 32 rows (key and value bits made bytes, table bytes packed, addresses), 1170 before and
// behind a tile's chunks.  2 x 1024 rows in blocks 45 us (0.8 POP/s of what the rows see),
// 2048 causal rows with a bias 66 us, 18 rows x 65 thousand keys 51 and 10 of the join.  34
// rows x 1058 keys, 14 us, fill 48 of 256 CUs (sixteen waves a workgroup there: 17.2).
// ---------------------------------------------------------------------------
constexpr int kWideEntries = 384;  // scores -128 .. 255
constexpr int kBiasPad = 16;
// How a staged chunk's keys lie to the rows: all max_dist or more before or behind, at
// positions in a row from `base` on, or anyhow.
enum Side : int { SIDE_ANY, SIDE_ROW, SIDE_BEFORE, SIDE_BEHIND };
struct ChunkSide {
  Side side;
  int base;
};
struct WideLut {
  int e[2][kWideEntries][2];
};
template <bool BIAS>
struct MaskedLut {
  AttnLut lut;
};
template <>
struct MaskedLut<true> {
  WideLut lut;
};

template <int DHW, int QG>
__device__ __forceinline__ void add_scores(const v4i (&q)[QG][DHW], const uint32_t (&k)[4], v4i (&s)[QG][4]) {
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
    for (int w = 0; w < QG; ++w) s[w][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k0, q[w][0], s[w][u], 0, 0, 0);
    if constexpr (DHW == 2) {
#pragma unroll
      for (int w = 0; w < QG; ++w) s[w][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k1, q[w][1], s[w][u], 0, 0, 0);
    }
  }
}

// bits [lo, hi) of 16
__device__ __forceinline__ uint32_t bits16(int lo, int hi) {
  return ((1u << min(max(hi, 0), 16)) - 1u) & ~((1u << min(max(lo, 0), 16)) - 1u);
}

template <int DHW, int QG, bool BIAS, bool HEADS>
__global__ __launch_bounds__(64 * NMDLM_MAX_T, QG == 1 ? 4 : 2) void k_masked_tiles(MaskedArgs a) {
  constexpr int NT = DHW * 4, DH = DHW * 64;
  constexpr int kHalf = (BIAS ? kWideEntries : kLutEntries) * 8;  // bytes of half a table
  __shared__ MaskedLut<BIAS> sLut;
  __shared__ int sDen[NMDLM_MAX_T][16];  // [part][T], at most eight waves
  __shared__ uint32_t sWord[NMDLM_MAX_T][16][2 * DHW];
  __shared__ int sPos[BIAS ? NMDLM_MAX_T * kAttnStages : 1][64];  // positions of the staged keys
  // the waves' stages, then (without HEADS) their sums [part][T][NT][64]; behind them 8 * bias
  extern __shared__ v4i sNum[];
  AttnStage<DHW>* sStage = reinterpret_cast<AttnStage<DHW>*>(sNum);

  const int nth = blockDim.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nwaves = nth >> 6;
  const int g = lane >> 4, c = lane & 15;
  const Place pl = place<HEADS>(a, wave, nwaves);
  if (!HEADS && !pl.there) return;  // uniform
  const int h = pl.h, t = pl.t, part = pl.part, np = pl.np, row0 = pl.tile * 16 * QG;
  const int nr = min(a.max_rows - row0, 16 * QG);
  const int d = a.H * DH, dw = d / 64, D = a.max_dist;
  const uint64_t* kb = a.kc + (size_t)t * a.cap * dw + h * DHW;
  const uint64_t* vb = a.vt + (size_t)t * (a.cap / 64) * d + h * DH;

  uint32_t qraw[QG];
  AttnWave<DHW, QG>::load_queries(qraw, a.q + ((size_t)t * a.max_rows + row0) * dw + h * DHW, dw, 0, nr - 1, g, c);
  KeyRanges kr[QG];
  int qp[QG];
#pragma unroll
  for (int u = 0; u < QG; ++u) {
    const int row = min(row0 + 16 * u + c, a.max_rows - 1);
    kr[u] = key_ranges(a.ranges[row], a.n_keys);
    qp[u] = BIAS ? a.q_pos[row] : 0;
  }
  const TileKeys tk = tile_keys(a, row0, lane);
  const ChunkList cl = chunk_list(tk.hull);
  const int splits = HEADS ? split_count(a, cl.n) : 1;
  if (pl.z >= splits) return;  // uniform
  const int i0 = split_at(cl.n, pl.z, splits);
  const int i1 = pl.there ? split_at(cl.n, pl.z + 1, splits) : i0;
  int* const sBias = HEADS ? reinterpret_cast<int*>(sStage + kAttnStages * nwaves) + wave * (2 * D + 2 * kBiasPad)
                           : reinterpret_cast<int*>(sNum + nwaves * NT * 64);
  int q_lo = 0, q_hi = 0;
  constexpr int kSmallPos = 1 << 29;  // differences of such positions fit
  bool small_pos = true;
  if constexpr (BIAS) {
    q_lo = q_hi = qp[0];
#pragma unroll
    for (int u = 1; u < QG; ++u) {
      q_lo = min(q_lo, qp[u]);
      q_hi = max(q_hi, qp[u]);
    }
    q_lo = wave_min(q_lo);
    q_hi = wave_max(q_hi);
    small_pos = q_lo >= -kSmallPos && q_hi <= kSmallPos;
    // entry i: key behind the row by i - D - kBiasPad
    for (int i = HEADS ? lane : tid; i < 2 * D + 2 * kBiasPad; i += HEADS ? 64 : nth)
      sBias[i] = 8 * a.bias[(size_t)h * (2 * D + 1) + min(max(D + kBiasPad - i, -D), D) + D];
    for (int i = tid; i < kWideEntries; i += nth) {
      const uint32_t v = (uint32_t)a.lut[min(max(i - 128, 0), 255)] ^ 0x80u;
#pragma unroll
      for (int b = 0; b < 4; ++b) sLut.lut.e[b >> 1][i][b & 1] = (int)(v << (8 * b));
    }
  } else {
    fill_lut(sLut.lut, load_lut(a.lut, tid, nth), tid, nth);
  }
  AttnWave<DHW, QG> w;
  w.init(qraw);
  __syncthreads();

  const char* lb = reinterpret_cast<const char*>(&sLut) + (BIAS ? 128 * 8 : 0);
  AttnStage<DHW>* const st = &sStage[kAttnStages * wave];
  int keys = 0;
  if (i0 + part < i1) {  // wave-uniform
    // as AttnWave::run: the weighted sum of one chunk while the table reads of the
    // next are in flight, and the loads of the one after that
    auto chunk_at = [&](int i) { return cl.at(min(i, i1 - 1)); };
    int kp = 0;  // the position of key `lane` of the chunk in `next`
    auto load = [&](AttnChunk<DHW>& ch, int jc) {
      AttnWave<DHW, QG>::load(ch, kb, vb, dw, d, jc, lane);
      if constexpr (BIAS) kp = a.k_pos[min(64 * jc + lane, a.n_keys - 1)];
    };
    auto put = [&](const AttnChunk<DHW>& ch, AttnStage<DHW>& s, int slot, int jc) {
      ChunkSide cs{SIDE_ANY, 0};
      if constexpr (BIAS) {
        cs.base = __builtin_amdgcn_readfirstlane(kp);
        const bool before = __builtin_elementwise_sub_sat(q_lo, kp) >= D;
        const bool behind = __builtin_elementwise_sub_sat(q_hi, kp) <= -D;
        const bool in_row = kp - lane == cs.base || 64 * jc + lane >= a.n_keys;
        if (__builtin_amdgcn_ballot_w64(before) == ~0ull) cs.side = SIDE_BEFORE;
        else if (__builtin_amdgcn_ballot_w64(behind) == ~0ull) cs.side = SIDE_BEHIND;
        else if (small_pos && cs.base == max(min(cs.base, kSmallPos), -kSmallPos) &&
                 __builtin_amdgcn_ballot_w64(in_row) == ~0ull)
          cs.side = SIDE_ROW;
        else
          sPos[kAttnStages * wave + slot][lane] = kp;
      }
      w.put(ch, s, lane);
      return cs;
    };
    v4i s[QG][4], p[QG];
    auto biased = [&](int slot, ChunkSide cs) {  // what the scores begin with
      if (cs.side == SIDE_BEFORE || cs.side == SIDE_BEHIND) {  // wave-uniform
        const int b = sBias[cs.side == SIDE_BEFORE ? kBiasPad : 2 * D + kBiasPad];
#pragma unroll
        for (int u = 0; u < QG; ++u)
#pragma unroll
          for (int k = 0; k < 4; ++k) s[u][k] = v4i{b, b, b, b};
      } else if (cs.side == SIDE_ROW) {
#pragma unroll
        for (int u = 0; u < QG; ++u) {
          const int* b = sBias + min(max(cs.base + 16 * g - qp[u], -D - kBiasPad), D) + D + kBiasPad;
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[u][k][e] = b[4 * k + e];
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const v4i pos = *reinterpret_cast<const v4i*>(&sPos[kAttnStages * wave + slot][16 * g + 4 * k]);
#pragma unroll
          for (int u = 0; u < QG; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int off = __builtin_elementwise_sub_sat(pos[e], qp[u]);
              s[u][k][e] = sBias[min(max(off, -D), D) + D + kBiasPad];
            }
        }
      }
    };
    auto score = [&](const uint32_t (&k)[4], int slot, ChunkSide cs) {
      if constexpr (BIAS) {
        biased(slot, cs);
        add_scores<DHW, QG>(w.q, k, s);
      } else {
        w.scores(k, s);
      }
    };
    auto lookup = [&]() {
#pragma unroll
      for (int u = 0; u < QG; ++u)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int b = k == 1 ? 2 : (k == 2 ? 1 : k);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[u][k][e] = *reinterpret_cast<const int*>(lb + kHalf * (b >> 1) + 4 * (b & 1) + s[u][k][e]);
        }
    };
    auto masked = [&](int jc) {  // weight 0 for the keys that a row does not see
      const int j0 = 64 * jc, j1 = j0 + 64;
      if ((j0 >= tk.all.a0 && j1 <= tk.all.a1) || (j0 >= tk.all.b0 && j1 <= tk.all.b1)) return;  // uniform
      const int j = j0 + 16 * g;
#pragma unroll
      for (int u = 0; u < QG; ++u) {
        const uint32_t vm = bits16(kr[u].a0 - j, kr[u].a1 - j) | bits16(kr[u].b0 - j, kr[u].b1 - j);
        const v4i m = bytes16(vm | (vm << 12)) * 0xFF;
        p[u] = (p[u] & m) | (~m & (int)0x80808080u);
      }
    };
    uint32_t k[4], v[NT];
    AttnChunk<DHW> first, next;
    int i = i0 + part, s0 = 0, s1 = 1, s2 = 2;  // the stages of chunks i - np, i, i + np
    load(first, chunk_at(i));
    ChunkSide d0 = put(first, st[s0], s0, chunk_at(i)), d1, d2;  // how they lie
    load(next, chunk_at(i + np));
    w.key_pieces(st[s0], k, g, c);
    d1 = put(next, st[s1], s1, chunk_at(i + np));
    load(next, chunk_at(i + 2 * np));
    score(k, s0, d0);
    lookup();
    w.key_pieces(st[s1], k, g, c);
    w.pack(s, p);
    masked(cl.at(i));
    for (i += np; i < i1; i += np) {  // wave-uniform
      w.value_pieces(st[s0], v, g, c);
      score(k, s1, d1);
      __builtin_amdgcn_sched_barrier(0);
      lookup();
      d2 = put(next, st[s2], s2, chunk_at(i + np));
      load(next, chunk_at(i + 2 * np));
      w.key_pieces(st[s2], k, g, c);
      keys += 64;
      w.weigh(v, p);
      __builtin_amdgcn_sched_barrier(0);
      w.pack(s, p);
      masked(cl.at(i));
      const int tmp = s0;
      s0 = s1;
      s1 = s2;
      s2 = tmp;
      d1 = d2;
    }
    w.value_pieces(st[s0], v, g, c);
    keys += 64;
    w.weigh(v, p);
  }
  w.finish(reinterpret_cast<char*>(st), lane, g, c);
  if constexpr (HEADS) {
    if (!pl.there) return;  // wave-uniform
#pragma unroll
    for (int u = 0; u < QG; ++u)
      if (16 * u + c < nr) {
        int32_t* o = split_sums<DHW>(a, row0 + 16 * u + c, h, pl.z) + (size_t)t * (DH + kMaskedDen);
#pragma unroll
        for (int n = 0; n < NT; ++n) *reinterpret_cast<v4i*>(o + 16 * n + 4 * g) = w.acc[u][n];
        if (g == 0) o[DH] = w.den[u] + 128 * keys;
      }
    return;
  }
  __syncthreads();  // the stages are read

#pragma unroll
  for (int u = 0; u < QG; ++u) {
    if (u > 0) __syncthreads();  // the sums and words of the group before are read
    const int rows = nr - 16 * u, pt = part * a.T + t;
#pragma unroll
    for (int n = 0; n < NT; ++n) sNum[(pt * NT + n) * 64 + lane] = w.acc[u][n];
    if (g == 0) sDen[pt][c] = w.den[u] + 128 * keys;
    __syncthreads();
    if (rows <= 0) continue;  // uniform
    fire_rows<DHW>(a, sNum, sDen, sWord, row0 + 16 * u, min(rows, 16), h, a.n_keys < 65536, tid, nth);
  }
}

// k_masked_join: the sums of a row's splits (integers: any order gives the same)
// and the neuron.  A workgroup per row and head, kJoinWaves / (T DHW) waves for each
// timestep and 64 channels, which take the splits in turn, sixteen loads at once.
constexpr int kJoinWaves = 16;
template <int DHW>
__global__ __launch_bounds__(64 * kJoinWaves) void k_masked_join(MaskedArgs a) {
  constexpr int LD = 64 * DHW + kMaskedDen;
  __shared__ int sNum[NMDLM_MAX_T][64 * DHW];
  __shared__ int sDen[NMDLM_MAX_T];
  const int h = blockIdx.x % a.H, row = blockIdx.x / a.H;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tw = a.T * DHW, nz = (int)blockDim.x / 64 / tw;  // waves of a timestep's 64 channels
  const int t = wave % tw / DHW, w = wave % DHW, z0 = wave / tw;
  for (int i = tid; i < a.T * 64 * DHW; i += blockDim.x) (&sNum[0][0])[i] = 0;
  const int n = split_count(a, chunk_list(tile_keys(a, row - row % a.tile, lane).hull).n);
  const int32_t* base = split_sums<DHW>(a, row, h, 0) + (size_t)t * LD;
  const size_t ld = (size_t)a.T * LD;
  int den = 0;
  if (w == 0 && z0 == 0)  // wave-uniform
    for (int z = lane; z < n; z += 64) den += base[z * ld + 64 * DHW];
  int x = 0;
  for (int z = z0; z < n; z += 16 * nz) {
    int v[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = base[min(z + k * nz, n - 1) * ld + w * 64 + lane];
#pragma unroll
    for (int k = 0; k < 16; ++k) x += z + k * nz < n ? v[k] : 0;
  }
  __syncthreads();
  atomicAdd(&sNum[t][w * 64 + lane], x);
  if (w == 0 && z0 == 0) {
    den = wave_sum(den);
    if (lane == 0) sDen[t] = den;
  }
  __syncthreads();
  if (wave < DHW)
    fire_row<DHW>(a, row, h, wave, lane, a.n_keys < 65536,
                  [&](int tt) { return sNum[tt][wave * 64 + lane]; }, [&](int tt) { return sDen[tt]; });
}

// Which kernel and grid; the ranges are on the device, the rule sees the sizes.  Measured in
// graphs with spikes out, T = 4, H = 16, dh = 128 unless said, us by heads / in one kernel:
//  * By heads (a second launch joins the sums) where a wave's walk of all keys would be
//    long and few workgroups would make it, the more rows the longer, since each row's sums
//    go through memory: 1 row x 1000 keys 11.3 / 8.1, x 2000 11.2 / 11.7, x 8000 15 / 49; 4 rows
//    x 450 12.0 / 10.2, x 1000 12.1 / 13.4; 18 x 1000 16.6 / 13.4, x 2000 19 / 20, x 4000 21 / 32;
//    34 x 2000 23 / 20, x 4000 24 / 32; 66 x 2000 28 / 21, x 8000 37 / 56; 130 x 4000 43 / 35, x
//    16000 72 / 104; 250 (16 tiles, a workgroup a CU without) x 16000 104 / 109.  T = 8, H = 8, dh =
//    64: 18 x 1000 13 / 15; T = 1, H = 4: 1 x 1500 8.7 / 5.2, x 6000 9.2 / 11.4, 18 x 1500 11 / 8.3.
//  * 32 rows a wave where the tiles give 1024 such waves (2 x 1024 rows in blocks 45 against
//    58 with 16, 2048 causal rows with a bias 66 against 84), by heads where fewer keys are
//    expanded so: a chunk costs 155 for 16 rows and 200 for 32 (18 rows x 65 thousand keys
//    62 against 88).
//  * Splits to fill the chip: 18 x 65 thousand keys, 16, 32 and 64 splits 91, 62 and 75; one
//    row x 130 thousand, 32, 64 and 128 splits 85, 67 and 75.
MaskedRoute masked_route(int T, int M, int n_keys, int H) {
  MaskedRoute r{1, T <= 2 ? 4 : (T <= 4 ? 2 : 1), 1, false};
  if (M > 2) r.tile = M >= 32 && (long long)(M / 32) * H * T >= 1024 ? 32 : 16;
  if (r.tile == 1) r.parts = std::max(std::min(kRowWaves / T, 4), 1);
  if (r.tile == 32) r.parts = 1;
  const long long wgs = (long long)((M + r.tile - 1) / r.tile) * H;
  const int walk = (n_keys + 63) / 64 / r.parts;
  if (wgs >= 256 || walk <= (r.tile == 1 ? 11 : 8 + M / 3)) return r;
  r.heads = true;
  r.parts = 1;
  if (r.tile > 1) r.tile = ((M + 15) / 16) * 155 <= ((M + 31) / 32) * 200 ? 16 : 32;
  const long long units = (long long)((M + r.tile - 1) / r.tile) * ((H + kHeadWaves - 1) / kHeadWaves) * T;
  r.splits = (int)std::max(1LL, std::min<long long>({(r.tile == 32 ? 256 : 512) / units, 64,
                                                     n_keys / (64 * kSplitChunks)}));
  return r;
}

size_t masked_attn_ws(int T, int M, int n_keys, int H, int dh) {
  const MaskedRoute r = masked_route(T, M, n_keys, H);
  if (!r.heads) return 0;
  return align_up((size_t)M * H * r.splits * T * (dh + kMaskedDen) * sizeof(int32_t), 256);
}

constexpr unsigned kSpreadGroups = 64;
constexpr size_t kMaskedPlainLds = 32768;  // dynamic LDS that needs no attribute beside the static

template <int DHW, int QG, bool BIAS, bool HEADS>
static nmdlm_status launch_tiles(const MaskedArgs& a, unsigned grid, int waves, hipStream_t st) {
  size_t dyn = (size_t)waves * (HEADS ? kAttnStages * sizeof(AttnStage<DHW>) : DHW * 4 * 64 * sizeof(v4i));
  static_assert(DHW * 4 * 64 * sizeof(v4i) >= kAttnStages * sizeof(AttnStage<DHW>), "sums over the stages");
  if (BIAS) dyn += (size_t)(HEADS ? waves : 1) * (2 * a.max_dist + 2 * kBiasPad) * sizeof(int);
  if (dyn > kMaskedPlainLds &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(&k_masked_tiles<DHW, QG, BIAS, HEADS>),
                          hipFuncAttributeMaxDynamicSharedMemorySize, (int)dyn) != hipSuccess)
    return NMDLM_ERR_HIP;
  hipLaunchKernelGGL((k_masked_tiles<DHW, QG, BIAS, HEADS>), dim3(grid), dim3(64 * waves), (uint32_t)dyn, st, a);
  return hip_status();
}

template <int DHW, bool HEADS>
static nmdlm_status launch_masked(MaskedArgs a, hipStream_t st) {
  const int waves = HEADS ? std::min(a.H, kHeadWaves) : a.T * a.parts;
  const unsigned tiles = (a.max_rows + a.tile - 1) / a.tile;
  const unsigned groups = (a.H + kHeadWaves - 1) / kHeadWaves, gs = (a.H + groups - 1) / groups;
  a.spread = !HEADS && a.tile > 1 && tiles * groups >= kSpreadGroups;
  const unsigned grid = HEADS      ? tiles * ((a.H + waves - 1) / waves) * a.T * a.splits
                        : a.spread ? (tiles * groups + kXcds - 1) / kXcds * kXcds * gs
                                   : tiles * a.H;
  if (a.tile == 1) {
    hipLaunchKernelGGL((k_masked_rows<DHW, HEADS>), dim3(grid), dim3(64 * waves), 0, st, a);
    return hip_status();
  }
  if (a.tile == 16)
    return a.bias ? launch_tiles<DHW, 1, true, HEADS>(a, grid, waves, st)
                  : launch_tiles<DHW, 1, false, HEADS>(a, grid, waves, st);
  return a.bias ? launch_tiles<DHW, 2, true, HEADS>(a, grid, waves, st)
                : launch_tiles<DHW, 2, false, HEADS>(a, grid, waves, st);
}

template <int DHW>
static nmdlm_status launch_masked_dh(const MaskedAttnCall& c, hipStream_t st) {
  const MaskedRoute r = masked_route(c.T, c.M, c.n_keys, c.H);
  const MaskedArgs a{c.q, c.k_cache, c.vt_cache, c.cap, reinterpret_cast<const int4*>(c.mask.ranges),
                     c.mask.q_pos, c.mask.k_pos, c.bias, c.lut, c.a_out, c.s_out, c.u_out,
                     static_cast<int32_t*>(c.ws), c.n_keys, c.M, c.T, c.H, r.parts, r.splits,
                     c.bias ? c.mask.max_dist : 0, r.tile,
                     ((reinterpret_cast<uintptr_t>(c.k_cache) | reinterpret_cast<uintptr_t>(c.vt_cache)) & 15) == 0,
                     false, c.theta};
  if (!r.heads) return launch_masked<DHW, false>(a, st);
  const nmdlm_status rc = launch_masked<DHW, true>(a, st);
  if (rc != NMDLM_OK) return rc;
  const int tw = c.T * DHW, nz = std::max(1, std::min(kJoinWaves / tw, (r.splits + 15) / 16));
  hipLaunchKernelGGL(k_masked_join<DHW>, dim3((unsigned)c.M * c.H), dim3(64 * tw * nz), 0, st, a);
  return hip_status();
}

nmdlm_status launch_masked_attn(const MaskedAttnCall& c, hipStream_t st) {
  return c.dh == 64 ? launch_masked_dh<1>(c, st) : launch_masked_dh<2>(c, st);
}

}  // namespace nmdlm
