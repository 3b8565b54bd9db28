// Attention on spike operands over paged caches: the formulas of attn_device.h
// for the packed rows of a plan, over all pages of a request or those selected
// for each row and head.
#include <algorithm>

#include "attn_device.h"
#include "pages.h"

namespace nmdlm {

// ---------------------------------------------------------------------------
// Pages of a request go to its splits as contiguous ranges.  A workgroup lists
// the pages of its range in LDS, kPageList at a time: all of them, or those that
// one of its rows selected.
// ---------------------------------------------------------------------------
constexpr int kPageList = 256;   // pages of a range that are listed at once
constexpr int kSplitPages = 8;   // a split has at least this many pages

struct PagedArgs {
  const PageTile* tiles;
  const int32_t* table;
  const uint64_t* q;
  const uint64_t* kp;
  const uint64_t* vp;
  const uint8_t* lut;
  const uint64_t* sel;
  int32_t* a_out;
  uint64_t* s_out;
  uint64_t* u_out;
  int32_t* part;  // sums of the splits [row][head][split][T][64 DHW + kPartDen]
  int max_pages, pool, max_rows, words;
  int T, H, parts, splits;
  int32_t theta;
};
constexpr int kPartDen = 4;  // the weights' sum behind the channels' sums, and padding

struct PageEntry {
  int id, keys;  // pool page, keys of it that count (0 outside the pool)
};

// Splits of a request of nP pages.
__device__ __forceinline__ int split_count(const PagedArgs& a, int nP) {
  return min(a.splits, max(nP / kSplitPages, 1));
}
struct PageRange {
  int p0, p1;
};
__device__ __forceinline__ PageRange split_range(int nP, int z, int n) {
  return PageRange{(int)((long long)nP * z / n), (int)((long long)nP * (z + 1) / n)};
}
__device__ __forceinline__ PageEntry page_entry(const PagedArgs& a, const int32_t* tab, int p, int J) {
  const int id = tab[p];
  const bool there = (unsigned)id < (unsigned)a.pool;
  return PageEntry{there ? id : 0, there ? min(64, J - 64 * p) : 0};
}
template <int DHW>
__device__ __forceinline__ int32_t* split_sums(const PagedArgs& a, int row, int h, int z) {
  return a.part + (((size_t)row * a.H + h) * a.splits + z) * a.T * (64 * DHW + kPartDen);
}
// ---------------------------------------------------------------------------
// k_paged_attn: a workgroup takes one tile of 16*QG rows, a head and one of the
// tile's splits; wave = (timestep, part).  A page is the 64-key chunk of a wave
// (attn_device.h).  With a selection an entry of the list has one bit per row
// that sees the page (a score that a row does not see weighs 0, byte -128).  The
// parts of a timestep take the list's entries in turn.
//
// Bound by instruction issue: a page and 16 rows cost 173 vector instructions, 16
// MFMAs and 32 LDS instructions (vector 72% of the busy cycles, matrix cores 27%, LDS
// 50%).  T = 4, 16 heads of 128: 32 requests x 16 rows x 2016 keys 34 us, 4.0 TB/s and
// 1.0 POP/s; 32 rows a wave, 3 x 2048 x 2048 243 us, 1.7 POP/s (one request 92 us,
// where the contiguous cache's kernel takes 87).
// ---------------------------------------------------------------------------

// One wave's loads of a page: key row `lane`, value words of channels lane (and
// lane + 64).
template <int DHW>
__device__ __forceinline__ void load_page(AttnChunk<DHW>& ch, const uint64_t* __restrict__ kp,
                                          const uint64_t* __restrict__ vp, size_t at, int lane) {
  typedef const __attribute__((address_space(1))) uint64_t gword;  // global, beyond the asm too
  gword *kr = (gword*)(kp + at), *vr = (gword*)(vp + at);
  // the page's address stays in scalar registers, the lane's offset in one of its own
  asm("" : "+s"(kr), "+s"(vr));
#pragma unroll
  for (int w = 0; w < DHW; ++w) {
    ch.k[w] = kr[(uint32_t)(lane * DHW + w)];
    ch.v[w] = vr[(uint32_t)(w * 64 + lane)];
  }
}

// The neuron of 16 rows over their sums: sNum [part][t][tile][lane] (row lane%16,
// channels 16n + 4(lane/16) + e) and sDen [part][t][row].  Waves share the NT
// tiles of 16 channels; a timestep's weights are summed and inverted once for
// all tiles of a wave.  All threads of the workgroup call it.
template <int DHW>
__device__ __forceinline__ void fire_rows(const PagedArgs& a, const v4i* sNum, const int (*sDen)[16],
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

// The rows that see page `lane` of a word (bit per row): lane r holds row r's word.
template <int ROWS>
__device__ __forceinline__ uint32_t seen_by(uint64_t word, int lane) {
  uint32_t m = 0u;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)word, r);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(word >> 32), r);
    const uint32_t x = lane < 32 ? lo : hi;
    m |= ((x >> (lane & 31)) & 1u) << r;
  }
  return m;
}

// Bits [p0, p1) of word w of a page range.
__device__ __forceinline__ uint64_t range_bits(int w, int p0, int p1) {
  const int lo = max(p0 - w * 64, 0), hi = min(p1 - w * 64, 64);
  if (lo >= hi) return 0ull;
  return (hi < 64 ? (1ull << hi) - 1 : ~0ull) & ~((1ull << lo) - 1);
}

// Lists the pages [p0, p1) (at most kPageList) that a row of the tile sees, with
// the rows; returns their number.  Words go to the waves in turn; sCount has a
// place for each.  All threads of the workgroup; two barriers.
constexpr int kListWords = kPageList / 64 + 1;  // a range may begin inside a word
template <int ROWS>
__device__ __forceinline__ int list_seen(const PagedArgs& a, const int32_t* tab, const PageTile& tl, int h,
                                         int p0, int p1, PageEntry* sList, uint32_t* sSeen, int* sCount,
                                         int lane, int wave, int nwaves) {
  const int w0 = p0 / 64, nr = tl.n_full & 63;
  uint32_t seen[kListWords];
  uint64_t any[kListWords];
#pragma unroll
  for (int k = 0; k < kListWords; ++k) {
    const int w = w0 + k;
    any[k] = 0;
    seen[k] = 0;
    if (k % nwaves != wave || w * 64 >= p1) continue;  // wave-uniform
    const uint64_t word =
        lane < nr ? a.sel[((size_t)(tl.row + lane) * a.H + h) * a.words + w] & range_bits(w, p0, p1) : 0ull;
    seen[k] = seen_by<ROWS>(word, lane);
    any[k] = __builtin_amdgcn_ballot_w64(seen[k] != 0u);
    if (lane == 0) sCount[k] = (int)__popcll(any[k]);
  }
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int k = 0; k < kListWords; ++k) {
    if ((w0 + k) * 64 >= p1) break;  // uniform
    if (seen[k] != 0u) {
      const int at = base + bits_before(any[k]);
      sList[at] = page_entry(a, tab, (w0 + k) * 64 + lane, tl.keys);
      sSeen[at] = seen[k];
    }
    base += sCount[k];
  }
  __syncthreads();
  return base;
}

template <int DHW, int QG, bool SEL>
__global__ __launch_bounds__(64 * NMDLM_MAX_T, QG == 1 ? 4 : 2) void k_paged_attn(PagedArgs a) {
  constexpr int NT = DHW * 4;
  __shared__ AttnLut sLut;
  __shared__ int sDen[NMDLM_MAX_T][16];  // [part][T], at most eight waves
  __shared__ uint32_t sWord[NMDLM_MAX_T][16][2 * DHW];
  __shared__ PageEntry sList[kPageList];
  __shared__ uint32_t sSeen[SEL ? kPageList : 1];
  __shared__ int sCount[SEL ? kListWords : 1];
  extern __shared__ v4i sNum[];  // the waves' stages, then their sums [part][T][NT][64]
  AttnStage<DHW>* sStage = reinterpret_cast<AttnStage<DHW>*>(sNum);

  touch_kernargs<sizeof(PagedArgs)>();
  const int nth = blockDim.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nwaves = nth >> 6;
  const int g = lane >> 4, c = lane & 15;
  const int h = blockIdx.x, z = blockIdx.y;
  const PageTile tl = a.tiles[blockIdx.z];
  const int nr = tl.n_full & 63, J = tl.keys, nP = (J + 63) / 64, splits = split_count(a, nP);
  if (nr == 0 || z >= splits) return;  // uniform
  const PageRange pr = split_range(nP, z, splits);
  const int32_t* tab = a.table + (size_t)tl.s * a.max_pages;
  const int np = a.parts, t = wave / np, part = wave - t * np;
  const int dw = a.H * DHW;

  const LutRegs lr = load_lut(a.lut, tid, nth);
  uint32_t qraw[QG];
  AttnWave<DHW, QG, true>::load_queries(qraw, a.q + ((size_t)t * a.max_rows + tl.row) * dw + h * DHW, dw, 0,
                                  nr - 1, g, c);
  AttnWave<DHW, QG, true> w;
  const char* lb = reinterpret_cast<const char*>(&sLut);
  // words of a pool page; a head's and timestep's keys and values in it
  const size_t page_words = (size_t)a.H * a.T * (64 * DHW), at_ht = ((size_t)h * a.T + t) * (64 * DHW);
  const uint64_t *kp = a.kp + at_ht, *vp = a.vp + at_ht;
  AttnStage<DHW>* const st = &sStage[kAttnStages * wave];
  int keys = 0;

  for (int b = pr.p0; b < pr.p1; b += kPageList) {  // uniform
    if (b > pr.p0) __syncthreads();  // the list of the piece before is read
    int m = min(pr.p1 - b, kPageList);
    if constexpr (SEL) {
      m = list_seen<16 * QG>(a, tab, tl, h, b, b + m, sList, sSeen, sCount, lane, wave, nwaves);
    } else {
      for (int i = tid; i < m; i += nth) sList[i] = page_entry(a, tab, b + i, J);
    }
    if (b == pr.p0) {
      w.init(qraw);
      fill_lut(sLut, lr, tid, nth);
    }
    __syncthreads();
    if (part >= m) continue;  // wave-uniform

    // as AttnWave::run: the weighted sum of one page while the table reads of the
    // next are in flight, and the loads of the one after that; what the list says of
    // a page is read before the table reads, which it would wait for
    auto id_at = [&](int i) { return sList[min(i, m - 1)].id; };
    auto load = [&](AttnChunk<DHW>& ch, int id) {
      load_page(ch, kp, vp, (size_t)(uint32_t)__builtin_amdgcn_readfirstlane(id) * page_words, lane);
    };
    AttnStage<DHW>*s0 = st, *s1 = st + 1, *s2 = st + 2;
    v4i s[QG][4], p[QG];
    uint32_t k[4], v[NT];
    AttnChunk<DHW> first, next;
    load(first, id_at(part));
    load(next, id_at(part + np));
    w.put(first, *s0, lane);
    w.key_pieces(*s0, k, g, c);
    w.put(next, *s1, lane);
    load(next, id_at(part + 2 * np));
    uint32_t seen = SEL ? sSeen[part] : 0u;
    w.scores(k, s);
    w.lookup(s, lb);
    w.key_pieces(*s1, k, g, c);
    w.pack(s, p);
    auto unseen = [&]() {  // weight 0 where the row does not see the page
      if constexpr (SEL) {
#pragma unroll
        for (int u = 0; u < QG; ++u)
          if (!((seen >> (16 * u + c)) & 1u)) p[u] = v4i{1, 1, 1, 1} * (int)0x80808080u;
      }
    };
    auto partial = [&](int nk) {  // keys past the request's last, or of no page
      if (nk < 64) {  // wave-uniform
        const int left = nk - 16 * g;
        const uint32_t vm = left >= 16 ? 0xFFFFu : (left <= 0 ? 0u : ((1u << left) - 1u));
        const v4i mk = bytes16(vm | (vm << 12)) * 0xFF;
#pragma unroll
        for (int u = 0; u < QG; ++u) p[u] &= mk;
#pragma unroll
        for (int n = 0; n < NT; ++n) v[n] &= vm;
      }
      keys += nk;
    };
    int i = part;
    unseen();
    for (i += np; i < m; i += np) {  // wave-uniform
      const int id = id_at(i + 2 * np), nk = sList[i - np].keys;
      if constexpr (SEL) seen = sSeen[i];
      w.value_pieces(*s0, v, g, c);
      w.scores(k, s);
      __builtin_amdgcn_sched_barrier(0);
      w.lookup(s, lb);
      w.put(next, *s2, lane);
      load(next, id);
      w.key_pieces(*s2, k, g, c);
      partial(__builtin_amdgcn_readfirstlane(nk));
      w.weigh(v, p);
      __builtin_amdgcn_sched_barrier(0);
      w.pack(s, p);
      unseen();
      AttnStage<DHW>* const tmp = s0;
      s0 = s1;
      s1 = s2;
      s2 = tmp;
    }
    w.value_pieces(*s0, v, g, c);
    partial(__builtin_amdgcn_readfirstlane(sList[i - np].keys));
    w.weigh(v, p);
  }
  w.finish(reinterpret_cast<char*>(st), lane, g, c);
  __syncthreads();  // the stages are read

#pragma unroll
  for (int u = 0; u < QG; ++u) {
    if (u > 0) __syncthreads();  // the sums and words of the group before are read
    const int rows = nr - 16 * u, pt = part * a.T + t;
#pragma unroll
    for (int n = 0; n < NT; ++n) sNum[(pt * NT + n) * 64 + lane] = w.acc[u][n];
    if (g == 0) sDen[pt][c] = w.den[u] + 128 * keys;
    __syncthreads();
    if (splits > 1) {  // uniform
      for (int i = tid; i < a.T * NT * 64; i += nth) {
        const int tt = i / (NT * 64), n = (i >> 6) % NT, r = i & 15, lg = (i >> 4) & 3;
        if (r < rows) {
          v4i x = sNum[i];
          for (int p = 1; p < np; ++p) x += sNum[p * a.T * NT * 64 + i];
          *reinterpret_cast<v4i*>(split_sums<DHW>(a, tl.row + 16 * u + r, h, z) +
                                  (size_t)tt * (64 * DHW + kPartDen) + 16 * n + 4 * lg) = x;
        }
      }
      for (int i = tid; i < a.T * 16; i += nth)
        if (i % 16 < rows) {
          int den = 0;
          for (int p = 0; p < np; ++p) den += sDen[p * a.T + i / 16][i % 16];
          split_sums<DHW>(a, tl.row + 16 * u + i % 16, h, z)[(size_t)(i / 16) * (64 * DHW + kPartDen) + 64 * DHW] =
              den;
        }
      continue;
    }
    if (rows <= 0) continue;  // uniform
    fire_rows<DHW>(a, sNum, sDen, sWord, tl.row + 16 * u, min(rows, 16), h, J < 65536, tid, nth);
  }
}

// ---------------------------------------------------------------------------
// The neuron of one row and head: num(t) is the channel's sum, den(t) the
// weights' sum; one wave per 64 channels.
// ---------------------------------------------------------------------------
template <int DHW, typename N, typename D>
__device__ __forceinline__ void fire_row(const PagedArgs& a, int row, int h, int w, int lane, bool small, N num,
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

// k_paged_join: the sums of a row's splits (integers: any order gives the same)
// and the neuron.  A workgroup per row and head, a wave per timestep and 64
// channels: 5 us for 32 rows of 16 heads in 8 splits, a chain of three loads (18 us
// with a workgroup per tile and head).
template <int DHW>
__global__ __launch_bounds__(64 * NMDLM_MAX_T * DHW) void k_paged_join(PagedArgs a, const PageTile* rows) {
  constexpr int LD = 64 * DHW + kPartDen;
  __shared__ int sNum[NMDLM_MAX_T][64 * DHW];
  __shared__ int sDen[NMDLM_MAX_T];
  touch_kernargs<sizeof(PagedArgs) + sizeof(void*)>();
  const int row = blockIdx.x, h = blockIdx.y;
  const PageTile tl = rows[row];
  const int n = split_count(a, (tl.keys + 63) / 64);
  if ((tl.n_full & 63) == 0 || n == 1) return;  // uniform; a single split fired by itself
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int t = wave / DHW, w = wave - t * DHW;
  const int32_t* base = split_sums<DHW>(a, row, h, 0) + (size_t)t * LD;
  const size_t ld = (size_t)a.T * LD;
  int x = 0, den = 0;
  for (int z0 = 0; z0 < n; z0 += 8) {
    int v[8], d[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int32_t* p = base + min(z0 + k, n - 1) * ld;
      v[k] = p[w * 64 + lane];
      d[k] = p[64 * DHW];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (z0 + k < n) {  // uniform
        x += v[k];
        den += d[k];
      }
  }
  sNum[t][w * 64 + lane] = x;
  if (w == 0 && lane == 0) sDen[t] = den;
  __syncthreads();
  if (wave < DHW)
    fire_row<DHW>(a, row, h, wave, lane, tl.keys < 65536, [&](int tt) { return sNum[tt][wave * 64 + lane]; },
                  [&](int tt) { return sDen[tt]; });
}

// ---------------------------------------------------------------------------
// k_paged_token: one row, for requests that bring a token or two.  The matrix
// cores would work for one query of sixteen; here a wave takes its pages bit by
// bit: lane = key for the scores (popcount of the key's row and the query, which
// is the same for all lanes), the weight's eight bits become eight 64-key masks
// by ballots, and with lane = channel
//     sum_j p_j V[j,c] = sum_b 2^b popcount(mask_b AND word of channel c).
// About 100 vector instructions a page of 128 channels, no exchange between
// lanes, and few registers: the loads of kTokenAhead pages are in flight in each
// of many waves.  Bound by HBM: T = 4, 16 heads of 128, 64 requests x 2048 keys, 268 MB,
// 45 us or 6.0 TB/s (64 us in tiles; a plain read reaches 6.3); with a selection of 8
// of the 31 pages, 75 MB 20 us, of 16 of 255 pages, 143 MB 30 us, the list and the table
// read one after the other before the pages.  A request has one workgroup a head where
// the plan has rows enough: 64 requests x 1 to 4000 keys, 271 MB, 52 us, the longest
// last; one of 100 thousand keys among 63 of a thousand 410 us.
// ---------------------------------------------------------------------------
// Two pages in flight in each of up to twelve waves a workgroup, at most four a
// timestep, against four in each of eight: 64 requests x 1 to 4000 keys 60.9 us
// against 62.1, x 2048 45.6 against 46.6, 128 x 512 30.9 against 32.0, T = 3, 32 x 1000
// 13.2 against 15.0, T = 6, 16 x 2 rows x 1000 17.2 against 20.3; twelve a timestep, T =
// 1, 64 x 2000 17.1 against 16.1 with four; sixteen waves, 128 x 512 41.
constexpr int kTokenAhead = 2;
constexpr int kTokenWaves = 12;

template <int DHW>
struct TokenPage {
  uint64_t k[DHW], v[DHW];  // key row `lane`; channels DHW*lane (and + 1)
};
template <int DHW>
__device__ __forceinline__ TokenPage<DHW> load_token_page(const PagedArgs& a, int id, int h, int t, int lane) {
  typedef const ulonglong2 __attribute__((may_alias)) pair;
  const size_t at = (((size_t)id * a.H + h) * a.T + t) * (64 * DHW);
  TokenPage<DHW> r;
  if constexpr (DHW == 2) {
    const ulonglong2 k = reinterpret_cast<pair*>(a.kp + at)[lane], v = reinterpret_cast<pair*>(a.vp + at)[lane];
    r.k[0] = k.x;
    r.k[1] = k.y;
    r.v[0] = v.x;
    r.v[1] = v.y;
  } else {
    r.k[0] = a.kp[at + lane];
    r.v[0] = a.vp[at + lane];
  }
  return r;
}

template <int DHW, bool SEL>
__global__ __launch_bounds__(64 * kTokenWaves) void k_paged_token(PagedArgs a) {
  constexpr int DH = 64 * DHW;
  __shared__ uint8_t sLut[256];
  __shared__ PageEntry sList[kPageList];
  __shared__ int sNum[NMDLM_MAX_T][DH];
  __shared__ int sDen[NMDLM_MAX_T];
  touch_kernargs<sizeof(PagedArgs)>();
  const int nth = blockDim.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nwaves = nth >> 6;
  const int h = blockIdx.x, z = blockIdx.y, row = blockIdx.z;
  const PageTile tl = a.tiles[row];
  const int J = tl.keys, nP = (J + 63) / 64, splits = split_count(a, nP);
  if ((tl.n_full & 63) == 0 || z >= splits) return;  // uniform
  const PageRange pr = split_range(nP, z, splits);
  const int32_t* tab = a.table + (size_t)tl.s * a.max_pages;
  const int np = a.parts, t = wave / np, part = wave - t * np;
  const uint64_t* qp = a.q + ((size_t)t * a.max_rows + row) * (a.H * DHW) + h * DHW;
  uint64_t q[DHW];
#pragma unroll
  for (int w = 0; w < DHW; ++w) {
    const uint64_t x = qp[w];
    q[w] = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
           (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
  }
  for (int i = tid; i < 256; i += nth) sLut[i] = a.lut[i];
  for (int i = tid; i < a.T * DH; i += nth) (&sNum[0][0])[i] = 0;
  if (tid < a.T) sDen[tid] = 0;

  int acc[8][DHW], den = 0;
#pragma unroll
  for (int b = 0; b < 8; ++b)
#pragma unroll
    for (int w = 0; w < DHW; ++w) acc[b][w] = 0;

  for (int b0 = pr.p0; b0 < pr.p1; b0 += kPageList) {  // uniform
    const int b1 = min(b0 + kPageList, pr.p1);
    int m = b1 - b0;
    if (b0 > pr.p0) __syncthreads();  // the list of the piece before is read
    if constexpr (SEL) {
      m = 0;
      const uint64_t* sw = a.sel + ((size_t)row * a.H + h) * a.words;
      for (int w = b0 / 64; w * 64 < b1; ++w) {
        const uint64_t word = sw[w] & range_bits(w, b0, b1);
        if (w % nwaves == wave && ((word >> lane) & 1))
          sList[m + bits_before(word)] = page_entry(a, tab, w * 64 + lane, J);
        m += (int)__popcll(word);
      }
      m = __builtin_amdgcn_readfirstlane(m);
    } else {
      for (int i = tid; i < m; i += nth) sList[i] = page_entry(a, tab, b0 + i, J);
    }
    __syncthreads();
    if (part >= m) continue;  // wave-uniform
    auto id_of = [&](int i) { return __builtin_amdgcn_readfirstlane(sList[min(i, m - 1)].id); };
    TokenPage<DHW> pg[kTokenAhead];
#pragma unroll
    for (int j = 0; j < kTokenAhead; ++j) pg[j] = load_token_page<DHW>(a, id_of(part + j * np), h, t, lane);
    for (int i = part; i < m; i += kTokenAhead * np) {
#pragma unroll
      for (int j = 0; j < kTokenAhead; ++j) {
        const int e = i + j * np;
        if (e < m) {  // wave-uniform
          const int keys = sList[e].keys;
          int s = 0;
#pragma unroll
          for (int w = 0; w < DHW; ++w) s += (int)__popcll(pg[j].k[w] & q[w]);
          int p = sLut[s];
          p = lane < keys ? p : 0;
          den += p;
#pragma unroll
          for (int b = 0; b < 8; ++b) {
            const uint64_t mask = __builtin_amdgcn_ballot_w64((p >> b) & 1);
#pragma unroll
            for (int w = 0; w < DHW; ++w) acc[b][w] += (int)__popcll(pg[j].v[w] & mask);
          }
        }
        pg[j] = load_token_page<DHW>(a, id_of(e + kTokenAhead * np), h, t, lane);
      }
    }
  }
  den = wave_sum(den);
  if (lane == 0) atomicAdd(&sDen[t], den);
#pragma unroll
  for (int w = 0; w < DHW; ++w) {
    int x = 0;
#pragma unroll
    for (int b = 7; b >= 0; --b) x = 2 * x + acc[b][w];
    atomicAdd(&sNum[t][DHW * lane + w], x);
  }
  __syncthreads();
  if (splits > 1) {  // uniform
    int32_t* o = split_sums<DHW>(a, row, h, z);
    for (int i = tid; i < a.T * DH; i += nth) o[(i / DH) * (DH + kPartDen) + i % DH] = (&sNum[0][0])[i];
    if (tid < a.T) o[tid * (DH + kPartDen) + DH] = sDen[tid];
    return;
  }
  for (int w = wave; w < DHW; w += nwaves)
    fire_row<DHW>(a, row, h, w, lane, J < 65536, [&](int tt) { return sNum[tt][w * 64 + lane]; },
                  [&](int tt) { return sDen[tt]; });
}

// ---------------------------------------------------------------------------
// Which kernel and grid; the lengths are on the device, the rule sees the plan's
// sizes.  All measured with spikes out, H = 16, T = 4, dh = 128 unless said.
//  * The token kernel up to 2 rows a request (and 8 rows more, a plan's spare
//    ones): 64 requests x 1 row x 4001 keys 100 us against 133 in tiles, x 501 keys 20
//    against 30; 2 rows 136 against 132 and 30 against 31; 3 rows 181 against 133.  One
//    request of 8 rows x 508 keys 6.2 against 9.8, x 4008 keys 18.1 against 12.6, x 64008
//    keys 104 against 36; of 4 rows 6.3 against 9.9, 12.1 against 12.4 and 79 against 35:
//    the spare rows pay for short contexts only.
//  * 32 rows a wave (QG = 2) where the tiles give 1024 such waves: 4 x 200 rows x
//    500 keys 24 us against 29 with 16, 1 x 2048 x 2348 109 against 135, T = 1, 16 x
//    100 x 400 17.0 against 18.5; below, T = 4, 1 x 300 x 600 19.5 against 17.6, T = 1,
//    1 x 1024 x 1324 26 against 18.
//  * Parts of tiles: eight waves a workgroup where T allows (32 x 16 x 2016 keys, one, two
//    and four parts: T = 1 26, 21 and 15 us, T = 2 34, 23 and 23, T = 4 38 and 36); sixteen
//    waves (T = 4, four parts) 46.
//  * Splits to give each CU one workgroup of tiles, or two of tokens: 1 x 16 rows x
//    64016 keys 391 us whole, 109 in 4, 42 in 16, 43 in 32; 4 x 16 x 16016 105 whole, 42 in
//    4 (one a CU), 47 in 6 (some CUs two), 42 in 8; 64 selected of 2047 pages, 32
//    rows, 70 whole, 25 in 8 (one a CU), 31 in 10 or 16.  16 x 16 x 2016 keys, a
//    workgroup a CU without: 23 whole, 40 in 2.  Idle slots count as if they had
//    rows: the 1 x 16 rows x 64016 keys in a plan of 64 blocks of 16 355 us, 36 in its own.
// ---------------------------------------------------------------------------
PagedRoute paged_route(const nmdlm_pages& pg, int T, int H) {
  PagedRoute r{pg.max_rows <= 2LL * pg.n_seq + 8, 1, T <= 2 ? 4 : (T <= 4 ? 2 : 1), 1};
  if (r.token) r.parts = std::max(std::min(kTokenWaves / T, 4), 1);
  const long long t32 = pg.max_rows / 32 + pg.n_seq;
  if (!r.token && pg.max_rows >= 32LL * pg.n_seq && t32 * H * T >= 1024) {
    r.groups = 2;
    r.parts = 1;
    return r;
  }
  // rows or tiles of every request, less what a plan may have to spare
  const long long units = std::max(r.token ? pg.max_rows / 2 : pg.max_rows / 16, pg.n_seq);
  r.splits = (int)std::max(1LL, std::min<long long>({(r.token ? 512 : 256) / (units * H), 64,
                                                     pg.max_pages / kSplitPages}));
  return r;
}

static size_t part_bytes(const nmdlm_pages& pg, const PagedRoute& r, int T, int H, int dh) {
  if (r.splits == 1) return 0;
  return align_up((size_t)pg.max_rows * H * r.splits * T * (dh + kPartDen) * sizeof(int32_t), 256);
}

size_t paged_attn_ws(const nmdlm_pages& pg, int T, int H, int dh) {
  return part_bytes(pg, paged_route(pg, T, H), T, H, dh);
}

constexpr size_t kPagedPlainLds = 49152;  // dynamic LDS that needs no attribute beside the static

template <int DHW, int QG, bool SEL>
static nmdlm_status launch_paged(const PagedArgs& a, dim3 grid, hipStream_t st) {
  const size_t dyn = (size_t)a.T * a.parts * std::max(DHW * 4 * 64 * sizeof(v4i),
                                                      kAttnStages * sizeof(AttnStage<DHW>));
  if (dyn > kPagedPlainLds &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(&k_paged_attn<DHW, QG, SEL>),
                          hipFuncAttributeMaxDynamicSharedMemorySize, (int)dyn) != hipSuccess)
    return NMDLM_ERR_HIP;
  hipLaunchKernelGGL((k_paged_attn<DHW, QG, SEL>), grid, dim3(64 * a.T * a.parts), (uint32_t)dyn, st, a);
  return hip_status();
}

template <int DHW>
static nmdlm_status launch_paged_dh(const nmdlm_pages& pg, const PagedAttnCall& c, hipStream_t st) {
  const PagedRoute r = paged_route(pg, c.T, c.H);
  PageIndex ix;
  page_index_layout(pg.n_seq, pg.max_rows, pg.index, &ix);
  PagedArgs a{};
  // heads first: where H is a multiple of 8 the tiles of a head share an XCD, and
  // the list's empty entries are the last
  const unsigned n_tiles = r.token ? pg.max_rows : (r.groups == 2 ? ix.n32 : ix.n16);
  static_assert(2 * NMDLM_MAX_REQUESTS + 8 < 65536 && NMDLM_MAX_PLAN_ROWS / 16 + NMDLM_MAX_REQUESTS < 65536,
                "tiles fit a grid's third dimension");
  const dim3 grid(c.H, r.splits, n_tiles);
  a.tiles = r.token ? ix.t1 : (r.groups == 2 ? ix.t32 : ix.t16);
  a.table = pg.table;
  a.q = c.q;
  a.kp = c.k_pages;
  a.vp = c.v_pages;
  a.lut = c.lut;
  a.sel = c.sel;
  a.a_out = c.a_out;
  a.s_out = c.s_out;
  a.u_out = c.u_out;
  a.part = static_cast<int32_t*>(c.ws);
  a.max_pages = pg.max_pages;
  a.pool = pg.pool;
  a.max_rows = pg.max_rows;
  a.words = (pg.max_pages + 63) / 64;
  a.T = c.T;
  a.H = c.H;
  a.parts = r.parts;
  a.splits = r.splits;
  a.theta = c.theta;
  nmdlm_status rc;
  if (r.token) {
    const dim3 block(64 * c.T * r.parts);
    if (c.sel) hipLaunchKernelGGL((k_paged_token<DHW, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_paged_token<DHW, false>), grid, block, 0, st, a);
    rc = hip_status();
  } else if (r.groups == 2) {
    rc = c.sel ? launch_paged<DHW, 2, true>(a, grid, st) : launch_paged<DHW, 2, false>(a, grid, st);
  } else {
    rc = c.sel ? launch_paged<DHW, 1, true>(a, grid, st) : launch_paged<DHW, 1, false>(a, grid, st);
  }
  if (rc != NMDLM_OK || r.splits == 1) return rc;
  hipLaunchKernelGGL(k_paged_join<DHW>, dim3(pg.max_rows, c.H), dim3(64 * c.T * DHW), 0, st, a, ix.t1);
  return hip_status();
}

nmdlm_status launch_paged_attn(const nmdlm_pages& pg, const PagedAttnCall& c, hipStream_t st) {
  return c.dh == 64 ? launch_paged_dh<1>(pg, c, st) : launch_paged_dh<2>(pg, c, st);
}

}  // namespace nmdlm
