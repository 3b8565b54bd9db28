// Attention on spike operands over paged caches: the formulas of attn_device.h
// for the packed rows of a plan, over all pages of a request or those selected
// for each row and head.
#include <algorithm>

#include "attn_device.h"
#include "pages.h"

namespace nmdlm {

// ---------------------------------------------------------------------------
// k_paged_attn: a workgroup takes one tile of 16*QG rows, a head and one of the
// tile's splits; wave = (timestep, part).  A page is the 64-key chunk of a wave
// (attn_device.h).  The pages to visit stand in an LDS list: all of the tile's
// pages, or those that at least one of its rows selected, with one bit per row
// that sees them (a score that a row does not see weighs 0, byte -128).  The
// parts of a timestep take the list's entries in turn.
// ---------------------------------------------------------------------------
constexpr int kPageList = 512;  // entries of the list (a longer one goes in pieces)

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
  int32_t* part;   // sums of the splits [tile][head][split][T][(16*DHW*... ) + 16]
  int32_t* nsplit; // [tile][head]: splits that hold sums (0, 1: none)
  int n_tiles, max_pages, pool, max_rows, words;
  int T, H, parts, splits;
  int32_t theta;
};

struct PageEntry {
  int id, keys;  // pool page, keys of it that count (0 outside the pool)
};

constexpr int kPagesPerSplit = 8;  // a split has at least this many pages

// Ints of one split's sums of a timestep: NT tiles of 64 lanes x 4, 16 weights.
template <int DHW>
constexpr int part_ints() { return DHW * 4 * 256 + 16; }

// One wave's loads of a page: key row `lane`, value words of channels lane (and
// lane + 64).
template <int DHW>
__device__ __forceinline__ void load_page(AttnChunk<DHW>& ch, const uint64_t* __restrict__ kp,
                                          const uint64_t* __restrict__ vp, size_t at, int lane) {
  const uint64_t* kr = kp + at * (64 * DHW);
  const uint64_t* vr = vp + at * (64 * DHW);
#pragma unroll
  for (int w = 0; w < DHW; ++w) {
    ch.k[w] = kr[(uint32_t)(lane * DHW + w)];
    ch.v[w] = vr[(uint32_t)(w * 64 + lane)];
  }
}

// The neuron of 16 rows: cur(t, n, lane) is the normalised current of row lane%16,
// channels 16n + 4(lane/16) + e; waves share the NT tiles.  All threads of the
// workgroup call it.
template <int DHW, typename F>
__device__ __forceinline__ void fire_rows(const PagedArgs& a, uint32_t (*sWord)[16][2 * DHW], int row0,
                                          int nr, int h, int tid, int nth, F cur) {
  constexpr int NT = DHW * 4, DH = DHW * 64;
  const int lane = tid & 63, wave = tid >> 6, nwaves = nth >> 6, g = lane >> 4, c = lane & 15;
  const int d = a.H * DH, dw = d / 64;
  const bool vec = (reinterpret_cast<uintptr_t>(a.a_out) & 15) == 0;
  for (int i = tid; i < a.T * 32 * DHW; i += nth) (&sWord[0][0][0])[i] = 0u;
  __syncthreads();
  for (int n = wave; n < NT; n += nwaves) {
    v4i V = v4i{0, 0, 0, 0};
    for (int t = 0; t < a.T; ++t) {
      const v4i x = cur(t, n, lane);
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
        V[e] += x[e];
        const bool s = V[e] >= a.theta;
        if (s) V[e] -= a.theta;
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

__device__ __forceinline__ v4i normalise(v4i x, int den, bool small) {
  if (small) return attn_norm4(x, den);
  v4i r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = attn_norm(x[e], den);
  return r;
}

// Word w of the tile's selections, row lane of it (0 for lanes without a row).
__device__ __forceinline__ uint64_t sel_word(const PagedArgs& a, int row0, int nr, int h, int w, int lane) {
  return lane < nr ? a.sel[((size_t)(row0 + lane) * a.H + h) * a.words + w] : 0ull;
}
// The rows that see page `lane` of the word (bit per row).
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

template <int DHW, int QG, bool SEL>
__global__ __launch_bounds__(64 * NMDLM_MAX_T) void k_paged_attn(PagedArgs a) {
  constexpr int NT = DHW * 4;
  __shared__ AttnLut sLut;
  __shared__ int sDen[NMDLM_MAX_T][16];
  __shared__ uint32_t sWord[NMDLM_MAX_T][16][2 * DHW];
  __shared__ PageEntry sList[kPageList];
  __shared__ uint32_t sSeen[SEL ? kPageList : 1];
  __shared__ int sCount[2];
  extern __shared__ v4i sNum[];  // the waves' stages, then the sums [T][NT][64]
  AttnStage<DHW>* sStage = reinterpret_cast<AttnStage<DHW>*>(sNum);

  const int nth = blockDim.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nwaves = nth >> 6;
  const int g = lane >> 4, c = lane & 15;
  const int lid = xcd_order(blockIdx.x, gridDim.x);
  const int ti = lid % a.n_tiles, hz = lid / a.n_tiles, h = hz / a.splits, z = hz - h * a.splits;
  const PageTile tl = a.tiles[ti];
  if ((tl.n_full & 63) == 0) return;  // uniform
  const int nr = tl.n_full & 63, J = tl.keys, nP = (J + 63) / 64;
  const int32_t* tab = a.table + (size_t)tl.s * a.max_pages;
  const int np = a.parts, t = wave / np, part = wave - t * np;
  const int dw = a.H * DHW;

  const LutRegs lr = load_lut(a.lut, tid, nth);
  uint32_t qraw[QG];
  AttnWave<DHW, QG>::load_queries(qraw, a.q + ((size_t)t * a.max_rows + tl.row) * dw + h * DHW, dw, 0,
                                  nr - 1, g, c);
  // pages to visit
  int cnt = nP;
  if constexpr (SEL) {
    if (tid == 0) sCount[0] = 0;
    __syncthreads();
    int mine = 0;
    for (int w = wave; w * 64 < nP; w += nwaves) {
      uint64_t x = sel_word(a, tl.row, nr, h, w, lane);
      for (int o = 32; o > 0; o >>= 1) x |= __shfl_xor((unsigned long long)x, o);
      if (nP - w * 64 < 64) x &= (1ull << (nP - w * 64)) - 1;
      mine += (int)__popcll(x);
    }
    if (lane == 0 && mine) atomicAdd(&sCount[0], mine);
    __syncthreads();
    cnt = sCount[0];
  }
  const int splits = min(a.splits, max((cnt + kPagesPerSplit - 1) / kPagesPerSplit, 1));
  if (z >= splits) return;  // uniform
  const int e0 = (int)((long long)cnt * z / splits), e1 = (int)((long long)cnt * (z + 1) / splits);

  AttnWave<DHW, QG> w;
  w.init(qraw);
  fill_lut(sLut, lr, tid, nth);
  const char* lb = reinterpret_cast<const char*>(&sLut);
  AttnStage<DHW>* const st = &sStage[kAttnStages * wave];
  int keys = 0;

  for (int b = e0; b < e1; b += kPageList) {  // uniform
    const int m = min(e1 - b, kPageList);
    __syncthreads();  // the list of the piece before is read
    if constexpr (SEL) {
      // entries [b, b + m) of the pages seen by a row, ascending: a wave walks all
      // words' counts and writes the entries of its own
      int base = 0;
      for (int wd = 0; wd * 64 < nP; ++wd) {
        uint64_t word = sel_word(a, tl.row, nr, h, wd, lane);
        const uint32_t seen = wd * 64 + lane < nP ? seen_by<16 * QG>(word, lane) : 0u;
        const uint64_t any = __builtin_amdgcn_ballot_w64(seen != 0u);
        const int at = base - b + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(any >> 32),
                                                                 __builtin_amdgcn_mbcnt_lo((uint32_t)any, 0));
        if (wd % nwaves == wave && seen != 0u && at >= 0 && at < m) {
          const int p = wd * 64 + lane, id = tab[p];
          const bool there = (unsigned)id < (unsigned)a.pool;
          sList[at] = PageEntry{there ? id : 0, there ? min(64, J - 64 * p) : 0};
          sSeen[at] = seen;
        }
        base += (int)__popcll(any);
      }
    } else {
      for (int i = tid; i < m; i += nth) {
        const int p = b + i, id = tab[p];
        const bool there = (unsigned)id < (unsigned)a.pool;
        sList[i] = PageEntry{there ? id : 0, there ? min(64, J - 64 * p) : 0};
      }
    }
    __syncthreads();
    if (part >= m) continue;  // wave-uniform

    // as AttnWave::run: the weighted sum of one page while the table reads of the
    // next and the loads of the one after are in flight
    auto entry = [&](int i) {
      const PageEntry e = sList[min(i, m - 1)];
      return PageEntry{__builtin_amdgcn_readfirstlane(e.id), __builtin_amdgcn_readfirstlane(e.keys)};
    };
    auto place = [&](int id) { return ((size_t)id * a.H + h) * a.T + t; };
    AttnStage<DHW>*s0 = st, *s1 = st + 1, *s2 = st + 2;
    v4i s[QG][4], p[QG];
    uint32_t k[4], v[NT];
    AttnChunk<DHW> first, nxt;
    PageEntry ec = entry(part), en = entry(part + np), ef = entry(part + 2 * np);
    load_page(first, a.kp, a.vp, place(ec.id), lane);
    load_page(nxt, a.kp, a.vp, place(en.id), lane);
    w.put(first, *s0, lane);
    w.key_pieces(*s0, k, g, c);
    w.put(nxt, *s1, lane);
    load_page(nxt, a.kp, a.vp, place(ef.id), lane);
    w.scores(k, s);
    w.lookup(s, lb);
    w.key_pieces(*s1, k, g, c);
    w.pack(s, p);
    auto unseen = [&](int i) {  // weight 0 where the row does not see the page
      if constexpr (SEL) {
        const uint32_t seen = sSeen[i];
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
    unseen(i);
    for (i += np; i < m; i += np) {
      w.value_pieces(*s0, v, g, c);
      w.scores(k, s);
      __builtin_amdgcn_sched_barrier(0);
      w.lookup(s, lb);
      w.put(nxt, *s2, lane);
      const PageEntry ex = entry(i + 2 * np);
      load_page(nxt, a.kp, a.vp, place(ex.id), lane);
      w.key_pieces(*s2, k, g, c);
      partial(ec.keys);
      w.weigh(v, p);
      __builtin_amdgcn_sched_barrier(0);
      w.pack(s, p);
      unseen(i);
      ec = en;
      en = ef;
      ef = ex;
      AttnStage<DHW>* const tmp = s0;
      s0 = s1;
      s1 = s2;
      s2 = tmp;
    }
    w.value_pieces(*s0, v, g, c);
    partial(ec.keys);
    w.weigh(v, p);
  }
  w.finish(reinterpret_cast<char*>(st), lane, g, c);
  __syncthreads();  // the stages are read

#pragma unroll
  for (int u = 0; u < QG; ++u) {
    if (u > 0) __syncthreads();  // the sums and words of the group before are read
    const int rows = nr - 16 * u;
    for (int i = tid; i < a.T * NT * 64; i += nth) sNum[i] = v4i{0, 0, 0, 0};
    for (int i = tid; i < a.T * 16; i += nth) (&sDen[0][0])[i] = 0;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        atomicAdd(reinterpret_cast<int*>(&sNum[(t * NT + n) * 64 + lane]) + e, w.acc[u][n][e]);
    if (g == 0) atomicAdd(&sDen[t][c], w.den[u] + 128 * keys);
    __syncthreads();
    if (splits > 1) {  // uniform; QG = 1
      int32_t* o = a.part + ((size_t)(ti * a.H + h) * a.splits + z) * a.T * part_ints<DHW>();
      for (int i = tid; i < a.T * NT * 64; i += nth) {
        const int tt = i / (NT * 64);
        *reinterpret_cast<v4i*>(o + (size_t)tt * part_ints<DHW>() + (i - tt * NT * 64) * 4) = sNum[i];
      }
      for (int i = tid; i < a.T * 16; i += nth)
        o[(size_t)(i / 16) * part_ints<DHW>() + NT * 256 + i % 16] = sDen[i / 16][i % 16];
      if (z == 0 && tid == 0) a.nsplit[ti * a.H + h] = splits;
      return;
    }
    if (a.splits > 1 && tid == 0) a.nsplit[ti * a.H + h] = 1;
    if (rows <= 0) continue;  // uniform
    const bool small = J < 65536;
    fire_rows<DHW>(a, sWord, tl.row + 16 * u, min(rows, 16), h, tid, nth, [&](int tt, int n, int l) {
      return normalise(sNum[(tt * NT + n) * 64 + l], sDen[tt][l & 15], small);
    });
  }
}

// k_paged_join: the sums of a tile's splits (integers: any order gives the same),
// normalised, and the neuron.
template <int DHW>
__global__ __launch_bounds__(64 * DHW * 4) void k_paged_join(PagedArgs a) {
  constexpr int NT = DHW * 4;
  __shared__ uint32_t sWord[NMDLM_MAX_T][16][2 * DHW];
  const int ti = blockIdx.x % a.n_tiles, h = blockIdx.x / a.n_tiles;
  const PageTile tl = a.tiles[ti];
  if ((tl.n_full & 63) == 0) return;
  const int splits = a.nsplit[ti * a.H + h];
  if (splits <= 1) return;
  const int32_t* base = a.part + (size_t)(ti * a.H + h) * a.splits * a.T * part_ints<DHW>();
  const size_t zs = (size_t)a.T * part_ints<DHW>();
  const bool small = tl.keys < 65536;
  fire_rows<DHW>(a, sWord, tl.row, tl.n_full & 63, h, threadIdx.x, blockDim.x, [&](int t, int n, int l) {
    const int32_t* o = base + (size_t)t * part_ints<DHW>();
    v4i x = v4i{0, 0, 0, 0};
    int den = 0;
    for (int z = 0; z < splits; ++z) {
      x += *reinterpret_cast<const v4i*>(o + z * zs + (n * 64 + l) * 4);
      den += o[z * zs + NT * 256 + (l & 15)];
    }
    return normalise(x, den, small);
  });
}

// ---------------------------------------------------------------------------
// Which grid.
// ---------------------------------------------------------------------------
struct PagedRoute {
  int groups, parts, splits;
};
static PagedRoute paged_route(const nmdlm_pages& pg, int T, int H) {
  const long long t16 = pg.max_rows / 16 + pg.n_seq, t32 = pg.max_rows / 32 + pg.n_seq;
  PagedRoute r{1, T <= 2 ? 4 : (T <= 4 ? 2 : 1), 1};
  if (pg.max_rows >= 32LL * pg.n_seq && t32 * H * T >= 2048) {
    r.groups = 2;
    r.parts = 1;
    return r;
  }
  const long long wgs = t16 * H;
  if (wgs < 256)
    r.splits = (int)std::max(1LL, std::min<long long>({(511 + wgs) / wgs, 64, pg.max_pages / kPagesPerSplit}));
  return r;
}

static int32_t* carve_paged(const nmdlm_pages& pg, const PagedRoute& r, int T, int H, int dh, void* ws,
                            int32_t** nsplit, size_t* bytes) {
  Carver cv{static_cast<char*>(ws), 0, (size_t)-1, true};
  int32_t* part = nullptr;
  *nsplit = nullptr;
  if (r.splits > 1) {
    const size_t th = (size_t)(pg.max_rows / 16 + pg.n_seq) * H;
    *nsplit = cv.take<int32_t>(th);
    part = cv.take<int32_t>(th * r.splits * T * (dh / 64 * 1024 + 16));
  }
  *bytes = align_up(cv.off, 256);
  return part;
}

size_t paged_attn_ws(const nmdlm_pages& pg, int T, int H, int dh) {
  int32_t* ns;
  size_t bytes;
  carve_paged(pg, paged_route(pg, T, H), T, H, dh, nullptr, &ns, &bytes);
  return bytes;
}

constexpr size_t kPagedPlainLds = 49152;  // dynamic LDS that needs no attribute beside the static

template <int DHW, int QG, bool SEL>
static nmdlm_status launch_paged(const PagedArgs& a, int n_wg, hipStream_t st) {
  const size_t dyn = std::max((size_t)a.T * DHW * 4 * 64 * sizeof(v4i),
                              (size_t)a.T * a.parts * kAttnStages * sizeof(AttnStage<DHW>));
  const auto fn = &k_paged_attn<DHW, QG, SEL>;
  if (dyn > kPagedPlainLds &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize,
                          (int)dyn) != hipSuccess)
    return NMDLM_ERR_HIP;
  hipLaunchKernelGGL((k_paged_attn<DHW, QG, SEL>), dim3((unsigned)n_wg), dim3(64 * a.T * a.parts),
                     (uint32_t)dyn, st, a);
  return hip_status();
}

template <int DHW>
static nmdlm_status launch_paged_dh(const nmdlm_pages& pg, const PagedAttnCall& c, hipStream_t st) {
  const PagedRoute r = paged_route(pg, c.T, c.H);
  PageIndex ix;
  page_index_layout(pg.n_seq, pg.max_rows, pg.index, &ix);
  PagedArgs a{};
  a.n_tiles = r.groups == 2 ? ix.n32 : ix.n16;
  a.tiles = r.groups == 2 ? ix.t32 : ix.t16;
  a.table = pg.table;
  a.q = c.q;
  a.kp = c.k_pages;
  a.vp = c.v_pages;
  a.lut = c.lut;
  a.sel = c.sel;
  a.a_out = c.a_out;
  a.s_out = c.s_out;
  a.u_out = c.u_out;
  size_t bytes;
  a.part = carve_paged(pg, r, c.T, c.H, c.dh, c.ws, &a.nsplit, &bytes);
  a.max_pages = pg.max_pages;
  a.pool = pg.pool;
  a.max_rows = pg.max_rows;
  a.words = (pg.max_pages + 63) / 64;
  a.T = c.T;
  a.H = c.H;
  a.parts = r.parts;
  a.splits = r.splits;
  a.theta = c.theta;
  // a launch has fewer than 2^32 threads
  if ((long long)a.n_tiles * c.H * r.splits * (64 * c.T * r.parts) >= 1LL << 32) return NMDLM_ERR_UNSUPPORTED;
  const int n_wg = a.n_tiles * c.H * r.splits;
  nmdlm_status rc;
  if (r.groups == 2)
    rc = c.sel ? launch_paged<DHW, 2, true>(a, n_wg, st) : launch_paged<DHW, 2, false>(a, n_wg, st);
  else
    rc = c.sel ? launch_paged<DHW, 1, true>(a, n_wg, st) : launch_paged<DHW, 1, false>(a, n_wg, st);
  if (rc != NMDLM_OK || r.splits == 1) return rc;
  hipLaunchKernelGGL(k_paged_join<DHW>, dim3((unsigned)(a.n_tiles * c.H)), dim3(64 * DHW * 4), 0, st, a);
  return hip_status();
}

nmdlm_status launch_paged_attn(const nmdlm_pages& pg, const PagedAttnCall& c, hipStream_t st) {
  return c.dh == 64 ? launch_paged_dh<1>(pg, c, st) : launch_paged_dh<2>(pg, c, st);
}

}  // namespace nmdlm
