// Paged spike caches: block tables and work lists from the requests' lengths,
// the store of packed rows into pages, and the choice of context pages by
// their spike counts.
#include <algorithm>

#include "pages.h"

namespace nmdlm {

// ---------------------------------------------------------------------------
// Plan.  Two steps: the sums over the requests in order (rows, pages taken,
// pages given back), by one workgroup; then every output entry by itself, its
// request found by bisection of cu_rows.
// ---------------------------------------------------------------------------
struct PlanArgs {
  nmdlm_pages pg;
  const int32_t* ctx;
  const int32_t* rows;
  int32_t* status;
  PageIndex ix;
};

constexpr int kPlanThreads = 1024;

// Inclusive sums over the workgroup; `total` is the sum of all.
template <typename V>
__device__ __forceinline__ V block_scan(V v, V* sWave, V& total) {
  constexpr int NW = kPlanThreads / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int o = 1; o < 64; o <<= 1) {
    const V u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  if (lane == 63) sWave[wave] = v;
  __syncthreads();
  V before = 0, all = 0;
  for (int w = 0; w < NW; ++w) {
    if (w < wave) before += sWave[w];
    all += sWave[w];
  }
  __syncthreads();  // sWave is free again
  total = all;
  return v + before;
}

// A chunk's sums fit 32 bits (1024 requests of at most 2^19 rows, 2^17 pages);
// the carries between chunks are 64 bits wide.
__device__ void plan_sums(const PlanArgs& a) {
  __shared__ int sRows[kPlanThreads / 64];
  __shared__ unsigned long long sPages[kPlanThreads / 64];
  __shared__ int sTaken;
  const int tid = threadIdx.x, n = a.pg.n_seq, pool = a.pg.pool;
  const int head = (int)((uint32_t)a.pg.ring_state[0] % (uint32_t)pool);
  const int free_pages = min(max(a.pg.ring_state[1], 0), pool);
  long long row_c = 0, need_c = 0, back_c = 0;
  int bits = 0;
  if (tid == 0) sTaken = 0;
  __syncthreads();
  for (int s0 = 0; s0 < n; s0 += kPlanThreads) {  // uniform
    const int s = s0 + tid;
    const bool in = s < n;
    const int ctx = in ? a.ctx[s] : 0, rows = in ? a.rows[s] : 0, held = in ? a.pg.held[s] : 0;
    const int r = rows > 0 && rows <= a.pg.max_rows ? rows : 0;
    int r_all;
    const long long row_end = row_c + block_scan(r, sRows, r_all);
    const long long end = (long long)ctx + rows;
    const bool held_ok = held >= 0 && held <= a.pg.max_pages;
    const bool fits = in && rows >= 0 && rows <= a.pg.max_rows && held_ok && ctx >= 0 &&
                      ctx <= (long long)held * NMDLM_PAGE &&
                      end <= (long long)a.pg.max_pages * NMDLM_PAGE && row_end <= a.pg.max_rows;
    const bool ended = in && rows == -1 && held_ok;
    const int pages = fits ? (int)((end + NMDLM_PAGE - 1) / NMDLM_PAGE) : 0;
    const unsigned need = max(pages - held, 0) * (fits ? 1 : 0), back = ended ? held : 0;
    unsigned long long p_all;
    const unsigned long long p =
        block_scan((unsigned long long)back << 32 | need, sPages, p_all);
    const long long need_end = need_c + (uint32_t)p, back_end = back_c + (long long)(p >> 32);
    const bool ok = fits && (need == 0 || need_end <= free_pages);
    if (in) {
      a.pg.cu_rows[s + 1] = (int)min(row_end, (long long)a.pg.max_rows);
      a.ix.req[s] = PageReq{ok ? (int)min(need_end - need, (long long)pool) : -1, held, ctx, rows};
      a.ix.back[s] = (int)min(back_end - back, (long long)pool);
      if (ended) a.pg.held[s] = 0;
      else if (ok) a.pg.held[s] = max(held, pages);
      if (!fits && !ended) bits |= NMDLM_STATUS_BAD_REQUEST;
      if (fits && !ok) bits |= NMDLM_STATUS_PAGES_SHORT;
      if (ok && need > 0) atomicMax(&sTaken, (int)need_end);
    }
    row_c += r_all;
    need_c += (uint32_t)p_all;
    back_c += (long long)(p_all >> 32);
  }
  if (bits && a.status) atomicOr(a.status, bits);
  __syncthreads();
  if (tid == 0) {
    // no more than the pool has room for (a table that repeats pages)
    const int back = (int)min(back_c, (long long)(pool - free_pages));
    a.pg.cu_rows[0] = 0;
    a.ix.head[0] = head;
    a.ix.head[1] = free_pages;
    a.ix.head[2] = back;
    a.pg.ring_state[0] = (int)(((long long)head + sTaken) % pool);
    a.pg.ring_state[1] = free_pages - sTaken + back;
  }
}

// The request of packed row m (n: none).
__device__ __forceinline__ int row_request(const int32_t* __restrict__ cu, int n, int m) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid + 1] <= m) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}
// The request whose entries (from cu[s] >> shift, plus mul s, on) hold entry i.
__device__ __forceinline__ int entry_request(const int32_t* __restrict__ cu, int n, int i, int shift,
                                             int mul) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((cu[mid] >> shift) + mul * mid <= i) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

struct PlanRing {
  int head, free_pages;
};

// Pool page of logical page lp of request s (-1 outside the pool): one it held,
// or one of those taken in this call.
__device__ __forceinline__ int plan_page(const PlanArgs& a, const PlanRing& g, const PageReq& q, int s,
                                         int lp) {
  int page;
  if (lp < q.held) {
    page = a.pg.table[(size_t)s * a.pg.max_pages + lp];
  } else {
    const long long i = (long long)g.head + q.first + (lp - q.held);
    page = a.pg.ring[i < a.pg.pool ? i : i - a.pg.pool];
  }
  return (unsigned)page < (unsigned)a.pg.pool ? page : -1;
}

__device__ __forceinline__ PageTile plan_tile(const PlanArgs& a, const int32_t* cu, int i, int shift) {
  const int s = entry_request(cu, a.pg.n_seq, i, shift, 1);
  const int at = (i - ((cu[s] >> shift) + s)) << shift;
  const PageReq q = a.ix.req[s];
  if (q.first < 0 || at >= q.rows) return PageTile{0, 0, 0, 0};
  return PageTile{s, cu[s] + at, min(q.rows - at, 1 << shift) | (q.ctx / NMDLM_PAGE) << 6, q.ctx + q.rows};
}

__device__ void plan_entries(const PlanArgs& a, const int32_t* cu, int tid, int nth) {
  const PlanRing g{a.ix.head[0], a.ix.head[1]};
  const int n = a.pg.n_seq;
  for (int m = tid; m < a.pg.max_rows; m += nth) {
    const int s = row_request(cu, n, m);
    long long slot = -1;
    int pos = 0;
    if (s < n) {
      const PageReq q = a.ix.req[s];
      if (q.first >= 0) {
        pos = q.ctx + m - cu[s];
        const int page = plan_page(a, g, q, s, pos / NMDLM_PAGE);
        if (page >= 0) slot = (long long)page * NMDLM_PAGE + pos % NMDLM_PAGE;
      }
    }
    a.pg.slot[m] = slot;
    a.pg.pos[m] = pos;
  }
  for (int i = tid; i < a.ix.n16; i += nth) a.ix.t16[i] = plan_tile(a, cu, i, 4);
  for (int i = tid; i < a.ix.n32; i += nth) a.ix.t32[i] = plan_tile(a, cu, i, 5);
  for (int i = tid; i < a.ix.n_runs; i += nth) {
    const int s = entry_request(cu, n, i, 6, 2);
    const PageReq q = a.ix.req[s];
    PageRun r{-1, 0, 0, 0};
    if (q.first >= 0) {
      const int lp = q.ctx / NMDLM_PAGE + (i - ((cu[s] >> 6) + 2 * s));
      const int b = max(q.ctx, lp * NMDLM_PAGE), e = min(q.ctx + q.rows, (lp + 1) * NMDLM_PAGE);
      if (b < e) {
        r = PageRun{plan_page(a, g, q, s, lp), b - lp * NMDLM_PAGE, cu[s] + b - q.ctx, e - b};
        // a page taken in this call has at least one of its rows
        if (lp >= q.held) a.pg.table[(size_t)s * a.pg.max_pages + lp] = r.page;
      }
    }
    a.ix.runs[i] = r;
  }
  // pages of ended requests, behind the ring's last
  const int back = a.ix.head[2];
  for (int i = tid; i < back; i += nth) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.ix.back[mid] <= i) lo = mid;
      else hi = mid - 1;
    }
    const long long at = (long long)g.head + g.free_pages + i;  // below 3 pool
    a.pg.ring[at % a.pg.pool] = a.pg.table[(size_t)lo * a.pg.max_pages + (i - a.ix.back[lo])];
  }
}

__global__ __launch_bounds__(kPlanThreads) void k_page_plan(PlanArgs a) {
  plan_sums(a);
  __syncthreads();
  plan_entries(a, a.pg.cu_rows, threadIdx.x, kPlanThreads);
}
__global__ __launch_bounds__(kPlanThreads) void k_page_sums(PlanArgs a) { plan_sums(a); }
__global__ __launch_bounds__(256) void k_page_entries(PlanArgs a) {
  plan_entries(a, a.pg.cu_rows, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

constexpr long long kPlanOneEntries = 4 * kPlanThreads;  // entries of a plan in one launch

nmdlm_status launch_page_plan(const nmdlm_pages& pg, const int32_t* ctx, const int32_t* rows,
                              int32_t* status, hipStream_t st) {
  PlanArgs a{pg, ctx, rows, status, {}};
  page_index_layout(pg.n_seq, pg.max_rows, pg.index, &a.ix);
  const long long entries = (long long)pg.max_rows + a.ix.n16 + a.ix.n32 + a.ix.n_runs;
  if (entries <= kPlanOneEntries) {
    hipLaunchKernelGGL(k_page_plan, dim3(1), dim3(kPlanThreads), 0, st, a);
    return hip_status();
  }
  hipLaunchKernelGGL(k_page_sums, dim3(1), dim3(kPlanThreads), 0, st, a);
  const nmdlm_status rc = hip_status();
  if (rc != NMDLM_OK) return rc;
  const unsigned grid = (unsigned)std::min<long long>((pg.max_rows + 255) / 256, 1024);
  hipLaunchKernelGGL(k_page_entries, dim3(grid), dim3(256), 0, st, a);
  return hip_status();
}

// ---------------------------------------------------------------------------
// Store.  A wave takes one run of rows (of one page), a head and a timestep:
// lane j = position j of the page.  Keys go to their rows as they are; values
// are a 64 x 64 bit transpose per 64 channels, lane j's word (channels) becoming
// lane c's word (positions); the keys are transposed too, for the counts.
// ---------------------------------------------------------------------------

// bit (lane i, bit j) <-> bit (lane j, bit i): for s = 32 .. 1 the blocks off
// the diagonal of every 2s x 2s block change places.
__device__ __forceinline__ uint64_t transpose64(uint64_t x, int lane) {
  constexpr uint64_t keep[6] = {0x00000000FFFFFFFFull, 0x0000FFFF0000FFFFull, 0x00FF00FF00FF00FFull,
                                0x0F0F0F0F0F0F0F0Full, 0x3333333333333333ull, 0x5555555555555555ull};
#pragma unroll
  for (int k = 0; k < 6; ++k) {
    const int s = 32 >> k;
    const uint64_t y = __shfl_xor((unsigned long long)x, s);
    x = lane & s ? (x & ~keep[k]) | ((y & ~keep[k]) >> s) : (x & keep[k]) | ((y & keep[k]) << s);
  }
  return x;
}

template <int DHW>
__global__ __launch_bounds__(256) void k_page_store(const PageRun* __restrict__ runs,
                                                    const uint64_t* __restrict__ k,
                                                    const uint64_t* __restrict__ v, int T, int H,
                                                    int max_rows, int pool,
                                                    uint64_t* __restrict__ k_pages,
                                                    uint64_t* __restrict__ v_pages,
                                                    uint8_t* __restrict__ counts) {
  const PageRun r = runs[blockIdx.x];
  const int unit = __builtin_amdgcn_readfirstlane((int)blockIdx.y * 4 + ((int)threadIdx.x >> 6));
  if ((unsigned)r.page >= (unsigned)pool || r.n < 1 || unit >= T * H) return;  // wave-uniform
  const int lane = threadIdx.x & 63;
  const int t = unit / H, h = unit - t * H;
  const int dw = H * DHW;
  const size_t at = ((size_t)r.page * H + h) * T + t;
  uint64_t* kp = k_pages + at * NMDLM_PAGE * DHW;
  uint64_t* vp = v_pages + at * 64 * DHW;
  const int i = lane - r.off;
  const bool in = i >= 0 && i < r.n;
  const size_t row = ((size_t)t * max_rows + r.row + (in ? i : 0)) * dw + h * DHW;
  uint64_t kw[DHW], vw[DHW], vo[DHW];
#pragma unroll
  for (int w = 0; w < DHW; ++w) {
    kw[w] = in ? k[row + w] : (lane < r.off ? kp[lane * DHW + w] : 0ull);
    vw[w] = in ? v[row + w] : 0ull;
    vo[w] = r.n < NMDLM_PAGE ? vp[w * 64 + lane] : 0ull;
  }
  const uint64_t mask = (r.n < 64 ? (1ull << r.n) - 1 : ~0ull) << r.off;
#pragma unroll
  for (int w = 0; w < DHW; ++w) {
    if (in) kp[lane * DHW + w] = kw[w];
    vp[w * 64 + lane] = (vo[w] & ~mask) | transpose64(vw[w], lane);
    counts[at * 64 * DHW + w * 64 + lane] = (uint8_t)__popcll(transpose64(kw[w], lane));
  }
}

nmdlm_status launch_page_store(const nmdlm_pages& pg, const uint64_t* k, const uint64_t* v, int T, int H,
                               int dh, uint64_t* k_pages, uint64_t* v_pages, uint8_t* counts,
                               hipStream_t st) {
  PageIndex ix;
  page_index_layout(pg.n_seq, pg.max_rows, pg.index, &ix);
  const dim3 grid((unsigned)ix.n_runs, (unsigned)((T * H + 3) / 4));
  if (dh == 64)
    hipLaunchKernelGGL(k_page_store<1>, grid, dim3(256), 0, st, ix.runs, k, v, T, H, pg.max_rows, pg.pool,
                       k_pages, v_pages, counts);
  else
    hipLaunchKernelGGL(k_page_store<2>, grid, dim3(256), 0, st, ix.runs, k, v, T, H, pg.max_rows, pg.pool,
                       k_pages, v_pages, counts);
  return hip_status();
}

// ---------------------------------------------------------------------------
// Select, scores.  S = Q . counts over T*dh channels on v_mfma_i32_16x16x64_i8
// (counts are at most 64, query bits 0 or 1: exact): A = 16 pages, row = page,
// B = the tile's 16 queries.  Lane (g, c) holds channels 16g .. 16g+15 of page c
// and of query c, and gets pages 4g + e of query c.
// ---------------------------------------------------------------------------
__device__ __forceinline__ v4i bits_to_bytes(uint32_t x) {  // byte j of 16 = bit j
  v4i r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (int)((((x >> (4 * i)) & 0xFu) * 0x00204081u) & 0x01010101u);
  return r;
}

template <int DHW>
__global__ __launch_bounds__(256) void k_page_scores(const PageTile* __restrict__ tiles,
                                                     const int32_t* __restrict__ table, int max_pages,
                                                     int pool, const uint64_t* __restrict__ q, int T, int H,
                                                     int max_rows, const uint8_t* __restrict__ counts,
                                                     int32_t* __restrict__ scores, int ld) {
  typedef const uint16_t __attribute__((may_alias)) u16_in;
  typedef const v4i __attribute__((may_alias)) v4i_in;
  const PageTile tl = tiles[blockIdx.x];
  if ((tl.n_full & 63) == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
  const int h = blockIdx.y, P = tl.n_full >> 6, nr = tl.n_full & 63;
  const int p0 = ((int)blockIdx.z * 4 + wave) * 16;
  if (p0 >= P) return;
  const int id = table[(size_t)tl.s * max_pages + min(p0 + c, P - 1)];
  const bool there = (unsigned)id < (unsigned)pool;
  const uint8_t* cp = counts + ((size_t)(there ? id : 0) * H + h) * T * (64 * DHW) + 16 * g;
  const uint64_t* qp = q + (size_t)(tl.row + min(c, nr - 1)) * (H * DHW) + h * DHW;
  v4i s = v4i{0, 0, 0, 0};
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int w = 0; w < DHW; ++w) {
      v4i x = *reinterpret_cast<v4i_in*>(cp + (t * DHW + w) * 64);
      if (!there) x = v4i{0, 0, 0, 0};
      const uint32_t b = reinterpret_cast<u16_in*>(qp + (size_t)t * max_rows * (H * DHW) + w)[g];
      s = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, bits_to_bytes(b), s, 0, 0, 0);
    }
  if (c < nr)
    *reinterpret_cast<v4i*>(scores + ((size_t)(tl.row + c) * H + h) * ld + p0 + 4 * g) = s;
}

// Select, choice: a wave per row and head.  The n_sel-th largest score is built
// bit by bit from the top (counting the scores that reach each candidate); the
// pages above it are taken, and of those equal to it the lowest.
__global__ __launch_bounds__(256) void k_page_pick(const PageTile* __restrict__ tiles, int H, int n_sel,
                                                   const int32_t* __restrict__ scores, int ld, int words,
                                                   uint64_t* __restrict__ sel) {
  const PageTile tl = tiles[blockIdx.x];
  if ((tl.n_full & 63) == 0) return;
  const int h = blockIdx.y, lane = threadIdx.x & 63;
  const int P = tl.n_full >> 6, nr = tl.n_full & 63, nP = (tl.keys + 63) / 64;
  for (int r = threadIdx.x >> 6; r < nr; r += 4) {  // wave-uniform
    const size_t at = (size_t)(tl.row + r) * H + h;
    const int32_t* sc = scores + at * ld;
    int thr = 0, take = 0;  // scores above thr, and the first `take` equal ones
    if (n_sel >= P) {
      thr = -1;
    } else if (n_sel > 0) {
      for (int bit = 1 << 16; bit > 0; bit >>= 1) {  // scores are at most 8*128*64 = 2^16
        int n = 0;
        for (int p = lane; p < P; p += 64) n += sc[p] >= (thr | bit) ? 1 : 0;
        for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
        if (n >= n_sel) thr |= bit;
      }
      int above = 0;
      for (int p = lane; p < P; p += 64) above += sc[p] > thr ? 1 : 0;
      for (int o = 32; o > 0; o >>= 1) above += __shfl_xor(above, o);
      take = n_sel - above;
    } else {
      thr = 1 << 30;
    }
    for (int w = 0; w < words; ++w) {
      const int p = w * 64 + lane;
      const int s = p < P ? sc[p] : -2;
      const uint64_t own = __builtin_amdgcn_ballot_w64(p >= P && p < nP);
      uint64_t eq = __builtin_amdgcn_ballot_w64(s == thr);
      uint64_t word = __builtin_amdgcn_ballot_w64(s > thr) | own;
      // the lowest `take` of the equal ones
      const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(eq >> 32),
                                                   __builtin_amdgcn_mbcnt_lo((uint32_t)eq, 0));
      word |= __builtin_amdgcn_ballot_w64(s == thr && before < take);
      take = max(take - (int)__popcll(eq), 0);
      if (lane == 0) sel[at * words + w] = word;
    }
  }
}

static int select_ld(const nmdlm_pages& pg) { return (pg.max_pages + 15) / 16 * 16; }

size_t page_select_ws(const nmdlm_pages& pg, int H) {
  return align_up((size_t)pg.max_rows * H * select_ld(pg) * sizeof(int32_t), 256);
}

nmdlm_status launch_page_select(const nmdlm_pages& pg, const uint64_t* q, int T, int H, int dh,
                                const uint8_t* counts, int n_sel, uint64_t* sel, void* ws,
                                hipStream_t st) {
  PageIndex ix;
  page_index_layout(pg.n_seq, pg.max_rows, pg.index, &ix);
  const int ld = select_ld(pg);
  int32_t* scores = static_cast<int32_t*>(ws);
  const dim3 grid((unsigned)ix.n16, (unsigned)H, (unsigned)((pg.max_pages + 63) / 64));
  if (dh == 64)
    hipLaunchKernelGGL(k_page_scores<1>, grid, dim3(256), 0, st, ix.t16, pg.table, pg.max_pages, pg.pool, q,
                       T, H, pg.max_rows, counts, scores, ld);
  else
    hipLaunchKernelGGL(k_page_scores<2>, grid, dim3(256), 0, st, ix.t16, pg.table, pg.max_pages, pg.pool, q,
                       T, H, pg.max_rows, counts, scores, ld);
  const nmdlm_status rc = hip_status();
  if (rc != NMDLM_OK) return rc;
  hipLaunchKernelGGL(k_page_pick, dim3((unsigned)ix.n16, (unsigned)H), dim3(256), 0, st, ix.t16, H, n_sel,
                     scores, ld, (pg.max_pages + 63) / 64, sel);
  return hip_status();
}

}  // namespace nmdlm
