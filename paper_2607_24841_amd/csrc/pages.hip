// Paged spike caches: block tables and work lists from the requests' lengths,
// the store of packed rows into pages, and the choice of context pages by
// their spike counts.
#include <algorithm>

#include "pages.h"

namespace nmdlm {

// ---------------------------------------------------------------------------
// Plan.  Two steps: sums over the requests in order (rows, pages taken and given
// back, list entries), by one workgroup; then every row by itself, its request
// found by bisection of cu_rows.  Latency bound, a chain of dependent loads, scans
// and barriers: 128 requests of 16 rows 8.2 us in one launch, 1000 requests of 90
// thousand rows 5.0 and 6.9 us in two.  The scans go by DPP within a wave and over
// the waves' sums (by shuffles and a loop over the sums the first launch took 13
// us, 4 KB of straight code).
// ---------------------------------------------------------------------------
struct PlanArgs {
  nmdlm_pages pg;
  const int32_t* ctx;
  const int32_t* rows;
  int32_t* status;
  PageIndex ix;
};

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;

// Inclusive sums of K values over the workgroup, in place; total: the sums of all.
template <int K>
__device__ __forceinline__ void block_scan(int (&x)[K], int (&total)[K], int (*sWave)[kPlanWaves]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    x[k] = wave_scan(x[k]);
    if (lane == 63) sWave[k][wave] = x[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {  // the waves' sums, one a lane of a row of 16
    const int y = row_scan(sWave[k][lane & 15]);
    total[k] = __builtin_amdgcn_readlane(y, 15);
    if (wave > 0) x[k] += __builtin_amdgcn_readlane(y, wave - 1);
  }
}
static_assert(kPlanWaves == 16, "a row of lanes holds the waves' sums");

// A chunk's sums fit 32 bits (1024 requests of at most 2^19 rows, 2^17 pages);
// the carries between chunks are 64 bits wide.
__device__ void plan_sums(const PlanArgs& a, int32_t* sCu, PageReq* sReq) {
  __shared__ int sRows[1][kPlanWaves], sPages[2][kPlanWaves], sLists[3][kPlanWaves];
  __shared__ int sTaken;
  const int tid = threadIdx.x, n = a.pg.n_seq, pool = a.pg.pool;
  const int first = a.pg.ring_state[0], head = (unsigned)first < (unsigned)pool ? first : 0;
  const int free_pages = min(max(a.pg.ring_state[1], 0), pool);
  long long row_c = 0, need_c = 0, back_c = 0;
  int t16_c = 0, t32_c = 0, run_c = 0;
  int bits = 0;
  if (tid == 0) sTaken = 0;
  for (int s0 = 0; s0 < n; s0 += kPlanThreads) {  // uniform
    const int s = s0 + tid;
    const bool in = s < n;
    const int ctx = in ? a.ctx[s] : 0, rows = in ? a.rows[s] : 0, held = in ? a.pg.held[s] : 0;
    const int r = rows > 0 && rows <= a.pg.max_rows ? rows : 0;
    int rs[1] = {r}, r_all[1];
    block_scan<1>(rs, r_all, sRows);
    const long long row_end = row_c + rs[0];
    const long long end = (long long)ctx + rows;
    const bool held_ok = held >= 0 && held <= a.pg.max_pages;
    const bool fits = in && rows >= 0 && rows <= a.pg.max_rows && held_ok && ctx >= 0 &&
                      ctx <= (long long)held * NMDLM_PAGE &&
                      end <= (long long)a.pg.max_pages * NMDLM_PAGE && row_end <= a.pg.max_rows;
    const bool ended = in && rows == -1 && held_ok;
    const int pages = fits ? (int)((end + NMDLM_PAGE - 1) >> 6) : 0;
    const int need = fits ? max(pages - held, 0) : 0, back = ended ? held : 0;
    int ps[2] = {need, back}, p_all[2];
    block_scan<2>(ps, p_all, sPages);
    const long long need_end = need_c + ps[0], back_end = back_c + ps[1];
    const bool ok = fits && (need == 0 || need_end <= free_pages);
    // list entries of a served request
    const int m = ok ? rows : 0;
    const int n16 = (m + 15) >> 4, n32 = (m + 31) >> 5, n_run = m > 0 ? pages - (ctx >> 6) : 0;
    int ls[3] = {n16, n32, n_run}, l_all[3];
    block_scan<3>(ls, l_all, sLists);
    if (in) {
      const int cu = (int)min(row_end - r, (long long)a.pg.max_rows);
      const PageReq q{ok ? (int)min(need_end - need, (long long)pool) : -1, held, ctx, rows, cu,
                      t16_c + ls[0] - n16, t32_c + ls[1] - n32, run_c + ls[2] - n_run};
      a.pg.cu_rows[s + 1] = (int)min(row_end, (long long)a.pg.max_rows);
      a.ix.req[s] = q;
      a.ix.back[s] = (int)min(back_end - back, (long long)pool);
      if (sCu) {
        sCu[s + 1] = (int)min(row_end, (long long)a.pg.max_rows);
        sReq[s] = q;
      }
      if (ended) a.pg.held[s] = 0;
      else if (ok) a.pg.held[s] = max(held, pages);
      if (!fits && !ended) bits |= NMDLM_STATUS_BAD_REQUEST;
      if (fits && !ok) bits |= NMDLM_STATUS_PAGES_SHORT;
      if (ok && need > 0) atomicMax(&sTaken, (int)need_end);
    }
    row_c += r_all[0];
    need_c += p_all[0];
    back_c += p_all[1];
    t16_c += l_all[0];
    t32_c += l_all[1];
    run_c += l_all[2];
  }
  if (bits && a.status) atomicOr(a.status, bits);
  __syncthreads();
  if (tid == 0) {
    // no more than the pool has room for (a table that repeats pages)
    const int back = (int)min(back_c, (long long)(pool - free_pages));
    a.pg.cu_rows[0] = 0;
    if (sCu) sCu[0] = 0;
    a.ix.head[0] = head;
    a.ix.head[1] = free_pages;
    a.ix.head[2] = back;
    a.ix.head[3] = t16_c;
    a.ix.head[4] = t32_c;
    a.ix.head[5] = run_c;
    const int next = head + sTaken;
    a.pg.ring_state[0] = next < pool ? next : next - pool;
    a.pg.ring_state[1] = free_pages - sTaken + back;
  }
}

// The request of packed row m (n: none).
__device__ __forceinline__ int row_request(const int32_t* cu, int n, int m) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid + 1] <= m) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

// Pool page of logical page lp of request s (-1 outside the pool): one it held,
// or one of those taken in this call.
__device__ __forceinline__ int plan_page(const PlanArgs& a, int head, const PageReq& q, int s, int lp) {
  int page;
  if (lp < q.held) {
    page = a.pg.table[(size_t)s * a.pg.max_pages + lp];
  } else {
    const int i = head + q.first + (lp - q.held);
    page = a.pg.ring[i < a.pg.pool ? i : i - a.pg.pool];
  }
  return (unsigned)page < (unsigned)a.pg.pool ? page : -1;
}

// Every row writes its slot and position; the first of a tile or of a page's
// rows writes the list entry and, for a page taken in this call (each has at
// least one row), the table's.
__device__ void plan_rows(const PlanArgs& a, const int32_t* cu, const PageReq* req, int tid, int nth) {
  const int head = a.ix.head[0], n = a.pg.n_seq;
  for (int m = tid; m < a.pg.max_rows; m += nth) {
    const int s = row_request(cu, n, m);
    long long slot = -1;
    int pos = 0;
    PageTile tl{0, 0, 0, 0};
    if (s < n) {
      const PageReq q = req[s];
      if (q.first >= 0) {
        const int i = m - q.row, end = q.ctx + q.rows, full = q.ctx >> 6 << 6;  // all at least 0
        pos = q.ctx + i;
        const int lp = pos >> 6, off = pos & 63, page = plan_page(a, head, q, s, lp);
        if (page >= 0) slot = (long long)page * NMDLM_PAGE + off;
        tl = PageTile{s, m, 1 | full, end};
        if ((i & 15) == 0) a.ix.t16[q.t16 + (i >> 4)] = PageTile{s, m, min(q.rows - i, 16) | full, end};
        if ((i & 31) == 0) a.ix.t32[q.t32 + (i >> 5)] = PageTile{s, m, min(q.rows - i, 32) | full, end};
        if (i == 0 || off == 0) {
          a.ix.runs[q.run + lp - (q.ctx >> 6)] = PageRun{page, off, m, min(NMDLM_PAGE - off, end - pos)};
          if (lp >= q.held) a.pg.table[(size_t)s * a.pg.max_pages + lp] = page;
        }
      }
    }
    a.pg.slot[m] = slot;
    a.pg.pos[m] = pos;
    a.ix.t1[m] = tl;
  }
  for (int i = a.ix.head[3] + tid; i < a.ix.n16; i += nth) a.ix.t16[i] = PageTile{0, 0, 0, 0};
  for (int i = a.ix.head[4] + tid; i < a.ix.n32; i += nth) a.ix.t32[i] = PageTile{0, 0, 0, 0};
  for (int i = a.ix.head[5] + tid; i < a.ix.n_runs; i += nth) a.ix.runs[i] = PageRun{-1, 0, 0, 0};
  // pages of ended requests, behind the ring's last
  const int back = a.ix.head[2], free_pages = a.ix.head[1];
  for (int i = tid; i < back; i += nth) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.ix.back[mid] <= i) lo = mid;
      else hi = mid - 1;
    }
    int at = head + free_pages + i;  // below 3 pool
    while (at >= a.pg.pool) at -= a.pg.pool;
    a.pg.ring[at] = a.pg.table[(size_t)lo * a.pg.max_pages + (i - a.ix.back[lo])];
  }
}

// One launch for few rows and requests: what the rows look up stays in LDS.  64
// requests of 8 rows 7.6 us (with the copy that puts the state back) against 9.6 in
// two launches, of 32 10.2 against 10.9, of 63 12.5 against 11.4; 1000 of one 9.9
// against 11.8; 8 of 250 8.5 against 9.5, of 500 10.3 against 9.4.
constexpr int kPlanOneRows = 2560;
__global__ __launch_bounds__(kPlanThreads) void k_page_plan(PlanArgs a) {
  __shared__ int32_t sCu[kPlanThreads + 1];
  __shared__ PageReq sReq[kPlanThreads];
  touch_kernargs<sizeof(PlanArgs)>();
  plan_sums(a, sCu, sReq);
  __syncthreads();
  plan_rows(a, sCu, sReq, threadIdx.x, kPlanThreads);
}

// Two for many.
constexpr int kPlanLdsRequests = 4096;  // bisection in LDS up to these
__global__ __launch_bounds__(kPlanThreads) void k_page_sums(PlanArgs a) {
  touch_kernargs<sizeof(PlanArgs)>();
  plan_sums(a, nullptr, nullptr);
}
__global__ __launch_bounds__(256) void k_page_rows(PlanArgs a) {
  __shared__ int32_t sCu[kPlanLdsRequests + 1];
  touch_kernargs<sizeof(PlanArgs)>();
  const int n = a.pg.n_seq;
  const int32_t* cu = a.pg.cu_rows;
  if (n <= kPlanLdsRequests) {  // uniform
    for (int i = threadIdx.x; i <= n; i += 256) sCu[i] = cu[i];
    __syncthreads();
    cu = sCu;
  }
  plan_rows(a, cu, a.ix.req, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

nmdlm_status launch_page_plan(const nmdlm_pages& pg, const int32_t* ctx, const int32_t* rows,
                              int32_t* status, hipStream_t st) {
  PlanArgs a{pg, ctx, rows, status, {}};
  page_index_layout(pg.n_seq, pg.max_rows, pg.index, &a.ix);
  if (pg.max_rows <= kPlanOneRows && pg.n_seq <= kPlanThreads) {
    hipLaunchKernelGGL(k_page_plan, dim3(1), dim3(kPlanThreads), 0, st, a);
    return hip_status();
  }
  hipLaunchKernelGGL(k_page_sums, dim3(1), dim3(kPlanThreads), 0, st, a);
  const nmdlm_status rc = hip_status();
  if (rc != NMDLM_OK) return rc;
  const unsigned grid = (unsigned)std::min<long long>((pg.max_rows + 255) / 256, 1024);
  hipLaunchKernelGGL(k_page_rows, dim3(grid), dim3(256), 0, st, a);
  return hip_status();
}

// ---------------------------------------------------------------------------
// Store.  A wave takes one run of rows (of one page), a head and a timestep:
// lane j = position j of the page.  Keys go to their rows as they are; values
// are a 64 x 64 bit transpose per 64 channels, lane j's word (channels) becoming
// lane c's word (positions); the keys are transposed too, for the counts.  The
// waves of a workgroup are the heads of one timestep, which share the rows'
// lines.  Six prompts, 5.7 thousand rows of 2048 channels, T = 4, 27.6 MB: 9.4 us,
// 2.9 TB/s, bound by the rows' loads (a lane's 16 bytes of a head are a line of
// their own); 64 requests of 4 rows, T = 8, 512 channels 4.3 us, the start of a launch.
// ---------------------------------------------------------------------------

// What a lane needs of the transpose's steps: the bits it keeps and how far the
// partner's are rotated.
struct TransposeLane {
  uint32_t sel8, keep4, rot4, keep2, rot2, keep1, rot1;
  __device__ __forceinline__ explicit TransposeLane(int lane) {
    sel8 = lane & 8 ? 0x03070105u : 0x06020400u;  // bytes of (partner, own): see step8
    keep4 = lane & 4 ? 0xF0F0F0F0u : 0x0F0F0F0Fu;
    rot4 = lane & 4 ? 4u : 28u;
    keep2 = lane & 2 ? 0xCCCCCCCCu : 0x33333333u;
    rot2 = lane & 2 ? 2u : 30u;
    keep1 = lane & 1 ? 0xAAAAAAAAu : 0x55555555u;
    rot1 = lane & 1 ? 1u : 31u;
  }
};

// bit (lane i, bit j) <-> bit (lane j, bit i): for s = 32 .. 1 the blocks off the
// diagonal of every 2s x 2s block change places.  Lanes 32 and 16 apart swap
// registers, nearer ones exchange by DPP; a partner's bits come rotated by s, what
// crosses a block's border falling on bits that are kept.
__device__ __forceinline__ uint64_t transpose64(uint64_t x, const TransposeLane& tl) {
  uint32_t lo = (uint32_t)x, hi = (uint32_t)(x >> 32);
  {
    const auto r = __builtin_amdgcn_permlane32_swap(lo, hi, false, false);
    lo = r[0];
    hi = r[1];
  }
  {
    const uint32_t p = __builtin_amdgcn_perm(hi, lo, 0x05040100u);  // the low halves
    const uint32_t q = __builtin_amdgcn_perm(hi, lo, 0x07060302u);  // the high halves
    const auto r = __builtin_amdgcn_permlane16_swap(p, q, false, false);
    lo = __builtin_amdgcn_perm(r[1], r[0], 0x05040100u);
    hi = __builtin_amdgcn_perm(r[1], r[0], 0x07060302u);
  }
  uint32_t d[2] = {lo, hi};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    uint32_t v = d[k], y;
    y = __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, true);  // row_ror:8: lane ^ 8
    v = __builtin_amdgcn_perm(y, v, tl.sel8);
    y = __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true);  // half mirror: lane ^ 7
    y = __builtin_amdgcn_update_dpp(0, y, 0x1B, 0xf, 0xf, true);   // quad_perm 3210: lane ^ 3
    v = (v & tl.keep4) | (__builtin_amdgcn_alignbit(y, y, tl.rot4) & ~tl.keep4);
    y = __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true);   // quad_perm 1032 of pairs: lane ^ 2
    v = (v & tl.keep2) | (__builtin_amdgcn_alignbit(y, y, tl.rot2) & ~tl.keep2);
    y = __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);   // lane ^ 1
    v = (v & tl.keep1) | (__builtin_amdgcn_alignbit(y, y, tl.rot1) & ~tl.keep1);
    d[k] = v;
  }
  return (uint64_t)d[1] << 32 | d[0];
}

constexpr int kStoreWaves = 16;

template <int DHW>
__global__ __launch_bounds__(64 * kStoreWaves) void k_page_store(
    const PageRun* __restrict__ runs, const uint64_t* __restrict__ k, const uint64_t* __restrict__ v, int T,
    int H, int max_rows, int pool, uint64_t* __restrict__ k_pages, uint64_t* __restrict__ v_pages,
    uint8_t* __restrict__ counts) {
  const PageRun r = runs[blockIdx.z];
  const int t = blockIdx.x;
  const int h = __builtin_amdgcn_readfirstlane((int)(blockIdx.y * (blockDim.x >> 6)) + ((int)threadIdx.x >> 6));
  if ((unsigned)r.page >= (unsigned)pool || r.n < 1 || h >= H) return;  // wave-uniform
  const int lane = threadIdx.x & 63;
  const TransposeLane tl(lane);
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
    vp[w * 64 + lane] = (vo[w] & ~mask) | transpose64(vw[w], tl);
    counts[at * 64 * DHW + w * 64 + lane] = (uint8_t)__popcll(transpose64(kw[w], tl));
  }
}

nmdlm_status launch_page_store(const nmdlm_pages& pg, const uint64_t* k, const uint64_t* v, int T, int H,
                               int dh, uint64_t* k_pages, uint64_t* v_pages, uint8_t* counts,
                               hipStream_t st) {
  PageIndex ix;
  page_index_layout(pg.n_seq, pg.max_rows, pg.index, &ix);
  // heads of a workgroup: evenly, at most kStoreWaves; empty runs are the grid's last
  const int groups = (H + kStoreWaves - 1) / kStoreWaves, waves = (H + groups - 1) / groups;
  const dim3 grid(T, groups, ix.n_runs), block(64 * waves);
  if (dh == 64)
    hipLaunchKernelGGL(k_page_store<1>, grid, block, 0, st, ix.runs, k, v, T, H, pg.max_rows, pg.pool,
                       k_pages, v_pages, counts);
  else
    hipLaunchKernelGGL(k_page_store<2>, grid, block, 0, st, ix.runs, k, v, T, H, pg.max_rows, pg.pool,
                       k_pages, v_pages, counts);
  return hip_status();
}

// ---------------------------------------------------------------------------
// Select, scores.  S = Q . counts over T*dh channels on v_mfma_i32_16x16x64_i8
// (counts are at most 64, query bits 0 or 1: exact): A = 16 queries, B = 16
// pages; lane (g, c) holds channels 16g .. 16g+15 of query c and of page c and
// gets queries 4g + e of page c.
//
// The counts of a page are one run of T*dh bytes.  Loaded as the operand wants
// them, adjacent lanes read different pages and a load costs 64 cache accesses;
// so four lanes take 64 bytes of one page and the operands come from LDS.  Query
// bits come from LDS too, where a workgroup's rows stand once.  32 rows and 16 heads
// of 128 over 2046 pages, T = 4, 16.8 MB of counts: 8.9 us (14.4 loaded as the operand
// wants them), of which half is the chain arguments, tile, table, counts.
// ---------------------------------------------------------------------------
__device__ __forceinline__ v4i bits_to_bytes(uint32_t x) {  // byte j of 16 = bit j
  v4i r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (int)((((x >> (4 * i)) & 0xFu) * 0x00204081u) & 0x01010101u);
  return r;
}

struct SelectArgs {
  const PageTile* tiles;
  const int32_t* table;
  const uint64_t* q;
  const uint8_t* counts;
  uint64_t* sel;
  int32_t* scores;  // [head of the launch][max_rows][ld], where they do not stay in LDS
  int max_pages, pool, max_rows, words;
  int T, H, n_sel, ld;
};

// k-steps (of 64 channels) staged at once, and the 16-byte units between a wave's
// staged pages (one of padding): as many as the call has, for more workgroups a CU.
constexpr int kScoreSteps = 8;
__host__ __device__ constexpr int score_ld(int steps) { return (steps < kScoreSteps ? steps : kScoreSteps) * 4 + 1; }

// The query bits of the tile's rows, [T][ROWS][DHW] words (rows past the last:
// the last).  All threads of the workgroup.
template <int DHW, int ROWS>
__device__ __forceinline__ void stage_queries(const SelectArgs& a, const PageTile& tl, int h,
                                              uint64_t* sQ) {
  const int nr = tl.n_full & 63;
  for (int i = threadIdx.x; i < a.T * ROWS * DHW; i += blockDim.x) {
    const int w = i % DHW, r = (i / DHW) % ROWS, t = i / (DHW * ROWS);
    sQ[i] = a.q[((size_t)t * a.max_rows + tl.row + min(r, nr - 1)) * (a.H * DHW) + h * DHW + w];
  }
}

// The pool page of the lane's four among 16 logical pages from p0 on.
__device__ __forceinline__ int score_id(const SelectArgs& a, const PageTile& tl, int p0, int lane) {
  return a.table[(size_t)tl.s * a.max_pages + max(min(p0 + (lane >> 2), (tl.n_full >> 6) - 1), 0)];
}

// Scores of 16 pages and QG groups of 16 rows.  The loads of a round of
// k-steps are all issued before the first is used.
template <int DHW, int QG>
__device__ __forceinline__ void score_pages(const SelectArgs& a, int id, int h, int lane, const uint64_t* sQ,
                                            v4i* st, v4i (&s)[QG]) {
  typedef const v4i __attribute__((may_alias)) v4i_in;
  typedef const uint16_t __attribute__((may_alias)) u16_in;
  const int g = lane >> 4, c = lane & 15;
  const bool there = (unsigned)id < (unsigned)a.pool;
  const uint8_t* cp = a.counts + ((size_t)(there ? id : 0) * a.H + h) * a.T * (64 * DHW) + 16 * (lane & 3);
  const int steps = a.T * DHW, ld = score_ld(steps);
#pragma unroll
  for (int u = 0; u < QG; ++u) s[u] = v4i{0, 0, 0, 0};
  for (int k0 = 0; k0 < steps; k0 += kScoreSteps) {  // uniform
    v4i x[kScoreSteps];
#pragma unroll
    for (int k = 0; k < kScoreSteps; ++k)
      x[k] = *reinterpret_cast<v4i_in*>(cp + min(k0 + k, steps - 1) * 64);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < kScoreSteps; ++k)
      if (k0 + k < steps) st[(lane >> 2) * ld + k * 4 + (lane & 3)] = there ? x[k] : v4i{0, 0, 0, 0};
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int k = 0; k < kScoreSteps; ++k) {
      if (k0 + k >= steps) break;  // uniform
      const int t = (k0 + k) / DHW, w = (k0 + k) % DHW;
      const v4i y = st[c * ld + k * 4 + g];
#pragma unroll
      for (int u = 0; u < QG; ++u) {
        const uint32_t b =
            reinterpret_cast<u16_in*>(sQ + (t * (16 * QG) + 16 * u + c) * DHW + w)[g];
        s[u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bits_to_bytes(b), y, s[u], 0, 0, 0);
      }
    }
    __builtin_amdgcn_wave_barrier();  // the stage is read before the next round's stores
  }
}

// Tiles of 32 rows, so that a block's rows read the counts once; a wave per 16
// pages.
template <int DHW>
__global__ __launch_bounds__(256) void k_page_scores(SelectArgs a) {
  touch_kernargs<sizeof(SelectArgs)>();
  extern __shared__ v4i sStage[];  // of the four waves
  __shared__ uint64_t sQ[NMDLM_MAX_T * 32 * DHW];
  const PageTile tl = a.tiles[blockIdx.x];
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, h = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int nr = tl.n_full & 63, P = tl.n_full >> 6;
  if (nr == 0 || (int)blockIdx.z * 64 >= P) return;  // uniform
  const int p0 = ((int)blockIdx.z * 4 + wave) * 16;
  const int id = score_id(a, tl, p0, lane);
  stage_queries<DHW, 32>(a, tl, h, sQ);
  __syncthreads();
  if (p0 >= P) return;  // wave-uniform
  v4i s[2];
  score_pages<DHW, 2>(a, id, h, lane, sQ, sStage + wave * 16 * score_ld(a.T * DHW), s);
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 16 * u + 4 * g + e;
      if (r < nr) a.scores[((size_t)h * a.max_rows + tl.row + r) * a.ld + p0 + c] = s[u][e];
    }
}

// Select, choice: a wave per row and head.  The scores stand in registers (score
// p in lane p % 64, register p / 64); the n_sel-th largest is found by bisection
// between 0 and the largest, and often earlier:
// where exactly n_sel scores reach the middle.  Of the scores equal to the last
// one taken the lowest pages are taken.  64 of 2046 for 512 rows and heads: 9.7 us
// (313 with the scores read again for each of 17 bits).  Half of it is the bisection,
// some 8 rounds of 32 comparisons and a sum over the wave: with the scores' kernel
// 17.5 us, and 12.7 with n_sel 0 or every page taken; the rest is the start of a launch
// and a chain of tile, scores and words.

struct Pick {
  int thr, ties;  // scores above thr, and the first `ties` equal to it
};
template <int NR>
__device__ __forceinline__ Pick pick_threshold(const int (&s)[NR], int P, int n_sel) {
  if (n_sel >= P) return Pick{-1, 0};  // every page (lanes past the last hold -1)
  if (n_sel == 0) return Pick{1 << 30, 0};
  int lo = 0, hi = 0;
#pragma unroll
  for (int r = 0; r < NR; ++r) hi = max(hi, s[r]);
  hi = wave_max(hi) + 1;
  int above = 0;  // scores >= hi; scores >= lo are at least n_sel
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    int n = 0;
    if constexpr (NR <= 8) {  // by the scalar unit: fewer instructions than a sum over lanes
#pragma unroll
      for (int r = 0; r < NR; ++r) n += (int)__popcll(__builtin_amdgcn_ballot_w64(s[r] >= mid));
    } else {
#pragma unroll
      for (int r = 0; r < NR; ++r) n += s[r] >= mid ? 1 : 0;
      n = wave_sum(n);
    }
    if (n == n_sel) return Pick{mid - 1, 0};
    if (n > n_sel) {
      lo = mid;
    } else {
      hi = mid;
      above = n;
    }
  }
  return Pick{lo, n_sel - above};
}

// The word of 64 pages whose scores the lanes hold; takes its ties off.
__device__ __forceinline__ uint64_t pick_word(int s, int thr, int& ties, int p, int P, int nP) {
  uint64_t word = __builtin_amdgcn_ballot_w64(s > thr || (p >= P && p < nP));
  if (ties > 0) {  // wave-uniform
    const uint64_t eq = __builtin_amdgcn_ballot_w64(s == thr);
    word |= __builtin_amdgcn_ballot_w64(s == thr && bits_before(eq) < ties);
    ties -= min((int)__popcll(eq), ties);
  }
  return word;
}

template <int NR>
__device__ __forceinline__ void pick_row(const int32_t* sc, int P, int nP, int n_sel, int words,
                                         uint64_t* __restrict__ out, int lane) {
  int s[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int p = r * 64 + lane, x = sc[max(min(p, P - 1), 0)];
    s[r] = p < P ? x : -1;
  }
  Pick k = pick_threshold<NR>(s, P, n_sel);
  uint64_t mine = 0;
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const uint64_t w = pick_word(s[r], k.thr, k.ties, r * 64 + lane, P, nP);
    if (lane == r) mine = w;
  }
  // words past the scores': the request's own pages, or none
  for (int w = lane; w < words; w += 64) {
    uint64_t x = mine;
    if (w >= NR) {
      const int a = max(P - w * 64, 0), b = min(nP - w * 64, 64);
      x = a < b ? ((b < 64 ? 1ull << b : 0ull) - (1ull << a)) : 0ull;
    }
    out[w] = x;
  }
}

// The same with the scores read again in every round, for contexts of more
// pages than the registers hold: 512 rows and heads, with the scores' kernel, 127 us
// over 3000 pages (30 with n_sel 0) and 1.9 ms over 20 thousand.
__device__ void pick_row_long(const int32_t* sc, int P, int nP, int n_sel, int words,
                              uint64_t* __restrict__ out, int lane) {
  int thr = n_sel > 0 ? 0 : 1 << 30, ties = 0;
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
    ties = n_sel - __builtin_amdgcn_readfirstlane(above);
  }
  for (int w = 0; w < words; ++w) {
    const int p = w * 64 + lane;
    const uint64_t word = pick_word(p < P ? sc[p] : -2, thr, ties, p, P, nP);
    if (lane == 0) out[w] = word;
  }
}

// P at most 128.
__device__ __forceinline__ void pick_few(const int32_t* sc, int P, int nP, int n_sel, int words,
                                         uint64_t* __restrict__ out, int lane) {
  if (P <= 64) pick_row<1>(sc, P, nP, n_sel, words, out, lane);
  else pick_row<2>(sc, P, nP, n_sel, words, out, lane);
}

__device__ __forceinline__ void pick_any(const int32_t* sc, int P, int nP, int n_sel, int words,
                                         uint64_t* __restrict__ out, int lane) {
  if (P <= 128) pick_few(sc, P, nP, n_sel, words, out, lane);
  else if (P <= 512) pick_row<8>(sc, P, nP, n_sel, words, out, lane);
  else if (P <= 2048) pick_row<32>(sc, P, nP, n_sel, words, out, lane);
  else pick_row_long(sc, P, nP, n_sel, words, out, lane);
}

__global__ __launch_bounds__(256) void k_page_pick(SelectArgs a) {
  touch_kernargs<sizeof(SelectArgs)>();
  const PageTile tl = a.tiles[blockIdx.x];
  const int r = __builtin_amdgcn_readfirstlane((int)blockIdx.z * 4 + ((int)threadIdx.x >> 6));
  if (r >= (tl.n_full & 63)) return;  // wave-uniform
  const int row = tl.row + r;
  pick_any(a.scores + ((size_t)blockIdx.y * a.max_rows + row) * a.ld, tl.n_full >> 6, (tl.keys + 63) / 64,
           a.n_sel, a.words, a.sel + ((size_t)row * a.H + blockIdx.y) * a.words, threadIdx.x & 63);
}

static int select_ld(const nmdlm_pages& pg) { return (pg.max_pages + 15) / 16 * 16; }

// Scores and choice in one kernel, for a tile of 16 rows and a head: the scores
// of at most kSelectPages pages meet in LDS; a wave per row.
constexpr int kSelectWaves = 8;
constexpr int kSelectPages = 128;
static_assert(kSelectPages <= 128, "pick_few");
template <int DHW>
__global__ __launch_bounds__(64 * kSelectWaves) void k_page_select(SelectArgs a) {
  touch_kernargs<sizeof(SelectArgs)>();
  __shared__ uint64_t sQ[NMDLM_MAX_T * 16 * DHW];
  extern __shared__ v4i sStage[];  // of the waves, then the scores [16][ld]
  int32_t* sScores = reinterpret_cast<int32_t*>(sStage + kSelectWaves * 16 * score_ld(a.T * DHW));
  const PageTile tl = a.tiles[blockIdx.x];
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, h = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int nr = tl.n_full & 63, P = tl.n_full >> 6;
  if (nr == 0) return;  // uniform
  int id = score_id(a, tl, wave * 16, lane);
  stage_queries<DHW, 16>(a, tl, h, sQ);
  __syncthreads();
  for (int p0 = wave * 16; p0 < P; p0 += kSelectWaves * 16) {
    v4i s[1];
    const int next = score_id(a, tl, p0 + kSelectWaves * 16, lane);
    score_pages<DHW, 1>(a, id, h, lane, sQ, sStage + wave * 16 * score_ld(a.T * DHW), s);
    id = next;
#pragma unroll
    for (int e = 0; e < 4; ++e) sScores[(4 * g + e) * a.ld + p0 + c] = s[0][e];
  }
  __syncthreads();
  for (int r = wave; r < nr; r += kSelectWaves) {
    const size_t at = (size_t)(tl.row + r) * a.H + h;
    pick_few(sScores + r * a.ld, P, (tl.keys + 63) / 64, a.n_sel, a.words, a.sel + at * a.words, lane);
  }
}

// One kernel where the table is narrow and its workgroups, which choose after
// they score, fill the chip: requests of 16 rows, 93 context pages, 16 heads, T = 4,
// 32 of them 10.1 us against 13.6 in two kernels, 16 of them 9.2 against 8.9, one 6.8
// in both; 256 with 125 pages 68 against 97.
bool select_fused(const nmdlm_pages& pg, int H) {
  return pg.max_pages <= kSelectPages && std::max(pg.max_rows / 16, pg.n_seq) * H >= 256;
}

// Heads that are scored before their pages are chosen: all, or an even share of
// them whose scores take at most this many bytes (one head's take what they need).
// 8192 rows, 16 heads, 2046 pages, T = 4, 1 GiB of scores: 1108 us at once, 1128 in
// four shares; 4096 rows 560 at once, 567 in two.
constexpr size_t kScoreBytes = (size_t)1 << 30;
static int select_heads(const nmdlm_pages& pg, int H) {
  const size_t head = (size_t)pg.max_rows * select_ld(pg) * sizeof(int32_t);
  const int fit = (int)std::min<size_t>(H, std::max<size_t>(kScoreBytes / head, 1));
  const int groups = (H + fit - 1) / fit;
  return (H + groups - 1) / groups;
}

size_t page_select_ws(const nmdlm_pages& pg, int H) {
  if (select_fused(pg, H)) return 0;
  return align_up((size_t)pg.max_rows * select_heads(pg, H) * select_ld(pg) * sizeof(int32_t), 256);
}

constexpr size_t kSelectPlainLds = 57344;  // dynamic LDS that needs no attribute beside the static

template <int DHW>
static nmdlm_status launch_select(const nmdlm_pages& pg, const uint64_t* q, int T, int H,
                                  const uint8_t* counts, int n_sel, uint64_t* sel, void* ws,
                                  hipStream_t st) {
  PageIndex ix;
  page_index_layout(pg.n_seq, pg.max_rows, pg.index, &ix);
  SelectArgs a{ix.t16, pg.table, q, counts, sel, static_cast<int32_t*>(ws), pg.max_pages, pg.pool,
               pg.max_rows, (pg.max_pages + 63) / 64, T, H, n_sel, select_ld(pg)};
  const size_t stage = 16 * score_ld(T * DHW) * sizeof(v4i);  // of a wave
  if (select_fused(pg, H)) {
    a.ld += 1;  // a row's bank past the row before's
    const size_t lds = kSelectWaves * stage + (size_t)a.ld * 16 * sizeof(int32_t);
    if (lds > kSelectPlainLds &&
        hipFuncSetAttribute(reinterpret_cast<const void*>(&k_page_select<DHW>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
      return NMDLM_ERR_HIP;
    hipLaunchKernelGGL(k_page_select<DHW>, dim3(ix.n16, H), dim3(64 * kSelectWaves), lds, st, a);
    return hip_status();
  }
  a.tiles = ix.t32;
  const int heads = select_heads(pg, H);
  for (int h0 = 0; h0 < H; h0 += heads) {
    const int n = std::min(heads, H - h0);
    // the kernels count heads from the launch's first
    a.q = q + (size_t)h0 * DHW;
    a.counts = counts + (size_t)h0 * T * 64 * DHW;
    a.sel = sel + (size_t)h0 * a.words;
    hipLaunchKernelGGL(k_page_scores<DHW>, dim3(ix.n32, n, (pg.max_pages + 63) / 64), dim3(256), 4 * stage, st, a);
    nmdlm_status rc = hip_status();
    if (rc != NMDLM_OK) return rc;
    hipLaunchKernelGGL(k_page_pick, dim3(ix.n32, n, 8), dim3(256), 0, st, a);
    if ((rc = hip_status()) != NMDLM_OK) return rc;
  }
  return NMDLM_OK;
}

nmdlm_status launch_page_select(const nmdlm_pages& pg, const uint64_t* q, int T, int H, int dh,
                                const uint8_t* counts, int n_sel, uint64_t* sel, void* ws,
                                hipStream_t st) {
  return dh == 64 ? launch_select<1>(pg, q, T, H, counts, n_sel, sel, ws, st)
                  : launch_select<2>(pg, q, T, H, counts, n_sel, sel, ws, st);
}

}  // namespace nmdlm
