// Work lists of a page plan (the `index` of nmdlm_pages) and the requests of
// the paged calls.
#pragma once

#include <algorithm>

#include "common.h"

namespace nmdlm {

// Over a wave, without LDS: within rows of 16 lanes, then across them.
__device__ __forceinline__ int row_scan(int x) {  // inclusive sums of a row of 16 lanes
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  return x;
}
__device__ __forceinline__ int wave_scan(int x) {
  x = row_scan(x);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31
  return x;
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }
__device__ __forceinline__ int wave_max(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x111, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x142, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x143, 0xf, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}
// of m, the bits below this lane
__device__ __forceinline__ int bits_before(uint64_t m) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

// What a plan knows of a request once its lengths are checked.
struct PageReq {
  int32_t first;  // its first page among those taken from the ring, or -1: refused
  int32_t held;   // pages it held before the call
  int32_t ctx, rows;
  int32_t row;            // first packed row
  int32_t t16, t32, run;  // first entries in the lists
};
// Up to TS rows of one request, for a workgroup that takes TS queries; no rows:
// no such tile (an index that is all zeros holds none).
struct PageTile {
  int32_t s, row;    // request, first packed row
  int32_t n_full;    // rows | full context pages << 6
  int32_t keys;      // ctx + new rows
};
// Consecutive rows of one page; page < 0 or n = 0: no such run.
struct PageRun {
  int32_t page, off, row, n;
};

// The lists are dense: entries past the last are cleared, so that workgroups
// without work are a grid's last (spread among the others they kept CUs idle
// that had been given fewer of the working ones).
struct PageIndex {
  int32_t* head;   // [8]: the ring's first free page and their number before the
                   // call, pages given back, tiles of 16 and 32 rows, runs
  PageReq* req;    // [n_seq]
  int32_t* back;   // [n_seq]: pages given back before request s
  PageTile* t1;    // [max_rows]: entry m is row m
  PageTile* t16;   // [n16]
  PageTile* t32;   // [n32]
  PageRun* runs;   // [n_runs]
  int n16, n32, n_runs;  // entries there is room for
};

// a request of r rows has at most r/16 + 1 tiles of 16, and its rows lie in at
// most r/64 + 2 pages
inline size_t page_index_layout(int n_seq, int max_rows, void* base, PageIndex* ix) {
  Carver cv{static_cast<char*>(base), 0, (size_t)-1, true};
  const int live = std::min(n_seq, max_rows);  // requests with rows
  ix->n16 = max_rows / 16 + live;
  ix->n32 = max_rows / 32 + live;
  ix->n_runs = max_rows / 64 + 2 * live;
  // Carver aligns offsets to 256 bytes of the base
  ix->head = cv.take<int32_t>(8);
  ix->req = cv.take<PageReq>(n_seq);
  ix->back = cv.take<int32_t>(n_seq);
  ix->t1 = cv.take<PageTile>(max_rows);
  ix->t16 = cv.take<PageTile>(ix->n16);
  ix->t32 = cv.take<PageTile>(ix->n32);
  ix->runs = cv.take<PageRun>(ix->n_runs);
  return align_up(cv.off, 256);
}

struct PagedAttnCall {
  const uint64_t* q;
  const uint64_t* k_pages;
  const uint64_t* v_pages;
  int T, H, dh;
  const uint8_t* lut;
  const uint64_t* sel;  // or null
  int32_t* a_out;       // or null
  int32_t theta;
  uint64_t* s_out;      // or null
  uint64_t* u_out;      // or null: per-row union over t
  void* ws;
};

// A block step over pages: each layer's k_cache / vt_cache are its pools.
struct PagedStep {
  const nmdlm_pages* pages;
  uint8_t* const* key_counts;  // host array [n_layers]
  int n_sel;                   // selected context pages, or below 0: all
};

nmdlm_status launch_page_plan(const nmdlm_pages& pg, const int32_t* ctx, const int32_t* rows,
                              int32_t* status, hipStream_t st);
nmdlm_status launch_page_store(const nmdlm_pages& pg, const uint64_t* k, const uint64_t* v, int T, int H,
                               int dh, uint64_t* k_pages, uint64_t* v_pages, uint8_t* counts,
                               hipStream_t st);
bool select_fused(const nmdlm_pages& pg, int H);  // scores and choice in one kernel
size_t page_select_ws(const nmdlm_pages& pg, int H);
nmdlm_status launch_page_select(const nmdlm_pages& pg, const uint64_t* q, int T, int H, int dh,
                                const uint8_t* counts, int n_sel, uint64_t* sel, void* ws,
                                hipStream_t st);
// The row kernel or tiles of 16 * groups rows, waves a timestep, most splits.
struct PagedRoute {
  bool token;
  int groups, parts, splits;
};
PagedRoute paged_route(const nmdlm_pages& pg, int T, int H);
size_t paged_attn_ws(const nmdlm_pages& pg, int T, int H, int dh);
nmdlm_status launch_paged_attn(const nmdlm_pages& pg, const PagedAttnCall& c, hipStream_t st);

}  // namespace nmdlm
