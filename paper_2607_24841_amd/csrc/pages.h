// Work lists of a page plan (the `index` of nmdlm_pages) and the requests of
// the paged calls.
#pragma once

#include "common.h"

namespace nmdlm {

// What a plan knows of a request once its lengths are checked.
struct PageReq {
  int32_t first;  // its first page among those taken from the ring, or -1: refused
  int32_t held;   // pages it held before the call
  int32_t ctx, rows;
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

// The tiles of request s start at entry cu_rows[s]/TS + s: its ceil(rows/TS)
// tiles fit before those of s + 1, without a prefix sum of their own.  Runs
// likewise from cu_rows[s]/64 + 2s (rows of r positions lie in at most r/64 + 2
// pages).  Entries between are marked.
struct PageIndex {
  int32_t* head;   // [4]: ring's first free page and their number before the
                   // call, pages given back
  PageReq* req;    // [n_seq]
  int32_t* back;   // [n_seq]: pages given back before request s
  PageTile* t16;   // [n16]
  PageTile* t32;   // [n32]
  PageRun* runs;   // [n_runs]
  int n16, n32, n_runs;
};

inline size_t page_index_layout(int n_seq, int max_rows, void* base, PageIndex* ix) {
  Carver cv{static_cast<char*>(base), 0, (size_t)-1, true};
  ix->n16 = max_rows / 16 + n_seq;
  ix->n32 = max_rows / 32 + n_seq;
  ix->n_runs = max_rows / 64 + 2 * n_seq;
  // Carver aligns offsets to 256 bytes of the base
  ix->head = cv.take<int32_t>(4);
  ix->req = cv.take<PageReq>(n_seq);
  ix->back = cv.take<int32_t>(n_seq);
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

nmdlm_status launch_page_plan(const nmdlm_pages& pg, const int32_t* ctx, const int32_t* rows,
                              int32_t* status, hipStream_t st);
nmdlm_status launch_page_store(const nmdlm_pages& pg, const uint64_t* k, const uint64_t* v, int T, int H,
                               int dh, uint64_t* k_pages, uint64_t* v_pages, uint8_t* counts,
                               hipStream_t st);
size_t page_select_ws(const nmdlm_pages& pg, int H);
nmdlm_status launch_page_select(const nmdlm_pages& pg, const uint64_t* q, int T, int H, int dh,
                                const uint8_t* counts, int n_sel, uint64_t* sel, void* ws,
                                hipStream_t st);
size_t paged_attn_ws(const nmdlm_pages& pg, int T, int H, int dh);
nmdlm_status launch_paged_attn(const nmdlm_pages& pg, const PagedAttnCall& c, hipStream_t st);

}  // namespace nmdlm
