/*
 * libnmdlm — the block-denoising step of a neuromorphic masked diffusion
 * language model (N-MDLM), for AMD Instinct MI355X (gfx950).
 *
 * Plain C ABI: device pointers, sizes and a HIP stream (passed as void*,
 * NULL = the default stream).  No call allocates or frees memory; scratch
 * memory is a caller-provided workspace whose size is given by the
 * *_workspace_size functions.  Every call validates its arguments on the
 * host first and, on error, returns a status without enqueueing any work.
 * Calls are asynchronous with respect to the host: outputs (and statistics)
 * are valid once the stream has reached them.  Apart from the static scratch
 * of nmdlm_qbsm_noalloc, the library keeps no global mutable state; two calls
 * may run concurrently on different streams when their workspaces and
 * outputs do not overlap.
 *
 * Spike tensors are {0,1}^{T x M x K} packed little-endian into uint64
 * words: tensor [T][M][ceil(K/64)], bit j of word w is channel 64*w + j.
 * Padding bits must be zero on input and are written as zero on output.
 *
 * Weight matrices are int8 [K][ldw] row-major: row k holds the weights that
 * leave input neuron k (its fan-out), so a product can skip whole rows.
 * ldw is a multiple of 16 and >= N; bytes [N, ldw) of a row may be read and
 * are ignored.  K * ldw must be below 2^31.
 */
#ifndef NMDLM_H
#define NMDLM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define NMDLM_ABI_VERSION 5

typedef enum nmdlm_status {
  NMDLM_OK = 0,
  NMDLM_ERR_INVALID_ARG = 1,  /* null pointer, size <= 0, threshold <= 0, ... */
  NMDLM_ERR_UNSUPPORTED = 2,  /* valid but outside the supported envelope     */
  NMDLM_ERR_WORKSPACE = 3,    /* workspace missing or smaller than required   */
  NMDLM_ERR_HIP = 4           /* a HIP launch reported an error               */
} nmdlm_status;

/* flags (bitwise OR) */
#define NMDLM_FORCE_DENSE 0x1u   /* read every weight row: the un-skipped product */
#define NMDLM_NO_HEAD     0x2u   /* block step without head/confidence/unmask    */
#define NMDLM_ATTN_FUSED  0x4u   /* block step: attention and the IF of its output
                                    in one kernel (a workgroup per head and 16
                                    queries, all timesteps); without it the
                                    grid and the context decide between one
                                    kernel and two.  Results do not depend on
                                    it.                                         */
#define NMDLM_ALL_PAGES   0x8u   /* block step over pages: no selection (n_sel
                                    below 0), whose room the workspace then
                                    lacks                                       */
/* bits 8..15 of the flags of nmdlm_qbsm: force the number of K splits
 * (0 = automatic).  Results do not depend on it. */
#define NMDLM_SPLIT_SHIFT 8u
/* bits 16..19: force rows per tile group (0 = automatic; 1,2,4,8 = 16..128
 * rows).  Results do not depend on it. */
#define NMDLM_ROWTILE_SHIFT 16u
/* bits 20..22: product kernel (0 = automatic; 1 = separate pass building the
 * active-row list; 2 = single kernel with an in-kernel list; 3 = single
 * kernel over 64-channel words, loading only active rows into registers;
 * 4 = as 3, gathering the active rows straight into LDS; 5 = as 3 with a
 * scalar gather-accumulate product in place of MFMA: per spike of a row,
 * the active weight row's columns are loaded and added; 6 = as 3 over the
 * blocked copy of the weights, nmdlm_qbsm_blocked only; 7 = as 6 with wide
 * tiles where the row tile is 64 rows: a workgroup takes four 64-column
 * tiles, each wave one of them over all of K).  Results do not depend on
 * it. */
#define NMDLM_PATH_SHIFT 20u
#define NMDLM_NO_FUSE (1u << NMDLM_PATH_SHIFT)

/* Supported envelope (NMDLM_ERR_UNSUPPORTED beyond it). */
#define NMDLM_MAX_TERNARY_K 16384
#define NMDLM_MAX_T 8
#define NMDLM_MAX_K 65536
#define NMDLM_MAX_HEAD_M 4096   /* block tokens of a step that runs the head */
#define NMDLM_MAX_KEYS 8388608  /* attention keys C+M per sequence (2^23): the
                                   sum of the table weights over the keys,
                                   at most 255 per key, stays below 2^31   */

/* bits of the device status word of a block step (nmdlm_step_io.status) */
#define NMDLM_STATUS_TOKEN_CLAMPED 0x1  /* a token id outside [0, V] was read as
                                           the nearest of 0 and V (the mask id) */
/* bits of the device status word of nmdlm_page_plan */
#define NMDLM_STATUS_PAGES_SHORT 0x2    /* the ring had too few pages for a request */
#define NMDLM_STATUS_BAD_REQUEST 0x4    /* lengths outside the bounds of the plan   */

/*
 * Statistics of one spike product, written by the device (int64 so the
 * host can sum them).  They count the block's union, whichever kernel ran:
 * weight_bytes = k_active * n is the per-block load of Eq. (13), the bytes of
 * the active rows.  The kernels over row-major weights read those; the lean,
 * tall and wide products over a blocked copy read more, up to every row (see
 * nmdlm_qbsm_blocked), and NMDLM_FORCE_DENSE counts every row.
 */
typedef struct nmdlm_qbsm_stats {
  int64_t k_total;       /* K                                             */
  int64_t k_active;      /* input neurons that spike at least once in the
                            block (active rows of W)                      */
  int64_t n;             /* N                                             */
  int64_t weight_bytes;  /* k_active * n                                  */
} nmdlm_qbsm_stats;

/* ------------------------------------------------------------------------
 * nmdlm_qbsm — quantised-weight x binary-spike product with row skipping
 *
 * Sec. IV-A: the linear operation over the B*T rows of a block,
 *     I[t,m,n] = bias[n] + sum_k S[t,m,k] * W[k,n],
 * where, by assumption (ii), row k of W is needed only if input neuron k
 * spikes at least once among all T*M rows, and only then read here (a row
 * block of the product reads the rows active in it).  The result is identical to the
 * dense product (integer arithmetic, no overflow for K*127 + |bias| < 2^31).
 *
 * Optional fused integrate-and-fire epilogue (Sec. II-B, Eqs. (3)-(4),
 * integrate-then-fire with soft reset, membrane starting at 0):
 *     V = 0; for t: V += I[t]; s[t] = (V >= theta); V -= s[t]*theta.
 *
 *   s_in      device, spikes [T][M][ceil(K/64)]
 *   T, M, K   1 <= T <= 8, M >= 1, T*M <= 2^19, 1 <= K <= 65536
 *   W, N, ldw device int8 [K][ldw] (see above), N >= 1
 *   bias      device int32 [N] or NULL (zero)
 *   cur_out   device int32 [T][M][N] or NULL: the currents I
 *   theta     threshold (> 0) used when s_out is given; ignored otherwise
 *   theta_vec device int32 [N] per-neuron thresholds (> 0) or NULL (use theta)
 *   s_out     device spikes [T][M][ceil(N/64)] or NULL; at least one of
 *             cur_out / s_out must be given
 *   stats     device, one nmdlm_qbsm_stats, or NULL
 *   flags     NMDLM_FORCE_DENSE, split/row-tile overrides
 *   ws        device workspace of ws_bytes >= nmdlm_qbsm_workspace_size();
 *             zero-filled before its first use; every call leaves its
 *             counter region zero again
 *   stream    hipStream_t or NULL
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_qbsm(const uint64_t* s_in, int T, int M, int K,
                        const int8_t* W, int N, int64_t ldw,
                        const int32_t* bias, int32_t* cur_out,
                        int32_t theta, const int32_t* theta_vec,
                        uint64_t* s_out, nmdlm_qbsm_stats* stats,
                        unsigned flags, void* ws, size_t ws_bytes, void* stream);

size_t nmdlm_qbsm_workspace_size(int T, int M, int K, int N);

/* ------------------------------------------------------------------------
 * Blocked weights — a second layout of a weight matrix for products over
 * many rows (prefills, steps over many sequences), where the block union is
 * dense and the products are plain int8 contractions.
 *
 * Sec. IV-A (Eqs. (12)-(13)): the row-load rule reads row k of W only if
 * input neuron k spikes in the block.  Over the blocked copy whole 64-row
 * words are read: rows that do not spike meet zero inputs, so the result is
 * unchanged, and at dense unions the bytes are those of the row-major path.
 * The copy's bytes sit in MFMA operand order, so a 64-row word of a 64-column
 * tile is four 16-byte loads per lane with no byte transposes.
 *
 * Layout: for word w (rows 64w..64w+63) and column tile x (columns
 * 64x..64x+63), 4096 bytes at offset (w * ceil(N/64) + x) * 4096; within
 * them, operand v (0..3), lane l = 16g + c (0..63), byte j (0..15) at
 * v*1024 + l*16 + j holds W[64w + 16g + j][64x + 4c + v], zero past K or N.
 *
 * nmdlm_weight_blocked_bytes: size of the copy (0 for invalid sizes).
 * nmdlm_weight_block: writes the copy Wb (device, 16-byte aligned, of
 *   nmdlm_weight_blocked_bytes) from W (as for nmdlm_qbsm); asynchronous on
 *   the stream.  The copy must be rebuilt whenever W changes.
 * nmdlm_qbsm_blocked: nmdlm_qbsm (same arguments, results and errors) with
 *   the blocked copy Wb of W also given.  Unforced, the sizes and options
 *   choose among
 *   - lean: products with neurons or a head, without bias, per-neuron
 *     thresholds or currents, of at least 64 rows T*M or a matrix of at most
 *     16 MB (less where K is below 512 or long, by measured lines).  Every
 *     word of the copy is read, also one without an active row: the loads do
 *     not wait for the union;
 *   - tall: such products, or currents alone, of many rows (at least 112 to
 *     160 tiles of 128 rows x 256 columns, by K).  Every word is read;
 *   - wide: others of 64-row tiles over at least 1536 output tiles of 64 x
 *     64 (and path 7 in the flags): four column tiles per workgroup; every
 *     word with an active row of the row block is read;
 *   - the others read a word without an active row not at all, and each wave
 *     takes the words from the copy when their union is dense: on average at
 *     least NMDLM_BLOCKED_MIN_ROWS active rows of 64 per active word, counted
 *     over the row blocks of the product that read the same words (the whole
 *     words then cost at most twice the active rows' bytes from HBM); else
 *     the row-major rows of W.  Path 6 in the flags: always from the copy.
 *   Results and statistics do not depend on which is used.
 *   NMDLM_ERR_UNSUPPORTED when the copy would exceed 2^31 bytes.
 * ------------------------------------------------------------------------ */
#define NMDLM_BLOCKED_MIN_ROWS 32
size_t nmdlm_weight_blocked_bytes(int K, int N);
nmdlm_status nmdlm_weight_block(const int8_t* W, int K, int N, int64_t ldw,
                                int8_t* Wb, void* stream);
nmdlm_status nmdlm_qbsm_blocked(const uint64_t* s_in, int T, int M, int K,
                                const int8_t* W, const int8_t* Wb, int N,
                                int64_t ldw, const int32_t* bias,
                                int32_t* cur_out, int32_t theta,
                                const int32_t* theta_vec, uint64_t* s_out,
                                nmdlm_qbsm_stats* stats, unsigned flags,
                                void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * nmdlm_qbsm_noalloc — nmdlm_qbsm without a workspace argument, for callers
 * that cannot allocate device memory (code under stream capture, tight
 * serving loops, harnesses that forbid allocation).  The call allocates
 * nothing: its scratch is a static device array of
 * NMDLM_NOALLOC_SCRATCH_BYTES that each GPU holds from the library's first
 * call on it until the process ends (that first call also clears it with a
 * fill kernel on the stream).  Every call on one GPU shares that GPU's array:
 * calls that overlap on one GPU (other streams, other host threads) race
 * and must not be issued.  Sequential calls on a stream are safe: every call
 * leaves the array's counter region at zero, as nmdlm_qbsm does.
 *
 * Arguments, results and errors are those of nmdlm_qbsm (same computation,
 * same kernels), less ws and ws_bytes; a product whose
 * nmdlm_qbsm_workspace_size() exceeds NMDLM_NOALLOC_SCRATCH_BYTES returns
 * NMDLM_ERR_UNSUPPORTED before any work is enqueued.
 * ------------------------------------------------------------------------ */
#define NMDLM_NOALLOC_SCRATCH_BYTES 16777216  /* 16 MiB per GPU */
nmdlm_status nmdlm_qbsm_noalloc(const uint64_t* s_in, int T, int M, int K,
                                const int8_t* W, int N, int64_t ldw,
                                const int32_t* bias, int32_t* cur_out,
                                int32_t theta, const int32_t* theta_vec,
                                uint64_t* s_out, nmdlm_qbsm_stats* stats,
                                unsigned flags, void* stream);

/* ------------------------------------------------------------------------
 * nmdlm_ternary_encode — adaptive quantisation and ternary bitwise coding of
 * integer activations (Sec. III-B, Eqs. (7)-(8)), per token m:
 *     S = sum_i |a_i|;  V_th = S / (D K)   (mean(|a|) / K, kept exact)
 *     q_i = round(a_i / V_th) = round(a_i D K / S), halves away from zero,
 *           0 when S = 0, |q_i| capped at 2^T - 1;
 *     s_{i,t} = sign(q_i) * bit t-1 of |q_i|,  t = 1..T  (q = sum 2^(t-1) s_t)
 *
 *   a       device int32 [M][D] (a layer's integer output)
 *   K       quantisation levels per mean magnitude (>= 1; D*K < 2^20)
 *   T       bits = timesteps (1..NMDLM_MAX_T)
 *   s_pos   device spikes [T][M][ceil(D/64)]: bit set where s = +1
 *   s_neg   device spikes [T][M][ceil(D/64)]: bit set where s = -1
 *   s_sum   device int64 [M] or NULL: S per token (V_th = S / (D K))
 * Integer arithmetic throughout: the result does not depend on rounding.
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_ternary_encode(const int32_t* a, int M, int D, int K, int T,
                                  uint64_t* s_pos, uint64_t* s_neg, int64_t* s_sum,
                                  void* stream);

/* ------------------------------------------------------------------------
 * nmdlm_qbsm_ternary — the spiking product on ternary bitwise-coded spikes
 * and its reconstruction (Sec. III-B, Eqs. (10)-(11); row-load rule of
 * Sec. IV-A on either spike plane):
 *     I_t[m,n] = sum_k (s_pos - s_neg)[t,m,k] * W[k,n]      t = 1..T
 *     acc[m,n] = sum_t 2^(t-1) I_t[m,n]   (= sum_k q[m,k] W[k,n], exact)
 * A weight row k is read only if input k spikes (either sign) somewhere in
 * the block.  The layer output is V_th[m] * acc[m,n] (V_th from
 * nmdlm_ternary_encode); acc can feed nmdlm_ternary_encode of the next
 * layer directly, since the per-token scale cancels in Eq. (7).
 *
 *   s_pos, s_neg  device spikes [T][M][ceil(K/64)] (never both set)
 *   W, ldw, N     as nmdlm_qbsm; K <= NMDLM_MAX_TERNARY_K and
 *                 (2^T - 1) * K * 127 < 2^31 (else NMDLM_ERR_UNSUPPORTED)
 *   acc_out       device int32 [M][N]
 *   stats         as nmdlm_qbsm (active rows of the union of both planes)
 *   flags, ws     as nmdlm_qbsm (ws of nmdlm_qbsm_workspace_size(T, M, K, N))
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_qbsm_ternary(const uint64_t* s_pos, const uint64_t* s_neg, int T,
                                int M, int K, const int8_t* W, int N, int64_t ldw,
                                int32_t* acc_out, nmdlm_qbsm_stats* stats,
                                unsigned flags, void* ws, size_t ws_bytes,
                                void* stream);

/* ------------------------------------------------------------------------
 * nmdlm_qbsm_ternary_if — the spiking product on ternary bitwise-coded
 * spikes followed by the modified IF neuron of Sec. III-B (Eqs. (9)-(10)),
 * which turns the per-timestep currents back into ternary spike planes;
 * row-load rule of Sec. IV-A on either input plane.  Per token m and output
 * neuron n, with I_t = sum_k (s_pos - s_neg)[t,m,k] * W[k,n] and the
 * threshold Vth = thr_num[m] / thr_den:
 *     V = 0; for t = 1..T:
 *       V += 2^(t-1) I_t
 *       s_t = +1 if V >= 2^(t-1) Vth, -1 if V <= -2^(t-1) Vth, else 0
 *       V -= 2^(t-1) s_t Vth
 * so that Vth sum_t 2^(t-1) s_t = sum_t 2^(t-1) I_t - V (Eq. (11), the final
 * membrane being its error).  Readings: the 2^t of Eqs. (9)-(10) counts steps
 * from 0 (weight 2^(t-1) for step t = 1..T, as in Eq. (8)); the membrane
 * integrates before it fires, as for Eqs. (3)-(4); a token with
 * thr_num[m] = 0 (Vth = 0, an all-zero activation vector) emits no spike.
 * The paper's threshold is the input's quantisation step: pass s_sum of
 * nmdlm_ternary_encode as thr_num and D*K as thr_den.  All arithmetic is
 * integer (the membrane is kept times thr_den in 64 bits): exact.
 *
 *   s_pos, s_neg  device spikes [T][M][ceil(K/64)] (never both set)
 *   W, ldw, N     as nmdlm_qbsm; K <= NMDLM_MAX_TERNARY_K
 *   thr_num       device int64 [M], each in [0, 2^55) (larger values give
 *                 undefined spikes)
 *   thr_den       1 <= thr_den <= NMDLM_MAX_THR_DEN (else INVALID_ARG /
 *                 UNSUPPORTED)
 *   out_pos       device spikes [T][M][ceil(N/64)]: bit set where s_t = +1
 *   out_neg       device spikes [T][M][ceil(N/64)]: bit set where s_t = -1
 *                 (padding bits written as zero; the planes can feed the next
 *                 nmdlm_qbsm_ternary_if directly)
 *   v_out         device int64 [M][N] or NULL: thr_den * final membrane
 *   stats, flags, ws   as nmdlm_qbsm_ternary
 * ------------------------------------------------------------------------ */
#define NMDLM_MAX_THR_DEN 16777216
nmdlm_status nmdlm_qbsm_ternary_if(const uint64_t* s_pos, const uint64_t* s_neg, int T,
                                   int M, int K, const int8_t* W, int N, int64_t ldw,
                                   const int64_t* thr_num, int64_t thr_den,
                                   uint64_t* out_pos, uint64_t* out_neg, int64_t* v_out,
                                   nmdlm_qbsm_stats* stats, unsigned flags, void* ws,
                                   size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * nmdlm_if_neuron — integrate-and-fire with soft reset (Sec. II-B,
 * Eqs. (3)-(4)), integrate-then-fire order, equality fires, no lower clamp:
 *     V = v_in (or 0); for t: V += cur[t] + theta*resid[t];
 *                             s[t] = (V >= theta); V -= s[t]*theta.
 *
 *   cur       device int32 [T][M][N]
 *   theta     threshold (> 0); theta_vec device int32 [N] or NULL
 *   resid     device spikes [T][M][ceil(N/64)] or NULL: membrane shortcut
 *   v_inout   device int32 [M][N] or NULL: initial membrane in, final out
 *   s_out     device spikes [T][M][ceil(N/64)]
 * Limits: T <= 8192 and M * ceil(N/64) <= 2^26, else NMDLM_ERR_UNSUPPORTED.
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_if_neuron(const int32_t* cur, int T, int M, int N,
                             int32_t theta, const int32_t* theta_vec,
                             const uint64_t* resid, int32_t* v_inout,
                             uint64_t* s_out, void* stream);

/* ------------------------------------------------------------------------
 * nmdlm_qnl_lut — 8-bit-in / 8-bit-out table non-linearity.
 * The paper names this operation only in its list of acronyms (QNL: a
 * quantised non-linearity implemented as a look-up table), as one of the
 * operations of the neuromorphic layers of Fig. 1; it gives no formula.
 * This library's reading, also used by the block step on the FFN up
 * current:
 *   NMDLM_QNL_S8: index = byte of clamp(floor(x / 2^shift), -128, 127)
 *   NMDLM_QNL_U8: index = clamp(x, 0, 255)            (shift ignored)
 *   y[i] = lut[index]  (the raw table byte; read it as int8 in S8 mode)
 *
 *   x    device int32 [n];  lut device uint8 [256];  y device uint8 [n]
 *   0 <= shift <= 31; n = 0 enqueues nothing
 * Errors: NMDLM_ERR_INVALID_ARG for n < 0, a missing pointer, a shift out of
 * range or an unknown mode (nothing is enqueued).
 * ------------------------------------------------------------------------ */
#define NMDLM_QNL_S8 0
#define NMDLM_QNL_U8 1
nmdlm_status nmdlm_qnl_lut(const int32_t* x, int64_t n, int shift, int mode,
                           const uint8_t* lut, uint8_t* y, void* stream);

/* ------------------------------------------------------------------------
 * nmdlm_bbm_attn — attention on spike operands.  The paper names the
 * operations involved only in its list of acronyms: binary-binary
 * multiplication (BBM, here the query-key product of two spike vectors),
 * quantised dynamic multiplication (QDM, the table weights times the value
 * spikes), a look-up-table non-linearity (QNL) and fixed-point arithmetic
 * (FixP, the integer normalisation); Fig. 1 places attention in every
 * neuromorphic layer.  The formula below is this library's reading.  For
 * every timestep t, head h, block query i < M and key j < C+M:
 *     s = popcount(Q[t,i,head h] AND K[t,j,head h])       in [0, dh]
 *     p = lut_att[s]                                       (uint8)
 *     a[t,i,c] = floor(256 * sum_j p * V[t,j,c] / sum_j p)   (0 if sum_j p = 0)
 * then optionally A = IF(a, theta_a) over t.  The block's own keys/values
 * must already be in rows [C, C+M) of the caches.
 *
 *   q         device spikes [T][M][d/64], d = H*dh
 *   k_cache   device spikes [T][cache_cap][d/64]  (token-major)
 *   vt_cache  device spikes, word-major: [T][cache_cap/64][d]; bit j%64 of
 *             word (t, j/64, c) is V[t,j,c] (the 64 positions of one word
 *             for every channel lie side by side)
 *   cache_cap multiple of 64, >= C+M
 *   dh        64 or 128 (else NMDLM_ERR_UNSUPPORTED): scores stay within
 *             the 256-entry table
 *   limits    T*M <= 2^19, d <= NMDLM_MAX_K and C+M <= NMDLM_MAX_KEYS, else
 *             NMDLM_ERR_UNSUPPORTED
 *   lut_att   device uint8 [256]
 *   a_out     device int32 [T][M][d] or NULL
 *   theta_a   threshold (> 0) when s_out is given
 *   s_out     device spikes [T][M][d/64] or NULL (at least one output)
 *   ws        workspace of nmdlm_bbm_attn_workspace_size() bytes (used when
 *             a_out is NULL)
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_bbm_attn(const uint64_t* q, const uint64_t* k_cache,
                            const uint64_t* vt_cache, int64_t cache_cap,
                            int T, int M, int C, int H, int dh,
                            const uint8_t* lut_att, int32_t* a_out,
                            int32_t theta_a, uint64_t* s_out,
                            void* ws, size_t ws_bytes, void* stream);

size_t nmdlm_bbm_attn_workspace_size(int T, int M, int H, int dh);

/* ------------------------------------------------------------------------
 * nmdlm_block_step — one denoising step z_{s+1} = f_dec(z_s, h) of block
 * diffusion (Sec. III-A, Eq. (6)) through a stack of spiking layers, or a
 * context prefill (Eq. (5): the same stack over the context tokens with
 * C = 0 and NMDLM_NO_HEAD).
 *
 * Per layer (Fig. 1: IF neurons in every layer; the wiring below is this
 * library's reading, the paper gives no layer internals):
 *   Q,K,V = IF(QBSM(X, W_qkv))   (thresholds q, k, v; K,V -> cache rows [C,C+M))
 *   A     = IF(attn(Q, caches), theta_a)
 *   X1    = IF(QBSM(A, W_o), theta_o, residual X)
 *   H     = IF(lut_act[QBSM(X1, W_up) >> s_up], theta_up)
 *   Y     = IF(QBSM(H, W_dn), theta_dn, residual X1)
 * Head (unless NMDLM_NO_HEAD): acc[m,v] = sum_t sum_c Y[t,m,c] W_head[c,v],
 * logit = (float)acc * head_scale[v]; pred = argmax (ties: smallest id);
 * conf = 1 / sum_v exp(logit_v - logit_pred) (fp64); then the k_unmask
 * masked positions of highest confidence (ties: lower position) take their
 * predicted token (B/S tokens per step, Sec. III-A).
 *
 * Several sequences in one step (io->n_seq > 1): n_seq independent
 * sequences at the same block (same M, C, pos0) share every product, so a
 * weight row counts once when it is active for any of their n_seq*M tokens
 * (the row-load rule of Sec. IV over the batch); attention, the caches and
 * the unmasking stay per sequence.  Token-indexed buffers then hold the
 * sequences one after the other: tokens/masked/pred/conf [n_seq][M], spikes
 * [T][n_seq*M][d/64], logits [n_seq*M][V], unmasked_pos [n_seq][k_unmask];
 * the caches of sequence s start s*T*cache_cap*d/64 words into k_cache and
 * vt_cache (both hold model->max_seq sequences).  With n_seq > 1, M must be
 * a multiple of 16/T (integer division) and NMDLM_ATTN_FUSED is ignored.
 *
 * Token ids: the block input reads the token table at row tokens[m] for an
 * unmasked position and at row V (the mask token) for a masked one; ids are
 * expected in [0, V).  An id outside [0, V] is read as the nearest of 0 and V
 * (never out of bounds) and flags NMDLM_STATUS_TOKEN_CLAMPED in io->status.
 * Limits: C+M <= NMDLM_MAX_KEYS and cache_cap/64 <= 2^31-1, else
 * NMDLM_ERR_UNSUPPORTED.
 * ------------------------------------------------------------------------ */
typedef struct nmdlm_layer {
  const int8_t* w_qkv;   /* device [d][3d]: columns Q | K | V */
  const int8_t* w_o;     /* device [d][d]  */
  const int8_t* w_up;    /* device [d][F]  */
  const int8_t* w_dn;    /* device [F][d]  */
  int32_t theta_q, theta_k, theta_v, theta_a, theta_o, theta_up, theta_dn;
  int32_t s_up;          /* right shift before lut_act (0..31) */
  const uint8_t* lut_att;/* device [256] attention score table */
  const uint8_t* lut_act;/* device [256] activation table (int8 bytes) */
  uint64_t* k_cache;     /* device [T][cache_cap][d/64]      */
  uint64_t* vt_cache;    /* device [T][cache_cap/64][d]: bit j%64 of word
                            (t, j/64, c) is value channel c of position j */
  /* Blocked copies (nmdlm_weight_block, ldw = N) of the four weights, or
   * NULL.  With a copy, the products choose as nmdlm_qbsm_blocked does (of 64
   * rows T*M and more, most read every word of it).  Path 6 in the flags
   * (every word from the copies) requires every copy, and the head's when
   * the step runs the head (NMDLM_ERR_INVALID_ARG otherwise).  Results do
   * not depend on it. */
  const int8_t* w_qkv_b;
  const int8_t* w_o_b;
  const int8_t* w_up_b;
  const int8_t* w_dn_b;
} nmdlm_layer;

typedef struct nmdlm_model {
  int n_layers, d, H, F, V, T;
  int64_t cache_cap;          /* multiple of 64 */
  int max_pos;                /* rows of pos_ch */
  const nmdlm_layer* layers;  /* HOST array [n_layers] */
  const uint64_t* emb;        /* device [V+1][T][d/64]; row V = mask token */
  const int32_t* pos_ch;      /* device [max_pos][T]: channel of the single
                                 position spike ORed into the token spikes */
  const int8_t* w_head;       /* device [d][V] (NULL allowed with NO_HEAD) */
  const float* head_scale;    /* device [V]                                */
  int max_seq;                /* sequences the caches hold (0 counts as 1):
                                 k_cache [max_seq][T][cache_cap][d/64],
                                 vt_cache [max_seq][T][cache_cap/64][d]     */
  const int8_t* w_head_b;     /* blocked copy of w_head (ldw = V) or NULL   */
} nmdlm_model;

typedef struct nmdlm_step_io {
  int M;                   /* tokens in the block (or context, in prefill)   */
  int C;                   /* cache rows already holding context            */
  int pos0;                /* sequence position of the first block token    */
  unsigned flags;          /* NMDLM_NO_HEAD, NMDLM_FORCE_DENSE              */
  const uint64_t* x_in;    /* device [T][M][d/64] block input spikes, or NULL:
                              assemble from tokens/masked, emb and pos_ch   */
  int32_t* tokens;         /* device [M] in/out (may be NULL with x_in and
                              NO_HEAD)                                       */
  uint8_t* masked;         /* device [M] in/out, 1 = still masked           */
  int k_unmask;            /* tokens revealed by this step                  */
  uint64_t* y_out;         /* device [T][M][d/64] last layer spikes or NULL */
  float* logits;           /* device [M][V] or NULL (workspace is used)     */
  int32_t* pred;           /* device [M] or NULL                            */
  double* conf;            /* device [M] or NULL                            */
  int32_t* unmasked_pos;   /* device [k_unmask] or NULL: chosen positions in
                              selection order, -1 when fewer were masked    */
  nmdlm_qbsm_stats* stats; /* device [4*n_layers + 1] or NULL: per product
                              (QKV, O, up, down per layer, then the head)  */
  void** prof_events;      /* HOST array of hipEvent_t or NULL: when given,
                              events 2i and 2i+1 take the start and end
                              times of the main kernel of product i (same
                              order as stats), stamped by its dispatch;
                              NMDLM_ERR_UNSUPPORTED inside stream capture  */
  int n_prof_events;       /* length of prof_events                         */
  int n_seq;               /* sequences in the step, 1..max(1, max_seq) (0
                              counts as 1); M is per sequence              */
  int32_t* status;         /* device int32 or NULL: the step ORs in
                              NMDLM_STATUS_* bits (the caller clears it);
                              a token id outside [0, V] is read as the
                              nearest of 0 and V and sets
                              NMDLM_STATUS_TOKEN_CLAMPED                   */
} nmdlm_step_io;

nmdlm_status nmdlm_block_step(const nmdlm_model* model, nmdlm_step_io* io,
                              void* ws, size_t ws_bytes, void* stream);

/* Workspace of a step over M block tokens in all (n_seq * M for a step of
 * several sequences). */
size_t nmdlm_block_step_workspace_size(const nmdlm_model* model, int M,
                                       unsigned flags);

/* ------------------------------------------------------------------------
 * Paged caches — requests of different lengths that share one pool of pages.
 *
 * A page holds the keys and values of NMDLM_PAGE = 64 consecutive positions of
 * one request (one word of the value cache).  A layer's pool:
 *   k_pages    device [pool][H][T][64][dh/64] words, 16-byte aligned: bit c%64
 *              of word c/64 is key channel c of the head at that position
 *   v_pages    device [pool][H][T][dh] words, 16-byte aligned: bit j is value
 *              channel c of the page's position j
 *   key_counts device [pool][H][T][dh] bytes, 16-byte aligned: in how many of
 *              the page's keys channel c spikes (what nmdlm_page_select scores
 *              by)
 * The layers of a model share the page numbers: one plan serves all of them.
 *
 * A plan covers n_seq requests, each with `held` pages (logical page p, its
 * positions 64p .. 64p+63, is pool page table[s][p]) and, in one step, new
 * rows that follow its context.  Packed rows are the new rows of all
 * requests one after the other: spikes [T][max_rows][H*dh/64], rows
 * [cu_rows[s], cu_rows[s+1]) being request s's.  Rows past the last
 * request's are not read as queries, keys or values, and nothing is written
 * for them.  A page belongs to one request.  The calls after nmdlm_page_plan read
 * what it left on the device, so they follow it in stream order.
 *
 * The plan is device memory of the caller.  The table, held, ring and
 * ring_state arrays live from step to step; initially held = 0, ring = the page numbers 0 .. pool-1
 * in any order and ring_state = {0, pool}.  The others are outputs of
 * nmdlm_page_plan.  Page numbers outside the pool are never followed: keys of
 * such a page count as absent and rows of it are not stored.
 * ------------------------------------------------------------------------ */
#define NMDLM_PAGE 64
#define NMDLM_MAX_REQUESTS 16384
#define NMDLM_MAX_PLAN_ROWS 524288   /* 2^19 packed rows                        */
#define NMDLM_MAX_PAGES 131072       /* pages of a request: NMDLM_MAX_KEYS / 64 */
#define NMDLM_MAX_POOL 33554432      /* pages of a pool (2^25)                  */

typedef struct nmdlm_pages {
  int n_seq;            /* requests, 1 .. NMDLM_MAX_REQUESTS                    */
  int max_rows;         /* packed rows, 1 .. NMDLM_MAX_PLAN_ROWS                */
  int max_pages;        /* width of the table, 1 .. NMDLM_MAX_PAGES             */
  int pool;             /* pages of the pool, 1 .. NMDLM_MAX_POOL               */
  int32_t* table;       /* device [n_seq][max_pages]                            */
  int32_t* held;        /* device [n_seq]: pages that request s holds           */
  int32_t* ring;        /* device [pool]: free pages, from ring_state[0] on,
                           wrapping at pool                                     */
  int32_t* ring_state;  /* device [2]: index of the first free page, their number */
  int32_t* cu_rows;     /* device [n_seq + 1]: first packed row of each request */
  int64_t* slot;        /* device [max_rows]: 64 * page + position within it, or
                           -1 for a row that has no page                        */
  int32_t* pos;         /* device [max_rows]: position of the row in its request
                           (0 for a row without a request)                      */
  void* index;          /* device, 16-byte aligned: work lists of the calls below */
  size_t index_bytes;   /* >= nmdlm_page_index_bytes(n_seq, max_rows)           */
} nmdlm_pages;

size_t nmdlm_page_index_bytes(int n_seq, int max_rows);

/* ------------------------------------------------------------------------
 * nmdlm_page_plan — block tables, slots and work lists of a step from the
 * requests' lengths.  Request s holds ctx[s] positions and brings new_rows[s]:
 *   new_rows > 0   rows for positions ctx .. ctx+new_rows-1.  The pages up to
 *                  ceil((ctx+new_rows)/64) that it does not hold are taken from
 *                  the ring, in the order of the requests
 *   new_rows = 0   idle: keeps its pages
 *   new_rows = -1  ended: its pages go behind the ring's last, held becomes 0
 *                  (free to be taken from the next call on)
 * A call with the same lengths again takes no further page, so the plan can
 * be made once a block and used by all of its steps.
 *
 * From the first request on whose pages the ring does not have, every
 * request that needs a page is refused (NMDLM_STATUS_PAGES_SHORT); one with
 * ctx < 0 or ctx > 64 held, new_rows < -1, ctx+new_rows > 64 max_pages, held
 * outside [0, max_pages] or rows past max_rows is refused as well
 * (NMDLM_STATUS_BAD_REQUEST).  A refused request takes no page; its rows (none
 * when new_rows > max_rows) have slot -1 and the calls below skip them.
 *
 *   ctx, new_rows  device int32 [n_seq]
 *   status         device int32 or NULL: bits are ORed in
 * Errors: NMDLM_ERR_INVALID_ARG for a missing or misaligned pointer or a size
 * below 1, NMDLM_ERR_UNSUPPORTED beyond the limits above,
 * NMDLM_ERR_WORKSPACE for an index that is too small.
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_page_plan(const nmdlm_pages* pages, const int32_t* ctx,
                             const int32_t* new_rows, int32_t* status, void* stream);

/* ------------------------------------------------------------------------
 * nmdlm_page_store — keys and values of the packed rows into their pages,
 * after nmdlm_page_plan.  key_counts of a page that takes rows are counted
 * again over its positions up to the last stored one (keys past it, of an
 * earlier holder of the page, are not counted).  Bits of other positions keep
 * their values.
 *
 *   k, v        device spikes [T][max_rows][H*dh/64], 16-byte aligned
 *   k_pages, v_pages, key_counts   see above
 *   T, H, dh    1 <= T <= 8, dh 64 or 128, T*max_rows <= 2^19, H*dh <= 65536
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_page_store(const nmdlm_pages* pages, const uint64_t* k,
                              const uint64_t* v, int T, int H, int dh,
                              uint64_t* k_pages, uint64_t* v_pages,
                              uint8_t* key_counts, void* stream);

/* ------------------------------------------------------------------------
 * nmdlm_page_select — for each packed row and head, the context pages that
 * matter most to it.  Page p of the ctx/64 full context pages scores
 *     S = sum_t sum_c Q[t,row,c] * key_counts[page][head][t][c],
 * the sum over the page's keys and the timesteps of the attention scores
 * popcount(Q AND K).  The n_sel pages of the largest S are selected (ties: the
 * lower p; all when there are no more), and every page from ctx/64 on: the
 * rest of the context and the new rows themselves.  The integers are exact.
 *
 *   q      device spikes [T][max_rows][H*dh/64], 16-byte aligned
 *   n_sel  >= 0
 *   sel    device [max_rows][H][ceil(max_pages/64)] words: bit p%64 of word
 *          p/64 is set when logical page p is selected; rows without a page
 *          keep their words
 *   ws     workspace of nmdlm_page_select_workspace_size() bytes: at most 1 GiB
 *          (or 4 bytes a row and page, where that is more)
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_page_select(const nmdlm_pages* pages, const uint64_t* q, int T,
                               int H, int dh, const uint8_t* key_counts, int n_sel,
                               uint64_t* sel, void* ws, size_t ws_bytes, void* stream);
size_t nmdlm_page_select_workspace_size(const nmdlm_pages* pages, int T, int H, int dh);

/* ------------------------------------------------------------------------
 * nmdlm_bbm_attn_paged — nmdlm_bbm_attn (its formulas, weights and neuron) of
 * the packed rows: row i of request s over the keys of its ctx+new_rows
 * positions, in its pages.  The rows' own keys and values must be stored
 * (nmdlm_page_store).  With sel, a row of a head sees only the keys of the
 * pages whose bit is set (0 where none is: a = 0).
 *
 *   q, T, H, dh, k_pages, v_pages   see above
 *   lut_att  device uint8 [256]
 *   sel      device [max_rows][H][ceil(max_pages/64)] words or NULL (all pages)
 *   a_out    device int32 [T][max_rows][H*dh] or NULL
 *   theta_a  threshold (> 0) when s_out is given
 *   s_out    device spikes [T][max_rows][H*dh/64] or NULL (at least one output);
 *            rows without a page keep what a_out and s_out hold
 *   ws       workspace of nmdlm_bbm_attn_paged_workspace_size() bytes
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_bbm_attn_paged(const nmdlm_pages* pages, const uint64_t* q, int T,
                                  int H, int dh, const uint64_t* k_pages,
                                  const uint64_t* v_pages, const uint8_t* lut_att,
                                  const uint64_t* sel, int32_t* a_out, int32_t theta_a,
                                  uint64_t* s_out, void* ws, size_t ws_bytes, void* stream);
size_t nmdlm_bbm_attn_paged_workspace_size(const nmdlm_pages* pages, int T, int H, int dh);

/* ------------------------------------------------------------------------
 * nmdlm_block_step_paged — nmdlm_block_step (the same layers, head and
 * unmasking) for the packed rows of a page plan: requests of different lengths
 * in one step, or a prefill of their prompts (NMDLM_NO_HEAD).  The plan is made
 * before (nmdlm_page_plan) and may serve several steps; per layer the step
 * makes the calls nmdlm_page_store, nmdlm_page_select (n_sel >= 0) and
 * nmdlm_bbm_attn_paged between its products.
 *
 *   model       layers[l].k_cache and vt_cache are the layer's k_pages and
 *               v_pages; cache_cap and max_seq are not read
 *   key_counts  HOST array [n_layers] of the layers' key_counts
 *   n_sel       context pages that a row and head sees besides its own request's
 *               last ones, or below 0: all pages.  A workspace sized with
 *               NMDLM_ALL_PAGES in the flags serves steps without a selection
 *               only; the flag with n_sel >= 0 is NMDLM_ERR_INVALID_ARG
 *   io          token-indexed buffers have max_rows rows (x_in, y_out
 *               [T][max_rows][d/64], tokens, masked, pred, conf [max_rows], logits
 *               [max_rows][V]), unmasked_pos [n_seq][k_unmask] holds positions
 *               within a request's rows (-1: fewer were masked).  M, C, pos0 and
 *               n_seq are not read; a row's position comes from the plan, and one
 *               at or past max_pos has no position spike and sets
 *               NMDLM_STATUS_BAD_REQUEST.  Of a request's rows the first
 *               NMDLM_MAX_HEAD_M can be unmasked; rows without a page are not,
 *               and their outputs mean nothing.
 * Limits: T*max_rows <= 2^19; errors as for nmdlm_block_step and the paged calls.
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_block_step_paged(const nmdlm_model* model, const nmdlm_pages* pages,
                                    uint8_t* const* key_counts, int n_sel,
                                    nmdlm_step_io* io, void* ws, size_t ws_bytes,
                                    void* stream);
size_t nmdlm_block_step_paged_workspace_size(const nmdlm_model* model,
                                             const nmdlm_pages* pages, unsigned flags);

/* ------------------------------------------------------------------------
 * Drafted decoding.  A block drafted by a cheaper model is checked in one pass
 * of the target: the drafted tokens and, for every position after them, a
 * masked row that sees the tokens before its position.  The target's logits at
 * the masked rows then say which drafts stand.  The pass needs rows that see
 * different keys (nmdlm_bbm_attn_masked, nmdlm_block_step_masked), the choice
 * draws from distributions (nmdlm_token_sample, nmdlm_draft_verify).
 *
 * nmdlm_mask — which cache rows a row sees, and the positions that a bias goes
 * by:
 *   ranges    device int32 [M][4], 16-byte aligned: row m sees the cache rows j
 *             with r0 <= j < r1 or r2 <= j < r3 (ends outside the keys count as
 *             the nearest end; a range with r1 <= r0 is empty).  Documents,
 *             prefixes, blocks, windows and drafted rows are such pairs
 *   q_pos     device int32 [M]: positions of the rows, or NULL
 *   k_pos     device int32 [n_keys]: positions of the cache rows, or NULL
 *   max_dist  0 .. NMDLM_MAX_DIST: distances beyond count as this
 * ------------------------------------------------------------------------ */
#define NMDLM_MAX_DIST 1024
typedef struct nmdlm_mask {
  const int32_t* ranges;
  const int32_t* q_pos;
  const int32_t* k_pos;
  int max_dist;
} nmdlm_mask;

/* ------------------------------------------------------------------------
 * nmdlm_bbm_attn_masked — nmdlm_bbm_attn (its sums, weights and neuron) of rows
 * that see the keys of their ranges, with a bias of the scores by distance:
 *     s = popcount(Q[t,i,head h] AND K[t,j,head h])
 *     x = s + bias[h][clamp(q_pos[i] - k_pos[j], -max_dist, max_dist) + max_dist]
 *     p = lut_att[clamp(x, 0, 255)] for the keys that row i sees
 *     a[t,i,c] = floor(256 * sum_j p * V[t,j,c] / sum_j p)   (0 if sum_j p = 0)
 * A cap of the scores is a matter of the table.  A row that sees nothing gets
 * a = 0.  The integers are exact and do not depend on how the work is split.
 *
 *   q, k_cache, vt_cache, cache_cap, T, M, H, dh, lut_att, a_out, theta_a, s_out
 *           as nmdlm_bbm_attn
 *   n_keys  cache rows that can be seen: 1 .. NMDLM_MAX_KEYS, at most cache_cap
 *   mask    HOST struct of device pointers
 *   bias    device int8 [H][2*max_dist + 1] or NULL (no bias; positions and
 *           max_dist are not read)
 *   ws      workspace of nmdlm_bbm_attn_masked_workspace_size() bytes
 * Errors: NMDLM_ERR_INVALID_ARG for a missing or misaligned pointer (positions
 * with a bias among them), a size below 1, max_dist outside its bounds, n_keys
 * past the cache; NMDLM_ERR_UNSUPPORTED as for nmdlm_bbm_attn.
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_bbm_attn_masked(const uint64_t* q, const uint64_t* k_cache,
                                   const uint64_t* vt_cache, int64_t cache_cap, int T,
                                   int M, int n_keys, int H, int dh, const uint8_t* lut_att,
                                   const nmdlm_mask* mask, const int8_t* bias,
                                   int32_t* a_out, int32_t theta_a, uint64_t* s_out,
                                   void* ws, size_t ws_bytes, void* stream);
size_t nmdlm_bbm_attn_masked_workspace_size(int T, int M, int n_keys, int H, int dh);

/* ------------------------------------------------------------------------
 * nmdlm_block_step_masked — nmdlm_block_step (the same layers, head and
 * unmasking) of one sequence's rows that see the keys of a mask: keys and values
 * of the M rows go to cache rows [C, C+M), and row m sees the cache rows of
 * ranges[m] among the C+M.  In one step it scores drafted tokens, several
 * documents or a whole sequence block by block.
 *
 *   mask   HOST struct; q_pos are the rows' positions (with x_in they are read for a
 *          bias only).  One outside the position table has no position spike and
 *          sets NMDLM_STATUS_BAD_REQUEST; k_pos [C+M], the new rows' own among them
 *   bias   HOST array [n_layers] of device tables (as nmdlm_bbm_attn_masked; NULL:
 *          none in this layer), or NULL
 *   io     as nmdlm_block_step; pos0 and NMDLM_ATTN_FUSED are not read, n_seq is 0 or 1
 *          (else NMDLM_ERR_UNSUPPORTED)
 *   ws     nmdlm_block_step_masked_workspace_size() for C+M keys (which does not
 *          fall as the keys grow), cleared as for nmdlm_block_step
 * Errors: as nmdlm_block_step and nmdlm_bbm_attn_masked.
 * ------------------------------------------------------------------------ */
nmdlm_status nmdlm_block_step_masked(const nmdlm_model* model, const nmdlm_mask* mask,
                                     const int8_t* const* bias, nmdlm_step_io* io, void* ws,
                                     size_t ws_bytes, void* stream);
size_t nmdlm_block_step_masked_workspace_size(const nmdlm_model* model, int M, int n_keys,
                                              unsigned flags);

/* ------------------------------------------------------------------------
 * nmdlm_token_sample — a token of each row of logits.  With the row's largest
 * logit l_max, temperature tau and w_v = exp((l_v - l_max) / tau) (float64, to
 * 4.6e-16 + 1.2e-16 |exponent| of itself; 0 for exponents below -700 and for NaN, 1
 * where l_v = l_max), the token is the first v with
 *     w_0 + ... + w_v > u * sum_j w_j
 * (the last of positive weight when none is); at tau = 0 the first of the
 * largest logits.  conf is w_token / sum_j w_j, at tau = 0 with tau = 1 in the
 * weights, as the block step has it.  A row of -inf and NaN alone: token -1,
 * conf 0.
 *
 *   logits  device float [M][V]
 *   u       device float [M] in [0, 1) (not read at tau = 0; may then be NULL)
 *   tokens  device int32 [M]
 *   conf    device double [M] or NULL
 *   ws      workspace of nmdlm_token_sample_workspace_size() bytes (any content)
 * Limits: M <= NMDLM_MAX_SAMPLE_M, V <= NMDLM_MAX_SAMPLE_V, else
 * NMDLM_ERR_UNSUPPORTED.  Errors: NMDLM_ERR_INVALID_ARG for a missing or misaligned
 * pointer, a size below 1, a temperature that is negative, infinite or NaN.
 * ------------------------------------------------------------------------ */
#define NMDLM_MAX_SAMPLE_V 16777216
#define NMDLM_MAX_SAMPLE_M 65535
nmdlm_status nmdlm_token_sample(const float* logits, int M, int V, double temperature,
                                const float* u, int32_t* tokens, double* conf, void* ws,
                                size_t ws_bytes, void* stream);
size_t nmdlm_token_sample_workspace_size(int M, int V);

/* ------------------------------------------------------------------------
 * nmdlm_draft_verify — which drafted tokens stand, and what replaces the first
 * that does not.  Row m has a draft x = draft[m] drawn from q (the
 * draft's distribution), and the target's distribution p, both as in
 * nmdlm_token_sample (at temperature 0: all on the first of the largest).  The
 * draft is taken when
 *     u[m][0] * q(x) < p(x);
 * else the token is drawn by u[m][1], as in nmdlm_token_sample, with the
 * weights max(p_v - q_v, 0) (p where these sum to 0).  Tokens that come out so
 * are distributed as p.  A row without a draft (an id outside [0, V)) is drawn
 * from p.
 *
 * Rows [cu_rows[s], cu_rows[s+1]) are request s's, in order: the rows up to its
 * first that takes no draft count, that one included (a row without a draft
 * behind the drafts gives the token that follows them all).  The rows after it
 * get token -1, accepted 0 and conf 0.  With NMDLM_VERIFY_EACH every row counts
 * (positions that were drafted independently).  Rows outside [cu_rows[0],
 * cu_rows[n_seq]) are left as they were.
 *
 *   logits        device float [M][V], the target's
 *   draft_logits  device float [M][V], the draft's, or NULL: drafts were certain
 *                 (q is 1 at the draft).  Not read in rows without a draft
 *   draft         device int32 [M]
 *   u             device float [M][2] in [0, 1)
 *   cu_rows       device int32 [n_seq + 1], not decreasing, within [0, M], or NULL:
 *                 one request of all M rows (n_seq = 1)
 *   tokens        device int32 [M];  accepted  device uint8 [M]
 *   n_accepted    device int32 [n_seq] or NULL: drafts taken that count
 *   conf          device double [M] or NULL: the target's probability of the
 *                 token, as in nmdlm_token_sample
 *   flags         0 or NMDLM_VERIFY_EACH
 *   ws            workspace of nmdlm_draft_verify_workspace_size() bytes (any content)
 * Limits and errors: as nmdlm_token_sample; n_seq <= NMDLM_MAX_PLAN_ROWS;
 * NMDLM_ERR_INVALID_ARG for other flags and for n_seq other than 1 without cu_rows.
 * ------------------------------------------------------------------------ */
#define NMDLM_VERIFY_EACH 0x1u
nmdlm_status nmdlm_draft_verify(const float* logits, const float* draft_logits, int M, int V,
                                const int32_t* draft, const float* u, double temperature,
                                double draft_temperature, const int32_t* cu_rows, int n_seq,
                                unsigned flags, int32_t* tokens, uint8_t* accepted,
                                int32_t* n_accepted, double* conf, void* ws,
                                size_t ws_bytes, void* stream);
size_t nmdlm_draft_verify_workspace_size(int M, int V);

/* Clears a workspace region with a fill kernel on the stream (use once on a
 * new workspace). */
nmdlm_status nmdlm_workspace_clear(void* ws, size_t ws_bytes, void* stream);

const char* nmdlm_status_string(nmdlm_status s);
int nmdlm_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* NMDLM_H */
