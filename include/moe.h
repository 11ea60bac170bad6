/*
 * moe.h -- C ABI of the MI355X (gfx950) routed MoE FFN forward, the hot path
 * of EPS-MoE (arXiv 2410.12247): top-k softmax gating, expert-sorted
 * dispatch, the SwiGLU expert FFN run as one grouped GEMM or as per-expert
 * dense GEMMs, and the weighted combine, for one GPU's share of experts.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Tensor pointers are DEVICE pointers owned by the caller; the library
 *   never frees or retains them.  moe_dims and moe_opts live in host memory.
 * - Layouts are row-major and dense.  bf16 tensors are passed as their
 *   16-bit patterns (moe_bf16).  Expert weights use the [out, in] layout of
 *   a linear layer, so both GEMM operands are contiguous along the reduced
 *   dimension:  w_gate, w_up [EL][I][H];  w_down [EL][H][I];  shared
 *   gate/up [Is][H], shared down [H][Is].
 * - Every call is asynchronous on `stream` (a hipStream_t; NULL is the null
 *   stream) unless stated otherwise.
 * - Arguments are checked on the host before anything is enqueued; a bad
 *   argument returns MOE_ERR_INVALID / MOE_ERR_UNSUPPORTED /
 *   MOE_ERR_WORKSPACE and leaves every buffer untouched.  A failing HIP call
 *   returns MOE_ERR_HIP.  moe_last_error() gives the message of the last
 *   failure on the calling thread.  Nothing aborts or throws.
 * - tokens == 0 is a valid no-op.
 * - Supported sizes: 1 <= experts <= 256, 1 <= top_k <= min(experts, 8),
 *   hidden, inter and shared_inter multiples of 64 up to 2^20, local experts
 *   [local_begin, local_begin + local_count) inside [0, experts),
 *   tokens * top_k < 2^31.
 * - Results are deterministic: the same inputs and options give the same
 *   bits on every run.  With MOE_FLAG_EXACT_ORDER (and in moe_ffn_group and
 *   moe_ffn_dense) every expert-GEMM output is one pass over K, so the bits
 *   are also the same for any pipeline number, stage kind, CU budget and
 *   either GEMM kind.  Without it the grouped GEMM may cut the tiles of its
 *   last, partial round into K pieces summed in a fixed order, and a launch
 *   of at most 16 rows per expert may run as a streaming GEMM that cuts every
 *   K into eight; which of them it does, and so the last bits, follows from
 *   the shape and the options (group_tile_rows, gemm_cu_budget or side_cus
 *   other than 0 switch the streaming form off).
 */
#ifndef MOE_H
#define MOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef uint16_t moe_bf16; /* bf16 bit pattern */
typedef uint8_t moe_e4m3;  /* OCP 8-bit float: 4 exponent, 3 mantissa bits, no infinity */
typedef uint8_t moe_scale; /* E8M0: 2^(byte - 127); 255 is NaN */

typedef enum {
    MOE_OK = 0,
    MOE_ERR_INVALID = 1,     /* null pointer, size out of range, bad option */
    MOE_ERR_UNSUPPORTED = 2, /* experts > 256 or top_k > 8 */
    MOE_ERR_WORKSPACE = 3,   /* workspace smaller than moe_workspace_bytes() */
    MOE_ERR_HIP = 4          /* a HIP runtime call failed */
} moe_status;

/* Problem shape.  T tokens of width H are routed over E experts (top-k);
 * this GPU computes local experts [local_begin, local_begin + local_count),
 * each a SwiGLU FFN of width I, plus optional shared experts applied to
 * every token whose concatenated width is shared_inter (0 = none). */
typedef struct {
    int64_t tokens;       /* T */
    int32_t hidden;       /* H */
    int32_t inter;        /* I */
    int32_t experts;      /* E, router width */
    int32_t top_k;        /* k */
    int32_t local_begin;  /* e0 */
    int32_t local_count;  /* EL */
    int32_t renormalize;  /* 1: softmax over the k selected; 0: over all E */
    int32_t shared_inter; /* Is (0 = no shared experts) */
} moe_dims;

enum { MOE_GEMM_AUTO = 0, MOE_GEMM_GROUP = 1, MOE_GEMM_DENSE = 2 };
/* Element types of tensors that may come in either. */
enum { MOE_BF16 = 0, MOE_FP32 = 1 };
enum { MOE_CHUNK_EXPERTS = 0, MOE_CHUNK_TOKENS = 1 };
enum {
    MOE_FLAG_TIMING = 1,
    MOE_FLAG_TIMING_GEMM = 2,
    MOE_FLAG_EXACT_ORDER = 4,
    MOE_FLAG_SERIAL = 8
};

/* Options of moe_ffn_forward (Sec. 4.3 of the paper: the GroupGemm /
 * DenseGemm switch by load, the pipeline number PN and how the work is cut
 * into pipeline stages).
 * chunk_mode MOE_CHUNK_EXPERTS (default): stage s is the expert group
 *   [s*EL/PN, (s+1)*EL/PN) with all of its rows, so each expert's weights
 *   are read by one stage only (the paper's horizontal split with weights
 *   split by expert, Sec. 4.3).  PN must divide local_count.
 * chunk_mode MOE_CHUNK_TOKENS: stage s is the token range
 *   [s*ceil(T/PN), (s+1)*ceil(T/PN)) over all local experts, so every stage
 *   reads every local expert's weights again (the split the paper argues
 *   against); kept as a measured comparison.  Needs PN*local_count <= 256.
 * Both modes give the same bits under MOE_FLAG_EXACT_ORDER. */
typedef struct {
    int32_t gemm_mode;      /* MOE_GEMM_AUTO, _GROUP or _DENSE */
    int32_t dense_min_rows; /* 0: AUTO weighs GroupGemm against DenseGemm
                               for each stage of at most two experts with
                               the library's launch-cost model (see
                               moe_gemm_plan) and takes GroupGemm for larger
                               stages.  > 0: AUTO picks DenseGemm for a
                               stage when every expert in it has at least
                               this many rows (Sec. 3.2 Conclusion 1's
                               threshold m), else GroupGemm */
    int32_t pipeline_n;     /* PN >= 1, the number of pipeline stages; 0 = chosen
                               by the library from the row counts (expert
                               stages only; see moe_pipeline_plan) */
    int32_t gemm_cu_budget; /* workgroups of the persistent grouped GEMM;
                               0 = one per compute unit */
    int32_t flags;          /* MOE_FLAG_TIMING: time each phase with HIP
                               events (read with moe_last_timing).
                               MOE_FLAG_TIMING_GEMM: time only the expert
                               GEMM launches (gate/up, down, shared), with
                               one event between consecutive launches of a
                               stream; the other phases read 0.  Every
                               event recorded between two kernels delays
                               the second, so this is the mode to time a
                               run whose wall time also matters.
                               MOE_FLAG_EXACT_ORDER: no K split in the
                               grouped GEMM (see the determinism note at
                               the top); slower when the tile count leaves
                               a partial last round of the grid.
                               MOE_FLAG_SERIAL: every step of every stage
                               (and the shared experts) runs on the caller's
                               stream in order, so nothing overlaps: the
                               paper's serial mode (Sec. 5.2), which
                               measures what cutting the work into PN stages
                               costs by itself.  Same bits as without it. */
    int32_t chunk_mode;     /* MOE_CHUNK_EXPERTS or MOE_CHUNK_TOKENS */
    int32_t dense_tile_rows;/* token rows of a DenseGemm tile: 0 = chosen per
                               expert from its row count (the height whose
                               tile count fills the chip best), or 128, 192,
                               256, 320 to force one */
    int32_t side_cus;       /* Sec. 5.2's SM control: when the forward uses
                               its side streams (PN != 1 or shared experts),
                               0 = no CU masks; > 0 = the gather and combine
                               streams run on this many CUs (spread over the
                               XCDs) and the GEMM stream, with its persistent
                               grid, on the others.  At most 248. */
    int32_t group_tile_rows;/* token rows of a GroupGemm tile: 0 = chosen per
                               stage by the launch-cost model (never taller
                               than the smallest height that holds the
                               stage's largest expert), or 128, 192, 256,
                               320 to force one */
} moe_opts;

/* Per-phase device time, in milliseconds summed over stages and over the
 * timed moe_ffn_forward calls (MOE_FLAG_TIMING or MOE_FLAG_TIMING_GEMM) this
 * thread made on one device since it last called moe_last_timing (`calls`
 * of them), so a timed loop needs one read at its end, not a host sync per
 * step.  Launch and stage counts add up the same way; pipeline_n is the
 * last call's. */
typedef struct {
    float route_ms, permute_ms, gather_ms, gateup_ms, down_ms, shared_ms,
        combine_ms, total_ms;
    int32_t gateup_launches, down_launches; /* GEMM kernel launches timed */
    int32_t dense_stages, group_stages;     /* policy decisions taken */
    int32_t pipeline_n;                     /* stages the last call ran */
    int32_t calls;                          /* timed calls summed */
} moe_timing;

/* The paper's pipeline-number analysis (Sec. 5.2 items 4-5) for one
 * forward, evaluated with the library's cost models. */
typedef struct {
    double t_comm_us;   /* T_comm before the split: the combine, one-GPU
                           stand-in for the dispatch and combine all2alls */
    double t_comp_us;   /* T_comp before the split: the expert GEMMs */
    double t_comm_n_us; /* N * S(m/N): the stages' combines, summed */
    double t_comp_n_us; /* N * G(m/N, E/N): the stages' GEMMs, summed */
    double eps0;        /* N * S(m/N) / S(m) - 1 */
    double eps1;        /* N * G(m/N, E/N) / G(m, E) - 1 */
    double overlap_frac;/* share of the CUs the GEMM grid leaves free for
                           the side streams (CU budget or side_cus): the
                           part of L(N) one GPU can realise */
    double gain_us;     /* L(N) - R(N): min(T_comm, T_comp) (N - 1) / N *
                           overlap_frac, minus the split's extra GEMM and
                           combine time and a fixed cost per added stage */
    int32_t enabled;    /* eps0 <= 0.32 and eps1 <= 0.03 (the values of the
                           paper's DeepSeekV2 test), or N = 1 */
    int32_t pipeline_n; /* N */
} moe_pipeline_eval;

/* Bytes of device workspace: with opts == NULL, what moe_permute needs;
 * with opts != NULL, what moe_ffn_forward needs with those options (a
 * superset).  Host-only; never touches the GPU.  Returns 0 for invalid dims
 * or options. */
size_t moe_workspace_bytes(const moe_dims *dims, const moe_opts *opts);

/* Guard gaps of the workspace layout (a debugging aid for out-of-region
 * writes; no passage of the paper defines it).  After every region of the
 * layout moe_workspace_bytes() sizes, the library leaves MOE_WS_GUARD_BYTES
 * bytes that no call reads or writes: a caller may fill them with a canary
 * before a call and compare them after it.  Writes the byte offsets of the
 * first `capacity` gaps (from the workspace start) to `offsets` and returns
 * how many gaps the layout has; -1 for invalid dims or options, or for
 * offsets == NULL with capacity > 0.  opts as in moe_workspace_bytes.
 * Host-only; never touches the GPU. */
#define MOE_WS_GUARD_BYTES 256
int32_t moe_workspace_guards(const moe_dims *dims, const moe_opts *opts, int64_t *offsets,
                             int32_t capacity);

/* Router (the topKGating operator of Sec. 3.3; k of E experts per token as
 * in Sec. 3.2).  For each token t:
 *   z[e] = fp32 fused-multiply-add chain over h = 0..H-1 (ascending, from
 *          +0) of x[t][h] * w_router[e][h], then + bias[e] (one fp32 add)
 *   topk_ids[t][0..k)  the k largest z, by (z descending, e ascending);
 *                      -0 and +0 are equal
 *   topk_w[t][j]       softmax weight, computed in fp64 and rounded to fp32:
 *                      over the k selected logits when renormalize, else
 *                      over all E logits.
 * x [T][H] bf16; w_router [E][H] fp32; bias [E] fp32 or NULL;
 * topk_ids [T][k] int32 (global expert ids); topk_w [T][k] fp32.
 * Logits are never materialised.  NaN logits are not supported (their weights
 * are undefined; a token's k experts stay distinct).  x and w_router may sit at
 * any address of their element type; x off 16 bytes takes slower kernels with
 * the same bits. */
moe_status moe_route(const moe_dims *dims, const moe_bf16 *x, const float *w_router,
                     const float *bias, int32_t *topk_ids, float *topk_w, void *stream);

/* Dispatch (Fig. 7a: each expert takes its tokens in ascending order;
 * Sec. 4.3: inputs split by rows, weights by expert).  Rows are ordered by
 * (local expert ascending, token ascending):
 *   counts [EL]        rows of each local expert
 *   offsets [EL+1]     exclusive prefix of counts (unpadded)
 *   sorted_slot [R]    row -> slot t*k+j   (R = offsets[EL] <= T*min(k,EL);
 *                      the buffer must hold T*min(k,EL) entries)
 *   slot_row [T*k]     slot -> row, -1 when the slot's expert is not local
 *   x_perm [R][H]      x_perm[r] = x[sorted_slot[r] / k]; may be NULL to
 *                      build the indices only (then x may be NULL too)
 * Deterministic: scan-based, no atomics decide an order.
 * ws: device workspace of at least moe_workspace_bytes(dims, NULL) bytes. */
moe_status moe_permute(const moe_dims *dims, const int32_t *topk_ids, const moe_bf16 *x,
                       int32_t *counts, int32_t *offsets, int32_t *sorted_slot,
                       int32_t *slot_row, moe_bf16 *x_perm, void *ws, size_t ws_bytes,
                       void *stream);

/* Gather of the rows of local experts [e_first, e_first + e_count) only:
 * x_perm[r] = x[sorted_slot[r] / k] for r in [offsets[e_first],
 * offsets[e_first + e_count]).  offsets and sorted_slot are device arrays
 * from moe_permute.  The dispatch of one pipeline stage. */
moe_status moe_gather(const moe_dims *dims, int32_t e_first, int32_t e_count,
                      const int32_t *offsets, const int32_t *sorted_slot,
                      const moe_bf16 *x, moe_bf16 *x_perm, void *stream);

/* GroupGemm expert FFN (Sec. 3.2, Conclusions 1-3; Fig. 3): ONE launch per
 * GEMM for all rows of local experts [e_first, e_first + e_count), each
 * expert with its own row count read on the device from offsets, so no
 * host synchronisation is needed.  For every such row r of expert e:
 *   act[r]    = bf16( silu(g) * u ), g = w_gate[e] x_perm[r],
 *                                     u = w_up[e] x_perm[r]   (fp32 accum)
 *   y_perm[r] = w_down[e] act[r]                               (fp32 accum)
 * bf16 MFMA with fp32 accumulation; silu(g) = g / (1 + exp(-g)).
 * w_gate/w_up/w_down point at the stacks of all EL local experts.
 * act [R][I] bf16 (caller scratch, rows indexed like x_perm);
 * y_perm [R][H] fp32.  cu_budget: persistent grid size (0 = all CUs).
 * Takes no workspace, so every tile is one pass over K (the bits of
 * moe_ffn_forward with MOE_FLAG_EXACT_ORDER). */
moe_status moe_ffn_group(const moe_dims *dims, int32_t e_first, int32_t e_count,
                         const int32_t *offsets, const moe_bf16 *x_perm,
                         const moe_bf16 *w_gate, const moe_bf16 *w_up,
                         const moe_bf16 *w_down, moe_bf16 *act, float *y_perm,
                         int32_t cu_budget, void *stream);

/* DenseGemm expert FFN (Sec. 4.3: with one expert per pipeline stage the
 * grouped GEMM becomes a dense one): one dense SwiGLU FFN over `rows`
 * contiguous rows whose count is known on the host, so the launch takes the
 * tile height (128 to 320 token rows) whose tile count fills the chip best:
 *   act[r] = bf16(silu(w_gate x[r]) * (w_up x[r])),  y[r] = w_down act[r]
 * x [rows][hidden] bf16; w_gate, w_up [inter][hidden]; w_down
 * [hidden][inter]; act [rows][inter] bf16 scratch; y [rows][hidden] fp32.
 * Usable for shared experts (inter = shared width, x = all tokens), which
 * moe_ffn_forward runs through the grouped scheduler instead (one expert
 * of T rows).  Same arithmetic and bits as moe_ffn_group for the same
 * rows. */
moe_status moe_ffn_dense(int64_t rows, int32_t hidden, int32_t inter, const moe_bf16 *x,
                         const moe_bf16 *w_gate, const moe_bf16 *w_up,
                         const moe_bf16 *w_down, moe_bf16 *act, float *y, void *stream);

/* Combine (LocalReduce, Fig. 7b) of the local experts [e_first,
 * e_first + e_count):  for every token t,
 *   y[t] = (accumulate ? y[t] : 0) + sum_j topk_w[t][j] * y_perm[slot_row[t*k+j]]
 * over the slots j whose expert lies in that range, the terms taken in
 * ascending expert order, each added with one fp32 fused multiply-add.
 * Running the stages of a pipeline in order (first with accumulate = 0, or
 * all with accumulate = 1 over a y that holds the shared experts' output)
 * gives the same bits as one call over all local experts.
 * y_perm [R][H] fp32; topk_ids, slot_row [T][k] int32; topk_w [T][k];
 * y [T][H] fp32. */
moe_status moe_combine(const moe_dims *dims, int32_t e_first, int32_t e_count,
                       const float *y_perm, const int32_t *topk_ids, const int32_t *slot_row,
                       const float *topk_w, float *y, int32_t accumulate, void *stream);

/* The whole forward of one MoE layer's routed FFN for this GPU's experts:
 * route -> dispatch -> per pipeline stage { gather ; GroupGemm or DenseGemm
 * (picked per stage from its row counts, Sec. 3.2 Conclusion 1 and
 * Sec. 4.3) ; combine }, with stage i+1's gather and stage i-1's combine
 * running on their own streams beside stage i's GEMMs (the one-GPU form of
 * the expert pipeline of Sec. 4.3-4.4).  The shared experts (if any) run
 * first, as one grouped-GEMM expert of all T rows, and write y; otherwise
 * the first combine writes every token.
 * topk_ids, topk_w, counts: optional outputs (NULL = keep them in the
 * workspace).  shared_*: required iff dims->shared_inter > 0.
 * ws: at least moe_workspace_bytes(dims, opts) bytes of device memory.
 * Ordered after prior work on `stream` and finished on `stream`.  When the
 * policy needs row counts on the host (gemm_mode != GROUP or PN > 1) the
 * call blocks the host once on a 4*EL-byte device-to-host copy (AUTO needs
 * the counts only when its threshold can be reached by some expert).
 * Thread safety: calls from several host threads on one device are
 * serialised inside the library (the side streams, ordering events and the
 * pinned copy of the counts are per device); moe_last_timing reads the
 * calling thread's own timed calls. */
moe_status moe_ffn_forward(const moe_dims *dims, const moe_opts *opts, const moe_bf16 *x,
                           const float *w_router, const float *bias,
                           const moe_bf16 *w_gate, const moe_bf16 *w_up,
                           const moe_bf16 *w_down, const moe_bf16 *shared_gate,
                           const moe_bf16 *shared_up, const moe_bf16 *shared_down,
                           float *y, int32_t *topk_ids, float *topk_w, int32_t *counts,
                           void *ws, size_t ws_bytes, void *stream);

/* moe_ffn_forward for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the same computation, arguments and bits as moe_ffn_forward with the same
 * options, but it takes no workspace.  Its scratch is a static device buffer
 * of 256 MiB in the library (each device the library runs on holds its own
 * copy until the process ends); the call allocates nothing, on the device or
 * the host.  Limits: moe_workspace_bytes(dims, opts) must not exceed
 * 256 MiB (e.g. up to 512 tokens of the Mixtral-, DBRX- and DeepSeekV2-shaped
 * layers, or decode batches), else MOE_ERR_UNSUPPORTED; options that need
 * the row counts on the host (pipeline_n > 1, MOE_GEMM_DENSE, or an AUTO
 * threshold some expert can reach) and the timing flags are refused with
 * MOE_ERR_UNSUPPORTED; every step runs on `stream` (shared experts
 * included), with the same bits as with side streams.  All calls on one
 * device share the buffer, and it keeps the last call's contents: calls from
 * several host threads are serialised, but calls that overlap on the GPU
 * (this one still running when another is enqueued on another stream) race
 * on it.  Nothing in the buffer needs to start zeroed. */
moe_status moe_ffn_forward_noalloc(const moe_dims *dims, const moe_opts *opts,
                                   const moe_bf16 *x, const float *w_router, const float *bias,
                                   const moe_bf16 *w_gate, const moe_bf16 *w_up,
                                   const moe_bf16 *w_down, const moe_bf16 *shared_gate,
                                   const moe_bf16 *shared_up, const moe_bf16 *shared_down,
                                   float *y, int32_t *topk_ids, float *topk_w, int32_t *counts,
                                   void *stream);

/* Timing of the timed moe_ffn_forward calls on this thread since the
 * previous read (waits for their events); the next timed call then starts a
 * new record.  Returns MOE_ERR_INVALID when no timed call was made. */
moe_status moe_last_timing(moe_timing *out);

/* The paper's enable condition and gain for PN = pipeline_n expert stages
 * (pipeline_n = 0: the PN moe_ffn_forward would choose with pipeline_n = 0,
 * i.e. the divisor of local_count with the largest gain among those
 * enabled, when that gain is at least 5% of the unsplit GEMM time (the
 * launch-cost model's error), else 1), from the host row counts
 * rows[0..local_count) of the local experts.  The GEMM terms use the launch-cost model of the GEMM
 * kind AUTO (or opts->gemm_mode) takes per stage; the communication terms
 * the combine's bytes at its measured streaming rate.  Expert stages only.
 * Host-only; never touches the GPU. */
moe_status moe_pipeline_plan(const moe_dims *dims, const moe_opts *opts, const int32_t *rows,
                             int32_t pipeline_n, moe_pipeline_eval *out);

/* The GEMM plan AUTO makes for one pipeline stage (Sec. 3.2 Conclusion 1:
 * GroupGemm and DenseGemm each win over part of the load range; Sec. 4.3:
 * with one expert per stage the grouped GEMM becomes a dense one), from the
 * host row counts of its n_experts experts, rows[0..n_experts).  The model
 * prices each launch from measured per-tile costs of every tile height:
 * GroupGemm is one launch over the stage with one tile height (the model's
 * cheapest up to the smallest height that holds the largest expert, taken
 * when at least 5% below that height's price; or opts->group_tile_rows), also
 * where a decode-sized launch would take the streaming or the one-wave form,
 * which the model does not know;
 * DenseGemm is one launch per expert with its own tile height.  Writes *dense (1 when
 * the stage would run DenseGemm under opts->gemm_mode, AUTO included) and,
 * when not NULL, tile_rows[e] (the tile height of expert e's launch, 0 for
 * an empty expert), *group_us and *dense_us (predicted GEMM microseconds
 * of the two kinds).  Uses dims->hidden / inter, opts->gemm_cu_budget,
 * dense_min_rows, dense_tile_rows, group_tile_rows and MOE_FLAG_EXACT_ORDER.  Host-only;
 * never touches the GPU (the grid is the current device's CU count, 256
 * when no device is visible). */
moe_status moe_gemm_plan(const moe_dims *dims, const moe_opts *opts, int32_t n_experts,
                         const int32_t *rows, int32_t *dense, int32_t *tile_rows,
                         double *group_us, double *dense_us);

/* Pipeline number from the overhead model of the paper's ablation (Sec. 5.2):
 * PN stages hide (PN - 1)/PN of C = min(T_comm, T_comp), the smaller of the
 * unsplit communication and computation times, and cost R(PN) = k*PN + b, so
 * the latency gain of PN > 1 is G(PN) = C - b - (C/PN + k*PN), largest near
 * PN = sqrt(C/k).  Writes to *pn the PN in [1, local_count] that divides
 * local_count and maximises G, with G(1) = 0 (no pipeline, no overhead); a
 * pipeline is chosen only when its gain is positive, and ties go to the
 * smaller PN.  k = 0 (no per-stage overhead) picks the largest PN whose gain
 * is positive.  *gain_ms (may be NULL) receives G(*pn).  Times in ms; c_ms
 * and k_ms must be finite and >= 0, b_ms finite, local_count in [1, 256],
 * else MOE_ERR_INVALID.  Host-only; never touches the GPU. */
moe_status moe_choose_pipeline_n(double c_ms, double k_ms, double b_ms, int32_t local_count,
                                 int32_t *pn, double *gain_ms);

/* ---- Block-scaled 8-bit operators ---------------------------------------
 * A value is an e4m3 number times the power of two of its block:
 *   activations  q [rows][C] with scales [rows][pitch(C)], one byte per row
 *                and 128 columns;
 *   weights      q [n][k] with scales [ceil(n/128)][pitch(k)], one byte per
 *                128 x 128 block; stacks of experts add a leading dimension.
 * pitch(k) = moe_scale_pitch(k): ceil(k/128) bytes padded to whole 4-byte
 * words; the padding is neither read as a scale nor written.  The last block
 * of a width that is no multiple of 128 (or of a matrix height) covers what is
 * left of it.
 *
 * Quantising takes the smallest power of two 2^e with |v| <= 448 * 2^e for
 * every value of the block (e in [-127, 120]; e = 0 for a block of zeros) and
 * rounds v * 2^-e to e4m3, to nearest, ties to even.  A NaN stays a NaN and an
 * infinity becomes one; beside an infinity (e = 120) a block's other values
 * are rounded to zero, or nearly.
 *
 * The products take any byte of 0 to 254 as a scale; 255 makes a NaN.  Launches of
 * some 17 to 100 rows per expert are slower by up to 2.4 times where bytes are below
 * 10 or above 246 (a block whose largest value is below 2^-108 or above 2^119).
 *
 * The products run on the matrix cores with fp32 accumulators and the scales
 * applied on the way.  Inside an 8-bit matrix instruction the products of
 * eight consecutive k are added as one group, each cut to 13 bits below the
 * group's largest exponent, so a sum's error is at most 2^-10 times the sum
 * over groups of the group's largest |product| (1.5e-5 of the result's norm
 * on Gaussian data), whatever the output type.  Launches of few rows, which the
 * weights' stream bounds, widen the values to bf16 instead and are exact to
 * fp32.  Which form a launch takes depends on its dims and widths alone: not on
 * the data, the expert range or the device's state, so results have the same
 * bits from run to run and from a range as from the whole.
 *
 * Tensors must be 16-byte aligned, scale tensors 4-byte aligned, else
 * MOE_ERR_INVALID, and belong to the current device.  Rows behind the last
 * expert's are not written.  Row counts below 2^31; a token matrix read
 * through sorted_slot must be smaller than 4 GiB, else MOE_ERR_UNSUPPORTED.
 * The calls allocate nothing, never synchronise and can be captured into a
 * graph.  No output may overlap an input unless stated. */

/* Bytes of one scale row of a width k; 0 unless k is a positive multiple of
 * 64 up to 2^20.  Host-only. */
size_t moe_scale_pitch(int32_t k);

/* q, scales = Q(x).  x [rows][cols] of x_type (MOE_BF16 or MOE_FP32); cols a
 * multiple of 64. */
moe_status moe_quant_rows(int64_t rows, int32_t cols, const void *x, int32_t x_type, moe_e4m3 *q,
                          moe_scale *scales, void *stream);

/* q, scales = Q(w) in 128 x 128 blocks, for `experts` (at most 256) stacked
 * weight matrices w [experts][n][k]; n and k multiples of 64. */
moe_status moe_quant_weights(int32_t experts, int32_t n, int32_t k, const moe_bf16 *w,
                             moe_e4m3 *q, moe_scale *scales, void *stream);

/* The normalisation in front of an MoE layer, with the residual's addition
 * and the quantised rows the products take:
 *   s = x + residual             (residual NULL: s = x)
 *   total = bf16(s)              the residual stream behind the addition (s
 *                                rounded to fp32 first)
 *   v = s * rsqrt(mean(s^2) + eps) * weight   (weight NULL: ones)
 *   y = bf16(v)                  what the router reads
 *   q, scales = Q(v)             from v before its rounding to bf16
 * v is computed in 64 bits.
 * x [rows][hidden] of x_type (MOE_FP32 is what moe_combine writes); residual,
 * total, y [rows][hidden] bf16; weight [hidden] bf16.  total, y and the pair
 * q, scales may each be NULL; y or q has to be given.  total may be the
 * residual itself, and y may be a bf16 x. */
moe_status moe_norm_quant(int64_t rows, int32_t hidden, const void *x, int32_t x_type,
                          const moe_bf16 *residual, const moe_bf16 *weight, float eps,
                          moe_bf16 *total, moe_bf16 *y, moe_e4m3 *q, moe_scale *scales,
                          void *stream);

/* Dense product y[r][j] = sum_k x[r][k] w[j][k], y [rows][n] of y_type
 * (MOE_BF16 or MOE_FP32), w [n][k]; n and k multiples of 64. */
moe_status moe_gemm_scaled(int64_t rows, int32_t n, int32_t k, const moe_e4m3 *x,
                           const moe_scale *x_scales, const moe_e4m3 *w,
                           const moe_scale *w_scales, void *y, int32_t y_type, void *stream);

/* The same grouped by expert: for every row r of the local experts [e_first,
 * e_first + e_count) (offsets from moe_permute, read on the device),
 *   y[r] = w[e] x_row(r),  x_row(r) = x[r], or with sorted_slot (from
 *   moe_permute too) the token row x[sorted_slot[r] / top_k].
 * w [EL][n][k] is the stack of all local experts; x [R][k], or [T][k] with
 * sorted_slot; y [R][n] of y_type.  dims gives the tokens, top_k and local
 * experts; its widths are not used. */
moe_status moe_gemm_group_scaled(const moe_dims *dims, int32_t e_first, int32_t e_count,
                                 const int32_t *offsets, const int32_t *sorted_slot, int32_t n,
                                 int32_t k, const moe_e4m3 *x, const moe_scale *x_scales,
                                 const moe_e4m3 *w, const moe_scale *w_scales, void *y,
                                 int32_t y_type, void *stream);

/* Workspace of moe_ffn_group_scaled: the activations between its two products.
 * One for some tokens serves fewer too.  Host-only; 0 for invalid dims. */
size_t moe_scaled_workspace_bytes(const moe_dims *dims);

/* moe_ffn_group in 8 bits, for the rows of local experts [e_first, e_first +
 * e_count):
 *   h[r]      = Q( silu(g) * u ), g = w_gate[e] x_row(r), u = w_up[e] x_row(r)
 *               (fp32 up to the quantisation)
 *   y_perm[r] = w_down[e] h[r]
 * x and sorted_slot as in moe_gemm_group_scaled with k = hidden; the weight
 * stacks as in moe_ffn_group; y_perm [R][H] of y_type (moe_combine takes
 * MOE_FP32).  ws: moe_scaled_workspace_bytes(dims) bytes, 16-byte aligned;
 * calls that may overlap on the GPU need their own.  Deterministic. */
moe_status moe_ffn_group_scaled(const moe_dims *dims, int32_t e_first, int32_t e_count,
                                const int32_t *offsets, const int32_t *sorted_slot,
                                const moe_e4m3 *x, const moe_scale *x_scales,
                                const moe_e4m3 *w_gate, const moe_scale *gate_scales,
                                const moe_e4m3 *w_up, const moe_scale *up_scales,
                                const moe_e4m3 *w_down, const moe_scale *down_scales,
                                void *y_perm, int32_t y_type, void *ws, size_t ws_bytes,
                                void *stream);

/* moe_combine over rows of either type: y_perm [R][H] of y_type.  The terms,
 * their order and y are moe_combine's (bf16 rows are widened exactly). */
moe_status moe_combine_rows(const moe_dims *dims, int32_t e_first, int32_t e_count,
                            const void *y_perm, int32_t y_type, const int32_t *topk_ids,
                            const int32_t *slot_row, const float *topk_w, float *y,
                            int32_t accumulate, void *stream);

/* A layer's quantised weights (moe_quant_weights): experts gate, up [EL][I][H]
 * and down [EL][H][I], shared gate, up [Is][H] and down [H][Is] (NULL without
 * shared experts).  The struct is host memory; its pointers are device ones. */
typedef struct {
    const moe_e4m3 *gate;
    const moe_scale *gate_scales;
    const moe_e4m3 *up;
    const moe_scale *up_scales;
    const moe_e4m3 *down;
    const moe_scale *down_scales;
    const moe_e4m3 *shared_gate;
    const moe_scale *shared_gate_scales;
    const moe_e4m3 *shared_up;
    const moe_scale *shared_up_scales;
    const moe_e4m3 *shared_down;
    const moe_scale *shared_down_scales;
} moe_scaled_weights;

/* Workspace of moe_forward_scaled; one for some tokens serves fewer too.
 * Host-only; 0 for invalid dims. */
size_t moe_forward_scaled_bytes(const moe_dims *dims);

/* The MoE layer in 8 bits, from the block's input to its output:
 *   moe_norm_quant (total = bf16(x + residual), the normalised rows in bf16
 *   and quantised) -> moe_route on the bf16 rows -> dispatch -> the shared
 *   experts (if any) and moe_ffn_group_scaled on the quantised rows, the
 *   routed rows in bf16 -> combine into y [T][H] fp32.
 * The next layer takes y and total as its x (MOE_FP32) and residual.
 * norm_weight NULL: x is bf16 rows that are normalised already (moe_ffn_forward's
 * input); then residual and total must be NULL and eps is not read.
 * topk_ids, topk_w, counts: optional outputs.  ws: moe_forward_scaled_bytes(dims)
 * bytes, 16-byte aligned.  Every step runs on `stream`; the call allocates
 * nothing, never synchronises and can be captured; calls that may overlap on
 * the GPU need a workspace each. */
moe_status moe_forward_scaled(const moe_dims *dims, const void *x, int32_t x_type,
                              const moe_bf16 *residual, const moe_bf16 *norm_weight, float eps,
                              moe_bf16 *total, const float *w_router, const float *bias,
                              const moe_scaled_weights *weights, float *y, int32_t *topk_ids,
                              float *topk_w, int32_t *counts, void *ws, size_t ws_bytes,
                              void *stream);

/* ---- Routing by scores ---------------------------------------------------
 * moe_route's softmax top-k with the rules that larger layers are trained with:
 * sigmoid scores, a bias that balances the experts' load, experts in groups.
 * The router's product comes from moe_route_logits or elsewhere. */

enum { MOE_SCORE_SOFTMAX = 0, MOE_SCORE_SIGMOID = 1 };
enum { MOE_GROUP_MAX = 0, MOE_GROUP_TOP_TWO = 1 };
/* Host memory. */
typedef struct {
    int32_t score;       /* MOE_SCORE_SOFTMAX (over all experts) or _SIGMOID */
    int32_t groups;      /* G, dividing the experts; group g holds experts
                            [g E/G, (g + 1) E/G).  1: no groups */
    int32_t top_groups;  /* groups kept, 1 .. G; they have to hold top_k experts */
    int32_t group_score; /* a group's value: its best choice (MOE_GROUP_MAX) or the
                            sum of its two best (MOE_GROUP_TOP_TWO) */
    float scale;         /* factor of the weights, finite */
} moe_routing;

/* The router's logits z[t][e], moe_route's chain without a bias: x [T][H] bf16,
 * 16-byte aligned; w_router [E][H] fp32; logits [T][E] fp32. */
moe_status moe_route_logits(const moe_dims *dims, const moe_bf16 *x, const float *w_router,
                            float *logits, void *stream);

/* Experts and weights from logits [T][E] of logits_type (MOE_FP32 or MOE_BF16).
 * For each token, with bias [E] fp32 or NULL:
 *   s[e] = softmax(z)[e] over all experts, or 1 / (1 + exp(-z[e]))
 *   c[e] = s[e] + bias[e]             the choice (without a bias its order is z's)
 *   groups: the top_groups largest values (descending; ties: the lower group)
 *   topk_ids[t][0..k)  the k largest c of the groups kept, by (c descending, e
 *                      ascending)
 *   topk_w[t][j] = scale * s[id_j], with dims->renormalize scale * s[id_j] / sum
 *                  of the chosen s
 * Choices and group values are compared in 64 bits, weights computed in 64 bits (the
 * softmax's sum over all experts to 2^-37) and rounded to fp32; choices nearer to each other than 2^-50 may come in either
 * order.  An expert is switched off by a logit of -inf, or by a choice of -inf or
 * NaN (its bias'); it is never chosen.  Where fewer than k are left, the last ids
 * are -1 with weight 0 (moe_permute and moe_combine pass over them).  A token with
 * a NaN logit, or with +inf under softmax, has NaN weights, and its experts are
 * the k largest logits of all groups, a NaN as the largest.
 * dims gives tokens (fewer than 2^28), experts, top_k and renormalize; the rest is
 * not used. */
moe_status moe_route_scores(const moe_dims *dims, const moe_routing *routing, const void *logits,
                            int32_t logits_type, const float *bias, int32_t *topk_ids,
                            float *topk_w, void *stream);

/* Its gradient: dlogits [T][E] (of logits_type, every element written) from the
 * chosen topk_ids and dtopk_w [T][k], the gradient of topk_w.  The choice itself
 * has none, nor has the bias.  An id outside [0, E) takes no part; one that is
 * named twice has the sum of both.  With dims->renormalize or sigmoid scores the
 * logits of experts that were not chosen are not read and get 0. */
moe_status moe_route_scores_backward(const moe_dims *dims, const moe_routing *routing,
                                     const void *logits, int32_t logits_type,
                                     const int32_t *topk_ids, const float *dtopk_w, void *dlogits,
                                     void *stream);

/* ---- Low-rank adapters ---------------------------------------------------
 * A batch holds rows of several requests, each with an adapter of its own beside
 * a projection y = x W^T that all share.  An adapter is a pair A [rank][k],
 * B [n][rank] and a scale.  Rows are ordered by adapter as tokens are by expert:
 * moe_permute with tokens = rows, experts = count, top_k = 1 and the rows'
 * adapters as topk_ids (-1: none) gives offsets, sorted_slot and slot_row, once
 * for all projections of a batch.
 * Tensors must be 16-byte aligned, scale and index tensors 4-byte aligned.  The
 * calls allocate nothing, never synchronise and can be captured; a workspace
 * (16-byte aligned) serves one call at a time, and one for some rows serves fewer
 * too.  Outputs overlap no input but base and dx_base as said below.  Results are
 * deterministic; their bits depend on rows, count and widths (which pick the tiles),
 * not on the other rows' adapters.  An infinity stays in the outputs that its formula
 * reaches, as an infinity or NaN.  Offsets ascend (where they do not, nothing outside the
 * outputs is touched); those outside [0, rows] are cut to it.  Entries of sorted_slot
 * outside [0, rows) are passed over.  A row whose place in slot_row has another entry, or
 * lies in no adapter's range, is a row without an adapter.
 * Rows and widths that need 2^32 lanes in a launch (some 5 10^10 values of y) are
 * MOE_ERR_UNSUPPORTED. */

/* Host memory; its pointers are device ones. */
typedef struct {
    int32_t count;      /* adapters, 1 .. 256 */
    int32_t rank;       /* a multiple of 8 up to 256; adapters of a smaller rank are
                           padded with zeros */
    int32_t n, k;       /* widths of the projection's output and input, multiples of
                           64 up to 2^20 */
    const moe_bf16 *a;  /* [count][rank][k] */
    const moe_bf16 *b;  /* [count][n][rank] */
    const float *scale; /* [count], or NULL for 1 */
} moe_adapters;

/* Workspace of moe_adapter_rows.  Host-only; 0 for invalid arguments. */
size_t moe_adapter_workspace_bytes(int64_t rows, const moe_adapters *adapters);

/* y[r] = base[r] + scale[e] * B[e] (A[e] x[r]) for every row r with an adapter e,
 * y[r] = base[r] for the others.  x [rows][k] bf16; base and y [rows][n] of y_type
 * (MOE_BF16 or MOE_FP32).  base may be y itself (the projection's output; rows
 * without an adapter are then not touched and slot_row may be NULL), or NULL for
 * zeros.  A x is held in fp32 and multiplied in its 24 bits, whatever y's type; so is
 * B^T dy below. */
moe_status moe_adapter_rows(int64_t rows, const moe_adapters *adapters, const int32_t *offsets,
                            const int32_t *sorted_slot, const int32_t *slot_row,
                            const moe_bf16 *x, const void *base, void *y, int32_t y_type, void *ws,
                            size_t ws_bytes, void *stream);

/* Workspace of moe_adapter_backward, no less than moe_adapter_rows': one serves both.
 * Host-only; 0 for invalid arguments. */
size_t moe_adapter_backward_bytes(int64_t rows, const moe_adapters *adapters);

/* Its gradient from dy [rows][n] bf16, the gradient of y (base's is dy itself):
 *   dx[r] = dx_base[r] + scale[e] * A[e]^T (B[e]^T dy[r])
 *   da[e] (+)= scale[e] * sum over e's rows of (B[e]^T dy[r]) x[r]^T
 *   db[e] (+)= scale[e] * sum over e's rows of dy[r] (A[e] x[r])^T
 * dx, dx_base [rows][k] of dx_type; dx_base (what the projection's own gradient
 * left) may be dx itself or NULL, as base above.  da [count][rank][k], db
 * [count][n][rank] fp32, added to what they hold with accumulate = 1; else
 * adapters without rows get zeros.  dx, or da and db together, may be NULL;
 * without da and db x is not read. */
moe_status moe_adapter_backward(int64_t rows, const moe_adapters *adapters,
                                const int32_t *offsets, const int32_t *sorted_slot,
                                const int32_t *slot_row, const moe_bf16 *x, const moe_bf16 *dy,
                                const void *dx_base, void *dx, int32_t dx_type, float *da,
                                float *db, int32_t accumulate, void *ws, size_t ws_bytes,
                                void *stream);

const char *moe_status_string(moe_status s);
const char *moe_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* MOE_H */
