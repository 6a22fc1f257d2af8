/*
 * seg_attn.h - C ABI of the segment-level causal attention library for NVIDIA B200 (sm_100a).
 *
 * The operation (names follow the paper; its total length T is `L` here, its tail length M is `T`):
 * a sequence of L positions is cut into non-overlapping segments of constant length S
 * (Section 3.1 "Setup", Section 3.5).  Every head runs scaled dot-product attention
 * softmax(Q K^T * sm_scale + mask) V (Appendix C, Eq. "attn") over a per-segment context
 * (Appendix C, Eq. "ctx"):
 *   - its own segment, causally (a query sees positions up to and including itself);
 *   - the carried KV tail: the last T key/value positions of the immediately preceding
 *     segment, the only differentiable cross-segment state (Section 3.4, "Local Continuity
 *     Channel"); the first segment has no carried state (Section 3.1, C_0 empty);
 *   - for KV heads of class SEGATTN_HEAD_PAST in `head_past_mask`, additionally every older
 *     key/value, read forward-only: stop-gradient, no gradient reaches those K/V (Definition 3.2;
 *     Section 3.4, "Long-Range Channel"; Appendix B, Lemma B.1);
 *   - KV heads of class SEGATTN_HEAD_OWN read their own segment and nothing else: the context of
 *     a long-range head in a layer that is not a long-range layer (Appendix C, Eq. "ctx", third
 *     case).
 * With global positions p (query) and j (key), i = p / S and a_i = max(0, i*S - T):
 *     visible(p, j, c) <=> lo_c(p) <= j <= p,  lo_c(p) = a_i (LOCAL), 0 (PAST), i*S (OWN)
 *     diff(p, j, c)    <=> max(lo_c(p), a_i) <= j <= p   (reads that carry gradient into K/V)
 * With seg_attn_params.seg_starts the segments have the lengths the caller gives instead of S: i is the
 * segment that holds p, i*S becomes its start s_i, and a_i = max(s_{i-1}, s_i - T) (the carried tail of a
 * segment shorter than T is the whole segment).
 * Query head h uses KV head c = h / (Hq / Hkv).
 *
 * Conventions that hold for every entry point unless it says otherwise:
 *   - Tensor pointers are DEVICE pointers owned by the caller; the library never frees or
 *     reallocates them.  Q, O, dO, dQ are bf16 [B][Lq][Hq][d]; K, V, dK, dV are bf16
 *     [B][kv_len][Hkv][d]; addressing is by the element strides in seg_attn_params (the last
 *     dimension is contiguous).  LSE is fp32, contiguous [B][Hq][Lq].
 *   - `head_past_mask` is a HOST array of Hkv bytes, one head class per KV head (0 = local,
 *     1 = past access, 2 = own segment only; any other value is SEGATTN_ERR_INVALID); it is read
 *     before the call returns.
 *   - `stream` is a cudaStream_t passed as void*.  Work is enqueued on it; no entry point
 *     synchronises the device except where stated.
 *   - Errors are return codes.  Arguments are validated on the host before anything is
 *     launched: SEGATTN_ERR_INVALID, _UNSUPPORTED_ARCH, _WORKSPACE and _TOO_LARGE mean that nothing
 *     was enqueued and the outputs are untouched.  SEGATTN_ERR_CUDA can also come from a launch or
 *     copy in the middle of a call's sequence (a backward is three kernels, the host-buffer step
 *     and the streamed prefill several launches and copies): what was enqueued before it still
 *     runs, so treat the outputs, and for the streamed prefill the handle's state, as undefined.
 *   - The kernels share a device status per process (see seg_attn_poll_status).  Once a bounded
 *     wait has run out, later kernels give up their waits early too, so outputs enqueued after
 *     that are undefined until seg_attn_poll_status has been called, which reads and clears it.
 *     An input that a kernel refused (an index or a length out of range) is recorded there as
 *     well and touches no other kernel.
 *   - Base pointers must be 16-byte aligned and every stride a multiple of 8 elements
 *     (tiles are moved by TMA).  d is 64 or 128.  0 <= T <= S.  Any Lq, kv_len >= 0.
 *   - Arithmetic: bf16 inputs, fp32 accumulation on the tensor cores, fp32 softmax
 *     statistics; P (and dS) are rounded to bf16 before the second product; outputs are
 *     rounded to bf16 (round-to-nearest-even).  A query row with no visible key present
 *     (possible only when kv_len does not reach it) yields O = 0, LSE = -inf.
 */
#ifndef SEG_ATTN_H_
#define SEG_ATTN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SEGATTN_OK = 0,
    SEGATTN_ERR_INVALID = 1,          /* bad shape, stride, alignment, null pointer, T > S, unsupported d */
    SEGATTN_ERR_UNSUPPORTED_ARCH = 2, /* the current device is not compute capability 10.x */
    SEGATTN_ERR_CUDA = 3,             /* a CUDA runtime/driver call failed; see seg_attn_last_cuda_error() */
    SEGATTN_ERR_TIMEOUT = 4,          /* a bounded wait inside a kernel expired (see seg_attn_poll_status) */
    SEGATTN_ERR_WORKSPACE = 5,        /* workspace/state buffer missing, misaligned or too small */
    SEGATTN_ERR_TOO_LARGE = 6         /* problem exceeds the fixed scratch of seg_attn_bwd_static */
} segattn_status;

/* Head classes, the entries of `head_past_mask` (Appendix C, Eq. "ctx"). */
#define SEGATTN_HEAD_LOCAL 0 /* own segment + carried tail, both differentiable */
#define SEGATTN_HEAD_PAST 1  /* own segment + carried tail + every older position (forward-only) */
#define SEGATTN_HEAD_OWN 2   /* own segment only */

/* seg_attn_params.flags, bit 0: for flagged KV heads the reads of the carried tail are stop-gradient
 * too, i.e. diff(p, j) <=> i*S <= j <= p for them.  This is the literal reading of Appendix C,
 * Eq. "ctx", where only local heads build and read the differentiable carried state and long-range
 * heads see their prefix forward-only.  The forward is the same in both readings; only the set of
 * (query, key) pairs that feed dK/dV changes. */
#define SEGATTN_FLAG_FLAGGED_TAIL_SG 1

typedef struct {
    int32_t B;       /* batch */
    int32_t Lq;      /* number of query rows per batch element */
    int32_t kv_len;  /* number of key/value rows present per batch element */
    int32_t Hq;      /* query heads */
    int32_t Hkv;     /* key/value heads; Hq % Hkv == 0; at most 64 */
    int32_t d;       /* head dimension: 64 or 128 */
    int32_t S;       /* segment length, >= 1 */
    int32_t T;       /* carried tail length, 0 <= T <= S */
    int32_t q_pos0;  /* global position of query row 0 (0 for a whole sequence; i*S when streaming) */
    int32_t kv_pos0; /* global position of key row 0 (may be negative: rows before position 0 are never visible) */
    float sm_scale;  /* softmax scale; the paper uses 1/sqrt(d) */
    int32_t flags;   /* bit set of SEGATTN_FLAG_*; 0 for the default semantics */
    int32_t detach_before; /* backward only: keys at global positions below this are read forward-only
                            * (no dK/dV from them, and their dK/dV rows come out zero): the boundary
                            * state of a truncated chain enters as a constant (K-truncated objective,
                            * Eq. "truncated-base").  A window of K+1 segments passes the position of
                            * its first segment.  0: none.  Must be >= 0. */
    int64_t q_stride[3]; /* element strides of Q (and dQ) for (batch, position, head) */
    int64_t k_stride[3]; /* element strides of K (and dK) */
    int64_t v_stride[3]; /* element strides of V (and dV) */
    int64_t o_stride[3]; /* element strides of O (and dO) */
    const int32_t* seg_starts; /* NULL: segments of constant length S.  Else a HOST array of n_segs ascending global
                                * positions, the first 0: segment i is [seg_starts[i], seg_starts[i+1]) and the last one
                                * is open-ended (segments of lengths m_i, Section 3.1).  S is then ignored, T may exceed
                                * a segment's length (the carried tail of a short segment is the whole segment).  The
                                * streamed prefill driver takes its lengths step by step instead (seg_prefill_step_len).  Read before the call returns. */
    int32_t n_segs;            /* 1 .. 256 when seg_starts is given */
} seg_attn_params;

/* Bytes of device scratch a call needs (is_bwd = 0: forward, none today; 1: backward, the
 * fp32 row dots D[B][Hq][Lq], rounded up to 256).  Returns 0 for invalid params. */
size_t seg_attn_workspace_bytes(const seg_attn_params* p, int is_bwd);

/* Forward (Appendix C, Eqs. "attn" and "ctx"; mask as stated at the top of this file).
 * O[b][r][h][:] = sum_j P_j V_j and LSE[b][h][r] = ln sum_j exp(sm_scale * <q,k_j>) over the
 * visible j (natural logarithm of the scaled scores).  Fully overwrites O and LSE.
 * `workspace` may be NULL (size 0). */
segattn_status seg_attn_fwd(const seg_attn_params* p, const void* Q, const void* K, const void* V,
                            const uint8_t* head_past_mask, void* O, float* LSE,
                            void* workspace, size_t workspace_bytes, void* stream);

/* Backward: the vector-Jacobian product of the forward for the cotangent dO (softmax VJP;
 * stop-gradient per Definition 3.2 and Lemma B.1; the tail as sole differentiable
 * cross-segment state per Section 3.4; one-transition reach of the K=1 discussion after
 * Definition 3.2).  With P = exp(s - LSE), D = <dO,O>, dS = P * (dO V^T - D):
 *   dQ_p = sm_scale * sum over visible j of dS_pj K_j          (stop-gradient keys included:
 *                                                               sg cuts the K/V side only)
 *   dK_j = sm_scale * sum over p with diff(p,j) of dS_pj Q_p,  dV_j = sum over the same p of P_pj dO_p
 * summed over the query heads of the KV head.  A key position thus receives gradient only
 * from queries of its own segment and, if it lies in the last T positions, of the next one.
 * O and LSE must be the forward's results for the same inputs.  dQ, dK, dV are fully
 * overwritten (no pre-zeroing).  `workspace` must hold seg_attn_workspace_bytes(p, 1) bytes,
 * 256-byte aligned; it is scratch, dead after the enqueued work has run. */
segattn_status seg_attn_bwd(const seg_attn_params* p, const void* Q, const void* K, const void* V,
                            const void* O, const float* LSE, const void* dO,
                            const uint8_t* head_past_mask, void* dQ, void* dK, void* dV,
                            void* workspace, size_t workspace_bytes, void* stream);

/* Backward for callers that cannot allocate device memory (the paper has no counterpart; this is
 * a packaging variant of seg_attn_bwd, not another operation).  Some hosts of this library may
 * not call cudaMalloc where the backward runs - a serving or training loop whose memory pool is
 * sized at start-up and frozen, a plugin that is handed tensors but no allocator, code that must
 * not trigger the implicit device synchronisation an allocation can cause - and so cannot provide
 * the `workspace` seg_attn_bwd asks for.  This entry point takes
 * no workspace: the fp32 row dots D live in a fixed array inside the library's device image,
 * SEG_ATTN_STATIC_MAX_ROWS floats (4 MiB) that every GPU loading the library holds until the
 * process exits.  It calls no cudaMalloc / cudaFree and no allocating library routine.
 *   - Same arguments, results and error codes as seg_attn_bwd otherwise (same kernels).
 *   - Problems with B * Hq * Lq > SEG_ATTN_STATIC_MAX_ROWS are rejected with
 *     SEGATTN_ERR_TOO_LARGE before anything is launched; use seg_attn_bwd with a workspace.
 *   - The first call on each device looks up the array's device address (one
 *     cudaGetSymbolAddress, with that device current).  Make that first call outside any stream
 *     capture.
 *   - All calls on a device share the one array and it keeps the previous call's contents (every
 *     element a call reads it has written first, so nothing needs clearing).  Two calls whose
 *     work overlaps on the GPU - different streams, or threads - race on it: serialise them. */
#define SEG_ATTN_STATIC_MAX_ROWS (1 << 20)
segattn_status seg_attn_bwd_static(const seg_attn_params* p, const void* Q, const void* K, const void* V,
                                   const void* O, const float* LSE, const void* dO,
                                   const uint8_t* head_past_mask, void* dQ, void* dK, void* dV, void* stream);

/* ---- Streamed prefill: the segment recurrence (C_i, o_i) = F(x_i, C_{i-1}, R_{i-1}) of
 * Definition 3.1 restricted to attention, with memory bounded as in Section 3.5 "Memory
 * Complexity": flagged KV heads keep their whole key/value history (the append-only
 * past-only pool of Section 3.4), the others keep only the T-position tail.
 *
 * The caller provides one device buffer for all persistent state.  In `p`, Lq is the
 * segment length fed per step (must equal S; seg_prefill_step_len feeds shorter ones), kv_len is the
 * maximum total length the pool must hold, q_pos0/kv_pos0 are ignored, and the Q/O strides describe the per-step
 * Q/O segment tensors [B][S][Hq][d], the K/V strides the per-step K/V segment tensors
 * [B][S][Hkv][d].  The handle itself is a small host object (malloc'd by create, freed by
 * destroy). */
typedef struct seg_prefill_handle seg_prefill_handle;

size_t seg_prefill_state_bytes(const seg_attn_params* p, const uint8_t* head_past_mask);
segattn_status seg_prefill_create(const seg_attn_params* p, const uint8_t* head_past_mask,
                                  void* state_mem, size_t state_bytes, seg_prefill_handle** out);
/* Processes the next segment: appends its K/V to the retained state, writes O_seg
 * [B][S][Hq][d] and LSE_seg [B][Hq][S] (the same values the whole-sequence forward gives for
 * those rows), then rolls the tail.  Call once per segment, in order, on one stream. */
segattn_status seg_prefill_step(seg_prefill_handle* h, const void* Qseg, const void* Kseg, const void* Vseg,
                                void* Oseg, float* LSEseg, void* stream);
/* The same for a segment of Lseg rows, 1 <= Lseg <= S: segments of lengths m_i (Section 3.1 lets them differ), and
 * in particular a shorter last segment.  The segment tensors hold Lseg rows per batch element and are addressed with
 * the strides given at creation; LSE_seg is [B][Hq][Lseg].  The carried tail of a segment shorter than T is the whole
 * segment (never more than one segment back), as with seg_attn_params.seg_starts, whose whole-sequence forward this
 * reproduces row for row.  seg_prefill_step(h, ...) is seg_prefill_step_len(h, S, ...). */
segattn_status seg_prefill_step_len(seg_prefill_handle* h, int32_t Lseg, const void* Qseg, const void* Kseg,
                                    const void* Vseg, void* Oseg, float* LSEseg, void* stream);
/* Backward of the segment stepped last (the streamed form of training with truncation depth 1: a
 * segment is run forward, its loss is differentiated, and credit stops where the carried state
 * entered - definition of the K-truncated objective with K = 1).  Valid after seg_prefill_step and
 * before the next one; the state still holds what that step attended over.  Qseg, Oseg, dOseg and
 * dQseg hold the Lseg rows of that step per batch element ([B][S][Hq][d] for a full segment) with the strides
 * given at creation, LSEseg as returned by the step.
 * dKctx and dVctx are contiguous bf16 [B][T+S][Hkv][d]: the gradients of the key/value rows at
 * global positions [pos - T, pos + Lseg), pos the segment's start - the T positions in front of the segment, of
 * which the previous segment's carried tail (its last min(T, length) positions) can be non-zero, then the segment
 * itself; rows before position 0 and the S - Lseg rows after a shorter segment are zero.  Older rows of past-access
 * heads are read forward-only and get none.  The caller adds the first T rows to the previous segment's gradients.  `workspace`: DEVICE,
 * 256-byte aligned, at least seg_prefill_bwd_workspace_bytes(h) bytes.  SEGATTN_ERR_INVALID when no segment
 * has been stepped yet or a pointer is null or misaligned, SEGATTN_ERR_WORKSPACE for the workspace; the state
 * is not modified. */
size_t seg_prefill_bwd_workspace_bytes(const seg_prefill_handle* h);
segattn_status seg_prefill_step_bwd(seg_prefill_handle* h, const void* Qseg, const void* Oseg, const float* LSEseg,
                                    const void* dOseg, void* dQseg, void* dKctx, void* dVctx, void* workspace,
                                    size_t workspace_bytes, void* stream);
segattn_status seg_prefill_reset(seg_prefill_handle* h); /* back to segment 0; state contents become dead */
void seg_prefill_destroy(seg_prefill_handle* h);

/* ---- Context of a head that reads a retrieved prefix (Appendix C, Eq. "ctx", first case: a
 * long-range head in a long-range layer attends over [K_ret ; K_i], R retrieved rows followed by
 * its own segment; Appendix D fixes R positions per head).  Given the R positions, builds
 *     K_ctx[b][r][c][:]     = K_pool[b][idx[b][c][r]][c][:]      0 <= r < R
 *     K_ctx[b][R + t][c][:] = K_seg[b][t][c][:]                  0 <= t < Lseg
 * and V_ctx alike.  K_pool/V_pool are bf16 with element strides pool_stride (batch, position, head)
 * and pool_len positions; K_seg/V_seg likewise with seg_stride; K_ctx/V_ctx are contiguous
 * [B][R + Lseg][Hkv][d].  idx is a DEVICE array of int32, [B][Hkv][R].  All pointers 16-byte
 * aligned, strides multiples of 8.  An index outside [0, pool_len) is not read: its row is zero
 * and the next seg_attn_poll_status returns SEGATTN_ERR_INVALID.  The attention itself is the
 * existing entry points on the context: seg_attn_fwd / seg_attn_bwd with Lq = Lseg, kv_len = R + Lseg,
 * q_pos0 = R, kv_pos0 = 0, S = R + Lseg, T = 0, class 0 heads, and, in the backward,
 * detach_before = R (the retrieved rows are forward-only: Definition 3.2, Lemma B.1); rows
 * [R, R + Lseg) of the dK/dV it returns are the segment's gradients.  The R positions come from the
 * caller or from seg_retrieval_select below. */
segattn_status seg_attn_gather_context(int32_t B, int32_t Hkv, int32_t d, int32_t R, int32_t Lseg, int32_t pool_len,
                                       const void* K_pool, const void* V_pool, const int64_t pool_stride[3],
                                       const void* K_seg, const void* V_seg, const int64_t seg_stride[3],
                                       const int32_t* idx, void* K_ctx, void* V_ctx, void* stream);

/* ---- Selection step of the top-k retrieval operator (Appendix D): which R pool positions a head
 * retrieves.  The paper names the steps and states none of the constants, so all are parameters here,
 * and the tie and overflow rules are this library's (equal scores: lower position first; windows are
 * added best anchor first until R positions are chosen; a short set is padded with the earliest
 * positions not yet chosen).  Steps per (batch, KV head): (1) query summaries of the last Lq_last
 * queries of the previous segment - the mean over each sliding window [u*stride, u*stride + window)
 * and the mean over the last `tail` rows, averaged over the group's query heads; (2) dot-product
 * scores of every summary against every pool key; (3) the top_k keys per summary, deduplicated;
 * (4) the n_anchors candidates of highest score; (5) positions anchor - off_lo .. anchor + off_hi,
 * padded to exactly R, ascending.  Arithmetic is fp32 with separately rounded products and
 * sequential sums, so the choice is reproducible bit for bit.  Q_last is bf16, contiguous
 * [B][Lq_last][Hq][d]; K_pool bf16 with element strides pool_stride (batch, position, head) and P
 * positions; idx (DEVICE, int32 [B][Hkv][R]) is what seg_attn_gather_context takes.  Limits: at most
 * 16 summaries, summaries * top_k <= 1024, R <= P, top_k <= P.  `workspace`: DEVICE, 256-byte aligned,
 * seg_retrieval_workspace_bytes(...) bytes (0 = invalid parameters).  Returns SEGATTN_ERR_INVALID for
 * parameters outside these limits or misaligned pointers and SEGATTN_ERR_WORKSPACE for a missing, misaligned
 * or short workspace, before anything is launched; the workspace's contents are scratch. */
typedef struct {
    int32_t Lq_last, window, stride, tail; /* query summaries */
    int32_t top_k, n_anchors;              /* candidates per summary; anchors kept */
    int32_t off_lo, off_hi;                /* window around an anchor */
    int32_t R;                             /* positions returned per head */
} seg_retrieval_params;
size_t seg_retrieval_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t d, int32_t P, const seg_retrieval_params* r);
segattn_status seg_retrieval_select(int32_t B, int32_t Hq, int32_t Hkv, int32_t d, int32_t P, const void* Q_last,
                                    const void* K_pool, const int64_t pool_stride[3], const seg_retrieval_params* r,
                                    int32_t* idx, void* workspace, size_t workspace_bytes, void* stream);

/* ---- RoPE re-indexing for prefix concatenation (Section 3.4, paragraph of that name; Appendix E).  When a
 * prefix of P key/value rows - the carried tail (P = T) or the retrieved rows (P = R) - is put in front of a
 * segment of m rows, the prefix keys are rotated with positions 0 .. P-1 and the segment's queries and keys with
 * positions P .. P+m-1; values are not rotated.  (For the carried tail this equals rotating everything at its
 * global position, since scores depend on position differences only; for retrieved rows it does not, which is
 * why the pool must hold keys BEFORE rotation.)  "Standard RoPE" is read as the rotation of the pairs
 * (x[i], x[i + d/2]), i < d/2, by the angle pos * base^(-2i/d):
 *     y[i] = x[i] cos a - x[i + d/2] sin a,   y[i + d/2] = x[i] sin a + x[i + d/2] cos a.
 * The angles' cosines and sines come from a table the caller keeps on the device:
 *   seg_rope_table_bytes   bytes of a table for positions [0, n_pos) (0: invalid d or n_pos; n_pos <= 2^24);
 *   seg_rope_table         fills `table` (DEVICE, 16-byte aligned, fp32 [n_pos][d/2][2] = (cos, sin)); the angles are
 *                          formed and their cosines and sines taken in double precision, then rounded to fp32;
 *   seg_rope_apply         Y[b][r][h][:] = Rot(pos0 + r) X[b][r][h][:] for bf16 X, Y [B][L][H][d] with the element
 *                          strides given (batch, row, head; multiples of 8; Y may be X); inverse != 0 applies the
 *                          transposed rotation, which maps a gradient with respect to the rotated tensor back to one
 *                          with respect to the unrotated tensor (dQ of the segment, and rows [R, R+m) of dK).
 *                          Arithmetic fp32, output rounded to bf16.  pos0 + L <= n_pos.
 *   seg_attn_gather_context_rope   seg_attn_gather_context with the re-indexed rotation applied to the keys while
 *                          they are copied: K_ctx[b][r][c] = Rot(r) K_pool[b][idx[b][c][r]][c] for r < R,
 *                          K_ctx[b][R + t][c] = Rot(R + t) K_seg[b][t][c]; V_ctx is the plain copy.  Same arguments,
 *                          limits and error behaviour as seg_attn_gather_context; R + Lseg <= n_pos.  The segment's
 *                          queries are rotated by seg_rope_apply with pos0 = R.
 * All four validate their arguments on the host (SEGATTN_ERR_INVALID) and enqueue one kernel on `stream`. */
size_t seg_rope_table_bytes(int32_t n_pos, int32_t d);
segattn_status seg_rope_table(int32_t n_pos, int32_t d, double base, float* table, void* stream);
segattn_status seg_rope_apply(int32_t B, int32_t L, int32_t H, int32_t d, const void* X, const int64_t x_stride[3],
                              void* Y, const int64_t y_stride[3], int32_t pos0, int32_t inverse, const float* table,
                              int32_t n_pos, void* stream);
segattn_status seg_attn_gather_context_rope(int32_t B, int32_t Hkv, int32_t d, int32_t R, int32_t Lseg, int32_t pool_len,
                                            const void* K_pool, const void* V_pool, const int64_t pool_stride[3],
                                            const void* K_seg, const void* V_seg, const int64_t seg_stride[3],
                                            const int32_t* idx, void* K_ctx, void* V_ctx, const float* table,
                                            int32_t n_pos, void* stream);

/* ---- Rotary positions in general form.  The paper's "standard RoPE" above rotates the whole head in the half pairing at
 * consecutive positions; models that are served through the paged cache below also come with neighbouring elements
 * paired, with only the first rot_dim elements of a head rotated, with frequencies scaled for contexts longer than the
 * trained one, and with rows at positions of their own.
 *   seg_rope_table_scaled  fills `table` (DEVICE, 16-byte aligned, fp32 [n_pos][rot_dim/2][2] = a (cos, sin)(pos w_i)) with
 *                          w_i = base^(-2i/rot_dim), a = amplitude, and by `kind`
 *                            SEGATTN_ROPE_PLAIN      w_i as it is;
 *                            SEGATTN_ROPE_LINEAR     w_i / factor (positions interpolated);
 *                            SEGATTN_ROPE_BY_PARTS   (1 - g_i) w_i / factor + g_i w_i with the ramp
 *                                                    g_i = clamp((t_i - turns_lo) / (turns_hi - turns_lo), 0, 1) over the
 *                                                    turns t_i = trained_len w_i / (2 pi) that pair i makes in the trained
 *                                                    length: slow pairs are interpolated, fast ones kept.
 *                          Angles, cosines and sines in double precision, rounded to fp32.  A table that seg_rope_table
 *                          filled serves as well (rot_dim = d).
 *   seg_rope_rotate        Y[b][r][h][:] = Rot(p) X[b][r][h][:] with p = positions[b*L + r] (DEVICE int32 [B][L]) or, where
 *                          `positions` is NULL, pos0 + r.  Pairs are (x[i], x[i + rot_dim/2]) for SEGATTN_ROPE_HALF and
 *                          (x[2i], x[2i+1]) for SEGATTN_ROPE_INTERLEAVED, i < rot_dim/2; elements from rot_dim on are
 *                          copied.  bf16, element strides (batch, row, head), multiples of 8; Y may be X (with its strides)
 *                          and may not overlap it otherwise.  inverse != 0 applies the transposed map (times the amplitude
 *                          again): the backward pass, which takes dY to dX.  fp32 arithmetic with separately rounded
 *                          products, one rounding to bf16.  A position outside [0, n_pos) is not looked up: its row comes
 *                          out zero and the next seg_attn_poll_status returns SEGATTN_ERR_INVALID.
 * d and rot_dim are multiples of 16, 16 <= rot_dim <= d <= 256, n_pos <= 2^24, B * L below 2^31, and
 * B * L * H * d at most 2^35. */
#define SEGATTN_ROPE_PLAIN 0
#define SEGATTN_ROPE_LINEAR 1
#define SEGATTN_ROPE_BY_PARTS 2
#define SEGATTN_ROPE_HALF 0
#define SEGATTN_ROPE_INTERLEAVED 1
typedef struct {
    int32_t kind;
    double base;                              /* > 1 */
    double factor;                            /* LINEAR, BY_PARTS: > 0 */
    double trained_len, turns_lo, turns_hi;   /* BY_PARTS: trained_len > 0, 0 <= turns_lo < turns_hi */
    double amplitude;                         /* > 0; 1 for a pure rotation */
} seg_rope_scaling;
segattn_status seg_rope_table_scaled(int32_t n_pos, int32_t rot_dim, const seg_rope_scaling* sc, float* table, void* stream);
segattn_status seg_rope_rotate(int32_t B, int32_t L, int32_t H, int32_t d, int32_t rot_dim, int32_t layout, const void* X,
                               const int64_t x_stride[3], void* Y, const int64_t y_stride[3], const int32_t* positions,
                               int32_t pos0, int32_t inverse, const float* table, int32_t n_pos, void* stream);

/* ---- Serving: a paged key/value cache, the attention of new tokens over it, and its eviction.  The paper stops at the
 * prefill; these continue it token by token under the same mask.  A sequence's rows lie in pages of page_size rows, slot j
 * in row j % page_size of page block_table[b][j / page_size]; a page that a call writes belongs to one sequence, one that
 * is only read may be shared (a common prefix).  kv_len[b] counts the rows
 * including the call's new ones: new row t of sequence b (t < q_len[b]) has slot kv_len[b] - q_len[b] + t and the global
 * position slot + pos_shift[b], where pos_shift counts the rows that evictions have taken out.
 * Everything the kernels read per sequence is in device memory, so a captured graph follows the lengths as they grow.
 * Numbers are checked where they are read: a page number outside [0, n_pages), a length outside [0, max_pages*page_size]
 * or a q_len outside [0, Lq] makes the next seg_attn_poll_status return SEGATTN_ERR_INVALID; such a page's rows are neither
 * read (they count as not visible) nor written.  Attention and eviction go on with such a length cut to its range (and a
 * negative pos_shift taken as 0); an append cuts nothing, it leaves out the rows that the numbers give no place. */
#define SEGATTN_KV_BF16 0
#define SEGATTN_KV_E4M3 1 /* 8-bit values, 1 + 4 + 3 bits, times a scale per KV head */
typedef struct {
    int32_t B, Hkv, d;           /* sequences, at most 65535; KV heads, at most 64; head dimension, 64 or 128 */
    int32_t dtype;               /* SEGATTN_KV_* */
    int32_t page_size, n_pages;  /* rows in a page, >= 1; pages in K and in V */
    int32_t max_pages;           /* entries of a sequence's row of the block table; max_pages*page_size <= 2^30 */
    int32_t table_stride;        /* elements between rows of the block table, >= max_pages */
    void *K, *V;                 /* DEVICE, 16-byte aligned */
    int64_t k_stride[3], v_stride[3]; /* elements, for (page, row, head); multiples of 16 bytes; the last dimension is contiguous */
    const float *k_scale, *v_scale;   /* E4M3: DEVICE [Hkv], > 0, finite, with finite inverses (not checked);
                                       * an eviction, which moves rows as they are, needs none.  BF16: NULL */
    const int32_t* block_table;  /* DEVICE [B][max_pages]; entries past a sequence's last page are not read */
    const int32_t* kv_len;       /* DEVICE [B] */
    const int32_t* q_len;        /* DEVICE [B], new rows of each sequence, or NULL: Lq for all */
    const int32_t* pos_shift;    /* DEVICE [B], >= 0, or NULL: 0 for all */
} seg_kv_cache;

/* Writes the new rows K_new, V_new (bf16 [B][Lq][Hkv][d]) into the cache.  With `table` (see seg_rope_rotate; rot_dim, layout
 * and n_pos as there) the keys are rotated by their positions first, and so are the queries Q (bf16 [B][Lq][Hq][d], may
 * be NULL; Q_out may be Q) into Q_out; without a table keys are copied and Q must be NULL.  An e4m3 cache stores x times
 * the scale's inverse (both rounded to fp32), rounded to nearest even and saturated at +-448.  Rows t >= q_len[b] are neither read nor written.  Not written
 * either (status as above) are a new row whose slot kv_len[b] - q_len[b] + t lies outside [0, max_pages*page_size) or whose
 * position is not in the table, and the rows of a sequence whose q_len is out of range or, with a table, whose pos_shift is negative.  One kernel;
 * B * Lq below 2^31, and B * Lq * (Hq + 2 Hkv) * d at most 2^35. */
segattn_status seg_kv_append(const seg_kv_cache* c, int32_t Lq, const void* K_new, const int64_t kn_stride[3],
                             const void* V_new, const int64_t vn_stride[3], int32_t Hq, const void* Q,
                             const int64_t q_stride[3], void* Q_out, const int64_t qo_stride[3], const float* table,
                             int32_t n_pos, int32_t rot_dim, int32_t layout, void* stream);

/* Attention of the new rows over the cache (which already holds them): for row t of sequence b at slot e and position p,
 * and KV head h of class head_past_mask[h] (HOST array, read before the call returns), slot j is visible when
 * lo <= j <= e, lo = 0 (PAST), max(0, max(0, i S - T) - pos_shift) (LOCAL), max(0, i S - pos_shift) (OWN), i = p / S: the
 * mask of seg_attn_fwd on what the cache retains.  (After an eviction that kept at least the last S + T rows, local and
 * own-segment heads see what they would have seen without it.)  S = 2^30 makes every head plainly causal.
 *   O bf16 [B][Lq][Hq][d], LSE fp32 contiguous [B][Hq][Lq] as in seg_attn_fwd; rows t >= q_len[b] are left as they were; a
 *   row that sees no key gets O = 0, LSE = -inf.  A row's result does not depend on rows it does not see, whatever they hold.
 *   O may be Q, with its strides (a view that shares some of its elements is SEGATTN_ERR_INVALID); not with weights_out and
 *   more than 32 rows to a KV head (Hq/Hkv * Lq) of a bf16 cache, whose weights read Q once more (SEGATTN_ERR_INVALID).
 *   weights_out (NULL: none): fp32 contiguous [B][Hkv][W]; for every slot j < kv_len[b] of sequences with new rows
 *     weights_out[b][h][j] = (weights_in ? weights_in[b][h][j] : 0) + sum over the new rows and the query heads of h of the
 *     row's attention weight on j;
 *   other entries are left as they were.  weights_in may be weights_out.  W >= max_pages*page_size.
 * SEGATTN_ERR_INVALID also where B * Hkv * (Hq/Hkv*Lq/8 rounded up) * (max_pages*page_size/64 + 3) passes 2^30.
 * `workspace`: DEVICE, 256-byte aligned, seg_attn_decode_workspace_bytes(...) bytes, scratch (0 = invalid parameters); calls
 * that may run at the same time, captured ones too, need one each.  Results do not change from run to run.
 * fp32 scores, statistics and accumulators; the weights are rounded to 16 bits before the product with V (bf16, or fp16
 * beside an e4m3 cache: half a step, 2^-11, down to 2^-27 of the row's largest weight, and 2^-38 of that one below). */
size_t seg_attn_decode_workspace_bytes(const seg_kv_cache* c, int32_t Lq, int32_t Hq, int32_t with_weights);
segattn_status seg_attn_decode(const seg_kv_cache* c, int32_t Lq, int32_t Hq, int32_t S, int32_t T, float sm_scale,
                               const uint8_t* head_past_mask, const void* Q, const int64_t q_stride[3], void* O,
                               const int64_t o_stride[3], float* LSE, const float* weights_in, float* weights_out, int32_t W,
                               void* workspace, size_t workspace_bytes, void* stream);

/* Eviction by accumulated attention weight.  With n = kv_len[b] and budget = sink + recent + heavy: a sequence of n <= budget
 * keeps all its rows; otherwise each KV head keeps the first `sink` slots, the last `recent` ones, and of those between them
 * the `heavy` ones of largest weights[b][h][.] (fp32 contiguous [B][Hkv][W]; equal weights: lower slot first; NaN ranks
 * lowest).  The kept rows of K and V are copied in ascending order to slots 0, 1, ... of the pages that dst_table (DEVICE
 * [B][dst_max_pages], row stride dst_stride) names in the same K and V, which must be none of the sequence's present pages.
 *   idx          int32 contiguous [B][Hkv][budget]: the slots kept, ascending, then -1
 *   kv_len_out   int32 [B]: min(n, budget);  pos_shift_out int32 [B]: pos_shift + n - kv_len_out.  Either may be the cache's own.
 *   weights_out  fp32 contiguous [B][Hkv][W]: the kept slots' weights, then zeros; may not overlap weights
 * W >= max_pages*page_size, 1 <= budget <= dst_max_pages*page_size and budget <= W.  q_len is ignored.  Two kernels, no
 * workspace. */
segattn_status seg_kv_evict(const seg_kv_cache* c, const float* weights, int32_t W, int32_t sink, int32_t recent,
                            int32_t heavy, const int32_t* dst_table, int32_t dst_max_pages, int32_t dst_stride, int32_t* idx,
                            int32_t* kv_len_out, int32_t* pos_shift_out, float* weights_out, void* stream);

/* ---- Pages from the lengths that requests ask for, on the device: so that a decoding loop admits, grows, rolls back and ends its
 * sequences without the host.  want (DEVICE int32 [B]) is the length every sequence is to have; with n = kv_len[b] and pages of
 * page_size rows, a sequence that shrinks (0: it is done) gives the pages behind its new length back to the list free_pages (DEVICE
 * int32 [n_pages], the first *free_count of them free), and one that grows takes pages from the list's end, after all that is given
 * back, in the order of b: the first that does not find enough of them, and every later one that needs any, stays as it is (what it
 * already has included), to be asked for again.  A page on the list and in a table belongs to one sequence: pages that sequences
 * share are not given back by a call of this kind.
 *   block_table     [B][max_pages], row stride table_stride: new entries are written, others are left as they were
 *   kv_len_out      int32 [B]: want[b] or, where the sequence stayed as it is, kv_len[b]; may be kv_len or want
 *   free_count_out  int32 [1]; may be free_count (else it is written for B = 0 too)
 *   q_len           int32 [B]: max(0, kv_len_out - kv_len), the new rows as the calls below take them
 *   slots           int64 [B][Lq]: page * page_size + row of new row t, -1 from q_len[b] on (8-byte aligned); for kernels that keep something
 *                   of their own beside the cache's rows: no call here needs it
 *   positions       int32 [B][Lq]: kv_len + t + pos_shift (NULL: 0) of new row t, 0 from q_len[b] on: what seg_rope_rotate takes
 * A sequence grows by at most Lq rows.  One out of range (want < 0 or past max_pages * page_size, a larger growth, a kv_len out of
 * range) stays as it is, a free_count outside [0, n_pages] is cut, a page number outside [0, n_pages) comes out as -1 in the table
 * and the slots, a pos_shift below 0, or one that brings a position past 2^31 - 1, counts as 0: each makes the next
 * seg_attn_poll_status return SEGATTN_ERR_INVALID.  B <= 65535, max_pages * page_size <= 2^30.
 * `workspace`: DEVICE, 256-byte aligned, seg_pages_workspace_bytes(B) bytes (0: invalid B), scratch (calls that may run
 * at the same time, captured ones too, need one each); not looked at, and may be NULL, where B <= 1024 and B * Lq <= 4096 (one kernel; two elsewhere). */
size_t seg_pages_workspace_bytes(int32_t B);
segattn_status seg_pages_resize(int32_t B, int32_t Lq, int32_t page_size, int32_t n_pages, const int32_t* want, int32_t* block_table,
                                int32_t max_pages, int32_t table_stride, const int32_t* kv_len, const int32_t* pos_shift,
                                int32_t* free_pages, const int32_t* free_count, int32_t* kv_len_out, int32_t* free_count_out,
                                int32_t* q_len, int64_t* slots, int32_t* positions, void* workspace, size_t workspace_bytes, void* stream);

/* ---- An 8-bit cache with a scale for each block of rows and head, instead of one for a head that has to be right before the first
 * token.  A block is `rows` (16, 32, 64 or 128; a divisor of page_size) rows of a page from a multiple of it on; the value of a
 * stored element x is x times its block's scale.  The seg_kv_cache beside it has dtype E4M3 and k_scale = v_scale = NULL. */
typedef struct {
    float *k, *v;                     /* DEVICE, addressed by (page, block of the page, head) */
    int64_t k_stride[3], v_stride[3]; /* elements, >= 0 */
    int32_t rows;
} seg_block_scales;

/* seg_kv_append (same arguments, same rows left out) into such a cache.  With m the largest finite magnitude that the call adds
 * to a block (of keys after their rotation), the block's scale becomes the smallest power of two 2^e >= m / 448, -40 <= e <= 119, or stays
 * where the block has rows of its sequence already and their scale is larger; where it grows those rows are brought to it (times
 * old / new, rounded to nearest even: exact, but for values below 2^-6 times the new scale).  (Of a scale that another program has left
 * there the magnitude counts; rows of one that is not finite become NaN or saturate.)  Stored is x times the scale's inverse,
 * rounded to nearest even and saturated at +-448; infinities saturate, and magnitudes past 448 * 2^119 = 2.98e38, a NaN stays one.  Scales of blocks that are written into for the
 * first time may hold anything before.  One kernel. */
segattn_status seg_blocks_append(const seg_kv_cache* c, const seg_block_scales* scales, int32_t Lq, const void* K_new,
                                 const int64_t kn_stride[3], const void* V_new, const int64_t vn_stride[3], int32_t Hq, const void* Q,
                                 const int64_t q_stride[3], void* Q_out, const int64_t qo_stride[3], const float* table,
                                 int32_t n_pos, int32_t rot_dim, int32_t layout, void* stream);

/* seg_kv_evict (same arguments, same rows kept) for such a cache: the kept rows' new blocks take the largest magnitude of their rows' finite
 * scales (2^-40 where that is zero), and a row of another scale is brought to it as above (one whose scale is not finite becomes NaN or saturates).  Scales must not share elements, neither here nor in the append (a zero stride
 * is SEGATTN_ERR_INVALID).  (seg_kv_evict itself moves rows as they are, without their blocks' scales.)  Neither moves means of blocks (see
 * below): those of the new pages are to be taken anew, by seg_blocks_summarise with Lq = max_pages * page_size.  Two kernels. */
segattn_status seg_blocks_evict(const seg_kv_cache* c, const seg_block_scales* scales, const float* weights, int32_t W, int32_t sink,
                                int32_t recent, int32_t heavy, const int32_t* dst_table, int32_t dst_max_pages, int32_t dst_stride,
                                int32_t* idx, int32_t* kv_len_out, int32_t* pos_shift_out, float* weights_out, void* stream);

/* ---- Sparse attention over the far past: a head of class PAST reads, of everything before its segment's tail, the n blocks whose mean
 * keys score highest against the query, found when the token is decoded.  (seg_retrieval_select is the paper's own operator, for a
 * segment at a time over keys that lie in one piece; this one is for rows of the paged cache, each with a choice of its own.)
 * Blocks are `block` slots (16, 32, 64 or 128; a divisor of page_size), block j the slots [j block, (j + 1) block) of a sequence.
 *   means   of a full block's keys: with m = their mean in double, rounded to fp32, and scale = max |m| times 1/127 (in fp32), q = m / scale
 *           (fp32) rounded to the nearest integer, -127 to 127.  A block with an infinite or NaN mean gets q = 0 and a NaN scale.
 *           q is int8 contiguous [n_pages][page_size / block][Hkv][d], 16-byte aligned, scale fp32 [n_pages][page_size / block][Hkv]. */
typedef struct {
    int8_t* q;      /* DEVICE */
    float* scale;   /* DEVICE */
    int32_t block;
} seg_block_means;
/* Means of every block that holds one of the sequence's newest q_len (NULL: Lq) rows and is full; other blocks' are left as they were.
 * With `scales` of more rows than a mean's block: of every full block in a scale's block that holds one, up to the sequence's end, since the
 * append that brought them may have raised that scale and rounded all its rows anew.
 * The cache's V is not read; `scales` is NULL or its blocks' (of which only those of K are read).  One kernel. */
segattn_status seg_blocks_summarise(const seg_kv_cache* c, const seg_block_scales* scales, int32_t Lq, const seg_block_means* means, void* stream);
/* The choice of each new row t and KV head.  For a head of class PAST, with lo the lowest slot that a head of class LOCAL would show
 * the row (seg_attn_decode), blocks j < R = lo / block (rounded down) are to choose from.  The query: the head's query heads summed in
 * double, rounded to fp32 (s), step = max |s| times 1/127, p = s / step rounded to the nearest integer (0 where s is not finite); block j scores
 * (float)(sum over p_i q_ji) * scale_j, exact but for that product.  The blocks below `sink` are chosen in any case, and of the others those of the
 * largest scores (equal: lower block; NaN lowest): n together, or all R where there are no more.
 *   idx   int32 contiguous [B][Lq][Hkv][n]: ascending, then -1; all -1 for heads of other classes.  Rows t >= q_len[b] are left as they were.
 * K, V and their strides in c are not used.  1 <= n <= 128, 0 <= sink <= n; max_pages * page_size / block at most 49152.  One kernel. */
segattn_status seg_blocks_select(const seg_kv_cache* c, int32_t Lq, int32_t Hq, int32_t S, int32_t T, const uint8_t* head_past_mask,
                                 const void* Q, const int64_t q_stride[3], const seg_block_means* means, int32_t n, int32_t sink,
                                 int32_t* idx, void* stream);
/* Blocks to attend to, as seg_blocks_select writes them or of any other origin: 1 <= n <= 128 for each [B][Lq][Hkv].  The entries that
 * count are those in front of the first that does not ascend within [0, R); if that one is not -1 the next seg_attn_poll_status
 * returns SEGATTN_ERR_INVALID.  Lists of heads of other classes are not read. */
typedef struct {
    const int32_t* idx; /* DEVICE, contiguous [B][Lq][Hkv][n] */
    int32_t n, block;
} seg_block_choice;

/* seg_attn_decode over a cache with a scale for each block (scales, or NULL: as c says) and, or, with chosen blocks (choice, or NULL).
 * With a choice a head of class PAST sees the slots of its row's blocks and every slot from R block (see above) to the row's own; the other classes see
 * what they do without one, and weights_out must be NULL.  Each new row's choice is its own: a call of many rows reads the
 * slots they all see once for each.  Scales may be any numbers, zero and negative ones too; those of V that are not zero should lie
 * within a factor of 2^100 of each other, wherever that is.  One of V that is not finite makes O of the rows that see its block not finite, all of it
 * (where their weight of the block is not below fp32's range), and leaves the LSE alone.  Those of unread blocks may hold anything.
 * Everything else is seg_attn_decode's, its workspace excepted: seg_attn_decode_blocks_workspace_bytes(...) of the same arguments. */
size_t seg_attn_decode_blocks_workspace_bytes(const seg_kv_cache* c, const seg_block_scales* scales, const seg_block_choice* choice,
                                              int32_t Lq, int32_t Hq, int32_t with_weights);
segattn_status seg_attn_decode_blocks(const seg_kv_cache* c, const seg_block_scales* scales, const seg_block_choice* choice, int32_t Lq,
                                      int32_t Hq, int32_t S, int32_t T, float sm_scale, const uint8_t* head_past_mask, const void* Q,
                                      const int64_t q_stride[3], void* O, const int64_t o_stride[3], float* LSE, const float* weights_in,
                                      float* weights_out, int32_t W, void* workspace, size_t workspace_bytes, void* stream);

/* ---- Whole training-step call with HOST buffers (pinned or pageable): copies Q, K, V, dO to
 * the device arena, runs forward and backward, copies O, LSE, dQ, dK, dV back, and
 * synchronises `stream` before returning.  Host tensors are contiguous in the layouts
 * above (strides in `p` are ignored).  dO_host == NULL runs the forward only (gradient
 * outputs are then ignored).  `arena` is a caller-owned DEVICE buffer of at least
 * seg_attn_host_arena_bytes(p) bytes, 256-byte aligned.  The work is processed in up to eight
 * chunks - ranges of batch elements or, for batches smaller than that, ranges of KV heads (with
 * their query heads) of one batch element, each an independent problem - whose copies in, kernels
 * (on `stream`) and copies out overlap; the two side streams and their events are created on first
 * use per device and kept for the life of the process.
 * With pageable host memory the copies do not overlap but the result is the same. */
size_t seg_attn_host_arena_bytes(const seg_attn_params* p);
segattn_status seg_attn_step_host(const seg_attn_params* p, const void* Q_host, const void* K_host,
                                  const void* V_host, const void* dO_host, const uint8_t* head_past_mask,
                                  void* O_host, float* LSE_host, void* dQ_host, void* dK_host, void* dV_host,
                                  void* arena, size_t arena_bytes, void* stream);

/* ---- Status and accounting */
/* Synchronises `stream`, then reads and clears the device status that kernels set when a
 * bounded wait expires or a kernel refuses its input.  Returns SEGATTN_OK, SEGATTN_ERR_TIMEOUT (also
 * where an input was refused besides), SEGATTN_ERR_INVALID (an index, position, page or length out of range
 * where a kernel read it) or SEGATTN_ERR_CUDA. */
segattn_status seg_attn_poll_status(void* stream);
const char* seg_attn_status_string(segattn_status s);
/* Last CUDA error code (cudaError_t or CUresult as int) recorded by this thread's failing call. */
int seg_attn_last_cuda_error(void);
/* Exact (query,key) pair counts of the mask summed over batch and query heads (the cost
 * model of Section 3.5 evaluated element-exactly), and the number of 128x128 tiles the
 * forward kernel visits.  Any of the output pointers may be NULL. */
segattn_status seg_attn_count_pairs(const seg_attn_params* p, const uint8_t* head_past_mask,
                                    int64_t* pairs_visible, int64_t* pairs_diff, int64_t* fwd_tiles);
/* Measurement aid (the paper has no counterpart): runs each of the four kernels of a training
 * step on its own - forward, row dots, dQ pass, dK/dV pass, in that order - once untimed and then
 * `iters` times back to back between two CUDA events recorded on `stream`, and returns the average
 * milliseconds per launch in ms_per_launch[0..3].  Arguments as for seg_attn_fwd / seg_attn_bwd
 * (O and LSE are written by the forward and read by the backward).  Synchronises `stream`. */
segattn_status seg_attn_profile_kernels(const seg_attn_params* p, const void* Q, const void* K, const void* V,
                                       void* O, float* LSE, const void* dO, const uint8_t* head_past_mask, void* dQ,
                                       void* dK, void* dV, void* workspace, size_t workspace_bytes, int iters,
                                       float ms_per_launch[4], void* stream);
/* Diagnostic aid (the paper has no counterpart): enqueues a one-warp kernel that waits, with a
 * 1 ms limit, on a barrier nothing ever signals - the way every wait inside the library's kernels
 * is bounded.  The wait gives up, the kernel ends normally, and the next seg_attn_poll_status
 * returns SEGATTN_ERR_TIMEOUT (seg_attn_last_cuda_error() then gives (4 << 8) | 99) and clears
 * the status word; the context stays usable. */
segattn_status seg_attn_selftest_wait_timeout(void* stream);
/* Number of kernel launches the library has enqueued so far in this process. */
int64_t seg_attn_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* SEG_ATTN_H_ */
