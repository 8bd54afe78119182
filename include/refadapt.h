/*
 * refadapt.h — C ABI of the RefAdapt-DiT hot path on one GB300 (sm_103a).
 *
 * RefAdapt-DiT (training-free reference reuse for reference-conditioned
 * diffusion transformers): every DiT block runs joint attention over
 * [text; reference; target] tokens. A block that reuses skips the reference
 * query rows and lets text and target queries attend to reference K/V cached
 * at the block's last materialisation; the first block whose head-mean score
 * D x M reaches theta reactivates and every deeper block recomputes
 * (paper Sec. 4, Algorithm 1).
 *
 * Conventions for every entry point:
 *  - All device pointers are caller-owned; the library allocates no device
 *    memory. Every call is asynchronous on `stream` (a cudaStream_t passed as
 *    void*; NULL = the legacy default stream) and performs no host sync.
 *  - Invalid arguments return RA_EINVAL before anything is launched;
 *    refadapt_last_error() then holds a one-line reason (thread-local).
 *  - A failed launch returns RA_ECUDA. A device-side wait that exceeded its
 *    time budget sets bit 0 of the caller's error word (see
 *    refadapt_check_error), never traps, and leaves the context usable.
 *  - No exceptions cross the ABI; nothing calls exit().
 *  - Calls may come from several host threads and target several GPUs: each
 *    works on the device current in the calling thread, and the library's
 *    one-time set-up (kernel shared-memory limits, SM counts, cluster
 *    occupancy) is kept per device under a mutex, the no-allocation scratch
 *    address per device and CUDA context. Work on one device follows the
 *    stream order the caller gives.
 *  - bf16 tensors are described by ra_seg: element (b, h, n, c) lives at
 *    ptr + b*stride_b + h*stride_h + n*stride_n + c (strides in elements,
 *    c contiguous). ptr and every stride must be 16-byte aligned
 *    (strides multiples of 8 elements).
 */
#ifndef REFADAPT_H
#define REFADAPT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  RA_OK = 0,
  RA_EINVAL = 1,        /* bad argument; nothing launched */
  RA_EUNSUPPORTED = 2,  /* valid but not supported here (e.g. no sm_103 device) */
  RA_ECUDA = 3,         /* a CUDA call failed */
  RA_ETIMEOUT = 4       /* a device-side wait ran out of its budget */
} ra_status;

/* Block execution modes (paper Sec. 4 "Execution and cache state";
 * Algorithm 1). REUSE: reference query rows skipped, text and target rows
 * attend to cached reference K/V. BOUNDARY: the first crossing block; every
 * row runs, reference K/V still from the cache, the cache is not updated.
 * COMPUTE: a block deeper than the boundary; fresh reference K/V are written
 * to the cache (a_b = t) and every row runs. FULL: bounded-age or step-0 full
 * refresh; same work as COMPUTE. */
typedef enum {
  RA_MODE_REUSE = 0,
  RA_MODE_BOUNDARY = 1,
  RA_MODE_COMPUTE = 2,
  RA_MODE_FULL = 3
} ra_mode;

/* Token roles (paper Sec. 3 "Setting"): R = reference rows, Y = the
 * remaining active-generation rows, split here into text and target. */
enum { RA_TEXT = 0, RA_REF = 1, RA_TGT = 2 };

/* Rows of one Q tile of the attention kernel; mass partials come per tile. */
#define RA_MASS_TILE_ROWS 128

typedef struct {
  void* ptr;          /* device, bf16 */
  int64_t stride_b;   /* elements */
  int64_t stride_h;   /* elements */
  int64_t stride_n;   /* elements */
  int32_t n;          /* rows (tokens) in this segment, >= 0 */
  int32_t reserved;   /* set to 0 */
} ra_seg;

/* ------------------------------------------------------------------ attention
 * refadapt_joint_attn — joint attention of one DiT block with the reference
 * mass as a by-product.
 *
 * Computes, per sample b and head h, O = Softmax(scale * Q K^T + bias) V
 * (paper Sec. 3.3, Attn(Q,K,V) = Softmax(QK^T / sqrt(d_h)) V) over the keys
 * [text; ref; target], bidirectional, no mask. Query rows: text and target
 * when mode[b] == RA_MODE_REUSE (reference rows skipped, their O rows left
 * untouched; App. A.4 removes the two reference-query score regions), every
 * row otherwise. The reference K/V segments are whatever the caller points
 * k[RA_REF] / v[RA_REF] at — normally the block's cache slot, so reuse costs
 * no copy.
 *
 * Mass (paper Eq. 4): for every executed query row q in the mass row set,
 * the softmax probability summed over reference keys, l_ref(q) / l(q), is
 * accumulated per 128-row Q tile into mass_partial[b][h][i] (fp32), i over
 * the text tiles (ceil(n_text/128)) then the target tiles
 * (ceil(n_tgt/128)), n counting query rows; refadapt_mass_partial_len()
 * gives the length. Mass row
 * set: target rows (mass_rows = 0), or text + target rows (mass_rows = 1);
 * partials of tiles outside the set are written as 0. M_{t,b,h} is the sum of
 * a (b, h) row of partials divided by the number of mass rows (the gate does
 * this). Every partial is written on every call, in a fixed reduction order
 * (deterministic).
 *
 * Arguments:
 *  q, k, v, o [3]   segments per role (RA_TEXT, RA_REF, RA_TGT). Per role q
 *                   and o share n (query rows) and k and v share n (key
 *                   rows); query and key rows of a role may differ (e.g. a
 *                   row sample of the queries). The target segment needs at
 *                   least one key row. q[RA_REF] / o[RA_REF] with ptr NULL:
 *                   the reference query rows are not computed, whatever the
 *                   mode.
 *  B, H, d          batch, heads, head dim; d in {64, 128}.
 *  softmax_scale    > 0; pass 0 for 1/sqrt(d).
 *  ref_logit_bias   device [H] fp32 or NULL: added to the logits of target
 *                   query rows against reference keys (natural-log units);
 *                   -inf leaves them out.
 *  mode             device [B] int32 (ra_mode) or NULL (= every row runs).
 *  mass_partial     device [B][H][refadapt_mass_partial_len(n_text, n_tgt)].
 *  mass_row_stride  the "sampled target-query rows" of Eq. 4 / Algorithm 1:
 *                   0 or 1 counts every mass row; k > 1 counts rows 0, k,
 *                   2k, ... of the target segment (and of the text segment
 *                   when mass_rows = 1); the partials then sum the sampled
 *                   rows only (divide by their count). O is unaffected.
 *  err_word         device int32 or NULL; bit 0 set on a device timeout.
 *
 * Fused reference-cache update (paper Eq. 11; Algorithm 1's compute and full
 * branches), optional: off when ref_fresh_q/k/v.ptr and a_b are all NULL
 * (the zero-initialised struct). Otherwise, for
 * every sample whose mode is RA_MODE_COMPUTE or RA_MODE_FULL, the reference
 * K/V (and the reference query) are read from ref_fresh_k / ref_fresh_v /
 * ref_fresh_q (this step's reference projections) instead of k/v/q[RA_REF],
 * and copied into k/v/q[RA_REF] (the block's cache slot) as a by-product:
 * one item of each (sample, head) bulk-stores every reference K/V tile it
 * streams through shared memory for its MMAs, each reference-row item its own
 * query tiles, and a_b[b] = step. Samples in REUSE or BOUNDARY read the
 * cache slot as before and leave it untouched. This replaces a separate
 * refadapt_ref_cache_update (and its reads of the fresh tensors) on the
 * attention's own pass over them.
 *
 * Results are deterministic for given arguments and modes. How a row's keys are
 * divided among CTAs (which sets the order of the fp32 sums) follows from the
 * sizes of the call and the modes of its samples.
 *  ref_fresh_k/v    segments with n = k[RA_REF].n (16-byte aligned as above;
 *                   ptr NULL only when n = 0).
 *  ref_fresh_q      n = q[RA_REF].n when q[RA_REF] is given; ptr NULL and
 *                   n = 0 otherwise.
 *  a_b              device [B] int32 or NULL: materialisation step per sample.
 *  step             the step index written into a_b.
 * A fresh segment whose ptr equals its cache segment's (same strides) is read
 * in place and not copied; K and V are both in place or both copied. The
 * cache segments must not overlap the fresh ones otherwise. Errors
 * (RA_EINVAL, nothing queued): n or stride mismatches as above.
 */
typedef struct {
  int32_t B, H, d;
  int32_t mass_rows;
  ra_seg q[3], k[3], v[3], o[3];
  float softmax_scale;
  int32_t mass_row_stride;  /* 0 or 1: every mass row; k > 1: rows 0, k, 2k, ... of each mass segment */
  const float* ref_logit_bias;
  const int32_t* mode;
  float* mass_partial;
  int32_t* err_word;
  ra_seg ref_fresh_q, ref_fresh_k, ref_fresh_v;  /* fused cache update; off when these ptrs and a_b are NULL */
  int32_t* a_b;
  int32_t step;
  int32_t reserved;  /* set to 0 */
} ra_attn_args;

ra_status refadapt_joint_attn(const ra_attn_args* args, void* stream);

int32_t refadapt_mass_partial_len(int32_t n_text, int32_t n_tgt);

/* ------------------------------------------------------------------ Q change
 * refadapt_q_delta — consecutive relative drift of the post-RoPE target
 * query, per sample and head (paper Eq. 1 applied to Q^{Y,h}, Sec. 4
 * "Runtime cues"):
 *   D[b][h] = ||q_cur - q_prev||_F / (||q_prev||_F + eps)
 * over the segment's n rows x d columns. Bandwidth-bound: reads both tensors
 * once through bulk copies into shared memory; fp32 per-thread sums and
 * butterflies, then compensated two-float sums across units, warps and
 * blocks, all in a fixed order (deterministic; relative error of D ~1e-7).
 *
 * Each slab (one sample and head) is reduced by one thread-block cluster of
 * up to 8 CTAs through distributed shared memory, leaving the workspace
 * untouched, when a slab has at most 8 x 384 units of 8 KB per tensor
 * (n <= 98304 rows at d = 128, 196608 at d = 64), all B * H clusters fit on
 * the GPU at once, and they fill at least 60 % of the SMs (or of the units,
 * for tiny inputs). Otherwise a
 * multi-block path spreads the units over all SMs; its ticket counters and
 * partial sums live in the workspace.
 *
 *  q_cur, q_prev    segments with equal n (>= 1); d in {64, 128}.
 *  d_out            device [B][H] fp32.
 *  workspace        device scratch of refadapt_q_delta_workspace_size(B, H)
 *                   bytes, 16-byte aligned, zero-filled once before its first
 *                   use; every call leaves it ready for the next. Calls that
 *                   share a workspace must be stream-ordered. Required (not
 *                   NULL) whatever the slab length.
 */
size_t refadapt_q_delta_workspace_size(int32_t B, int32_t H);
ra_status refadapt_q_delta(const ra_seg* q_cur, const ra_seg* q_prev, int32_t B, int32_t H, int32_t d,
                           float eps, float* d_out, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------ Q change, no allocation
 * refadapt_q_delta_noalloc — the same D as refadapt_q_delta, for callers that
 * cannot allocate device memory and have no workspace to hand over: for
 * example a plugin inside a host framework that owns the whole device memory
 * pool and forbids direct cudaMalloc, or a latency-critical loop that must not
 * pay cudaMalloc's implicit device synchronisation. The paper has no
 * counterpart; this is an interface convenience only.
 *
 * The scratch that the long-slab path needs (ticket counters and per-block
 * partial sums; slabs that fit one cluster use none) lives in a
 * file-scope static device array inside the library, sized for at most
 * RA_Q_DELTA_NOALLOC_MAX_BH (= B * H) slabs, about 193 KB; every GPU that loads
 * the library holds it until the process exits. Larger B * H returns RA_EINVAL
 * (use refadapt_q_delta with a workspace). The call allocates nothing: no
 * cudaMalloc, no cudaFree, no allocating library routine. Its first call on a
 * device looks the array's device address up (cudaGetSymbolAddress with that
 * device current) and caches it for the CUDA context current at that moment;
 * a later call in another context (for instance after cudaDeviceReset tore
 * the primary context down) looks it up again. Make the first call, and the
 * first call after a reset, before any stream capture. A call that takes the
 * multi-block path clears that path's ticket counters on `stream` right
 * before its kernel, after every argument check; a call that returns
 * RA_EINVAL queues nothing. All calls share the one array, so calls that
 * overlap on the GPU (different streams, or different host threads without
 * ordering) race and must not be issued. Arguments and results are those of
 * refadapt_q_delta.
 */
#define RA_Q_DELTA_NOALLOC_MAX_BH 96
ra_status refadapt_q_delta_noalloc(const ra_seg* q_cur, const ra_seg* q_prev, int32_t B, int32_t H, int32_t d,
                                   float eps, float* d_out, void* stream);

/* ------------------------------------------------------------------ gate
 * Controller state of Algorithm 1 for one trajectory (opaque, device
 * resident): a_full (step of the last full refresh), whether the current
 * step is a full refresh, and per sample the reactivated latch and boundary.
 */
typedef struct ra_state ra_state;
size_t refadapt_state_size(int32_t B);
ra_status refadapt_state_init(ra_state* state, int32_t B, void* stream);

/* refadapt_gate — one block's decision (paper Eqs. 12-13, App. A.2 head
 * mean, bounded-age refresh of Sec. 4 / Algorithm 1), on the device.
 *
 * Must be called for blocks 0, 1, ... in order within a step. At b == 0 it
 * opens step t: t == 0 forces FULL (and a_full = 0); else t - a_full >=
 * delta_max forces FULL for every block of the step (and a_full = t); else
 * the reactivated latch is cleared. Per sample: g_h = D[b][h] * M_{t-1,b,h}
 * (M from the previous step's mass partials of this block), gbar = mean_h
 * g_h; FULL if the step is a full refresh, COMPUTE if already reactivated,
 * else BOUNDARY (and latch) if gbar >= theta — or b >= forced_boundary when
 * forced_boundary >= 0 — else REUSE.
 *
 * cue selects the per-head trigger of the controller ablation (paper Sec. 5.3,
 * Tab. 4; App. A.2), everything else unchanged: RA_CUE_PRODUCT g_h = D_h M_h
 * (the method), RA_CUE_CHANGE g_h = D_h (target-Q change only),
 * RA_CUE_EXPOSURE g_h = M_h (exposure only). The anchor-relative variant is
 * RA_CUE_PRODUCT fed with the change to the block's last materialisation
 * (c^anchor of App. A.2) in q_delta; the fixed-interval baseline is
 * theta = +inf with delta_max = the interval.
 *
 *  q_delta            device [B][H] (refadapt_q_delta for this step/block);
 *                     may be NULL at t == 0.
 *  mass_partial_prev  device [B][H][mass_partial_len] from step t-1, block b;
 *                     may be NULL at t == 0.
 *  mass_row_count     number of rows the partials cover (n_tgt, or
 *                     n_text + n_tgt when mass_rows = 1).
 *  mode_out           device [B] int32, read by refadapt_joint_attn and
 *                     refadapt_ref_cache_update.
 *  gbar_out, m_out    device [B] and [B][H] fp32 or NULL (logging; gbar is
 *                     NaN at t == 0).
 */
typedef struct {
  double theta;
  int32_t t, b, B, H;
  int32_t delta_max;
  int32_t forced_boundary;
  int32_t mass_partial_len;
  int32_t mass_row_count;
  int32_t cue;         /* ra_cue */
  int32_t reserved;    /* set to 0 */
  const float* q_delta;
  const float* mass_partial_prev;
  ra_state* state;
  int32_t* mode_out;
  float* gbar_out;
  float* m_out;
} ra_gate_args;

typedef enum { RA_CUE_PRODUCT = 0, RA_CUE_CHANGE = 1, RA_CUE_EXPOSURE = 2 } ra_cue;

ra_status refadapt_gate(const ra_gate_args* args, void* stream);

/* refadapt_q_delta_gate — refadapt_q_delta, then refadapt_gate on the D it
 * produced (paper Eq. 1, then Eqs. 12-13 / App. A.2 / Algorithm 1), with the
 * results of the two calls, bit for bit. When the Q change takes its cluster
 * path this is one launch: each cluster's leader writes its slab's D and takes
 * a ticket from the workspace; the leader that takes the last one runs the
 * decision on all B x H values in its CTA. No CTA waits for another. On the
 * multi-block path the gate is a second launch behind the Q change.
 *
 *  q_cur ... workspace_bytes   as for refadapt_q_delta (the workspace also
 *                              holds the ticket; same size function).
 *  gate                        as for refadapt_gate with gate->B == B,
 *                              gate->H == H, gate->t >= 1 (step 0 has no Q
 *                              change: call refadapt_gate), and gate->q_delta
 *                              NULL or equal to d_out.
 * Errors: RA_EINVAL for either call's argument errors, nothing queued.
 */
ra_status refadapt_q_delta_gate(const ra_seg* q_cur, const ra_seg* q_prev, int32_t B, int32_t H, int32_t d,
                                float eps, float* d_out, void* workspace, size_t workspace_bytes,
                                const ra_gate_args* gate, void* stream);

/* ------------------------------------------------------------------ cache
 * refadapt_ref_cache_update — materialise a block's reference K/V into its
 * cache slot (paper Eq. 11, Z_b = (H_b, K_b, V_b, a_b); Algorithm 1: a
 * COMPUTE or FULL block updates K_b, V_b and sets a_b = t).
 *
 * For each sample b with mode[b] in {COMPUTE, FULL}: copies k_src -> k_cache,
 * v_src -> v_cache and, when x_src is not NULL, x_src -> x_cache (the
 * block's cached reference hidden state, any bf16 [B, x_heads, n, x_width]
 * tensor), then sets a_b[b] = t. Samples in other modes are untouched. A copy
 * whose source and destination pointers are equal is skipped (in-place
 * producer). 16-byte vector copies.
 *
 *  k_*, v_*      segments [B, H, n_ref, d]; all n equal; d in {64, 128}.
 *  x_src/x_cache optional segments [B, x_heads, n_ref, x_width];
 *                x_width a multiple of 8.
 *  mode          device [B] int32.
 *  a_b           device [B] int32 or NULL.
 */
ra_status refadapt_ref_cache_update(const ra_seg* k_src, const ra_seg* v_src, const ra_seg* k_cache,
                                    const ra_seg* v_cache, int32_t B, int32_t H, int32_t d,
                                    const ra_seg* x_src, const ra_seg* x_cache, int32_t x_heads,
                                    int32_t x_width, const int32_t* mode, int32_t t, int32_t* a_b,
                                    void* stream);

/* ------------------------------------------------------------------ DiT block around the attention
 * The paper's models are DiTs whose blocks run joint attention over
 * [text; reference; target] rows (Sec. 3, "Setting"). Under reuse the
 * reference-side QKV projections and the other reference-stream operations
 * are skipped because the layer-wise reference K/V are cached (App. A.4);
 * at the boundary the cached reference hidden state is restored, its query
 * runs against the current target and the reference output becomes the next
 * block's cached hidden state (Algorithm 1, App. A.3). The paper does not
 * give the block's layers; these entry points build a dual-stream MMDiT
 * block (text rows with one weight set, reference and target rows with
 * another) from: a modulated LayerNorm (refadapt_ln_modulate), linear layers
 * with fused epilogues (refadapt_gemm) and the RoPE table the QKV epilogue
 * reads (refadapt_rope_table).
 *
 * Rows come in up to three segments (text, reference, target), each with its
 * own pointers and strides; row r of sample s of a segment lives at
 * ptr + s * stride_s + r * stride_r (elements, features contiguous). A
 * segment with gated = 1 is skipped for samples whose mode (device [B],
 * written by refadapt_gate) is RA_MODE_REUSE. All calls are asynchronous on
 * `stream` and allocate nothing; invalid arguments return RA_EINVAL before
 * anything is launched.
 */

/* refadapt_rope_table — table[pos][i] = (cos, sin)(pos * base^(-2i/d)),
 * fp32, pos in [0, n_pos), i in [0, d/2): [n_pos][d/2][2] floats, 16-byte
 * aligned (device, caller-owned). Angles in fp64. d a multiple of 4. */
ra_status refadapt_rope_table(float* table, int32_t n_pos, int32_t d, double base, void* stream);

/* refadapt_ln_modulate — x = LN(h) * (1 + scale[s]) + shift[s] per row:
 * LN without affine over C features, fp32 mean and variance, eps added to
 * the variance; shift and scale are the block's AdaLN vectors for the row's
 * stream and sample, fp32 [B][C] (row stride mod_stride_s). bf16 in and out;
 * h and x must not overlap. C a multiple of 256, at most 4096; pointers
 * 16-byte aligned, row strides >= C and multiples of 8 elements. The call waits
 * only for its own copies and has no error word: rows whose copy did not end
 * within the wait budget (at least 0.5 s) become NaN. */
typedef struct {
  const void* h;
  int64_t h_stride_s, h_stride_r;
  void* x;
  int64_t x_stride_s, x_stride_r;
  const float* shift;
  const float* scale;
  int64_t mod_stride_s;
  int32_t rows;       /* rows per sample, >= 0 */
  int32_t gated;
} ra_lnmod_seg;

typedef struct {
  int32_t B, C, n_seg, reserved;
  float eps, reserved2;
  ra_lnmod_seg seg[3];
  const int32_t* mode;  /* device [B]; required when a segment is gated */
} ra_lnmod_args;

ra_status refadapt_ln_modulate(const ra_lnmod_args* args, void* stream);

/* refadapt_gemm — out = epilogue(A W^T + bias) on tcgen05 tensor cores:
 * A bf16 rows of each segment (K features), W bf16 [N][K] (nn.Linear
 * layout, one weight matrix per segment, so text and image streams differ),
 * bias fp32 [N] or NULL, fp32 accumulation. N a multiple of 256, K of 64.
 * Epilogues (fp32 until one final rounding to bf16):
 *   RA_EPI_STORE  out = acc + bias
 *   RA_EPI_GELU   out = gelu_tanh(acc + bias)
 *   RA_EPI_RESID  out = resid + gate[s] * (acc + bias); gate fp32 [B][N]
 *                 (row stride gate_stride_s); resid may equal out
 *                 (in-place update of a residual stream) but must not
 *                 partially overlap it.
 *   RA_EPI_QKV    N = 3 H d, columns [q | k | v], head h at h*d within each
 *                 part: q and k of each head are RMS-normalised over d
 *                 (fp32, norm_eps added to the mean square) and scaled by
 *                 q_norm / k_norm [d], then rotated by RoPE on interleaved
 *                 pairs (2i, 2i+1) at position pos_offset + r, reading
 *                 rope[pos][i] (refadapt_rope_table, rope_len rows); v gets
 *                 the bias only. Written head-major to q_out, k_out, v_out
 *                 (ra_seg, n = rows): for a gated segment (the reference
 *                 rows) the K and V tiles are also skipped when the mode is
 *                 RA_MODE_BOUNDARY (the block keeps its cached K/V), so k_out
 *                 and v_out can point straight at the block's cache slot.
 * Pointers 16-byte aligned; row strides multiples of 8 elements; out rows
 * hold N columns (out_stride_r >= N); A rows K (a_stride_r >= K).
 * err_word: device int32 or NULL; bit 0 set if a device wait timed out.
 * tile_mode: 0 picks CTA pairs (a cluster of two SMs running one cta_group::2
 * MMA on a tile of 256 rows, each SM staging half of the operands) or one CTA
 * per tile of 128 rows, whichever a model of the call's time prefers; 1 and 2
 * force either. Tiles are up to 256 columns wide, narrower where that saves a
 * round of tiles; modes 1 and 2 give the same results. Mode 0 also lets the CTAs
 * of a cluster share a tile's K where tiles are few and K is long: the fp32 sums
 * of up to four parts of K are then added in a fixed order, so a call's results
 * are deterministic, but a row's last rounding may depend on the call's other
 * rows and on the modes.
 */
typedef enum { RA_EPI_STORE = 0, RA_EPI_GELU = 1, RA_EPI_RESID = 2, RA_EPI_QKV = 3 } ra_epilogue;

typedef struct {
  const void* a;
  int64_t a_stride_s, a_stride_r;
  int32_t rows;        /* rows per sample, >= 0 */
  int32_t gated;
  const void* w;       /* bf16 [N][K] */
  const float* bias;   /* [N] or NULL */
  void* out;           /* STORE / GELU / RESID */
  int64_t out_stride_s, out_stride_r;
  const void* resid;   /* RESID */
  int64_t resid_stride_s, resid_stride_r;
  const float* gate;   /* RESID: [B][N] */
  int64_t gate_stride_s;
  ra_seg q_out, k_out, v_out;          /* QKV: [B, H, rows, d] */
  const float* q_norm;                 /* QKV: [d] */
  const float* k_norm;                 /* QKV: [d] */
  int32_t pos_offset;                  /* QKV: RoPE position of row 0 */
  int32_t reserved;
} ra_gemm_seg;

typedef struct {
  int32_t B, N, K, epilogue;
  int32_t H, d, n_seg, rope_len;       /* H, d, rope_len: QKV only */
  ra_gemm_seg seg[3];
  const int32_t* mode;                 /* device [B]; required when a segment is gated */
  const float* rope;                   /* QKV: [rope_len][d/2][2] */
  float norm_eps;
  int32_t tile_mode;                   /* 0 auto, 1 one CTA per 128-row tile, 2 CTA pairs on 256-row tiles */
  int32_t* err_word;
} ra_gemm_args;

ra_status refadapt_gemm(const ra_gemm_args* args, void* stream);

/* ------------------------------------------------------------------ layers of gated DiT blocks
 * Further layers that DiT blocks put around the joint attention: rotary
 * positions with several axes, norms before and after a branch, and the gated
 * feed-forward. Each has its backward pass, for training such blocks (the
 * paper's method itself trains nothing). Rows come in segments as above. All
 * calls are asynchronous on `stream` and allocate nothing; invalid arguments
 * return RA_EINVAL before anything is launched.
 */

/* refadapt_rope_axes — rotary positions with several axes (time, height,
 * width, ...) on up to two tensors (a block's q and k; their head counts may
 * differ):
 *   the columns of a head are cut into n_axes runs of axis_dim[a] columns; pair
 *   i of run a, columns (2i, 2i + 1) of the run, turns by the angle
 *   pos[s][r][a] * base^(-2i / axis_dim[a])
 * Columns past the last run are copied. inverse = 1 turns by the negative
 * angle: the inverse, and the gradient of the forward turn.
 *
 *  pos         device fp32 [n][n_axes] per sample, samples pos_stride_s
 *              elements apart (0: all samples share the positions). Any finite
 *              values (negative and fractional ones too); the angle is formed
 *              in two-float arithmetic, exact to fp32 for |angle| < 2^24.
 *  axis_dim    even, >= 2, sum <= d; 1 to 4 axes; base > 1.
 *  d           a multiple of 8, at most 256; n * d / 8 < 2^31.
 *  t[i].x, .out  bf16 segments of n rows; out may equal x (same strides) but
 *              must not partially overlap it, nor the other tensor. The strides
 *              of an output are at least d; those of axes with one entry say
 *              nothing. */
typedef struct {
  ra_seg x, out;
  int32_t heads, reserved;
} ra_rope_tensor;

typedef struct {
  int32_t B, n, d, n_axes;
  int32_t axis_dim[4];
  double base;
  const float* pos;
  int64_t pos_stride_s;
  int32_t n_tensors, inverse;
  ra_rope_tensor t[2];
} ra_rope_args;

ra_status refadapt_rope_axes(const ra_rope_args* args, void* stream);

/* refadapt_rope_axes_table — the same angles as a table for the QKV epilogue
 * of refadapt_gemm: table[r][i] = (cos, sin) of pair i at the coordinates
 * pos[r], fp32, [n][d/2][2] (16-byte aligned); a segment's pos_offset is then
 * its first row of the table. Pairs past the last run get (1, 0). d a multiple
 * of 4. axis_dim: host array of n_axes entries. */
ra_status refadapt_rope_axes_table(float* table, const float* pos, int32_t n, int32_t d, int32_t n_axes,
                                   const int32_t* axis_dim, double base, void* stream);

typedef enum { RA_NORM_NONE = 0, RA_NORM_LAYER = 1, RA_NORM_RMS = 2 } ra_norm;

/* refadapt_residual_norm — what stands between two branches of a block, in
 * one pass over the rows: the norm after the branch, its gate, the residual sum
 * and the norm before the next branch with its modulation:
 *   h_out = alpha * h + gate[s] * (N_post(y) * post_w)
 *   x     = N_pre(h_out) * pre_w * (1 + scale[s]) + shift[s]
 * N_LAYER(v) = (v - mean) / sqrt(var + eps), N_RMS(v) = v / sqrt(mean(v^2) +
 * eps) over the C features of a row, N_NONE(v) = v; fp32 throughout, x from the
 * unrounded h_out, one rounding to bf16 per output.
 *
 *  h, y         bf16 rows; y NULL: h_out = alpha * h.
 *  h_out, x     bf16 rows; either may be NULL (not both). Each may equal h or
 *               y (same strides), in place, but must not partially overlap them.
 *  gate, scale, shift  fp32 [B][C] (rows gate_stride_s; mod_stride_s for both
 *               scale and shift); NULL: 1, 0 and 0.
 *  post_w, pre_w  fp32 [C] or NULL (1).
 * C a multiple of 8, at most 5120; pointers 16-byte aligned, row strides >= C
 * and multiples of 8 elements (of 4 for the fp32 vectors). A segment with
 * gated = 1 is skipped for samples whose mode is RA_MODE_REUSE. B * rows of all
 * segments below 2^30. */
typedef struct {
  const void* h;
  int64_t h_stride_s, h_stride_r;
  const void* y;
  int64_t y_stride_s, y_stride_r;
  void* h_out;
  int64_t h_out_stride_s, h_out_stride_r;
  void* x;
  int64_t x_stride_s, x_stride_r;
  const float* gate;
  int64_t gate_stride_s;
  const float* scale;
  const float* shift;
  int64_t mod_stride_s;
  const float* post_w;
  const float* pre_w;
  int32_t rows;       /* rows per sample, >= 0 */
  int32_t gated;
} ra_resnorm_seg;

typedef struct {
  int32_t B, C, n_seg, post, pre, reserved;  /* post, pre: ra_norm */
  float eps, alpha;
  ra_resnorm_seg seg[3];
  const int32_t* mode;  /* device [B]; required when a segment is gated */
} ra_resnorm_args;

ra_status refadapt_residual_norm(const ra_resnorm_args* args, void* stream);

/* refadapt_residual_norm_backward — gradients of refadapt_residual_norm for
 * one segment. From h (the forward call's h_out), y, dx and dh_out (gradients
 * with respect to x and h_out; one of them may be NULL, taken as zero):
 *   dh, dy                  bf16 rows, gradients of the forward call's h and y
 *   dgate, dscale, dshift   fp32 [B][C], contiguous
 *   dpost_w, dpre_w         fp32 [C], summed over the samples
 * Any output may be NULL. y may be NULL (then dy, dgate and dpost_w too).
 * dh and dy may each equal an input (same strides), in place, but must not
 * overlap one another. Column sums are fp32 in a fixed order (deterministic).
 *  workspace   device scratch of
 *              refadapt_residual_norm_backward_workspace_size(B, rows, C) bytes
 *              (on the device that is current), 16-byte aligned; calls that
 *              share it must be stream-ordered.
 *  err_word    device int32 or NULL; bit 0 set if a device wait timed out (the
 *              sums are NaN then). */
typedef struct {
  int32_t B, C, rows, post, pre, reserved;
  float eps, alpha;
  const void* h;
  int64_t h_stride_s, h_stride_r;
  const void* y;
  int64_t y_stride_s, y_stride_r;
  const void* dx;
  int64_t dx_stride_s, dx_stride_r;
  const void* dh_out;
  int64_t dh_out_stride_s, dh_out_stride_r;
  void* dh;
  int64_t dh_stride_s, dh_stride_r;
  void* dy;
  int64_t dy_stride_s, dy_stride_r;
  const float* gate;
  int64_t gate_stride_s;
  const float* scale;
  int64_t mod_stride_s;
  const float* post_w;
  const float* pre_w;
  float* dgate;
  float* dscale;
  float* dshift;
  float* dpost_w;
  float* dpre_w;
  void* workspace;
  size_t workspace_bytes;
  int32_t* err_word;
} ra_resnorm_grad_args;

size_t refadapt_residual_norm_backward_workspace_size(int32_t B, int32_t rows, int32_t C);
ra_status refadapt_residual_norm_backward(const ra_resnorm_grad_args* args, void* stream);

/* refadapt_glu — the gated feed-forward's projections, activation and product
 * in one kernel, on tcgen05 tensor cores:
 *   out = act(x Wg^T) o (x Wu^T)
 * x bf16 rows of C features, Wg and Wu bf16 [F][C] contiguous (nn.Linear
 * layout; halves of one [2 F][C] matrix will do), one pair per segment, fp32
 * accumulation, one rounding to bf16 per output. act: RA_ACT_SILU g / (1 + e^-g)
 * or RA_ACT_GELU (tanh form). The down projection is refadapt_gemm.
 *  pre_gate, pre_up   bf16 rows of F, the products before the activation, for
 *                     refadapt_glu_backward; both or neither (NULL).
 * C and F multiples of 8, at least 64; pointers 16-byte aligned, row strides
 * multiples of 8 elements and at least the row's length. A segment with gated =
 * 1 is skipped for samples whose mode is RA_MODE_REUSE. err_word: device int32
 * or NULL; bit 0 set if a device wait timed out. No output of any segment may
 * overlap an input or another output (refused where tensors start at one address
 * or fill ranges that meet); B * rows below 2^30. Deterministic; how a call is cut into
 * tiles follows from its sizes. */
typedef enum { RA_ACT_SILU = 0, RA_ACT_GELU = 1 } ra_act;

typedef struct {
  const void* x;
  int64_t x_stride_s, x_stride_r;
  const void* w_gate;  /* bf16 [F][C] */
  const void* w_up;    /* bf16 [F][C] */
  void* out;
  int64_t out_stride_s, out_stride_r;
  void* pre_gate;
  int64_t pre_gate_stride_s, pre_gate_stride_r;
  void* pre_up;
  int64_t pre_up_stride_s, pre_up_stride_r;
  int32_t rows;        /* rows per sample, >= 0 */
  int32_t gated;
} ra_glu_seg;

typedef struct {
  int32_t B, F, C, act, n_seg, reserved;
  ra_glu_seg seg[3];
  const int32_t* mode;  /* device [B]; required when a segment is gated */
  int32_t* err_word;
} ra_glu_args;

ra_status refadapt_glu(const ra_glu_args* args, void* stream);

/* refadapt_glu_backward — gradients of the gated feed-forward of one segment,
 *   y = hidden Wd^T,  hidden = act(g) o w,  g = x Wg^T,  w = x Wu^T,
 * from dy and what refadapt_glu kept (pre_gate = g, pre_up = w, hidden = out):
 *   du = dy Wd,  dg = du o w o act'(g),  dw = du o act(g),
 *   dx = dg Wg + dw Wu,  dw_gate = dg^T x,  dw_up = dw^T x,  dw_down = dy^T hidden
 * dg and dw are formed in the epilogue of dy Wd from its fp32 sums (du is never
 * stored) and rounded to bf16 once, as operands of the products after them.
 * Two or three launches, and one more where a long sum is split.
 *  dy                  bf16 rows of O features; w_down bf16 [O][F].
 *  dx, dw_*            bf16, contiguous [F][C] and [O][F] for the weights; any
 *                      may be NULL (frozen weights), not all. hidden may be NULL
 *                      without dw_down, x without dw_gate and dw_up.
 *  workspace           device scratch of refadapt_glu_backward_workspace_size()
 *                      bytes (on the device that is current), 16-byte aligned;
 *                      calls that share it must be stream-ordered.
 * C, F, O multiples of 8, at least 64; pointers and strides as for refadapt_glu;
 * neither outputs nor the workspace may overlap inputs, one another or themselves. Rows of
 * zero: the weights' gradients are zero. Deterministic. */
typedef struct {
  int32_t B, rows, C, F, O, act;
  const void* dy;
  int64_t dy_stride_s, dy_stride_r;
  const void* x;
  int64_t x_stride_s, x_stride_r;
  const void* pre_gate;
  int64_t pre_gate_stride_s, pre_gate_stride_r;
  const void* pre_up;
  int64_t pre_up_stride_s, pre_up_stride_r;
  const void* hidden;
  int64_t hidden_stride_s, hidden_stride_r;
  const void* w_gate;
  const void* w_up;
  const void* w_down;
  void* dx;
  int64_t dx_stride_s, dx_stride_r;
  void* dw_gate;
  void* dw_up;
  void* dw_down;
  void* workspace;
  size_t workspace_bytes;
  int32_t* err_word;
} ra_glu_grad_args;

size_t refadapt_glu_backward_workspace_size(int32_t B, int32_t rows, int32_t C, int32_t F, int32_t O);
ra_status refadapt_glu_backward(const ra_glu_grad_args* args, void* stream);

/* ------------------------------------------------------------------ linear layers in 4 bits
 * Products of microscaled 4-bit matrices, on the tensor cores' 4-bit rate: rows
 * and weights in 4 bits with a scale for every few columns, the sums in fp32, the
 * epilogues of refadapt_gemm. All calls are asynchronous on `stream` and allocate
 * nothing; invalid arguments return RA_EINVAL before anything is launched.
 *
 * A 4-bit matrix of R rows and K columns:
 *  codes   two e2m1 values a byte, the even column in the low half: [R][K / 2].
 *          e2m1: sign in bit 3, then 0, 0.5, 1, 1.5, 2, 3, 4, 6.
 *  scales  one byte for each block of columns of a row, in tiles of 128 rows by
 *          four blocks, 512 bytes, [ceil(R / 128)][ceil(K / (4 block))][512]: row r
 *          and block j of a tile at 16 (r % 32) + 4 (r / 32) + j. What lies behind
 *          the last row or block is zero.
 *            RA_Q4_E4M3  blocks of 16; e4m3 value times 2^exponent (one exponent
 *                        for the matrix, of the caller's choice)
 *            RA_Q4_E8M0  blocks of 32; 2^(byte - 127); exponent 0
 * A value is its e2m1 value times its scale. refadapt_quant4_scales_size: bytes of
 * one matrix's scales; 0 if rows or K are negative or the format is unknown.
 */
typedef enum { RA_Q4_E4M3 = 0, RA_Q4_E8M0 = 1 } ra_q4_format;

size_t refadapt_quant4_scales_size(int32_t rows, int32_t K, int32_t format);

/* refadapt_quant4 — bf16 rows to 4 bits, along their features (codes, scales: each
 * sample's rows a matrix of C columns), along the rows (codes_t, scales_t: the
 * transposed matrix of all samples' rows, C rows of ceil(B rows / 64) * 64 columns,
 * zeros behind the last), or both. Per block, amax its largest magnitude:
 *   RA_Q4_E4M3  scale = e4m3(amax / 2^exponent / 6), at most 448 (exact to the
 *               nearest, ties to even; larger blocks saturate)
 *   RA_Q4_E8M0  scale = the smallest power of two (2^-126 or more) with
 *               amax <= 6 scale
 *   value       x / (scale 2^exponent) to the nearest e2m1 value, ties to even,
 *               saturating; 0 where the scale is 0
 * A block with a value that is not finite gets a scale that is NaN (0x7f, 0xff).
 *
 *  x           bf16 rows of C features; pointer 16-byte aligned, strides multiples
 *              of 8 elements, row stride >= C.
 *  codes       [B][rows][C / 2], 16-byte aligned, strides in bytes, multiples of 16;
 *              C a multiple of 64.
 *  scales      [B][ceil(rows / 128)][..][512] contiguous, 16-byte aligned.
 *  codes_t     C rows of codes_t_stride bytes (a multiple of 16), 16-byte aligned; C
 *              a multiple of 8.
 *  scales_t    as of one matrix of C rows, contiguous, 16-byte aligned.
 *  exponent    -64 to 64; 0 for RA_Q4_E8M0.
 * codes and scales go together, codes_t and scales_t too; no output may overlap an input,
 * another output or itself. A segment with gated = 1 is skipped for samples whose mode is
 * RA_MODE_REUSE (not with codes_t). B * rows of a segment below 2^30. */
typedef struct {
  const void* x;
  int64_t x_stride_s, x_stride_r;
  void* codes;
  int64_t codes_stride_s, codes_stride_r;  /* bytes */
  void* scales;
  void* codes_t;
  int64_t codes_t_stride;                  /* bytes */
  void* scales_t;
  int32_t rows;       /* rows per sample, >= 0 */
  int32_t gated;
  int32_t exponent, reserved;
} ra_quant4_seg;

typedef struct {
  int32_t B, C, n_seg, format;
  ra_quant4_seg seg[3];
  const int32_t* mode;  /* device [B]; required when a segment is gated */
} ra_quant4_args;

ra_status refadapt_quant4(const ra_quant4_args* args, void* stream);

/* refadapt_gemm4 — refadapt_gemm with 4-bit operands of one format:
 *   out = epilogue(2^(a_exponent + w_exponent) A W^T + bias)
 * with exact products and fp32 sums (a_exponent + w_exponent up to 127). lin.a: codes, its
 * strides in bytes (multiples of 16, a_stride_r >= K / 2); lin.w: codes [N][K / 2];
 * a_scales, w_scales as above; all 16-byte aligned. N a multiple of 64 (QKV: as for
 * refadapt_gemm), K of 64. The other fields, the epilogues, gates, tile_mode and err_word
 * are refadapt_gemm's. No output may overlap an input (but out may be resid), another
 * output or itself. Deterministic; the order of the fp32 sums follows from the sizes of
 * the call. */
typedef struct {
  ra_gemm_seg lin;
  const void* a_scales;
  const void* w_scales;
  int32_t a_exponent, w_exponent;
} ra_gemm4_seg;

typedef struct {
  int32_t B, N, K, epilogue;
  int32_t H, d, n_seg, rope_len;       /* H, d, rope_len: QKV only */
  ra_gemm4_seg seg[3];
  const int32_t* mode;                 /* device [B]; required when a segment is gated */
  const float* rope;                   /* QKV: [rope_len][d/2][2] */
  float norm_eps;
  int32_t tile_mode;                   /* as ra_gemm_args */
  int32_t* err_word;
  int32_t format;                      /* ra_q4_format */
  int32_t reserved;
} ra_gemm4_args;

ra_status refadapt_gemm4(const ra_gemm4_args* args, void* stream);

/* refadapt_linear4_backward — gradients of y = x W^T through 4-bit products, all
 * operands in RA_Q4_E8M0 along the axis that is summed over (Q):
 *   dx = Q(dy) Q(W^T)^T,   dw = Q(dy^T) Q(x^T)^T
 *  dy, x        bf16 rows of N and K features; w bf16 [N][K] contiguous.
 *  dx           bf16 rows of K features, each sample's right behind those of the one
 *               before (dx_stride_s = rows * dx_stride_r), or NULL (then w may be NULL).
 *  dw           bf16 [N][K] contiguous, or NULL (then x may be NULL). Not both NULL.
 *  workspace    device scratch of refadapt_linear4_backward_workspace_size() bytes,
 *               16-byte aligned; calls that share it must be stream-ordered.
 * N and K multiples of 64; pointers 16-byte aligned, strides multiples of 8 elements;
 * neither outputs nor the workspace may overlap inputs, one another or themselves. Rows of zero:
 * dw is zero. B * rows below 2^30. Deterministic. */
typedef struct {
  int32_t B, rows, K, N;
  const void* dy;
  int64_t dy_stride_s, dy_stride_r;
  const void* x;
  int64_t x_stride_s, x_stride_r;
  const void* w;
  void* dx;
  int64_t dx_stride_s, dx_stride_r;
  void* dw;
  void* workspace;
  size_t workspace_bytes;
  int32_t* err_word;
} ra_linear4_grad_args;

size_t refadapt_linear4_backward_workspace_size(int32_t B, int32_t rows, int32_t K, int32_t N);
ra_status refadapt_linear4_backward(const ra_linear4_grad_args* args, void* stream);

/* ------------------------------------------------------------------ the optimiser's step
 * What turns gradients into weights, over any number of tensors in one call.
 */

typedef enum { RA_F32 = 0, RA_BF16 = 1 } ra_type;

/* refadapt_grad_norm — out[0] = sqrt(sum of g^2) over the elements of all tensors,
 * out[1] = min(1, max_norm / out[0]), the factor that clips them to max_norm (out[1]
 * is NaN where the norm is not finite). Squares are formed in fp32 (a gradient beyond
 * 1.8e19 makes the norm infinite, a thousand beyond 5e17 may; below 1.1e-19 they lose bits,
 * below 2.6e-23 they are zero), summed in fp32 over up to 1024 elements, at most 32 in a
 * row, and in fp64 above that, in a fixed order (deterministic).
 *  tensors    host array; g device, fp32 or bf16, aligned to its type, n >= 0 elements.
 *  max_norm   > 0 (INFINITY: no clipping).
 *  out        device fp32 [2].
 *  workspace  device scratch of refadapt_grad_norm_workspace_size() bytes, 16-byte
 *             aligned, zero-filled once before its first use; every call leaves it ready
 *             for the next. Calls that share it must be stream-ordered. Its second 32-bit
 *             word counts the calls whose norm was finite, the steps that refadapt_adamw
 *             takes (a step_dev that needs no launch of its own). */
typedef struct {
  const void* g;
  int64_t n;
  int32_t type;       /* ra_type */
  int32_t reserved;
} ra_grad;

size_t refadapt_grad_norm_workspace_size(void);
ra_status refadapt_grad_norm(const ra_grad* tensors, int32_t n_tensors, float max_norm, float* out, void* workspace,
                             size_t workspace_bytes, void* stream);

/* refadapt_adamw — one step of Adam with decoupled weight decay, over all tensors:
 *   g' = c g                   c = *grad_scale (device), or 1
 *   m  = beta1 m + (1 - beta1) g'
 *   v  = beta2 v + (1 - beta2) g'^2
 *   p  = p - lr decay p - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * in fp32, p in place, its rounding to bf16 in w (a |g'| beyond 1.8e19, whose square passes
 * fp32's end, makes v infinite). Where c is not finite the call changes nothing.
 *  bits = 32  m and v are fp32.
 *  bits = 8   m and v are e4m3 in blocks of 32 elements, with a power of two (e8m0
 *             byte, 2^(byte - 127)) for each in m_scale and v_scale: the smallest one
 *             (2^-126 or more) with amax <= 448 scale. New moments are rounded to one
 *             of the two e4m3 values beside them so that the mean is kept: with r of 16
 *             random bits, the upper one where the part above the lower one is at least
 *             1 - (16 r + 8) / 2^20 of the step. (Rounding to the nearest would hold v
 *             where it is: a step changes it by 0.1 %.) A second moment above zero is
 *             at least the smallest step. The update uses the moments before this
 *             rounding. A block with a moment that is not finite gets the scale NaN
 *             (0xff). r is the low (m) and the high (v) half of
 *               mix(i * 0x9e3779b1 ^ key),  i the element, counted over the call's
 *             tensors, each from the next multiple of 32 on; key = mix(mix(mix(low
 *             half of seed) ^ high half) ^ t), and where i passes 32 bits mix(key ^ its
 *             upper half); mix(x): x ^= x >> 16, x *= 0x243f6a89, x ^= x >> 15,
 *             x *= 0xb7e15163, x ^= x >> 16, all in 32 bits.
 *  tensors    host array. p fp32, g fp32 or bf16, w bf16 or NULL; n >= 0 elements,
 *             contiguous, each pointer aligned to its type (16 bytes is fastest). No
 *             output may overlap an input or another output.
 *  lr, step   the rate and the number t >= 1 of the step; lr_dev, step_dev: device fp32
 *             and int32, or NULL, which count instead (a captured call then goes on with
 *             what they hold when it is replayed; a step below 1 there counts as 1).
 *  beta1, beta2 in [0, 1), eps >= 2^-126 (1.2e-38), decay >= 0, lr >= 0, all finite in fp32. */
typedef struct {
  void* p;
  const void* g;
  void* m;
  void* v;
  void* m_scale;      /* bits = 8: [ceil(n / 32)] */
  void* v_scale;
  void* w;
  int64_t n;
  int32_t g_type;     /* ra_type */
  int32_t reserved;
} ra_adamw_tensor;

typedef struct {
  const ra_adamw_tensor* tensors;
  int32_t n_tensors, bits;
  double lr, beta1, beta2, eps, decay;
  int64_t step;
  const float* lr_dev;
  const int32_t* step_dev;
  const float* grad_scale;
  uint64_t seed;
} ra_adamw_args;

ra_status refadapt_adamw(const ra_adamw_args* args, void* stream);

/* ------------------------------------------------------------------ misc */
const char* refadapt_status_string(ra_status s);
const char* refadapt_last_error(void);

/* Diagnostic: how this thread's last refadapt_joint_attn, refadapt_gemm,
 * refadapt_gemm4 or refadapt_ln_modulate was launched, e.g. "clusters of 2" (text for people and
 * tests, valid until the thread's next call of this function). */
const char* refadapt_last_launch(void);

/* Budget, in nanoseconds, of every device-side mbarrier wait of kernels
 * launched afterwards by this process (default 2e9). */
void refadapt_set_wait_budget_ns(uint64_t ns);

/* Synchronises `stream`, reads the device error word, clears it and returns
 * RA_ETIMEOUT if a device wait ran out, RA_ECUDA on a CUDA error, else RA_OK. */
ra_status refadapt_check_error(int32_t* err_word, void* stream);

int32_t refadapt_version(void);

/* Diagnostic for the timeout path: launches one thread that waits, with the
 * given budget, on an mbarrier that nothing ever arrives at — the same bounded
 * wait every kernel uses. The wait gives up, sets bit 0 of *err_word and the
 * kernel returns normally, so refadapt_check_error then reports RA_ETIMEOUT
 * with the context still usable. budget_ns is capped at 1e9. */
ra_status refadapt_selftest_wait_timeout(int32_t* err_word, uint64_t budget_ns, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* REFADAPT_H */
