/*
 * al.h -- C ABI of the MI355X (gfx950) quantized optimizer-step library
 * (libal.so).
 *
 * The library implements the fused quantized optimizer step of "Beyond Dense
 * Adam States: Adaptive Log-Space Quantization for Memory-Efficient
 * Optimizers": each step decodes block-wise optimizer state, applies the
 * optimizer update and re-encodes the state, for AdamW (dense M, V), Adafactor
 * (factored V) and CAME (dense M, factored V and factored confidence C),
 * section 3.1.
 *
 * Codes (section 4):
 *   AL8 / AL16  non-negative states. Per block of B consecutive elements of
 *               the row-major flattening: l_min = max(l_floor, log2 of the
 *               smallest positive value), l_max = log2 of the largest,
 *               capped at 126 (Eq. al_bounds); positive x -> 1 +
 *               round((L-2) clip((log2 x - l_min)/(l_max - l_min), 0, 1)),
 *               zero -> 0 (Eq. al_quant); decode 2^(l_min + (q-1)/(L-2) *
 *               delta) (Eq. al_dequant). L = 256 (AL8, uint8 codes) or
 *               65,536 (AL16, uint16 codes). q = 0 iff x = 0 (Eq.
 *               exact_zero). Equal positives widen the interval upward by
 *               one log2 unit; the width is at least 1e-12.
 *               Metadata: 2 floats per block, {l_min, delta}.
 *   UF8         signed momentum (section 4.3): symmetric int8 in
 *               [-127, 127] with a per-block absmax scale; code =
 *               round(127 x / absmax), decode code * absmax / 127.
 *               Metadata: 1 float per block, {absmax}.
 *   FP32        the state is a plain float array (no metadata).
 *
 * Storage (section 4.4, Eq. al_memory): a state of n elements under block B
 * holds ceil(n/B)*B codes -- padded per tensor; padded codes are written as
 * 0 -- plus its metadata. al_code_bytes / al_meta_floats / al_state_bytes
 * give the sizes.
 *
 * Numeric contract. State arithmetic (decode, EMA, marginal means, factor
 * reconstruction, residuals) is binary64, each state rounded once to fp32
 * per step, sums exact to binary64 rounding; codes are decided from binary64
 * positions. The parameter update itself is fp32.
 *
 * Memory and execution. Every pointer argument is device memory owned by
 * the caller, except that tensor lists and config structs are host memory
 * read during the call. The library keeps no pointer after a call returns.
 * All device work is enqueued on `stream` (a hipStream_t; NULL = the null
 * stream) of the current device, whose memory the pointers are, in order; calls return without synchronizing. The library never
 * allocates device memory: each step takes a caller workspace whose size the
 * matching *_workspace_bytes query returns. Calls on distinct streams with
 * distinct buffers may run concurrently; calls that share a workspace or
 * state buffers must be ordered by the caller.
 *
 * Fresh state: all codes and metadata zero (code 0 is exact zero).
 *
 * Errors. Every call returns an al_status. All argument checks run on the
 * host before any HIP call, so a rejected call has enqueued nothing.
 * al_last_error() returns a thread-local description of the last failure on
 * the calling thread. Non-finite or negative values in a non-negative state
 * are not detected; their codes are unspecified.
 *
 * Alignment. Every device pointer must be 16-byte aligned (AL_EALIGN), except
 * the matrices of the al_act_*, al_norm_*, al_swiglu_*, al_linear_wgrad and
 * al_orthogonalize calls, and the matrices, ids and vectors of al_embed_* and
 * al_linear_xent (see there).
 */
#ifndef AL_H
#define AL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum al_status {
    AL_OK = 0,
    AL_EINVAL = 1,       /* bad argument: NULL, n < 0, bad codec/block/dtype, rows*cols mismatch */
    AL_EALIGN = 2,       /* a device pointer is not 16-byte aligned */
    AL_EWORKSPACE = 3,   /* workspace missing or smaller than the query returned */
    AL_EUNSUPPORTED = 4, /* a valid combination the library does not implement */
    AL_EHIP = 5          /* a HIP runtime call or launch failed */
} al_status;

typedef enum al_codec {
    AL_CODEC_FP32 = 0,
    AL_CODEC_AL8 = 1,
    AL_CODEC_AL16 = 2,
    AL_CODEC_UF8 = 3
} al_codec;

typedef enum al_dtype { AL_DTYPE_F32 = 0, AL_DTYPE_BF16 = 1 } al_dtype;

/* Which code a state gets ("representation and state policy", section 4.3).
 * block: 64, 128, 256, 512, 1024 or 2048 (ignored for FP32).
 * log_floor: l_floor of Eq. al_bounds (AL codecs only); the optimizer path
 * supplies it, typically log2 of its squared numerical floor (section 4.1). */
typedef struct al_state_spec {
    int32_t codec;
    int32_t block;
    float log_floor;
} al_state_spec;

/* One parameter tensor and its optimizer state buffers.
 * rows, cols: the row-major shape; a 1-D tensor has rows == 1 (such tensors,
 * and any tensor with rows == 1, keep an unfactored second moment in `v`).
 * param: rows*cols fp32, updated in place. grad: rows*cols of the call's
 * grad dtype.
 * m, m_meta:       momentum (AdamW, CAME).
 * v, v_meta:       dense second moment (AdamW), or the unfactored second
 *                  moment of a rows == 1 tensor (Adafactor, CAME).
 * vr/vc (+meta):   factored second moment, row (len rows) / column (len cols)
 *                  statistics (Adafactor, CAME; rows > 1 only).
 * cr/cc (+meta):   CAME factored confidence, row / column (rows > 1 only).
 * Slots a path does not use must be NULL. Metadata pointers are NULL for
 * FP32 states. */
typedef struct al_tensor {
    float* param;
    const void* grad;
    int64_t rows;
    int64_t cols;
    void* m;
    float* m_meta;
    void* v;
    float* v_meta;
    void* vr;
    float* vr_meta;
    void* vc;
    float* vc_meta;
    void* cr;
    float* cr_meta;
    void* cc;
    float* cc_meta;
} al_tensor;

/* AdamW (section 3.1, Eq. adam_update; decoupled weight decay and bias
 * corrections as in PyTorch AdamW). m: UF8 (block 256) or FP32.
 * v: AL8, AL16 or FP32. */
typedef struct al_adamw_cfg {
    double lr, beta1, beta2, eps, weight_decay;
    int32_t grad_dtype;
    int32_t reserved;
    al_state_spec m, v;
} al_adamw_cfg;

/* Flags of the factored steps (al_adafactor_cfg / al_came_cfg .flags).
 * AL_FLAG_EXACT_SUMS: every row and column mean behind the factored states is
 * recomputed with exact sums (slow). The default path already yields the same
 * fp32 states bit for bit -- its fast sums are kept only where they provably
 * round the same way -- so this flag is a check of that path, not a
 * different result. */
#define AL_FLAG_EXACT_SUMS 1

/* Adafactor (factored second moment, section 3.1): beta2_t = 1 - t^decay_rate,
 * G2 = g^2 + eps1, R/C = EMA of row/column means of G2, update
 * u = g / sqrt(R_i C_j / mean(R)), clipped by max(1, RMS(u)/clip_threshold);
 * no first moment, no relative step, no parameter scaling.
 * v: AL8, AL16 or FP32 for R, C and 1-D v. flags: 0 or AL_FLAG_EXACT_SUMS. */
typedef struct al_adafactor_cfg {
    double lr, eps1, clip_threshold, decay_rate, weight_decay;
    int32_t grad_dtype;
    int32_t flags;
    al_state_spec v;
} al_adafactor_cfg;

/* CAME (confidence-guided factored optimizer, section 3.1): factored V as
 * Adafactor with a constant beta2 and no bias correction; clipped update
 * uhat; m = EMA(beta1) of uhat; residual (uhat - m)^2 + eps2 feeds factored
 * confidence R', C' (EMA beta3); update m / sqrt(R'_i C'_j / mean(R')).
 * 1-D tensors: unfactored v, update = m, no confidence.
 * m: UF8 (block 256) or FP32; v and conf: AL8, AL16 or FP32.
 * flags: 0 or AL_FLAG_EXACT_SUMS. */
typedef struct al_came_cfg {
    double lr, beta1, beta2, beta3, eps1, eps2, clip_threshold, weight_decay;
    int32_t grad_dtype;
    int32_t flags;
    al_state_spec m, v, conf;
} al_came_cfg;

/* APOLLO, the projected-state path (section 3.1: first and second moments
 * kept in a low-rank projection of the gradient derive a channel-wise scale
 * of the original gradient; section 6 setup: rank 256, channel-wise scaling,
 * projection refreshed every 200 steps; Table 4: UF8 momentum, AL8 second
 * moment). A rows x cols tensor has C = max(rows, cols) channels of
 * L = min(rows, cols) inputs: rows >= cols projects the columns (channel c is
 * row c), otherwise the rows (channel c is column c). Per step:
 *   R   = fl32(A Pi) in binary64, A = G (rows >= cols) or G^T as C x L,
 *         Pi = proj (L x rank, row-major fp32; the caller draws it, N(0, 1/rank),
 *         and refreshes it every gap steps);
 *   m, v: the AdamW moments of R (rank * C elements, channel-major: element
 *         c * rank + k), with AdamW's codes, bias corrections and eps; the
 *         direction Rt = (m / bc1) / (sqrt(v / bc2) + eps) is fp32;
 *   s_c = ||Rt_c|| / (||R_c|| + 1e-8), G~ = G with channel c scaled by s_c;
 *   limiter (gamma > 0): from step 2, lam = max(||G~|| / (*norm_state + 1e-8),
 *         gamma) / gamma and *norm_state = fl32(||G~|| / lam); at step 1
 *         lam = 1 and *norm_state = fl32(||G~||);
 *   param = fl32(param (1 - lr wd) - lr g (s_c / lam)), binary64.
 * The token embedding, LM head and 1-D tensors are not projected: they take
 * al_adamw_step with the same codes. With more columns than rows,
 * min(rows - 1, 15) rows of the gradient must span less than 4 GiB (about 71
 * million fp32 columns; AL_EUNSUPPORTED beyond). */
typedef struct al_apollo_tensor {
    float* param;
    const void* grad;
    int64_t rows;
    int64_t cols;
    const float* proj; /* L x rank fp32 */
    void* m;           /* projected momentum, rank * C elements */
    float* m_meta;
    void* v;           /* projected second moment, rank * C elements */
    float* v_meta;
    float* norm_state; /* 1 float: the limiter's last update norm (unused when gamma <= 0) */
} al_apollo_tensor;

/* rank: 64, 128 or 256. gamma: the limiter's growth bound (<= 0: no limiter).
 * m: UF8 (block 256) or FP32; v: AL8, AL16 or FP32. */
typedef struct al_apollo_cfg {
    double lr, beta1, beta2, eps, weight_decay, gamma;
    int32_t rank;
    int32_t grad_dtype;
    al_state_spec m, v;
} al_apollo_cfg;

/* Library version string, e.g. "0.1.0 gfx950". */
const char* al_version(void);

/* Thread-local text of the last failure on this thread ("" if none). */
const char* al_last_error(void);

/* Storage accounting (section 4.4). Bytes of the code array of an n-element
 * state (padded to whole blocks), metadata floats, and their total in bytes.
 * Return -1 for an invalid codec, block or n < 0. */
int64_t al_code_bytes(int32_t codec, int64_t n, int32_t block);
int64_t al_meta_floats(int32_t codec, int64_t n, int32_t block);
int64_t al_state_bytes(int32_t codec, int64_t n, int32_t block);

/* Encode n fp32 values x (non-negative for AL codecs) into codes + meta
 * (Eq. al_bounds and al_quant for AL8/AL16; section 4.3 for UF8).
 * codec: AL8, AL16 or UF8. codes: al_code_bytes(codec, n, block) bytes;
 * meta: al_meta_floats(codec, n, block) floats. log_floor is ignored for
 * UF8. n == 0 is a no-op. */
al_status al_quantize(int32_t codec, const float* x, int64_t n, int32_t block, float log_floor,
                      void* codes, float* meta, void* stream);

/* Decode n values (Eq. al_dequant for AL8/AL16; section 4.3 for UF8) into
 * out (n floats). */
al_status al_dequantize(int32_t codec, const void* codes, const float* meta, int64_t n,
                        int32_t block, float* out, void* stream);

/* Workspace size (bytes) that al_adamw_step needs for this tensor list and
 * config: the step's tensor descriptor table (64 + 8 bytes per non-empty
 * tensor, 256-byte aligned parts). 0 for a list with no elements. */
al_status al_adamw_workspace_bytes(const al_tensor* tensors, int32_t nt, const al_adamw_cfg* cfg, size_t* bytes);

/* One fused AdamW step over a list of nt tensors (section 3.1, Eq.
 * adam_update, with PyTorch AdamW's decoupled weight decay and bias
 * corrections; codes of section 4). step = the 1-based step count after
 * increment. One pass over HBM: read p, g, m, v (+meta), write p, m, v
 * (+meta). Uses per tensor: param, grad, m, m_meta, v, v_meta; the other
 * slots must be NULL. ws: device workspace of at least
 * al_adamw_workspace_bytes, 256-byte aligned (AL_EWORKSPACE otherwise); the
 * call writes the descriptor table there on the stream (small copy kernels;
 * the descriptors of up to 8 tensors travel in the step kernel's arguments
 * instead) and runs the whole list in one launch of the step kernel (several
 * for lists beyond 2^32 chunks of 512-2048 elements). ws is scratch: its
 * contents need not survive between calls, and calls that share it must be
 * ordered on one stream. */
al_status al_adamw_step(const al_tensor* tensors, int32_t nt, const al_adamw_cfg* cfg, int64_t step, void* ws,
                        size_t ws_bytes, void* stream);

/* For callers that cannot allocate device memory or hand over a workspace
 * (code under HIP graph capture, tight serving loops, harnesses that forbid
 * allocation): al_adamw_step without ws, same arguments otherwise and the
 * same results bit for bit (the same kernels). The descriptor table lives in
 * a fixed device array of the library instead, 288 KiB per GPU, held until
 * the process ends: at most 4096 non-empty tensors per call (more:
 * AL_EUNSUPPORTED, before any HIP call). The first call on a device looks up
 * that array's address once (hipGetSymbolAddress). The call allocates
 * nothing (no hipMalloc, hipFree or host heap). Every call on one GPU writes
 * the same array: calls in order on one stream are safe, calls that may
 * overlap on one GPU (several streams or threads) race and must be
 * serialized by the caller. */
al_status al_adamw_step_noalloc(const al_tensor* tensors, int32_t nt, const al_adamw_cfg* cfg, int64_t step,
                                void* stream);

/* Workspace size (bytes) that al_adafactor_step / al_came_step need for this
 * tensor list and config. A part of a list (frozen tensors left out, one
 * parameter group) never needs more than the list, so one workspace sized for
 * the whole list serves every part of it. */
al_status al_adafactor_workspace_bytes(const al_tensor* tensors, int32_t nt,
                                       const al_adafactor_cfg* cfg, size_t* bytes);
al_status al_came_workspace_bytes(const al_tensor* tensors, int32_t nt, const al_came_cfg* cfg,
                                  size_t* bytes);

/* One Adafactor step over nt tensors. Uses per tensor: param, grad and
 * (rows > 1) vr, vr_meta, vc, vc_meta or (rows == 1) v, v_meta.
 * ws: device workspace of at least the queried size, 256-byte aligned. */
al_status al_adafactor_step(const al_tensor* tensors, int32_t nt, const al_adafactor_cfg* cfg,
                            int64_t step, void* ws, size_t ws_bytes, void* stream);

/* One CAME step over nt tensors. Uses per tensor: param, grad, m, m_meta and
 * (rows > 1) vr, vc, cr, cc with metadata or (rows == 1) v, v_meta. */
al_status al_came_step(const al_tensor* tensors, int32_t nt, const al_came_cfg* cfg,
                       int64_t step, void* ws, size_t ws_bytes, void* stream);

/* Workspace size (bytes) that al_apollo_step needs for this list and config:
 * per tensor R (rank * C floats), below rank 256 also Rt (as many floats),
 * per-channel binary64 sums, and the descriptor tables of the step's
 * launches. */
al_status al_apollo_workspace_bytes(const al_apollo_tensor* tensors, int32_t nt, const al_apollo_cfg* cfg,
                                    size_t* bytes);

/* One APOLLO step over nt projected tensors (rows, cols >= 1). Kernels, in
 * stream order: the binary64 projection on the matrix cores (also sums of
 * squares per channel of G), the fused AdamW step over the projected moments
 * (fp32 R as its gradient, lr 1, no weight decay; at rank 256 it forms the
 * channel scales itself, one channel per 256-element sub-tile, from the
 * direction it computes; below rank 256 it writes the direction as its
 * parameter Rt in the workspace and a separate pass forms the channel
 * scales), the limiter per tensor, and the parameter update. ws: device
 * workspace of at least the queried size, 256-byte aligned. */
al_status al_apollo_step(const al_apollo_tensor* tensors, int32_t nt, const al_apollo_cfg* cfg, int64_t step,
                         void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Orthogonalised updates. O(G) replaces the singular values of a matrix by
 * numbers near 1, by products alone (Newton-Schulz):
 *   X = G / (|G| + eps), |G| the Frobenius norm, then `steps` times
 *   X <- a X + (b A + c A A) X, A = X X^T        (rows <= cols)
 *   X <- a X + X (b A + c A A), A = X^T X        (rows > cols).
 * A zero matrix gives zeros (also with eps = 0), one that holds an infinity or a NaN gives NaN.
 * parts: what X, A and b A + c A A are held in between the products, whose
 * sums are fp32: 1 = one fp16 number each (11 bits: the result is 1e-3 to 3.5e-3 off for normal matrices, up to 4e-3 where singular values
 * fall as 1 / k), 2 = the sum of two (22 bits; 1e-6 to 6e-6, of the fp32 sums too; three products for one). Both hold an element of X to no less than 2^-35 of X's norm: in one part
 * elements below 2^-24 of the norm have fewer bits, in two those below 2^-13. Where that is less work, two steps are taken at
 * once, as X <- a a X + D X with a second A = M A M, M = a I + b A + c A A (the same polynomial of A, other roundings). |G| is a binary64 sum in a fixed order:
 * the same call gives the same bits. (How the products are cut, and whether steps go two at a time, is chosen by the sizes that go together: see al_muon_step.)
 * a, b, c: for singular values of at most 1 to begin with, those of X must stay within 4 and those of b A + c A A within
 * 128 (AL_EINVAL; a = 3.4445, b = -4.7750, c = 2.0315 are usual). steps: 1 to 64.
 * rows, cols up to 2^21, the smaller of them up to 2^16, 2^33 elements (AL_EUNSUPPORTED). */
typedef struct al_ortho_cfg {
    double a, b, c, eps;
    int32_t steps, parts;
} al_ortho_cfg;

/* Workspace bytes of al_orthogonalize. */
al_status al_orthogonalize_workspace_bytes(int64_t rows, int64_t cols, const al_ortho_cfg* cfg, size_t* bytes);

/* out = O(x), x of dtype and out of out_dtype (al_dtype): rows x cols, element (i, j) at i * ld + j, any alignment of the element
 * type and any ld >= cols (ignored for rows <= 1). out may be x itself (same type and ld); they must not overlap otherwise. ws: at least
 * the queried bytes, 256-byte aligned. */
al_status al_orthogonalize(int32_t dtype, const void* x, int64_t ldx, int64_t rows, int64_t cols, const al_ortho_cfg* cfg, int32_t out_dtype,
                           void* out, int64_t ldout, void* ws, size_t ws_bytes, void* stream);

/* The step of a matrix by its orthogonalised momentum (the Muon optimizer):
 *   m = fl32(beta m + (1 - beta) g), u = m or, with nesterov, fl32(beta m + (1 - beta) g),
 *   param = fl32(param (1 - lr wd) - lr s O(u))
 * in binary64 but for O (ortho), whose result is fp32; m is coded as m (UF8, block 256) or kept as FP32, and u is formed from m before it
 * is coded. s by `scale`: 0 = 1, 1 = sqrt(max(1, rows / cols)), 2 = 0.2 sqrt(max(rows, cols)) (the RMS of an AdamW update). */
typedef enum al_muon_scale { AL_MUON_SCALE_NONE = 0, AL_MUON_SCALE_SPECTRAL = 1, AL_MUON_SCALE_RMS = 2 } al_muon_scale;
typedef struct al_muon_cfg {
    double lr, beta, weight_decay;
    al_ortho_cfg ortho;
    int32_t nesterov, scale;
    int32_t grad_dtype;
    int32_t reserved;
    al_state_spec m;
} al_muon_cfg;

/* Workspace size (bytes) that al_muon_step needs for this tensor list and config. A part of a list never needs more than the list.
 * Up to 32 matrices of any shapes share launches, longest sides first, while they take no more than 2^30 bytes (one matrix at least): for each an fp32
 * update or X twice, and A and b A + c A A, 2 or 4 bytes an element, sides padded to multiples of 64. */
al_status al_muon_workspace_bytes(const al_tensor* tensors, int32_t nt, const al_muon_cfg* cfg, size_t* bytes);

/* One step over nt matrices (rows, cols >= 1; a list's 1-D tensors, embedding and head take al_adamw_step). Uses per tensor: param, grad, m, m_meta;
 * the other slots must be NULL, and no two tensors may share memory. step: the 1-based step count, which the update does not depend on. m's codes are al_quantize's, but for values half way between
 * two codes (the position is x fl(127 fl(1 / absmax)) in binary64 here). Per group: the momentum pass (which also sums the squares of u), the norms of matrices of more than 2^23
 * elements, u into 16-bit parts with its norm, and three products a step of O, the last of which ends in the parameters. A matrix's parameters may differ by
 * O's roundings with the list that it is stepped in: the group's sizes choose the tiles and whether steps go two at a time. Its momentum does not. Processes that have to agree bit for bit step
 * the same lists. ws: device workspace
 * of at least the queried size, 256-byte aligned. */
al_status al_muon_step(const al_tensor* tensors, int32_t nt, const al_muon_cfg* cfg, int64_t step, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Activations in 8 bits, and the operators that save and use them: the code
 * itself, layer / RMS norm and their backward pass, the gated activation
 * silu(gate) * up and its backward pass, and a linear layer's weight gradient
 * from its saved input. The weight gradients come out in the types the
 * optimizer steps read (al_tensor.grad).
 *
 * Matrices. rows x cols, one row per token, element (i, j) at i * ld + j with
 * ld >= cols (ignored for rows <= 1). fp32 or bf16; any alignment of the
 * element type and any ld will do (16-byte aligned rows are fastest). Outputs
 * must not overlap inputs except where an entry point says so. rows up to
 * 2^31 - 1, cols up to 2^31 - 8193, rows * ld up to 2^48.
 *
 * Activation code E8 (block: 32, 64 or 128 columns; blocks do not cross rows;
 * the last block of a row may be short). For a block with largest magnitude a:
 *   E = max(1, floor(log2 a) + 121)        (a = 0: E = 1)
 *   code = clamp(rint(x 2^(127 - E)), -127, 127), ties to even
 *   decode: code * 2^(E - 127), exact in bf16 and fp32.
 * The step 2^(E - 127) is between a / 128 and a / 64, so a decoded value is
 * within half a step of x (up to one step where |x| > 127 steps). A block
 * holding a NaN or an infinity has E = 255 and codes 0, and decodes to NaN
 * throughout. codes: int8, rows of nb * block bytes, nb = ceil(cols / block),
 * columns past cols coded 0; exps: uint8, rows of nb bytes. Both 16-byte
 * aligned.
 *
 * Sums and statistics are fp32 and independent of scheduling: every result
 * repeats bit for bit. */
typedef enum al_norm_kind { AL_NORM_LAYER = 0, AL_NORM_RMS = 1 } al_norm_kind;

/* Bytes of the codes and of the exponents of a rows x cols matrix. -1 for a
 * bad block, a negative size or one past the limits above. */
int64_t al_act_code_bytes(int64_t rows, int64_t cols, int32_t block);
int64_t al_act_exp_bytes(int64_t rows, int64_t cols, int32_t block);

/* Encode x (dtype: al_dtype) into codes and exps, and decode them into out. */
al_status al_act_quantize(int32_t dtype, const void* x, int64_t ld, int64_t rows, int64_t cols, int32_t block,
                          void* codes, void* exps, void* stream);
al_status al_act_dequantize(const void* codes, const void* exps, int64_t rows, int64_t cols, int32_t block,
                            int32_t dtype, void* out, int64_t ld, void* stream);

/* Norm over each row: xhat = (x - mean) rstd, rstd = (var + eps)^-1/2 with the
 * biased variance about the mean (AL_NORM_RMS: mean = 0, var = the mean
 * square), y = xhat gamma + beta. gamma, beta: cols floats, NULL = 1 and 0;
 * beta only for AL_NORM_LAYER. x and y have dtype; y may be x itself (same
 * ld). eps >= 0, taken as fp32; a row without variance needs eps > 0, and a row whose squares add up to
 * more than fp32 holds has rstd = 0. mean (AL_NORM_LAYER only, else NULL) and rstd: rows floats, NULL where not
 * wanted. codes, exps: the E8 code of xhat, both NULL where it is not saved
 * (block is then ignored). xhat is what a backward pass needs of x, and a
 * linear layer that reads y needs nothing else either (al_linear_wgrad). */
al_status al_norm_forward(int32_t kind, int32_t dtype, const void* x, int64_t ldx, int64_t rows, int64_t cols,
                          double eps, const float* gamma, const float* beta, void* y, int64_t ldy, float* mean,
                          float* rstd, int32_t block, void* codes, void* exps, void* stream);

/* Workspace bytes of an al_norm_backward that is asked for dgamma or dbeta:
 * partial sums of the weight gradients. */
al_status al_norm_backward_workspace_bytes(int32_t kind, int32_t dtype, int64_t rows, int64_t cols, size_t* bytes);

/* Backward pass of al_norm_forward. With a = dy gamma and n = cols,
 *   dx = rstd (a - sum(a) / n [AL_NORM_LAYER] - xhat sum(a xhat) / n) + add
 *   dgamma = sum over rows of dy xhat, dbeta = sum over rows of dy.
 * xhat comes from x, mean and rstd (codes = exps = NULL), or from its E8 code
 * (x = mean = NULL). dy, x, add and dx have dtype; add (NULL: none) is the
 * gradient that reaches x past the norm; dx may be add itself (same ld).
 * dgamma, dbeta: cols values of grad_dtype, NULL where not wanted (dbeta only
 * for AL_NORM_LAYER). ws: at least the queried bytes, 256-byte aligned, may be NULL
 * when neither is wanted. rows == 0 writes zero weight gradients. */
al_status al_norm_backward(int32_t kind, int32_t dtype, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                           const float* mean, const float* rstd, int32_t block, const void* codes, const void* exps,
                           int64_t rows, int64_t cols, const float* gamma, const void* add, int64_t ldadd, void* dx,
                           int64_t lddx, int32_t grad_dtype, void* dgamma, void* dbeta, void* ws, size_t ws_bytes,
                           void* stream);

/* h = silu(gate) * up, silu(g) = g / (1 + e^-g), in fp32, rounded once to
 * dtype; optionally the E8 codes of gate and up (all four pointers or none).
 * Here and in the backward pass 1 / (1 + e^-g) is within 2^-22 of its value
 * (relative) for fp32, within (|g| + 5) 2^-24 for bf16, and 0 where e^-g
 * overflows. */
al_status al_swiglu_forward(int32_t dtype, const void* gate, int64_t ldgate, const void* up, int64_t ldup,
                            int64_t rows, int64_t cols, void* h, int64_t ldh, int32_t block, void* gate_codes,
                            void* gate_exps, void* up_codes, void* up_exps, void* stream);

/* Backward pass from the codes: with s = 1 / (1 + e^-gate),
 *   dup = dh gate s, dgate = dh up s (1 + gate (1 - s)),
 * and optionally (h_codes, h_exps: both or none) the E8 code of the recomputed
 * h = gate s up, the input that the next linear layer's weight gradient needs. dgate and dup
 * may share a buffer (two column ranges of one matrix). */
al_status al_swiglu_backward(int32_t dtype, const void* dh, int64_t lddh, int64_t rows, int64_t cols, int32_t block,
                             const void* gate_codes, const void* gate_exps, const void* up_codes,
                             const void* up_exps, void* dgate, int64_t lddgate, void* dup, int64_t lddup,
                             void* h_codes, void* h_exps, void* stream);

/* Workspace bytes of al_linear_wgrad (partial sums of products split over the
 * tokens, and of the bias gradient). */
al_status al_linear_wgrad_workspace_bytes(int32_t dtype, int64_t tokens, int64_t out_features, int64_t in_features,
                                          size_t* bytes);

/* Weight gradient of y = z W^T (+ bias), W out_features x in_features row-major, z = xhat gamma +
 * beta, xhat saved as an E8 code (tokens x in_features):
 *   dw[n][k] = gamma[k] sum_t dy[t][n] xhat[t][k] + beta[k] sum_t dy[t][n] + base[n][k]
 *   dbias[n] = sum_t dy[t][n]
 * dy: tokens x out_features of dtype. gamma, beta: in_features floats, NULL = 1 and 0 (a layer
 * that does not follow a norm has its own input as xhat). base, dw: packed
 * out_features x in_features of grad_dtype; base NULL = 0, base may be dw
 * itself (gradient accumulation). dbias: out_features values of grad_dtype or
 * NULL. The products are exact (both factors are bf16 numbers, an fp32 dy is three
 * of them but for bits below 2^-133, which are dropped) and summed in fp32 on the
 * matrix cores. tokens == 0: dw = base, dbias = 0.
 * out_features below 2^22, in_features below 2^29, at most 2^38 weights (AL_EUNSUPPORTED otherwise).
 * One launch where the outputs fill the device (beta or dbias take two more); fewer
 * outputs split the tokens, and a second launch adds the parts, and up to 16384
 * tokens those of dy's sums, in order. */
al_status al_linear_wgrad(int32_t dtype, const void* dy, int64_t lddy, const void* codes, const void* exps,
                          int32_t block, int64_t tokens, int64_t out_features, int64_t in_features,
                          const float* gamma, const float* beta, int32_t grad_dtype, const void* base, void* dw,
                          void* dbias, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * The two ends of a token model: the lookup of embeddings and its gradient,
 * and softmax cross entropy of a linear head with its gradients. Matrices as
 * for the activations above, except that the head's weight begins at a 16-byte
 * aligned address; weight gradients are packed, in the types the optimizer steps read. scale: finite in fp32.
 *
 * Token ids and targets: tokens values of index_dtype, one behind the other. An
 * id or a target below 0 or from vocab on stands for no token: its embedding is zero, and it takes part in no loss and no
 * gradient, whatever its row holds.
 *
 * Sums are fp32 and independent of scheduling: every result repeats bit for
 * bit. tokens and vocab up to 2^31 - 1; with a gradient of the table vocab up to 2^26, cols up to
 * 65535 * 1024 and floor(tokens / 32) below floor(2^23 / ceil(cols / 1024)) (AL_EUNSUPPORTED). */
typedef enum al_index { AL_INDEX_I32 = 0, AL_INDEX_I64 = 1 } al_index;

/* out[t] = scale table[ids[t]], in fp32, rounded once to out_dtype. table:
 * vocab x cols of table_dtype, out: tokens x cols. */
al_status al_embed_forward(int32_t table_dtype, const void* table, int64_t ldtable, int64_t vocab, int64_t cols, int32_t index_dtype,
                           const void* ids, int64_t tokens, double scale, int32_t out_dtype, void* out, int64_t ldout, void* stream);

/* Workspace bytes of al_embed_backward: the sorted tokens, and sums of every 32 of them. */
al_status al_embed_backward_workspace_bytes(int64_t tokens, int64_t vocab, int64_t cols, size_t* bytes);

/* Gradient of the table: dw[v] = base[v] + scale * sum of dy[t] over the tokens t with ids[t] = v, in the order of the tokens.
 * dy: tokens x cols of dtype. base, dw: packed vocab x cols of grad_dtype, 16-byte aligned; base NULL = 0, base may be dw itself
 * (gradient accumulation, or a head's gradient where the table is tied: then rows without a token are not touched). ws: at least the
 * queried bytes, 256-byte aligned. The tokens are sorted by id (runs of 1024, then up to 64 of them merged in a launch), sums over
 * 32 sorted tokens of one id are taken apart from the rows, and each row is written once. */
al_status al_embed_backward(int32_t dtype, const void* dy, int64_t lddy, int32_t index_dtype, const void* ids, int64_t tokens, int64_t vocab,
                            int64_t cols, double scale, int32_t grad_dtype, const void* base, void* dw, void* ws, size_t ws_bytes, void* stream);

/* Workspace bytes of al_linear_xent; dh, dw: whether these gradients are wanted. */
al_status al_linear_xent_workspace_bytes(int64_t tokens, int64_t hidden, int64_t vocab, int64_t ldw, int32_t want_dh, int32_t dh_dtype,
                                         int32_t want_dw, int32_t grad_dtype, size_t* bytes);

/* Softmax cross entropy of logits = h w^T (h: tokens x hidden, w: vocab x hidden, both bf16) against target, with its gradients, without
 * a tokens x vocab matrix:
 *   lse[t] = log sum over v of exp(logit[t][v]),  loss[t] = lse[t] - logit[t][target[t]]
 *   d[t][v] = scale weight[t] (exp(logit[t][v] - lse[t]) - [v = target[t]])
 *   dh = d w,  dw = d^T h + base                  (of scale * sum over t of weight[t] loss[t])
 * loss, lse: tokens floats, 0 for a token without a target, NULL where not wanted. weight: tokens floats, NULL = 1. dh: tokens x hidden of
 * dh_dtype; base, dw: packed vocab x hidden of grad_dtype, 16-byte aligned, base NULL = 0, base may be dw itself (dw NULL: base too); NULL where not wanted.
 * Products of bf16 numbers with fp32 sums; d is rounded to bf16 for a bf16 gradient and to the sum of two bf16 numbers (16 bits) for an fp32
 * one. Logits are taken once for the losses and, where a gradient is wanted, again, a piece of the vocabulary at a time: the workspace holds 2^26
 * elements of d (256 columns at least) and, with several pieces, dh in fp32; besides a copy of h, the statistics (8 bytes for each 64 columns, 32 in small calls, of up to 16384 tokens at a
 * time) and what products that are split over their sums leave, up to 256 MiB. Besides the logits' own fp32 sums a loss is as near for large logits as for small ones: it is taken from
 * differences to a row's largest, and nothing is rounded at the logits' size, but lse. A weight of minus infinity takes its row out of the softmax where h is positive there (dh then has no value).
 * w: 16-byte aligned; ldw or hidden that is no multiple of 8 costs a copy of w in the
 * workspace. tokens * vocab up to 2^38, tokens * hidden and vocab * hidden up to 2^34, tokens and vocab
 * up to 2^24, hidden up to 2^22 (AL_EUNSUPPORTED). */
al_status al_linear_xent(const void* h, int64_t ldh, const void* w, int64_t ldw, int64_t tokens, int64_t hidden, int64_t vocab,
                         int32_t index_dtype, const void* target, const float* weight, double scale, float* loss, float* lse, int32_t dh_dtype, void* dh,
                         int64_t lddh, int32_t grad_dtype, const void* base, void* dw, void* ws, size_t ws_bytes, void* stream);

/* Diagnostic: evaluate, elementwise on the device, a math primitive the
 * codes rely on, so tests can bound it against the host: fn 0 = hardware
 * fp32 log2 of (float)x (the fast code position uses it on mantissas in
 * [1/2, 1)), 1 = the binary64 exp2 used by decoding, 2 = binary64 log2 (block
 * endpoints and near-boundary positions), 3 = binary64 sqrt, 4 = 1/sqrt(x)
 * (factored second-moment reconstruction), 5 = x / 127 and 6 = 127 / x by
 * the division-free sequences of the UF8 code (exact for x a finite fp32
 * value, x > 0 for 6), 7 = fl32(x / 3) by the multiply-and-check quotient of
 * the clipped updates, 8 = the binary64 log2 of (float)x that fits the AdamW
 * step's second-moment blocks (x > 0), 9 = the clipped update of the CAME
 * passes, fl32(fl64(fl64(r c) x) / d) for fixed binary64 r, c, d from the
 * quotient with fl64(1 / d) folded into r and the decision test over eight
 * consecutive inputs (n a multiple of 8), 10 = the same for bf16 values x with
 * r = d = 1 and c = 0x1.00008c3a4f91dp7 (about 2^7 (1 + 2^-17)), where the residual pass's range test is
 * known to pass and only the midpoint test runs. x, out: n doubles (device). */
al_status al_diag_math(int32_t fn, const double* x, int64_t n, double* out, void* stream);

/* The AL8 levels of the fused AdamW step's split-table decode (section 4.1,
 * Eq. al_dequant): for each of nblocks blocks with metadata {l_min, delta}
 * (fp32 pairs, the AL8 layout), out[255 b + q - 1] is the binary64 value of
 * the level of code q = 1..255 before its rounding to fp32, computed by the
 * same device functions as the step: kind 0 = two factors (blocks of 128 and
 * more), 1 = three factors (blocks of 64). meta, out: device, 16-byte
 * aligned; out holds 255 nblocks doubles. For measuring the decode's error
 * against 2^E. */
al_status al_diag_levels(int32_t kind, const float* meta, int64_t nblocks, double* out, void* stream);

/* Sums of squares behind the relative update error of section 3.2 (Eq.
 * update_error): with U = a, U_ref = b (two updates of the same n elements,
 * fp32 device arrays), writes out[0] = sum_i (a_i - b_i)^2 and out[1] =
 * sum_i b_i^2, each term formed in binary64 and summed double-double (fixed
 * order: the result is reproducible and within an ulp of the exact sum).
 * out: device buffer of at least AL_DIFF_NORMS_OUT doubles, 16-byte aligned;
 * out[2 ..] is scratch. n = 0 writes zeros. Enqueued on stream; allocates
 * nothing. The error is sqrt(out[0]) / (sqrt(out[1]) + eps). */
#define AL_DIFF_NORMS_OUT 4098
al_status al_diff_norms(const float* a, const float* b, int64_t n, double* out, void* stream);

/* Diagnostic: how al_linear_wgrad cuts a product, a rule on its sizes alone:
 * plan[0] = width of the tiles of outputs (64, 128 or 256), plan[1] = splits
 * of the tokens (1: one launch), plan[2] = slabs that dy's sums are taken in,
 * plan[3] = 1 where these are taken in the product's own launch, else 0. (Rows of dy
 * that are 2^25 elements apart, or code rows of 2^26 bytes, are taken in
 * 64-wide tiles with the same splits.) plan: host memory. No HIP call; the
 * sizes that al_linear_wgrad refuses are refused. For tests that have to
 * reach a kernel. */
al_status al_diag_wgrad_plan(int32_t dtype, int64_t tokens, int64_t out_features, int64_t in_features, int32_t plan[4]);

/* Diagnostic: streaming rates of the fused AdamW byte mix. Reads p (n fp32),
 * g (n bf16), m and v (n bytes each) and writes p, m, v with no optimizer
 * arithmetic. mode selects the access shape:
 *   0, 1  the shape of al_adamw_step at block 2048 (one 2048-element chunk per
 *         wavefront in two load phases, 4 consecutive elements per lane,
 *         XCD-contiguous workgroup order); mode 1 uses non-temporal loads and stores. Writes
 *         p[4i] += g[4i], p[4i+3] += g[4i+3] (g as bf16), m ^= v, v += 1 per
 *         byte. n must be a multiple of 2048.
 *   2, 3  the fastest shape found for the mix (one 4096-element chunk per
 *         wavefront, 16 bytes per lane from every stream, all loads before any
 *         store, non-temporal): a reference rate, not the step's layout.
 *         Writes p += 1, m ^= v, v += 1 per byte; g is only read. n must be a
 *         multiple of 4096.
 * v += 1 carries into the next byte where a byte is 0xFF. Timing it gives the
 * achievable HBM bandwidth for the step's exact byte mix. Enqueued on stream;
 * allocates nothing. AL_EINVAL for a bad mode, n or NULL buffer, AL_EALIGN
 * for a buffer not 16-byte aligned. */
al_status al_diag_stream(int32_t mode, float* p, const void* g, void* m, void* v, int64_t n, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* AL_H */
