/*
 * jd.h - C ABI of the judge-decoding verification step for NVIDIA B200 (sm_100a).
 *
 * One call, jd_verify, performs what follows every target-model forward over a block of M
 * draft tokens in judge decoding (arXiv 2501.19309):
 *   1. LM-head projection of the target's last-layer embeddings, L = H W^T      (Sec. 3.1, Eq. 2)
 *   2. softmax over the vocabulary, p_j = softmax(L[j,:]), and q_j = softmax(draft logits)
 *   3. the standard speculative-sampling test u_j q_j[x_j] < p_j[x_j]            (Sec. 3.1, Eq. 4)
 *      and the judge test sigmoid(w . H[b,j+1] + b0) > tau                      (Sec. 4.1 "Inference")
 *   4. mask = standard OR judge (or one of them), accepted prefix length        (Sec. 4.1; App. B.2)
 *   5. the next token: from normalised max(0, p - q) at the first rejection, from the extra
 *      row p_M after a fully accepted block                                     (Sec. 3.1, after Eq. 4)
 * The logits exist only on chip; they are never written to device memory unless the
 * test-only logits_debug pointer is set.
 *
 * Conventions
 *   - Indices are 0-based. Row j of H[b] (j = 0..M) yields p_j, the target distribution of draft
 *     slot j; row 0 belongs to the last context token, row j >= 1 to draft token j-1. The judge
 *     score of draft token j is read from row j+1. Row M also yields the bonus distribution.
 *   - All tensors are dense, row-major (last index fastest).
 *   - Unless a function says "host", every data pointer is a DEVICE pointer owned by the caller.
 *     The library never frees or keeps caller memory, except that W and w_judge given to
 *     jd_set_head are borrowed until the next jd_set_head or jd_destroy.
 *   - jd_verify is asynchronous on the given CUDA stream and never synchronises it.
 *   - No function throws, prints or exits; every failure is a jd_status_t.
 *   - Uniforms: Philox4x32-10, key = (seed low word, seed high word), counter =
 *     (b, slot, stream, 0), first output word, u = (word >> 8) * 2^-24. stream 0 is the
 *     acceptance draw of slot j, stream 1 the token draw at slot accept_len[b].
 */
#ifndef JD_H_
#define JD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  JD_OK = 0,
  JD_ERR_INVALID_ARG = 1, /* null pointer, size out of range, bad enum, misaligned pointer */
  JD_ERR_UNSUPPORTED = 2, /* shape or dtype that no kernel variant covers */
  JD_ERR_ARCH = 3,        /* the current device is not compute capability 10.x */
  JD_ERR_ALLOC = 4,       /* device or host allocation failed */
  JD_ERR_CUDA = 5,        /* a CUDA runtime or driver call failed */
  JD_ERR_TIMEOUT = 6,     /* device status: a bounded wait inside a kernel ran out */
  JD_ERR_BAD_TOKEN = 7,   /* device status: a draft token was outside [0, V) and was clamped */
  JD_ERR_PAGES = 8,       /* device status: a cache has too few free pages, or a sequence too many; nothing was reserved */
  JD_ERR_BAD_INDEX = 9    /* device status: a slot, page, node or length of a cache call was out of range, named twice or
                             not held; that entry was skipped */
} jd_status_t;

/* Storage type of the head. F32 / BF16: W, H and w_judge all have that type. FP8_E4M3: W holds
 * FP8 E4M3 codes (1 sign, 4 exponent bits with bias 7, 3 mantissa bits, no infinities) with one
 * float32 scale per vocabulary row, registered with jd_set_head_fp8; H and w_judge are bf16. */
typedef enum { JD_DTYPE_F32 = 0, JD_DTYPE_BF16 = 1, JD_DTYPE_FP8_E4M3 = 2 } jd_dtype_t;

/* Which tests form the accept mask (Sec. 4.1 "Inference"): the standard test alone (Eq. 4),
 * the judge alone, or their logical OR (the paper's judge decoding). */
typedef enum { JD_MODE_STANDARD = 0, JD_MODE_JUDGE = 1, JD_MODE_JUDGE_OR_STANDARD = 2 } jd_mode_t;

/* Distribution of the token drawn at the first rejected slot a < M.
 * RESIDUAL: normalised max(0, p_a - q_a), the form under which the standard test is lossless;
 *           an identically zero residual falls back to p_a.
 * TARGET_P: p_a itself, which is how Sec. 3.1 words the correction when read literally.
 * After a fully accepted block the token always comes from p_M. */
typedef enum { JD_RESAMPLE_RESIDUAL = 0, JD_RESAMPLE_TARGET_P = 1 } jd_resample_t;

/* How the standard (non-judge) test decides, and how the next token is chosen.
 * SAMPLING: the stochastic test of Eq. 4 with the residual / bonus draw described above.
 * TOPK:     deterministic verification: the candidate passes iff it is among the top_k highest-valued
 *           entries of p_j (Sec. 5.1 "Training-free baseline"); top_k = 1 is greedy verification
 *           (acceptance against a greedily decoded target, Sec. 3.2), top_k = V accepts everything. The next
 *           token is the target's greedy token argmax p_a, at a rejection and after a full block.
 *           Equal logits rank by token id (lower id first); the batched variant compares the row against
 *           a float32 dot product for the candidate, so there an entry equal to the candidate's logit to
 *           within float32 summation order may rank on either side of it. No uniform is drawn; the
 *           draft logits only feed the q_draft output. */
typedef enum { JD_RULE_SAMPLING = 0, JD_RULE_TOPK = 1 } jd_rule_t;

/* Normalisation applied to the rows of H in front of the LM head. The paper's judge takes the last
 * embedding ahead of the model's final RMS norm and LM head (Sec. 4.1 "Model design and training"):
 * with JD_NORM_RMS the logits are W . (H[b,j] / sqrt(mean_k H[b,j,k]^2 + rms_eps)) while the judge
 * dot product still uses H[b,j+1] as given. The norm's gain vector is expected folded into W. */
typedef enum { JD_NORM_NONE = 0, JD_NORM_RMS = 1 } jd_norm_t;

/* Kernel family used by jd_verify. AUTO picks the fastest one that supports the shape. */
typedef enum {
  JD_VARIANT_AUTO = 0,
  JD_VARIANT_SIMT = 1,   /* CUDA-core reference pipeline: any shape; f32, bf16 or FP8 head */
  JD_VARIANT_FUSED = 2,  /* one persistent tcgen05/TMA kernel, logits parked in tensor memory;
                            bf16 with d % 64 == 0 or FP8 head with d % 128 == 0, B*(M+1) <= 96, V
                            small enough for every CTA to keep its vocabulary tiles on chip
                            (128256 fits on 148 SMs) */
  JD_VARIANT_BATCHED = 3 /* tcgen05 GEMM with fused statistics + second pass over the selected
                            rows (one launch per 64 sequences beyond 96); same dtypes and d as
                            the fused variant, any number of rows and sequences */
} jd_variant_t;

typedef struct {
  int32_t max_B;    /* largest number of sequences per call, >= 1 */
  int32_t max_M;    /* largest number of draft tokens per sequence, >= 1 */
  int32_t d;        /* embedding width */
  int32_t V;        /* vocabulary size */
  int32_t dtype;    /* jd_dtype_t: storage type of W, H and w_judge */
  int32_t device;   /* CUDA device ordinal the handle lives on */
} jd_config_t;

typedef struct jd_handle_s* jd_handle_t;

typedef struct {
  int32_t B;                   /* sequences in this call, 1..max_B */
  int32_t M;                   /* draft tokens per sequence, 1..max_M */
  const void* H;               /* [B, M+1, d] embeddings, dtype of the handle (bf16 for an FP8 head),
                                  16-byte aligned */
  const int32_t* draft_tokens; /* [B, M] drafted token ids x_j in [0, V) */
  const float* draft_logits;   /* [B, M, V] draft-model logits; q_j = softmax at temperature 1. 4-byte aligned
                                  like every int32 / float array here; a 16-byte aligned base with V % 4 == 0
                                  lets the kernels use 16-byte loads, anything else takes 4-byte loads */
  float tau;                   /* judge threshold in [0, 1]; accept iff score > tau (strict) */
  uint64_t seed;               /* Philox key */
  int32_t mode;                /* jd_mode_t */
  int32_t resample;            /* jd_resample_t */
  int32_t variant;             /* jd_variant_t; JD_VARIANT_AUTO in production */
  int32_t rule;                /* jd_rule_t */
  int32_t top_k;               /* K of JD_RULE_TOPK, >= 1; ignored by JD_RULE_SAMPLING */
  int32_t norm;                /* jd_norm_t */
  float rms_eps;               /* epsilon of JD_NORM_RMS, >= 0 */
  /* outputs, always written */
  int32_t* accept_len;         /* [B] number of accepted draft tokens, 0..M */
  int32_t* next_token;         /* [B] the corrected (accept_len < M) or bonus (== M) token */
  float* judge_scores;         /* [B, M] sigmoid(w . H[b,j+1] + b0) */
  float* p_draft;              /* [B, M] p_j[x_j] */
  /* optional outputs, may be NULL */
  float* q_draft;              /* [B, M] q_j[x_j] */
  uint8_t* masks;              /* [B, M] bit0 = standard test passed, bit1 = judge test passed */
  float* row_max;              /* [B, M+1] max_v L[b,j,v] */
  float* row_lse;              /* [B, M+1] log sum_v exp L[b,j,v] */
  float* logits_debug;         /* [B, M+1, V] the logits as the softmax sees them (normalisation and FP8
                                  scales applied); tests only: every variant honours it, at the price of
                                  writing R x V floats */
} jd_verify_args_t;

/* Library version, major*10000 + minor*100 + patch. */
int jd_version(void);

/* Static text for a status code; never NULL. */
const char* jd_status_string(jd_status_t s);

/* Bytes of device workspace a handle with this configuration allocates (informational;
 * the handle owns its workspace). Returns 0 for an invalid configuration. */
size_t jd_workspace_bytes(const jd_config_t* cfg);

/* Creates a handle on cfg->device: checks the architecture (JD_ERR_ARCH unless compute
 * capability 10.x), allocates the workspace (JD_ERR_ALLOC) and stores the configuration.
 * *out is set only on JD_OK. Not thread-safe per handle; distinct handles are independent. */
jd_status_t jd_create(jd_handle_t* out, const jd_config_t* cfg);

/* Frees the workspace. Synchronises the device first. NULL is accepted. */
jd_status_t jd_destroy(jd_handle_t h);

/* Registers the LM head W [V, d] and the judge head (w_judge [d], bias b_judge); device
 * pointers in the handle's dtype, 16-byte aligned, borrowed until replaced or jd_destroy.
 * The judge head is the paper's linear map R^d -> R (Sec. 4.1 "Model design and training",
 * App. B.1). Builds the TMA descriptors of W. Must precede jd_verify. */
jd_status_t jd_set_head(jd_handle_t h, const void* W, const void* w_judge, float b_judge);

/* 8-bit head (the paper runs its targets with 8-bit weights: Table 1 caption, App. B.3). Handles
 * created with JD_DTYPE_FP8_E4M3 register W8 [V, d] (uint8 E4M3 codes, 16-byte aligned) and w_scale [V]
 * (float32): the logical weight is w_scale[v] * e4m3(W8[v,k]). Every call then quantises the rows
 * of H the same way on the device, s_r = max_k |H[r,k]| / 448 and h8 = e4m3(H[r,k] * 448 / max_k |H[r,k]|)
 * rounded to nearest even, and the tensor cores multiply FP8 by FP8 with fp32 accumulation:
 * L[r,v] = w_scale[v] * s_r * sum_k e4m3(W8[v,k]) * h8[r,k]. The judge still reads the bf16 rows.
 * h8 is the E4M3 value nearest to that quotient, ties to the even mantissa (the device computes
 * H * 448 in float32, exactly, and divides with one rounding, which yields the same codes as the
 * exact quotient for bf16 rows). w_judge [d] is bf16. Pointers are borrowed like those of
 * jd_set_head. The fused and the batched tensor-core variants need d % 128 == 0; the CUDA-core
 * variant takes any d. */
jd_status_t jd_set_head_fp8(jd_handle_t h, const void* W8, const float* w_scale, const void* w_judge,
                            float b_judge);

/* One verification call (steps 1-5 above) enqueued on `cuda_stream` (a cudaStream_t, NULL =
 * default stream). Host-side checks return JD_ERR_INVALID_ARG / JD_ERR_UNSUPPORTED before
 * anything is launched. Device-side conditions (clamped tokens, timed-out waits) are recorded
 * in the handle's device status word, read with jd_last_device_status. Calls on one handle
 * must be ordered on the device (same stream or explicit dependencies): they share the
 * workspace. */
jd_status_t jd_verify(jd_handle_t h, const jd_verify_args_t* args, void* cuda_stream);

/* Same call for callers whose per-step data live in HOST memory: `args` holds HOST pointers
 * for H, draft_tokens, draft_logits and for every output (pinned memory recommended; W stays
 * on the device via jd_set_head). Inputs are copied to handle-owned device staging buffers,
 * the verification runs, the outputs are copied back (one copy through a pinned mirror), and the
 * stream is synchronised before returning. The draft logits, most of the bytes, travel on a second
 * stream of the handle while the verification already runs; each variant waits for them where it
 * first reads them (the fused kernel on a device word that the copy's stream sets, with a bounded
 * wait). Pinned host buffers are needed for that overlap; pageable ones work, serially.
 * logits_debug must be NULL. */
jd_status_t jd_verify_host(jd_handle_t h, const jd_verify_args_t* args, void* cuda_stream);

/* Synchronises the stream of the handle's last jd_verify and reads the device status of that call:
 * *out = JD_OK, JD_ERR_TIMEOUT or JD_ERR_BAD_TOKEN. Consecutive calls of the fused variant enqueue
 * no memset between them (the kernel keeps its grid-barrier counters clean and tags its status
 * writes with a launch number, so a clamped token of an earlier call is not reported for a later
 * one). JD_ERR_TIMEOUT is different: a call in which a wait ran out leaves those counters in an
 * unknown state, so every later fused call on the handle gives up at once and reports
 * JD_ERR_TIMEOUT too, until this function has been called; the next jd_verify then starts from a
 * cleared block. */
jd_status_t jd_last_device_status(jd_handle_t h, int* out);

/* Test helper for the failure path: launches a two-CTA kernel whose barrier wait can never be
 * satisfied and gives up after `spin_limit` polls (1 .. 2^20, about 40 ns each). No memory is
 * touched beyond the handle's status word; afterwards jd_last_device_status reports
 * JD_ERR_TIMEOUT and the handle stays usable. Every wait inside the real kernels is bounded the
 * same way (limit 2^22). */
jd_status_t jd_selftest_timeout(jd_handle_t h, uint32_t spin_limit, void* cuda_stream);

/* Test helper for the fail-stop rule described at jd_last_device_status: marks the handle's device
 * status as a fused call that gave up would have left it (nothing waits, nothing runs out, the host
 * side of the handle is not told). A fused jd_verify enqueued afterwards must return at once with
 * device status JD_ERR_TIMEOUT, and the first call after jd_last_device_status has reported it must
 * run normally again. */
jd_status_t jd_selftest_stale_timeout(jd_handle_t h, void* cuda_stream);

/* Variant the last jd_verify on this handle ran (jd_variant_t), 0 before the first call, and
 * the number of kernels it launched. Either pointer may be NULL. */
jd_status_t jd_last_launch_info(jd_handle_t h, int* variant, int* kernel_launches);

/* Measurement aid (the paper has no counterpart): reads the first bytes/16*16 bytes at `data`
 * (device pointer, 16-byte aligned) exactly once with streaming loads and XORs all 32-bit words
 * read into *out (device pointer, one word, which the caller zeroes beforehand). The call's
 * device time over the LM head is the read-only streaming ceiling a verification call that must
 * fetch W once can approach. Asynchronous on the stream; uses the current device. */
jd_status_t jd_stream_read_probe(const void* data, size_t bytes, uint32_t* out, void* cuda_stream);

/* Measurement aid (the paper has no counterpart). A library built with -DJD_PHASE_STAMPS
 * (python -m paper_2501_19309_b200.build --stamps) makes thread 0 of every CTA of the fused kernel
 * record the GPU's global timer at the phase boundaries of the call; this function copies the
 * stamps of the most recent fused launch on the current device to the HOST array `out`:
 * 256 CTAs x 16 slots of nanosecond values (capacity >= 4096 entries), slot meanings as printed by
 * paper_2501_19309_b200/phase_times.py. Synchronise the stream first. The normal library records
 * nothing and returns JD_ERR_UNSUPPORTED. */
jd_status_t jd_debug_phase_stamps(uint64_t* out, int32_t capacity);

/* Test helper: fills out[i] = Philox uniform for (seed, b[i], slot[i], stream[i]), i < n, with
 * the device generator; device pointers. Used to compare the generator bit for bit with an
 * independent host implementation. */
jd_status_t jd_philox_uniforms(uint64_t seed, const int32_t* b, const int32_t* slot,
                               const int32_t* stream, int32_t n, float* out, void* cuda_stream);

/* Test helper for the FP8 head: quantises `rows` bf16 rows of width d (device pointer, 16-byte
 * aligned) exactly as jd_verify does for a JD_DTYPE_FP8_E4M3 handle and writes the E4M3 codes
 * [rows, d] (device pointer, 16-byte aligned) and the per-row scales [rows] (float32). Asynchronous
 * on the stream; uses the current device. */
jd_status_t jd_quantize_rows_e4m3(const void* H, int32_t rows, int32_t d, uint8_t* codes, float* scale,
                                  void* cuda_stream);

/* Test helper (the paper has no counterpart): the handle's workspace regions are separated by guard
 * blocks of a fixed byte pattern that no kernel may touch. Synchronises the device and sets
 * *damaged to the number of guard blocks whose pattern is no longer intact (0 = no kernel wrote
 * past the end of a region). */
jd_status_t jd_check_workspace_guards(jd_handle_t h, int32_t* damaged);

/* Handle-free form of jd_verify for callers that must not allocate device memory when they
 * verify: servers whose own pool already owns the whole device, decode loops that cannot afford
 * the synchronisation an allocation implies, code barred from allocating after start-up.
 * (The paper has no counterpart; this is a deployment convenience of this library.)
 * It runs the fused tensor-core variant only: bf16, d % 64 == 0, B*(M+1) <= 96, and V small
 * enough for that variant; anything else returns JD_ERR_UNSUPPORTED and launches nothing.
 * The kernel's scratch (592,896 bytes) is a fixed array inside the library's device image: every
 * GPU that loads the library holds it until the process exits. No cudaMalloc, cudaFree or other
 * allocating call is made here.
 *   d, V, W, w_judge, b_judge : the head, as for jd_set_head (device pointers, 16-byte aligned)
 *   args                     : as for jd_verify (device pointers); variant must be AUTO or FUSED,
 *                              rule JD_RULE_SAMPLING, norm JD_NORM_NONE, logits_debug NULL
 *   device_status            : optional device pointer to one uint32 that receives the call's
 *                              device status (JD_OK, JD_ERR_TIMEOUT, JD_ERR_BAD_TOKEN); NULL to skip
 * The call uses the CURRENT device. Its first call on a device looks up the array's device
 * address and the SM count and loads every instantiation of the kernel (so that no later call has
 * to load code); make that first call outside any stream capture. First calls from several host
 * threads are serialised by a lock. All calls on a
 * device share the one array, which keeps the previous call's contents (the words that must
 * start at zero are cleared on the stream each time): calls that overlap on the GPU, from any
 * stream or thread, race with each other, so order them. Asynchronous on `cuda_stream`. */
jd_status_t jd_verify_static(int32_t d, int32_t V, const void* W, const void* w_judge, float b_judge,
                             const jd_verify_args_t* args, uint32_t* device_status, void* cuda_stream);

/* =========================================================================================
 * Around the verification call: rotary positions, a paged key / value cache and the attention
 * of a drafted block over it. One decoding step of a target layer stack is
 *
 *   jd_cache_reserve   pages for the block's T nodes            (once a step)
 *   jd_cache_append    rotate q and k, write k and v            (every layer)
 *   jd_cache_attend    attention over context + visible nodes   (every layer)
 *   jd_verify          accept_len, next_token                   (once a step)
 *   jd_cache_commit    keep the accepted nodes' rows, drop the others, advance the lengths
 *
 * Lengths, page tables and accept_len stay on the device throughout: no call of a step waits for
 * the host, and a whole step can be captured in a CUDA graph. A block is what Sec. 3.1 forwards in
 * parallel: node 0 is the last context token, nodes 1..T-1 are draft tokens, in a chain or in a
 * tree (a node's number is larger than its parent's).
 *
 * A prompt goes in the same way, without jd_verify, in chains of up to max_nodes tokens that are kept whole: reserve, append and
 * attend with T tokens, commit with accept_len = T - 1 and no paths (prompts of different lengths: num_nodes, and slot -1 where
 * one has ended).
 * ========================================================================================= */

/* Which elements of a head turn together. HALF: i with i + rot_dim / 2; INTERLEAVED: 2 i with 2 i + 1. */
typedef enum { JD_ROPE_HALF = 0, JD_ROPE_INTERLEAVED = 1 } jd_rope_layout_t;

/* How the frequencies base^(-2 i / rot_dim) are changed for contexts longer than the model was trained on.
 * LINEAR: divided by `factor`.
 * BANDS:  by wavelength: those shorter than original_len / high are kept, those longer than
 *         original_len / low divided by `factor`, and linearly blended in between (in turns per
 *         original_len).
 * YARN:   the same blend along the index i, between the indices whose frequencies make `high` and
 *         `low` turns in original_len (rounded down and up, kept to 0..rot_dim - 1: the upper one
 *         may lie behind the last index), and the outputs are multiplied by 0.1 ln(factor) + 1. */
typedef enum { JD_ROPE_SCALE_NONE = 0, JD_ROPE_SCALE_LINEAR = 1, JD_ROPE_SCALE_BANDS = 2, JD_ROPE_SCALE_YARN = 3 } jd_rope_scaling_t;

/* HOST helper: writes the rot_dim / 2 frequencies (HOST array) and the amplitude (HOST, may be NULL).
 * rot_dim even, 2..256; base > 1; factor >= 1, original_len >= 1 and 0 < low < high where the scaling uses them. */
jd_status_t jd_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double original_len,
                                double low, double high, float* inv_freq, float* amplitude);

typedef struct {
  const float* inv_freq;   /* [rot_dim / 2] radians per position, 4-byte aligned */
  int32_t rot_dim;         /* elements of a head that turn, even, 2..min(head_dim, 256); the rest pass through */
  int32_t layout;          /* jd_rope_layout_t */
  float amplitude;         /* factor on the turned elements, 1 without scaling; finite */
} jd_rope_t;

typedef struct {
  int64_t tokens;          /* 0..2^31 - 1; 0 launches nothing */
  int32_t heads, head_dim; /* >= 1; head_dim 1..256 */
  int32_t dtype;           /* JD_DTYPE_F32 or JD_DTYPE_BF16 */
  int32_t inverse;         /* 1: turn by the negative angle. The map is linear and this is its transpose:
                              with the output's gradient as x it returns the input's gradient. */
  const void* x;           /* [tokens][heads][head_dim], x_stride elements between tokens (0: dense) */
  void* out;               /* same shape, out_stride elements between tokens (0: dense). out == x with the same
                              stride turns in place; any other overlap is undefined */
  int64_t x_stride, out_stride;
  const int32_t* positions;  /* [tokens], any int32 */
  jd_rope_t rope;
} jd_rope_args_t;

/* Rotary positions: (a, b) -> amplitude (a cos t - b sin t, b cos t + a sin t) with t = position x inv_freq,
 * for every token and head. The angle is formed and reduced in float64, so that far positions lose nothing;
 * the products are float32, rounded once. Asynchronous on the stream; uses the current device. */
jd_status_t jd_rope(const jd_rope_args_t* args, void* cuda_stream);

/* ---------------------------------------------------------------- paged cache */

typedef struct {
  int32_t num_layers;   /* >= 1 */
  int32_t num_pages;    /* pages of a layer's pool, >= 1 */
  int32_t page_size;    /* tokens of a page: a power of two, 8..1024 */
  int32_t q_heads;      /* a multiple of kv_heads */
  int32_t kv_heads;
  int32_t head_dim;     /* a multiple of 8, 8..256 */
  int32_t max_seqs;     /* slots for sequences */
  int32_t max_pages;    /* page-table entries of a slot; max_pages * page_size <= 2^24 */
  int32_t max_nodes;    /* largest block, 1..128 */
  int32_t dtype;        /* JD_DTYPE_F32 or JD_DTYPE_BF16: K, V, q and outputs */
  int32_t device;       /* CUDA device ordinal that every buffer lives on */
} jd_cache_config_t;

/* DEVICE buffers, all owned by the caller and borrowed until jd_cache_destroy. A new cache starts from
 * page_table = -1, seq_len = held = refs = 0, every free_bits bit of a page = 1 and the bits behind the last page = 0,
 * and a workspace of zeroes. The calls below keep them; between calls a caller may read them, in stream order. */
typedef struct {
  void* k_pages;        /* [num_layers][num_pages][kv_heads][page_size][head_dim], 16-byte aligned */
  void* v_pages;        /* same */
  int32_t* page_table;  /* [max_seqs][max_pages] page numbers, -1 where none */
  int32_t* seq_len;     /* [max_seqs] committed tokens */
  int32_t* held;        /* [max_seqs] leading page-table entries in use */
  int32_t* refs;        /* [num_pages] sequences that hold the page, 0 = free */
  uint32_t* free_bits;  /* [ceil(num_pages / 32)] bit p % 32 of word p / 32: page p is free */
  void* workspace;      /* zero-filled, 256-byte aligned, jd_cache_workspace_bytes() */
  size_t workspace_bytes;
} jd_cache_buffers_t;

typedef struct jd_cache_s* jd_cache_t;

/* Bytes of workspace a cache of this configuration needs, 0 for an invalid one. */
size_t jd_cache_workspace_bytes(const jd_cache_config_t* cfg);

/* Creates a handle: host memory and tensor maps only, no device allocation and nothing enqueued. Calls on one
 * handle share its workspace and must be ordered on the device (one stream, or explicit dependencies); graphs
 * captured from one handle must not run at the same time. Streams that attend at the same time take two handles
 * on the same buffers, each with a workspace of its own; calls that change the cache are always ordered. */
jd_status_t jd_cache_create(jd_cache_t* out, const jd_cache_config_t* cfg, const jd_cache_buffers_t* buffers);
jd_status_t jd_cache_destroy(jd_cache_t c);   /* frees host memory only; NULL is accepted */

/* Slots: every call below takes B sequences, 1..min(max_seqs, 1024), and `slots` [B] (device) with the slot of
 * each, or NULL for slots 0..B-1. Entry -1 marks a padding sequence: skipped, its outputs are left as they were.
 * Other slots outside [0, max_seqs) are skipped and reported. jd_cache_attend may name a slot several times; in the
 * calls that change the cache the first naming counts, later ones are skipped and reported. */

/* Makes room for n more tokens (1..) of every sequence: pages for [seq_len, seq_len + n), the lowest free ones, in the
 * sequences' order; and where the page that holds token seq_len has rows in use and other owners, a copy of those
 * rows in a page of the sequence's own (all layers). A sequence named later in the call counts as owner until its turn,
 * so that the last one keeps the page. All or nothing: if pages are short, or a table is, nothing changes and
 * JD_ERR_PAGES is reported. Reserve before append, and fork only between commit and reserve: behind a fork the page that a
 * block begins in has two owners, and append writes nothing there. */
jd_status_t jd_cache_reserve(jd_cache_t c, int32_t B, const int32_t* slots, int32_t n, void* cuda_stream);

/* The block of drafted tokens of a step. */
typedef struct {
  int32_t nodes;              /* T, 1..max_nodes */
  int32_t per_seq;            /* 0: one mask and depth for all sequences, 1: one for each */
  const uint32_t* mask;       /* [T][W] or [B][T][W], W = ceil(T / 32): bit j % 32 of word j / 32 of row i: node i sees
                                 node j (its own bit included). NULL: a chain, node i sees 0..i. Bits >= T are ignored */
  const int32_t* depth;       /* [T] or [B][T] tokens between the context's end and the node: position = seq_len + depth.
                                 NULL: depth = node number */
  const int32_t* num_nodes;   /* [B] nodes of each sequence, 0..T (clamped), or NULL: T. Rows behind them are neither
                                 read nor written, in no output */
} jd_tree_t;

typedef struct {
  int32_t B, layer;
  const int32_t* slots;
  jd_tree_t tree;
  const void* k;              /* [B][T][kv_heads][head_dim], k_stride elements between tokens (0: dense) */
  const void* v;              /* same, v_stride */
  const void* q;              /* [B][T][q_heads][head_dim], q_stride; NULL: no queries */
  void* q_out;                /* same shape, q_out_stride; may be q itself with the same stride */
  int64_t k_stride, v_stride, q_stride, q_out_stride;
  const jd_rope_t* rope;      /* HOST struct; NULL: keys and queries as they are */
} jd_append_args_t;

/* Writes keys (turned to their positions) and values of a block behind the sequences' tokens, node j at token
 * seq_len + j, and the turned queries to q_out. seq_len stays. Rows whose page is missing or has other owners are
 * skipped and reported (jd_cache_reserve has to come first). Pointers 16-byte aligned, strides multiples of 16 bytes. */
jd_status_t jd_cache_append(jd_cache_t c, const jd_append_args_t* args, void* cuda_stream);

/* Kernel family of jd_cache_attend. TENSOR: tcgen05 kernel, bf16 with head_dim 64 or 128. SIMT: any cache. */
typedef enum { JD_ATTEND_AUTO = 0, JD_ATTEND_SIMT = 1, JD_ATTEND_TENSOR = 2 } jd_attend_variant_t;

typedef struct {
  int32_t B, layer;
  const int32_t* slots;
  jd_tree_t tree;             /* depth is not read */
  const void* q;              /* [B][T][q_heads][head_dim], q_stride elements between tokens (0: dense); head h reads
                                 kv head h / (q_heads / kv_heads) */
  void* out;                  /* same shape and type, out_stride; not q */
  int64_t q_stride, out_stride;
  float* lse;                 /* [B][T][q_heads] log sum exp of the scaled scores, or NULL */
  float scale;                /* on q . k, positive and finite */
  int32_t variant;            /* jd_attend_variant_t */
} jd_attend_args_t;

/* Attention of a block's nodes over the sequence's seq_len cached tokens and the nodes they may see:
 * out = softmax(scale q k^T) v, statistics and sums in float32; the bf16 kernel rounds the softmax weights to
 * bf16 in front of their product with v. A row that sees nothing gets out = 0 and lse = -inf. Whatever stands
 * in rows that a node may not see (infinities and NaN too) stays without effect on it. A value of a seen row that is not finite
 * makes that element of the output what the sum has it be, the infinity or NaN, as long as the row's weight is one that
 * float32 holds; below that NaN may stand for the infinity. Numerators are divided at the end, so a value times the
 * number of tokens has to stay below 2^119. Pointers 16-byte aligned, strides multiples of 16 bytes. */
jd_status_t jd_cache_attend(jd_cache_t c, const jd_attend_args_t* args, void* cuda_stream);

typedef struct {
  int32_t B;
  const int32_t* slots;
  const int32_t* accept_len;  /* [B][num_paths] accepted draft tokens, as jd_verify writes them */
  int32_t num_paths;          /* >= 1 candidate paths of every sequence; the one with the largest accept_len is kept, the
                                 first of equals. (With several, verify by JD_RULE_TOPK: under the sampling rule the pick
                                 would bias the tokens.) */
  int32_t path_len;           /* entries of a path, 0..max_nodes - 1 */
  const int32_t* paths;       /* [B][num_paths][path_len] nodes of the draft tokens along the path, rising; NULL:
                                 nodes 1, 2, .. (path_len then bounds accept_len; use T - 1) */
  int32_t* chosen;            /* [B] the kept path, or NULL */
} jd_commit_args_t;

/* Ends a step: node 0 and the first accept_len nodes of the kept path become the sequence's next tokens. Their rows
 * are moved together in all layers, seq_len grows by accept_len + 1 and the pages behind are released. accept_len is
 * clamped to 0..path_len; where a path does not rise, or reaches max_nodes or a row that the sequence does not hold or not
 * alone, it is cut there and reported; where that is node 0's row, seq_len stays. A sequence that had no nodes in the step
 * (num_nodes 0) is left out by slot -1. */
jd_status_t jd_cache_commit(jd_cache_t c, const jd_commit_args_t* args, void* cuda_stream);

/* dst[i] becomes a copy of src[i] (device arrays [n], n <= 1024) that shares its pages; jd_cache_reserve gives each its
 * own where they part. dst must be empty, named once and no source of the same call, else it is skipped and reported;
 * entries with src or dst -1 are padding. */
jd_status_t jd_cache_fork(jd_cache_t c, int32_t n, const int32_t* src, const int32_t* dst, void* cuda_stream);

/* Cuts the sequences to length[b] tokens (device [B]; NULL: 0, which frees them) and releases the pages behind, uncommitted
 * ones too. A length outside 0..seq_len is skipped and reported. */
jd_status_t jd_cache_truncate(jd_cache_t c, int32_t B, const int32_t* slots, const int32_t* length, void* cuda_stream);

/* Moves the pages in use to the lowest numbers, in all layers, so that the first `used` pages hold everything and the rest
 * of the pool can go: the highest pages in use fill the lowest free ones, the k-th of those moved into the k-th of those
 * free, both counted from below. Page numbers change; sequences do not. used: device pointer to one int32, or NULL. */
jd_status_t jd_cache_compact(jd_cache_t c, int32_t* used, void* cuda_stream);

/* Synchronises the stream of the cache's last call and returns and clears the device status: *out = JD_OK, JD_ERR_PAGES,
 * JD_ERR_BAD_INDEX or JD_ERR_TIMEOUT, the first since the last query. That stream has to exist still. Not during a capture. */
jd_status_t jd_cache_last_status(jd_cache_t c, int* out);

#ifdef __cplusplus
}
#endif
#endif /* JD_H_ */
