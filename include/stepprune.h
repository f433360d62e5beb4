/*
 * stepprune.h -- C ABI of the GB300 (sm_103a) StepPrune inference path.
 *
 * StepPrune (arXiv 2609.13804) prunes the visual prefix of a multimodal LLM by
 * sequential selection: a pointer decoder picks visual tokens one round at a
 * time, conditioned on what it already picked and on the text, until a learned
 * STOP action wins (Sec. 3.1-3.2, Eq. 2 and Eq. 4; grouped rounds of g tokens,
 * Sec. 3.5, Eq. 11).  The kept tokens are restored to native order and
 * physically gathered before the language-model prefill (Algorithm 1 steps 4-5).
 * This library runs that path on one GPU:
 *
 *   sp_select    text projection + cross-modal encoder (Eq. 3), candidate
 *                precompute, the sequential selection loop, restore.
 *   sp_compact   gather of the kept visual rows and the text rows into a packed
 *                variable-length buffer with cu_seqlens and positions.
 *   sp_project   the frozen multimodal projector on the kept rows, scattered
 *                into their packed slots.
 *   sp_prefill   the LM prefill over the packed prefix (hidden states after the
 *                final RMSNorm).
 *   sp_pipeline  all four, back to back on one stream.
 * and the generation after it: sp_decode over a cache per sequence, and over
 * pages that sequences share (sp_prefill_paged, sp_decode_paged and the
 * operators they, beam search and speculative sampling are made of).
 *
 * Conventions (all entry points):
 *   - Pointers marked DEVICE are device memory owned by the caller; HOST marks
 *     host memory read during the call only.  Matrices are row-major; weights
 *     use the nn.Linear layout [out_features, in_features].  bf16 data is
 *     passed as raw 16-bit patterns (void*).
 *   - Calls are asynchronous on the given stream and never synchronise the
 *     host.  Hot calls (sp_select, sp_compact, sp_project, sp_prefill,
 *     sp_pipeline) allocate nothing: scratch comes from the caller's workspace,
 *     sized by the matching *_workspace() query.  Handles allocate at create
 *     time only and free at destroy.
 *   - Sizes that depend on the selection (the kept counts, the packed length T)
 *     stay on the device; grids are sized from host-known caps and kernels
 *     skip rows past the device count, so no call reads results back.
 *   - A status is returned for every call; argument problems are detected on
 *     the host before any launch (nothing is launched then).  The message of
 *     the last failure on the calling thread is in sp_last_error().
 *   - Device-side failures (a bounded wait that ran out, an index out of
 *     range) set bits in the optional DEVICE int error word passed in the
 *     call; read it after synchronising (see SP_DEVERR_*).  Kernels never trap.
 *   - No C++ exception crosses the ABI.
 */
#ifndef STEPPRUNE_H
#define STEPPRUNE_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define SP_API __attribute__((visibility("default")))
#else
#define SP_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

#define SP_ABI_VERSION 1

/* Limits checked on the host (SP_ERR_SHAPE when exceeded). */
#define SP_MAX_BATCH 256          /* images per call */
#define SP_MAX_ENC_LAYERS 4       /* cross-modal encoder blocks */
#define SP_MAX_DEC_LAYERS 4       /* pointer-decoder layers */
#define SP_MAX_LM_LAYERS 96       /* decoder layers of the LM */
#define SP_MAX_KMAX 1024          /* per-episode cap on retained tokens */
#define SP_MAX_NVIS 16384         /* visual tokens of one image */
#define SP_MAX_BEAMS 16           /* beams of one element */
#define SP_MAX_DRAFT_ROWS 1024    /* rows of one sequence that sp_draft_verify looks at */
#define SP_MAX_TABLE_ROWS 4096    /* rows of a table that sp_pages_* work on */

typedef enum {
  SP_OK = 0,
  SP_ERR_INVALID_ARG = 1,   /* NULL where a pointer is required, bad enum, ... */
  SP_ERR_SHAPE = 2,         /* a size outside the supported set or a limit */
  SP_ERR_ALIGN = 3,         /* a device pointer not 16-byte aligned */
  SP_ERR_WORKSPACE = 4,     /* workspace NULL or smaller than *_workspace() */
  SP_ERR_CUDA = 5,          /* a CUDA runtime call failed (message has the code) */
  SP_ERR_TIMEOUT = 6,       /* reported by sp_device_error_status() */
  SP_ERR_UNSUPPORTED = 7,   /* device is not sm_103 / feature not built */
  SP_ERR_DEVICE = 8         /* reported by sp_device_error_status() */
} sp_status;

/* Bits of the DEVICE error word. */
#define SP_DEVERR_TIMEOUT 0x1   /* a bounded wait (mbarrier / flag) ran out */
#define SP_DEVERR_INDEX 0x2     /* an index outside its range was skipped */
#define SP_DEVERR_PAGES 0x4     /* a cache had too few free pages */

typedef struct CUstream_st* sp_stream; /* a cudaStream_t; NULL is the legacy default stream */

/* Thread-local message of the last failed call ("" if none). */
SP_API const char* sp_last_error(void);
/* SP_ABI_VERSION of the loaded library. */
SP_API int sp_abi_version(void);
/* Maps a device error word read back by the caller to SP_OK / SP_ERR_TIMEOUT / SP_ERR_DEVICE. */
SP_API sp_status sp_device_error_status(int device_error_word);

/* ------------------------------------------------------------------------ */
/* Selector (Sec. 3.2: cross-modal encoder, STOP row, pointer decoder).      */
/* ------------------------------------------------------------------------ */

typedef struct {
  int D;             /* visual feature width = width of the candidate memory M; multiple of 128 */
  int D_text;        /* width of the prompt embeddings E_text */
  int h;             /* pointer-decoder width; multiple of 128 in 128..1024 */
  int n_enc_layers;  /* encoder blocks (the paper uses 2); 0..SP_MAX_ENC_LAYERS */
  int enc_head_dim;  /* encoder head dim: 64 or 128; D must be a multiple */
  int enc_ffn;       /* encoder MLP width (4 D in a ViT block) */
  float ln_eps;      /* LayerNorm epsilon */
  float g_text;      /* text gate g_text of E~ = g_text LN(W_p E) (1 at inference) */
  int n_dec_layers;  /* pointer-decoder layers, 1..SP_MAX_DEC_LAYERS (0 is read as 1) */
} sp_selector_cfg;

/*
 * Weights of the selector.  The encoder and text projection are bf16 (tensor
 * cores); the pointer decoder is fp32.  LayerNorm gain/bias pointers may be
 * NULL (gain 1 / bias 0).  All DEVICE; borrowed by the handle, so they must
 * outlive it (the handle keeps folded copies of the decoder matrices).
 *
 * Reading of the decoder (Sec. 3.2, Eq. 4; the paper fixes no layer count or
 * width): one pre-LN decoder layer of width h with single-head attention.  A
 * decoder token is y = W_in q with q_1 = s_start and q_{t+1} = M[a_t]; causal
 * self-attention gives u_t = y_t + Wo_s sum_i softmax_i(<Wq_s x_t, Wk_s x_i>/sqrt h)
 * Wv_s x_i with x_i = LN1(y_i); the pointer logits are the cross-attention
 * scores l_t(j) = <Wq_p LN2(u_t), Wk_p M_j>/sqrt h over the N+1 rows of
 * M = [H; s_stop], plus a per-episode stop_bias on the STOP row.
 *
 * With n_dec_layers = L > 1 the fields below (ln1, Wq_s .. Wo_s, ln2, Wq_p,
 * Wk_p) describe the LAST layer, and dec_lower[0 .. L-2] the layers before it,
 * each a whole pre-LN decoder layer of width h (Sec. 3.2: self-attention,
 * cross-attention to the memory, feed-forward network):
 *   a  = x + Wo_s SelfAttn(LN1(x))            causal over the history
 *   c  = a + Wo_c CrossAttn(LN2(a), M)        all N+1 rows of M, unmasked
 *   x' = c + W2 GELU(W1 LN3(c))               hidden width 4h, exact-erf GELU
 * x of layer 0 is y = W_in q; x' of layer L-2 enters the last layer.
 */
typedef struct {
  const float* ln1_g; const float* ln1_b;  /* [h] */
  const float* Wq_s; const float* Wk_s; const float* Wv_s; const float* Wo_s;  /* [h, h] fp32 */
  const float* ln2_g; const float* ln2_b;  /* [h] */
  const float* Wq_c; const float* Wo_c;    /* [h, h] fp32 */
  const float* Wk_c; const float* Wv_c;    /* [h, D] fp32 */
  const float* ln3_g; const float* ln3_b;  /* [h] */
  const void* W1;                          /* [4h, h] bf16 */
  const void* W2;                          /* [h, 4h] bf16 */
} sp_dec_layer_weights;

typedef struct {
  const void* W_p;                         /* [D, D_text] bf16 text projection */
  const float* ln_text_g; const float* ln_text_b;    /* [D] */
  const void* enc_wqkv[SP_MAX_ENC_LAYERS]; /* [3D, D] bf16, rows q|k|v */
  const void* enc_wo[SP_MAX_ENC_LAYERS];   /* [D, D] bf16 */
  const void* enc_w1[SP_MAX_ENC_LAYERS];   /* [enc_ffn, D] bf16 */
  const void* enc_w2[SP_MAX_ENC_LAYERS];   /* [D, enc_ffn] bf16 */
  const float* enc_ln1_g[SP_MAX_ENC_LAYERS]; const float* enc_ln1_b[SP_MAX_ENC_LAYERS];
  const float* enc_ln2_g[SP_MAX_ENC_LAYERS]; const float* enc_ln2_b[SP_MAX_ENC_LAYERS];
  const float* s_stop;                     /* [D] learned STOP embedding */
  const float* s_start;                    /* [D] learned START embedding (q_1) */
  const float* W_in;                       /* [h, D] decoder input projection */
  const float* ln1_g; const float* ln1_b;  /* [h] */
  const float* Wq_s; const float* Wk_s; const float* Wv_s; const float* Wo_s; /* [h, h] */
  const float* ln2_g; const float* ln2_b;  /* [h] */
  const float* Wq_p;                       /* [h, h] pointer query */
  const float* Wk_p;                       /* [h, D] pointer key */
  const sp_dec_layer_weights* dec_lower;   /* HOST [n_dec_layers - 1] (copied at creation; the
                                              DEVICE pointers inside are borrowed), or NULL */
} sp_selector_weights;

typedef struct sp_selector_s sp_selector;

/* Validates cfg, allocates the folded decoder matrices and encodes the weight
 * tensor maps.  Synchronous (uses the legacy stream once). */
SP_API sp_status sp_selector_create(const sp_selector_cfg* cfg, const sp_selector_weights* w,
                             sp_selector** out);
SP_API void sp_selector_destroy(sp_selector* s);

/*
 * One batch of images for selection.  Image b owns visual rows
 * [sum_{c<b} n_vis[c], +n_vis[b]) of X (or H) and text rows likewise of E_text.
 * Candidate groups: with group_size > 0 the candidates of an image are cut into
 * consecutive groups of group_size (the last may be shorter); each group is an
 * independent episode with its own mask, history, cap k_max and stop_bias, all
 * sharing s_start / s_stop; group_size 0 = one episode per image.  Episodes are
 * numbered image-major, group-minor.
 */
typedef struct {
  int B;                 /* images, 1..SP_MAX_BATCH */
  const int* n_vis;      /* HOST [B] visual tokens per image (N_b, 1..SP_MAX_NVIS) */
  const int* n_txt;      /* HOST [B] text tokens per image (L_b, >= 0) */
  const void* X;         /* DEVICE [sum N_b, D] bf16 visual tokens; ignored when H is set */
  const void* E_text;    /* DEVICE [sum L_b, D_text] bf16 prompt embeddings; ignored when H is set */
  const float* H;        /* DEVICE [sum N_b, D] fp32 encoded candidates, or NULL to run the
                            text projection and encoder on X / E_text (Eq. 3) */
  const float* stop_bias;/* DEVICE [n_episodes] fp32 added to the STOP logit */
  int group_size;        /* candidates per episode (0: whole image) */
  int g;                 /* visual tokens kept per non-STOP round (1..16); Eq. 11 */
  int k_max;             /* per-episode cap, 1..SP_MAX_KMAX */
} sp_select_in;

/*
 * Outputs.  idx row b holds image b's kept visual indices (image-local) in
 * ascending (native) order, then -1 up to k_cap.  k_cap must be at least the
 * largest possible count of an image: sum over its episodes of min(k_max, size).
 * order / ep_count / margin / gap are optional per-episode traces:
 *   order[e*k_max + i]   episode-local index taken i-th (step order)
 *   ep_count[e]          tokens kept by episode e
 *   margin[e*(k_max+1)+r] round r's smallest gap between consecutive values
 *                        among the top g+1 available visual logits and STOP
 *   gap[e*(k_max+1)+r]   round r's best available visual logit minus the raw
 *                        STOP logit (before stop_bias): STOP wins iff
 *                        stop_bias > gap, which calibrates stop_bias
 *   rounds[e]            evaluated rounds of episode e
 * Unwritten trace entries are left as they were.
 */
typedef struct {
  int* idx;          /* DEVICE [B, k_cap] */
  int k_cap;
  int* count;        /* DEVICE [B] kept tokens per image (K_b) */
  int* order;        /* DEVICE [n_episodes, k_max] or NULL */
  int* ep_count;     /* DEVICE [n_episodes] or NULL */
  float* margin;     /* DEVICE [n_episodes, k_max + 1] or NULL */
  float* gap;        /* DEVICE [n_episodes, k_max + 1] or NULL */
  int* rounds;       /* DEVICE [n_episodes] or NULL */
  float* memory;     /* DEVICE [sum N_b, D] fp32 or NULL: receives the candidate memory H
                        (the encoder output of Eq. 3, or a copy of the given H) */
  int* err;          /* DEVICE error word (SP_DEVERR_*) or NULL */
} sp_select_out;

/* Number of episodes of a batch (host arithmetic; -1 on bad arguments). */
SP_API int sp_num_episodes(int B, const int* n_vis, int group_size);
/* Workspace bytes sp_select needs for this batch (0 on bad arguments). */
SP_API size_t sp_select_workspace(const sp_selector* s, const sp_select_in* in);
/* Algorithm 1 steps 1-4 for every image of the batch (see sp_select_in).
 * A selector with n_dec_layers > 1 takes g = 1 only (each new history position
 * runs through every layer before the next decision; SP_ERR_UNSUPPORTED
 * otherwise, before any launch). */
SP_API sp_status sp_select(const sp_selector* s, const sp_select_in* in, const sp_select_out* out,
                    void* workspace, size_t workspace_bytes, sp_stream stream);

/*
 * sp_select without a caller workspace.  The paper has no counterpart: this is
 * for callers that cannot allocate device memory (a plug-in whose host
 * application owns all device memory, a plain-C caller with no allocator, a
 * path that may not pay for cudaMalloc).  It runs the same selection as
 * sp_select; its scratch is one static device array of
 * SP_SELECT_NOALLOC_SCRATCH_BYTES that every GPU loading the library holds
 * until exit.  Inputs and outputs are still the caller's.
 *   - A batch whose sp_select_workspace() exceeds that size is rejected with
 *     SP_ERR_WORKSPACE before any launch.
 *   - It calls no cudaMalloc / cudaFree and no allocating library routine.
 *   - The first call on a device looks up the array's device address (with
 *     that device current); make that first call before any stream capture.
 *   - All calls share the array and it keeps the last call's contents: calls
 *     whose GPU work overlaps (several streams or threads) race; serialise them.
 *   - The device address found by the first call is kept for the process's
 *     life: do not use this entry point across a device reset
 *     (cudaDeviceReset tears down the context the address belongs to).
 */
#define SP_SELECT_NOALLOC_SCRATCH_BYTES (64u << 20)
SP_API sp_status sp_select_noalloc(const sp_selector* s, const sp_select_in* in, const sp_select_out* out,
                                   sp_stream stream);

/* ------------------------------------------------------------------------ */
/* Training-time continuous pathway, forward only (Sec. 3.3, Eqs. 5-9).      */
/* ------------------------------------------------------------------------ */

/*
 * The trajectory aggregates of Eqs. 5-7, accumulated along the hard rollout:
 * at every evaluated step t of an episode, p_t = softmax(l_t / tau) over its
 * available candidates and STOP (l_t as in sp_select, stop_bias included:
 * pass zeros for the paper's training), and
 *   A_1 = 1,  A_{t+1} = A_t (1 - p_t(STOP))                       (Eq. 5)
 *   s_i  += A_t p_t(i) beta^t                                      (Eq. 6)
 *   Kbar += A_t (1 - p_t(STOP))                                    (Eq. 7)
 * The rollout is sp_select's (Eq. 4, hard argmax): it ends at the first hard
 * STOP, at k_max kept tokens or with only STOP left; later steps contribute
 * nothing.
 */
typedef struct {
  float tau;        /* pointer temperature, > 0 */
  float beta;       /* discount of Eq. 6, in (0, 1] */
  float* score;     /* DEVICE [sum N_b] fp32 out: s_i, same rows as X / H (4-byte aligned) */
  float* kbar;      /* DEVICE [n_episodes] fp32 out: Kbar per episode */
} sp_train_args;

/*
 * sp_select plus the aggregates above, in the same launches (same workspace
 * size as sp_select_workspace).  Requires g = 1 (one token per step, the
 * rollout the aggregates are defined on) and an episode size whose keys fit
 * the selection kernel's shared memory (up to 2,032 candidates per episode);
 * otherwise SP_ERR_UNSUPPORTED before any launch.  SP_ERR_INVALID_ARG for a
 * NULL score / kbar or tau <= 0 or beta outside (0, 1].
 */
SP_API sp_status sp_select_train(const sp_selector* s, const sp_select_in* in, const sp_select_out* out,
                                 const sp_train_args* train, void* workspace, size_t workspace_bytes,
                                 sp_stream stream);

/*
 * Eq. 8: alpha = SoftTopK_{k,tau}(s) per image, k = the batch mean of the
 * images' soft counts (an image's count is the sum of its episodes' Kbar),
 * detached, clamped to [0, N_b].  SoftTopK is the entropic optimal transport
 * of an image's scores (mass 1/N_b each) onto the anchors 0 and 1 with masses
 * (N_b - k, k) / N_b, cost (s_i - y)^2, regularisation tau; alpha_i is N_b
 * times token i's mass sent to anchor 1, which equals
 * sigmoid(2 (s_i - theta) / tau) with sum_i alpha_i = k (theta is solved for).
 *   n_vis / group_size: HOST, as in sp_select_in (episodes image-major)
 *   score: DEVICE [sum N_b] fp32, kbar: DEVICE [n_episodes] fp32
 *   alpha: DEVICE [sum N_b] fp32 out;  k_out: DEVICE [1] fp32 out or NULL
 * Errors: SP_ERR_INVALID_ARG / SP_ERR_SHAPE on bad sizes or pointers.
 */
SP_API sp_status sp_soft_topk(int B, const int* n_vis, int group_size, const float* score, const float* kbar,
                              float tau, float* alpha, float* k_out, sp_stream stream);

/*
 * Eq. 9: x~ = sqrt(alpha_r) x + sqrt(1 - alpha_r) eps for every row r, fp32
 * arithmetic, bf16 in and out.  X, noise, out: DEVICE [rows, D] bf16, 16-byte
 * aligned, D a multiple of 8; alpha: DEVICE [rows] fp32 (clamped to [0, 1]).
 * The Gaussian draws eps are the caller's.  out may alias X.
 */
SP_API sp_status sp_vp_gate(int rows, int D, const void* X, const void* noise, const float* alpha, void* out,
                            sp_stream stream);

/* ------------------------------------------------------------------------ */
/* Compaction (Algorithm 1 step 5: X_S = Gather(X, S), then [X_S; text]).    */
/* ------------------------------------------------------------------------ */

/*
 * Sequence b of the packed output is image b's kept visual rows (native order)
 * followed by its text rows; positions restart at 0 for every sequence.
 * T = cu_seqlens[B] is written on the device; T_cap = sum_b (min(n_vis[b], k_cap)
 * + n_txt[b]) bounds it.
 *   direct (vis_packed == NULL): W_vis must equal W_txt and visual rows go
 *     straight into their packed slots (no projector, or one already applied).
 *   projector mode (vis_packed != NULL): visual rows go to vis_packed, image-
 *     major and contiguous (vis_cu[b] is image b's first row), and
 *     vis_row_map[i] is the packed row that projected row i belongs to; the
 *     visual slots of packed are left for sp_project.
 */
typedef struct {
  int B;
  const int* n_vis;      /* HOST [B] */
  const int* n_txt;      /* HOST [B] */
  const void* X;         /* DEVICE [sum N_b, W_vis] bf16 */
  int W_vis;             /* multiple of 8 */
  const void* text;      /* DEVICE [sum L_b, W_txt] bf16 (LM-width prompt embeddings) */
  int W_txt;             /* multiple of 8 */
  const int* idx;        /* DEVICE [B, k_cap] from sp_select */
  int k_cap;
  const int* count;      /* DEVICE [B] */
} sp_compact_in;

typedef struct {
  void* packed;          /* DEVICE [T_cap, W_txt] bf16 */
  int* cu_seqlens;       /* DEVICE [B + 1] */
  int* pos;              /* DEVICE [T_cap] */
  void* vis_packed;      /* DEVICE [sum_b min(n_vis[b], k_cap), W_vis] bf16, or NULL (direct / index mode) */
  int* vis_row_map;      /* DEVICE [same rows] (projector and index modes) */
  int* vis_cu;           /* DEVICE [B + 1] (projector and index modes) */
  int* err;              /* DEVICE error word or NULL */
  int* vis_src;          /* DEVICE [same rows] int32, or NULL.  Index mode (vis_src set,
                            vis_packed NULL): no visual row is copied; vis_src[i] is the row of
                            X that kept visual row i comes from, and sp_project (io.vis_src)
                            gathers those rows itself: Alg. 1 step 5's gather folded into the
                            projector's operand load.  An invalid index gives vis_src -1. */
} sp_compact_out;

/* T_cap of a batch (host arithmetic; -1 on bad arguments). */
SP_API int sp_packed_cap(int B, const int* n_vis, const int* n_txt, int k_cap);
SP_API sp_status sp_compact(const sp_compact_in* in, const sp_compact_out* out, sp_stream stream);

/* ------------------------------------------------------------------------ */
/* Language model: projector + decoder-only prefill.                          */
/* ------------------------------------------------------------------------ */

typedef enum { SP_PROJ_NONE = 0, SP_PROJ_LINEAR = 1, SP_PROJ_MLP2_GELU = 2 } sp_proj_kind;

typedef struct {
  int n_layers;      /* 1..SP_MAX_LM_LAYERS */
  int d;             /* model width; multiple of 128 */
  int n_heads;       /* query heads */
  int n_kv_heads;    /* key/value heads; divides n_heads (GQA when smaller) */
  int head_dim;      /* 64 or 128 */
  int ffn;           /* SwiGLU width; multiple of 128 */
  int max_pos;       /* positions covered by the rotary table (> longest sequence) */
  float rope_theta;
  float rms_eps;
  int proj_kind;     /* sp_proj_kind */
  int proj_in;       /* visual width entering the projector */
  int proj_hidden;   /* hidden width of SP_PROJ_MLP2_GELU */
  int mrope_section[3]; /* 3-D mRoPE (the Qwen2.5-VL backbone, Sec. 1): rotation pairs given to the
                           (t, h, w) position components, consecutive from pair 0; the three sum
                           to head_dim / 2, each even.  All zero: 1-D RoPE on pos. */
} sp_model_cfg;

/*
 * Weights (DEVICE, borrowed; bf16 unless stated).  Per layer:
 *   wqkv  [(n_heads + 2 n_kv_heads) head_dim, d]  rows q | k | v
 *   wo    [d, n_heads head_dim]
 *   wgu   [2 ffn, d]  rows gate | up   (SwiGLU: down(silu(gate x) * up x))
 *   wdown [d, ffn]
 *   attn_norm / mlp_norm  fp32 [d] RMSNorm gains, or NULL (1)
 * final_norm fp32 [d] or NULL.  Projector: proj_w1 [proj_hidden or d, proj_in],
 * proj_w2 [d, proj_hidden] (SP_PROJ_MLP2_GELU only).
 */
typedef struct {
  const void* wqkv[SP_MAX_LM_LAYERS];
  const void* wo[SP_MAX_LM_LAYERS];
  const void* wgu[SP_MAX_LM_LAYERS];
  const void* wdown[SP_MAX_LM_LAYERS];
  const float* attn_norm[SP_MAX_LM_LAYERS];
  const float* mlp_norm[SP_MAX_LM_LAYERS];
  const float* final_norm;
  const void* proj_w1;
  const void* proj_w2;
} sp_model_weights;

typedef struct sp_model_s sp_model;

/* Validates cfg, uploads the rotary table (fp64 on the host, stored fp32) and
 * encodes the weight tensor maps.  Synchronous. */
SP_API sp_status sp_model_create(const sp_model_cfg* cfg, const sp_model_weights* w, sp_model** out);
SP_API void sp_model_destroy(sp_model* m);

/*
 * Projector on the kept rows (Sec. 3.3, last paragraph: restored, then
 * projected): packed[vis_row_map[i]] = P(x_i) for i < vis_cu[B] (device
 * count), P = W1 x, or W2 GELU(W1 x), with x_i = vis_packed[i], or, when
 * vis_src is given, x_i = X[vis_src[i]] read by the first GEMM's operand loads
 * (row-gather TMA) so that the kept rows are never copied.  rows_cap bounds
 * vis_cu[B].
 */
typedef struct {
  int B;
  int rows_cap;
  const void* vis_packed;   /* DEVICE [rows_cap, proj_in] bf16 (ignored with vis_src) */
  const int* vis_row_map;   /* DEVICE [rows_cap] */
  const int* vis_cu;        /* DEVICE [B + 1] */
  void* packed;             /* DEVICE [T_cap, d] bf16 (visual slots written) */
  int* err;
  const void* X;            /* DEVICE [rows_X, proj_in] bf16 visual tokens (with vis_src) */
  int rows_X;               /* rows of X (with vis_src) */
  const int* vis_src;       /* DEVICE [rows_cap] rows of X (sp_compact's index mode), or NULL */
} sp_project_io;

SP_API size_t sp_project_workspace(const sp_model* m, int rows_cap);
SP_API sp_status sp_project(const sp_model* m, const sp_project_io* io, void* workspace,
                     size_t workspace_bytes, sp_stream stream);

/*
 * Prefill of the packed sequences: the frozen LM run over the pruned prefix
 * that Algorithm 1 hands it (Sec. 3.3, last paragraph: the kept tokens,
 * restored to native order and projected, precede the text; Sec. 1: the
 * prefill cost the selection removes is that of the dropped visual tokens).
 * The layers are those of the evaluated backbones (Sec. 4.1): causal attention
 * within each sequence (cu_seqlens), grouped-query heads, rotary positions
 * pos, pre-RMSNorm Llama-style layers with SwiGLU, and the final RMSNorm.
 * hidden rows t < T = cu_seqlens[B] are written; rows >= T are untouched.  residual (optional) receives the last residual stream (fp32,
 * before the final norm).  kv (optional) receives the key / value cache the
 * generation that follows reads (sp_decode): per layer l, sequence b and
 * position p = pos[row] the rotated key at
 *   kv + (((l * 2 + 0) * B + b) * kv_S_cap + p) * (n_kv_heads * head_dim)
 * and the value at the same offset with 1 in place of 0 (bf16).  Positions
 * must be < kv_S_cap (else SP_DEVERR_INDEX).
 * With an mRoPE model (mrope_section set), pos3 gives every row's rotary
 * (t, h, w) position (sp_mrope_positions writes it for a pruned batch); pos is
 * then only the row's index within its sequence (its cache slot).  A rotary
 * position >= max_pos sets SP_DEVERR_INDEX.
 */
typedef struct {
  int B;
  int T_cap;                /* bound on cu_seqlens[B] */
  int max_seqlen_cap;       /* bound on every sequence length */
  const void* x;            /* DEVICE [T_cap, d] bf16 packed LM input */
  const int* cu_seqlens;    /* DEVICE [B + 1] */
  const int* pos;           /* DEVICE [T_cap] */
  float* hidden;            /* DEVICE [T_cap, d] fp32 output */
  float* residual;          /* DEVICE [T_cap, d] fp32 or NULL */
  int* err;
  void* kv;                 /* DEVICE [n_layers][2][B][kv_S_cap][n_kv_heads * head_dim] bf16, or NULL */
  int kv_S_cap;             /* positions per sequence in kv */
  const int* pos3;          /* DEVICE [T_cap, 4] int32 (t, h, w, unused); required iff mRoPE, else NULL */
} sp_prefill_io;

/*
 * mRoPE positions of a pruned batch (reading of Sec. 3.3's last paragraph: the
 * kept tokens are restored to native order so that the backbone's positional
 * convention holds).  Image b's N_b tokens form a grid of ceil(N_b / grid_w[b])
 * rows of grid_w[b] tokens at time 0; a kept token idx keeps its grid position
 * (0, idx / grid_w, idx % grid_w); the text after it continues on all three
 * components from max(rows, grid_w[b]) (the unpruned image block's largest
 * position + 1).  Row cu + j of sequence b (cu = sum over earlier images of
 * count + n_txt, the packing of sp_compact) gets the j-th position.
 *   n_vis, n_txt, grid_w: HOST [B];  idx [B, k_cap], count [B]: DEVICE (sp_select)
 *   pos3: DEVICE [T_cap, 4] int32 out (rows >= the packed length untouched)
 * Errors: bad sizes -> SP_ERR_SHAPE; on the device, an index outside its image
 * or a row >= T_cap sets SP_DEVERR_INDEX (the row is skipped).
 */
SP_API sp_status sp_mrope_positions(int B, const int* n_vis, const int* n_txt, const int* grid_w, const int* idx,
                                    int k_cap, const int* count, int* pos3, int T_cap, int* err, sp_stream stream);

SP_API size_t sp_prefill_workspace(const sp_model* m, int T_cap, int max_seqlen_cap);
SP_API sp_status sp_prefill(const sp_model* m, const sp_prefill_io* io, void* workspace,
                     size_t workspace_bytes, sp_stream stream);

/*
 * One generation step after the prefill (the decode whose per-token latency
 * the pruned prefix lowers): every sequence b appends one token x[b] at
 * position lens[b], which attends to the cached keys / values 0..lens[b]-1
 * (written by sp_prefill's kv, or by earlier steps) and to itself; the layers
 * are the prefill's, applied to that one row.  The step writes the new
 * token's rotated key / value into the cache at position lens[b], the final
 * RMSNorm of its last residual into hidden[b], and then increments lens[b]
 * (on the device, so steps chain without a host round trip).
 * Errors: a position >= kv_S_cap sets SP_DEVERR_INDEX (nothing is written
 * for that sequence's cache row); more than 8 query heads per key / value
 * head -> SP_ERR_UNSUPPORTED.  max_len_cap sizes the attention's key split
 * only: a longer sequence is still attended in full (its ranges grow).
 */
typedef struct {
  int B;                    /* sequences, as in the prefill that wrote kv */
  const void* x;            /* DEVICE [B, d] bf16: the new token of each sequence */
  int* lens;                /* DEVICE [B] int32: cached positions per sequence; incremented */
  void* kv;                 /* DEVICE cache, layout of sp_prefill_io.kv */
  int kv_S_cap;             /* positions per sequence in kv */
  int max_len_cap;          /* bound on lens[b] + 1 (sizes the attention launch) */
  float* hidden;            /* DEVICE [B, d] fp32 output */
  int* err;
  int* rope_pos;            /* DEVICE [B] int32 rotary position of each new token, or NULL (= lens);
                               incremented with lens.  After an mRoPE prefix: the position the
                               next text token takes (on all three components, so the 1-D
                               rotation at that position) */
} sp_decode_io;

SP_API size_t sp_decode_workspace(const sp_model* m, int B);
SP_API sp_status sp_decode(const sp_model* m, const sp_decode_io* io, void* workspace, size_t workspace_bytes,
                           sp_stream stream);

/* ------------------------------------------------------------------------ */
/* Several sequences over one prefix: a paged cache and beams.                */
/* ------------------------------------------------------------------------ */

/*
 * Samples and beams of a question continue the same pruned prefix (another
 * question keeps other tokens; questions share an unpruned one).  In a paged cache
 * they share its keys and values: a pool of pages of page_size positions, and per
 * sequence a table of its pages.  Position p of a sequence is row p % page_size of
 * page table[p / page_size].  One layer's pool is
 *   kv  DEVICE [2][n_pages][page_size][n_kv_heads * head_dim] bf16 (K, then V).
 * Table entries behind a sequence's pages are not read (-1, say).  A page
 * outside 0..n_pages-1 where one is needed sets SP_DEVERR_INDEX; nothing is
 * written for it, and read it counts as keys and values of zero.
 */
typedef struct {
  void* kv;                 /* DEVICE pool of one layer, 16-byte aligned */
  int n_pages;              /* n_pages * page_size <= 2^30 */
  int page_size;            /* a power of two, 16..1024 */
  const int* table;         /* DEVICE [B, max_pages] int32 */
  int max_pages;
  const int* lens;          /* DEVICE [B] int32 positions per sequence (each call says which) */
} sp_paged_kv;

/*
 * Appends rows to the cache, rotated on the way: row j of sequence b goes to
 * position cache.lens[b] + j (lens: the positions cached before; NULL: 0).
 *   rope  DEVICE [max_pos, head_dim / 2, 2] fp32 (cos, sin) of each rotary
 *         position and pair; pair i of a head is its elements i and
 *         i + head_dim / 2 (as in sp_prefill).  NULL: rows are already rotated.
 *   pos   DEVICE [T_cap] rotary position of each row; or
 *   pos3  DEVICE [T_cap, 4] (t, h, w, unused) with mrope_section as in
 *         sp_model_cfg (sp_mrope_positions writes it).
 * Queries and keys are rotated in fp32 and rounded once; values are copied.
 * q_out may be qkv itself (with ld_q = ld): the queries are then rotated in
 * place.  lens is not changed.  Rows outside cu_rows[0] .. cu_rows[B] - 1 are
 * not read.  A position outside its table or a rotary position outside
 * 0..max_pos-1 sets SP_DEVERR_INDEX and the row's keys and values (for a rotary
 * position its queries too) are skipped.
 */
typedef struct {
  int B;                    /* sequences, 1..SP_MAX_BATCH */
  int T_cap;                /* rows of qkv, at most 2^31 - 1; B without cu_rows */
  const int* cu_rows;       /* DEVICE [B + 1] ascending: sequence b's rows; NULL: row b is sequence b's */
  const void* qkv;          /* DEVICE [T_cap, ld] bf16: q | k | v of every row */
  long long ld;             /* elements between rows, a multiple of 8 */
  void* q_out;              /* DEVICE [T_cap, ld_q] bf16, or NULL: keys and values only */
  long long ld_q;
  int n_heads, n_kv_heads, head_dim;  /* head_dim 64 or 128 */
  const float* rope;
  int max_pos;
  const int* pos;
  const int* pos3;
  int mrope_section[3];
  sp_paged_kv cache;
  int* err;                 /* DEVICE error word or NULL */
} sp_paged_append_io;

SP_API sp_status sp_paged_append(const sp_paged_append_io* io, sp_stream stream);

/*
 * Attention of rows whose sequences share prefixes.  The sequences
 * group_cu[g] .. group_cu[g+1] - 1 share prefix g: prefix_lens[g] positions of
 * the same pool, in the pages of prefix_table.  Row j of sequence b (of its
 * n_b rows) sees its group's whole prefix and, of the sequence's own
 * cache.lens[b] positions (these rows' own keys, appended before, among them),
 * those up to lens[b] - n_b + j.  Sequences outside every group have no prefix.
 *   out = softmax(scale <q, k>) v over the visible keys, lse = log sum exp of
 *   the scaled scores; a row that sees no key, or only keys with a score of
 *   -infinity, gets zeros and lse -infinity.
 * A prefix is read once for all rows that share it (in small calls by several
 * CTAs, from the L2 cache).  Scores, statistics and sums are fp32; the weights are rounded to bf16 for the product with V.
 * Lengths are read on the device (they may change between replays of a graph);
 * the workspace depends on the arguments of its query alone and keeps nothing
 * (calls whose GPU work overlaps need one each).
 * A call may have as much work as the arguments' limits allow while the sum, over
 * the prefixes and the sequences, of (rows * n_heads + 128 n_kv_heads) *
 * (keys + 1024) is at most 2^38 (its rows are those that read these keys); a call
 * of several times that sets SP_DEVERR_INDEX and gives zeros and lse -infinity.
 * A NaN in a query, or in a key that it sees, makes that query's output and lse
 * NaN.
 * A NaN or infinity in V at a sequence's own position can also reach that
 * sequence's earlier rows of the same call (a weight of zero times it is NaN),
 * never another sequence.
 * Rows outside cu_rows[0] .. cu_rows[B] - 1 are left as they were.  The result
 * does not depend on timing (no atomics); it is summed in an order that depends
 * on the lengths of the whole batch and on how wide the tables are (which also
 * decide how the call is cut: tables much wider than their contents cost time).
 */
typedef struct {
  int B;                    /* sequences, 1..SP_MAX_BATCH */
  int T_cap;                /* rows of q; B without cu_rows; T_cap * n_heads <= 2^28 */
  const int* cu_rows;       /* DEVICE [B + 1] ascending, or NULL: one row per sequence */
  const void* q;            /* DEVICE [T_cap, ld_q] bf16 rotated queries */
  long long ld_q;           /* elements between rows, a multiple of 8 */
  void* out;                /* DEVICE [T_cap, ld_out] bf16 (must not overlap q) */
  long long ld_out;
  float* lse;               /* DEVICE [T_cap, n_heads] fp32 or NULL */
  int n_heads, n_kv_heads, head_dim;
  float scale;              /* 0: 1 / sqrt(head_dim) */
  sp_paged_kv cache;        /* lens: own positions, the rows of this call included */
  int n_groups;             /* 0..SP_MAX_BATCH; 0: no prefixes (the group arguments are ignored) */
  const int* group_cu;      /* DEVICE [n_groups + 1] ascending */
  const int* prefix_table;  /* DEVICE [n_groups, prefix_max_pages] int32 */
  int prefix_max_pages;
  const int* prefix_lens;   /* DEVICE [n_groups] */
  int* err;                 /* DEVICE error word or NULL */
} sp_prefix_attention_io;

SP_API size_t sp_prefix_attention_workspace(int T_cap, int B, int n_groups, int n_heads, int n_kv_heads,
                                            int head_dim);
SP_API sp_status sp_prefix_attention(const sp_prefix_attention_io* io, void* workspace, size_t workspace_bytes,
                                     sp_stream stream);

/*
 * The model over a paged cache.  pools is the pools of all layers one after the
 * other (kv [n_layers][2][n_pages][page_size][n_kv_heads * head_dim]), lens is
 * ignored.
 * sp_prefill_paged: sp_prefill (workspace and results are its) with the keys and
 * values put into pages: row j of sequence b at position j of table row b;
 * io.kv must be NULL.
 */
SP_API sp_status sp_prefill_paged(const sp_model* m, const sp_prefill_io* io, const sp_paged_kv* pools, void* workspace,
                                  size_t workspace_bytes, sp_stream stream);

/*
 * One generation step over pages, sequences sharing prefixes: the layers of
 * sp_decode applied to the new token x[b] of every sequence (queries and keys
 * rotated in fp32 and rounded once, as there), its keys and values appended at
 * the sequence's own position lens[b] (sp_paged_append) and its attention over
 * its group's prefix and its own pages (sp_prefix_attention).
 * lens and rope_pos are then incremented on the device, so steps chain.  (After a
 * prefix of L positions rope_pos starts at L, after an mRoPE prefix at the
 * position its next text token takes.)  A position outside the table, or a rotary
 * position outside 0..max_pos-1, sets SP_DEVERR_INDEX and is not written.
 */
typedef struct {
  int B;                    /* sequences, 1..SP_MAX_BATCH */
  const void* x;            /* DEVICE [B, d] bf16: the new token of each sequence */
  int* lens;                /* DEVICE [B] own cached positions; incremented */
  int* rope_pos;            /* DEVICE [B] rotary position of each new token; incremented */
  sp_paged_kv cache;        /* pools of all layers; table [B, max_pages]: the sequences' own pages; lens ignored */
  int n_groups;             /* as in sp_prefix_attention_io */
  const int* group_cu;
  const int* prefix_table;
  int prefix_max_pages;
  const int* prefix_lens;
  float* hidden;            /* DEVICE [B, d] fp32 output */
  int* err;                 /* DEVICE error word or NULL */
} sp_decode_paged_io;

SP_API size_t sp_decode_paged_workspace(const sp_model* m, int B, int n_groups);
SP_API sp_status sp_decode_paged(const sp_model* m, const sp_decode_paged_io* io, void* workspace,
                                 size_t workspace_bytes, sp_stream stream);

/*
 * Beam search's selection: of the W beams of each of B elements and the V
 * tokens, the n_out continuations with the largest
 *   cum[w] + log softmax(logits[w])[v],
 * best first.  Scores are compared in 64 bits; equal ones go to the lower beam,
 * then the lower token (within a beam the order is that of the logits).  A
 * row's sum is taken in fp32, good to about 2^-20 of it: scores of two beams that
 * are nearer than that can change places.  Beams of an element with equal logits
 * have equal sums, to the bit.  (Row strides that are no multiple of 16 bytes take
 * up to a fifth longer.)
 *   - A beam with cum -infinity (or NaN) is not alive: it proposes nothing.
 *   - A finished beam (done != 0) proposes only itself: token eos, score cum;
 *     its logits have no effect, whatever they hold (some of them are read).
 *   - NaN and -infinity logits have no weight and are never chosen; a row with
 *     +infinity spreads its weight over them (the softmax's limit).
 * Places for which no continuation is left get score -infinity, parent and
 * token -1.  The workspace keeps nothing; calls whose GPU work overlaps need one
 * each.
 */
typedef struct {
  int B, W, V;              /* 1..SP_MAX_BATCH, 1..SP_MAX_BEAMS, 1..2^24 */
  const void* logits;       /* DEVICE [B * W, ld] fp32 or bf16, aligned to its type */
  int logits_f32;           /* 1: fp32, 0: bf16 */
  long long ld;             /* elements between rows, at least V */
  const float* cum;         /* DEVICE [B, W] */
  const unsigned char* done;/* DEVICE [B, W] or NULL */
  int eos;
  int n_out;                /* 1..2 SP_MAX_BEAMS */
  float* score;             /* DEVICE [B, n_out] */
  int* parent;              /* DEVICE [B, n_out] beam of the element */
  int* token;               /* DEVICE [B, n_out] */
} sp_beam_select_io;

SP_API size_t sp_beam_select_workspace(int B, int W, int V, int n_out);
SP_API sp_status sp_beam_select(const sp_beam_select_io* io, void* workspace, size_t workspace_bytes,
                                sp_stream stream);

/*
 * Puts the cache of every element's beams into a new order: beam w becomes a
 * continuation of beam parent[w] (of the same element; -1: of itself).  Row
 * e * W + w of table and own_table belongs to beam w of element e; lens are the
 * positions cached, equal for the beams of an element.
 * own_table names pages of each beam's own for every place of its table, in
 * which no other row of own_table has a page; it does not change.  table starts
 * as a copy of it.  A beam appends to table[len / page_size], which is then its
 * own page: after this call table holds the parent's entries for full pages
 * (never written again, so shared) and the beam's own behind them, and the rows
 * of the partly filled page are copied from the parent's own page, all layers.
 * Unequal lengths, a length outside the table or a parent outside -1..W-1 set
 * SP_DEVERR_INDEX: such an element stays as it was (such a parent: -1).
 */
typedef struct {
  int B, W;                 /* elements, beams */
  int n_layers;             /* pools, one after the other */
  void* kv;                 /* DEVICE [n_layers][2][n_pages][page_size][row_elems] bf16 */
  int n_pages, page_size;   /* as in sp_paged_kv */
  int row_elems;            /* n_kv_heads * head_dim, a multiple of 8 */
  int* table;               /* DEVICE [B * W, max_pages], updated */
  const int* own_table;     /* DEVICE [B * W, max_pages] */
  int max_pages;
  const int* lens;          /* DEVICE [B * W] */
  const int* parent;        /* DEVICE [B, ld_parent] (sp_beam_select's) */
  int ld_parent;
  int* err;                 /* DEVICE error word or NULL */
} sp_beam_reorder_io;

SP_API sp_status sp_beam_reorder(const sp_beam_reorder_io* io, sp_stream stream);

/*
 * Verification of drafted tokens (speculative sampling), and without drafts the
 * sampling of a token for every sequence.  Sequence b has the rows
 * cu_rows[b] .. cu_rows[b + 1] - 1 of logits, n of them: row j holds the target's
 * logits behind its j-th drafted token draft[row j], the last row those behind
 * all of them (its draft is not read).  With t = temperature[b],
 * p_j = softmax(logits[row j] / t) and q_j = softmax(draft_logits[row j] / t):
 *   - draft j stays iff u[row j] q_j(d_j) < p_j(d_j) and those before it do;
 *   - the token after the a that stay is argmax r(v) / noise[b, v] over the tokens
 *     with r(v) > 0, of equal ones the lowest, with r = max(p_a - q_a, 0) where a
 *     draft was rejected (p_a if that leaves nothing) and r = p_a behind the last.
 *     With u uniform in [0, 1) and noise exponentially distributed with mean 1
 *     tokens are distributed as the target's.
 *   - Drafts without draft_logits are taken as certain (q_j is 1 at d_j): of a
 *     rejected one's row the others are left.
 * A sequence is greedy where temperature[b] is not above 0, and every one is
 * without noise: drafts stay while they are the target's largest logit (of equal
 * ones the lowest token), which is the next token too; u, noise and draft_logits
 * have no effect on it, and log-probabilities are those at temperature 1.
 *   n_accept[b] = a, token[b] = the drafts that stay, the next token and -1 behind
 *   it, logp[b] = log p of each (0 behind them).  A sequence without rows gets
 *   n_accept -1, one with more than max_rows, or rows outside 0 .. T_cap - 1, sets
 *   SP_DEVERR_INDEX besides.  A draft outside the vocabulary is rejected; where that
 *   ends its sequence SP_DEVERR_INDEX is set.
 * NaN and -infinity logits have no weight, nor have those whose weight is below 2^-126
 * of the row's largest; a row with +infinity spreads its weight over them.  A token
 * whose noise is NaN or below 0 is not drawn.  Where no token can be drawn (a row
 * without weight) the next token is -1, its logp -infinity.  A draft with u NaN is
 * rejected.
 * Sums are fp32, good to 2^-17.5: the answers move only where u q and p, or the two
 * best scores of a race, are nearer than (200 + 5 z) 2^-24 of p and q, for tokens
 * 2^-z times as likely as the row's likeliest (2^-16 for z up to 11).
 * The workspace keeps nothing; calls whose GPU work overlaps need one each.  One for
 * T_cap, B and V is enough for every call of no more of each.  max_rows is to be near
 * what sequences have: thread blocks are launched for B * max_rows rows (256 sequences
 * of two rows: 24 us with max_rows 2 or 9, 47 with 64, 440 with 1,024).
 */
typedef struct {
  int B, V;                 /* 1..SP_MAX_BATCH, 1..2^24 */
  int T_cap;                /* rows of logits, 0..2^24; B without cu_rows */
  int max_rows;             /* of a sequence, 1..SP_MAX_DRAFT_ROWS: drafts + 1 */
  const int* cu_rows;       /* DEVICE [B + 1] ascending, or NULL: one row per sequence */
  const void* logits;       /* DEVICE [T_cap, ld] fp32 or bf16, aligned to its type */
  int logits_f32;           /* 1: fp32, 0: bf16 (draft_logits too) */
  long long ld;             /* elements between rows, at least V */
  const int* draft;         /* DEVICE [T_cap]; may be NULL with max_rows 1 */
  const void* draft_logits; /* DEVICE [T_cap, ld_draft], or NULL (a sequence's last row is not read) */
  long long ld_draft;
  const float* u;           /* DEVICE [T_cap]; may be NULL with max_rows 1 or without noise */
  const float* noise;       /* DEVICE [B, ld_noise], or NULL: every sequence is greedy */
  long long ld_noise;
  const float* temperature; /* DEVICE [B], or NULL: 1 */
  int* n_accept;            /* DEVICE [B] */
  int* token;               /* DEVICE [B, max_rows] */
  float* logp;              /* DEVICE [B, max_rows] or NULL */
  int* err;                 /* DEVICE error word or NULL */
  int clear_err;            /* 1: the call sets *err to 0 first (a word of its own) */
} sp_draft_verify_io;

SP_API size_t sp_draft_verify_workspace(int T_cap, int B, int V);
SP_API sp_status sp_draft_verify(const sp_draft_verify_io* io, void* workspace, size_t workspace_bytes,
                                 sp_stream stream);

/*
 * The pages of a cache that sequences share.  Row s of table names the pages of
 * sequence s (negative: none), lens[s] its cached positions, and refs[p] is the
 * number of table entries that name page p: 0 where it is free.  Prefixes that
 * sequences share (sp_prefix_attention's) are rows as well.  A program begins with
 * an empty table (-1) and zeros in lens and refs; these calls keep the books, and
 * it adds to lens what it appends.  They all work on the state of the tables
 * before the call: order of the rows matters only where pages run out.
 *   sp_pages_trim     entries behind the page of a row's last position are
 *                     released: what a rejected draft had, or (with lens 0) all of
 *                     an ended sequence's.
 *   sp_pages_fork     row s becomes a continuation of row parent[s] (-1 or s: it
 *                     stays): it takes the pages of the parent's lens positions,
 *                     and its length; its own are released.  Nothing is copied.
 *   sp_pages_reserve  row s gets room for add[s] positions behind its lens: a page
 *                     where its table has none, and one of its own in place of one
 *                     that other entries name, into which the positions it has there
 *                     are copied (all layers).  lens does not change.  (A page that
 *                     several rows of a call write to is copied for each of them.)
 *   sp_pages_compact  row s keeps positions keep[s][0 .. count[s] - 1], in that
 *                     order (count -1: it stays): leading pages whose positions stay
 *                     in place are kept, the others go to pages of its own and the
 *                     old ones are released; lens[s] becomes count[s].  Other rows
 *                     that share the old pages keep them as they are.
 * Fresh pages are the free ones of the lowest numbers before the call, in order of
 * rows and their places.  If they do not suffice, rows are served from the first on
 * until one does not fit: it and those behind it stay as they were, and
 * SP_DEVERR_PAGES is set.
 * A length outside the table, a parent outside -1 .. S - 1, or a count outside
 * -1 .. keep_cap sets SP_DEVERR_INDEX and the row stays as it was.  An entry of
 * n_pages or more that a call takes, replaces or releases sets SP_DEVERR_INDEX and
 * counts as none; a position of keep outside the row (keep[i] = i at or behind its
 * length, too) sets it and what it would have moved is undefined.
 * The workspace (reserve, compact) keeps nothing; calls whose GPU work overlaps need
 * one each.
 */
typedef struct {
  void* kv;                 /* DEVICE [n_layers][2][n_pages][page_size][row_elems] bf16 (reserve, compact) */
  int n_layers;             /* 1..SP_MAX_LM_LAYERS */
  int n_pages, page_size;   /* as in sp_paged_kv */
  int row_elems;            /* n_kv_heads * head_dim, a multiple of 8 */
  int S;                    /* rows of table, 1..SP_MAX_TABLE_ROWS */
  int* table;               /* DEVICE [S, max_pages] */
  int max_pages;            /* S * max_pages at most 2^30 */
  int* lens;                /* DEVICE [S] */
  int* refs;                /* DEVICE [n_pages], 16-byte aligned */
  int* err;                 /* DEVICE error word or NULL */
} sp_pages;

SP_API sp_status sp_pages_trim(const sp_pages* p, sp_stream stream);
SP_API sp_status sp_pages_fork(const sp_pages* p, const int* parent, sp_stream stream);
SP_API size_t sp_pages_workspace(int S, int max_pages);
SP_API sp_status sp_pages_reserve(const sp_pages* p, const int* add, void* workspace, size_t workspace_bytes,
                                  sp_stream stream);
/* keep: DEVICE [S, ld_keep], its first keep_cap columns; S * keep_cap at most 2^30.  count: DEVICE [S]. */
SP_API sp_status sp_pages_compact(const sp_pages* p, const int* keep, long long ld_keep, int keep_cap,
                                  const int* count, void* workspace, size_t workspace_bytes, sp_stream stream);

/* ------------------------------------------------------------------------ */
/* The whole path: select -> compact -> project -> prefill.                  */
/* ------------------------------------------------------------------------ */

/*
 * Algorithm 1 (Sec. 3.5) end to end on the device, followed by the prefill
 * over its result: the text projection and the encoder (Eq. 3), the pointer
 * rounds of Eq. 4 / Eq. 11 with the STOP action per episode, the restore to
 * native order, the gather into packed sequences [kept visual rows; text
 * rows] (Sec. 3.3, last paragraph), the projector on the kept rows, and the
 * LM prefill of sp_prefill.  One stream, no host synchronisation: sizes that
 * depend on the selection stay on the device (grids are sized from caps).
 * Outputs: idx / count as sp_select's, cu_seqlens as sp_compact's, hidden as
 * sp_prefill's.  Errors: the union of those of the four calls; the
 * workspace must hold sp_pipeline_workspace() bytes (SP_ERR_WORKSPACE).
 */
typedef struct {
  sp_select_in sel;          /* X and E_text required (H ignored); E_text is also the
                                text rows of the LM input, so D_text must equal d */
  int k_cap;                 /* row stride of idx */
  int* idx;                  /* DEVICE [B, k_cap] */
  int* count;                /* DEVICE [B] */
  int* cu_seqlens;           /* DEVICE [B + 1] */
  float* hidden;             /* DEVICE [T_cap, d] fp32 (T_cap = sp_packed_cap(...)) */
  int* err;                  /* DEVICE error word or NULL */
} sp_pipeline_io;

SP_API size_t sp_pipeline_workspace(const sp_selector* s, const sp_model* m, const sp_pipeline_io* io);
SP_API sp_status sp_pipeline(const sp_selector* s, const sp_model* m, const sp_pipeline_io* io,
                      void* workspace, size_t workspace_bytes, sp_stream stream);

/*
 * The same path from HOST buffers: copies X, E_text and stop_bias (HOST, best
 * pinned) into the workspace, runs sp_pipeline, and copies idx, count,
 * cu_seqlens and the T_cap hidden rows back into the HOST outputs, all on
 * `stream`.  The host buffers must stay valid until the stream reaches the end
 * of the call.  The io's DEVICE pointer fields are ignored; host_* are used.
 */
typedef struct {
  sp_select_in sel;          /* X, E_text, stop_bias are HOST pointers here */
  int k_cap;
  int* host_idx;             /* HOST [B, k_cap] */
  int* host_count;           /* HOST [B] */
  int* host_cu_seqlens;      /* HOST [B + 1] */
  float* host_hidden;        /* HOST [T_cap, d] */
} sp_pipeline_host_io;

SP_API size_t sp_pipeline_host_workspace(const sp_selector* s, const sp_model* m,
                                  const sp_pipeline_host_io* io);
SP_API sp_status sp_pipeline_host(const sp_selector* s, const sp_model* m, const sp_pipeline_host_io* io,
                           void* workspace, size_t workspace_bytes, sp_stream stream);

/* ------------------------------------------------------------------------ */
/* Failure-detection self-test (the paper has no counterpart).               */
/* ------------------------------------------------------------------------ */

/*
 * Every wait in this library's kernels is bounded (2 s): one that runs out
 * sets SP_DEVERR_TIMEOUT in the call's error word and the kernel returns, so a
 * lost arrival never hangs the GPU.  This call runs the two wait helpers the
 * kernels use, with limit_us microseconds (1 .. 2,000,000) in place of 2 s:
 *   out[0] = 1 if a wait on an mbarrier completed, 0 if it timed out,
 *   out[1] = 1 if a wait for *flag == 1 completed, 0 if it timed out.
 * The mbarrier gets no arrival (so the wait runs out) unless `complete` is
 * non-zero; the flag wait completes iff the caller's DEVICE int *flag is 1.
 * A timeout ORs SP_DEVERR_TIMEOUT into *err (DEVICE, may be NULL);
 * sp_device_error_status() maps it to SP_ERR_TIMEOUT.  The stream and the
 * context stay usable.  flag, out: DEVICE.  Asynchronous on `stream`.
 * Errors: SP_ERR_INVALID_ARG (NULL flag / out), SP_ERR_SHAPE (limit out of
 * range), SP_ERR_CUDA.
 */
SP_API sp_status sp_wait_probe(const int* flag, unsigned int limit_us, int complete, int* out, int* err,
                               sp_stream stream);

/* ------------------------------------------------------------------------ */
/* Per-kernel timing (CUDA events recorded around every launch).             */
/* ------------------------------------------------------------------------ */

typedef enum {
  SP_K_GEMM = 0, SP_K_SGEMM = 1, SP_K_ATTN = 2, SP_K_NORM = 3, SP_K_SELECT = 4,
  SP_K_RESTORE = 5, SP_K_COMPACT = 6, SP_K_MISC = 7, SP_K_TRAIN = 8, SP_K_COUNT = 9
} sp_kernel_kind;

/* Starts (capacity > 0) or stops (0) recording launch events; host-allocated. */
SP_API sp_status sp_profile_begin(int capacity);
/* Synchronises on the recorded events and returns, per sp_kernel_kind, the
 * summed milliseconds, launch counts and algorithmic flops / bytes. */
SP_API sp_status sp_profile_end(double* ms, long long* launches, double* flops, double* bytes);

#ifdef __cplusplus
}
#endif
#endif /* STEPPRUNE_H */
