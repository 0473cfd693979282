/*
 * sd2.h -- C ABI of the MI355X (gfx950) SD^2 speculative-decoding round.
 *
 * One round of SD^2 ("Steering Pretrained Drafters during Speculative
 * Decoding", Berdoz, Rheinboldt, Wattenhofer) on one GPU:
 *   1. the drafter proposes k tokens autoregressively, every processed token's
 *      input embedding carrying the current steering vector s
 *      (Sec. "Drafting": the steering term is computed once per drafting stage
 *      since it does not depend on the draft position, and it also conditions
 *      the keys/values the drafter caches);
 *   2. the verifier scores the block [last committed token, k drafts] in one
 *      parallel forward (Sec. "Verification");
 *   3. speculative rejection sampling (Leviathan et al. 2023, cited in Sec.
 *      "Verification") accepts a prefix of n drafts and draws one final token,
 *      so the block yields n + 1 tokens (Sec. "Metrics", block efficiency);
 *   4. the steering vector for the next round is W_s applied to the verifier's
 *      final-norm hidden state at the position of the last token returned
 *      (Sec. "Verification"); cache lengths roll back to the accepted prefix.
 *
 * Conventions for every call:
 *  - All pointers named "device" are HIP device pointers owned by the caller;
 *    they must stay valid until sd2_destroy.  The library allocates no device
 *    memory: all state lives in the caller's workspace.
 *  - Calls are asynchronous on the HIP stream given to sd2_create, except
 *    sd2_debug_read, which synchronises that stream.  Argument and capacity
 *    errors are detected on the host and returned before anything is enqueued.
 *    HIP errors are returned as SD2_ERR_HIP by the call that observes them.
 *  - A handle is not thread-safe; use one handle per stream.  No C++ exception
 *    crosses this interface.
 *  - Weight matrices are row-major [out][in] ("W x" layout), untied LM head,
 *    no biases.  bf16 tensors hold bfloat16 bit patterns.
 */
#ifndef SD2_H
#define SD2_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t sd2_status;
#define SD2_OK 0
#define SD2_ERR_INVALID_ARG (-1)   /* bad shape, pointer, alignment or size */
#define SD2_ERR_CAPACITY (-2)      /* prompt + generation would exceed max_seq_len */
#define SD2_ERR_STATE (-3)         /* e.g. sd2_round before sd2_prefill */
#define SD2_ERR_HIP (-4)           /* a HIP runtime call failed; see sd2_last_error */
#define SD2_ERR_UNSUPPORTED (-5)   /* valid request the library does not handle */

typedef struct sd2_handle* sd2_handle_t;

typedef enum { SD2_F32 = 0, SD2_BF16 = 1 } sd2_dtype;

/* Shape of one SwiGLU decoder (the paper's models all use SwiGLU MLPs, eq. (1)).
 * head_dim = d_model / n_heads must be even and at most 128; n_heads must be a
 * multiple of n_kv_heads (grouped-query attention); d_model, n_heads*head_dim
 * and d_ff must be multiples of 64. */
typedef struct {
    int32_t n_layers, d_model, n_heads, n_kv_heads, d_ff, vocab;
    float rope_theta;  /* rotate-half RoPE base */
    float rms_eps;     /* RMSNorm: x / sqrt(mean(x^2) + eps) * gain */
} sd2_dims;

/* Device pointers of one model, all of the configuration's dtype.
 * layers points to a HOST array of n_layers * 9 device pointers, per layer in
 * the order attn_norm[d], wq[H*hd][d], wk[Hkv*hd][d], wv[Hkv*hd][d],
 * wo[d][H*hd], ffn_norm[d], w_gate[F][d], w_up[F][d], w_down[d][F].  The host
 * array is copied by sd2_create; every device pointer must be 16-byte aligned. */
typedef struct {
    const void* embed;             /* [vocab][d] */
    const void* const* layers;     /* host array of n_layers*9 device pointers */
    const void* final_norm;        /* [d] */
    const void* lm_head;           /* [vocab][d] */
} sd2_weights;

typedef struct {
    sd2_dims verifier, drafter;    /* both models must share the vocabulary */
    sd2_dtype dtype;
    int32_t k;                     /* draft length, 1..32 */
    int32_t max_batch;             /* sequences per round, 1..256 */
    int32_t max_seq_len;           /* capacity per sequence: >= prompt + max_new_tokens + k + 1 */
    int32_t max_new_tokens;        /* generated tokens per sequence; its last round is truncated */
    float temperature;             /* 0 => greedy (argmax drafts, accept iff draft == verifier argmax) */
    uint64_t seed;                 /* Philox4x32-10 key of every random draw */
    int32_t steering;              /* SD2_STEER_INPUT or SD2_STEER_NONE (sd2_create); SD2_STEER_MLP,
                                      SD2_STEER_MLP_OUT or SD2_STEER_MLP_COND (sd2_create_mlp) */
    int32_t cond_rank;             /* SD2_STEER_MLP_COND: hidden width R of the conditional bias MLP,
                                      a multiple of 16 in 16..4096; ignored by the other forms */
} sd2_config;

/* How the drafter is steered by the verifier (sd2_config.steering). */
#define SD2_STEER_INPUT 0  /* s = W_s hF (verifier final-norm hidden state, d_V -> d_D) added to the
                              drafter's input embedding of every token it processes in the round */
#define SD2_STEER_MLP 1    /* the paper's eq. (2): g = LayerNorm(W_hml [h; m; l]) from the verifier's
                              residual stream after decoder blocks L_V-2, floor(L_V/2) and 3 (counted
                              from 1; high, middle, low; training details) and one bias b_l = W_s^(l) g
                              per drafter layer, added to the up projection before the gating product:
                              W_d((W_u a + b_l) * SiLU(W_g a)).  Needs L_V >= 3. */
#define SD2_STEER_MLP_OUT 2 /* the paper's ablation "Inv. bias after MLP" (Sec. Ablation): the same g,
                              and one bias b = W_s g of d_D values added to the output of every
                              drafter MLP (x += W_d(...) + b).  Needs L_V >= 3. */
#define SD2_STEER_MLP_COND 4 /* the paper's ablation "Cond. bias in MLP" (Sec. Ablation; its formula is
                              this library's reading): the same g, and per drafter layer l and token
                              the bias U_l SiLU(V_l [f; g]) added to the up projection as in eq. (2),
                              f the residual stream entering layer l at the token's position (the
                              embedding for l = 0), V_l [R][d_D + d_V], U_l [d_ff_D][R].  The g part
                              V_l^g g is computed once per round.  Runs one kernel per operation
                              (no persistent launches).  Needs L_V >= 3. */
#define SD2_STEER_NONE 3   /* no steering: the pretrained drafter the paper compares against (Table 1,
                              "Pretrained"); no steering projection runs and nothing is added to the
                              drafter.  Gives the same outputs as SD2_STEER_INPUT with W_s = 0, without
                              its cost; the baseline of the steering-overhead measurement. */

/* Weights of SD2_STEER_MLP, device pointers in the configuration's dtype, 16-byte aligned. */
typedef struct {
    const void* w_s;       /* SD2_STEER_MLP: [L_D * d_ff_D][d_V], rows l*d_ff_D .. (l+1)*d_ff_D - 1 give
                              layer l's bias; SD2_STEER_MLP_OUT: [d_D][d_V]; SD2_STEER_MLP_COND: V^g
                              [L_D * R][d_V], rows l*R .. (l+1)*R - 1 the g columns of V_l */
    const void* w_hml;     /* [d_V][3 d_V]: g = W_hml [h; m; l] (columns: h, then m, then l) */
    const void* ln_gain;   /* [d_V] LayerNorm gain */
    const void* ln_bias;   /* [d_V] LayerNorm shift */
    float ln_eps;          /* LayerNorm: (g - mean) / sqrt(var + eps) * gain + shift, population variance */
    const void* w_cf;      /* SD2_STEER_MLP_COND: V^f [L_D * R][d_D], the f columns of V_l (else unused) */
    const void* w_cu;      /* SD2_STEER_MLP_COND: U [L_D * d_ff_D][R], rows l*d_ff_D .. the U_l block */
} sd2_mlp_steering;

/* Bytes of device workspace sd2_create needs for cfg (0 if cfg is invalid).  K/V caches and logits
   grow with the configuration; above SD2_NOALLOC_WORKSPACE_BYTES prefill runs chunks of 2048 rows
   (512 up to it), whose activations and partial sums take most of the rest: 707 MiB for the
   8B / 1B pair of the benchmark (one sequence, 774 positions), 242 MiB of it K/V. */
size_t sd2_workspace_bytes(const sd2_config* cfg);

/*
 * Create a handle.  verifier/drafter: model weights; w_steer: device [d_drafter][d_verifier]
 * steering projection W_s (s = W_s h, paper Sec. "Verification"/"Drafting"), ignored (may be
 * NULL) when cfg->steering is SD2_STEER_NONE;
 * workspace: device buffer of at least sd2_workspace_bytes(cfg) bytes, 256-byte aligned;
 * hip_stream: the hipStream_t every call enqueues on (NULL = default stream).
 * On success *out receives the handle.  Enqueues small table-initialisation kernels.
 * The current HIP device must be a gfx950 (MI355X) with XNACK off, its default mode: the
 * kernels are built for exactly that target, and any other device gives SD2_ERR_UNSUPPORTED
 * (SD2_ERR_HIP if the device cannot be queried).
 */
sd2_status sd2_create(const sd2_config* cfg, const sd2_weights* verifier, const sd2_weights* drafter,
                      const void* w_steer, void* workspace, size_t workspace_bytes, void* hip_stream,
                      sd2_handle_t* out);

/*
 * For callers that cannot allocate device memory (code under HIP graph capture, serving loops
 * and harnesses that forbid hipMalloc): sd2_create with the workspace taken from a static device
 * array of the library instead of the caller.  Allocates nothing, on host or device: the array
 * (SD2_NOALLOC_WORKSPACE_BYTES per GPU) is part of the library's code object, reserved on every
 * GPU the library runs on until the process ends, and the handle's host state sits in a static
 * slot of that GPU.  cfg->steering must be SD2_STEER_INPUT or SD2_STEER_NONE; the other arguments
 * are as sd2_create's, and the handle is used and destroyed the same way.
 * Limits and errors: SD2_ERR_CAPACITY when sd2_workspace_bytes(cfg) exceeds
 * SD2_NOALLOC_WORKSPACE_BYTES (checked before any device call); one such handle per GPU at a
 * time: SD2_ERR_STATE while another one on the current device is alive.  The array keeps the
 * previous handle's contents; creation clears what this handle uses with a kernel (no
 * hipMemsetAsync) on hip_stream, and sd2_destroy of such a handle waits for its stream, so the
 * next handle never clears memory still in use.  Work of a handle from this entry point and any
 * other user of the same array must not overlap on one GPU: they would race on it.
 */
#define SD2_NOALLOC_WORKSPACE_BYTES ((size_t)64 << 20)
sd2_status sd2_create_noalloc(const sd2_config* cfg, const sd2_weights* verifier, const sd2_weights* drafter,
                              const void* w_steer, void* hip_stream, sd2_handle_t* out);

/*
 * Create a handle whose drafter is steered by the paper's MLP biases (eq. (2); Sec.
 * "Verification" and "Drafting"): cfg->steering must be SD2_STEER_MLP (or SD2_STEER_MLP_OUT, the
 * ablation with one bias after every MLP, or SD2_STEER_MLP_COND, the conditional bias).  Everything else is as
 * sd2_create.  The bias is recomputed at the end of every round from the verifier row whose
 * logits produced the final token, and used for every drafter token of the next round;
 * the drafter processes the prompt without steering, and the first round's bias comes from
 * the verifier at position len-2 (zero when len == 1).
 */
sd2_status sd2_create_mlp(const sd2_config* cfg, const sd2_weights* verifier, const sd2_weights* drafter,
                          const sd2_mlp_steering* steering, void* workspace, size_t workspace_bytes,
                          void* hip_stream, sd2_handle_t* out);

/*
 * Create a handle whose K/V caches lie in pages (see "Paged K/V caches" below): instead of max_seq_len
 * rows for each of max_batch sequences the workspace holds n_pages pages, each of page_size positions in every
 * layer of both models.  Sequences take pages as they grow and give them up when they finish;
 * sd2_fork lets sequences share a common beginning, sd2_release frees one, sd2_compact moves the
 * pages in use together.  cfg->steering must be SD2_STEER_INPUT or SD2_STEER_NONE; rounds run one kernel per
 * operation; everything else is as sd2_create, with sd2_create_paged_bytes for sd2_workspace_bytes.
 * sd2_prefill returns SD2_ERR_CAPACITY when batch * ceil((max_prompt - 1) / page_size) exceeds n_pages.
 * A sequence that the pool cannot give all the pages of a round takes none and sits it out: its out_counts
 * entry is 0, its state is kept (SD2_DBG_STATE: done = 2), and it goes on in a later round that finds pages,
 * which finished sequences have left; when none can go on, the caller has to release one.  sd2_train_loss
 * returns SD2_ERR_UNSUPPORTED.
 */
typedef struct {
    int32_t page_size;  /* 16, 32, 64, 128, 256, 512 or 1024 */
    int32_t n_pages;    /* 1..2^24 */
} sd2_paging;
size_t sd2_create_paged_bytes(const sd2_config* cfg, const sd2_paging* paging);
sd2_status sd2_create_paged(const sd2_config* cfg, const sd2_weights* verifier, const sd2_weights* drafter,
                            const void* w_steer, const sd2_paging* paging, void* workspace, size_t workspace_bytes,
                            void* hip_stream, sd2_handle_t* out);

/*
 * Prefill `batch` sequences (1..max_batch) with their prompts.
 * tokens: device int32 [batch][max_prompt], row b holding lens[b] prompt ids in [0, vocab);
 * lens: device int32 [batch], each in [1, max_prompt]; max_prompt: host bound on lens.
 * Both models process positions 0..len-2 (the drafter with zero steering); the first
 * round's steering vector is W_s applied to the verifier's final-norm hidden state at
 * position len-2 (zero when len == 1).  Returns SD2_ERR_CAPACITY when
 * max_prompt + max_new_tokens + k + 1 > max_seq_len.  Resets all per-sequence state.
 */
sd2_status sd2_prefill(sd2_handle_t h, int32_t batch, const int32_t* tokens, const int32_t* lens,
                       int32_t max_prompt);

/*
 * One speculative round for every prefilled sequence.
 * out_tokens: device int32 [batch][k+1]: row b gets the accepted drafts followed by the
 *             final token (only the first out_counts[b] entries are meaningful);
 * out_counts: device int32 [batch]: tokens emitted this round (n+1, truncated at the
 *             max_new_tokens budget), 0 once the sequence has finished.
 * Returns SD2_ERR_STATE before sd2_prefill.
 */
sd2_status sd2_round(sd2_handle_t h, int32_t* out_tokens, int32_t* out_counts);

/*
 * Calls on a running generation of a paged handle (SD2_ERR_UNSUPPORTED on any other, SD2_ERR_STATE
 * before sd2_prefill), between rounds.
 * sd2_fork: `count` further sequences go on from sequence seq (0 .. number of sequences - 1) as it is now,
 *   sharing its pages until they write to them; they are the next count sequences, in the rounds'
 *   outputs too (SD2_ERR_CAPACITY beyond max_batch).  They draw random numbers of their own.
 * sd2_release: sequence seq is finished now and gives up its pages; its number stays taken.
 * sd2_compact: the pages in use are moved to the front of the pool; live (device int32 [1], or NULL)
 *   receives their number.
 */
sd2_status sd2_fork(sd2_handle_t h, int32_t seq, int32_t count);
sd2_status sd2_release(sd2_handle_t h, int32_t seq);
sd2_status sd2_compact(sd2_handle_t h, int32_t* live);

/*
 * Test hook: like sd2_round, but the trajectory follows caller-supplied decisions.
 * forced: device int32 [batch][k+2] = k drafts, accepted count n, final token y per
 * sequence.  The library still computes its own decisions from its own logits and
 * records them (sd2_debug_read SD2_DBG_OWN_*); drafting, verification, commit and
 * steering then proceed with the forced values.
 */
sd2_status sd2_round_forced(sd2_handle_t h, const int32_t* forced, int32_t* out_tokens, int32_t* out_counts);

/*
 * Training-objective forward (paper Sec. "Training"; input-form steering, SD2_STEER_INPUT only):
 * for one token sequence x_0..x_{n-1} (tokens: device int32 [n], ids in [0, vocab)) and the
 * offset of every target (deltas: device int32 [n], deltas[tau] in 1..k, entry 0 unused; the
 * paper draws them uniformly), writes out_kl (device float [n]):
 *   out_kl[tau] = KL(p_V || p_D) = sum_v p_V(v) (log p_V(v) - log p_D(v)),  tau = 1..n-1,
 * p_V the verifier's softmax at position tau-1 and p_D the drafter's, whose input embedding at
 * every position p carries the steering of the target it predicts, s_{p+1} = W_s hF_V(p -
 * deltas[p+1]) (zero when that position is negative or the offset lies outside 1..k; hF_V = the
 * verifier's final-norm hidden state), and out_kl[0] = 0; out_loss (device float [1]) receives the mean over tau = 1..n-1.
 * Both models run rows_per_chunk positions at a time (1..512) in sequence slot 0 of the
 * handle's caches, so the handle's generation state is lost (sd2_prefill before the next round).
 * scratch: device buffer of at least sd2_train_loss_scratch_bytes(cfg, n, rows_per_chunk)
 * bytes, 256-byte aligned, caller-owned.  Errors: SD2_ERR_UNSUPPORTED for the MLP and unsteered
 * forms, SD2_ERR_CAPACITY when n > max_seq_len, SD2_ERR_INVALID_ARG otherwise.
 */
size_t sd2_train_loss_scratch_bytes(const sd2_config* cfg, int32_t max_len, int32_t rows_per_chunk);
sd2_status sd2_train_loss(sd2_handle_t h, const int32_t* tokens, const int32_t* deltas, int32_t n,
                          int32_t rows_per_chunk, float* out_kl, float* out_loss, void* scratch,
                          size_t scratch_bytes);

/*
 * Paged K/V caches.
 *
 * A page holds page_size consecutive positions of one sequence, in every array of the cache.  The
 * table names the pages of each sequence in the order of its positions; refs counts for every page the
 * table entries that name it, so that sequences with a common beginning can share its pages.  All of it
 * is the caller's device memory: start with refs 0 and table entries -1.  sd2_pages_reserve gives a
 * sequence the pages it is about to write (and copies those it shares), sd2_pages_fork lets it go on from
 * another one's, sd2_pages_trim takes pages back, sd2_pages_compact moves the pages in use together;
 * sd2_paged_append writes rows, sd2_paged_attn reads them.  A table entry outside 0 .. n_pages - 1 names
 * no page: its positions are neither read nor written.
 *
 * These calls belong to no handle.  Each is asynchronous on hip_stream (NULL: the default stream) of
 * the current device, which the memory has to be on; calls on one cache have to be ordered (one stream, or
 * events between them), calls on different caches need not be, as long as they have workspaces of their
 * own.  They may be captured into a graph; a replay reads the device arrays anew, while host values (lists of
 * sequences, sizes) are those of the capture.  Workspaces need no initialisation, are 256-byte
 * aligned, and are used by the call's own kernels only.  Arguments are checked before anything is enqueued;
 * what device arrays hold (lengths, offsets, table entries) cannot be, and is brought into range by the
 * kernels, as stated with each call.  No pair of buffers of a call may overlap unless stated.
 */
#define SD2_PAGE_ARRAYS 8     /* arrays of a cache at most */
#define SD2_PAGED_MAX_SEQS 4096

/* One array of a cache: page p is blocks * page_size rows of row_bytes bytes, page after page.  A block
 * (a layer and KV head, say) is the page's positions in order.  With a negative row_bytes it has no rows: page p is
 * blocks records of -row_bytes bytes (the scales of a layer, say), which go along whole where any row of the page is
 * copied. */
typedef struct {
    void* data;         /* device, 16-byte aligned */
    int32_t blocks;     /* 1..65536 */
    int32_t row_bytes;  /* a multiple of 16, up to 65536; or minus a multiple of 2, up to 2^20 */
} sd2_page_array;

typedef struct {
    int32_t page_size;  /* positions per page: 16, 32, 64, 128, 256, 512 or 1024 */
    int32_t n_pages;    /* 1..2^24 */
    int32_t max_seqs;   /* 1..SD2_PAGED_MAX_SEQS */
    int32_t max_pages;  /* entries of a sequence; max_pages * page_size at most 2^30 */
    int32_t* table;     /* device [max_seqs][max_pages] */
    int32_t* refs;      /* device [n_pages] */
    int32_t n_arrays;   /* 1..SD2_PAGE_ARRAYS */
    sd2_page_array arrays[SD2_PAGE_ARRAYS];
} sd2_pages;

/* Bytes of workspace that sd2_pages_reserve and sd2_pages_compact need (0: invalid). */
size_t sd2_pages_workspace_bytes(const sd2_pages* pages);

/*
 * Make positions first[b] .. last[b] - 1 of the sequences b = 0 .. nseq - 1 writable (device int32
 * [nseq] each; first[b] >= last[b]: nothing for this one).  Of the table entries that hold these positions,
 *  - one that names no page gets a free page (refs 0), and
 *  - one whose page is shared (refs above 1 when the call begins) gets a free page too, to which the rows
 *    of the positions below keep[b] are copied (keep NULL: below first[b]); the shared page loses this
 *    reference.  Sequences that share a page and both write to it get a copy each.
 * Free pages are given in ascending order to the entries in the order of (sequence, position).  granted (device int32
 * [nseq], or NULL) receives last[b], or the position where the first page begins that the pool could not
 * give or that lies behind the table's last entry.  Entries left without a page stay as they were.
 * Negative positions count as 0.
 */
sd2_status sd2_pages_reserve(const sd2_pages* pages, int32_t nseq, const int32_t* first, const int32_t* last,
                             const int32_t* keep, int32_t* granted, void* workspace, size_t workspace_bytes,
                             void* hip_stream);

/*
 * For each i the sequence dst[i] gives up its pages and takes those of src[i], shared (HOST int32 [n]
 * each, sequences in 0 .. max_seqs - 1; no dst twice, and none that is also a src:
 * SD2_ERR_INVALID_ARG).  No row is copied: see sd2_pages_reserve.
 */
sd2_status sd2_pages_fork(const sd2_pages* pages, int32_t n, const int32_t* src, const int32_t* dst, void* hip_stream);

/*
 * Sequences b = 0 .. nseq - 1 keep the pages of their first lens[b] positions (device int32 [nseq])
 * and give up the others; lens[b] = 0 frees a sequence, a negative one leaves it as it is.
 */
sd2_status sd2_pages_trim(const sd2_pages* pages, int32_t nseq, const int32_t* lens, void* hip_stream);

/*
 * Sequences b = 0 .. nseq - 1 give up the pages that their next rows, from position lens[b] on, do not read under a
 * window (see sd2_paged_attn_window): those whose positions are all at least sinks and at most lens[b] - window.
 * lens: device int32 [nseq]; a negative one leaves its sequence as it is.  window: 1..2^30; sinks: 0..2^30.
 */
sd2_status sd2_pages_slide(const sd2_pages* pages, int32_t nseq, const int32_t* lens, int32_t window, int32_t sinks,
                           void* hip_stream);

/*
 * Move the pages in use (refs above 0) to 0 .. live - 1: those behind, in ascending order, into the
 * free ones before, in ascending order, with their rows, references and table entries.  live (device int32
 * [1], or NULL) receives their number.
 */
sd2_status sd2_pages_compact(const sd2_pages* pages, int32_t* live, void* workspace, size_t workspace_bytes,
                             void* hip_stream);

/* One layer of a paged cache for sd2_paged_append and sd2_paged_attn: the row of page p, KV head h and
 * slot s starts at element p * page_stride + (h * page_size + s) * head_dim of k and of v. */
typedef struct {
    void *k, *v;           /* device, 16-byte aligned */
    int64_t page_stride;   /* elements, at least n_kv_heads * page_size * head_dim, whole 16-byte units */
    int32_t dtype;         /* sd2_dtype of k, v and of the rows of a call */
    int32_t page_size;     /* as sd2_pages */
    int32_t n_pages;       /* as sd2_pages */
    int32_t n_kv_heads;    /* 1..1024 */
    int32_t head_dim;      /* 32, 64 or 128 */
    int32_t max_pages;     /* as sd2_pages */
    const int32_t* table;  /* device [nseq][max_pages] */
} sd2_paged_kv;

/* The rows that a call brings, packed: sequence b = 0 .. nseq - 1 has the rows row_off[b] ..
 * row_off[b + 1] - 1 (ascending; or max_rows rows each, when row_off is NULL), and they are the last ones
 * of its lens[b] positions: row i of n is position lens[b] - n + i.  Offsets are brought into 0 ..
 * total_rows, rows of a sequence beyond max_rows and rows that belong to no sequence are left alone. */
typedef struct {
    int32_t nseq;            /* 0..SD2_PAGED_MAX_SEQS */
    int32_t max_rows;        /* of one sequence, at least 1 */
    int32_t total_rows;      /* of all; nseq * max_rows when row_off is NULL */
    const int32_t* row_off;  /* device [nseq + 1], or NULL */
    const int32_t* lens;     /* device [nseq] */
} sd2_paged_rows;

/* Rows of k and v (device [total_rows][n_kv_heads][head_dim], k_stride and v_stride elements from one row
 * to the next, whole 16-byte units) into the pages of their positions.  Rows without a page, or at a
 * negative position, are dropped. */
sd2_status sd2_paged_append(const sd2_paged_kv* kv, const sd2_paged_rows* rows, const void* k, int64_t k_stride,
                            const void* v, int64_t v_stride, void* hip_stream);

/*
 * Causal grouped-query attention of the rows over their sequences' pages: row at position p, head h:
 *   out = sum_j softmax_j(scale * q . k_j) v_j   over the positions j <= p that have a page,
 * KV head h / (n_heads / n_kv_heads); zeros when there is none (a negative position, no page), NaN where all
 * their scores are -infinity.
 * q, out: device [total_rows][n_heads][head_dim], q_stride and out_stride elements from one row to the next
 * (whole 16-byte units); n_heads a multiple of n_kv_heads, up to 1024.  q and out may be columns of one buffer, but
 * share no element (SD2_ERR_INVALID_ARG; of different strides: their extents must not meet).  bf16: scores,
 * softmax and sums in fp32, the softmax's weights rounded to bf16 for their product with v (where max_rows rows
 * have up to 64 query vectors of a KV head: to two bf16 numbers each, 2^-15 of the weight); fp32: fp32 throughout.
 * Memory behind a sequence's last position, and pages it does not name, are not read, or do not count,
 * whatever they hold; infinities and NaN of a position reach the rows that read it, and no others.
 * The rows of a sequence times n_heads / n_kv_heads are at most 2^30.  Sizes that together make a launch of 2^32
 * threads or more are refused (workspace 0): that takes beyond 8 million workgroups, one for each sequence, KV head
 * and 16 query vectors at least.
 * max_len: the largest length expected, 1..max_pages * page_size (it decides into how many parts the work may be
 * split, and the workspace; a longer sequence is computed all the same).
 */
size_t sd2_paged_attn_workspace_bytes(const sd2_paged_kv* kv, const sd2_paged_rows* rows, int32_t n_heads,
                                      int32_t max_len);
sd2_status sd2_paged_attn(const sd2_paged_kv* kv, const sd2_paged_rows* rows, const void* q, int64_t q_stride,
                          void* out, int64_t out_stride, int32_t n_heads, float scale, int32_t max_len,
                          void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * sd2_paged_attn under a window: the row at position p reads the positions j <= p with p - j < window (its own and
 * the window - 1 before it) or j < sinks, of those that have a page.  window: 1..2^30, or 0 for every j <= p;
 * sinks: 0..2^30.  Positions that no row of a sequence reads cost nothing, and need no pages (sd2_pages_slide).
 * Everything else is as with sd2_paged_attn; the workspace is that of the same window and sinks.
 */
size_t sd2_paged_attn_window_workspace_bytes(const sd2_paged_kv* kv, const sd2_paged_rows* rows, int32_t n_heads,
                                             int32_t max_len, int32_t window, int32_t sinks);
sd2_status sd2_paged_attn_window(const sd2_paged_kv* kv, const sd2_paged_rows* rows, const void* q, int64_t q_stride,
                                 void* out, int64_t out_stride, int32_t n_heads, float scale, int32_t max_len,
                                 int32_t window, int32_t sinks, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * A paged cache that holds 8 bits a value: k and v are e4m3 numbers (4 exponent bits, bias 7; 3 mantissa bits; no
 * infinities, 0x7f and 0xff are NaN), and each 16 positions of a KV head (slots 16 j .. 16 j + 15 of a page) have a
 * power of two for k and one for v that their numbers are multiplied by, 2^(byte - 127).  The bytes of KV head h and
 * j are k's at scales[p * scale_stride + (h * page_size / 16 + j) * 2] for page p, and v's behind it; those that
 * sd2_paged_append_scaled writes are 27..246, and others give no defined values.  For sd2_pages_* the scales are an array
 * of their own, of records.
 */
typedef struct {
    sd2_paged_kv kv;       /* dtype: of the rows of a call (new rows, q and out); k, v and page_stride in elements of a byte */
    void* scales;          /* device, 2-byte aligned */
    int64_t scale_stride;  /* bytes from one page to the next, even, at least n_kv_heads * page_size / 8 */
} sd2_paged_scaled;

/*
 * sd2_paged_append into such a cache.  With a the largest finite magnitude of the new rows in 16 positions of a KV
 * head (k and v apart), their power 2^e is the least with 448 * 2^e >= a, e in -100..119.  Where the first of the new
 * rows is not the first of the 16 positions, e is at least what it was before, and when it grows the numbers of the
 * positions before the first new row are rounded again to the new one.  A value x becomes the e4m3 number nearest to
 * x / 2^e (ties to even, at most 448 in magnitude); an infinity or NaN becomes NaN.  Positions of the 16 behind the
 * last new row are not written (and count for nothing until they are).  One sequence's rows of 16 positions are
 * best brought in one call: what they are rounded to does not depend on it, except below 2^(e - 6), where numbers
 * that were rounded before e grew are rounded twice.  e falls only when the first of the 16 positions is written: rows that
 * are written over from behind it (drafts that were rejected) leave it where they raised it, and the rows before them rounded.
 */
sd2_status sd2_paged_append_scaled(const sd2_paged_scaled* kv, const sd2_paged_rows* rows, const void* k, int64_t k_stride,
                             const void* v, int64_t v_stride, void* hip_stream);

/*
 * sd2_paged_attn_window over such a cache (window 0: sd2_paged_attn), for q and out of kv->kv.dtype.  The cache's values enter
 * both products exactly; bf16: q, sums and softmax are as there; fp32: q and the softmax's weights enter as three bf16
 * numbers each, which together hold their 24 bits, and all sums are in fp32.
 */
size_t sd2_paged_attn_scaled_workspace_bytes(const sd2_paged_scaled* kv, const sd2_paged_rows* rows, int32_t n_heads,
                                       int32_t max_len, int32_t window, int32_t sinks);
sd2_status sd2_paged_attn_scaled(const sd2_paged_scaled* kv, const sd2_paged_rows* rows, const void* q, int64_t q_stride,
                           void* out, int64_t out_stride, int32_t n_heads, float scale, int32_t max_len,
                           int32_t window, int32_t sinks, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Destroy a handle (NULL is a no-op).  Does not free caller memory. */
sd2_status sd2_destroy(sd2_handle_t h);

/* Static text for a status code. */
const char* sd2_status_string(sd2_status s);

/* Text of the last HIP error observed by handle h (empty if none). */
const char* sd2_last_error(sd2_handle_t h);

/* What sd2_debug_read copies (all host-side, after synchronising the stream). */
#define SD2_DBG_LOGITS_V 1    /* float [batch][k+1][vocab]: last round's verifier logits */
#define SD2_DBG_LOGITS_D 2    /* float [batch][k][vocab]: last round's drafter logits (row j drew draft j) */
#define SD2_DBG_STEER 3       /* float [batch][d_drafter]: current steering vector s (SD2_STEER_INPUT) */
#define SD2_DBG_OWN_DRAFTS 4  /* int32 [batch][k]: drafts the library drew itself last round */
#define SD2_DBG_OWN_N 5       /* int32 [batch]: accepted count the library computed itself */
#define SD2_DBG_OWN_Y 6       /* int32 [batch]: final token the library drew itself */
#define SD2_DBG_STATE 7       /* int32 [batch][5]: t, len_verifier, len_drafter, produced, done (2: without pages
                                 in the last round) */
#define SD2_DBG_HIST 8        /* int32 [batch][max_seq_len]: committed tokens */
#define SD2_DBG_HIDDEN_V 9    /* float [batch][k+1][d_verifier]: last verify pass's final-norm hidden states */
#define SD2_DBG_PATH 10       /* int32 [2]: round execution path (0: one kernel per operation, 1: one persistent
                                 launch per drafter step and per verify pass), and 1 if one of those launches
                                 ever timed out at a grid barrier (its results are then invalid) */
#define SD2_DBG_TRACE 11      /* int64 [33][1024]: persistent path, last profiled round, device clock
                                 (100 MHz): entry 0 = start of launch j (0: verify pass, 1..k: drafter
                                 steps), entry p+1 = end of its phase p; SD2_ERR_STATE when that path
                                 is unavailable */

#define SD2_DBG_UBIAS 12      /* float [batch][L_D][d_ff_D]: current up-projection biases (SD2_STEER_MLP),
                                 float [batch][d_D]: the bias after every MLP (SD2_STEER_MLP_OUT);
                                 SD2_ERR_STATE for SD2_STEER_INPUT */
#define SD2_DBG_NONFINITE 13  /* int32 [1]: 1 if a verifier or drafter logit of a round since the last read of
                                 this selector was a NaN or an infinity (every logit the round's decisions use
                                 is checked as the sampler reads it), else 0; the read clears it */

#define SD2_DBG_REFS 14       /* int32 [n_pages]: table entries that name each page; SD2_ERR_STATE without pages */
#define SD2_DBG_TABLE 15      /* int32 [max_batch][ceil(max_seq_len / page_size)]: the page table (-1: none) */

/* Copy a debug buffer of the last round into host memory dst (bytes must match). */
sd2_status sd2_debug_read(sd2_handle_t h, int32_t what, void* dst_host, size_t bytes);

/* Kernel classes for sd2_profile_read. */
#define SD2_PROF_GEMV 1      /* weight-streaming projections and LM heads */
#define SD2_PROF_ATTN 2      /* attention over the KV cache */
#define SD2_PROF_SAMPLER 3   /* draft picks, accept test, final draw, commit */
#define SD2_PROF_OTHER 4     /* embedding/planning, RoPE and cache append */
#define SD2_PROF_PROGRAM 5   /* persistent launches (one per drafter step, one per verify pass) */

/*
 * Measurement hook.  enable != 0: following rounds are launched one kernel at a time (not from
 * the recorded graph) with a HIP event pair recorded on the handle's stream around every
 * launch; enable == 0 returns to graph replay.  Rounds stay functionally identical.
 */
sd2_status sd2_profile(sd2_handle_t h, int32_t enable);

/*
 * For the last profiled round (synchronises the stream): number of launches of class cls,
 * the sum of their event-to-event durations in milliseconds, and the sum of their algorithmic
 * bytes (SD2_PROF_GEMV: weights + input rows + output rows; SD2_PROF_PROGRAM: the weights the
 * launch streams, KV-cache reads not included; 0 for other classes).
 */
sd2_status sd2_profile_read(sd2_handle_t h, int32_t cls, int32_t* launches, double* total_ms, double* bytes);

#ifdef __cplusplus
}
#endif
#endif /* SD2_H */
