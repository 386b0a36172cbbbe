/*
 * asd.h - C ABI of libasd, the GB300 (sm_103a) verifier of Approximate
 * Speculative Decoding (ASD, arXiv 2608.03447).
 *
 * One verifier step takes the target model's teacher-forced logits for a batch
 * of draft blocks and, per request, returns the accepted prefix length, the
 * committed tokens, the recovery (or bonus) token and the updated regret
 * ledger (Sec. 3.2-3.3, Alg. 1).
 *
 * Conventions shared by every entry point
 *   - Every array argument is DEVICE memory owned by the caller, contiguous,
 *     row-major unless it comes with strides. The library allocates nothing and keeps no per-call state
 *     outside the caller's workspace (but for the word that asd_weigh_error reads).
 *   - Calls are asynchronous and ordered on `stream` (a cudaStream_t; NULL is
 *     the legacy default stream). Nothing synchronises with the host.
 *   - Indices are 0-based: request b in [0, B), draft position j in [0, K)
 *     (the paper's i = j + 1), target row j in [0, K] (row K is the bonus row).
 *   - A return value other than ASD_OK means that nothing was launched, except
 *     ASD_ERR_CUDA, which reports a failed launch.
 *   - Per-request data errors never abort the call: they set bits of
 *     status[b] (ASD_STATUS_*). Such a request accepts nothing (a = 0), emits
 *     y*_0 as its recovery token and keeps its ledger; for a NaN logit the
 *     argmax is deterministic but unspecified.
 *   - A workspace serves one call at a time: two calls that share a workspace
 *     must be ordered on one stream (or otherwise serialised).
 */
#ifndef ASD_H
#define ASD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

struct CUstream_st;
typedef struct CUstream_st* asd_stream_t; /* == cudaStream_t */

/* The persistent per-request ledger (B, s) of Sec. 3.2: the request's total
 * regret budget and the regret already spent in earlier rounds. budget = 0
 * selects exact strict greedy verification (Alg. 1); budget = +INFINITY is
 * allowed. Valid ledgers have 0 <= spent <= budget and no NaN. */
typedef struct {
  float budget;
  float spent;
} asd_ledger;

/* One vocabulary shard's reduction of one target row (asd_shard_partials):
 * what the tensor-parallel remark of Sec. 3.3 says the verifier needs from
 * each shard, with no logit buffer. */
typedef struct {
  uint64_t key;        /* order-preserving (top logit, GLOBAL vocabulary index): larger wins */
  float top;           /* the shard's top logit, exactly as stored (sign of zero kept) */
  float draft_logit;   /* z(x) if the row's draft token is in this shard, else -INFINITY */
  uint32_t flags;      /* ASD_STATUS_NAN_LOGIT if the shard saw a NaN in the row's request */
  uint32_t reserved;
} asd_partial;

/* Storage types. Logits are ASD_F32 or ASD_BF16; the cache entry points also take ASD_F16. */
enum { ASD_F32 = 0, ASD_BF16 = 1, ASD_F16 = 2 };

/* Flag ORed into the dtype argument of the verify entry points: the logits and
 * draft tokens are resident, i.e. no kernel that is still running or queued
 * ahead of this call on the stream writes them (they were written by work that
 * has completed, by a copy, or by the host). The row stage then starts
 * streaming them while the previous kernel on the stream finishes (programmatic
 * dependent launch), which overlaps consecutive calls. Without the flag the row
 * stage still launches early but reads nothing before the previous kernel has
 * completed and its writes are visible, so a producer kernel (such as the
 * model's LM head) may write the logits right before the call. Results are the
 * same either way; only the overlap differs. */
#define ASD_RESIDENT_INPUTS 0x100

/* Return codes. */
enum {
  ASD_OK = 0,
  ASD_ERR_NULL = 1,      /* a required pointer is NULL */
  ASD_ERR_SHAPE = 2,     /* B < 0, K < 0, K > 31, V < 1, or H invalid; cache entry points: a size, head
                          * count, stride or rotation out of its range */
  ASD_ERR_DTYPE = 3,     /* unknown dtype code */
  ASD_ERR_CONTROL = 4,   /* gate < 0 or NaN, cap < 0; eps < 0 or NaN, scale not finite or
                          * past 2e38 */
  ASD_ERR_WORKSPACE = 5, /* workspace smaller than the size query returns */
  ASD_ERR_ALIGN = 6,     /* pointer not aligned as documented */
  ASD_ERR_CUDA = 7,      /* a CUDA call failed (launch or device query) */
  ASD_ERR_DEVICE = 8,    /* the current device cannot run the kernel (not sm_103) */
  ASD_ERR_TIMEOUT = 9,   /* reported by asd_workspace_error and asd_weigh_error: a kernel gave up waiting */
  ASD_ERR_SCRATCH_LIMIT = 10 /* asd_verify_noalloc: the problem needs more than its scratch */
};

/* Per-request status bits (status[b]). */
#define ASD_STATUS_DRAFT_RANGE 1u /* a draft id outside [0, V) */
#define ASD_STATUS_NAN_LOGIT 2u   /* a NaN among the request's K+1 logit rows */
#define ASD_STATUS_BAD_LEDGER 4u  /* budget < 0 or NaN, spent < 0 or NaN, spent > budget */
#define ASD_STATUS_OVERFLOW 8u    /* asd_commit: the token history has no room for the block */
#define ASD_STATUS_INCOMPLETE 16u /* the workspace's error word was set when the request was
                                   * selected (asd_workspace_error): a kernel gave up waiting on
                                   * its copy pipeline, so row results may be missing. Set for
                                   * every request of such a call until asd_workspace_init.
                                   * asd_tree_attention: also by the call that gives up. */

#define ASD_STATUS_LENGTH 32u     /* cache entry points: kv_len < 0, a token count outside its range, or
                                   * more slots than the request's row of the page table covers */
#define ASD_STATUS_PAGE 64u       /* cache entry points: a page id outside [0, pages) */
#define ASD_STATUS_POSITION 128u  /* asd_kv_append: a position outside the rotation's table;
                                   * asd_kv_evict_numbered: numbers that are not a sequence's */
#define ASD_STATUS_PATH 256u      /* asd_kv_compact: path[i] < i or not ascending; asd_kv_weigh: path[i] outside
                                   * [0, T) */
#define ASD_STATUS_TOKEN 512u     /* asd_tokens_record, asd_tokens_bias: a token id >= V */
#define ASD_STATUS_EMPTY_ROW 1024u /* asd_rules_verify with ASD_FLAG_EMPTY_ROWS: no token may come where the recovery
                                   * token does. The accepted drafts and the ledger stand. */

/* Largest draft length: one warp lane per target row of a block. */
#define ASD_MAX_K 31

/* Bytes of workspace that asd_verify / asd_verify_strict need for (B, K, V,
 * dtype). Writes *bytes; returns ASD_ERR_SHAPE / ASD_ERR_DTYPE / ASD_ERR_NULL
 * on bad arguments. */
int asd_workspace_size(int B, int K, int V, int dtype, size_t* bytes);

/* Zero a workspace (cudaMemsetAsync on `stream`). Required once before the
 * first call that uses it; every verify call leaves the workspace zeroed again
 * when it completes, so it can be reused for any shape (and captured in a CUDA
 * graph) with no further initialisation. */
int asd_workspace_init(void* workspace, size_t bytes, asd_stream_t stream);

/* Read the workspace's sticky error word (synchronises `stream`): 0, or
 * ASD_ERR_TIMEOUT if a kernel that used this workspace gave up waiting on its
 * own copy pipeline (a bounded wait of about one second; it does not happen in
 * normal operation). After a non-zero word the outputs of that call are
 * incomplete and the workspace must be re-initialised with asd_workspace_init. */
int asd_workspace_error(const void* workspace, int* error, asd_stream_t stream);

/* Self-test of the failure detection above (the paper has no counterpart):
 * launches one CTA whose thread waits, with the same bounded mbarrier wait as
 * the pipeline kernels, on a barrier that nothing signals. After about one
 * second the wait gives up, the kernel writes ASD_ERR_TIMEOUT to the
 * workspace's error word and returns; nothing faults and the context stays
 * usable. `workspace` is any workspace of at least 4 bytes (16-byte aligned);
 * read the result with asd_workspace_error and re-initialise the workspace
 * before its next verify call. Returns ASD_ERR_NULL / ASD_ERR_WORKSPACE /
 * ASD_ERR_ALIGN on bad arguments, ASD_ERR_CUDA if the launch fails. */
int asd_selftest_wait_timeout(void* workspace, size_t workspace_bytes, asd_stream_t stream);

/*
 * ASD verification of B draft blocks (Eq. 1, 3, 5-13; Alg. 1).
 *
 * logits        [B, K+1, V], dtype ASD_F32 or ASD_BF16; row b*(K+1)+j holds
 *               z_{j+1}. Aligned to its element size; any further alignment
 *               is handled.
 * draft         [B, K] int32 draft tokens x (may be NULL when K = 0)
 * ledger        [B] in/out. spent is updated to s' = fl(s + C_a) (Eq. 13);
 *               left untouched when budget == 0 or the request is flagged.
 * gate          g of Eq. 7 (>= 0; +INFINITY disables the gate)
 * cap           M of Eq. 10 (>= 0; INT32_MAX disables the cap)
 * accepted_len  [B]       a = longest feasible prefix (Eq. 12)
 * committed     [B, K+1]  x_0..x_{a-1}, y*_a, then -1 padding
 * recovery      [B]       y*_a: the recovery token (a < K) or the bonus (a = K)
 * row_argmax    [B, K+1]  y*_j (lowest index on ties); may be NULL
 * row_regret    [B, K]    r_j = fl32(z_j(y*_j) - z_j(x_j)), NaN for an
 *                         out-of-range draft; may be NULL
 * status        [B]       ASD_STATUS_* bits; may be NULL
 * workspace     >= asd_workspace_size(...) bytes, 16-byte aligned, zeroed
 *               by asd_workspace_init before first use
 * dtype         ASD_F32 or ASD_BF16, optionally | ASD_RESIDENT_INPUTS (above)
 *
 * Arithmetic (all fp32, round to nearest): argmax by IEEE comparison
 * (-0 == +0), then per request, left to right over the mismatches d_j = 1:
 * C' = C + r_j; accept while r_j / (K - j) <= g, fl(s + C') <= budget and
 * N' <= M; a is the first position that fails (else K). budget == 0
 * dispatches to the strict rule (Eq. 2) and keeps the ledger.
 */
int asd_verify(const void* logits, int dtype, int B, int K, int V, const int32_t* draft,
               asd_ledger* ledger, float gate, int cap, int32_t* accepted_len,
               int32_t* committed, int32_t* recovery, int32_t* row_argmax, float* row_regret,
               int32_t* status, void* workspace, size_t workspace_bytes, asd_stream_t stream);

/*
 * Strict greedy verification (Eq. 2): a = the first j with x_j != y*_j (else
 * K); committed and recovery as in asd_verify (the bonus y*_K is appended when
 * a = K). No ledger. Same arguments, layouts and workspace as asd_verify.
 */
int asd_verify_strict(const void* logits, int dtype, int B, int K, int V, const int32_t* draft,
                      int32_t* accepted_len, int32_t* committed, int32_t* recovery,
                      int32_t* row_argmax, float* row_regret, int32_t* status, void* workspace,
                      size_t workspace_bytes, asd_stream_t stream);

/*
 * Fused LM-head + verify (Sec. 3.1 Eq. 1 with Sec. 3.3's remark that the
 * verifier needs only the top token, the top logit and the draft token's logit,
 * so no [T, V] logit buffer is needed). The logits z = h W^T are computed on
 * the tensor cores (bf16 inputs, fp32 accumulation) and reduced on chip; they
 * are never written to memory. The selection is then the one of asd_verify.
 *
 * hidden        [B*(K+1), H] bf16 (as uint16 bits or __nv_bfloat16): the
 *               target's final hidden state of every row of every block,
 *               16-byte aligned
 * weight        [V, H] bf16 LM-head weight, 16-byte aligned
 * H             hidden size, a multiple of 8 (rows must be 16-byte pitched)
 * row_top       [B, K+1] the top logit z_j(y*_j) of each row; may be NULL
 * everything else as in asd_verify; the workspace size comes from
 * asd_lmhead_workspace_size. Requires a Blackwell (sm_10x) device: other
 * devices get ASD_ERR_DEVICE.
 * Precision: the logits are fp32 sums of bf16 products in the tensor core's
 * order, so ties and near-ties (within about 1e-5 of the row's scale) may
 * resolve differently from an exact (fp64) evaluation; exact ties between
 * equal fp32 logits go to the lowest index, as in asd_verify.
 * Launch: clusters of two CTAs, one per SM of a pair, each with up to 227 KB
 * of shared memory and all 512 tensor-memory columns of its SM, so a call
 * occupies the GPU's SM pairs while it runs; the selection runs in a small
 * kernel right behind.
 */
int asd_lmhead_workspace_size(int B, int K, int V, int H, size_t* bytes);
int asd_lmhead_verify(const void* hidden, const void* weight, int H, int B, int K, int V,
                      const int32_t* draft, asd_ledger* ledger, float gate, int cap,
                      int32_t* accepted_len, int32_t* committed, int32_t* recovery,
                      int32_t* row_argmax, float* row_regret, float* row_top, int32_t* status,
                      void* workspace, size_t workspace_bytes, asd_stream_t stream);

/*
 * The same tensor-core LM-head GEMM writing its fp32 logits [T, V] (row-major,
 * device memory) instead of reducing them: for callers that need the logits
 * themselves, and to check the GEMM against an exact evaluation. No workspace.
 */
int asd_lmhead_logits(const void* hidden, const void* weight, int H, int T, int V, float* logits,
                      asd_stream_t stream);

/* Bytes of the fixed device scratch that asd_verify_noalloc uses. */
#define ASD_NOALLOC_SCRATCH_BYTES (1u << 20)

/*
 * asd_verify without a caller workspace and without allocating anything: for
 * callers that may not allocate device memory when they verify (a serving loop
 * with a fixed device-memory budget, a plug-in whose host framework owns every
 * device allocation, a latency-bound path where cudaMalloc / cudaFree could
 * synchronise the device). The paper has no counterpart; it is an interface
 * convenience around the same computation as asd_verify, with the same
 * arguments minus the workspace and the same results.
 *
 * Scratch: a fixed ASD_NOALLOC_SCRATCH_BYTES array of device memory inside the
 * library, held by every GPU that loads it until the process exits. A call
 * whose asd_workspace_size(B, K, V, dtype) exceeds it returns
 * ASD_ERR_SCRATCH_LIMIT and launches nothing.
 * Set-up: the first call made with a given device current looks up the
 * array's device address (cudaGetSymbolAddress); make that first call outside
 * any stream capture. The address is kept for the life of the process:
 * cudaDeviceReset unloads the library's device code, so after it this entry
 * point must not be called again in that process.
 * Each call clears the part of the array it uses (cudaMemsetAsync on
 * `stream`, which also clears the array's error word) and then launches the
 * verify kernels. Every call on every stream shares the one array: calls that
 * can overlap on the GPU (different streams, no ordering between them) race
 * and give wrong results. Order them on one stream. Allocates nothing: no
 * cudaMalloc, cudaFree or allocating library call.
 * Failure report: the array's error word is not readable by the caller, so a
 * call whose kernels gave up waiting on their copy pipeline (the bounded wait
 * of asd_workspace_error) flags every request ASD_STATUS_INCOMPLETE in
 * status[b] instead (a = 0, ledger kept); pass a status array to see it.
 */
int asd_verify_noalloc(const void* logits, int dtype, int B, int K, int V, const int32_t* draft,
                       asd_ledger* ledger, float gate, int cap, int32_t* accepted_len,
                       int32_t* committed, int32_t* recovery, int32_t* row_argmax,
                       float* row_regret, int32_t* status, asd_stream_t stream);

/*
 * Several sequential draft blocks of the same B requests in one call: block i
 * of request b is verified with the ledger left by block i-1 (Sec. 3.2: the
 * ledger (B, s) persists across decoding rounds). The result is bit for bit
 * that of nblk asd_verify calls made in order, block 0 first.
 *
 * logits        [nblk, B, K+1, V]; draft [nblk, B, K]; ledger [B] in/out
 * accepted_len, recovery, status  [nblk, B]; committed, row_argmax [nblk, B, K+1];
 * row_regret    [nblk, B, K]
 * workspace     asd_blocks_workspace_size(nblk, B, K, V, dtype) bytes
 * The logits of all blocks stream in one pass; only each request's selection
 * runs block after block, the ledger handed from one to the next.
 */
int asd_blocks_workspace_size(int nblk, int B, int K, int V, int dtype, size_t* bytes);
int asd_verify_blocks(const void* logits, int dtype, int nblk, int B, int K, int V,
                      const int32_t* draft, asd_ledger* ledger, float gate, int cap,
                      int32_t* accepted_len, int32_t* committed, int32_t* recovery,
                      int32_t* row_argmax, float* row_regret, int32_t* status, void* workspace,
                      size_t workspace_bytes, asd_stream_t stream);

/*
 * The verifier-side opportunity rate of Eq. 4 (Sec. 3.1), as counts added to
 * `counts` (device, uint64, accumulated over calls; zero it to start):
 *   counts[t * np + u] += #{ mismatch positions (x, i) with r_i <= tau[t],
 *                            i + p[u] <= K and x_l = y*_l for l = i+1 .. i+p[u] }
 *   counts[ntau * np]  += |M|, the number of mismatch positions
 * so Omega(tau[t], p[u]) = counts[t * np + u] / counts[ntau * np].
 * row_argmax [n, K+1], draft [n, K], row_regret [n, K]: asd_verify's row
 * outputs for n block-requests (device); status [n] or NULL (block-requests
 * with a non-zero status are skipped). tau [ntau] and p [np] are HOST arrays,
 * 1 <= ntau, np <= ASD_OPPORTUNITY_MAX; tau not NaN, p >= 0.
 */
#define ASD_OPPORTUNITY_MAX 16
int asd_opportunity(const int32_t* row_argmax, const int32_t* draft, const float* row_regret,
                    const int32_t* status, int n, int K, const float* tau, int ntau, const int32_t* p,
                    int np, unsigned long long* counts, asd_stream_t stream);

/*
 * Vocabulary-sharded verify (Sec. 3.3: under tensor parallelism the verifier
 * needs only the top token, the top logit and the draft token's logit, which
 * each vocabulary shard can reduce locally). Step 1 on every shard:
 *   asd_shard_partials: logits [B, K+1, Vs] hold the shard's vocabulary entries
 *   v_offset .. v_offset+Vs-1 of a V-entry vocabulary; draft [B, K] holds
 *   GLOBAL token ids; writes partials [B*(K+1)]. Workspace and its rules as for
 *   asd_verify, sized with asd_workspace_size(B, K, Vs, dtype).
 * Step 2, once the S shards' partials sit side by side (an all-gather across
 * ranks, or S slices of one GPU):
 *   asd_shard_combine: partials [S, B*(K+1)] -> the outputs of asd_verify for
 *   the whole vocabulary, bit for bit (same keys, same fp32 arithmetic). No
 *   workspace. The ledger, gate, cap and outputs are as in asd_verify.
 */
int asd_shard_partials(const void* logits, int dtype, int B, int K, int Vs, int v_offset, int V,
                       const int32_t* draft, asd_partial* partials, void* workspace,
                       size_t workspace_bytes, asd_stream_t stream);
int asd_shard_combine(const asd_partial* partials, int S, int B, int K, int V, const int32_t* draft,
                      asd_ledger* ledger, float gate, int cap, int32_t* accepted_len,
                      int32_t* committed, int32_t* recovery, int32_t* row_argmax, float* row_regret,
                      int32_t* status, asd_stream_t stream);

/* Step 1 of the same scheme with the LM head fused (the remark of Sec. 3.3 as
 * a tensor-parallel rank would run it: no logit buffer anywhere):
 * weight [Vs, H] bf16 holds rows v_offset .. v_offset+Vs-1 of the LM-head
 * weight of a V-entry vocabulary; hidden [B*(K+1), H] bf16 and draft [B, K]
 * (GLOBAL ids) as in asd_lmhead_verify; writes partials [B*(K+1)] for
 * asd_shard_combine. The top logit in a partial is the value the key holds
 * (a zero maximum is +0). Workspace from asd_lmhead_workspace_size(B, K, Vs,
 * H). Same precision and launch notes as asd_lmhead_verify. */
int asd_lmhead_partials(const void* hidden, const void* weight, int H, int B, int K, int Vs, int v_offset,
                        int V, const int32_t* draft, asd_partial* partials, void* workspace,
                        size_t workspace_bytes, asd_stream_t stream);

/*
 * Advance along the emitted sequence (Sec. 3.3: the target cache, the draft
 * cache and the ledger advance only along the emitted tokens; proposal-only
 * state past the returned prefix is discarded). For each request b with
 * a = accepted_len[b]:
 *   tokens [B, max_tokens], token_len [B] (in/out): the a + 1 emitted tokens
 *     committed[b][0..a] are appended at token_len[b]; token_len[b] += a + 1
 *   kv_len [B] (in/out): kv_len[b] += pending + a -- the cache keeps the
 *     pending input token of the pass (pending = 1 when the verification pass
 *     consumed the previous round's recovery token before the drafts, else 0)
 *     and the a accepted drafts; positions from the new length on held
 *     proposal-only state and may be overwritten (call once per cache)
 *   status [B] (out, may be NULL): ASD_STATUS_OVERFLOW when the history has
 *     no room; such a request changes nothing.
 * tokens / token_len may be NULL together, kv_len may be NULL. Device arrays.
 * accepted_len values are those asd_verify writes (0..K); others are clamped.
 */
int asd_commit(int B, int K, const int32_t* accepted_len, const int32_t* committed, int pending,
               int32_t* kv_len, int32_t* tokens, int32_t* token_len, int max_tokens, int32_t* status,
               asd_stream_t stream);

/* ------------------------------------------------------------------------
 * The cache side of a verified block. The target pass that precedes a verify
 * call feeds every request's pending token and drafts (a chain, or a tree in
 * which several drafts share a prefix) through the model; per layer their keys
 * and values enter a paged cache (asd_kv_append) and each of those tokens
 * attends to the request's context and to its own ancestors
 * (asd_tree_attention). Once a path of the tree has been verified, its keys and
 * values move next to the context (asd_kv_compact) and asd_commit advances
 * kv_len over them. The paper leaves these to the serving engine (Sec. 3.3,
 * cache semantics).
 *
 * A paged cache. Element (layer, page, i, head, d) of the keys lies at
 * k[layer * layer_stride + page * page_stride + i * token_stride +
 *   head * head_stride + d], the values likewise from v: any order of the
 * page's tokens and heads. Strides count elements; all are >= 0 and offsets are
 * formed in 64 bits. Slot s of request b (its token number s) is place
 * s % page_size of page page_table[b * table_width + s / page_size]. No two
 * requests may share a page that a call writes.
 */
typedef struct {
  void* k;
  void* v;
  int dtype;     /* ASD_F32, ASD_BF16 or ASD_F16 */
  int layers;    /* >= 1 */
  int pages;     /* >= 0 */
  int page_size; /* >= 1 tokens */
  int heads;     /* >= 1 key/value heads */
  int head_dim;  /* 1 .. ASD_MAX_HEAD_DIM */
  int64_t layer_stride, page_stride, token_stride, head_stride;
  const int32_t* page_table; /* [B, table_width] device memory */
  int B;                     /* requests */
  int table_width;           /* pages that a request's row has room for */
} asd_kv_cache;
#define ASD_MAX_HEAD_DIM 256
#define ASD_MAX_PATH 256 /* longest path that asd_kv_compact moves */

/*
 * Appends T tokens' keys and values to one layer of the cache, with an optional
 * norm per head and the position rotation on the way; the queries of the same
 * tokens take the same norm and rotation to q_out in the same pass.
 *
 * The tokens go to slots kv_len[b] + t (t < T) of request b. kv_len is not
 * changed (asd_commit advances it). A request flagged ASD_STATUS_LENGTH writes
 * nothing, a token whose position is out of range is left out, and one whose page
 * is out of range leaves its key and value out.
 *
 * Arithmetic: x is widened to fp32; with a norm x <- x / sqrt(mean(x^2) + eps)
 * * w; then (a, b) <- (a cos - b sin, b cos + a sin); one rounding at the end.
 * Values are copied bit for bit.
 */
/* B * T * (q_heads + 2 * heads) <= 2^30. */
typedef struct {
  int64_t batch, token, head; /* strides in elements of a [B, T, heads, head_dim] array of the cache's dtype: any, as
                               * in the rows of a fused projection; the last dimension is contiguous */
} asd_strides;
typedef struct {
  const void* k; /* [B, T, heads, head_dim] */
  const void* v;
  const void* q; /* [B, T, q_heads, head_dim], or NULL with q_heads = 0 */
  void* q_out;   /* [B, T, q_heads, head_dim] contiguous; may be q itself where q is contiguous */
  asd_strides k_strides, v_strides, q_strides;
  const int32_t* kv_len;    /* [B] tokens that each request has in the cache */
  const int32_t* new_len;   /* [B] how many of the T tokens exist (0..T), or NULL: all. Nothing is written for the
                             * others, q_out included */
  const int32_t* positions; /* [B, T] rotation positions (a tree's nodes take their depth), or NULL: kv_len[b] + t */
  const float* cos;         /* [rot_positions, rot_dim / 2], or both NULL: no rotation */
  const float* sin;
  const void* q_norm; /* [head_dim] weights of the cache's dtype, or NULL: no norm */
  const void* k_norm;
  int32_t* status;    /* [B] or NULL: ASD_STATUS_* bits are ORed in (zero it to start; one array can serve all
                       * layers of a pass) */
  int layer;
  int T;              /* tokens per request, >= 0 */
  int q_heads;        /* >= 0 */
  int rot_dim;        /* even, 2 .. head_dim: the leading elements that turn; 0 without tables */
  int rot_positions;  /* >= 0 */
  int interleaved;    /* 0: element i turns with i + rot_dim / 2; 1: 2i with 2i + 1 */
  float eps;          /* >= 0, of the norm */
  int reserved;       /* 0 */
} asd_append;
int asd_kv_append(const asd_kv_cache* cache, const asd_append* args, asd_stream_t stream);

/*
 * Attention of each request's T newest tokens over its paged cache: the tokens
 * of a draft chain or tree after asd_kv_append has put them there (T = 1: plain
 * decoding).
 *
 * Token t of request b sees every slot s < kv_len[b], and of the slots
 * kv_len[b] + u (u < new_len[b]) those with bit u % 32 of word u / 32 of its row
 * of tree_mask set (a node's row holds itself and its ancestors).
 *
 * Query head h reads key/value head h / group with group = q_heads / heads, a
 * whole number. B * heads * (T * group / 16 + 1) * (slots of the page table's row
 * / 64 + 1) < 2^31. A request flagged ASD_STATUS_LENGTH counts as one without
 * tokens, a slot on a page out of range as zeros.
 *
 * A row that sees nothing (new_len[b] <= t, or an empty context and an empty
 * mask row) is 0 with lse = -INFINITY. What a row does not see does not reach
 * it, NaN and infinities included.
 * Arithmetic: scores, softmax statistics and sums in fp32, one rounding at the
 * end. 16-bit types with head_dim <= 128 and a multiple of 8, rows on 16-byte
 * boundaries and scale > 0 run on the tensor cores, where the softmax weights
 * are rounded to the 16-bit type for the second product. The result does not
 * depend on the order in which CTAs finish.
 */
typedef struct {
  const void* q;             /* [B, T, q_heads, head_dim] of the cache's dtype */
  void* out;                 /* [B, T, q_heads, head_dim] contiguous */
  float* lse;                /* [B, T, q_heads] natural log of the sum of exp(score), or NULL */
  asd_strides q_strides;
  const int32_t* kv_len;     /* [B] the context, without the T new tokens */
  const int32_t* new_len;    /* [B] (0..T), or NULL: T */
  const uint32_t* tree_mask; /* [B, T, ceil(T / 32)], or NULL: a chain (u <= t) */
  int32_t* status;           /* as in asd_append */
  void* workspace;           /* 16-byte aligned, zeroed by asd_workspace_init before first use; one for a larger T or
                              * cache serves any smaller one. A call that gives up waiting on its own pipeline sets
                              * the error word (asd_workspace_error) and flags all its requests
                              * ASD_STATUS_INCOMPLETE; while the word is set calls write nothing and flag theirs */
  size_t workspace_bytes;    /* >= asd_attention_workspace_size */
  int layer;
  int T;
  int q_heads;
  float scale;               /* |scale| <= 2e38; scores are scale * (q . k) */
} asd_attention;
int asd_attention_workspace_size(const asd_kv_cache* cache, int T, int q_heads, size_t* bytes);
int asd_tree_attention(const asd_kv_cache* cache, const asd_attention* args, asd_stream_t stream);

/*
 * Moves the keys and values of a verified path next to the context, in place
 * and in every layer: slot kv_len[b] + path[b][i] goes to slot kv_len[b] + i for
 * i < path_len[b]. Call it before asd_commit advances kv_len.
 *
 * path          [B, P] int32 tree nodes, ascending, path[i] >= i (a topological
 *               numbering gives both); a node that stays where it is costs
 *               nothing. P <= ASD_MAX_PATH
 * path_len      [B] int32, 0..P
 * status        as above; a flagged request moves nothing
 */
int asd_kv_compact(const asd_kv_cache* cache, int P, const int32_t* kv_len, const int32_t* path,
                   const int32_t* path_len, int32_t* status, asd_stream_t stream);

/*
 * Which cached slots a request still needs: the attention weight that each slot of
 * each key/value head has received. asd_kv_weigh adds up what the rows of one pass
 * give (after asd_tree_attention, which leaves their lse; the rows of a verified
 * path after asd_kv_compact has moved it), asd_kv_evict keeps the heaviest slots.
 *
 * weight_out[b][h][s] = w + sum of exp(scale * (q . k_s) - lse) over the rows of
 * request b's heads h * group .. h * group + group - 1 that see slot s; w is decay *
 * weight[b][h][s] for s < kv_len[b] and 0 for the new slots (kv_len[b] .. kv_len[b] +
 * n - 1), whose weights begin here; with decay = 0 weight is not read. Slots from
 * kv_len[b] + n on are left as they were.
 *
 * Row i (i < n = new_len[b]) sees the slots below kv_len[b] and the new slots
 * kv_len[b] .. kv_len[b] + i: a chain. It is token i of q and lse, or with a path
 * token path[b][i] (a tree's accepted nodes, as asd_kv_compact takes them). A row
 * whose lse is infinite adds nothing (a token that saw nothing has -INFINITY).
 * Slots that a row does not see do not reach it, NaN included.
 *
 * A request without rows (new_len 0) and one flagged ASD_STATUS_LENGTH write
 * nothing; a row whose path entry is outside [0, T) (ASD_STATUS_PATH) adds nothing,
 * and a slot on a page out of range (ASD_STATUS_PAGE) counts as a key of zeros.
 * Arithmetic: scores, exponentials and sums in fp32, rows added in a fixed order.
 * 16-bit types with a head_dim that is a multiple of 8 and rows on 16-byte
 * boundaries run on the tensor cores; a call that gives up waiting on its own
 * pipeline flags all its requests ASD_STATUS_INCOMPLETE and is remembered until
 * asd_weigh_error reads it. No workspace. Values of the cache are not read. The limits on sizes are
 * those of asd_tree_attention, with `rows` for T.
 */
typedef struct {
  const void* q;           /* [B, T, q_heads, head_dim] of the cache's dtype */
  const float* lse;        /* [B, T, q_heads] as asd_tree_attention writes it */
  asd_strides q_strides;
  const float* weight;     /* [B, heads, width]; may be NULL with decay = 0 */
  float* weight_out;       /* [B, heads, width]; may be weight itself */
  const int32_t* kv_len;   /* [B] slots that all rows see */
  const int32_t* new_len;  /* [B] (0..rows), or NULL: rows */
  const int32_t* path;     /* [B, rows] or NULL: row i is token i, and rows = T */
  int32_t* status;         /* as in asd_append */
  double scale;            /* |scale| <= 2e38; a rounding of it would be in every weight */
  float decay;             /* finite, >= 0 */
  int layer;
  int T;                   /* tokens of q and lse */
  int rows;                /* rows of a request, >= 0 */
  int q_heads;
  int width;               /* slots that a head's weights have room for, >= kv_len + new_len of every request */
} asd_weigh;
int asd_kv_weigh(const asd_kv_cache* cache, const asd_weigh* args, asd_stream_t stream);

/* Whether an asd_kv_weigh on the current device has given up a wait (about one second; it does
 * not happen in normal operation) since the last call of this function: 0 or ASD_ERR_TIMEOUT.
 * Weights that such a call was to write may be missing. Synchronises `stream`, whose calls it
 * tells of, and clears what it has read. */
int asd_weigh_error(int* error, asd_stream_t stream);

/*
 * Cuts every request's cache to its budget, in place and in every layer. Of
 * request b's kv_len[b] slots n = min(keep[b], kv_len[b]) stay in each layer and
 * head: the first f = min(first, n), the last r = min(last, n - f), and the n - f -
 * r heaviest of those between (a NaN weighs as much as -INFINITY; of equal weights
 * the lower slot stays). Different heads keep different slots.
 *
 * A slot that stays and lies below n is not moved; the others that stay go, in
 * ascending order, to the places below n that became free, in ascending order,
 * their weights with them. Attention does not depend on the order of the slots
 * (keys are rotated by their positions when they are appended), so nothing else
 * moves. The last slots are the newest tokens as long as tokens lie in their order: at
 * the first eviction, and at a later one if at least `last` tokens have been appended
 * since the one before. With fewer in between `last` holds on to slots that are no longer
 * the newest ones; asd_kv_evict_numbered knows the tokens. Later tokens take positions of their
 * own (asd_append.positions): kv_len is no longer a token's number. A request's pages
 * are its own: of a page that two requests' tables share, both move slots.
 *
 * weight        [layers, B, heads, width]; weight_out the same or weight itself. Slots
 *               of weight_out from n on are left as they were.
 * kv_len_out    [B] = n; neither kv_len nor keep itself (every head reads them while the
 *               call runs)
 * keep          [B] >= 0
 * status        ASD_STATUS_LENGTH (kv_len < 0 or past the table or the width, keep <
 *               0): such a request moves nothing and keeps its length.
 *               ASD_STATUS_PAGE: a move from or to a page out of range is left out,
 *               its weight is not.
 * width         <= ASD_MAX_EVICT_SLOTS
 */
typedef struct {
  const float* weight;
  float* weight_out;
  const int32_t* kv_len;
  int32_t* kv_len_out;
  const int32_t* keep;
  int32_t* status;
  int first, last; /* >= 0 */
  int width;
  int reserved;    /* 0 */
} asd_evict;
#define ASD_MAX_EVICT_SLOTS 360448
int asd_kv_evict(const asd_kv_cache* cache, const asd_evict* args, asd_stream_t stream);

/*
 * The same, and the newest tokens stay however many have been appended since the last
 * eviction: of request b's tokens 0 .. tokens[b] - 1, in the order in which they were
 * appended, the last r = min(last, n - f), wherever their slots are, instead of the last r
 * slots. A head keeps fewer of them where an eviction with a smaller `last` or `keep` has
 * left some out, and more of the heaviest.
 *
 * number        [layers, B, heads, width] the token of each slot; negative: the slot has
 *               been appended since the last eviction (or there was none), and holds token
 *               tokens[b] - kv_len[b] + s. Filled with -1 before a request's first eviction,
 *               and only evictions write it: a request that loses slots has the numbers of the
 *               slots below n, moved with them, and -1 in those from n to kv_len[b] - 1.
 * tokens        [B] >= kv_len: how many tokens have been appended to the request's cache
 *               and not taken back, evicted ones included; not kv_len_out. Tokens can be taken
 *               back (kv_len and tokens made smaller) that no eviction has seen yet.
 * status        ASD_STATUS_LENGTH: also tokens < kv_len. ASD_STATUS_POSITION: a head whose
 *               numbers are not of one such sequence (more newest tokens than places): it
 *               moves nothing, its slots below n stay.
 */
int asd_kv_evict_numbered(const asd_kv_cache* cache, const asd_evict* args, int32_t* number, const int32_t* tokens,
                          asd_stream_t stream);

/* ------------------------------------------------------------------------
 * Rules: what a request's own text, its caller and its grammar do to the logits
 * of a draft block before they are compared. The paper verifies raw logits; a
 * serving engine changes them first, and since row j of a block continues the
 * drafts x_0 .. x_{j-1}, every row is changed differently.
 *
 * Token v of row j, all in fp32, each operation rounded:
 *   c = times said (record) + #{ i < j : x_i = v }
 *   if c > 0 or v is in the prompt:  z <- z > 0 ? z / repetition : z * repetition
 *   if c > 0:                        z <- z - c * frequency, then z <- z - presence
 *   if v has a record:               z <- z + bias
 *   if the grammar does not allow v: z <- -INFINITY, whatever it was
 *
 * A record says what is known of a token; a set bit of `marks` (bit v % 32 of word
 * v / 32) that token v has one. Records without a mark are not read, so marks and
 * records of zeros are a request without text. asd_tokens_record and
 * asd_tokens_bias write both.
 */
typedef struct {
  uint32_t seen; /* ASD_TOKEN_PROMPT if the token is in the prompt | how often it has been said (below 2^31) */
  float bias;
} asd_token_record;
#define ASD_TOKEN_PROMPT 0x80000000u
typedef struct {
  uint32_t* marks;           /* [B, ceil(V / 32)] */
  asd_token_record* records; /* [B, V], 8-byte aligned */
  const float* repetition;   /* [B], > 0, or NULL: 1 */
  const float* frequency;    /* [B] or NULL: 0 */
  const float* presence;     /* [B] or NULL: 0 */
  const uint32_t* allow;     /* ceil(V / 32) words a row as in marks, or NULL: every token may come */
  int64_t allow_batch;       /* words from a request's rows to the next one's, and from a row to the next (>= 0; 0: */
  int64_t allow_row;         /* one for all) */
  int B, V;
} asd_token_rules;

/*
 * asd_verify of the logits under the rules, which are applied as the rows are read:
 * no changed logits are written. Arguments, outputs, workspace and status as
 * for asd_verify (or, with ledger = NULL, asd_verify_strict); a NaN counts where the
 * grammar allows its token. Regrets are differences of changed logits, which stay
 * fp32: a draft that is not allowed has an infinite one, NaN where no token is
 * allowed (then y* = 0). ASD_RESIDENT_INPUTS is not taken.
 *
 * A draft whose changed logit is -INFINITY (not allowed by the grammar, or banned by its
 * bias) is never accepted, whatever gate, budget and cap are, not even where it equals
 * y* = 0 because no token is allowed. The recovery token of a row without any is y* = 0
 * all the same; with ASD_FLAG_EMPTY_ROWS in dtype such a request's status tells.
 */
#define ASD_FLAG_EMPTY_ROWS 0x200
typedef struct {
  const void* logits;     /* [B, K+1, V] */
  const int32_t* draft;   /* [B, K] */
  asd_ledger* ledger;     /* [B], or NULL: strict */
  int32_t* accepted_len;
  int32_t* committed;
  int32_t* recovery;
  int32_t* row_argmax;    /* may be NULL, as row_regret and status may */
  float* row_regret;
  int32_t* status;
  void* workspace;
  size_t workspace_bytes; /* >= asd_workspace_size(B, K, V, dtype) */
  int dtype;              /* ASD_F32 or ASD_BF16, ASD_FLAG_EMPTY_ROWS ORed in if wanted */
  int K;
  float gate;
  int cap;
} asd_rules_block;
int asd_rules_verify(const asd_token_rules* rules, const asd_rules_block* block, asd_stream_t stream);

/*
 * The changed logits themselves, for callers that sample: logits and out [B, rows,
 * V] (1 <= rows <= ASD_MAX_K + 1; out may be logits itself) of dtype ASD_F32 or
 * ASD_BF16, rounded once. draft [B, rows - 1], or NULL: no row has drafts before it.
 * Draft ids outside [0, V) count for nothing. Logits that no rule names are copied
 * bit for bit. No workspace.
 */
int asd_rules_logits(const asd_token_rules* rules, const void* logits, int dtype, int rows, const int32_t* draft,
                     void* out, asd_stream_t stream);

/*
 * Adds tokens to the records: tokens [B, n] int32, of which request b has the first
 * token_len[b] (0..n; NULL: n). Negative ids are skipped, so asd_verify's `committed`
 * can be passed as it is. prompt = 0: each is said once more; 1: each is in the prompt.
 * status [B] or NULL: ASD_STATUS_TOKEN (an id >= V, skipped) and ASD_STATUS_LENGTH
 * (a token_len out of range: nothing of the request is recorded) are ORed in.
 */
int asd_tokens_record(const asd_token_rules* rules, const int32_t* tokens, int n, const int32_t* token_len, int prompt,
                      int32_t* status, asd_stream_t stream);

/* Sets the bias of tokens: ids and bias [B, n] (n <= ASD_MAX_BIAS), lengths, negative
 * ids and status as above; where an id comes twice the later one counts. A bias of 0
 * is one like any other; -INFINITY bans a token. */
#define ASD_MAX_BIAS 1024
int asd_tokens_bias(const asd_token_rules* rules, const int32_t* ids, const float* bias, int n, const int32_t* length,
                    int32_t* status, asd_stream_t stream);

/* The device address through which kernels read page-locked (pinned) host
 * memory, e.g. logits that stay in host memory and stream to the GPU over the
 * host link while asd_verify runs, with no separate copy. `host` should lie in
 * a pinned, mapped allocation (cudaHostAlloc / cudaHostRegister; runtime
 * contexts map pinned memory by default). On systems whose GPU reads pageable
 * memory through the host's page tables the runtime also accepts pageable
 * memory (slower to read); where neither applies the call returns
 * ASD_ERR_ALIGN. The alias is valid as long as the allocation is.
 * Synchronous, no allocation. */
int asd_host_alias(const void* host, void** device);

/* How many kernels one asd_verify / asd_verify_strict call launches for this
 * shape (1 or 2: the row stage, and unless the row stage selects as well a
 * selection kernel launched right behind it); 0 for B = 0. For accounting only. */
int asd_verify_launches(int B, int K, int V, int dtype, int* launches);

/* Launch options of the logit-streaming entry points (asd_verify,
 * asd_verify_strict, asd_verify_blocks, asd_shard_partials, asd_verify_noalloc).
 * The paper has no counterpart: these choose among kernels that compute the
 * same results bit for bit, for tests that cover each kernel and for
 * measurements; the defaults (all fields 0) are what production calls want.
 *   path          ASD_PATH_AUTO picks the row-stage kernel by size (one CTA or
 *                 one cluster of CTAs per request, selection included, for few
 *                 requests that fit it; the TMA pipeline for
 *                 ASD_RESIDENT_INPUTS in long rows (few, or more than 21 MB)
 *                 and, with fused_select, for more than 80 MB in long rows;
 *                 the register-streaming kernel for everything else); the
 *                 others force one (a forced ASD_PATH_SMALL falls back to AUTO
 *                 where the shape does not fit it).
 *   fused_select  1: the row stage runs the selection itself (the CTA that
 *                 completes a request selects it) instead of launching
 *                 select_kernel right behind it.
 *   no_pdl        1: launch without programmatic dependent launch.
 * Process-wide; each call reads the options once when it is issued, and a CUDA
 * graph keeps the kernels chosen at capture. asd_set_launch_options(NULL)
 * restores the defaults. Returns ASD_ERR_CONTROL for an unknown path. */
enum { ASD_PATH_AUTO = 0, ASD_PATH_SMALL = 1, ASD_PATH_STREAM = 2, ASD_PATH_TMA = 3 };
typedef struct {
  int path;
  int fused_select;
  int no_pdl;
} asd_launch_options;
int asd_set_launch_options(const asd_launch_options* options);
int asd_get_launch_options(asd_launch_options* options);

/* Human-readable text of a return code. Never NULL. */
const char* asd_status_string(int code);

#ifdef __cplusplus
}
#endif

#endif /* ASD_H */
