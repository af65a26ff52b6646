/*
 * startrail.h -- C ABI of the one-GPU ring-attention share (StarTrail hot path) for gfx950.
 *
 * The library computes what ONE GPU of a (concentric) ring computes for one
 * attention layer in training: blockwise attention of a resident query shard
 * against the KV chunks the ring delivers step by step, folded into a running
 * (O, lse) state, and the matching backward accumulation of dQ, dK, dV.
 * The ring itself is simulated by visiting chunks that are already resident
 * in device memory; nothing here communicates.
 *
 * General rules for every entry point
 *   - All tensor pointers are DEVICE pointers unless a parameter says "host".
 *     Descriptor structs and the small integer tables are HOST memory and are
 *     read before the call returns.
 *   - The library allocates nothing and owns nothing: every buffer, including
 *     workspaces, is the caller's.  Calls enqueue work on the given HIP stream
 *     (a hipStream_t passed as void*, NULL = the default stream) and return
 *     without synchronising.
 *   - Errors are returned as st_status; nothing aborts or throws.  Arguments
 *     are validated on the host before any launch; on error nothing is enqueued.
 *     st_last_error() gives a text for the calling thread's last failure.
 *   - Tensors Q, K, V, dO are 4-D [B, S, heads, D] views described by element
 *     strides with the D dimension contiguous (st_tensor).  Base pointers and
 *     strides must keep every row 16-byte aligned (ST_ERR_ALIGNMENT otherwise).
 *   - Partial / running outputs are dense fp32: O-like [B, Sq, Hq, D],
 *     lse-like [B, Hq, Sq]; chunk gradients [B, Sk, Hkv, D].
 *   - Query head h reads KV head h / (Hq / Hkv).  Causal masking is by GLOBAL
 *     token position: key t of a chunk is visible to query i iff
 *     k_offset + t <= q_offset + i.  lse is the natural-log log-sum-exp of
 *     scale * <q, k> over visible keys; a row with no visible key has O = 0
 *     and lse = -inf.
 *   - Supported: ST_F32 with D <= 256 and D % 8 == 0 (fp32 MFMA kernels), ST_BF16
 *     with D == 128 or D == 64 (bf16 MFMA kernels, fp32 accumulation).  Anything
 *     else returns ST_ERR_UNSUPPORTED.
 *   - Precision of the ST_BF16 path: P and dS are rounded to bf16 before the
 *     second contractions, and every kernel, forward and backward, evaluates
 *     the scores from the same operand Q' = bf16(Q * scale * log2 e), so that
 *     the matrix units deliver exponents directly.  That is attention of a
 *     query perturbed by at most 2^-9 relative per element: the scores move by
 *     about 1e-3 of their spread (standard deviation over a row), lse likewise,
 *     and backward and forward stay consistent with each other (recomputed
 *     probabilities sum to one over a row).
 */
#ifndef STARTRAIL_H
#define STARTRAIL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  ST_OK = 0,
  ST_ERR_INVALID_ARG = 1,   /* null pointer, negative size, Hq % Hkv != 0, bad layout (P, C, rank) ... */
  ST_ERR_UNSUPPORTED = 2,   /* dtype / head_dim / size combination that has no kernel */
  ST_ERR_ALIGNMENT = 3,     /* pointer or stride breaks the 16-byte row alignment */
  ST_ERR_HIP = 4,           /* a HIP call or launch failed; see st_last_error() */
  ST_ERR_WORKSPACE = 5      /* workspace missing or smaller than st_ring_workspace_bytes() */
} st_status;

typedef enum { ST_F32 = 0, ST_BF16 = 1, ST_E4M3 = 2 /* of a cache's pages only */ } st_dtype;

/* How the driver walks the visit order. */
typedef enum {
  ST_RING_STEPWISE = 0,     /* one st_attn_block_fwd/bwd + st_attn_merge per visited chunk */
  ST_RING_FUSED = 1         /* one launch per pass; the running state stays in registers */
} st_ring_mode;

#define ST_MAX_CHUNKS 256   /* most chunks one st_ring_* call accepts */

/* 4-D view [B, S, heads, D]; strides in ELEMENTS; D contiguous (stride 1). */
typedef struct {
  void*   ptr;              /* device */
  int64_t stride_b, stride_s, stride_h;
} st_tensor;

/* One (Q shard, KV chunk) pair: the operands of one ring iteration
 * (Algorithm 1, the forward_iteration step). */
typedef struct {
  int32_t dtype;            /* st_dtype of Q, K, V, dO */
  int32_t B, Hq, Hkv, D;
  int32_t Sq, Sk;           /* tokens in the Q shard / in this chunk; Sk may be 0 */
  int64_t q_offset;         /* global position of Q row 0 */
  int64_t k_offset;         /* global position of chunk row 0 */
  int32_t causal;           /* 0: every key visible; 1: visible iff k_offset+t <= position of query row i */
  float   scale;            /* softmax scale, finite and > 0, normally 1/sqrt(D) (Section 2.1 attention equation) */
  int32_t q_seg;            /* 0: the Q rows are one run from q_offset.  > 0: rows [q_seg, Sq) are a second run */
  int64_t q_offset2;        /*    whose row q_seg sits at q_offset2 >= q_offset + q_seg (appendix "Sequence
                             *    Parallelism Dataloader": a rank holds an early and a late piece of the sequence so
                             *    that causal work is equal across ranks); 0 < q_seg < Sq */
} st_block_desc;

/* One GPU's whole share: the Q shard plus the table of chunks the ring delivers
 * (Section 3.2: after the team all-gather each delivered buffer is a run of
 * sequence shards; here every shard is one chunk with its own base pointer). */
typedef struct {
  int32_t dtype;
  int32_t B, Hq, Hkv, D;
  int32_t Sq, Sk;           /* every chunk has Sk tokens */
  int64_t q_offset;
  int32_t causal;
  float   scale;
  int32_t n_chunks;         /* 1 .. ST_MAX_CHUNKS */
  const void* const* k_ptr; /* host array [n_chunks] of device base pointers, chunk j = [B,Sk,Hkv,D] */
  const void* const* v_ptr; /* host array [n_chunks] */
  int64_t k_stride_b, k_stride_s, k_stride_h;   /* shared by all K chunks */
  int64_t v_stride_b, v_stride_s, v_stride_h;   /* shared by all V chunks */
  const int64_t* k_offset;  /* host array [n_chunks]: global position of row 0 of chunk j */
  int32_t q_seg;            /* second run of query rows, as in st_block_desc (0: none) */
  int64_t q_offset2;
} st_ring_desc;

/* ---- ring iteration, forward (Algorithm 1: forward_iteration before its fold) ----
 * Attention of the Q shard against ONE chunk.
 *   o_part   fp32 [B,Sq,Hq,D]  (overwritten)   partial output, already divided by its own row sum
 *   lse_part fp32 [B,Hq,Sq]    (overwritten)
 * A fully masked chunk (or Sk == 0) is legal and writes O = 0, lse = -inf. */
st_status st_attn_block_fwd(const st_block_desc* desc, const st_tensor* q, const st_tensor* k,
                            const st_tensor* v, float* o_part, float* lse_part, void* hip_stream);

/* ---- online-softmax fold / the arithmetic of ReduceScatter_combine (Algorithm 1;
 * Section 3.2 "Forward Propagation": lse and O are updated step by step) ----
 * In place: (o_acc, lse_acc) <- merge((o_acc, lse_acc), (o_part, lse_part)) with
 *   lse' = log(exp(lse_acc) + exp(lse_part)),
 *   O'   = exp(lse_acc - lse') O_acc + exp(lse_part - lse') O_part.
 * A state with lse = -inf is empty (the neutral element; start from O = 0, lse = -inf).
 * One whose lse is NaN makes the row NaN.
 * o_out_lowp (nullable): also write O' rounded to out_dtype, dense [B,Sq,Hq,D].
 * o_acc/o_part fp32 [B,Sq,Hq,D]; lse_acc/lse_part fp32 [B,Hq,Sq].  o_part may not alias o_acc. */
st_status st_attn_merge(float* o_acc, float* lse_acc, const float* o_part, const float* lse_part,
                        int32_t B, int32_t Sq, int32_t Hq, int32_t D, int32_t out_dtype,
                        void* o_out_lowp, void* hip_stream);

/* ---- ReduceScatter_combine on one GPU (Algorithm 1, last step; Section 3.2 "Forward Propagation": the team
 * members' intermediate results are amalgamated and each member keeps its own portion of the rows) ----
 * n_states partial states of the SAME Sq_in query rows, each over a different part of the keys, are
 * combined in one pass, and only rows [row0, row0 + Sq_out) are kept:
 *   lse' = log(sum_x exp(lse_x)),   O' = sum_x exp(lse_x - lse') O_x.
 *   o_parts, lse_parts  host arrays [n_states] of device pointers: fp32 [B,Sq_in,Hq,D] / fp32 [B,Hq,Sq_in]
 *   o_out fp32 [B,Sq_out,Hq,D], lse_out fp32 [B,Hq,Sq_out] (overwritten; may not alias an input)
 *   o_out_lowp (nullable): O' rounded to out_dtype, dense [B,Sq_out,Hq,D]
 * A state with lse = -inf on a row is empty there; a row empty in every state gives O = 0, lse = -inf, and one whose lse is NaN
 * in some state gives NaN.
 * Requires 1 <= n_states <= 64, D <= 256, D % 8 == 0, 0 <= row0, row0 + Sq_out <= Sq_in. */
st_status st_attn_combine(const float* const* o_parts, const float* const* lse_parts, int32_t n_states,
                          int32_t B, int32_t Sq_in, int32_t Hq, int32_t D, int32_t row0, int32_t Sq_out,
                          float* o_out, float* lse_out, int32_t out_dtype, void* o_out_lowp, void* hip_stream);

/* ---- backward preparation (Section 3.2 "Backward Propagation": each iteration mirrors the
 * FlashAttention backward, which needs Delta_i = <dO_i, O_i> of the FINAL merged O) ----
 *   d_o      [B,Sq,Hq,D] in desc->dtype;  o: the final O, in o_dtype (ST_F32 or desc->dtype)
 *   delta    fp32 [B,Hq,Sq] (overwritten).   Only B, Sq, Hq, D, dtype of desc are used. */
st_status st_attn_delta(const st_block_desc* desc, const st_tensor* d_o, const st_tensor* o,
                        int32_t o_dtype, float* delta, void* hip_stream);

/* ---- ring iteration, backward (Section 3.2 "Backward Propagation") ----
 * The Q shard (with its FINAL lse and Delta) meets ONE chunk:
 *   P = exp(scale q k^T - lse),  dV += P^T dO,  dS = P o (dO v^T - Delta),
 *   dQ += scale dS k,  dK += scale dS^T q   (dK, dV summed over the query heads of a KV group).
 *   dq_acc fp32 [B,Sq,Hq,D]   ACCUMULATED (+=): the circulating query gradient
 *   dk_acc, dv_acc fp32 [B,Sk,Hkv,D] ACCUMULATED (+=): stay with the chunk
 * The caller zeroes the accumulators once.  Every accumulator element is owned by one workgroup per
 * launch (read, add, write; no atomic adds), so results are bit-reproducible; calls that add into the same
 * accumulator must be ordered on one stream. */
st_status st_attn_block_bwd(const st_block_desc* desc, const st_tensor* q, const st_tensor* k,
                            const st_tensor* v, const st_tensor* d_o, const float* lse_final,
                            const float* delta, float* dq_acc, float* dk_acc, float* dv_acc,
                            void* workspace, size_t workspace_bytes, void* hip_stream);
/* workspace (nullable): device, 256-byte aligned, best st_attn_block_bwd_workspace_bytes(desc) bytes (0 for
 * ST_F32).  With it the ST_BF16 path keeps a scaled copy of Q there, which is what its hand-scheduled dK/dV kernel
 * reads (B Sq Hq D 2 bytes, rounded up to 256: the least that is accepted), and behind it the partial sums of a
 * launch with few key tiles; with less room it runs on fewer workgroups.  Without a workspace the same values are
 * computed by the general kernel, at a lower rate.  Contents mean nothing between calls; calls that share a
 * workspace must be ordered on one stream. */
size_t st_attn_block_bwd_workspace_bytes(const st_block_desc* desc);

/* ---- fp32 -> storage dtype (round to nearest even), n contiguous elements ---- */
st_status st_cast_from_f32(const float* src, void* dst, int64_t n, int32_t dst_dtype, void* hip_stream);

/* ---- chunk-visit order of the concentric layout (appendix algorithms get_init_send and
 * get_P2P_config; Section 3.2: teams of C, team groups of P/C^2 teams, sub-rings) ----
 * For the Q shard of global rank `rank` (team rank/C): one GPU plays the C members of the team
 * in turn; member a' walks its P/C^2 sub-ring iterations, each delivering the gathered KV of one
 * team = C consecutive sequence shards.
 *   shard_idx host [P] (out): sequence-shard index met at each of the P visits
 *   member_of host [P] (out): team member (0..C-1) whose running state the visit folds into
 * Requires C >= 1, C*C | P, 0 <= rank < P (else ST_ERR_INVALID_ARG).  C = 1 is the plain ring. */
st_status st_visit_order(int32_t P, int32_t C, int32_t rank, int32_t* shard_idx, int32_t* member_of);

/* ---- the literal per-GPU schedule of the concentric layout (Section 3.2: after the team all-gather every
 * member holds the team's Q, K, V of C N/P tokens; member a of team t then walks its sub-ring of P/C^2
 * GPUs and meets one gathered team buffer per iteration) ----
 * For global rank `rank` = t*C + a:
 *   team_buffer host [P/C^2] (out): index tau of the team whose gathered KV (sequence shards
 *                                   tau*C .. tau*C+C-1) is met at iteration i = 0 .. P/C^2-1
 * The rank's partial state covers the C N/P query rows of its team against those buffers; the C members'
 * partial states combined (st_attn_combine) give the team's attention output.
 * Requires C >= 1, C*C | P, 0 <= rank < P (else ST_ERR_INVALID_ARG). */
st_status st_team_visit_order(int32_t P, int32_t C, int32_t rank, int32_t* team_buffer);

/* ---- communication the schedule implies (Section 3.2 "Theoretical Analysis": the three communication
 * expressions, ring attention's P2P, the concentric layout's collectives and its P2P) ----
 * For one attention block forward on one GPU: P GPUs, team size C, batch B, sequence N, hidden size H,
 * bytes_per_element of the exchanged tensors (2 for bf16), link bandwidth W in bytes per second and
 * per-message latency L in seconds.  Byte counts are exact integers, times are fp64:
 *   ring_iterations            P - 1                      startrail_iterations            P / C^2 - 1
 *   ring_p2p_bytes_per_iter    2 B N H e / P              startrail_p2p_bytes_per_iter    2 C B N H e / P
 *   ring_p2p_bytes             product of the two         startrail_p2p_bytes             product of the two
 *   startrail_collective_bytes 4 B N H e (C - 1) / P      (team all-gather of Q, K, V + reduce-scatter of O)
 *   ring_p2p_seconds           iterations * (bytes_per_iter / W + L)        likewise startrail_p2p_seconds
 *   startrail_collective_seconds   collective_bytes / W   (the paper's expression has no latency term)
 * Requires C >= 1, C*C | P, P | N, positive sizes, W > 0, L >= 0 (else ST_ERR_INVALID_ARG).  Host-only,
 * `out` is host memory. */
typedef struct {
  int32_t ring_iterations;
  int32_t startrail_iterations;
  int64_t ring_p2p_bytes_per_iter;
  int64_t startrail_p2p_bytes_per_iter;
  int64_t ring_p2p_bytes;
  int64_t startrail_p2p_bytes;
  int64_t startrail_collective_bytes;
  double ring_p2p_seconds;
  double startrail_p2p_seconds;
  double startrail_collective_seconds;
} st_comm_report;
st_status st_schedule_report(int32_t P, int32_t C, int64_t B, int64_t N, int64_t H, int32_t bytes_per_element,
                             double W, double L, st_comm_report* out);

/* ---- driver: the whole share (Algorithm 1 loop + combine; backward loops of Section 3.2) ----
 * order host [n_visit]: chunk indices into the desc tables, in visit order (each at most once).
 * member_of host [n_visit] (nullable = all 0): running state each visit folds into; the member
 *   states are merged at the end (the combine step).  Chunks lying entirely in the causal future
 *   of the shard are skipped.
 * Forward outputs: o_acc fp32 [B,Sq,Hq,D], lse fp32 [B,Hq,Sq] (overwritten); o_lowp nullable,
 *   [B,Sq,Hq,D] in desc->dtype.
 * workspace: device, >= st_ring_workspace_bytes(desc, mode, backward) bytes, 256-byte aligned.  Its contents
 *   are the library's (partial states, Delta, the tile counters of the dK/dV launch, the scaled copy of Q, partial
 *   sums of backward launches that would leave part of the chip idle) and mean nothing between calls; calls that share a
 *   workspace must be ordered on one stream.  Sizes depend on the whole descriptor, under a causal mask on the positions
 *   too.  What is there beyond that size changes nothing; with less room a backward runs on fewer workgroups, down to the
 *   room its Delta, counters and copy of Q need. */
size_t st_ring_workspace_bytes(const st_ring_desc* desc, int32_t mode, int32_t backward);

st_status st_ring_fwd(const st_ring_desc* desc, const st_tensor* q, const int32_t* order,
                      const int32_t* member_of, int32_t n_visit, int32_t mode,
                      float* o_acc, float* lse, void* o_lowp,
                      void* workspace, size_t workspace_bytes, void* hip_stream);

/* Backward outputs (all ACCUMULATED, caller zeroes once): dq_acc fp32 [B,Sq,Hq,D];
 * dk_acc, dv_acc host arrays [n_chunks] of device fp32 [B,Sk,Hkv,D] buffers (entries of chunks
 * that are not visited may be NULL).  o: final O in o_dtype; lse_final from st_ring_fwd.
 * Workgroups of a launch may pass sums on to one another; should one be kept waiting for seconds, which no schedule of them
 * does, all gradients of the launch are NaN. */
st_status st_ring_bwd(const st_ring_desc* desc, const st_tensor* q, const st_tensor* d_o,
                      const st_tensor* o, int32_t o_dtype, const float* lse_final,
                      const int32_t* order, int32_t n_visit, int32_t mode,
                      float* dq_acc, float* const* dk_acc, float* const* dv_acc,
                      void* workspace, size_t workspace_bytes, void* hip_stream);

/* st_ring_bwd for callers that cannot allocate device memory or hand over a workspace: code under HIP graph
 * capture, tight serving or training loops, harnesses that forbid hipMalloc.  Same arguments and results as
 * st_ring_bwd with a workspace of st_ring_workspace_bytes() (bit for bit) without one: Delta, the tile counters of the
 * dK/dV launch and the scaled copy of Q live in a static device array of st_ring_bwd_noalloc_max_bytes() = 40 MiB that
 * every GPU the library runs on holds until the process ends.  The call allocates and frees nothing (no hipMalloc /
 * hipFree, no allocating library routine); the array's device address is looked up once per device, on the first call.
 * A share whose Delta, counters and copy of Q exceed the array returns ST_ERR_WORKSPACE and enqueues nothing;
 * partial sums of launches that are split over more workgroups, or of one that makes all three gradients, have a second static array of
 * 96 MiB, which is also the most that st_ring_bwd uses of its workspace for them (320 MiB for shares that this call refuses).  Every call on a GPU uses
 * that GPU's one array (what must start at zero is cleared by the call itself): calls that overlap on one GPU, on different streams or from different threads, race; order them. */
st_status st_ring_bwd_noalloc(const st_ring_desc* desc, const st_tensor* q, const st_tensor* d_o,
                              const st_tensor* o, int32_t o_dtype, const float* lse_final,
                              const int32_t* order, int32_t n_visit, int32_t mode,
                              float* dq_acc, float* const* dk_acc, float* const* dv_acc, void* hip_stream);
size_t st_ring_bwd_noalloc_max_bytes(void);

/* st_ring_bwd for the LAST visit of the listed chunks, with the work that follows a chunk's last visit folded
 * into the kernels that produce dK / dV (Section 3.2 "Backward Propagation": the key and value gradients are
 * complete once the chunk has met every query shard).
 *   kv_flags   ST_KV_ASSIGN: dk_acc[j], dv_acc[j] of every chunk in `order` are OVERWRITTEN with this call's
 *              contribution instead of added to (they need not be zeroed; a listed chunk that lies entirely in
 *              the shard's causal future is set to zero).  0: accumulate, as st_ring_bwd.
 *   dk_lowp, dv_lowp  nullable; host arrays [n_chunks] of device pointers, entries nullable (both or neither of a
 *              chunk): the final dk_acc[j] / dv_acc[j] rounded to desc->dtype, dense [B,Sk,Hkv,D], 16-byte
 *              aligned.  ST_BF16 descriptors only.
 * dq_acc is accumulated as in st_ring_bwd.  Same workspace. */
enum { ST_KV_ASSIGN = 1 };
st_status st_ring_bwd_last(const st_ring_desc* desc, const st_tensor* q, const st_tensor* d_o,
                           const st_tensor* o, int32_t o_dtype, const float* lse_final,
                           const int32_t* order, int32_t n_visit, int32_t mode,
                           float* dq_acc, float* const* dk_acc, float* const* dv_acc,
                           int32_t kv_flags, void* const* dk_lowp, void* const* dv_lowp,
                           void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- attention with modified scores: capped by a tanh, biased by distance, masked by documents and prefixes ----
 * One (Q shard, KV chunk) pair as in st_attn_block_fwd / st_attn_block_bwd, with scores
 *   u = scale <q, k>,   y = softcap tanh(u / softcap),   s = y - slope_h |p_q - p_k|
 * over the keys of the row's span.  The states fold with st_attn_merge and st_attn_combine, Delta comes from st_attn_delta.
 *   softcap  0: scores are not capped; otherwise finite and positive.  ST_BF16: at most 1024, and capped scores are some 2^-22 softcap
 *            off (the hardware's exponential and reciprocal); ST_F32: tanhf
 *   slopes   nullable; device fp32 [Hq], finite, as their products with the distances have to be (ST_BF16: and those over scale):
 *            what a unit of distance between the positions of query and key takes off the score; chunks of at most 2^24 keys
 *   spans    nullable; device int64 [B,Sq,2], 16-byte aligned: query row i of batch entry b sees the keys at global positions
 *            spans[b][i][0] <= p < spans[b][i][1] (and, with desc->causal, p <= its own); an empty span is legal (O = 0,
 *            lse = -inf, no gradient).  st_mask_spans makes them; any other interval (a sliding window) is as good.
 * Precision of ST_BF16: scores, softmax, sums in fp32 from the stored Q and K (Q is not scaled and rounded first, as the kernels
 * of the plain scores do); P and the gradient of the scores are rounded to bf16 before the second contractions.
 * Delta has the rounding of the O that st_attn_delta is handed: none with o_part, half a step of bf16 a value with o_lowp.
 * The states' lse is fp32, like everything that is folded from it: with a bias, where a row sees nothing of a sequence but keys
 * far away, its probabilities in the backward carry half a step of an lse of that size, 2^-24 slope distance.
 * Infinities and NaN in rows of Q, K, V, dO reach the results of the rows and keys that see them, and no others.  Outputs overlap
 * neither each other nor an input. */
typedef struct {
  float softcap;
  const float* slopes;      /* device */
  const int64_t* spans;     /* device */
} st_score;

/* Spans of a packed batch (host sizes, device tensors): documents lie one behind the other in every batch entry.
 *   bounds  int64 [B,n_docs+1], rising (equal: an empty document): document d holds the positions bounds[d] <= p < bounds[d+1]
 *   prefix  nullable, int64 [B,n_docs]: so many first tokens of document d are seen by all of its tokens, whatever `causal` says
 *   spans   int64 [B,Sq,2] (out): a row sees its own document, with `causal` up to its own position or the prefix' end;
 *           a row in no document gets an empty span.  Hand them on with desc->causal = 0: the causal order is in them.
 * q_offset, q_seg, q_offset2 place the rows as in st_block_desc.  B Sq <= 2^30, n_docs < 2^30. */
st_status st_mask_spans(int32_t B, int32_t Sq, int64_t q_offset, int32_t q_seg, int64_t q_offset2, int32_t causal,
                        const int64_t* bounds, int32_t n_docs, const int64_t* prefix, int64_t* spans, void* hip_stream);

/* Workspace of the two calls below, for these sizes (0: none is needed): device, 256-byte aligned; its contents mean nothing
 * between calls, and calls that share one must be ordered on one stream.  What score holds does not count. */
size_t st_attn_score_workspace_bytes(const st_block_desc* desc, const st_score* score, int32_t backward);

/* score: nullable (plain scores).  o_part fp32 and / or o_lowp in desc->dtype, dense [B,Sq,Hq,D] (one may be NULL, overwritten);
 * lse_part fp32 [B,Hq,Sq] (overwritten). */
st_status st_attn_score_fwd(const st_block_desc* desc, const st_score* score, const st_tensor* q, const st_tensor* k,
                            const st_tensor* v, float* o_part, float* lse_part, void* o_lowp, void* workspace,
                            size_t workspace_bytes, void* hip_stream);

/* Gradients of the pair from the FINAL lse and Delta: dense fp32 accumulators as in st_attn_block_bwd, ADDED to (flags = 0) or
 * OVERWRITTEN (ST_GRAD_ASSIGN), and / or *_lowp, the same values rounded to desc->dtype, dense.  With ST_GRAD_ASSIGN one of
 * accumulator and *_lowp may be NULL for each gradient; without it the accumulators are needed.  Every element has one writer and
 * every sum a fixed order: results are bit-reproducible.  slopes have no gradient. */
enum { ST_GRAD_ASSIGN = 1 };
st_status st_attn_score_bwd(const st_block_desc* desc, const st_score* score, const st_tensor* q, const st_tensor* k,
                            const st_tensor* v, const st_tensor* d_o, const float* lse_final, const float* delta,
                            int32_t flags, float* dq_acc, float* dk_acc, float* dv_acc, void* dq_lowp, void* dk_lowp,
                            void* dv_lowp, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- norms of queries and keys for each head, and the rotation by their positions, in one pass ----
 * For every token and head x[0 .. D):  n = x rsqrt(mean(x^2) + eps) weight (norm = 0: n = x), then the first `rot` values are
 * rotated in pairs, (a, b) -> (a cos t - b sin t, a sin t + b cos t) with t = p f for the pair's axis position p and frequency f.
 *   pairing     ST_ROPE_HALVES: pair j is (j, j + rot / 2); ST_ROPE_NEIGHBOURS: (2 j, 2 j + 1)
 *   n_axes      1 .. ST_ROPE_MAX_AXES; the first axis_pairs[0] pairs turn by the positions of axis 0, the next axis_pairs[1] by
 *               those of axis 1 (time, height, width of a video patch); they add up to rot / 2
 *   positions   nullable; device int32 [n_axes,B,S].  NULL (one axis): the rows are those of a shard, at offset, and from row seg
 *               on at offset2 (q_offset, q_seg, q_offset2 of st_block_desc)
 *   freq        device fp64 [rot/2], radians per position (any: scaled ones too); angles are made in fp64, for far positions, and
 *               their fraction of a turn is rounded to fp32, 1e-7 radians at most, before its sine and cosine
 *   q_weight, k_weight  nullable (ones); device fp32 [D], for norm = 1 only
 * q, k: [B,S,Hq,D] and [B,S,Hkv,D] views (k is not read where Hkv = 0); arithmetic is fp32, rounded once.  q_out, k_out: views of
 * the same type, which may be q and k themselves.  D <= 256, D % 8 == 0, rot even, 0 <= rot <= D, Hq + Hkv <= 16384, B S <= 2^25. */
enum { ST_ROPE_HALVES = 0, ST_ROPE_NEIGHBOURS = 1, ST_ROPE_MAX_AXES = 4 };
typedef struct {
  int32_t dtype, B, S, Hq, Hkv, D;
  int32_t rot, pairing, norm;
  float   eps;
  int32_t n_axes;
  int32_t axis_pairs[ST_ROPE_MAX_AXES];
  int64_t offset;
  int32_t seg;
  int64_t offset2;
} st_rope_desc;
st_status st_qk_rope_fwd(const st_rope_desc* desc, const st_tensor* q, const st_tensor* k, const float* q_weight,
                         const float* k_weight, const double* freq, const int32_t* positions, const st_tensor* q_out,
                         const st_tensor* k_out, void* hip_stream);

/* Gradients of the same pass.  q, k: its inputs (not read with norm = 0); d_q, d_k: gradients of its outputs, views in d_dtype
 * (ST_F32, as the attention backward leaves them, or desc->dtype); dx_q, dx_k (out): gradients of q and k, views in desc->dtype
 * (may be d_q, d_k where the types agree).  dw_q, dw_k: nullable fp32 [D], with norm = 1: gradients of the weights, added to, or
 * overwritten with ST_GRAD_ASSIGN; sums have a fixed order.  workspace: st_qk_rope_bwd_workspace_bytes(desc) bytes, 256-byte
 * aligned, needed with dw_q or dw_k only. */
size_t st_qk_rope_bwd_workspace_bytes(const st_rope_desc* desc);
st_status st_qk_rope_bwd(const st_rope_desc* desc, const st_tensor* q, const st_tensor* k, const st_tensor* d_q,
                         const st_tensor* d_k, int32_t d_dtype, const float* q_weight, const float* k_weight,
                         const double* freq, const int32_t* positions, int32_t flags, const st_tensor* dx_q,
                         const st_tensor* dx_k, float* dw_q, float* dw_k, void* workspace, size_t workspace_bytes,
                         void* hip_stream);

/* ---- a cache of keys and values in pages, for serving: appending to it, reading chunks of it, attention that reads it ----
 * Token x of sequence b lies in page table[b][x / page] at row x % page.  Every size that changes from step to step (tokens of the
 * sequences, their new rows, the pages) is read from device memory by the kernels, so that a captured call can be replayed.
 *   dtype          what the pages hold: the dtype of the calls' tensors, or ST_E4M3
 *   page           16, 32, 64, 128 or 256
 *   k, v           [n_pages, page, Hkv, D] views (stride_b of a page, stride_s of a token, below 2^20, stride_h of a head), rows
 *                  16-byte aligned
 *   k_scale, v_scale  ST_E4M3 only: device bytes [n_pages, Hkv]; a stored value stands for its e4m3 value times 2^(scale - 127)
 *                  (1 <= scale <= 254; of pages that hold no token anything), an infinity where fp32 does not hold that.  Whole powers
 *                  of two: every value is exact in bf16, and a page whose scale grows keeps its rows but for what falls below the
 *                  least e4m3 value
 *   table          device int32 [B, width].  An entry that is no page (negative, or >= n_pages: a page that a window has left behind)
 *                  holds nothing: its tokens are not stored, not seen, and read as zeros
 *   lens           device int32 [B]: tokens of every sequence, those that a call appends among them; at most width page of them
 * Rows of a call are packed: T rows, of which sequence b has the n_b = starts[b + 1] - starts[b] from starts[b] on (device int32
 * [B + 1], rising, in 0 .. T; n_b may be 0).  Row i of sequence b is its token lens[b] - n_b + i.  Rows of no sequence (T may be
 * more than there are, as for a captured call) are left as they were.
 * A page may be in the tables of several sequences (a common beginning), but only one of them may append to it, in one call at a time,
 * and of the pages that a call appends to each stands once in its sequence's table.
 * D: multiples of 8 up to 256 (ST_E4M3: of 16); B <= 65535, T <= 2^25, width page <= 2^30. */
typedef struct {
  int32_t  dtype, n_pages, page, Hkv, D, B, width;
  st_tensor k, v;
  uint8_t *k_scale, *v_scale;
  const int32_t *table, *lens;
} st_cache;

/* The norms and rotations of st_qk_rope_fwd over new rows, and their keys and values into the cache.
 *   desc        B = 1, S = T, seg = 0; Hq may be 0 (then q and q_out are not read); positions are the tokens' places in their
 *               sequences + offset, or come from `positions` int32 [n_axes,1,T].  Hkv and D are the cache's
 *   q, k, v     [1,T,heads,D] views in desc->dtype; q_out as q, which it may be
 * ST_E4M3: the scale of a page and head is 2^e with the least e for which all new values of the page are within 448 2^e, and not
 * below what the rows have that were there before, which are rescaled where it grows; values that are not finite are stored as NaN and
 * do not count for the scale.  Keys for pages in fewer bits than fp32 are normed and rotated in fp64 (angles to 2^-52 of themselves), so that
 * in ST_E4M3 each is the nearest stored value to the exact one, in ST_BF16 that of the exact one in fp32, but where the exact one is as
 * close to the middle of two; queries, and keys in ST_F32, in fp32.
 * Repeating a call with the same tensors, q_out not q, changes nothing. */
st_status st_cache_append(const st_rope_desc* desc, const st_cache* cache, const int32_t* starts, const st_tensor* q, const st_tensor* k,
                          const st_tensor* v, const float* q_weight, const float* k_weight, const double* freq, const int32_t* positions,
                          const st_tensor* q_out, void* hip_stream);

/* Tokens first[b] .. first[b] + count - 1 of every sequence (first: device int32 [B], NULL: 0) as chunks [B,count,Hkv,D], views in
 * `dtype` (that of the cache; of ST_E4M3 either other); tokens past a sequence's end are zeros.  k_out or v_out may be NULL.
 * count <= 2^28, count Hkv D < 2^34. */
st_status st_cache_read(const st_cache* cache, const int32_t* first, int32_t count, int32_t dtype, const st_tensor* k_out,
                        const st_tensor* v_out, void* hip_stream);

/* Attention of packed rows against the cache, with the scores of st_score: a row at position p sees the tokens x < lens[b] of its
 * sequence with x <= p (causal) and p - x < window (window > 0).
 *   q_first     nullable; device int64 [B]: position of a sequence's first row, counted from the cache's first token (a GPU that has a
 *               share of a sequence's tokens passes the distance from the share's beginning).  NULL: lens[b] - n_b
 *   max_rows    no sequence has more rows than this; rows behind are not computed
 *   softcap, slopes  as in st_score
 *   o_part fp32 and / or o_lowp in dtype, dense [1,T,Hq,D]; lse_part fp32 [1,Hq,T]: a state that st_attn_merge and st_attn_combine fold
 *   (B = 1, Sq = T).  A row that sees nothing has O = 0, lse = -inf.
 * ST_BF16 with D = 64 or 128 (pages of ST_BF16 or ST_E4M3), ST_F32 with any D (pages of ST_F32 or ST_E4M3).  Scores, softmax and sums
 * are fp32; of bf16 rows exp(s - max) meets the values as two bf16 parts (2^-16), whatever else is in the call, in sequences of up to 128
 * rows of a KV head's query heads (n_b Hq / Hkv), and in all of a call with min(max_rows, T) Hq / Hkv <= 256 and few tiles of 128 rows (64, KV heads
 * counted); as one (2^-8, as in st_score) in longer ones.  Infinities and NaN reach the rows that see them, and no others.
 * Results do not depend on the order of the pages. */
typedef struct {
  int32_t dtype, T, Hq, max_rows, causal, window;
  float   scale, softcap;
  const float* slopes;      /* device */
} st_cache_rows;
size_t st_attn_cache_workspace_bytes(const st_cache_rows* rows, const st_cache* cache);   /* device, 256-byte aligned; as for st_attn_score_fwd */
st_status st_attn_cache(const st_cache_rows* rows, const st_cache* cache, const int32_t* starts, const int64_t* q_first, const st_tensor* q,
                        float* o_part, float* lse_part, void* o_lowp, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- per-kernel timing for benchmarks (not part of the method) ----
 * Between st_profile_begin() and st_profile_end() the library records a HIP event on the launch
 * stream before and after every kernel it launches (this creates hipEvent_t objects; at most 4096
 * launches are recorded, later ones run untimed).  st_profile_end() waits for the recorded events,
 * sums the durations per kernel name into out[0 .. *n_entries) (host memory, at most max_entries
 * entries) and stops recording.  Process-wide; not meant to be used from several threads at once. */
typedef struct {
  char    name[48];
  int32_t launches;
  float   total_ms;
} st_profile_entry;
st_status st_profile_begin(void);
st_status st_profile_end(st_profile_entry* out, int32_t max_entries, int32_t* n_entries);

/* ---- the device as the library sees it, for benchmark reports (not part of the method) ----
 * Facts of the current HIP device: compute units, XCDs (accelerator dies with an L2 each; 8 when the runtime
 * does not tell), the maximum shader and memory clocks, bus width and memory size.  `out` is host memory. */
typedef struct {
  char    name[64];
  char    arch[32];
  int32_t compute_units;
  int32_t xcds;
  int32_t max_clock_mhz;
  int32_t memory_clock_mhz;
  int32_t memory_bus_bits;
  int64_t hbm_bytes;
} st_device_report;
st_status st_device_facts(st_device_report* out);

/* ---- MFMA loops for benchmarks (not part of the method) ----
 * One workgroup of four wavefronts per compute unit; every wavefront loads 16 operand fragments (16 bytes per
 * lane each) from `operands` and then runs `iters` iterations of a loop of v_mfma_f32_32x32x16_bf16 on them.
 * Timed by the caller (events on the stream), it gives the rate the matrix units sustain on THAT data, which is
 * the ceiling to compare an attention kernel with: the chip runs at its power limit, and the limit depends on
 * the operand values and on what is issued beside the MFMAs.
 *   mix       0: nothing but MFMAs (32 per iteration).  1 .. st_mfma_probe_mixes(): side instructions with
 *             independent operands are spread between the MFMAs (st_mfma_probe_mix_name: "valu2" two v_mul_f32
 *             per MFMA, "exp1" one v_exp_f32, "pack2" two v_cvt_pk_bf16_f32, "lds1" one 16-byte LDS read,
 *             "ldstr1" one transposing 8-byte LDS read; "fwd", "dq", "dkv", "one" and "fwd64", "dq64", "dkv64",
 *             "one64": the instruction counts per key block of the forward, dQ and dK/dV loops and of the one that
 *             makes all gradients at head sizes 128 and 64, without their dependencies, barriers and global memory
 *             operations - what such a mix reaches bounds that loop on the same data)
 *   operands  device, 16-byte aligned, operand_bytes >= 65536 bytes of bf16 values (read with wrap-around)
 *   sink      device, sink_floats >= 256 * compute units floats (overwritten; keeps the loop alive)
 *   flop      host, nullable: floating point operations of the MFMAs the launch executes (2 per multiply-add) */
st_status st_mfma_probe(const void* operands, int64_t operand_bytes, int32_t mix, int32_t iters, float* sink,
                        int64_t sink_floats, double* flop, void* hip_stream);
int32_t     st_mfma_probe_mixes(void);
const char* st_mfma_probe_mix_name(int32_t mix);   /* "" for a mix out of range */

/* ---- misc ---- */
const char* st_status_str(st_status s);
const char* st_last_error(void);      /* thread-local text of the last failure, "" if none */
int32_t     st_version(void);         /* major*10000 + minor*100 + patch */

#ifdef __cplusplus
}
#endif
#endif /* STARTRAIL_H */
