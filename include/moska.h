/*
 * moska.h -- C ABI of the MoSKA decode-attention hot path for NVIDIA B200 (sm_100a).
 *
 * MoSKA (Mixture of Shared KV Attention) splits the KV context of a batch of decoding requests
 * into a large SHARED store, partitioned into chunks that many requests attend to, and a
 * per-request UNIQUE KV.  One decode step of one attention layer is
 *
 *   route  ->  group_by_chunk  ->  { shared_attn  ||  unique_attn }  ->  merge
 *
 * (Section III-A "Shared KV Attention", Section III-B "The MoSKA Architecture", Fig. 2.)
 *
 * Conventions that hold for every entry point
 * -------------------------------------------
 *  * All tensor arguments are DEVICE pointers owned by the caller, unless a parameter is
 *    documented as a host pointer.  The library never allocates, frees or keeps a pointer
 *    after the call returns.  Scratch memory comes from a caller-provided workspace.
 *  * Every call only enqueues work on `stream` and returns without synchronising, and nothing
 *    produced on the device is read back by the host.  The exceptions say so at their
 *    declaration: moska_device_status and the *_host forms of the step wait for the device.
 *  * bf16 tensors are passed as `const uint16_t*` (raw bfloat16 bit patterns).
 *  * Symbols: B requests, Hq query heads, Hkv KV heads, G = Hq / Hkv (1..8), D head dimension
 *    (64 or 128), C shared chunks of L tokens each, k chunks routed per (request, KV head).
 *    Query row r = b * Hq + hq; its KV head is h = hq / G.
 *  * Partial results: every query row owns `n_slots = shared_slots + n_unique_splits` slots.
 *        o_part   float [B][Hq][n_slots][D]   softmax-normalised partial output
 *        lse_part float [B][Hq][n_slots]      natural-log sum of exp(scale * q.k) over the
 *                                             tokens of that slot; -inf marks an empty slot
 *    Shared attention writes slots [0, shared_slots), unique attention writes slots
 *    [shared_slots, n_slots).  Both write EVERY slot of their range (empty ones as -inf, o = 0),
 *    so the caller never has to clear the buffers.
 *  * Return value: MOSKA_OK or a negative moska_status.  moska_last_error() gives a text for
 *    the last failure on the calling thread.  Invalid arguments are detected on the host
 *    before anything is launched.
 *  * What a kernel can only find out while it runs (routing indices that break the grouping's
 *    preconditions, an entry outside the batch, a bounded wait that ran out) goes to one sticky
 *    status word per device, read and cleared by moska_device_status().  A kernel that raises it
 *    never traps and never writes outside the caller's buffers; the results of that step are not
 *    valid.
 *  * Hidden state: none that outlives a call on the device side.  On the host side the library
 *    keeps, per device ordinal, the address of its status word (and of the built-in scratch of
 *    moska_group_by_chunk_noalloc), and per (host thread, device) the two CUDA events that order
 *    the side stream of a two-stream moska_decode_step; all are created on first use with that
 *    device current and are not valid across a cudaDeviceReset.
 */
#ifndef MOSKA_H_
#define MOSKA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum moska_status {
    MOSKA_OK              = 0,
    MOSKA_ERR_INVALID_ARG = -1, /* null pointer, k > C, Hq % Hkv != 0, misaligned pointer ...   */
    MOSKA_ERR_UNSUPPORTED = -2, /* D not in {64,128}, G > 8, L % 128 != 0, device is not sm_100 */
    MOSKA_ERR_WORKSPACE   = -3, /* workspace missing or smaller than moska_workspace_bytes()    */
    MOSKA_ERR_CUDA        = -4, /* a CUDA runtime call or kernel launch failed                  */
    MOSKA_ERR_TIMEOUT     = -5, /* device side: a bounded wait inside a kernel ran out          */
    MOSKA_ERR_CORRUPT     = -6  /* device side, debug build: workspace guard words overwritten  */
} moska_status;

/* Problem shape of one decode step of one layer. */
typedef struct moska_shape {
    int32_t B;               /* concurrent requests                                              */
    int32_t Hq;              /* query heads                                                      */
    int32_t Hkv;             /* KV heads, Hq % Hkv == 0, G = Hq / Hkv <= 8                       */
    int32_t D;               /* head dimension: 64 or 128                                        */
    int32_t C;               /* number of shared chunks                                          */
    int32_t L;               /* tokens per shared chunk, a multiple of 128                       */
    int32_t k;               /* chunks routed per (request, KV head), 1 <= k <= C                */
    int32_t shared_slots;    /* partial slots written by shared attention: k in routed mode;     */
                             /* in dense mode (no routing) the C chunks are cut into this many   */
                             /* runs of ceil(C / shared_slots) consecutive chunks                */
    int32_t n_unique_splits; /* partial slots written by unique attention (split-K), >= 1        */
    int64_t unique_tokens;   /* optional hint: the private tokens of all requests together, if   */
                             /* the host knows them, else 0.  Only moska_decode_step reads it,   */
                             /* to divide the SMs between shared and unique attention; results   */
                             /* never depend on it                                               */
    int32_t q_len;           /* query tokens per request (speculative decoding, chunked prefill;  */
                             /* Section II-A's multi-turn reuse): 0 or 1 = one.  With q_len > 1   */
                             /* the B batch rows are B / q_len requests, row b = r * q_len + i is */
                             /* token i of request r, kv_start / kv_len have B / q_len entries,   */
                             /* kv_len[r] counts the tokens the LAST query token sees and token i */
                             /* sees the first kv_len[r] - (q_len - 1 - i) of them.  Routing and  */
                             /* shared attention treat every row as a request of its own; unique  */
                             /* attention reads the request's K/V once for all its rows (needs    */
                             /* D = 128 and q_len * G <= 16; <= 8 with the FP8 store)             */
} moska_shape;

typedef void* moska_stream; /* a cudaStream_t */

/* Optional per-stage device timing of moska_decode_step (CUDA events recorded on the stream each
 * stage is launched on).  Stage order of the arrays below. */
enum { MOSKA_STAGE_ROUTE = 0, MOSKA_STAGE_GROUP, MOSKA_STAGE_SHARED, MOSKA_STAGE_UNIQUE,
       MOSKA_STAGE_MERGE, MOSKA_N_STAGES };
typedef struct moska_profiler moska_profiler;

/* Library version, major * 100 + minor. */
int moska_version(void);

/* Text of the last error raised on the calling thread ("" if none). Host pointer, never NULL. */
const char* moska_last_error(void);

/* Waits for the current device to finish, stores the sticky device-side status word in
 * *status_host (host pointer) and clears it.  0 means no kernel of the library raised anything.
 * MOSKA_ERR_TIMEOUT: a CTA of the tensor-core Shared KV Attention kernel, or a warp of the 4-bit
 * paged attention or tree attention, gave up on one of its bounded waits (TMA, MMA or bulk-copy completion).
 * MOSKA_ERR_INVALID_ARG: a grouping call (either entry point) met a chunk index outside [0, C) or
 * a (request, KV head) list that is not strictly ascending, shared attention met an entry of
 * seg_entries outside [0, B*Hkv*k), a call on a paged store met a page index, a length or a
 * position that is out of range, or one on trees a parent, a row range or a path that is none.  In every
 * case the outputs of the steps since the last read are not valid.  MOSKA_ERR_CORRUPT (debug
 * build only): guard words of the workspace were overwritten or a work list would have overflowed.
 * The most negative code raised since the last read is the one reported. */
int moska_device_status(int32_t* status_host);

/* n_slots = shared_slots + n_unique_splits; negative status if the shape is invalid. Host only. */
int moska_partial_slots(const moska_shape* shape);

/* Bytes of workspace that moska_route / moska_group_by_chunk / moska_shared_attn[_fp8] need for
 * this shape (one workspace serves all of them; 256-byte aligned base required): the grouping's bit
 * sets and work lists, the router's scores beyond 256 chunks, and, for D = 128, room for an f16
 * copy of the queries (B*Hq*D*2 bytes, used by the FP8 shared store only).  Host only, pure.  */
size_t moska_workspace_bytes(const moska_shape* shape);

/* A reasonable n_unique_splits for a batch whose longest unique context has `max_len` tokens.
 * Host only, pure.                                                                              */
int moska_default_unique_splits(int32_t B, int32_t Hkv, int32_t max_len);

/* The same for a private store in FP8 (moska_unique_attn_fp8, moska_decode_step_fp8kv), whose
 * kernel has more and shorter-lived CTAs per SM.  Host only, pure.                             */
int moska_default_unique_splits_fp8(int32_t B, int32_t Hkv, int32_t max_len);

/*
 * Chunk embeddings used by the router (Section III-B: "precomputed chunk embeddings"; the
 * embedding of a chunk is the arithmetic mean of its L keys, per KV head).  Offline step.
 *   k_shared   bf16  [Hkv][C][L][D]   (16-byte aligned)
 *   summaries  float [Hkv][C][D]      out
 */
int moska_build_chunk_summaries(const uint16_t* k_shared, float* summaries,
                                const moska_shape* shape, moska_stream stream);

/*
 * A second training-free chunk embedding for the same `summaries` buffer (Section II-B and III-B
 * cite two lightweight routers: one pools a chunk's keys uniformly -- the mean above -- the other
 * weights a chunk's tokens by an attention pass inside the chunk).  Here the chunk's mean key
 * kbar probes the chunk's own keys:
 *     w_t = softmax_t(probe_scale * <kbar, k_t>),   summaries[h][c] = sum_t w_t k_t,
 * so tokens aligned with the chunk's centre count more and outliers less; probe_scale = 0 gives
 * the mean.  Everything downstream (moska_route and on) is unchanged.  Offline step; fp32.
 *   probe_scale  finite, >= 0 (1/sqrt(D) is the natural choice); L <= 10240
 */
int moska_build_chunk_summaries_attn(const uint16_t* k_shared, float* summaries, float probe_scale,
                                     const moska_shape* shape, moska_stream stream);

/*
 * Router (Section III-B): relevance of chunk c for (request b, KV head h) is the inner product
 * of the pooled query  qbar[b][h] = sum_{g<G} q[b][h*G+g]  with summaries[h][c]; the k chunks
 * with the largest score are selected, exact ties going to the lower chunk index.
 *   q           bf16  [B][Hq][D]
 *   summaries   float [Hkv][C][D]
 *   topk_idx    int32 [B][Hkv][k]   out, chunk indices in ASCENDING order
 *   topk_score  float [B][Hkv][k]   out, score of topk_idx[...] (same order); may be NULL
 * Up to 256 chunks one warp scores and selects for one (b, h) out of shared memory and `ws` may
 * be NULL; beyond that the scores are computed as a tiled fp32 product into `ws` (which must
 * then hold moska_workspace_bytes(); the grouping call may reuse the same workspace afterwards)
 * and selected by one warp per (b, h).
 */
int moska_route(const uint16_t* q, const float* summaries, int32_t* topk_idx, float* topk_score,
                const moska_shape* shape, void* ws, size_t ws_bytes, moska_stream stream);

/*
 * Query aggregation (Section III-A: the N concurrent queries that hit the same shared chunk are
 * gathered into one query matrix).  Let p = (b*Hkv + h)*k + j be the flat position of the j-th
 * routed chunk of (b, h) and key(p) = h*C + topk_idx[p].  This is a stable counting sort of the
 * positions by key:
 *   seg_offsets  int32 [Hkv*C + 1]  out, exclusive scan of the number of positions per key
 *   seg_entries  int32 [B*Hkv*k]    out, positions p, key-major, ascending p inside one key
 * The result is deterministic.  It also writes the tile work lists that moska_shared_attn
 * consumes into `ws` (give both calls the same, unmodified workspace).
 * Precondition (what moska_route produces): every list topk_idx[b][h][0..k) is STRICTLY ASCENDING,
 * hence without repeated chunks, and lies in [0, C).  The sort is done on one bit per (key,
 * request), which only describes such lists.  The marking pass checks it on the device: an index
 * outside [0, C) is skipped and a list out of order is flagged, both as MOSKA_ERR_INVALID_ARG in
 * the device status word (moska_device_status); seg_entries then still holds only positions that
 * exist, but a repeated or skipped chunk is missing from it, so the step's results are not valid.
 */
int moska_group_by_chunk(const int32_t* topk_idx, int32_t* seg_offsets, int32_t* seg_entries,
                         const moska_shape* shape, void* ws, size_t ws_bytes, moska_stream stream);

/*
 * moska_group_by_chunk for callers that cannot allocate device memory.  (The paper has no
 * counterpart; this is a packaging variant of the call above.)
 *
 * Some hosts of this library may not call cudaMalloc at the point where they need the grouping:
 * a serving engine that gave all device memory to its own pool at start-up and has no bytes left
 * to carve a workspace from, or a latency-critical loop in which an allocation (which can
 * synchronise the whole device) is not acceptable.  For them the scratch of the grouping passes
 * lives in a fixed buffer of MOSKA_NOALLOC_SCRATCH_BYTES inside the library image; every GPU
 * that loads the library keeps that buffer until the process exits.  The call allocates and
 * frees nothing, neither directly nor through another library.
 *
 *   inputs / outputs      as moska_group_by_chunk (topk_idx in; seg_offsets, seg_entries out),
 *                         same precondition on topk_idx, same report through moska_device_status
 *   limit                 shapes whose grouping scratch (moska_workspace_bytes) exceeds the
 *                         buffer are rejected with MOSKA_ERR_WORKSPACE before anything runs
 *   first call            the first call on each device looks up the buffer's device address
 *                         (with that device current); make it before any stream capture
 *   shared state          all calls on a device use the same buffer and each call first clears
 *                         what it needs zeroed, so calls in stream order are independent; calls
 *                         that overlap on the GPU (different streams, no ordering) race
 *   work lists            the tile lists for moska_shared_attn stay inside the buffer and are not
 *                         exported; pair moska_shared_attn with moska_group_by_chunk instead
 */
#define MOSKA_NOALLOC_SCRATCH_BYTES (8u << 20)
int moska_group_by_chunk_noalloc(const int32_t* topk_idx, int32_t* seg_offsets,
                                 int32_t* seg_entries, const moska_shape* shape,
                                 moska_stream stream);

/*
 * Debug aid (no counterpart in the paper).  A library compiled with -DMOSKA_DEBUG_GUARDS
 * (`python -m paper_2511_06010_b200.build --debug` -> csrc/libmoska_debug.so) leaves 256 guard
 * bytes behind every region of the workspace (moska_workspace_bytes grows accordingly), fills them
 * and the regions' alignment padding with a pattern at the start of moska_route /
 * moska_group_by_chunk, compares them at the end of the grouping, and checks every work-list write
 * against the list's capacity.  This call compares the guard words once more, at any later point
 * (after shared attention, after the step): a mismatch raises MOSKA_ERR_CORRUPT in the device
 * status word (moska_device_status).  Nothing traps; a write beyond a list's capacity is skipped.
 *   ws, ws_bytes   the workspace the grouping call was given (device pointer, 256-byte aligned)
 * Returns MOSKA_ERR_UNSUPPORTED in a library built without the guard words (the regular build:
 * its workspace layout has no room for them and its kernels carry no checks).
 */
int moska_debug_check_workspace(void* ws, size_t ws_bytes, const moska_shape* shape,
                                moska_stream stream);

/*
 * Shared KV Attention (Section III-A, Fig. 2a): for every non-empty segment (h, c) the query rows
 * of all requests routed to chunk c form the rows of one Q matrix; S = scale * Q Kc^T, row-wise
 * softmax statistics and O = softmax(S) Vc are computed as one batched tensor-core product, so
 * the chunk's K/V tile leaves HBM once per step however many requests use it.
 * For entry p = (b*Hkv+h)*k + j and each g < G it writes slot j of row (b, h*G+g).
 *   q                      bf16 [B][Hq][D]
 *   k_shared, v_shared     bf16 [Hkv][C][L][D]   (128-byte aligned)
 *   topk_idx/seg_offsets/seg_entries   as produced by moska_route / moska_group_by_chunk,
 *       or all three NULL for DENSE mode: no routing, every row attends every chunk; run s of
 *       ceil(C/shared_slots) consecutive chunks goes to slot s (needs no prior grouping call).
 *   o_part, lse_part       see "Partial results" above; slots [0, shared_slots) are written
 *   softmax_scale          multiplies q.k before the softmax (usually 1/sqrt(D))
 */
int moska_shared_attn(const uint16_t* q, const uint16_t* k_shared, const uint16_t* v_shared,
                      const int32_t* topk_idx, const int32_t* seg_offsets,
                      const int32_t* seg_entries, float* o_part, float* lse_part,
                      float softmax_scale, const moska_shape* shape, void* ws, size_t ws_bytes,
                      moska_stream stream);

/*
 * Shared KV Attention over a shared store kept in FP8 (E4M3), the KV precision the paper's
 * evaluation assumes (Section IV) applied to the batched product of Section III-A.  Token t of chunk
 * c of KV head h has key k_scale[h][c] * e4m3(k8[h][c][t][:]) and value v_scale[h][c] *
 * e4m3(v8[h][c][t][:]): ONE scale per (KV head, chunk) and tensor, so the key scale joins the softmax
 * scale and the value scale the final normalisation.  The code tiles arrive by TMA (half the bytes
 * of the bf16 store), are widened exactly to f16 in shared memory and multiplied on the tensor cores
 * with f16 Q and P and fp32 accumulation.  Routed or dense mode as for moska_shared_attn (in dense
 * mode a partial slot covers a run of chunks with different scales: the running maximum is kept in
 * scaled units and a chunk's value scale, relative to the run's first, joins its P tiles), D = 128.  Segments of at most 8 query rows are streamed by a
 * kernel of their own (codes widened in registers, f16 warp MMAs), as with the bf16 store.
 *   k8_shared, v8_shared  uint8 [Hkv][C][L][D]  OCP FP8 E4M3 codes (128-byte aligned)
 *   k_scale, v_scale      float [Hkv][C]        positive
 *   ws                    as for moska_shared_attn (the grouping's work lists); the call also keeps
 *                         an f16 copy of q in it, so it WRITES the workspace and needs it in dense
 *                         mode too
 * Chunk embeddings for the router are built from whichever copy of the keys the caller has in
 * bf16 (moska_build_chunk_summaries*); they are an offline step.
 */
int moska_shared_attn_fp8(const uint16_t* q, const uint8_t* k8_shared, const uint8_t* v8_shared,
                          const float* k_scale, const float* v_scale, const int32_t* topk_idx,
                          const int32_t* seg_offsets, const int32_t* seg_entries, float* o_part,
                          float* lse_part, float softmax_scale, const moska_shape* shape, void* ws,
                          size_t ws_bytes, moska_stream stream);

/*
 * Unique KV Attention (Section III-A: per-request attention over private KV, a memory-bound
 * GEMV-like pass).  Split-K over the request's tokens: each of the n_unique_splits slots holds
 * the partial result over a disjoint token range (which range is an implementation detail);
 * slots without tokens are written as lse = -inf, o = 0.
 *   k_unique, v_unique  bf16 [T_total][Hkv][D]  token-major ragged store (16-byte aligned)
 *   kv_start            int64 [B]  first token of request b in the store
 *   kv_len              int32 [B]  number of tokens of request b (0 allowed)
 */
int moska_unique_attn(const uint16_t* q, const uint16_t* k_unique, const uint16_t* v_unique,
                      const int64_t* kv_start, const int32_t* kv_len, float* o_part,
                      float* lse_part, float softmax_scale, const moska_shape* shape,
                      moska_stream stream);

/*
 * Unique KV Attention over a private KV store kept in FP8 (E4M3), the KV precision the paper's
 * evaluation assumes (Section IV) applied to the memory-bound per-request pass of Section III-A.
 * Token t of KV head h has key k_scale[t][h] * e4m3(k8[t][h][:]) and value v_scale[t][h] *
 * e4m3(v8[t][h][:]); everything else (split-K slots, empty requests, outputs) is as in
 * moska_unique_attn.  The codes are widened exactly to f16 and multiplied on tensor cores with
 * fp32 accumulation; P is rounded to f16.  D must be 128.
 *   k8, v8            uint8 [T_total][Hkv][D]   OCP FP8 E4M3 codes (16-byte aligned)
 *   k_scale, v_scale  float [T_total][Hkv]
 */
int moska_unique_attn_fp8(const uint16_t* q, const uint8_t* k8, const uint8_t* v8,
                          const float* k_scale, const float* v_scale, const int64_t* kv_start,
                          const int32_t* kv_len, float* o_part, float* lse_part,
                          float softmax_scale, const moska_shape* shape, moska_stream stream);

/*
 * Combination of the shared and unique partial results.  The paper leaves this step implicit;
 * the log-sum-exp merge is the only combination that equals softmax attention over the union of
 * the tokens (Section III-A/III-B).  Per row: M = max_i lse_i, w_i = exp(lse_i - M),
 * out = sum_i w_i o_i / sum_i w_i, lse = M + ln sum_i w_i.  Slots with lse = -inf contribute
 * nothing; if every slot is -inf then out = 0 and lse = -inf (never NaN).
 *   out      bf16  [B][Hq][D]        out
 *   out_f32  float [B][Hq][D]        out, unrounded copy; may be NULL
 *   lse_out  float [B][Hq]           out; may be NULL
 */
int moska_merge(const float* o_part, const float* lse_part, uint16_t* out, float* out_f32,
                float* lse_out, const moska_shape* shape, moska_stream stream);

/*
 * Measured comparison, not part of the method: the unbatched form that Shared KV Attention
 * replaces (Section I, Section III-A: one memory-bound GEMV pass per request over each routed
 * chunk).  Same results as moska_shared_attn, same slots; reads every routed chunk once per
 * (request, KV head) instead of once per step.  topk_idx == NULL selects dense mode.
 */
int moska_gemv_baseline(const uint16_t* q, const uint16_t* k_shared, const uint16_t* v_shared,
                        const int32_t* topk_idx, float* o_part, float* lse_part,
                        float softmax_scale, const moska_shape* shape, moska_stream stream);

/* Creates a profiler able to hold `max_steps` recorded steps (host object owning CUDA events). */
int moska_profiler_create(moska_profiler** out, int32_t max_steps);
void moska_profiler_destroy(moska_profiler* prof);
/* Restricts recording to the stages whose bit (1 << MOSKA_STAGE_x) is set in stage_mask (all
 * stages by default).  Every recorded stage costs two event records per step on the stream it
 * runs on -- about 3 us per stage on a B200 -- so a caller timing whole steps records only the
 * stage it needs.  Stages that are not recorded read as 0. */
int moska_profiler_select(moska_profiler* prof, uint32_t stage_mask);
/* Waits for the recorded events, adds up the elapsed milliseconds per stage over the steps
 * recorded since the last read into stage_ms[MOSKA_N_STAGES] (host), stores their number in
 * *n_steps (host) and clears the profiler. */
int moska_profiler_read(moska_profiler* prof, float* stage_ms, int32_t* n_steps);

/*
 * One whole decode step on device buffers.  Without `side_stream` everything runs on `stream`
 * in the order route, group, unique, shared, merge.  With it, unique attention is enqueued first
 * on `stream`; route, group and shared attention follow on `side_stream` (both ordered after the
 * work already on `stream`), and the merge waits for both.  `side_stream` must have a HIGHER
 * priority than `stream`: its CTAs then take SMs over as unique-attention CTAs retire.  The
 * persistent tensor-core kernel of shared attention is given only a share of the SMs (derived
 * from the two kernels' estimated work, see shape->unique_tokens), so the HBM-bound unique
 * attention keeps running on the others: the two resource profiles overlap on one GPU.
 * Dense mode (no routing) when summaries == NULL.
 * Scratch buffers topk_idx [B*Hkv*k], seg_offsets [Hkv*C+1], seg_entries [B*Hkv*k], o_part,
 * lse_part and ws are caller-owned as in the individual calls.  `prof` may be NULL; otherwise
 * the step's stage boundaries are recorded into it (steps beyond its capacity are not recorded).
 */
int moska_decode_step(const uint16_t* q, const float* summaries, const uint16_t* k_shared,
                      const uint16_t* v_shared, const uint16_t* k_unique,
                      const uint16_t* v_unique, const int64_t* kv_start, const int32_t* kv_len,
                      int32_t* topk_idx, int32_t* seg_offsets, int32_t* seg_entries,
                      float* o_part, float* lse_part, uint16_t* out, float* lse_out,
                      float softmax_scale, const moska_shape* shape, void* ws, size_t ws_bytes,
                      moska_stream stream, moska_stream side_stream, moska_profiler* prof);

/*
 * moska_decode_step with the private KV store in FP8 (E4M3 codes + per-(token, head) fp32 scales,
 * laid out as for moska_unique_attn_fp8); the shared store stays bf16.  Same schedule, buffers,
 * outputs and error behaviour; D must be 128.
 */
int moska_decode_step_fp8kv(const uint16_t* q, const float* summaries, const uint16_t* k_shared,
                            const uint16_t* v_shared, const uint8_t* k8_unique,
                            const uint8_t* v8_unique, const float* k_scale, const float* v_scale,
                            const int64_t* kv_start, const int32_t* kv_len, int32_t* topk_idx,
                            int32_t* seg_offsets, int32_t* seg_entries, float* o_part,
                            float* lse_part, uint16_t* out, float* lse_out, float softmax_scale,
                            const moska_shape* shape, void* ws, size_t ws_bytes, moska_stream stream,
                            moska_stream side_stream, moska_profiler* prof);

/*
 * moska_decode_step with the SHARED store in FP8 (laid out as for moska_shared_attn_fp8); the
 * private store stays bf16.  Same schedule, buffers, outputs and error behaviour (summaries NULL
 * selects dense mode); D = 128; the workspace is needed in dense mode too.
 */
int moska_decode_step_fp8shared(const uint16_t* q, const float* summaries, const uint8_t* k8_shared,
                                const uint8_t* v8_shared, const float* k_scale_shared,
                                const float* v_scale_shared, const uint16_t* k_unique,
                                const uint16_t* v_unique, const int64_t* kv_start, const int32_t* kv_len,
                                int32_t* topk_idx, int32_t* seg_offsets, int32_t* seg_entries,
                                float* o_part, float* lse_part, uint16_t* out, float* lse_out,
                                float softmax_scale, const moska_shape* shape, void* ws, size_t ws_bytes,
                                moska_stream stream, moska_stream side_stream, moska_profiler* prof);

/*
 * moska_decode_step with BOTH stores in FP8, the KV precision of the paper's evaluation (Section
 * IV) on the whole path: the shared store as for moska_shared_attn_fp8 (one scale per (KV head,
 * chunk)), the private store as for moska_unique_attn_fp8 (one scale per (token, KV head)).  Same
 * schedule, buffers, outputs and error behaviour as moska_decode_step (summaries NULL selects dense
 * mode); D = 128; the workspace is needed in dense mode too.
 */
int moska_decode_step_fp8(const uint16_t* q, const float* summaries, const uint8_t* k8_shared,
                          const uint8_t* v8_shared, const float* k_scale_shared, const float* v_scale_shared,
                          const uint8_t* k8_unique, const uint8_t* v8_unique, const float* k_scale_unique,
                          const float* v_scale_unique, const int64_t* kv_start, const int32_t* kv_len,
                          int32_t* topk_idx, int32_t* seg_offsets, int32_t* seg_entries, float* o_part,
                          float* lse_part, uint16_t* out, float* lse_out, float softmax_scale,
                          const moska_shape* shape, void* ws, size_t ws_bytes, moska_stream stream,
                          moska_stream side_stream, moska_profiler* prof);

/*
 * moska_decode_step for a caller whose step inputs live in HOST memory: copies q_host (bf16
 * [B][Hq][D], ideally pinned) into q_dev, runs the step, copies `out` back into out_host (bf16
 * [B][Hq][D]) and waits for the stream.  The KV stores and all scratch stay on the device.
 * q_host must be 16-byte aligned.  With a side stream and buffers of 4 MiB or more the copies
 * leave the critical path: a PAGE-LOCKED q_host is copied on the side stream in front of the
 * router while unique attention reads its query rows straight from host memory, and the result
 * is merged in four row ranges, each copied to out_host on the side stream while the next one is
 * merged.  Pageable buffers and small ones take one copy before and one after the step.  Both
 * host buffers belong to the call until it returns.
 */
int moska_decode_step_host(const uint16_t* q_host, uint16_t* q_dev, const float* summaries,
                           const uint16_t* k_shared, const uint16_t* v_shared,
                           const uint16_t* k_unique, const uint16_t* v_unique,
                           const int64_t* kv_start, const int32_t* kv_len, int32_t* topk_idx,
                           int32_t* seg_offsets, int32_t* seg_entries, float* o_part,
                           float* lse_part, uint16_t* out_dev, uint16_t* out_host,
                           float softmax_scale, const moska_shape* shape, void* ws,
                           size_t ws_bytes, moska_stream stream, moska_stream side_stream,
                           moska_profiler* prof);

/*
 * moska_decode_step_fp8 (both stores in FP8, Section IV's precision) for a caller whose step inputs
 * live in HOST memory: q_host in, out_host out, the call returns when the result is there.  Copies,
 * their overlap with the step and the conditions on the host buffers are those of
 * moska_decode_step_host.
 */
int moska_decode_step_fp8_host(const uint16_t* q_host, uint16_t* q_dev, const float* summaries,
                               const uint8_t* k8_shared, const uint8_t* v8_shared,
                               const float* k_scale_shared, const float* v_scale_shared,
                               const uint8_t* k8_unique, const uint8_t* v8_unique,
                               const float* k_scale_unique, const float* v_scale_unique,
                               const int64_t* kv_start, const int32_t* kv_len, int32_t* topk_idx,
                               int32_t* seg_offsets, int32_t* seg_entries, float* o_part, float* lse_part,
                               uint16_t* out_dev, uint16_t* out_host, float softmax_scale,
                               const moska_shape* shape, void* ws, size_t ws_bytes, moska_stream stream,
                               moska_stream side_stream, moska_profiler* prof);

/* ---- a paged private store ------------------------------------------------------------------------
 * The private contexts of Section III-A in a pool of pages: a request's tokens live in the pages that
 * its row of the page table names, so a context grows a token at a time without moving.  Two storage
 * formats (n_pages, page_size and the table are the caller's; a page holds all KV heads):
 *
 *   MOSKA_KV_BF16  k_pages, v_pages bf16 [n_pages][page_size][Hkv][D]   (16-byte aligned)
 *   MOSKA_KV_FP4   k_pages uint8 [n_pages][Hkv][page_size / 16][18 D]   (16-byte aligned), v_pages
 *                  not read.  Keys and values as E2M1 codes (the 4-bit type of the tensor cores:
 *                  0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives) with one f16 scale per (token, KV
 *                  head, 32 dimensions): value = scale * e2m1(code), 4.5 bits an element.
 *
 * A block of 16 tokens of one KV head in the 4-bit format is 18 D bytes; token t of the block
 * (0..15), dimension d, an even dimension in the low half of its byte and d + 1 in the high half:
 *   keys          t (D/2) + ((d % 32) / 8) (D/8) + (d / 32) 4 + (d % 8) / 2
 *   values        8 D + (t/2) D + (x ^ s) (D/8) + (t % 2) (D/16) + (d % (D/8)) / 2,  x = d / (D/8),
 *                 s = 2 ((t/2) % 4) for D = 128, 4 ((t/4) % 2) for D = 64
 *   key scales    16 D + 2 (t (D/32) + d / 32)          (bytes; little-endian f16)
 *   value scales  17 D + 2 ((d / 32) 16 + t)
 * which is the order the attention kernel's lanes read: whole 16-byte (8-byte at D = 64) pieces,
 * eight different bank groups a quarter warp, without a shuffle.
 *
 * Context token t of request r is row t % page_size of page page_table[r][t / page_size].  Entries
 * behind the last page that a context reaches are not read.  A page index outside [0, n_pages), a
 * context longer than max_pages pages or a negative length raise MOSKA_ERR_INVALID_ARG in the device
 * status word: attention then reads page 0 (the pages that the row has, an empty context), appended
 * and gathered rows are left out, and the results of that call are not valid.  Two requests may share pages that only one
 * call at a time writes.
 */
enum { MOSKA_KV_BF16 = 0, MOSKA_KV_FP4 = 1 };

typedef struct moska_paged_kv {
    int32_t format;            /* MOSKA_KV_BF16 or MOSKA_KV_FP4                                    */
    int32_t page_size;         /* tokens per page: a power of two, 16..32768, at most 2^30 elements */
    int32_t n_pages;           /* pages in the pool, >= 1                                          */
    int32_t max_pages;         /* entries in a row of the page table, >= 1                         */
    void* k_pages;             /* keys, or the 4-bit pool (keys and values)                        */
    void* v_pages;             /* values; MOSKA_KV_FP4: not read, may be NULL                      */
    const int32_t* page_table; /* int32 [B / q_len, or n_requests][max_pages]                      */
    const int32_t* kv_len;     /* int32 [same]: context tokens, those that an append call of this
                                  step writes included; 0 = no context                             */
} moska_paged_kv;

/* Bytes of one pool tensor: of k_pages and of v_pages each (bf16), or of the one 4-bit pool. 0 if a
 * field is out of range.  Host only, pure. */
size_t moska_paged_pool_bytes(int32_t format, int32_t n_pages, int32_t page_size, int32_t Hkv, int32_t D);

/* A reasonable n_unique_splits for a paged store whose longest context has `max_len` tokens.  Host
 * only, pure. */
int moska_default_paged_splits(int32_t format, int32_t n_requests, int32_t Hkv, int32_t D, int32_t max_len);

/*
 * Appends new tokens to a paged store, with the position rotation applied on the way.  For every new
 * row: its key is rotated and written, its value is written, its queries are rotated into q_out.
 *   q, k, v     bf16, row i at q + i q_stride ([Hq][D] dense inside a row), k + i k_stride, v + i
 *               v_stride ([Hkv][D]); strides in elements, multiples of 8, >= the row; pointers
 *               16-byte aligned: the three may be columns of one projection's output.  q and q_out
 *               may both be NULL (keys and values only).
 *   positions   int32 [B], the rotation's position of row i, in [0, n_positions); a row outside is left
 *               out and raises MOSKA_ERR_INVALID_ARG in the device status word
 *   cos_sin     float [n_positions][rot_dim]: cos of the rot_dim / 2 angles, then their sin (16-byte
 *               aligned)
 *   rot_dim     leading dimensions that are rotated: a multiple of 16 up to D; 0 = no rotation
 *               (positions and cos_sin are not read, the queries are copied)
 *   interleaved 0: dimension p is paired with p + rot_dim / 2; 1: 2p with 2p + 1
 *   row_start   NULL: shape->B rows, shape->q_len (0 or 1 = one) for each of n_requests = B / q_len
 *               requests, in order.  Else int32 [n_requests + 1], ascending: request r has rows
 *               row_start[r] .. row_start[r+1] - 1; rows from row_start[n_requests] to B are padding.
 *   q_out       bf16 [B][Hq][D] (16-byte aligned)
 * Rows are read and written at once, in no order: q_out, the pools and the range from the first to the last
 * row of q, of k and of v may not overlap, but for q, k and v with one another.  A call where they do, or
 * whose k_pages and v_pages do, is refused.
 * With n_r rows, row i of request r becomes context token kv_len[r] - n_r + i: kv_len counts the
 * tokens after the call.  Where that is negative the row is padding.  For padding rows nothing is
 * written, q_out included (they keep what the buffer held).  The rotation is (a, b) -> (a cos - b sin, b cos + a sin) in fp32, each
 * product and sum rounded, the result rounded once to bf16, or to 4 bits: scale = f16(max|x| / 6) (at
 * most 10912), code = the E2M1 value nearest to x / scale, ties to the even code.  A NaN or an
 * infinity makes its 32 dimensions NaN.  Rows of one call must be different tokens; nothing outside
 * them is changed.  shape: B, Hq, Hkv, D and q_len are read.
 */
int moska_kv_append_paged(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride,
                          const uint16_t* v, int64_t v_stride, const int32_t* positions,
                          const float* cos_sin, int32_t n_positions, int32_t rot_dim,
                          int32_t interleaved, const int32_t* row_start, int32_t n_requests,
                          uint16_t* q_out, const moska_paged_kv* kv, const moska_shape* shape,
                          moska_stream stream);

/*
 * Reads the last rows of paged contexts back as bf16 (for the 4-bit format: the values that the codes
 * stand for, rounded to bf16), for instance to make a private context a chunk of the shared store.
 * Rows and requests as in moska_kv_append_paged: row i of request r is context token kv_len[r] - n_r
 * + i (kv->kv_len may be another array than the store's own lengths, to read an earlier range).
 * Padding rows are left as they were.
 *   k_out, v_out  bf16 [B][Hkv][D]   (16-byte aligned), overlapping neither one another nor the pools
 */
int moska_kv_gather_paged(const int32_t* row_start, int32_t n_requests, uint16_t* k_out, uint16_t* v_out,
                          const moska_paged_kv* kv, const moska_shape* shape, moska_stream stream);

/*
 * Unique KV Attention over a paged private store: the same partial results and slots as
 * moska_unique_attn.  With q_len > 1: q_len * G <= 16, and D = 128 for bf16.  Scores are summed in fp32,
 * softmax and row sums are fp32.  Held in 16 bits:
 *   bf16 format   P in bf16 (half a step: 2^-8)
 *   4-bit format  queries in f16, scaled by a power of two per row: exact down to 2^-17 of the row's largest
 *                 element, below that within 2^-25 of it; codes (exact); values as code * scale in f16 (2^-11,
 *                 or 2^-25 absolute below 2^-14; value scales above 10912, which append does not write, overflow);
 *                 P in f16 (2^-11; below 2^-21 of the row's largest within 2^-32 of that, so what is smaller
 *                 counts in the row sum alone)
 *   softmax_scale  finite, > 0
 */
int moska_unique_attn_paged(const uint16_t* q, const moska_paged_kv* kv, float* o_part, float* lse_part,
                            float softmax_scale, const moska_shape* shape, moska_stream stream);

/*
 * Attention of requests that have a paged private context and no shared store: the final rows,
 * without a separate merge.
 *   out      bf16  [B][Hq][D]   (16-byte aligned); a row without context is 0
 *   lse_out  float [B][Hq]      may be NULL; -inf for such a row
 *   ws       moska_paged_attn_workspace_bytes(shape) bytes, 256-byte aligned; calls that share it
 *            must not overlap.  Not read or written (may be NULL) with n_unique_splits = 1.
 * shape: B, Hq, Hkv, D, q_len and n_unique_splits are read.
 */
int moska_paged_attn(const uint16_t* q, const moska_paged_kv* kv, uint16_t* out, float* lse_out,
                     float softmax_scale, const moska_shape* shape, void* ws, size_t ws_bytes,
                     moska_stream stream);
size_t moska_paged_attn_workspace_bytes(const moska_shape* shape);

/*
 * moska_decode_step with a paged private store.  The shared store is bf16 (k_shared, v_shared bf16,
 * both scales NULL) or FP8 (E4M3 codes with k_scale_shared and v_scale_shared, as for
 * moska_shared_attn_fp8, D = 128).  Same schedule, buffers, outputs and error behaviour (summaries
 * NULL selects dense mode).
 */
int moska_decode_step_paged(const uint16_t* q, const float* summaries, const void* k_shared,
                            const void* v_shared, const float* k_scale_shared, const float* v_scale_shared,
                            const moska_paged_kv* kv, int32_t* topk_idx, int32_t* seg_offsets,
                            int32_t* seg_entries, float* o_part, float* lse_part, uint16_t* out,
                            float* lse_out, float softmax_scale, const moska_shape* shape, void* ws,
                            size_t ws_bytes, moska_stream stream, moska_stream side_stream,
                            moska_profiler* prof);

/* ---- speculative decoding over a paged private store -----------------------------------------------
 * A request's drafted tokens are a TREE.  Its nodes are consecutive batch rows, a parent before its
 * children; parents[row] is the index, within the request, of the parent of that row's node, -1 for
 * none.  Node 0 is the token that the last step sampled, the others are drafts.  The nodes' keys and values are
 * appended like any rows (moska_kv_append_paged, a node's position being its depth behind the committed
 * tokens), so that with T nodes they are context tokens kv_len[r] - T .. kv_len[r] - 1.  Then follow
 * attention (each node sees the committed tokens, its ancestors and itself), verification, and the
 * commit that keeps the accepted path's rows.
 *   row_start   NULL: shape->q_len nodes for each of n_requests = B / q_len requests.  Else int32
 *               [n_requests + 1], ascending: request r has rows row_start[r] .. row_start[r+1] - 1, at most
 *               shape->q_len (more raise MOSKA_ERR_INVALID_ARG in the device status word, and the first
 *               q_len count); rows from row_start[n_requests] to B are padding and left as they were.
 *   parents     int32 [B].  A value that is not in -1 .. i - 1 for node i raises MOSKA_ERR_INVALID_ARG in the
 *               device status word and counts as -1.  NULL (attention): a chain, node i under node i - 1.
 * q_len is 1 .. MOSKA_TREE_MAX_NODES in these calls (0 = 1).  A request whose kv_len is smaller than its
 * number of nodes is (partly) padding: nodes whose token index is negative hold nothing and see nothing.
 */
#define MOSKA_TREE_MAX_NODES 64

/*
 * Attention of the trees' nodes over the paged contexts that they end: final rows, both storage formats,
 * D = 64 and 128.
 *   q        bf16  [B][Hq][D]   (16-byte aligned)
 *   out      bf16  [B][Hq][D]   (16-byte aligned); a row that sees nothing is 0
 *   lse_out  float [B][Hq]      may be NULL; -inf for such a row
 *   ws       moska_tree_attn_workspace_bytes(shape) bytes (20 MB for D = 128), 256-byte aligned; calls that
 *            share it must not overlap.  Not read or written (may be NULL) with n_unique_splits = 1.
 * out, lse_out and ws may not overlap one another or what is read: the call is refused.
 * shape: B, Hq, Hkv, D, q_len and n_unique_splits are read: a context is cut into at most that many parts, as the
 * work of all contexts is shared among the SMs; 64 lets any batch be shared evenly, and costs no more than 2.  What a
 * node does not see has no influence on it, infinities and NaN included; a value that it sees and that is not finite makes that
 * dimension of its rows not finite.  Scores, softmax statistics, row sums and results
 * are held in fp32.  In 16 bits: bf16 pages, the probabilities (bf16, half a step 2^-8 of each); 4-bit pages, the
 * probabilities (f16, 2^-11; below 2^-21 of the row's largest within 2^-32 of that, so what is smaller counts in the row sum
 * alone) and a value as scale * code (f16, 2^-11, or 2^-25 absolute below 2^-14; above 65504, which takes a value scale above
 * the 10912 that append writes at most, it is infinite); keys are exact for every finite scale, as two bf16 numbers that add
 * up to scale * code, and so are the queries.  out is rounded once more.
 * A part of a context may take as long as it needs, but fp32 sums of very many tokens lose what is below their last bits: the
 * tensor cores cut off each product's bits below about 2^-25 of the sum.  With values of one sign and weights alike the result
 * of a part of 2^18 tokens is 0.03 % too small, of 2^20 0.4 %, of 2^22 2.3 % (a part of 4-bit pages up to 32 rows a
 * head: 0.02, 0.1, 0.6 %): cut such contexts (n_unique_splits).
 */
int moska_tree_attn(const uint16_t* q, const moska_paged_kv* kv, const int32_t* parents, const int32_t* row_start,
                    int32_t n_requests, uint16_t* out, float* lse_out, float softmax_scale, const moska_shape* shape,
                    void* ws, size_t ws_bytes, moska_stream stream);
size_t moska_tree_attn_workspace_bytes(const moska_shape* shape);

/* A reasonable n_unique_splits of moska_unique_attn_tree and the step below, for trees of up to `nodes` nodes
 * that end contexts of up to `max_len` tokens.  Host only, pure. */
int moska_default_tree_splits(int32_t n_requests, int32_t nodes, int32_t Hq, int32_t Hkv, int32_t max_len);

/* Unique KV Attention of trees of shape->q_len nodes each: the partial results and slots of
 * moska_unique_attn_paged, for a step that also attends to a shared store. */
int moska_unique_attn_tree(const uint16_t* q, const moska_paged_kv* kv, const int32_t* parents, float* o_part,
                           float* lse_part, float softmax_scale, const moska_shape* shape, moska_stream stream);

/* moska_decode_step_paged for trees of shape->q_len nodes each: the shared store is attended to by every
 * node as by a request of its own, the private context as in moska_tree_attn.  A request with fewer nodes has its rows filled
 * up with nodes behind them that no other node has above it (parent -1, any token): they are seen by themselves alone, and
 * moska_kv_commit_paged leaves them behind.  All runs on `stream`, one stage after another: attention of trees takes every SM, and
 * side_stream is not used. */
int moska_decode_step_tree(const uint16_t* q, const float* summaries, const void* k_shared,
                           const void* v_shared, const float* k_scale_shared, const float* v_scale_shared,
                           const moska_paged_kv* kv, const int32_t* parents, int32_t* topk_idx, int32_t* seg_offsets,
                           int32_t* seg_entries, float* o_part, float* lse_part, uint16_t* out,
                           float* lse_out, float softmax_scale, const moska_shape* shape, void* ws,
                           size_t ws_bytes, moska_stream stream, moska_stream side_stream,
                           moska_profiler* prof);

/*
 * Verification of drafted tokens against the target's probabilities, from given random numbers: the walk
 * down each tree that keeps the target's distribution.  With cur = 0, P = row cur of target_probs and Z = 1,
 * for the nodes j = 1, 2, .. whose parent is cur, in order, with x = tokens[j]:
 *   accepted if P(x) > 0 and u_accept[j] q Z < P(x), q = draft_probs[cur][x] (1 without draft_probs): cur = j,
 *   P = row j of target_probs, Z = 1; children of the new cur follow.  Else, with Q = row cur of draft_probs,
 *   P becomes max(P / Z - Q, 0) and Z its sum (both stay where that sum is 0); without draft_probs (a draft that
 *   was picked, not drawn) Z loses P(x) and P(x) becomes 0.
 * At the end next_token is the first v with P(0) + .. + P(v) > u_next[r] sum(P) and P(v) > 0 (the last v with
 * P(v) > 0 if there is none, -1 if P is 0 everywhere).  P, Z and the sums are held in 64 bits.
 *   target_probs  [B][V] of prob_type, row i (elements i target_stride ..) behind node i; entries that are
 *                 not > 0 (NaN included) count as 0, none is infinite
 *   draft_probs   the same, with draft_stride; row i is what the children of node i were drawn from, each on its
 *                 own from the whole row (with replacement): for siblings that were drawn to be different the walk
 *                 above does not keep the target's distribution.  May be NULL, for children that were picked
 *                 without chance (the likeliest ones, for instance)
 *   tokens        int32 [B]; a node whose token is not in [0, V) is not tried
 *   u_accept      float [B], u_next float [n_requests]: in [0, 1)
 *   path          int32 [n_requests][max_nodes]: the accepted nodes, 0 first, then -1
 *   n_path        int32 [n_requests]: how many (0 for a request without nodes, whose next_token is -1)
 *   next_token    int32 [n_requests]
 * B, row_start and max_nodes as B, row_start and q_len above.  The results may not overlap one another or the inputs.
 */
enum { MOSKA_PROB_F32 = 0, MOSKA_PROB_BF16 = 1 };
int moska_verify_tree(const void* target_probs, int64_t target_stride, const void* draft_probs, int64_t draft_stride,
                      int32_t prob_type, int32_t V, const int32_t* tokens, const int32_t* parents,
                      const float* u_accept, const float* u_next, const int32_t* row_start, int32_t n_requests,
                      int32_t max_nodes, int32_t B, int32_t* path, int32_t* n_path, int32_t* next_token,
                      moska_stream stream);

/*
 * Keeps the rows of accepted paths: with T nodes and c = kv_len[r] - T committed tokens, context token
 * c + path[r][j] is moved to c + j for every j < n_path[r], keys and values, as the bytes that they are, and
 * kv_len_out[r] = c + n_path[r] (what is behind it stays in the pages and counts no more).
 *   path        int32 [n_requests][path_stride], strictly ascending within n_path[r], each in [0, T)
 *   n_path      int32 [n_requests], 0 .. min(T, path_stride)
 *   kv_len_out  int32 [n_requests], apart from kv->kv_len
 * A path that is not so, a page outside the pool, a row range outside B or of more than q_len nodes, or a length that is
 * negative or more than max_pages pages hold, raises MOSKA_ERR_INVALID_ARG in the device status word; the request is left
 * as it was, kv_len_out[r] = kv_len[r].  The same, without an error, for a request with 0 <= kv_len[r] < T (padding).
 * Nodes' pages belong to one request alone.  shape: B, Hkv, D and q_len are read.
 */
int moska_kv_commit_paged(const int32_t* path, int32_t path_stride, const int32_t* n_path, const int32_t* row_start,
                          int32_t n_requests, int32_t* kv_len_out, const moska_paged_kv* kv, const moska_shape* shape,
                          moska_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* MOSKA_H_ */
