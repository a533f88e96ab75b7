/*
 * dblp.h -- C ABI of libdblp: the receive-side data path of the Dynamic Bounded-Loss Protocol (DBLP)
 * for W simulated workers whose gradients are resident on one CUDA device (sm_100a).
 *
 * One communication round is four steps:
 *
 *   dblp_packetize   gradients            -> header ring + payload ring      (Algorithm 1, first step)
 *   dblp_apply_loss  seeded loss process  -> delivered bitmap + arrival list (Sections II-C, V-B; property 1)
 *   dblp_aggregate   arrival list + rings -> received bitmap + aggregate     (Algorithm 2; Algorithm 3 "mean")
 *   dblp_check_bound received bitmap      -> per-worker loss counts, stop / continue decision (Section III-B)
 *
 * Each is a call of its own on the caller's stream.  dblp_round_device runs all four as one call and overlaps what is
 * independent: apply_loss (ALU-bound) beside packetize (HBM-bound), and the bitmap + tolerance test beside the masked
 * reduce, on a high-priority stream that the plan owns; dblp_round_host does the same from host buffers with the
 * copies overlapped.  Results are identical either way.
 *
 * Conventions
 *   - Every function returns DBLP_OK (0) or a negative dblp_status_t; nothing throws, aborts or traps.
 *     dblp_last_error() gives the text of the calling thread's most recent failure.
 *   - Unless an argument is marked HOST it is a DEVICE pointer owned by the caller, on the device that was
 *     current when the plan was created.  The library allocates device memory, streams and events only in
 *     dblp_plan_create.
 *   - Per-round calls only enqueue work on the given stream (a cudaStream_t passed as void*; NULL = the
 *     legacy default stream) and do not synchronise.  Counts that a later step needs stay on the device.
 *   - Anomalies found on the device (bad slot index, header that contradicts the plan, wrong round, repeated
 *     packet) are counted in dblp_counters_t and skipped; they never fault.
 *   - Alignment: ring and aggregate base pointers 16-byte aligned; payload_bytes a multiple of 16.
 *     Tensor sizes need no alignment (ragged edges take a scalar path).
 *   - Limits: W * C < 2^31 packets per round, ring slots < 2^32 - 1, payload_bytes <= 65536.
 */
#ifndef DBLP_H
#define DBLP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    DBLP_OK = 0,
    DBLP_EINVAL = -1,    /* null pointer, zero size, value out of range */
    DBLP_EALIGN = -2,    /* pointer or payload size not 16-byte aligned */
    DBLP_ECAPACITY = -3, /* a limit above is exceeded, or the workspace is too small */
    DBLP_ECUDA = -4,     /* a CUDA runtime call failed; text in dblp_last_error() */
    DBLP_ETIMEOUT = -5   /* reserved: waits inside kernels are bounded and counted, see dblp_wait_timeouts */
} dblp_status_t;

typedef enum { DBLP_F32 = 0, DBLP_BF16 = 1, DBLP_F16 = 2 } dblp_dtype_t; /* F16: worker-side operators only, not plans */
typedef enum { DBLP_LOSS_NONE = 0, DBLP_LOSS_IID = 1, DBLP_LOSS_GE = 2, DBLP_LOSS_MICROBURST = 3 } dblp_loss_kind_t;
enum { DBLP_SUM = 0, DBLP_MEAN = 1, DBLP_OUT_BF16 = 2 }; /* flags of dblp_aggregate; OUT_BF16 only with dblp_aggregate_reduce_ex */

/* Packet header, 32 bytes, stored beside (not inside) the payload.  seq, round and len_bytes are the paper's
 * three fields (Section IV-A); tensor_id and offset_elems are the id/offset tags of the prior work the paper
 * builds on (Section III-A), redundant with seq given the plan and verified against it on receipt; worker stands
 * for the per-worker UDP port (Section IV-D). */
typedef struct {
    uint32_t seq;          /* unique per (worker, round), 0 .. C-1 */
    uint32_t round;        /* communication round the packet was sent in */
    uint32_t len_bytes;    /* valid payload bytes (the last chunk of a tensor is short) */
    uint32_t tensor_id;    /* index into the plan's tensor list */
    uint64_t offset_elems; /* first element of the chunk inside its tensor */
    uint32_t worker;       /* 0 .. W-1 */
    uint32_t reserved;     /* written as 0 */
} dblp_hdr_t;

/* Loss process in integers: a packet's 32-bit draw u drops it iff u < threshold, thresholds in [0, 2^32].
 * The paper injects loss without naming a generator (Sections II-C, V-B); the processes are:
 *   IID         drop iff u0 < t_drop.
 *   MICROBURST  one window of window_len consecutive sequence numbers, the same for every worker;
 *               drop iff u0 < (inside ? t_drop_in : t_drop_out).
 *   GE          two-state chain per worker in seq order: starts Bad iff u_init < t_init_bad; drop iff
 *               u0 < (Bad ? t_drop_bad : t_drop_good); then Bad -> Good iff u1 < t_bg, Good -> Bad iff u1 < t_gb.
 * Draws are Philox4x32-10 with key = seed and counter = (id low, id high, stream | attempt << 8, round),
 * id = worker * C + seq. */
typedef struct {
    uint32_t kind; /* dblp_loss_kind_t */
    uint32_t pad;
    uint64_t t_drop;
    uint64_t t_gb, t_bg, t_init_bad;
    uint64_t t_drop_good, t_drop_bad;
    uint64_t window_len;
    uint64_t t_drop_in, t_drop_out;
} dblp_loss_model_t;

/* Receiver statistics of a round (device memory; all fields accumulate until dblp_round_reset).  n_accepted and n_dup
 * are settled by the bitmap step of the bookkeeping (dblp_aggregate_bitmap): between a dblp_aggregate_claim and its
 * dblp_aggregate_bitmap every valid packet of the call is still counted under n_dup. */
typedef struct {
    uint64_t n_arrived;  /* arrival-list entries examined */
    uint64_t n_accepted; /* packets whose bit was newly set */
    uint64_t n_dup;      /* valid packets of this round whose chunk had already arrived */
    uint64_t n_stale;    /* valid packets of another round (Section III-A: dropped) */
    uint64_t n_invalid;  /* slot outside the ring, or header contradicting the plan (Algorithm 2 integrity check) */
    uint64_t n_late;     /* valid packets of this round that came after their worker's receiver had stopped */
    uint32_t status;     /* bit 0: arrival numbers exceeded 32 bits */
    uint32_t pad;
} dblp_counters_t;

typedef struct dblp_plan dblp_plan_t;

/* ---- plan: the constants exchanged once before training (Section IV-A) -------------------------------------
 * tensor_numel (HOST, T values > 0): elements of each gradient tensor in flat order.  Chunking is per tensor:
 * tensor t yields ceil(n_t / E) chunks, E = payload_bytes / element size; C is their total.
 * bucket_seq_bounds (HOST, B+1 ascending sequence numbers from 0 to C, or NULL with B = 1): the ranges over
 * which dblp_check_bound counts; one bucket is the paper's single bitmap per worker stream.
 * Allocates the plan's device tables on the current device; *out is owned by the caller until dblp_plan_destroy. */
int dblp_plan_create(const uint64_t* tensor_numel, uint32_t T, int dtype, uint32_t payload_bytes, uint32_t W,
                     const uint64_t* bucket_seq_bounds, uint32_t B, dblp_plan_t** out);
int dblp_plan_destroy(dblp_plan_t* plan);
/* C = chunks per worker, N = elements per worker, M = W * C, row_words = ceil(C / 32) words per bitmap row.
 * Any out pointer may be NULL. */
int dblp_plan_query(const dblp_plan_t* plan, uint64_t* C, uint64_t* N, uint64_t* M, uint64_t* row_words);
/* Where packets live.  DBLP_WIRE_RINGS (default): a header ring of 32-byte entries and a payload ring of payload_bytes
 * entries.  DBLP_WIRE_DATAGRAMS: one ring of (32 + payload_bytes)-byte datagrams, header first, as a packet looks on
 * the wire (Section IV-B: chunk and header together fill the UDP payload); pass the ring's base as both hdr_ring and
 * payload_ring to every call.  Set before the first round; results do not depend on it. */
enum { DBLP_WIRE_RINGS = 0, DBLP_WIRE_DATAGRAMS = 1 };
int dblp_plan_set_wire_format(dblp_plan_t* plan, int format);
/* A server split over several devices (Section IV-D's server, sharded by offset range): each device owns a contiguous
 * run of the tensors with a plan of its own, whose packets are the chunks seq_offset .. seq_offset + C - 1 of worker
 * streams that are stream_chunks long in all.  After this call the loss process draws each packet's fate by its number
 * in the whole stream (and runs the burst chain and places the microburst window along the whole stream), so that the
 * shards' delivered bitmaps, side by side, are exactly the delivered bitmap of the unsplit round.  Headers, sequence
 * numbers and the arrival permutation stay local to the shard.  dblp_workspace_bytes grows by one stream-wide bitmap.
 * dblp_apply_loss_resend with a send set and DBLP_LOSS_GE is refused on such a plan (DBLP_EINVAL): the chain would need
 * the send set of the whole stream.  Call before the first round. */
int dblp_plan_set_shard(dblp_plan_t* plan, uint64_t stream_chunks, uint64_t seq_offset);
/* Expert knob: pins the launch shape of the masked reduce (dblp_aggregate_reduce) -- chunks summed per tile and
 * number of persistent blocks; 0 = choose automatically (what dblp_plan_create does).  Results do not depend on it.
 * DBLP_ECAPACITY if the tile's slot entries do not fit in shared memory.  Not to be called while work that uses the
 * plan is being enqueued from another thread. */
int dblp_plan_tune_reduce(dblp_plan_t* plan, uint32_t chunks_per_tile, uint32_t grid_blocks);
/* Bytes of scratch that dblp_apply_loss / dblp_apply_loss_resend need.  dblp_aggregate_book_stop has its own query
 * (dblp_stop_workspace_bytes); the remaining calls need none. */
int dblp_workspace_bytes(const dblp_plan_t* plan, size_t* bytes);

/* HOST helper: rates -> thresholds floor(prob * 2^32).  IID uses mean_loss.  GE is the simple Gilbert chain
 * (every packet sent in Bad is lost): P(Bad->Good) = 1 / mean_burst_len, P(Good->Bad) chosen so the stationary loss
 * is mean_loss, start state drawn from the stationary law; DBLP_EINVAL if that P(Good->Bad) would exceed 1 (the mean
 * loss cannot be reached with bursts that short).  MICROBURST: window_len = ceil(window_frac * C). */
int dblp_loss_model_from_rates(int kind, double mean_loss, double mean_burst_len, double window_frac, double p_in,
                               double p_out, uint64_t C, dblp_loss_model_t* out);

/* ---- packetize (Algorithm 1 "split data into chunks"; Sections IV-A, IV-B) ----------------------------------
 * grads: HOST array of W device pointers, each a flat gradient of N elements of the plan's dtype (element-aligned).
 * Writes M headers to hdr_ring and M payload slots of payload_bytes each to payload_ring; packet (w, seq) goes to
 * slot w * C + seq; bytes of a slot past len_bytes are written as zero.  Rings may hold more than M slots (the
 * rest is untouched). */
int dblp_packetize(const dblp_plan_t* plan, const void* const* grads, uint32_t round, dblp_hdr_t* hdr_ring,
                   void* payload_ring, void* stream);

/* ---- apply_loss: which packets survive, and in which order they arrive ---------------------------------------
 * model: HOST.  delivered_bits: W rows of row_words u32, bit (seq % 32) of word (seq / 32) set iff packet
 * (w, seq) survives; padding bits zero.  arrival: capacity M u32; receives the surviving slot numbers in the order
 * pi(0), pi(1), ... where pi is a seeded permutation of [0, M) (4-round Feistel network on the smallest even
 * number of bits covering M, cycle-walked; round function = one Philox draw).  *n_arrived_dev (u64) = their count.
 * ws: scratch of at least dblp_workspace_bytes(); contents need not be preserved between calls. */
int dblp_apply_loss(const dblp_plan_t* plan, const dblp_loss_model_t* model, uint64_t seed, uint32_t round,
                    uint32_t attempt, uint32_t* delivered_bits, uint32_t* arrival, uint64_t* n_arrived_dev, void* ws,
                    size_t ws_bytes, void* stream);

/* ---- retransmission attempts (Algorithm 1: "for each unsent chunk ... send"; Section III-B: the sender retransmits
 * from the most recent bitmap) -------------------------------------------------------------------------------------
 * dblp_missing_bits: sent_bits <- the chunks whose bit is 0 in recv_bitmap (padding bits stay 0): what a sender
 * transmits after a bitmap reply.  Same layout as the bitmaps.
 * dblp_apply_loss_resend: dblp_apply_loss restricted to the chunks in sent_bits (NULL = all, which is
 * dblp_apply_loss): a chunk that is not sent cannot arrive, and the burst chain, which models the channel while
 * packets cross it, advances only over the packets that are sent.  Draws are keyed by (packet id, attempt), so the
 * fate of a sent packet under a memoryless process does not depend on what else is sent. */
int dblp_missing_bits(const dblp_plan_t* plan, const uint32_t* recv_bitmap, uint32_t* sent_bits, void* stream);
int dblp_apply_loss_resend(const dblp_plan_t* plan, const dblp_loss_model_t* model, uint64_t seed, uint32_t round,
                           uint32_t attempt, const uint32_t* sent_bits, uint32_t* delivered_bits, uint32_t* arrival,
                           uint64_t* n_arrived_dev, void* ws, size_t ws_bytes, void* stream);

/* ---- apply_loss without any allocation (the paper has no counterpart: this entry point exists for the sake of
 * callers, not of the protocol) ---------------------------------------------------------------------------------
 * Same results as dblp_apply_loss, bit for bit, but the scratch is a fixed array inside the library's own device
 * image instead of a caller-provided workspace.  It is meant for callers that hold no allocator for device memory
 * and must not call one: code running inside a memory pool whose owner forbids side allocations, plug-ins loaded
 * into a host process that has already handed all device memory to another runtime, and hard real-time loops where
 * an allocation's latency (or its implicit device synchronisation) is not acceptable.  Inputs and outputs are still
 * the caller's buffers.
 *   - Limit: the plan's dblp_workspace_bytes() must not exceed DBLP_STATIC_SCRATCH_BYTES (4 MiB + 64 KiB, i.e.
 *     roughly W * C <= 2^20 packets per round); larger plans get DBLP_ECAPACITY and a message naming both sizes.
 *   - Cost: every GPU on which the library is loaded keeps those bytes reserved until the process exits.
 *   - The first call on a device looks up the array's device address (one cudaGetSymbolAddress, no allocation) and
 *     caches it; make that first call before starting any stream capture on that device.  The plan's device must be
 *     the current device.
 *   - All calls on a device share the one array.  Nothing in it has to start at zero (each pass overwrites what the
 *     next reads), but two calls whose kernels overlap on the GPU -- different streams, or different host threads
 *     without ordering between them -- race on it.  Order them on one stream or with events.
 *   - Calls no cudaMalloc, cudaFree or other allocating routine. */
#define DBLP_STATIC_SCRATCH_BYTES (4u * 1024u * 1024u + 64u * 1024u)
int dblp_apply_loss_static(const dblp_plan_t* plan, const dblp_loss_model_t* model, uint64_t seed, uint32_t round,
                           uint32_t attempt, uint32_t* delivered_bits, uint32_t* arrival, uint64_t* n_arrived_dev,
                           void* stream);

/* ---- aggregate = bookkeeping + masked reduce ------------------------------------------------------------------
 * dblp_aggregate_book (Algorithm 2, chunk branch; Section III-A round filter): examines arrival[0 .. *n_arrived_dev)
 * (at most arrival_cap entries).  An entry is invalid if its slot >= n_slots or its header contradicts the plan
 * (worker < W, tensor_id < T, offset on a chunk boundary inside the tensor, len_bytes = that chunk's length,
 * seq = that chunk's number); stale if header.round != round; otherwise it claims cell (worker, seq) of slot_key.
 * slot_key: W * C u64, all-ones = nothing arrived yet, else (arrival number << 32) | slot; the claim is an atomic
 * minimum, so the earliest arrival keeps the cell whatever order threads run in, and later ones count as n_dup.
 * Arrival numbers continue from counters->n_arrived, so a further call in the same round (a retransmission
 * attempt) never displaces an earlier packet.  recv_bitmap (W rows of row_words u32) is rewritten from slot_key.
 *
 * dblp_aggregate_reduce (Algorithm 2 "unreceived chunks remain 0-filled / reconstruct"; Algorithm 3 mean): for
 * every element i of chunk c:  agg[i] = (+0.0f + x_0 + x_1 + ...) over the workers w = 0 .. W-1, in that order,
 * whose cell (w, c) is claimed, x_w read from the claimed payload slot (bf16 widened exactly), plain fp32
 * additions; with DBLP_MEAN the sum is divided by (float)W -- all workers, not the number that arrived.
 * The destination is the plan's (tensor base + chunk offset), never the slot's position.  agg_out: N fp32.
 *
 * dblp_aggregate runs both.  slot_key, recv_bitmap and counters are in/out round state (dblp_round_reset). */
/* dblp_aggregate_book = dblp_aggregate_claim (examine the arrivals, claim cells, count stale and invalid ones) followed
 * by dblp_aggregate_bitmap (rewrite recv_bitmap from slot_key; the bits that are new are the packets accepted by this
 * call, the other valid ones were repeats; fold this call's arrival count into counters->n_arrived).  recv_bitmap must
 * be the round's bitmap as the previous bookkeeping call (or dblp_round_reset) left it.
 * The reduce needs only the claims, the tolerance test only the bitmap, so a caller with two streams can run the
 * bitmap and dblp_check_bound beside dblp_aggregate_reduce.  Call dblp_aggregate_bitmap exactly once after each
 * dblp_aggregate_claim, with the same n_arrived_dev and arrival_cap, before the round's next claim. */
int dblp_aggregate_claim(const dblp_plan_t* plan, const dblp_hdr_t* hdr_ring, uint64_t n_slots, const uint32_t* arrival,
                         const uint64_t* n_arrived_dev, uint64_t arrival_cap, uint32_t round, uint64_t* slot_key,
                         dblp_counters_t* counters, void* stream);
/* dblp_aggregate_claim_grouped: the same claims with the same results (claim table and counters are identical), made
 * in a cheaper order for rounds whose headers and claim table do not fit in L2.  The arrival list is first grouped by
 * slot range (a counting sort in three small passes into (position, slot) pairs in ws), then the claims are made range
 * by range, so that the headers and cells they touch stay in L2 instead of costing two random DRAM sectors per packet;
 * a packet's arrival number travels with it, so "first arrival wins" is unchanged.  On 12 M packets the claim stage
 * drops from 0.53 to 0.29 ms; below about 3 M packets the plain order is the faster one.
 * dblp_aggregate_claim chooses by itself: a plan whose headers and claim table exceed the L2 owns a scratch of
 * dblp_claim_workspace_bytes(M, M) bytes (allocated in dblp_plan_create, 8 bytes per packet) and groups every call
 * with n_slots <= M and arrival_cap <= M; such a plan serves one claim at a time.  This entry point is for callers who
 * want the grouping elsewhere or with a scratch of their own.  ws: dblp_claim_workspace_bytes(n_slots, arrival_cap)
 * bytes, 256-byte aligned, contents need not be preserved. */
int dblp_claim_workspace_bytes(const dblp_plan_t* plan, uint64_t n_slots, uint64_t arrival_cap, size_t* bytes);
int dblp_aggregate_claim_grouped(const dblp_plan_t* plan, const dblp_hdr_t* hdr_ring, uint64_t n_slots,
                                 const uint32_t* arrival, const uint64_t* n_arrived_dev, uint64_t arrival_cap,
                                 uint32_t round, uint64_t* slot_key, dblp_counters_t* counters, void* ws, size_t ws_bytes,
                                 void* stream);
int dblp_aggregate_bitmap(const dblp_plan_t* plan, const uint64_t* slot_key, const uint64_t* n_arrived_dev,
                          uint64_t arrival_cap, uint32_t* recv_bitmap, dblp_counters_t* counters, void* stream);
int dblp_aggregate_book(const dblp_plan_t* plan, const dblp_hdr_t* hdr_ring, uint64_t n_slots, const uint32_t* arrival,
                        const uint64_t* n_arrived_dev, uint64_t arrival_cap, uint32_t round, uint32_t* recv_bitmap,
                        uint64_t* slot_key, dblp_counters_t* counters, void* stream);
int dblp_aggregate_reduce(const dblp_plan_t* plan, const void* payload_ring, const uint64_t* slot_key, float* agg_out,
                          uint32_t flags, void* stream);

/* ---- masked reduce with fused extras ---------------------------------------------------------------------------------
 * dblp_aggregate_reduce plus, in the same pass over the data:
 *   norm (Eq. 1 needs the L2 norm of the aggregated gradient): norm_out[0] = sum of agg[i]^2 in fp64, norm_out[1] = its
 *     square root.  Squares of fp32 values are exact in fp64; the additions follow a fixed tree (per thread, warp
 *     shuffle, warps in order, tiles in a fixed order), so the result is reproducible for a given plan and within
 *     about 64 ulp of the exactly rounded sum.  norm_scratch: dblp_norm_scratch_count() doubles (changes when
 *     dblp_plan_tune_reduce changes the tile height).  Both NULL = off.
 *   update (Algorithm 4, worker: w <- w - alpha * g): params[i] = params[i] - lr * agg[i], an fp32 multiply then an
 *     fp32 subtract (no fused multiply-add), for every element; chunks nobody delivered leave params unchanged because
 *     their aggregate is +0.  params: N fp32, in/out.  NULL = off.
 *   bf16 output (flag DBLP_OUT_BF16, may be or-ed with DBLP_MEAN): agg_out is N bf16 values, each the fp32 result
 *     rounded to nearest even (NaN stays a quiet NaN); norm and update still use the fp32 value.
 * For the broadcast half of a round (Algorithm 3 "DBLP_SEND(mean)", Algorithm 4 "DBLP_RECV"), packetize the mean with a
 * W = 1 plan, apply loss, book, and call this with params: the worker's reconstruction and its update in one pass. */
int dblp_norm_scratch_count(const dblp_plan_t* plan, uint64_t* count);
int dblp_aggregate_reduce_ex(const dblp_plan_t* plan, const void* payload_ring, const uint64_t* slot_key, float* agg_out,
                             uint32_t flags, double* norm_scratch, double* norm_out, float* params, float lr,
                             void* stream);

/* ---- order-free reduce (property 1: "gradients should be applied as soon as they arrive") --------------------------
 * Same inputs and the same mathematical result as dblp_aggregate_reduce, but every received payload is added into the
 * aggregate with floating-point atomics in whatever order the hardware runs them, so the fp32 sums are not
 * reproducible bit for bit: each element is within (W - 1) * 2^-24 * sum_w |x_w| of the exact sum.  Provided to measure
 * what the fixed worker order costs; zeroes agg_out first, and scales by 1 / W in a second pass for DBLP_MEAN. */
int dblp_aggregate_reduce_atomic(const dblp_plan_t* plan, const void* payload_ring, const uint64_t* slot_key,
                                 float* agg_out, uint32_t flags, void* stream);

/* ---- bookkeeping with early stop (Algorithm 2, the branch without a probe: "if the loss-tolerance threshold is
 * satisfied, send stop") ------------------------------------------------------------------------------------------
 * As dblp_aggregate_book, but each worker's receiver stops the moment its own missing / C <= bound_ppm / 10^6 holds
 * (one bitmap per worker stream): of a worker's valid packets of this round, taken in arrival order, only those up
 * to and including the one that satisfies the threshold are booked; the rest count as n_late and leave no trace.
 * Integrity and round checks come first, as for a running receiver.  The result equals a sequential walk over the
 * arrival list.  Needs W <= 4096 and a workspace of dblp_stop_workspace_bytes(arrival_cap) bytes, 256-byte aligned. */
int dblp_stop_workspace_bytes(const dblp_plan_t* plan, uint64_t arrival_cap, size_t* bytes);
int dblp_aggregate_book_stop(const dblp_plan_t* plan, const dblp_hdr_t* hdr_ring, uint64_t n_slots,
                             const uint32_t* arrival, const uint64_t* n_arrived_dev, uint64_t arrival_cap,
                             uint32_t round, uint32_t bound_ppm, uint32_t* recv_bitmap, uint64_t* slot_key,
                             dblp_counters_t* counters, void* ws, size_t ws_bytes, void* stream);
int dblp_aggregate(const dblp_plan_t* plan, const dblp_hdr_t* hdr_ring, const void* payload_ring, uint64_t n_slots,
                   const uint32_t* arrival, const uint64_t* n_arrived_dev, uint64_t arrival_cap, uint32_t round,
                   uint32_t* recv_bitmap, uint64_t* slot_key, dblp_counters_t* counters, float* agg_out,
                   uint32_t flags, void* stream);

/* Start of a round (Algorithm 2: bitmap <- 0): recv_bitmap <- 0, slot_key <- all-ones, counters <- 0. */
int dblp_round_reset(const dblp_plan_t* plan, uint32_t* recv_bitmap, uint64_t* slot_key, dblp_counters_t* counters,
                     void* stream);

/* ---- check_bound (Section III-B: stop once missing / total <= p; Algorithm 2: stop signal or bitmap reply) ----
 * For each worker w and bucket b: recv_cnt[w*B+b] = set bits of row w over the bucket's sequence range,
 * missing_cnt = total - recv_cnt, ok = (missing * 10^6 <= bound_ppm * total) in 64-bit integers;
 * *all_ok = 1 iff every ok is 1.  bound_ppm: HOST, n_bounds = 1 (one tolerance for all) or B (per bucket), in parts
 * per million (Table I: 0.8 % = 8000).  Outputs: recv_cnt, missing_cnt u32[W*B], ok u8[W*B], all_ok u32[1].
 * A plan serves one dblp_check_bound at a time (calls on one stream, or ordered by events). */
int dblp_check_bound(const dblp_plan_t* plan, const uint32_t* recv_bitmap, const uint32_t* bound_ppm,
                     uint32_t n_bounds, uint32_t* recv_cnt, uint32_t* missing_cnt, uint8_t* ok, uint32_t* all_ok,
                     void* stream);

/* HOST, pure: the rule above for counts summed over several shards of one worker stream (each GPU of a sharded server
 * counts its own chunk range): 1 iff missing * 10^6 <= bound_ppm * total.  Counts below 2^43 cannot overflow. */
int dblp_bound_ok(uint64_t missing, uint64_t total, uint32_t bound_ppm);

/* ---- phase-aware tolerance (HOST, pure) ----------------------------------------------------------------------
 * dblp_clr: Eq. 1, |norm_prev - norm_curr| / norm_prev >= eta in fp64; norm_prev == 0 counts as critical.
 * dblp_select_bound: Section IV-D / Algorithm 3: the first iteration uses P_low; at the start of an epoch the
 * tolerance becomes P_high unless dblp_clr fires, then P_low; at any other iteration it stays current_ppm. */
int dblp_clr(double norm_prev, double norm_curr, double eta);
uint32_t dblp_select_bound(double norm_prev, double norm_curr, double eta, uint32_t p_low_ppm, uint32_t p_high_ppm,
                           int at_epoch_start, int first_iteration, uint32_t current_ppm);

/* ---- whole rounds ---------------------------------------------------------------------------------------------------
 * The device buffers of a round, all allocated by the caller with the sizes given. */
typedef struct {
    void* grads;               /* W * N elements of the plan's dtype, worker-major; dblp_round_host only */
    dblp_hdr_t* hdr_ring;      /* M headers */
    void* payload_ring;        /* M * payload_bytes */
    uint32_t* delivered_bits;  /* W * row_words */
    uint32_t* arrival;         /* M */
    uint64_t* n_arrived;       /* 1 */
    uint32_t* recv_bitmap;     /* W * row_words */
    uint64_t* slot_key;        /* W * C */
    dblp_counters_t* counters; /* 1 */
    float* agg;                /* N */
    uint32_t* recv_cnt;        /* W * B */
    uint32_t* missing_cnt;     /* W * B */
    uint8_t* ok;               /* W * B */
    uint32_t* all_ok;          /* 1 */
    void* ws;                  /* dblp_workspace_bytes (max with dblp_stop_workspace_bytes(M) for dblp_round_until_stop) */
    size_t ws_bytes;
    uint32_t* sent_bits;       /* W * row_words; used by dblp_round_until_stop only */
} dblp_device_buffers_t;

/* Optional stage marks: CUDA events (cudaEvent_t passed as void*, created by the caller) that a whole-round call
 * records where a stage begins or ends, on the stream that runs the stage, so that a caller can time the stages of the
 * overlapped schedule.  NULL members are skipped; a NULL struct pointer means no marks. */
typedef struct {
    void* begin;          /* caller's stream, before anything */
    void* packetize_end;  /* caller's stream */
    void* loss_begin;     /* side stream: round_reset + apply_loss */
    void* loss_end;
    void* receive_begin;  /* caller's stream, once packetize and apply_loss have both finished */
    void* claim_end;      /* caller's stream: arrivals examined, cells claimed */
    void* reduce_end;     /* caller's stream */
    void* bound_begin;    /* side stream: bitmap + check_bound */
    void* bound_end;
    void* end;            /* caller's stream, after the side stream has been joined */
} dblp_round_marks_t;

/* dblp_round_device = one round of the server on gradients resident in device memory (Algorithm 3: receive from
 * every worker, then the mean; Algorithm 2 inside; Section III-B for the tolerance test):
 *   dblp_round_send     round_reset and apply_loss (attempt 0) on the plan's side stream beside dblp_packetize on the
 *                       caller's stream; returns with the caller's stream waiting for both.
 *   dblp_round_receive  dblp_aggregate_claim, then dblp_aggregate_bitmap + dblp_check_bound (one tolerance for all) on
 *                       the side stream beside dblp_aggregate_reduce; the caller's stream waits for both at the end.
 * grads: HOST array of W device pointers as for dblp_packetize.  flags: DBLP_SUM or DBLP_MEAN.  Packets occupy ring slots
 * 0 .. M-1.  Nothing is allocated and the host is not blocked.  The side stream and its events belong to the plan, so a
 * plan serves one whole-round call at a time (calls on one stream, or ordered by the caller). */
int dblp_round_send(const dblp_plan_t* plan, const void* const* grads, const dblp_loss_model_t* model, uint64_t seed,
                    uint32_t round, const dblp_device_buffers_t* dev, const dblp_round_marks_t* marks, void* stream);
int dblp_round_receive(const dblp_plan_t* plan, uint32_t round, uint32_t bound_ppm, uint32_t flags,
                       const dblp_device_buffers_t* dev, const dblp_round_marks_t* marks, void* stream);
int dblp_round_device(const dblp_plan_t* plan, const void* const* grads, const dblp_loss_model_t* model, uint64_t seed,
                      uint32_t round, uint32_t bound_ppm, uint32_t flags, const dblp_device_buffers_t* dev,
                      const dblp_round_marks_t* marks, void* stream);

/* dblp_round_host = the same round from HOST gradients (grads_host: HOST array of W host pointers, pinned memory
 * recommended).  Gradients of 32 MiB per worker and more are taken in up to 16 parts, contiguous ranges of chunks: the
 * host-to-device copies into dev->grads run back to back on a copy stream of the plan, part by part and worker by
 * worker; each slice is packetized as soon as it has landed; once a part is there for all workers its packets are
 * claimed, its chunks reduced, and its range of the aggregate starts back to agg_host on another stream of the plan,
 * so the copy back overlaps the copies in of the later parts.  The loss process runs beside all of it, the bitmap and
 * the tolerance test after the last claims.  Results are those of dblp_round_device.  The aggregate, the counters and
 * the bound outputs are copied back to the host pointers (NULL to skip) and the call waits for all of it.  Nothing is
 * allocated. */
int dblp_round_host(const dblp_plan_t* plan, const void* const* grads_host, const dblp_loss_model_t* model,
                    uint64_t seed, uint32_t round, uint32_t bound_ppm, uint32_t flags,
                    const dblp_device_buffers_t* dev, float* agg_host, dblp_counters_t* counters_host,
                    uint32_t* recv_cnt_host, uint32_t* missing_cnt_host, uint8_t* ok_host, uint32_t* all_ok_host,
                    void* stream);

/* ---- one round's control loop (Algorithms 1 + 2 together; HOST-blocking) ----------------------------------------------
 * After dblp_round_reset and dblp_packetize: attempt k = 0, 1, ... transmits what the bitmap reports missing
 * (dblp_missing_bits), redraws loss and arrival order with the attempt number (dblp_apply_loss_resend), books the
 * arrivals (dblp_aggregate_book, or dblp_aggregate_book_stop when early_stop != 0) and tests the tolerance
 * (dblp_check_bound, one value for all).  The decision is read back after every attempt -- the protocol's
 * probe / bitmap / stop exchange is a round trip -- and the loop ends when every worker passes or after max_attempts.
 * Packets are read from ring slots 0 .. M-1.  *attempts_used and *all_ok_host are HOST outputs.  The masked reduce is
 * left to the caller (dblp_aggregate_reduce). */
int dblp_round_until_stop(const dblp_plan_t* plan, const dblp_loss_model_t* model, uint64_t seed, uint32_t round,
                          uint32_t bound_ppm, uint32_t max_attempts, int early_stop, const dblp_device_buffers_t* dev,
                          uint32_t* attempts_used, uint32_t* all_ok_host, void* stream);

/* ---- worker side: operators of the training step whose gradients a round carries -----------------------------------
 * Algorithm 4 (worker): compute the gradient, send it, receive the mean, update.  These calls compute pieces of that
 * gradient for token models: the embedding table and its gradient, dropout, attention and its gradient.  They need no
 * plan; they run on the current device, whose memory all device pointers are in, allocate nothing, only enqueue work
 * on the given stream, and the order of every floating-point addition is fixed by the arguments, so results repeat bit for bit.
 * Calls can be captured in a graph; make a call of each kind once on a device before (it looks up symbols and sets limits).
 * dtype arguments are dblp_dtype_t; strides are in elements and may be anything that keeps rows apart (inputs may also
 * repeat: stride 0).  Zero-sized calls return DBLP_OK without touching memory. */

/* dblp_embed: out[i, :] = scale * table[tokens[i], :], an fp32 multiply rounded once to out_dtype.
 * table: rows x width, row stride table_stride.  tokens: n ids of token_bytes (4 or 8) bytes each, signed.  out: n rows,
 * row stride out_stride.  A token equal to `padding` (any value outside [0, rows) = no padding id) gives a zero row.  A
 * token outside [0, rows) gives a zero row too, whatever `padding` is, and is counted in *bad_tokens (u64, device,
 * accumulates; NULL = not counted); it never faults. */
int dblp_embed(const void* table, int64_t table_stride, uint64_t rows, uint32_t width, int table_dtype,
               const void* tokens, uint32_t token_bytes, uint64_t n, int64_t padding, float scale, void* out,
               int64_t out_stride, int out_dtype, uint64_t* bad_tokens, void* stream);

/* dblp_embed_grad: the table's gradient, dense.  For every row v
 *     dtable[v, :] = round(scale * sum of dout[i, :] over the i with tokens[i] = v, ascending [+ dtable[v, :]])
 * The sum is in fp32: the occurrences of all tokens, sorted by (token, i), are cut into tiles of 32; inside a tile a
 * row's terms are added one after the other, and a row that spans several tiles adds their partial sums in tile order
 * (from 17 partial sums on in 8 contiguous parts, joined in order).  Rows that no token names are written as zero.
 * flags: DBLP_ACCUMULATE adds to what dtable holds (rows that no token names are not touched), e.g. the output layer's
 * gradient of a tied table.  Padding and bad tokens contribute nothing (bad_tokens as above).
 * ws: dblp_embed_grad_workspace_bytes() bytes, 256-byte aligned, contents need not be preserved.  n < 2^31, rows < 2^31. */
enum { DBLP_ACCUMULATE = 1 };
int dblp_embed_grad_workspace_bytes(uint64_t n, uint64_t rows, uint32_t width, size_t* bytes);
int dblp_embed_grad(const void* dout, int64_t dout_stride, int dout_dtype, const void* tokens, uint32_t token_bytes,
                    uint64_t n, int64_t padding, float scale, void* dtable, int64_t dtable_stride, uint64_t rows,
                    uint32_t width, int dtable_dtype, uint32_t flags, uint64_t* bad_tokens, void* ws, size_t ws_bytes,
                    void* stream);

/* dblp_dropout: out = dropout(x) [+ residual], rows x cols, each with a row stride of its own; out may be x or residual.
 * Element i = row * cols + col (whatever the strides) draws 16 bits: group i / 8 is one Philox4x32-10 draw with key =
 * seed and counter = (group low, group high, 5 | site << 8, step), element i takes half i % 2 (low first) of word
 * (i % 8) / 2.  It is dropped iff its bits are below t = floor(p * 65536); a kept element is scaled by
 * 65536 / (65536 - t), the inverse of the share that is really kept, so the expectation is exact for every p.  The mask
 * is never stored: dblp_dropout_grad draws it again.  p in [0, 1] (1 drops everything), site < 2^24; (seed, step, site)
 * names a mask: site tells the dropouts of one training step apart.  residual NULL = none.  The product and the sum are
 * fp32 (two roundings), the result is rounded once more to dtype. */
int dblp_dropout(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, void* out,
                 int64_t out_stride, uint64_t rows, uint32_t cols, int dtype, double p, uint64_t seed, uint32_t step,
                 uint32_t site, void* stream);
/* dx = the gradient of x given dout (the residual's gradient is dout itself).  dx may be dout. */
int dblp_dropout_grad(const void* dout, int64_t dout_stride, void* dx, int64_t dx_stride, uint64_t rows, uint32_t cols,
                      int dtype, double p, uint64_t seed, uint32_t step, uint32_t site, void* stream);

/* Heads of a [batch, token, head, head_dim] tensor; the head_dim elements of a head are contiguous.  Data and strides
 * (in elements; unused where the extent is 1) are multiples of 16 bytes.  Strides are not negative; inputs may have stride 0 over batch
 * or heads (broadcast); the sections of outputs must not overlap. */
typedef struct {
    void* data;
    int64_t batch_stride, token_stride, head_stride;
} dblp_heads_t;

enum { DBLP_ATTENTION_CAUSAL = 1 };
typedef struct {
    uint32_t batch, q_tokens, k_tokens; /* extents of the tensors */
    uint32_t q_heads, kv_heads;         /* kv_heads divides q_heads; query head h reads key head h / (q_heads / kv_heads) */
    uint32_t head_dim;                  /* a multiple of 8, at most 128 */
    int dtype;                          /* DBLP_BF16 or DBLP_F16 */
    uint32_t flags;                     /* 0 or DBLP_ATTENTION_CAUSAL */
    float scale;                        /* of the scores, usually 1 / sqrt(head_dim); finite, > 0 */
    const int32_t* q_lens;              /* device, [batch]: tokens that count in each sequence; NULL = all.  Values are */
    const int32_t* k_lens;              /* clamped to the extents; what lies beyond is never used, NaN included */
} dblp_attention_t;

/* dblp_attention, per sequence and head, with lq = q_lens[b] and lk = k_lens[b]:
 *     s_ij = scale * <q_i, k_j>,  i < lq, j < lk, with DBLP_ATTENTION_CAUSAL also j <= i + lk - lq (the last query
 *                                 sees every key)
 *     lse_i = log sum_j exp(s_ij),  out_i = sum_j exp(s_ij - lse_i) v_j
 * A query that sees no key or lies beyond lq gets out = 0 and lse = -infinity and has no part in any gradient, whatever its q
 * and dout hold; so does one with finite q and dout that has no score above -infinity.  A score of NaN or +infinity makes its
 * row of out NaN, and its gradients.  What is not finite can, as 0 * NaN, reach more than the formulas say where only the
 * causal mask is between: v_j the rows of out before j, q_i and dout_i the gradients of keys after i.
 * lse: fp32 [batch, q_heads, q_tokens], contiguous (NULL = not wanted).
 * dblp_attention_grad: with D_i = <dout_i, out_i>, p_ij = exp(s_ij - lse_i) computed again from q, k and lse,
 *     ds_ij = p_ij (<dout_i, v_j> - D_i),  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,
 *     dv_j = sum_i p_ij dout_i;  shared key heads sum over their query heads.
 * p_ij is computed from s_ij and lse_i in fp32, so it is off by about 2^-22 |lse_i| of itself: below 0.1 % up to |lse| = 4000, and
 * of no use from about 10^6 on (the forward pass holds for any size of scores).
 * out and lse are dblp_attention's for the same arguments.  Every element of dq, dk and dv is written (zero where
 * nothing contributes).  Scores, statistics and accumulators are fp32; p and ds are rounded to dtype where they enter a
 * product.
 * With DBLP_F16, p or ds below 2^-25 vanishes where it is rounded: scale the loss so that dout is not tiny.
 * ws: dblp_attention_workspace_bytes() bytes (fwd for dblp_attention, grad for dblp_attention_grad; either may be 0),
 * 256-byte aligned, contents need not be preserved.  The gradient's holds 8 bytes a query row and 1 to 32 copies of dq in
 * fp32, head_dim rounded up to 64 or 128: one a share of the keys, as many as make the heads fill the device; where query heads
 * share key heads also up to q_heads / kv_heads copies of dk and dv.  (1 sequence, 8192 tokens, 16 heads on 4 of 128: 672 MB; 131072
 * tokens, 8 heads of 128: 9.7 GB.) */
int dblp_attention_workspace_bytes(const dblp_attention_t* a, size_t* fwd_bytes, size_t* grad_bytes);
int dblp_attention(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                   const dblp_heads_t* out, float* lse, void* ws, size_t ws_bytes, void* stream);
int dblp_attention_grad(const dblp_attention_t* a, const dblp_heads_t* q, const dblp_heads_t* k, const dblp_heads_t* v,
                        const dblp_heads_t* out, const dblp_heads_t* dout, const float* lse, const dblp_heads_t* dq,
                        const dblp_heads_t* dk, const dblp_heads_t* dv, void* ws, size_t ws_bytes, void* stream);

/* dblp_norm_rotate: what stands between a projection and dblp_attention.  For every token and head of q, and of k,
 *     r = 1 / sqrt(mean of x_i^2 over the head's head_dim elements + eps),  y_i = x_i r weight_i
 * and the first rotary_dim columns of y are turned, pair by pair: pair i (i < rotary_dim / 2) is columns (i, i +
 * rotary_dim / 2), with DBLP_ROTATE_INTERLEAVED columns (2 i, 2 i + 1), and
 *     (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = position * freqs[i].
 * The angle is a 64-bit product reduced to one turn before it is rounded, so far positions lose nothing; the rest is fp32,
 * rounded once.  The squares of a head must not add up beyond fp32 (elements up to about 10^18).  Heads are as for
 * dblp_attention (data and strides multiples of 16 bytes); q_out may be q and k_out may be k (the same data and strides); nothing of
 * q lies over anything of k where either is written.
 * dblp_norm_rotate_grad: with d = the gradient of the output turned back by -t,
 *     dx_i = r weight_i d_i - x_i r^3 / head_dim * sum_j weight_j d_j x_j,  dweight_i = sum over tokens and heads of d_i x_i r,
 * from the inputs of the forward call; dq may be dq_out and dk may be dk_out.  With DBLP_ACCUMULATE dweight is added to.
 * Sums over tokens are fp32, in an order that the shapes fix; dweight is rounded once to weight_dtype.
 * ws: dblp_norm_rotate_grad_workspace_bytes() bytes, 256-byte aligned, contents need not be preserved. */
enum { DBLP_ROTATE_INTERLEAVED = 2 };
typedef struct {
    uint32_t batch, tokens;         /* batch * tokens * heads < 2^31 */
    uint32_t q_heads, k_heads;      /* k_heads 0: no k, its pointers are not looked at */
    uint32_t head_dim;              /* a multiple of 8, at most 256 */
    uint32_t rotary_dim;            /* <= head_dim; a multiple of 16, interleaved of 2; 0 = no rotation */
    int dtype, weight_dtype;        /* any */
    uint32_t flags;                 /* DBLP_ROTATE_INTERLEAVED, for the gradient also DBLP_ACCUMULATE */
    float eps;                      /* > 0, finite */
    const int32_t* positions;       /* device; token t of sequence b is at positions[b * position_stride + t] */
    int64_t position_stride;
    const double* freqs;            /* device, rotary_dim / 2 angles in radians a position */
} dblp_norm_rotate_t;
/* weights: contiguous, head_dim elements; NULL = all ones */
int dblp_norm_rotate(const dblp_norm_rotate_t* a, const dblp_heads_t* q, const void* q_weight, const dblp_heads_t* q_out,
                     const dblp_heads_t* k, const void* k_weight, const dblp_heads_t* k_out, void* stream);
int dblp_norm_rotate_grad_workspace_bytes(const dblp_norm_rotate_t* a, size_t* bytes);
/* dq_weight, dk_weight NULL = not wanted (both NULL: no workspace needed); a weight that q and k share has two gradients, in two
 * places, which the caller adds up */
int dblp_norm_rotate_grad(const dblp_norm_rotate_t* a, const dblp_heads_t* q, const void* q_weight, const dblp_heads_t* dq_out,
                          const dblp_heads_t* dq, void* dq_weight, const dblp_heads_t* k, const void* k_weight,
                          const dblp_heads_t* dk_out, const dblp_heads_t* dk, void* dk_weight, void* ws, size_t ws_bytes,
                          void* stream);

/* A matrix: element (r, c) at data + r * row_stride + c * col_stride, in elements.  "Rows" means col_stride = 1. */
typedef struct {
    void* data;
    int64_t row_stride, col_stride;
} dblp_matrix_t;

typedef enum { DBLP_ACT_NONE = 0, DBLP_ACT_RELU = 1, DBLP_ACT_GELU = 2, DBLP_ACT_GELU_TANH = 3, DBLP_ACT_SILU = 4 } dblp_activation_t;
typedef struct {
    uint32_t rows, in, out;     /* x is rows x in, w is in x out; each below 2^31, workspaces below 2^62 bytes */
    int dtype;                  /* DBLP_BF16 or DBLP_F16: of x, w, pre, dy, dx, and the residual of dx */
    int out_dtype;              /* of out and its residual, for the gradient of dw: dtype or DBLP_F32 */
    int bias_dtype;             /* of bias, for the gradient of dbias: any */
    int activation;             /* dblp_activation_t */
    uint32_t flags;             /* the gradient: 0 or DBLP_ACCUMULATE (dw and dbias are added to) */
} dblp_linear_t;

/* dblp_linear: z = x w + bias, out = act(z) + residual; pre = z, for the backward pass.  x, residual, pre, out: rows; w: one
 * of its two strides is 1 (weights held as [out, in] are the transposed view).  bias: contiguous.  bias, residual, pre:
 * NULL = none.  out may be the residual (the same place and stride); apart from that out and pre lie over nothing else that is passed:
 * an in-place step x += x w needs a second place.  The product's operands are 16-bit, everything after that is fp32 and rounded
 * once.  The tensor cores' own sums truncate: sums of one sign lose up to 2.8e-6 of themselves where the result is fp32 (taken in runs of 512
 * terms), and an eighth of half a step where it has 16 bits.  relu: max(z, 0), NaN stays; gelu: z Phi(z); gelu_tanh: z / 2 (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))); silu:
 * z / (1 + exp(-z)).
 * dblp_linear_grad: dx = (dy w^T + residual) * act'(pre), dw = x^T dy, dbias = sum of dy's rows.  `pre` belongs to the
 * layer BEFORE: where x = act(pre) was that layer's output, dx is the gradient of its pre-activation, ready to be its dy;
 * without an activation pre is NULL.  residual (of dx, NULL = none): the gradient that reaches x on another way.  relu' is
 * 0 at 0 and NaN at NaN.  dx, dw, dbias: NULL = not wanted; dx may be the residual or pre (the same place and stride)
 * or lie over x, which is read before; no other result lies over an operand or another result.  dw: one of its strides is 1.
 * Every sum over the rows or columns is fp32, in an order that the shapes, types and alignments fix.
 * ws: dblp_linear_workspace_bytes() bytes for the same x, w and dy (NULL: forward only), 256-byte aligned, contents need not
 * be preserved.  It holds copies of operands whose data or strides are not multiples of 16 bytes, and partial sums where
 * few rows or a long sum are split over the device. */
int dblp_linear_workspace_bytes(const dblp_linear_t* l, const dblp_matrix_t* x, const dblp_matrix_t* w, const dblp_matrix_t* dy,
                                size_t* fwd_bytes, size_t* grad_bytes);
int dblp_linear(const dblp_linear_t* l, const dblp_matrix_t* x, const dblp_matrix_t* w, const void* bias,
                const dblp_matrix_t* residual, const dblp_matrix_t* pre, const dblp_matrix_t* out, void* ws, size_t ws_bytes,
                void* stream);
int dblp_linear_grad(const dblp_linear_t* l, const dblp_matrix_t* dy, const dblp_matrix_t* x, const dblp_matrix_t* w,
                     const dblp_matrix_t* residual, const dblp_matrix_t* pre, const dblp_matrix_t* dx, const dblp_matrix_t* dw,
                     void* dbias, void* ws, size_t ws_bytes, void* stream);

/* dblp_orthogonalize: an update whose singular values are brought near 1 by Newton-Schulz products, matrix by matrix:
 *     X = x / (|x|_F + eps);  for each (a, b, c):  A = X X^T, X = a X + (b A + c A A) X;  out = scale X
 * (with X^T X and X (b A + c A A) where x is taller than wide: the products are always those of the shorter side).
 * Used on the mean of a round (Algorithm 3) before the weights are updated.
 * The norm is summed in 64 bits.  X and A enter the products scaled by powers of two (1024 and 256) and rounded to f16; X itself is
 * kept in two f16 words (22 bits), so that what rounding adds is not amplified with the small singular values.  How far results are from
 * the iteration in 64 bits, in parts of their norm, with five steps of the usual coefficients:
 *   out_dtype BF16  the result's own rounding, 1.7e-3, up to 1.1 times that below 512 on the shorter side, where products read both words in
 *                   the last three steps (below 64 in all), and up to 1.5 times that for larger matrices, whose products are of one f16 word
 *                   each (1.7 times where all singular values are alike).
 *   F32 or F16      the products are of both words (three products each, about three times the work of large matrices): up to 5e-6, and up to 6e-5 for
 *                   matrices of one or a few directions (iterated in fp32: 5e-6, 1.6e-4); F16 results are rounded besides.
 * For a bf16 result as near as the fp32 iteration's take F32 and convert.
 * Coefficients must keep the entries of X below 63 and those of A and b A + c A A below 255 (singular values up to about 2 do), beyond
 * which they become infinite.  An x of zeros gives zeros.  NaN or infinity in a matrix spreads over that matrix alone.
 * out may be x (the same place, strides and dtype).
 * ws: dblp_orthogonalize_workspace_bytes() bytes, 256-byte aligned, contents need not be preserved. */
enum { DBLP_ORTHOGONALIZE_STEPS = 16 };
typedef struct {
    uint32_t batch, rows, cols;         /* rows, cols <= 32768; batch < 65536 */
    int x_dtype, out_dtype;             /* any */
    uint32_t steps;                     /* 1 .. DBLP_ORTHOGONALIZE_STEPS */
    const float* coefficients;          /* HOST, steps times (a, b, c), finite */
    float eps;                          /* >= 0 */
    float scale;                        /* finite */
    int64_t x_batch_stride, x_row_stride, out_batch_stride, out_row_stride;  /* in elements */
} dblp_orthogonalize_t;
int dblp_orthogonalize_workspace_bytes(const dblp_orthogonalize_t* a, size_t* bytes);
int dblp_orthogonalize(const dblp_orthogonalize_t* a, const void* x, void* out, void* ws, size_t ws_bytes, void* stream);

/* ---- diagnostics -----------------------------------------------------------------------------------------------*/
const char* dblp_strerror(int status);
const char* dblp_last_error(void);  /* HOST string, valid until the calling thread's next failing call */
/* Waits inside kernels that gave up after their limit (about two seconds), on the current device since the library was
 * loaded; 0 unless something is wrong, else the results of the calls before it are incomplete.  Reads the device:
 * synchronises with the default stream. */
int dblp_wait_timeouts(uint64_t* count);
uint64_t dblp_launch_count(void);   /* kernels launched by this library since it was loaded */

#ifdef __cplusplus
}
#endif
#endif /* DBLP_H */
