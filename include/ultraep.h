/*
 * ultraep.h — C ABI of the MI355X (gfx950) library for UltraEP's
 * per-microbatch, per-layer balancing path (arXiv 2606.04101):
 *
 *   1. ultraep_count          exact per-expert loads from top-k routing ids
 *   2. ultraep_plan           quota-driven replication (SolveReplication) and
 *                             reroute split (SolveReroute), Algorithm 1
 *   3. ultraep_dispatch       token-to-replica assignment and bf16 row scatter
 *                             into per-destination, per-replica blocks
 *   4. ultraep_pack_replicas  local half of weight distribution: the blobs of
 *                             this rank's replicated main experts copied into
 *                             per-destination staging
 *      ultraep_relay_plan     relay trees for hot-expert fan-out, and
 *      ultraep_pack_relay     the packing that follows them
 *   5. ultraep_combine        reverse reroute: gate-weighted gather of the
 *                             experts' output rows back to token order
 *   6. ultraep_grad_reduce    local half of the gradient reduction: replica
 *                             gradients accumulated into main gradients
 *
 * and the operators of the MoE layer around it:
 *
 *   7. ultraep_route          router: top-k ids, gates, per-expert counts and
 *      ultraep_balance_loss   score sums; the balance loss over them
 *      ultraep_route_grad     and the logits' gradient from both
 *   8. ultraep_combine_grad   backward pass of the combine
 *   9. ultraep_quant_rows     rows to 8-bit integers with a scale each, and
 *      ultraep_expert_matmul  the experts' products on them, block by block
 *  10. ultraep_expert_matmul_bf16   the experts' products in bf16, forward and
 *                             for the gradient of their input, and
 *      ultraep_expert_weight_grad   the gradient of their weights
 *  11. ultraep_quant_blocks   rows to 8-bit floating point with a scale for each
 *                             128 elements, and
 *      ultraep_expert_matmul_fp8    the experts' products on them
 *
 * Conventions for every call:
 *   - Buffer pointers are DEVICE pointers unless marked "host".  The caller
 *     owns and allocates every buffer; the library never allocates, never
 *     frees, never synchronises the host, keeps no state between calls and
 *     issues no memset, so every call can be captured into a HIP graph.
 *     (ultraep_plan_noalloc takes its workspace from a fixed array in the
 *     library's device memory instead of a caller buffer; see there.)
 *   - Work is enqueued on `stream` in order; results are ready when the
 *     stream reaches that point.  Calls on different streams must use
 *     distinct output and workspace buffers.
 *   - Return value: ULTRAEP_OK, or ULTRAEP_EINVAL for an argument problem
 *     that the host can see (nothing is launched), or ULTRAEP_EDEVICE when a
 *     launch fails.
 *   - Problems visible only in device data are reported through a device
 *     status word: the first failing kernel stores its (negative) code into
 *     *status if it still holds 0.  The caller zeroes the word before a
 *     sequence of calls and reads it after its own synchronisation.  When
 *     the status is nonzero the outputs of the failing call are undefined.
 *   - Layouts are row-major.  With n_main = E / R main experts per rank,
 *     home rank h(e) = e / n_main (main experts in contiguous blocks),
 *     S = n_main + n_slot physical slots per rank (slot p < n_main is main
 *     expert r*n_main + p, slot n_main + s is redundant slot s) and
 *     ncol = E + R * n_slot CSR entries at most.
 *   - bf16 data are moved as raw 16-bit patterns (never converted).
 *
 * Supported sizes (else ULTRAEP_EINVAL): 1 <= R <= 64, E % R == 0,
 * E <= 1024, 0 <= n_slot, R * n_slot <= 256, u_min >= 1,
 * 1 <= beta_den <= beta_num <= 2^20, 1 <= k <= min(E, 64), T >= 0,
 * T * k < 2^31, H % 8 == 0, W % 8 == 0, 16-byte aligned x / send / w_main /
 * staging; other buffers aligned to their elements unless their call asks for
 * more, workspaces to 8 bytes (not checked).  The total load of a plan must not exceed 2^30 tokens (device
 * status ULTRAEP_EDATA otherwise).
 */
#ifndef ULTRAEP_H
#define ULTRAEP_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  ULTRAEP_OK = 0,
  ULTRAEP_EINVAL = -1,  /* bad argument (host-visible); nothing launched */
  ULTRAEP_ENOSPC = -2,  /* device: staging capacity too small */
  ULTRAEP_EDEVICE = -3, /* a kernel launch failed */
  ULTRAEP_EDATA = -4    /* device: ids out of range, negative or oversized
                           loads, or a load row that disagrees with topk */
};

/* EP group metadata and the planner's constants (host struct).
 * Table 1 of the paper: R ranks, E logical experts, N_slot redundant slots per
 * rank, quota floor u_min (1024 in the paper) and balancing target
 * beta = beta_num / beta_den (1.01 in the paper, i.e. 101/100). */
typedef struct {
  int32_t R;
  int32_t E;
  int32_t n_slot;
  int64_t u_min;
  int32_t beta_num;
  int32_t beta_den;
} ultraep_group;

/* Plan outputs (device buffers; element counts from ultraep_plan_sizes).
 *   slot_expert [R * n_slot]   X (Table 1): x_{t,s} = expert hosted by
 *                              redundant slot s of rank t, -1 when empty;
 *                              slots fill in the order replicas are accepted.
 *   quota       [E * R]        U (Table 1): u_{e,t} at e * R + t.
 *   host_ptr    [E + 1]        CSR row pointers over the hosts H(e).
 *   host_rank   [ncol]         H(e) in order: home first, then replica ranks
 *                              ascending; -1 padding after host_ptr[E].
 *   host_pslot  [ncol]         physical slot of that instance on its rank;
 *                              -1 padding.
 *   reroute     [R * ncol]     Q (Table 1): q_{r,e,t} at r * ncol + j where j
 *                              is the CSR entry of (e, t); 0 padding.
 *   stats       [8] int64      tau*, tau_lo0, tau_hi0, number of bisection
 *                              probes, number of replicas, max |H(e)|,
 *                              status (0 or ULTRAEP_EDATA), total load L. */
typedef struct {
  int32_t *slot_expert;
  int32_t *quota;
  int32_t *host_ptr;
  int32_t *host_rank;
  int32_t *host_pslot;
  int32_t *reroute;
  int64_t *stats;
} ultraep_plan_buf;

/* Host only.  Element counts of the seven plan buffers, in struct order, for
 * group *g (host pointer).  Returns ULTRAEP_EINVAL for an unsupported group. */
int ultraep_plan_sizes(const ultraep_group *g, size_t counts_out[7]);

/* Step 1 — exact load acquisition (Sec. 4.2 forward pipeline; lambda_{r,e} of
 * Table 1): counts[b * E + e] = number of (token, k) slots of block b routed
 * to expert e, for n_groups blocks of T * k ids stored back to back in topk
 * ([n_groups][T][k] int32).  Id -1 means "not routed" and is skipped; ids
 * outside [-1, E) are skipped and raise ULTRAEP_EDATA in *status.  One count
 * per routed slot (no per-token deduplication).  counts is fully written.
 * 1 <= n_groups <= 65535, 1 <= k <= min(E, 64), E <= 1024, T * k < 2^31. */
int ultraep_count(const int32_t *topk, int64_t T, int32_t k, int32_t E,
                  int32_t n_groups, int32_t *counts, int32_t *status,
                  hipStream_t stream);

/* Step 2 — Algorithm 1 on the load matrix (device, [R][E] int32, row r =
 * lambda_{r,.}).  SolveReplication binary-searches the integer threshold tau
 * from tau_lo = ceil(beta * ceil(L / R)) to tau_hi = max_r ell_r with
 * tau = floor((lo + hi) / 2), running the greedy probe of Sec. 5.1 at each
 * step (overloaded ranks by descending excess, their main experts by
 * descending load, transfers of min(excess, slack, remaining load) to the
 * admissible rank of largest slack, a transfer below u_min ends the expert;
 * all ties go to the lower id).  The last feasible probe gives X and U; with
 * no feasible probe every expert stays on its home.  SolveReroute (Sec. 5.2)
 * lets each host's own tokens consume its quota first, then splits every
 * source's residual demand over the residual quotas in proportion, sources
 * in ascending rank order, by largest remainder against the quotas still
 * unconsumed (ties to the earlier host), which keeps both margins of Q
 * exact.  Every output buffer is fully written (padding included).  Data
 * errors (negative loads, L > 2^30) set stats[6] = ULTRAEP_EDATA.
 *   ws  device workspace of ws_bytes >= ultraep_plan_ws_bytes(g); its
 *       contents on entry do not matter. */
int ultraep_plan(const int32_t *load, const ultraep_group *g,
                 const ultraep_plan_buf *out, void *ws, size_t ws_bytes,
                 hipStream_t stream);

/* ultraep_plan for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the same kernels and outputs as ultraep_plan, with the planner workspace
 * taken from a fixed array in the library's device memory instead of a
 * caller buffer.  The array holds ULTRAEP_PLAN_STATIC_WS_BYTES (4.25 MiB),
 * enough for every supported group (R <= 64, E <= 1024, R * n_slot <= 256);
 * a group that would need more is rejected with ULTRAEP_EINVAL before any
 * launch.  Each device the library runs on holds its own copy from the
 * first call on that device (made with that device current) until the
 * process ends.  The call allocates nothing and launches the planner's
 * kernels only; the first kernel clears the part of the array that must
 * start at zero.  Every call on one device shares that device's array:
 * calls that overlap in time on one device (on different streams without
 * an ordering between them, or from several host threads) race on it, so
 * the caller serialises them.  ULTRAEP_EDEVICE if the array's device
 * address cannot be obtained or a launch fails. */
#define ULTRAEP_PLAN_STATIC_WS_BYTES ((size_t)17 << 18)
int ultraep_plan_noalloc(const int32_t *load, const ultraep_group *g,
                         const ultraep_plan_buf *out, hipStream_t stream);

/* The two halves of ultraep_plan, in this order on one stream (or with the
 * second made to wait for the first): SolveReplication writes slot_expert,
 * quota, host_ptr, host_rank, host_pslot and stats; SolveReroute then writes
 * reroute from the load matrix and those buffers.  They are separate so a
 * caller can run the reroute alongside the weight distribution
 * (ultraep_pack_replicas needs only slot_expert), as in the forward pipeline
 * of Sec. 4.2 and Eq. (1). */
int ultraep_plan_replicate(const int32_t *load, const ultraep_group *g,
                           const ultraep_plan_buf *out, void *ws, size_t ws_bytes,
                           hipStream_t stream);
int ultraep_plan_reroute(const int32_t *load, const ultraep_group *g,
                         const ultraep_plan_buf *out, hipStream_t stream);

/* Bytes of device workspace ultraep_plan needs for group *g (host only; 0
 * for an unsupported group): per-expert orders and the outcome and transfer
 * record of every speculatively evaluated bisection probe. */
size_t ultraep_plan_ws_bytes(const ultraep_group *g);

/* Bytes of device workspace ultraep_dispatch / ultraep_dispatch_layout need
 * (host only; 0 for unsupported arguments). */
size_t ultraep_dispatch_ws_bytes(int64_t T, int32_t k, const ultraep_group *g);

/* Step 3 — token assignment and dispatch permutation of source rank `rank`
 * (Sec. 5.2 Token Assignment).  The j-th local slot routed to expert e
 * (counted over the (token, k) slots in token-major order) goes to the first
 * instance of H(e) whose cumulative quota q_{rank,e,.} exceeds j.  The send
 * buffer holds one block per (destination rank t, physical slot p) in
 * (t, p) order, block (t, p) holding q_{rank, e(t,p), t} rows in ascending
 * token order.
 *   x            [T][H] bf16 token rows of this rank
 *   topk         [T][k] int32 expert ids (-1 = not routed)
 *   plan         outputs of ultraep_plan (device buffers)
 *   send         [T*k][H] bf16: routed rows at their positions, rows from
 *                block_off[R*S] to T*k - 1 zero-filled
 *   row_of_slot  [T*k] int32 row of send for each slot, -1 if not routed
 *   block_off    [R*S + 1] int64 first row of each block, last = routed rows
 *   ws           device workspace of ws_bytes >= ultraep_dispatch_ws_bytes
 * A plan row that does not describe exactly the routed ids of topk raises
 * ULTRAEP_EDATA. */
int ultraep_dispatch(const uint16_t *x, const int32_t *topk, int64_t T,
                     int32_t k, int32_t H, int32_t rank,
                     const ultraep_group *g, const ultraep_plan_buf *plan,
                     uint16_t *send, int32_t *row_of_slot, int64_t *block_off,
                     void *ws, size_t ws_bytes, int32_t *status,
                     hipStream_t stream);

/* The two halves of ultraep_dispatch, for callers that move the rows
 * themselves or time them apart: the layout (row_of_slot, block_off) and the
 * scatter (send rows; n_routed = block_off + R * S, the routed row count,
 * read on the device: rows n_routed .. T*k - 1 are zero-filled, none when
 * the count lies outside [0, T*k]). */
int ultraep_dispatch_layout(const int32_t *topk, int64_t T, int32_t k,
                            int32_t rank, const ultraep_group *g,
                            const ultraep_plan_buf *plan, int32_t *row_of_slot,
                            int64_t *block_off, void *ws, size_t ws_bytes,
                            int32_t *status, hipStream_t stream);
int ultraep_dispatch_scatter(const uint16_t *x, int64_t T, int32_t k,
                             int32_t H, const int32_t *row_of_slot,
                             const int64_t *n_routed, uint16_t *send,
                             hipStream_t stream);

/* Step 4 — local half of the forward weight distribution (Sec. 6.1; the
 * remote peer stores are not part of this library).  Every redundant slot
 * (t, s) whose expert e has home `rank` receives a bit copy of
 * w_main[e - rank * n_main]; entries are ordered by destination rank t, then
 * slot s.
 *   w_main    [n_main][W] bf16 blobs of this rank's main experts (W elements
 *             each; an expert's gate, up and down matrices as stored)
 *   staging   [cap][W] bf16; entries 0 .. n_out-1 written, the rest untouched
 *   dest_off  [R + 1] int64 first entry of each destination rank, last = n_out
 * If n_out > cap, ULTRAEP_ENOSPC is raised, dest_off is still written and no
 * entry is copied. */
int ultraep_pack_replicas(const uint16_t *w_main, int64_t W, int32_t rank,
                          const ultraep_group *g, const ultraep_plan_buf *plan,
                          uint16_t *staging, int64_t cap, int64_t *dest_off,
                          int32_t *status, hipStream_t stream);

/* SolveReroute of ultraep_plan_reroute and the packing of
 * ultraep_pack_replicas in one launch, overlapped as the forward pipeline of
 * Sec. 4.2 overlaps the reroute with the weight distribution (Eq. (1)): the
 * same results as the two calls.  Needs the buffers ultraep_plan_replicate
 * wrote; arguments and errors as for the two calls. */
int ultraep_reroute_and_pack(const int32_t *load, const ultraep_group *g,
                             const ultraep_plan_buf *plan, const uint16_t *w_main, int64_t W,
                             int32_t rank, uint16_t *staging, int64_t cap, int64_t *dest_off,
                             int32_t *status, hipStream_t stream);

/* Relay trees for hot-expert fan-out (Sec. 6.2, load-aware relay
 * scheduling), from a plan (slot_expert and the host lists).  Each rank's
 * sending volume starts at one expert blob per replica of its main experts.
 * Every expert with more than `threshold` replicas (the paper uses 4), by
 * replica count descending then id ascending, gets the integer nearest
 * sqrt(replicas) first-stage relays: its replica ranks of smallest volume;
 * each other replica, by ascending rank, is served by the relay whose
 * volume is smallest (one blob added at once); the source's volume then
 * drops to one blob per relay.  Ties go to the smaller rank.
 *   threshold    >= 0
 *   slot_src     [R * n_slot] int32: the rank that sends redundant slot
 *                (t, s) its blob (the expert's home rank or a relay), -1 for
 *                an empty slot
 *   send_vol     [R] int32: blobs each rank sends under the trees
 *   relay_stats  [4] int64: experts with relays, relays in total, largest
 *                sending volume before and after
 * A plan whose host lists do not match its slot map, or whose stats[6] is
 * nonzero, raises ULTRAEP_EDATA (outputs undefined).  Every output element
 * is written otherwise. */
int ultraep_relay_plan(const ultraep_group *g, const ultraep_plan_buf *plan, int32_t threshold,
                       int32_t *slot_src, int32_t *send_vol, int64_t *relay_stats,
                       int32_t *status, hipStream_t stream);

/* Local half of the weight distribution with relay trees (Sec. 6.1 tile
 * copy, Sec. 6.2 trees): every redundant slot (t, s) whose sender
 * slot_src[t * n_slot + s] is `rank` receives a bit copy of its expert's
 * blob, entries ordered by destination rank t, then slot s.  The blob of a
 * main expert of `rank` comes from w_main; the blob of an expert that
 * `rank` relays comes from relay_src[s'], this rank's own redundant slot s'
 * holding that expert (the buffer the first stage fills).
 *   relay_src  [n_slot][W] bf16 (needed when n_slot > 0)
 *   staging, dest_off, cap as for ultraep_pack_replicas.
 * A slot this rank should relay without hosting its expert raises
 * ULTRAEP_EDATA; n_out > cap raises ULTRAEP_ENOSPC. */
int ultraep_pack_relay(const uint16_t *w_main, const uint16_t *relay_src, int64_t W, int32_t rank,
                       const ultraep_group *g, const ultraep_plan_buf *plan,
                       const int32_t *slot_src, uint16_t *staging, int64_t cap,
                       int64_t *dest_off, int32_t *status, hipStream_t stream);

/* Reverse reroute: the combine gather (Sec. 4.2, the scatter-to-gather
 * inversion of the token assignment).  Token t's output row is the sum of
 * its routed slots' rows weighted by their gates:
 *   out[t] = bf16( sum_{kk ascending, row_of_slot[t*k+kk] >= 0}
 *                  gate[t*k+kk] * y[row_of_slot[t*k+kk]] )
 * in fp32: every product and every partial sum rounded to fp32 (no fused
 * multiply-add), from +0; the result rounded to bf16 to nearest-even, every
 * NaN to 0x7FC0.  The paper fixes bf16 activations only; this order and
 * precision are the library's reading.
 *   y            [n_rows][H] bf16: rows in the dispatch layout (the experts'
 *                outputs for the rows ultraep_dispatch sent)
 *   gate         [T][k] fp32 top-k gate weights
 *   row_of_slot  [T*k] int32 from ultraep_dispatch (-1 = not routed)
 *   out          [T][H] bf16, fully written
 * A row outside [-1, n_rows) raises ULTRAEP_EDATA (that slot is skipped).
 * 1 <= k <= 64, H % 8 == 0, 16-byte aligned y and out. */
int ultraep_combine(const uint16_t *y, int64_t n_rows, const float *gate,
                    const int32_t *row_of_slot, int64_t T, int32_t k, int32_t H, uint16_t *out,
                    int32_t *status, hipStream_t stream);

/* Gradient reduction, local half (Sec. 4.2 backward pass, tile streaming of
 * Sec. 6.1): every replica of a main expert of `rank` returns an fp32
 * gradient blob, laid out like the forward staging (one [W] entry per
 * redundant slot (t, s) whose expert has home `rank`, destination rank
 * ascending, then slot).  Each main gradient is updated in place to
 *   main_grad[l] = (...(main_grad[l] + r_0) + r_1 ...) + r_{f-1}
 * element by element in fp32, its replicas' entries taken in that staging
 * order, and every replica entry is then zeroed for reuse by the next layer.
 *   main_grad  [n_main][W] fp32, read and written
 *   rgrad      [cap][W] fp32, entries 0 .. n_out-1 read and zeroed
 * n_out > cap raises ULTRAEP_ENOSPC and changes nothing.  W % 4 == 0,
 * 16-byte aligned buffers. */
int ultraep_grad_reduce(float *main_grad, float *rgrad, int64_t W, int32_t rank,
                        const ultraep_group *g, const ultraep_plan_buf *plan, int64_t cap,
                        int32_t *status, hipStream_t stream);

/* Element types of the operators below that take more than one. */
enum {
  ULTRAEP_F32 = 0,
  ULTRAEP_BF16 = 1
};

enum {
  ULTRAEP_SOFTMAX = 0,
  ULTRAEP_SIGMOID = 1
};

/* A router (host struct): E experts, k of them a token, 1 <= k <= min(E, 64),
 * E <= 1024.
 *   score      of a token's logits z: ULTRAEP_SOFTMAX  s = softmax(z), or
 *              ULTRAEP_SIGMOID  s = 1 / (1 + exp(-z))
 *   renorm     1: a token's gates are scale * s_i / (sum of its chosen s);
 *              0: scale * s_i
 *   n_group,   0, 0: every expert is eligible.  Else the experts form n_group
 *   top_group  contiguous groups of at least two (n_group <= 64 divides E);
 *              a group scores the sum of its two largest keys and the
 *              token's ids come from its top_group best (ties: the lower
 *              group; k <= top_group * E / n_group).  One with fewer than two
 *              experts that can be chosen scores -inf.  1, 1 is as 0, 0
 *   scale      finite
 *   seq_len    tokens of a sequence for the statistics: token t belongs to
 *              sequence t / seq_len.  0: all T tokens are one */
typedef struct {
  int32_t E;
  int32_t k;
  int32_t score;
  int32_t renorm;
  int32_t n_group;
  int32_t top_group;
  float scale;
  int64_t seq_len;
} ultraep_router;

/* Router.  A token's ids are the k experts of largest key, in falling order,
 * equal keys by rising id, where the key is
 *   softmax  z + bias
 *   sigmoid  s + bias; z itself where there is neither bias nor groups
 * in fp32 (bias enters the selection only).  So a softmax's bias is on the
 * logits' scale, and its groups rank by sums of two logits: a router that adds
 * its bias to the probabilities, or ranks groups by their largest one, chooses
 * other ids.  An expert whose logit or bias is
 * -inf is never chosen: the ids left over are -1, their gates 0.  A token that is
 * masked, or has no logit above -inf, gets ids -1 and gates 0 and counts in no
 * statistic; so does one with a NaN or +inf logit, which raises ULTRAEP_EDATA.
 * The ids are what ultraep_count and ultraep_dispatch take, the gates what
 * ultraep_combine takes, and counts (with seq_len 0) this rank's row of the
 * load matrix.
 *   logits    [T] rows of E elements of `type`, ld elements apart (E <= ld <= 2^20)
 *   bias      [E] fp32, or null.  +inf is as the largest finite number; a NaN
 *             raises ULTRAEP_EDATA, and its expert is not chosen
 *   mask      [T] bytes, 0 = masked; or null
 *   topk      [T][k] int32
 *   gate      [T][k] fp32
 * Statistics of each of the n_seg = ceil(T / seq_len) sequences (1 with
 * seq_len 0, also for T = 0); all three, or null for each:
 *   counts    [n_seg][E] int32: ids by expert
 *   prob_sum  [n_seg][E] fp32: sum over tokens of p = s / (sum of all E s)
 *             (softmax: p = s)
 *   tokens    [n_seg] int32: tokens that have an id
 *   ws        workspace of ws_bytes >= ultraep_route_ws_bytes for this T or a
 *             larger one, 4-byte aligned
 *             (may be null without statistics)
 * Sums run in one fixed order for given T and router: equal calls give equal
 * bits.  T <= 2^23. */
int ultraep_route(const void *logits, int32_t type, int64_t T, int64_t ld,
                  const ultraep_router *r, const float *bias, const uint8_t *mask,
                  int32_t *topk, float *gate, int32_t *counts, float *prob_sum,
                  int32_t *tokens, void *ws, size_t ws_bytes, int32_t *status,
                  hipStream_t stream);

/* Bytes of device workspace that ultraep_route needs for its statistics with up
 * to T tokens, so one workspace does for the largest batch and all smaller ones
 * (host only; 0 for unsupported arguments, at least 4 otherwise). */
size_t ultraep_route_ws_bytes(int64_t T, const ultraep_router *r);

/* Balance loss over n_seg sequences: with c, F = counts, load_tokens (this
 * rank's own, or summed over all ranks), P, n = prob_sum, tokens
 *   coef[s][e] = alpha * E * c[s][e] / (n_seg * k * F[s] * n[s])
 *   loss       = sum over s, e of coef[s][e] * P[s][e]
 * coef is 0 for a sequence whose F or n is not positive; it is the loss's
 * gradient with respect to each of the sequence's score rows p, which
 * ultraep_route_grad takes.  Neither aliases an input.  n_seg >= 0 (0: loss 0). */
int ultraep_balance_loss(const int32_t *counts, const int32_t *load_tokens,
                         const float *prob_sum, const int32_t *tokens, int64_t n_seg,
                         const ultraep_router *r, float alpha, float *loss, float *coef,
                         hipStream_t stream);

/* Gradient of the router: of  sum dgate * gate + dloss * sum coef * p  with
 * respect to the logits (topk and coef are constants).
 *   topk     [T][k] from ultraep_route
 *   dgate    [T][k] fp32, or null (0)
 *   coef     [n_seg][E] from ultraep_balance_loss, or null (0)
 *   dloss    one fp32 on the device, or null (1)
 *   dlogits  rows like logits': type, ld; all T * E elements are written, the
 *            ld - E between them are not; may be logits itself
 * Masked tokens, tokens whose first id is -1, and logits of -inf, get 0.  An id outside
 * [-1, E), a NaN or a +inf logit raises ULTRAEP_EDATA.  bias and groups only
 * choose ids and do not enter.  T <= 2^23. */
int ultraep_route_grad(const void *logits, int32_t type, int64_t T, int64_t ld,
                       const ultraep_router *r, const uint8_t *mask, const int32_t *topk,
                       const float *dgate, const float *coef, const float *dloss,
                       void *dlogits, int32_t *status, hipStream_t stream);

/* Backward pass of ultraep_combine: from dout [T][H] bf16, the gradient of its
 * output rows,
 *   dy[row_of_slot[t*k+i]] = bf16(gate[t*k+i] * dout[t])
 *   dgate[t*k+i]           = sum_h dout[t][h] * y[row_of_slot[t*k+i]][h]  (fp32)
 * rounded to nearest-even, NaN to 0x7FC0; a masked slot (row -1) has dgate 0.
 * The backward pass of the dispatch is ultraep_combine with gates 1.
 *   y, dy     [n_rows][H] bf16 in the dispatch layout; dy may not be y
 *   n_routed  device, block_off + R * S of the dispatch: dy's rows from there
 *             to n_rows - 1 are zero-filled
 * A row outside [-1, n_routed) (that slot is skipped, its dgate 0), or n_routed
 * outside [0, n_rows] (dy is left alone and dgate 0), raises ULTRAEP_EDATA.
 * Sizes and alignment as for ultraep_combine; n_rows < 2^31. */
int ultraep_combine_grad(const uint16_t *dout, const uint16_t *y, int64_t n_rows,
                         const float *gate, const int32_t *row_of_slot, int64_t T, int32_t k,
                         int32_t H, const int64_t *n_routed, uint16_t *dy, float *dgate,
                         int32_t *status, hipStream_t stream);

/* Rows to 8-bit integers with a scale each.  With a = max |x| over a row,
 *   scale = a / 127,  q = round-to-nearest-even(x * (127 / a))
 * each operation in fp32; a row with a <= 2^-100 has q 0 and scale 0, a row
 * with an infinity or a NaN q 0 and scale NaN.  A weight [n][N][K] takes n * N
 * rows.
 *   x      rows of K elements of `type`, ld elements apart
 *   q      rows of ldq bytes, ldq >= K: K integers, then zeros
 *   scale  [rows] fp32
 * K, ld % 8 == 0, ldq % 16 == 0, ld, ldq <= 2^20, rows < 2^31, 16-byte aligned x
 * and q. */
int ultraep_quant_rows(const void *x, int32_t type, int64_t rows, int64_t K, int64_t ld,
                       int8_t *q, int64_t ldq, float *scale, hipStream_t stream);

/* The experts' products on 8-bit integers.  Row m of block g (rows block_off[g]
 * to block_off[g + 1] - 1, as the dispatch writes them) meets weight
 * w = block_w[g]:
 *   v[n] = (sum_k xq[m][k] * wq[w][n][k]) * x_scale[m] * w_scale[w][n]
 * the sum in 32-bit integers (exact), the rest in fp32.  y[m] = v, or with
 * act 1 (SwiGLU, gate rows of the weight first)
 *   y[m][n] = v[n] / (1 + exp(-v[n])) * v[N/2 + n],  n < N/2
 * rounded to nearest-even to `type`.
 *   xq         [M][K] int8, x_scale [M] fp32
 *   wq         [n_w][N][K] int8, w_scale [n_w][N] fp32
 *   block_off  [n_block + 1] int64 (a part of the dispatch's is fine: rows
 *              outside the blocks are neither read nor written)
 *   block_w    [n_block] int32, or null (block g takes weight g)
 *   y          [M][N], or [M][N / 2] with act
 * Blocks that are not in rising order within [0, M], and a nonempty block
 * whose weight is outside [0, n_w), raise ULTRAEP_EDATA; then no row is written.
 * 1 <= n_block <= 2048, n_w >= 1, M < 2^31; K % 16 == 0, K <= 2^16 (the sum
 * stays within 32 bits), N % 8 == 0 (N % 16 == 0 with act), N <= 2^20,
 * M * N < 2^38; 16-byte aligned xq, wq and y.  M = 1 is the decode form: any M takes any blocks. */
int ultraep_expert_matmul(const int8_t *xq, const float *x_scale, int64_t M,
                          const int8_t *wq, const float *w_scale, int32_t n_w, int32_t N,
                          int32_t K, const int64_t *block_off, const int32_t *block_w,
                          int32_t n_block, int32_t act, void *y, int32_t type,
                          int32_t *status, hipStream_t stream);

enum {
  ULTRAEP_NO_ACT = 0,
  ULTRAEP_SWIGLU = 1,
  ULTRAEP_SWIGLU_GRAD = 2
};

/* The experts' products in bf16.  Row m of block g (rows block_off[g] to
 * block_off[g + 1] - 1, as the dispatch writes them) meets weight
 * w = block_w[g]:
 *   trans 0  v[n] = sum_k x[m][k] * w[n][k], weights [N][K]: the forward product
 *   trans 1  v[n] = sum_k x[m][k] * w[k][n], weights [K][N]: on the forward
 *            product's own weights this is the gradient of its input, x being
 *            the gradient of its output
 * exact products summed in fp32.  What leaves is
 *   ULTRAEP_NO_ACT       y[m][n] = v[n]
 *   ULTRAEP_SWIGLU       y[m][n] = v[n] / (1 + exp(-v[n])) * v[N/2 + n], n < N/2
 *                        (gates first), and pre[m] = v unless pre is null
 *   ULTRAEP_SWIGLU_GRAD  v is the gradient of such a y; with a, b = pre[m][n],
 *                        pre[m][N + n] and s = 1 / (1 + exp(-a)),
 *                        y[m][n]     = v[n] * b * s * (1 + a * (1 - s))
 *                        y[m][N + n] = v[n] * a * s
 * in fp32 (the SwiGLU of v itself, not of the rounded pre), rounded to
 * nearest-even to `type`, pre to bf16.  The exponential and the quotient are the
 * hardware's exp2 and reciprocal: v / (1 + exp(-v)) is off by (1.25 |v| + 6) * 2^-24
 * of its value at most, and 0 where v < -87.3 (it is under 2e-36 in magnitude there);
 * the gradients by (3 |a| + 20) * 2^-24 of |v| |b| s (1 + |a| (1 - s)) and |v| |a| s.
 *   x          [M][K] bf16
 *   w          n_w weights of N * K bf16, w_stride elements apart (so they may
 *              lie in blobs that hold an expert's other weights too)
 *   block_off  [n_block + 1] int64 (a part of the dispatch's is fine: rows
 *              outside the blocks are neither read nor written)
 *   block_w    [n_block] int32, or null (block g takes weight g)
 *   pre        SWIGLU: [M][N] bf16, written, or null; SWIGLU_GRAD: [M][2 N]
 *              bf16, read; NO_ACT: null
 *   y          rows of N, N / 2 (SWIGLU) or 2 N (SWIGLU_GRAD) elements; with
 *              SWIGLU_GRAD and bf16 it may be pre itself; otherwise neither y nor a
 *              written pre overlaps another buffer
 * Blocks that are not in rising order within [0, M], and a nonempty block
 * whose weight is outside [0, n_w), raise ULTRAEP_EDATA; then no row is written.
 * 1 <= n_block <= 2048, n_w >= 1, M < 2^31; K, N % 8 == 0 (N % 16 == 0 with
 * SWIGLU), 8 <= K, N <= 2^20, M * N < 2^38; N * K <= w_stride <= 2^40,
 * w_stride % 8 == 0; 16-byte aligned x, w, pre and y. */
int ultraep_expert_matmul_bf16(const uint16_t *x, int64_t M, const uint16_t *w, int32_t n_w,
                               int64_t w_stride, int32_t N, int32_t K, int32_t trans,
                               const int64_t *block_off, const int32_t *block_w,
                               int32_t n_block, int32_t act, uint16_t *pre, void *y,
                               int32_t type, int32_t *status, hipStream_t stream);

/* Gradient of the weights of y = x w^T: for every weight w of n_w
 *   dw[w][n][k] = sum over the blocks g with block_w[g] = w, in rising order,
 *                 and their rows m, of dy[m][n] * x[m][k]
 * exact products summed in fp32, rounded to nearest-even to `type`; with
 * accumulate 1 added to the dw that is there (in fp32).  A weight without rows
 * gets zeros (accumulate: stays as it is).  dw are weights [N][K]; where the
 * forward pass keeps [K][N], swap dy and x.  fp32 gradients dw_stride apart are
 * what ultraep_grad_reduce takes.
 *   dy         [M][N] bf16, x [M][K] bf16 (they may be the same)
 *   block_off, block_w, n_block  as for ultraep_expert_matmul_bf16
 *   dw         n_w gradients of N * K elements of `type`, dw_stride elements
 *              apart; what lies between them is not written; dw overlaps neither
 *              dy nor x
 *   ws         workspace of ws_bytes >= ultraep_expert_weight_grad_ws_bytes,
 *              16-byte aligned, or null: where the weights are few and small,
 *              their rows are summed in parts, side by side, with it (the
 *              result then differs in the order of the sums)
 * Equal calls give equal bits.  An unsound list raises ULTRAEP_EDATA as there;
 * then nothing is written to dw.
 * N, K % 8 == 0, 8 <= N, K <= 2^20, n_w <= 2^20, ceil(N / 64) * ceil(K / 64) *
 * n_w < 2^31, M < 2^31; N * K <= dw_stride <= 2^40, dw_stride % 8 == 0;
 * 16-byte aligned dy, x and dw. */
int ultraep_expert_weight_grad(const uint16_t *dy, const uint16_t *x, int64_t M, int32_t N,
                               int32_t K, const int64_t *block_off, const int32_t *block_w,
                               int32_t n_block, int32_t n_w, int64_t dw_stride,
                               int32_t accumulate, void *dw, int32_t type, void *ws,
                               size_t ws_bytes, int32_t *status, hipStream_t stream);

/* Bytes of that workspace for up to M rows (host only; 0 for unsupported
 * arguments, at least 16 otherwise). */
size_t ultraep_expert_weight_grad_ws_bytes(int64_t M, int32_t N, int32_t K, int32_t n_w);

/* Rows to 8-bit floating point (e4m3: 4 bits of exponent, 3 of mantissa, largest
 * 448, no infinities) with a power-of-two scale for each 128 elements.  In each
 * block of 128 (the row's last may be shorter), e is the least integer with
 * |x| <= 448 * 2^e throughout, -127 at least, and
 *   q = x * 2^-e rounded to nearest-even to e4m3,  scale byte = e + 127
 * (the value of q is q * 2^e; scale bytes are e8m0).  A block with an infinity
 * or a NaN has every q NaN (0x7F) and scale byte 255 (NaN).  A weight [n][N][K]
 * takes n * N rows.
 *   x      rows of K elements of `type`, ld elements apart
 *   q      rows of ldq bytes, ldq >= K: K values, then zeros
 *   scale  rows of 4 * ceil(K / 512) bytes: ceil(K / 128) scales, then zeros;
 *          4-byte aligned; q and scale do not overlap x
 * K, ld % 8 == 0, ldq % 16 == 0, ld, ldq <= 2^20, rows < 2^31, 16-byte aligned x
 * and q. */
int ultraep_quant_blocks(const void *x, int32_t type, int64_t rows, int64_t K, int64_t ld,
                         uint8_t *q, int64_t ldq, uint8_t *scale, hipStream_t stream);

/* The experts' products on such values.  Row m of block g meets weight
 * w = block_w[g]; with b = k / 128,
 *   v[n] = sum_k xq[m][k] * wq[w][n][k] * 2^(x_scale[m][b] + w_scale[w][n][b] - 254)
 * summed by the matrix unit, which applies the scales, in fp32 with what follows.
 * y[m] = v, or with act ULTRAEP_SWIGLU (as accurate as ultraep_expert_matmul_bf16's)
 *   y[m][n] = v[n] / (1 + exp(-v[n])) * v[N/2 + n],  n < N/2
 * rounded to nearest-even to `type`.
 *   bf16 results are sums of the unit's 8-bit products, of which it cuts 8
 * neighbours (k from a multiple of 8 on) 13 bits below the exponent of the largest
 * before it adds them.  Besides fp32's roundings v is then off by up to
 *   7 * 2^-13 * the sum over the 8s of max|x| * max|w|,  with their scales
 * whatever v itself is: the largest products set it, and where they cancel it may
 * be more than bf16's rounding, or than v.  Normal values, K = 7168: 1.5e-5 of the
 * results' norm before they are rounded, and 1 % of them more than 0.0036 off, with
 * the rounding, where the rounding alone is up to 2^-8; with every 512th channel of x
 * 100 times larger 1 % more than 0.0044.  What is lost of an 8 is below 2^-10 of its
 * largest product, whose factors' own roundings to e4m3 are up to 2^-4 each.
 *   For fp32 results the values are taken to bf16 (exactly, from 2^-126 in
 * magnitude to its largest, 2^128 - 2^120; what a scale takes above that is
 * infinite) and every product is exact and summed in fp32, at half the rate: a caller
 * whose sums may not be cut takes these and rounds them.
 *   A weight whose scales are held for blocks of 128 x 128 repeats each for 128 rows.
 *   xq         [M][K] e4m3, x_scale [M][4 * ceil(K / 512)] bytes
 *   wq         [n_w][N][K] e4m3, w_scale [n_w][N][4 * ceil(K / 512)] bytes
 *   block_off, block_w, n_block, y, errors  as for ultraep_expert_matmul
 * K % 16 == 0, N % 8 == 0 (N % 16 == 0 with act), 16 <= K <= 2^18, 8 <= N <= 2^20,
 * M < 2^31, M * N < 2^38; 16-byte aligned xq, wq and y, 4-byte aligned scales. */
int ultraep_expert_matmul_fp8(const uint8_t *xq, const uint8_t *x_scale, int64_t M,
                              const uint8_t *wq, const uint8_t *w_scale, int32_t n_w, int32_t N,
                              int32_t K, const int64_t *block_off, const int32_t *block_w,
                              int32_t n_block, int32_t act, void *y, int32_t type,
                              int32_t *status, hipStream_t stream);

/* Host only.  Static description of a status code. */
const char *ultraep_strerror(int code);

#ifdef __cplusplus
}
#endif

#endif /* ULTRAEP_H */
