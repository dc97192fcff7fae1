/*
 * railsched - batched LPT rail spraying of MoE all-to-all traffic on one AMD MI355X (gfx950).
 *
 * C ABI of the hot path of RailS (arXiv 2510.19262): router logits -> top-k routing ->
 * GPU-to-GPU byte matrix D^(1) -> fixed-size chunks -> per-node descending sort ->
 * greedy least-loaded-rail assignment -> per-NIC send/receive loads, completion time,
 * lower bound.  The rails are simulated arithmetically; nothing is transmitted.
 *
 * Notation (Section 4.1, System Model): M domains (nodes); N GPUs = NICs = rails per domain;
 * G = M*N GPUs; GPU id g = d*N + n, 0-based; C = chunk bytes; R2 = rate of one rail.
 * "batch" is the number of independent traffic matrices (e.g. MoE layers) processed in one call;
 * an *instance* is one (matrix b, source node k) pair, numbered b*M + k.  Instances are scheduled
 * independently: each node decides from local information only (Sections 1 and 3.2).
 *
 * Conventions
 *   - Every pointer is a DEVICE pointer unless its name starts with h_.  The caller owns every
 *     buffer (inputs, outputs, workspace); the library allocates nothing, keeps no state between
 *     calls (LoadState is reset for every all-to-all round, Section 5.2) and never frees anything.
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).  All work is enqueued
 *     asynchronously on it; no call but railsched_check_capacity synchronises the host with the device.
 *   - Every function returns 0 (RAILSCHED_OK) or a negative railsched_status.  Arguments are
 *     validated on the host before anything is launched; on an error nothing has been enqueued.
 *   - All outputs are integers and are defined bit-exactly, but for those of the operators on a router in training
 *     (railsched_route_logprobs, _balance, _distill and their gradients), which are defined by formulas.
 *   - Capacity.  Every call that reads or writes the per-chunk arrays (chunk_w, chunk_flow, perm, rail, port) takes
 *     `capacity`, the number of records those arrays hold.  The chunk count chunk_off[batch*M] exists on the device
 *     only; when it exceeds `capacity` the call touches none of the per-chunk arrays and fills its remaining outputs
 *     with -1 instead (S for stage 4, R and stats for stage 5, all three for railsched_schedule), so a caller that
 *     never synchronises still finds the overflow in whatever it reads back; chunk_off is complete either way.
 *     railsched_check_capacity reports the same condition to the host as RAILSCHED_ERR_CAPACITY.
 *   - Limits: 1 <= N <= 64, 1 <= M, G <= 16384, N*G <= 16384 for chunk_sort, 1 <= k <= E <= 1024,
 *     1 <= C < 2^32, every instance holds fewer than 2^32 chunks and fewer than 2^56 bytes.
 */
#ifndef RAILSCHED_H
#define RAILSCHED_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum railsched_status {
    RAILSCHED_OK = 0,
    RAILSCHED_ERR_INVALID_ARG = -1, /* a size or count is out of its documented range           */
    RAILSCHED_ERR_NULL_PTR    = -2, /* a required pointer is NULL                               */
    RAILSCHED_ERR_UNSUPPORTED = -3, /* valid in the paper's model but beyond this library's limits */
    RAILSCHED_ERR_CAPACITY    = -4, /* railsched_check_capacity: more chunks than the arrays hold */
    RAILSCHED_ERR_WORKSPACE   = -5, /* workspace missing or smaller than *_workspace_bytes()     */
    RAILSCHED_ERR_HIP         = -6, /* the HIP runtime refused a launch                          */
    RAILSCHED_ERR_SCRATCH     = -7  /* railsched_schedule_static: needs more than the static buffer */
} railsched_status;

/* Topology and chunking of the Rail fabric (Section 4.1; chunk size: Section 5.1, "Flow Splitting
 * and Atomicity").  Plain data, passed by HOST pointer. */
typedef struct railsched_topo {
    int32_t nodes;              /* M                                                             */
    int32_t rails;              /* N                                                             */
    int64_t chunk_bytes;        /* C                                                             */
    int64_t rail_bw_Bps;        /* R2 in bytes/s; only used by callers to turn bytes into time   */
    int32_t include_intra_node; /* 0: traffic inside a node is not inter-domain and is skipped   */
    int32_t reserved;           /* must be 0                                                     */
} railsched_topo_t;

const char *railsched_version(void);
const char *railsched_strerror(int status);

/* Waits until `stream` has drained, reads the chunk count chunk_off[batch*M] back and compares it with `capacity`
 * (Section 5.1: the number of atomic flows depends on the traffic, so record arrays sized ahead of time can turn
 * out too small).  The only call of the library that synchronises the host with the device.
 *   chunk_off [batch*M + 1] int64, as written by stage 3        (in)
 *   h_total   HOST pointer, receives the chunk count            (out, nullable)
 * Returns RAILSCHED_OK, RAILSCHED_ERR_CAPACITY (count > capacity; *h_total is still set), NULL_PTR, INVALID_ARG, HIP. */
int railsched_check_capacity(const int64_t *chunk_off, int32_t batch, const railsched_topo_t *h_topo, int64_t capacity,
                             int64_t *h_total, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Stage 1 - gating decision (Algorithm 1 step 1; Top-K expert selection of Section 6.3).
 * For every token row the indices of the k largest logits, largest first; equal logits (IEEE
 * comparison, so -0 == +0) are ordered by ascending expert index.  Logits must be finite.
 *   logits   [rows][E] fp32, row-major            (in)
 *   topk_idx [rows][k] int32                      (out)
 * rows may be 0.  Errors: NULL_PTR, INVALID_ARG (rows < 0, E < 1, k < 1, k > E), UNSUPPORTED (E > 1024).
 * ------------------------------------------------------------------------------------------- */
int railsched_route_topk(const float *logits, int64_t rows, int32_t E, int32_t k,
                         int32_t *topk_idx, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Stage 2 - GPU-to-GPU traffic matrix D^(1) (Section 4.1; Algorithm 1 step 2, selection of input
 * slices by gate and expert assignment).  Row r of matrix b belongs to source GPU
 * s = r / tokens_per_gpu; its slot j goes to GPU expert_gpu[topk_idx[r][j]][t mod R] with
 * t = r mod tokens_per_gpu (R replicas of every expert; R = 1 puts an expert on a single GPU);
 * every (token, slot) adds payload_bytes to D1[b][s][d].  A token whose slots hit the same GPU
 * counts once per slot.
 *   topk_idx   [batch*G*tokens_per_gpu][k] int32, values in [0,E)  (in; out-of-range values are ignored)
 *   expert_gpu [E][R] int32, values in [0,G)                        (in; same rule)
 *   D1         [batch][G][G] int64                                  (out, fully overwritten)
 *   ws         railsched_traffic_matrix_workspace_bytes(...) bytes of device memory, 4-byte aligned
 *              (scratch: destination counts of the slices a (matrix, source GPU) pair is cut into; summed in a
 *              fixed order by a second kernel, so no atomics leave the workgroups; contents undefined afterwards)
 * Errors: NULL_PTR, INVALID_ARG, UNSUPPORTED (G > 16384), WORKSPACE.
 * ------------------------------------------------------------------------------------------- */
size_t railsched_traffic_matrix_workspace_bytes(int32_t batch, int64_t tokens_per_gpu, int32_t k,
                                                const railsched_topo_t *h_topo);
int railsched_traffic_matrix(const int32_t *topk_idx, int32_t batch, int64_t tokens_per_gpu, int32_t k,
                             const int32_t *expert_gpu, int32_t E, int32_t R, int64_t payload_bytes,
                             const railsched_topo_t *h_topo, int64_t *D1, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Stages 1 and 2 in one call (Algorithm 1 steps 1-2: gate, then selection of input slices by gate
 * and expert assignment).  Same inputs, same rules and bit-identical outputs as
 * railsched_route_topk over all batch*G*tokens_per_gpu rows followed by railsched_traffic_matrix;
 * for E <= 8 both are produced in a single pass over the logits and the indices are never read back; so they are for
 * 8 < E <= 32 with k <= 8 when the indices are wanted, and so is D1 for 32 < E <= 256 with k <= 8 when they are not
 * (topk_idx == NULL); both need 16-byte aligned logits, E a multiple of 4 and G <= 8192 and 4096.  Everything else runs the
 * two stages.
 *   logits     [batch*G*tokens_per_gpu][E] fp32                     (in)
 *   expert_gpu [E][R] int32, values in [0,G)                        (in; out-of-range values are ignored)
 *   topk_idx   [batch*G*tokens_per_gpu][k] int32                    (out; may be NULL for the single-pass shapes:
 *                                                                    the picks are then counted but not stored)
 *   D1         [batch][G][G] int64                                  (out, fully overwritten)
 *   ws         railsched_route_traffic_workspace_bytes(...) bytes of device memory, 4-byte aligned
 *              (scratch: per-slice destination counts; contents undefined afterwards)
 * Errors: NULL_PTR (also topk_idx == NULL for a shape that runs the two stages), INVALID_ARG, UNSUPPORTED (E > 1024, G > 16384),
 * WORKSPACE (ws missing, misaligned or smaller than the query's answer).
 * ------------------------------------------------------------------------------------------- */
size_t railsched_route_traffic_workspace_bytes(int32_t batch, int64_t tokens_per_gpu, int32_t E, int32_t k,
                                               const railsched_topo_t *h_topo);
int railsched_route_traffic(const float *logits, int32_t batch, int64_t tokens_per_gpu, int32_t E, int32_t k,
                            const int32_t *expert_gpu, int32_t R, int64_t payload_bytes,
                            const railsched_topo_t *h_topo, int32_t *topk_idx, int64_t *D1, void *ws, size_t ws_bytes,
                            void *stream);

/* ---------------------------------------------------------------------------------------------
 * Stage 3 - flow splitting and LPT sorting (Section 5.1 "Flow Splitting and Atomicity";
 * Algorithm 2 steps 1-2).  For instance (b,k) the flows of node k's N GPUs are taken in canonical
 * order (local GPU n ascending, destination GPU ascending; destinations inside node k skipped
 * unless include_intra_node); a flow of B bytes yields floor(B/C) chunks of C bytes and one of
 * B mod C bytes if that is non-zero.  The instance's chunks are then ordered by descending weight,
 * ties by source GPU, destination GPU and position in the flow (a stable sort of the canonical list).
 *   D1         [batch][G][G] int64, entries >= 0                     (in)
 *   chunk_off  [batch*M + 1] int64: exclusive scan of instance sizes (out)
 *   chunk_w    [capacity] uint32: chunk weight in bytes              (out, nullable)
 *   chunk_flow [capacity] uint32: n*G + destination GPU              (out)
 *   perm       [capacity] uint32: canonical position inside the instance of the chunk now at this
 *              sorted position                                      (out, nullable)
 * With chunk_w == NULL only chunk_off is produced (a count query: railsched_check_capacity then
 * returns the total to size the record arrays with).  If the total chunk count exceeds `capacity`
 * the record arrays are left untouched and chunk_off is still complete.
 * Workspace: railsched_chunk_sort_workspace_bytes(batch, topo) bytes, 256-byte aligned.
 * Errors: NULL_PTR, INVALID_ARG, UNSUPPORTED (N*G > 16384, C >= 2^32), WORKSPACE.
 * ------------------------------------------------------------------------------------------- */
size_t railsched_chunk_sort_workspace_bytes(int32_t batch, const railsched_topo_t *h_topo);
int railsched_chunk_sort(const int64_t *D1, int32_t batch, const railsched_topo_t *h_topo,
                         int64_t *chunk_off, uint32_t *chunk_w, uint32_t *chunk_flow, uint32_t *perm,
                         int64_t capacity, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Stage 4 - LPT iterative allocation (Algorithm 2, initialisation and step 3).  Per instance:
 * LoadState[0..N) = 0; for every chunk in stored order j* = the lowest-numbered rail of minimum
 * LoadState; rail[i] = j*; LoadState[j*] += w_i.  The final LoadState is the send load S[b][k][.]
 * (Section 4.1, load matrix S).  Weights need not come from stage 3: any sequence is scheduled in
 * the order given (the guarantees of Theorem 4 need it non-increasing).
 *   chunk_off [batch*M + 1] int64   (in)
 *   chunk_w   [capacity] uint32     (in; the first chunk_off[batch*M] are read)
 *   rail      [capacity] uint8, values in [0,N)            (out; the first chunk_off[batch*M] are written)
 *   S         [batch][M][N] int64                          (out; every entry -1 if chunk_off[batch*M] > capacity,
 *                                                           and then chunk_w is not read and rail not written)
 *   ws        optional (NULL, 0 = none): railsched_lpt_spray_workspace_bytes(batch, topo) bytes, 256-byte aligned.
 *             Instances are independent (Sections 1 and 3.2), so the order they are worked on is free: with a
 *             workspace, batches of thousands of instances are taken longest chain first from a queue (the few far
 *             longer than the rest on a wavefront of their own), which evens out the load of the SIMDs; the outputs
 *             do not depend on it.  It pays for railsched_lpt_spray_chunkwise; railsched_lpt_spray, whose chains
 *             are what the closed forms leave over, accepts it and leaves it unused.
 * Errors: NULL_PTR, INVALID_ARG, UNSUPPORTED (N > 64), WORKSPACE (ws given but misaligned or too small).
 * ------------------------------------------------------------------------------------------- */
size_t railsched_lpt_spray_workspace_bytes(int32_t batch, const railsched_topo_t *h_topo);
int railsched_lpt_spray(const int64_t *chunk_off, const uint32_t *chunk_w, int32_t batch,
                        const railsched_topo_t *h_topo, int64_t capacity, uint8_t *rail, int64_t *S, void *ws,
                        size_t ws_bytes, void *stream);

/* Same function, same arguments, same outputs bit for bit (Algorithm 2 step 3), but every single chunk
 * goes through the cross-lane argmin; railsched_lpt_spray above additionally assigns whole periods of
 * equal-weight chunks in closed form when the rail loads are within one weight of each other (the
 * bound L_max <= L_opt + w_max of the Theorem 4 proof is what makes that state the common one).
 * Kept as the plain reference kernel for measurements and cross-checks. */
int railsched_lpt_spray_chunkwise(const int64_t *chunk_off, const uint32_t *chunk_w, int32_t batch,
                                  const railsched_topo_t *h_topo, int64_t capacity, uint8_t *rail, int64_t *S, void *ws,
                                  size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Stage 5 - load evaluation (Section 4.1 load matrices S and R; Theorem 2; Theorem 3).
 * Rail n of a source node ends on NIC n of the destination node, so a chunk whose destination GPU
 * lies in node f and that was put on rail n adds its weight to R[b][f][n].
 *   R     [batch][M][N] int64                                   (out)
 *   stats [batch][8] int64                                      (out)
 *     [0] makespan = max over all entries of S[b] and R[b]  (Theorem 2: T = makespan / R2)
 *     [1] max send load   [2] max receive load
 *     [3] lower bound max( max_k ceil(sum_n S[b][k][n] / N), max_f ceil(sum_n R[b][f][n] / N), w_max )
 *         (uniform split of Theorem 3; one chunk is indivisible, Theorem 4 proof)
 *     [4] total bytes scheduled  [5] w_max  [6] chunk count
 *     [7] max over nodes k of (max_n S[b][k][n] - min_n S[b][k][n])
 * S is read as produced by stage 4.  No global atomics are used (the bins of a workgroup are
 * LDS-private integer atomics): every workgroup writes its partial receive loads to the workspace
 * and a second kernel adds them in a fixed order.
 * chunk_w, chunk_flow, rail hold `capacity` records; if chunk_off[batch*M] > capacity none of them is
 * read and every entry of R and stats is -1.
 * Workspace: railsched_eval_workspace_bytes(batch, topo) bytes, 256-byte aligned.
 * Errors: NULL_PTR, INVALID_ARG, UNSUPPORTED, WORKSPACE.
 * ------------------------------------------------------------------------------------------- */
size_t railsched_eval_workspace_bytes(int32_t batch, const railsched_topo_t *h_topo);
int railsched_eval(const int64_t *chunk_off, const uint32_t *chunk_w, const uint32_t *chunk_flow,
                   const uint8_t *rail, const int64_t *S, int32_t batch, const railsched_topo_t *h_topo,
                   int64_t capacity, int64_t *R, int64_t *stats, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Stages 3-5 in one call (Algorithm 2 steps 1-3 and 6; Section 4.1 S and R; Theorems 2-3): the outputs of
 * railsched_chunk_sort, railsched_lpt_spray and railsched_eval run one after the other on the same
 * arguments, bit for bit, with less work: stage 3 knows that every instance starts with a run of full chunks,
 * whose allocation from empty rails is round robin, so their rails are written with the records, stage 4 only
 * runs behind them and stage 5 takes their receive loads in closed form.  Batches of at most 1024 instances
 * with N*G <= 2048 flows (256 with N*G <= 4096) and capacity <= 65536 chunks per instance (131072 for at most 256
 * instances) are served by one workgroup per instance (two launches after the counts instead of six), which leaves the
 * full chunks of instances far longer than the rest to further workgroups of its launch.
 *   D1 [batch][G][G] int64 (in);  chunk_off [batch*M+1];  chunk_w, chunk_flow, perm (perm may be NULL),
 *   rail: `capacity` records each;  S, R [batch][M][N] int64;  stats [batch][8] int64   (out)
 *   ws: railsched_schedule_workspace_bytes(batch, topo) bytes, 256-byte aligned.
 * If chunk_off[batch*M] > capacity the record arrays are left alone and every entry of S, R and stats is -1.
 * Errors: NULL_PTR, INVALID_ARG, UNSUPPORTED (as the three stages), WORKSPACE.
 * ------------------------------------------------------------------------------------------- */
size_t railsched_schedule_workspace_bytes(int32_t batch, const railsched_topo_t *h_topo);
int railsched_schedule(const int64_t *D1, int32_t batch, const railsched_topo_t *h_topo, int64_t *chunk_off,
                       uint32_t *chunk_w, uint32_t *chunk_flow, uint32_t *perm, int64_t capacity, uint8_t *rail,
                       int64_t *S, int64_t *R, int64_t *stats, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * railsched_schedule for callers that cannot allocate device memory or carry a workspace around: code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation.  Same arguments without the
 * workspace, same outputs bit for bit; the workspace is an array of RAILSCHED_STATIC_SCRATCH_BYTES bytes inside
 * the library's device image (every GPU the library runs on holds its own copy until the process ends).  The
 * call allocates and frees nothing; the first call on a device asks the runtime for the array's address there.
 * Batches whose railsched_schedule_workspace_bytes(batch, topo) exceeds RAILSCHED_STATIC_SCRATCH_BYTES are
 * refused with RAILSCHED_ERR_SCRATCH before anything is enqueued (4 MiB covers e.g. 32 matrices of 8 nodes x
 * 8 rails, or 1024 matrices of 4 x 4).
 * All calls on one GPU share that GPU's array: calls that can overlap there (different streams, or several
 * host threads) race on it and must be ordered by the caller; on one stream they are ordered already.
 * Errors: as railsched_schedule without WORKSPACE, plus SCRATCH, and HIP when the device has no such array.
 * ------------------------------------------------------------------------------------------- */
#define RAILSCHED_STATIC_SCRATCH_BYTES (4u << 20)
int railsched_schedule_static(const int64_t *D1, int32_t batch, const railsched_topo_t *h_topo, int64_t *chunk_off,
                              uint32_t *chunk_w, uint32_t *chunk_flow, uint32_t *perm, int64_t capacity, uint8_t *rail,
                              int64_t *S, int64_t *R, int64_t *stats, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Second all-to-all of an MoE layer (Algorithm 1 step 4: expert outputs return to the token owners):
 * its traffic is the first one's reversed, D1T[b][d][s] = D1[b][s][d]; stages 3-5 then run on D1T.
 *   D1, D1T [batch][G][G] int64, distinct buffers.
 * Errors: NULL_PTR, INVALID_ARG (also D1 == D1T), UNSUPPORTED.
 * ------------------------------------------------------------------------------------------- */
int railsched_transpose_matrix(const int64_t *D1, int32_t batch, const railsched_topo_t *h_topo, int64_t *D1T,
                               void *stream);

/* ---------------------------------------------------------------------------------------------
 * The path-selection schemes RailS is compared with (Sections 1, 2.2 and 6.1), reduced to arithmetic
 * on the chunk records of stage 3: same inputs and outputs as stage 4, another rule for the rail.
 *   RAILSCHED_POLICY_NIC_DIRECT   a GPU's traffic leaves through its own NIC: rail = flow id div G
 *   RAILSCHED_POLICY_FLOW_HASH    static per-flow hashing (ECMP-like): hash(instance*N*G + flow id) mod N
 *   RAILSCHED_POLICY_RANDOM_SPRAY per chunk: hash(index of the chunk in the record arrays) mod N
 *   RAILSCHED_POLICY_ROUND_ROBIN  chunk i of the instance, in stored order, takes rail i mod N
 * hash(x) = splitmix64 finaliser of (seed + 0x9E3779B97F4A7C15 * (x + 1)), 64-bit wrapping.
 *   rail [capacity] uint8 (out), S [batch][M][N] int64 send loads (out); feed both to railsched_eval.
 * If chunk_off[batch*M] > capacity the per-chunk arrays are left alone and every entry of S is -1.
 * Errors: NULL_PTR, INVALID_ARG (unknown policy), UNSUPPORTED.
 * ------------------------------------------------------------------------------------------- */
enum { RAILSCHED_POLICY_NIC_DIRECT = 0, RAILSCHED_POLICY_FLOW_HASH = 1, RAILSCHED_POLICY_RANDOM_SPRAY = 2,
       RAILSCHED_POLICY_ROUND_ROBIN = 3 };
int railsched_assign_policy(int32_t policy, uint64_t seed, const int64_t *chunk_off, const uint32_t *chunk_w,
                            const uint32_t *chunk_flow, int32_t batch, const railsched_topo_t *h_topo,
                            int64_t capacity, uint8_t *rail, int64_t *S, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Spraying execution, port choice (Algorithm 2 step 4: round-robin port choice inside the chosen NIC):
 * each rail of a node hands its chunks to its `ports` queue pairs in turn; the chunk that is the c-th
 * one (c = 0, 1, ...) put on its rail inside its instance, in stored order, takes port c mod ports.
 *   rail [chunks] uint8 (in), port [chunks] uint8 (out), 1 <= ports <= 256.
 * `capacity` is the number of records rail and port hold and sizes the workspace:
 * railsched_port_round_robin_workspace_bytes(batch, topo, capacity) bytes, 256-byte aligned.
 * If chunk_off[batch*M] exceeds capacity, rail is not read and port not written.
 * Errors: NULL_PTR, INVALID_ARG, UNSUPPORTED (ports > 256), WORKSPACE.
 * ------------------------------------------------------------------------------------------- */
size_t railsched_port_round_robin_workspace_bytes(int32_t batch, const railsched_topo_t *h_topo, int64_t capacity);
int railsched_port_round_robin(const int64_t *chunk_off, const uint8_t *rail, int32_t batch,
                               const railsched_topo_t *h_topo, int32_t ports, int64_t capacity, uint8_t *port,
                               void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Operators on the logits of a router in training (the "Gate" of Algorithm 1 step 1).  They read the same rows of
 * logits as stage 1 and, like stage 2, its picks; their outputs are floating point and are defined by the formulas
 * below, evaluated in fp32 (sums over rows in fp32 per part and in fp64 over the parts), with one rounding to the
 * type of the logits where a gradient has that type.  The order of every sum is fixed: equal inputs give equal bits.
 *
 * Common to all of them:
 *   logits    rows of E values of type `dtype` (railsched_dtype), row r at logits + r*ld elements, ld >= E    (in)
 *             A logit may be -infinity: that expert is out for this row (probability 0).  A row with NaN or
 *             +infinity makes NaN of the floating outputs it enters and of no others.
 *   row_mask  [rows] uint8, NULL = all rows count.  A row whose entry is 0 (padding) does not count, and neither does a
 *             row whose logits are all -infinity: whatever a masked row holds enters nothing, its picks are not counted, its
 *             floating outputs and its gradient are 0, its alternatives -1.
 *   temperature  tau, within 2^-60 .. 2^60 (distillation: 2^-8 .. 2^8): z = logits / tau, p = softmax(z) over the row, lse = log sum exp z.
 *   d_logits  the gradient, type `dtype`, row r at d_logits + r*ld_d, ld_d >= E; not the same memory as logits.  Places
 *             between the rows are left as they are.  accumulate = 0: overwritten; 1: added to what is there (each
 *             sum rounded to `dtype`; rows that do not count are left as they are).
 *   An index outside [0,E) is ignored.
 * Limits: E <= 1024, k, m and K <= E, m and K <= 64, rows < 2^31, ld and ld_d <= 2^31, groups <= 2^23.  rows may be 0 (nothing is written but the groups' outputs).
 * Errors: NULL_PTR, INVALID_ARG (sizes, ld < E, unknown dtype, temperature out of range, accumulate not 0 or 1 (or 2 where it says so),
 * d_logits == logits), UNSUPPORTED (limits), WORKSPACE.
 * ------------------------------------------------------------------------------------------- */
typedef enum railsched_dtype { RAILSCHED_F32 = 0, RAILSCHED_BF16 = 1, RAILSCHED_F16 = 2 } railsched_dtype;

/* Log probabilities of given experts, with log-sum-exp, entropy and the most likely experts of every row.
 *   topk_idx  [rows][k] int32: the experts asked for (stage 1's picks, or another router's); NULL iff k == 0   (in)
 *   logp      [rows][k] fp32: z[topk_idx] - lse; exp(logp) is the gate weight of the pick; 0 where ignored      (out)
 *   lse       [rows] fp32                                                                                     (out, nullable)
 *   entropy   [rows] fp32: -sum p log p                                                                       (out, nullable)
 *   alt_idx   [rows][m] int32: the experts of the m largest logits in stage 1's order; -1 where fewer are left (out; NULL iff m == 0).
 *             NaN is no number and never among them; +infinity is
 *   alt_logp  [rows][m] fp32: their z - lse; -infinity where alt_idx is -1 in a row that counts               (out; NULL iff m == 0)
 * The logits of a row are read once; the picks' logits are fetched from the cache. */
int railsched_route_logprobs(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, float temperature,
                             const uint8_t *row_mask, const int32_t *topk_idx, int32_t k, int32_t m, float *logp, float *lse,
                             float *entropy, int32_t *alt_idx, float *alt_logp, void *stream);

/* Its gradient: d_logits[e] = (sum over slots j of e of d_logp[j] - p_e (sum over slots of d_logp - d_lse
 * + d_entropy (log p_e + entropy))) / tau.  d_lse carries a loss on lse (its square: the z-loss).
 *   d_logp [rows][k], d_lse [rows], d_entropy [rows] fp32 (in, each nullable = 0; d_logp NULL if k == 0) */
int railsched_route_logprobs_backward(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, float temperature,
                                      const uint8_t *row_mask, const int32_t *topk_idx, int32_t k, const float *d_logp,
                                      const float *d_lse, const float *d_entropy, int32_t accumulate, void *d_logits, int64_t ld_d,
                                      void *stream);

/* Balance loss of groups of rows (layers, sequences, micro-batches), with the counts of picks per expert.  Group g
 * holds the rows [group_off[g], group_off[g+1]), or with group_off NULL the g-th of `groups` equal parts of the rows.
 * With n its rows that count, c_e its picks of expert e and P_e the sum of p_e over its rows that count:
 *   loss[g] = coef * E / (k n^2) * sum_e c_e P_e        (0 if n == 0; temperature 1)
 * which is coef where picks and probabilities are spread evenly.
 *   group_off [groups+1] int64, not decreasing, within [0, rows]; nullable      (in; values outside are clamped)
 *   topk_idx  [rows][k] int32                                                   (in)
 *   counts    [groups][E] int64: c_e                                            (out)
 *   tokens    [groups] int64: n                                                 (out)
 *   prob_sum  [groups][E] fp32: P_e                                             (out)
 *   loss      [groups] fp32                                                     (out)
 *   ws        railsched_route_balance_workspace_bytes(rows, groups, E) bytes, 256-byte aligned (contents undefined before and after; calls
 *             that can run at the same time, captured graphs among them, need one each)
 * Errors as above, also INVALID_ARG where group_off is NULL and rows is not a multiple of groups, groups < 0, k < 1. */
size_t railsched_route_balance_workspace_bytes(int64_t rows, int32_t groups, int32_t E);
int railsched_route_balance(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, const uint8_t *row_mask,
                            const int32_t *topk_idx, int32_t k, const int64_t *group_off, int32_t groups, float coef,
                            int64_t *counts, int64_t *tokens, float *prob_sum, float *loss, void *ws, size_t ws_bytes, void *stream);

/* Its gradient through the probabilities (the counts are constants): with a_e = d_loss[g] coef E c_e / (k n^2),
 * d_logits[e] = p_e (a_e - sum_f a_f p_f).  counts and tokens are inputs: a caller that adds them up over ranks first trains on
 * the balance of all of them.  Rows of no group are left as they are, but set to 0 with accumulate = 2, which is 0 otherwise
 * (with groups = 0 and group_off given that is every row; counts, tokens and d_loss may be NULL then).
 *   counts [groups][E] int64, tokens [groups] int64, d_loss [groups] fp32       (in) */
int railsched_route_balance_backward(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, const uint8_t *row_mask,
                                     int32_t k, const int64_t *group_off, int32_t groups, float coef, const int64_t *counts,
                                     const int64_t *tokens, const float *d_loss, int32_t accumulate, void *d_logits, int64_t ld_d,
                                     void *stream);

/* Distillation: the divergence of a router from the top logits of another one (the teacher), so that a forecaster of the
 * routing can be trained before it feeds stage 1.  The teacher's list of a row is (t_idx[j], t_logit[j]), j < K; an entry
 * with an index outside [0,E) or the logit -infinity is absent.  Its probabilities are
 *   without t_lse: q = softmax(t_logit / tau) over the list;
 *   with t_lse:    q = exp(t_logit / tau - t_lse), t_lse the teacher's log-sum-exp over all its experts at this temperature, and the
 *                  rest q_r = max(0, 1 - sum q) is held against p_r, the sum of p outside the list (left out where p_r is 0: below 2^-126).
 *   loss[r] = tau^2 (sum_j q_j (log q_j - log p[t_idx[j]]) + q_r (log q_r - log p_r))
 * A row without entries has the loss 0 (also with t_lse).  +infinity where q_j > 0 meets an expert that is out.
 * An expert listed twice counts with the sum of its entries' terms.
 * temperature is within 2^-8 .. 2^8: log p - log q, from which loss and gradient are formed, is off by a few 2^-24 of 1 + |logit - t_logit| / tau + |t_lse|, while it is
 * itself of order 1 / tau for a large tau.  Where student and teacher differ by about 1 that is up to about 2^-11 of a row's gradient at 2^8, and 2^-14 of tau d_loss at 2^-8.  t_lse counts as the
 * number that it is in fp32 (with a list that leaves p no rest, half a step of t_lse changes the loss by tau^2 times that).
 *   t_idx [rows][K] int32, t_logit [rows][K] fp32, t_lse [rows] fp32 (nullable)  (in; alt_idx and alt_logp of railsched_route_logprobs
 *                                                                                will do, with t_lse = 0 at temperature 1)
 *   loss  [rows] fp32                                                            (out) */
int railsched_route_distill(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, float temperature,
                            const uint8_t *row_mask, const int32_t *t_idx, const float *t_logit, const float *t_lse, int32_t K,
                            float *loss, void *stream);

/* Its gradient: with Q = sum q, d_logits[e] = tau d_loss (p_e (Q + q_r) - sum over entries of e of q) in the list and
 * tau d_loss p_e (Q + q_r - q_r / p_r) outside (without t_lse, or where p_r is 0: q_r = 0).
 *   d_loss [rows] fp32 (in) */
int railsched_route_distill_backward(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, float temperature,
                                     const uint8_t *row_mask, const int32_t *t_idx, const float *t_logit, const float *t_lse, int32_t K,
                                     const float *d_loss, int32_t accumulate, void *d_logits, int64_t ld_d, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* RAILSCHED_H */
