/*
 * poseidon.h -- C ABI of libposeidon.so: batched evaluation of Poseidon's
 * DAG training-time model and the exact parallelism search built on it,
 * on one GB300 (sm_103a).
 *
 * Model (paper Sec. 4.1): for a pipeline of N = S stages and M micro-batches
 * the DAG has nodes F_{s,m}, B_{s,m} (Sec. 4.1.1), inter-stage edges
 * F_{s,m} -> F_{s+1,m} and B_{s+1,m} -> B_{s,m}, an intra-stage chain in 1F1B
 * order, B_{s,M} -> R_s and R_s -> E (Sec. 4.1.2).  Node weights are the
 * per-layer times summed over the stage's layers, inter-stage edges carry the
 * activation-transfer time, R_s the gradient all-reduce time (Sec. 4.1.3).
 * The makespan T is the longest path: T = max_s (finish(B_{s,M}) + d_s).
 *
 * Conventions shared by every entry point:
 *  - every call returns a pos_status; no C++ exception crosses the ABI;
 *    poseidon_last_error() describes the last failure of the calling thread;
 *  - the caller owns every buffer it passes; the library copies what it keeps;
 *  - costs are int32 microseconds, memory int64 bytes; the planner's
 *    arithmetic is integer, so its results are exact and reproducible;
 *  - class k = type * n_tp + tp_idx indexes every per-class table.
 */
#ifndef POSEIDON_H
#define POSEIDON_H
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t pos_status;
#define POS_OK 0
#define POS_EINVAL 1        /* bad argument, table or problem */
#define POS_EOVERFLOW 2     /* a makespan could exceed int32 (guard below) */
#define POS_ENOMEM 3        /* device or host allocation failed */
#define POS_ECUDA 4         /* a CUDA runtime call failed */
#define POS_ETIMEOUT 5      /* a bounded device loop hit its iteration limit */
#define POS_EINFEASIBLE 6   /* the search space has no memory-feasible plan */
#define POS_ENOTIMPL 7

/* Pipeline schedules (the intra-stage order of Sec. 4.1.2).  Stage s
 * (1-based) of N runs W_s forwards, then (B_i, F_{W_s+i}) for
 * i = 1..M-W_s, then the remaining backwards, and holds the activations of
 * W_s micro-batches at once:
 *   POS_SCHED_1F1B        W_s = min(N-s+1, M)
 *   POS_SCHED_EAGER_1F1B  W_s = min(2(N-s)+1, M)   (Eager 1F1B, App. B)
 *   POS_SCHED_INTERLEAVED_1F1B  Interleaved 1F1B (Sec. 4.1.4) for candidates
 *       whose V field is >= 2, 1F1B for the others.  The S = N devices each
 *       hold V model chunks; the L layers are split over the J = N*V
 *       virtual stages in order, virtual stage j (0-based) being chunk j / N
 *       on device j % N, so the DAG has 2VNM compute nodes, 2(NV-1)M
 *       inter-stage and N(2VM-1) intra-stage edges.  M must be a multiple
 *       of N.  Device d (0-based) runs the interleaved order of Narayanan et
 *       al. (2021), which the paper cites: its k-th forward (k = 0..VM-1)
 *       is chunk (k mod NV) / N of micro-batch (k / NV)*N + k mod N, its
 *       k-th backward chunk V-1 - (k mod NV) / N of the same micro-batch;
 *       it runs w_d = min(2(N-d-1) + (V-1)N, VM) forwards (all VM when
 *       M = N), then alternates one forward and one backward, then runs
 *       the remaining backwards.  Memory: the largest sum of activations
 *       the device holds along that order (a forward of chunk c adds its
 *       mem_a, the matching backward releases it) plus the mem_w of all its
 *       chunks must fit cap of its class.  The edge between virtual stages
 *       j and j+1 uses the classes of their devices (p2p_f[k_{j%N}][k_{(j+1)%N}],
 *       p2p_b[k_{(j+1)%N}][k_{j%N}]); R_d sums dsync over the device's chunks
 *       and follows its last op.  poseidon_eval_batch evaluates such
 *       records; poseidon_search searches over them (pos_problem.V). */
#define POS_SCHED_1F1B 0
#define POS_SCHED_EAGER_1F1B 1
#define POS_SCHED_INTERLEAVED_1F1B 2

#define POS_PLACE_FREE 0    /* any device type on any stage */
#define POS_PLACE_EXACT 1   /* exactly type_counts[t] stages of type t */
#define POS_PLACE_DEVICES 2 /* a (device type, TP index) per stage; the stages of
                               type t use exactly type_counts[t] devices: the sum
                               over them of D * tp_list[tp index] (per-stage TP) */

#define POS_MAX_STAGES 16
#define POS_MAX_LAYERS 127
#define POS_MAX_TYPES 4
#define POS_MAX_TP 8

/*
 * Profiled cost tables (Sec. 3.2 and Sec. 4.1.3), host pointers, row-major:
 *   fwd, bwd, dsync [K][L]   per-layer forward, backward and DP all-reduce
 *                            time in us (>= 0);
 *   p2p_f, p2p_b    [K][K]   activation / gradient transfer time per
 *                            micro-batch, indexed [sending class][receiving
 *                            class]; the F edge s->s+1 uses p2p_f[k_s][k_s+1],
 *                            the B edge s+1->s uses p2p_b[k_s+1][k_s];
 *   mem_w, mem_a    [K][L]   bytes per layer: resident (weights, optimizer)
 *                            and activations per in-flight micro-batch (>= 0);
 *   cap             [K]      device memory per class, bytes.
 * A stage s (1-based) holding layers [a, b) on class k fits when
 *   sum mem_w + W_s * sum mem_a <= cap[k],   W_s = min(S - s + 1, M),
 * W_s being the 1F1B in-flight micro-batches of that stage.
 * Limits: 1 <= L <= 127, 1 <= n_types <= 4, 1 <= n_tp <= 8, and per class
 * sum_l (fwd + bwd) and sum_l dsync below 2^31.
 */
typedef struct pos_tables {
    int32_t L, n_types, n_tp;
    const int32_t *fwd, *bwd, *dsync;
    const int32_t *p2p_f, *p2p_b;
    const int64_t *mem_w, *mem_a;
    const int64_t *cap;
} pos_tables;

/*
 * One encoded candidate plan, 16 bytes:
 *   map_rank   lexicographic rank of the layer composition (l_1..l_S) among
 *              all C(L-1, S-1) compositions of L into S non-empty stages;
 *              rank 0 = (1, ..., 1, L-S+1);
 *   type_code  device type of stage s (0-based) in bits [2s, 2s+2);
 *   S          stages (1..16), M micro-batches (1..255), tp_idx < n_tp;
 *   V          model chunks per device under POS_SCHED_INTERLEAVED_1F1B
 *              (V >= 2: S is the device count N, map_rank ranks the
 *              composition of L into the J = S*V virtual stages among
 *              C(L-1, J-1), J <= 16, and M must be a multiple of S);
 *              ignored by the other schedules and when V < 2.
 */
typedef struct pos_candidate {
    uint64_t map_rank;
    uint32_t type_code;
    uint8_t S, M, tp_idx, V;
} pos_candidate;

/*
 * A candidate whose stages may use different TP indices (the per-stage
 * heterogeneous TP of the Metis and HexiScale plans in the paper's Table 1),
 * 24 bytes:
 *   map_rank, type_code, S, M, V   as in pos_candidate;
 *   tp_code    TP index of stage s (0-based; of device s for interleaved
 *              records) in bits [2s, 2s+2), so the class of stage s is
 *              type_s * n_tp + tp_s; needs n_tp <= 4.
 * The tables' TP axis may stand for any per-stage parallel setting (TP
 * degree, and the data-parallel degree of the stage's all-reduce and
 * memory); every stage still runs the pipeline's M micro-batches.
 */
typedef struct pos_candidate_ex {
    uint64_t map_rank;
    uint32_t type_code;
    uint32_t tp_code;
    uint8_t S, M, V, pad0;
    uint32_t pad1;
} pos_candidate_ex;

/* feasible[] codes written by poseidon_eval_batch */
#define POS_FEAS_NO 0        /* some stage exceeds its memory capacity */
#define POS_FEAS_YES 1
#define POS_FEAS_INVALID 2   /* a field is out of range; makespan = -1 */
#define POS_FEAS_OVERFLOW 3  /* guard U(S,M) >= 2^31; makespan = -1 */

/*
 * Overflow guard: every DAG path visits each node once, so
 *   T <= U(S,M) = M * sum_l max_k (fwd + bwd) + sum_l max_k dsync
 *                 + 2 M (S-1) max_{k,k'} max(p2p_f, p2p_b).
 * Candidates with U(S,M) >= 2^31 are not evaluated.
 */

/*
 * Copy the tables to the current CUDA device and build the per-class
 * exclusive prefix sums used by every kernel (hot-path step a1, Sec. 4.1.3)
 * and, when it takes at most 32 KB, a byte table of each class's largest
 * memory-feasible stage end per start layer and in-flight count (the
 * evaluator's memory check).
 * *handle owns the device copies until poseidon_tables_destroy.  schedule
 * (POS_SCHED_1F1B, POS_SCHED_EAGER_1F1B or POS_SCHED_INTERLEAVED_1F1B)
 * applies to every evaluation through the handle.
 * Errors: POS_EINVAL (null pointer, limits, negative cost or memory),
 * POS_EOVERFLOW (a class's summed costs reach 2^31), POS_ENOTIMPL (schedule),
 * POS_ENOMEM, POS_ECUDA.
 */
pos_status poseidon_tables_create(const pos_tables *tables, int32_t schedule, void **handle);
pos_status poseidon_tables_destroy(void *handle);

/*
 * Evaluate n candidates: makespan (Sec. 4.1) and memory feasibility
 * (Sec. 3.2).  d_cands (16-byte aligned), d_makespan (int32[n]) and
 * d_feasible (uint8[n]) are DEVICE pointers on the handle's device; outputs
 * are in input order; the call is asynchronous on `stream` (a cudaStream_t,
 * NULL = legacy default stream) and returns after the launches.  Part of the
 * work runs on library-owned side streams of the device, forked from
 * `stream` after the sort and joined back into it before the call's last
 * operation, so every effect is still ordered after earlier work on
 * `stream` and before later work on it.  Infeasible
 * plans still get their makespan.  Scratch: the batch is counting-sorted by
 * S and M (and by (N, V, M/N) for interleaved records) and decoded into a
 * 38*n + 13 KB (Interleaved 1F1B: 38*n + 78 KB) stream-ordered allocation
 * (decoded record 32 B, sorted position 4 B and sort key 2 B per candidate,
 * key histograms) from a library-owned memory pool (per device, kept
 * between calls); batches above 2^24 candidates go in chunks of 2^24, one
 * after another.
 * Errors: POS_EINVAL (null handle or pointers, n < 0, misaligned
 * candidates), POS_ENOMEM, POS_ECUDA (launch failure).
 */
pos_status poseidon_eval_batch(void *handle, const pos_candidate *d_cands, int64_t n,
                               int32_t *d_makespan, uint8_t *d_feasible, void *stream);

/*
 * poseidon_eval_batch for 24-byte pos_candidate_ex records (a TP index per
 * stage): same outputs, flags, schedules, scratch and stream semantics;
 * a record whose TP field of some stage s < S is >= n_tp is flagged
 * POS_FEAS_INVALID.  d_cands must be 8-byte aligned.
 * Errors: those of poseidon_eval_batch, and POS_EINVAL when the handle's
 * tables have n_tp > 4.
 */
pos_status poseidon_eval_batch_ex(void *handle, const pos_candidate_ex *d_cands, int64_t n,
                                  int32_t *d_makespan, uint8_t *d_feasible, void *stream);

/*
 * Same as poseidon_eval_batch but with HOST buffers: copies the candidates
 * to the device, evaluates, copies the results back and synchronises.
 * Takes n*21 bytes from the library's memory pool for the duration of the
 * call (the default stream orders the work).
 */
pos_status poseidon_eval_batch_host(void *handle, const pos_candidate *cands, int64_t n,
                                    int32_t *makespan, uint8_t *feasible);

/*
 * Deterministic argmin over eval_batch outputs (hot-path step a9): the
 * smallest makespan among entries with feasible == 1, ties broken to the
 * lowest index.  Device pointers; *d_out (int64, device) receives the index
 * or -1 when no entry is feasible.  Asynchronous on `stream`; above 16384
 * entries it uses a stream-ordered scratch allocation of at most 16 bytes per
 * SM * 4 from the library's pool (per device, kept between calls).
 */
pos_status poseidon_argmin(const int32_t *d_makespan, const uint8_t *d_feasible, int64_t n,
                           int64_t *d_out, void *stream);

/*
 * poseidon_argmin_noalloc: same inputs, output and result as poseidon_argmin,
 * for callers that cannot allocate device memory during a call -- a process
 * whose device memory belongs to another allocator (a framework's caching
 * allocator holding the free memory, or a service that reserves everything
 * at start-up and forbids allocation afterwards).  The paper has no
 * counterpart; this is a library convenience.
 * It allocates nothing: its per-block partial results live in a fixed
 * 64 KB array of device global memory (4096 partial results) that every GPU
 * loading the library holds until the process exits.  The first call on a
 * device looks up that array's device address (cudaGetSymbolAddress) with
 * the device current; make that first call before any stream capture.
 * That address is kept for the life of the process: do not use the
 * library across a cudaDeviceReset (the array may move when the module is
 * loaded again).
 * All calls on a device share the array and it keeps the last call's
 * contents (every slot a call reads is written earlier in the same call, so
 * nothing needs clearing); calls that overlap on the GPU, e.g. on two
 * streams at once, race on it.  Errors: POS_EINVAL for bad arguments or
 * when the GPU would need more than 4096 partial results (more than 1024
 * SMs), POS_ECUDA for a failed address lookup or launch.
 */
pos_status poseidon_argmin_noalloc(const int32_t *d_makespan, const uint8_t *d_feasible,
                                   int64_t n, int64_t *d_out, void *stream);

/*
 * Search problem (Sec. 4.2.3): choose M from M_list, a TP index, a
 * device-type-to-stage placement and a layer composition for S stages.
 * Slices are (m_idx, tp_idx, placement) in this nesting order; placements
 * are the allowed type sequences in lexicographic order.  Global index of a
 * plan = (((m_idx*n_tp + tp_idx)*n_place + place_rank)*n_map + map_rank),
 * n_map = C(L-1, S-1).  Objective: time per sample T/(D*M), compared exactly;
 * ties go to the lowest global index.
 * POS_PLACE_DEVICES (per-stage TP, as in the mixed-TP plans of the paper's
 * Table 1): slices are (m_idx, d_idx, class sequence), the classes
 * k_s = type_s * n_tp + tp_s of the S stages chosen freely among those whose
 * stages of every type t use exactly type_counts[t] devices (sum of
 * D_list[d_idx] * tp_list[tp_s]); the sequences of one D in lexicographic
 * order of (k_1, ..., k_S); slice ordinal = m_idx * P + (sequences of
 * D_list[0..d_idx-1]) + place_rank, P = the sequences of every D; global
 * index = ordinal * n_map + map_rank.  The tables must hold every class's
 * costs for each D tried; ridge pruning is not available (POS_EINVAL);
 * under POS_SCHED_INTERLEAVED_1F1B the sequence is over the S devices and
 * needs n_tp <= 4 (POS_EINVAL).
 */
/* Stage-level pruning (Sec. 4.2.1).  Every mode returns the same plan.
 *   POS_PRUNE_NONE   exhaustive enumeration (memory cut only).
 *   POS_PRUNE_EQ2    cut a prefix S_x when g(S_x) > T_min, g of Eq. 2 as
 *                    printed (Theorem 1).
 *   POS_PRUNE_TIGHT  a larger valid bound, not in the paper: Eq. 2 with the
 *                    inter-stage F and B edges on its path added, and the
 *                    largest of two bounds over the stages not yet placed.
 *                    For a complete plan and 1-based stages i <= y, the path
 *                    through the first micro-batch's forwards up to y, stage
 *                    y's whole chain, the last micro-batch's backwards down
 *                    to i and R_i has length
 *                      P(y, i) = sum_{j<y} (F_j + pf_j) + M (F_y + B_y)
 *                                + sum_{j=i}^{y-1} (B_j + pb_j) + d_i <= T;
 *                    the prefix bound is max( max_{i<=x} P(x, i),
 *                    min over memory-feasible completions of max_{y>x} P(y, y),
 *                    min over them of max_{y>x, i<=x} P(y, i) ), the minima
 *                    taken from per-slice tables built by a dynamic program
 *                    over (stage, first layer). */
#define POS_PRUNE_NONE 0
#define POS_PRUNE_EQ2 1
#define POS_PRUNE_TIGHT 2

typedef struct pos_problem {
    pos_tables tables;
    int32_t S;
    int32_t n_M;
    const int32_t *M_list;      /* [n_M], 1..255 */
    const int32_t *tp_list;     /* [n_tp] TP degree of each TP index (reported) */
    const int32_t *dp_list;     /* [n_tp] data-parallel degree D of each TP index */
    int32_t placement;          /* POS_PLACE_FREE or POS_PLACE_EXACT */
    const int32_t *type_counts; /* [n_types] stages per type (POS_PLACE_EXACT) */
    int32_t warmup;             /* random feasible samples seeding T_min (paper: 500) */
    int32_t prune;              /* POS_PRUNE_NONE, POS_PRUNE_EQ2 or POS_PRUNE_TIGHT */
    uint64_t seed;              /* warm-up sampling seed */
    int32_t schedule;           /* POS_SCHED_1F1B, POS_SCHED_EAGER_1F1B or
                                   POS_SCHED_INTERLEAVED_1F1B (with V below) */
    int64_t frontier_cap;       /* entries that a frontier buffer holds; 0 = default
                                   2^24; raised to at least 32*L */
    int32_t profile;            /* 1: device time per kernel kind in the stats (CUDA
                                   events around every launch); 0: those fields are 0 */
    int32_t ridge;              /* 1: layer-level pruning (Theorem 2): only plans whose
                                   layer counts over the stages of each device type rise,
                                   then fall ("ridge-like") are enumerated or returned.
                                   Theorem 2 guarantees a ridge-like optimum only under
                                   its assumptions: the result may be worse than the
                                   exact optimum (never better); 0: exact search */
    int32_t V;                  /* POS_SCHED_INTERLEAVED_1F1B: model chunks per device
                                   (>= 2, S*V <= 16); ignored by the other schedules */
    int32_t cas_limit;          /* rounds of the incumbent's compare-and-swap loop before
                                   the search gives up with POS_ETIMEOUT: 0 = default
                                   (2^20); < 0 = no round, so every update that would
                                   lower the incumbent gives up (tests the time-out path) */
    int32_t n_D;                /* POS_PLACE_DEVICES: data-parallel degrees tried */
    const int32_t *D_list;      /* [n_D] (>= 1); dp_list is not read there */
} pos_problem;

typedef struct pos_plan {
    int32_t found;
    int32_t m_idx, tp_idx, M, tp, D, S;  /* tp_idx, tp: -1 under POS_PLACE_DEVICES */
    int32_t makespan;           /* T in us */
    int32_t type[POS_MAX_STAGES];    /* device type per stage (per device, interleaved) */
    int32_t layers[POS_MAX_STAGES];  /* layers per stage (per virtual stage, interleaved) */
    uint64_t place_rank, map_rank, global_index;
    int32_t tp_stage[POS_MAX_STAGES];  /* TP index per stage (per device); -1 past S */
    int32_t d_idx;              /* POS_PLACE_DEVICES: index of D in D_list; else -1 */
} pos_plan;

typedef struct pos_search_stats {
    uint64_t evaluated;         /* complete plans whose makespan was computed */
    uint64_t warmup_evaluated;  /* of which in the warm-up */
    uint64_t prefixes;          /* partial plans generated (all depths) */
    uint64_t pruned_bound;      /* children cut by g(S_x) > T_min */
    uint64_t pruned_memory;     /* children cut by memory feasibility */
    uint64_t relaxations;       /* DAG node relaxations (2*S*M per evaluation) */
    uint64_t slices, slices_feasible;
    uint64_t launches;          /* kernel launches */
    double ms_setup, ms_warmup, ms_search, ms_total;  /* host wall clock */
    /* device time per kernel kind, CUDA events on the search's stream */
    double ms_expand, ms_complete, ms_leaf;
    uint64_t expand_launches, complete_launches, leaf_launches;
    /* frontier entries read by the expansion / completion kernels, and
       complete plans written by the completion kernel */
    uint64_t parents_expand, parents_complete, leaves;
    /* POS_PRUNE_TIGHT: device time and launches of the completion-bound
       tables (one launch per batch of slices) */
    double ms_bound;
    uint64_t bound_launches;
    /* batches of slices run a second time, host-driven, because a frontier
       of their pipelined pass overflowed frontier_cap */
    uint64_t reruns;
    /* per parent depth x (stages 0..x-1 placed; x = S-2 is the completion):
       device time of its level kernels (profile only), their launches, the
       frontier entries they read and the children (plans) they wrote */
    double ms_depth[POS_MAX_STAGES];
    uint64_t launches_depth[POS_MAX_STAGES];
    uint64_t parents_depth[POS_MAX_STAGES];
    uint64_t children_depth[POS_MAX_STAGES];
    uint64_t pruned_ridge;      /* children cut by the layer-level (ridge) rule */
} pos_search_stats;

/*
 * Exact search (Sec. 4.2.3) on the current CUDA device: warm-up sampling,
 * then enumeration of every slice's layer compositions with the memory cut
 * and the stage-level prune chosen by problem->prune (Eq. 2 / Theorem 1, or
 * the tighter bound); the result equals the exhaustive optimum.  Host pointers in, host plan out;
 * synchronous.  stats may be NULL.
 * Under POS_SCHED_INTERLEAVED_1F1B the S = N devices hold problem->V chunks
 * each: a plan is a slice (M, TP index, type placement over the N devices)
 * and a composition of L into the N*V virtual stages (C(L-1, NV-1) per
 * slice in the global index); M values that are not multiples of N are
 * skipped (their indices still count).  Prune modes there: POS_PRUNE_EQ2
 * cuts a prefix when some device's serial work over its placed chunks,
 * M * sum (F + B) + sum dsync, is already worse than the incumbent;
 * POS_PRUNE_TIGHT adds, per device whose first chunk is placed, the path
 * through the fill forwards, its chain and the drain backwards.  Layer-level
 * (ridge) pruning is not defined there (POS_EINVAL).
 * Errors: POS_EINVAL, POS_EOVERFLOW (guard fails for some M), POS_ENOMEM,
 * POS_ECUDA, POS_ETIMEOUT, POS_EINFEASIBLE (no memory-feasible plan; *out
 * has found = 0).
 * Limits (checked on the host before the device is touched; POS_EINVAL):
 * at most 2^22 slices (M values x TP indices x placements; M values x
 * class sequences of every D under POS_PLACE_DEVICES) and 2^22 placements;
 * under POS_PLACE_DEVICES at most 65536 devices per type; the global index
 * (slices x compositions) must fit in 64 bits; the lcm of all D*M must be
 * below 2^32.  Memory-feasible slices are
 * enumerated in batches of at most 65535 slices, one after another.
 * Memory: the work buffers (one frontier of frontier_cap 32-byte entries per
 * depth, a leaf buffer of the same length, each with a share of slots that
 * may stay empty beside them when frontier_cap is above 1.9 million (at most
 * 25 %, 11 % at the default; GB300), slice and feasibility tables,
 * and with POS_PRUNE_TIGHT 1 KB of bound tables per stage and slice of a
 * batch),
 * a stream and pinned counters are kept per device between calls, grown on
 * demand and released at process exit; concurrent searches on one device
 * are serialised.
 */
pos_status poseidon_search(const pos_problem *problem, pos_plan *out, pos_search_stats *stats);

/* ------------------------------------------------------------------------
 * Layer operators: what a pipeline stage keeps of a micro-batch in 8 bits
 * between its forward and its backward pass.  A stage holds the activations
 * of W_s micro-batches at once and fits when mem_w + W_s * mem_a <= cap, so
 * the bytes that poseidon_ckpt_bytes returns for the tensors a layer keeps
 * are what goes into mem_a.
 *
 * Every pointer below is a device pointer on the current device unless a
 * line says otherwise; every call is asynchronous on `stream`.  Strides are
 * in elements and may be any number >= 0 on tensors that are read (0
 * repeats a row); rows that are written must not overlap.
 */
#define POS_BF16 0
#define POS_F16 1
#define POS_F32 2

/*
 * Checkpoint of a matrix [rows][cols], one buffer: rows of
 * pitch = 32 * ceil(cols / 32) code bytes (zeros past the last column), then,
 * from byte rows * pitch, rows of 4 * ceil(groups / 4) scale bytes, one per
 * group of 32 columns (groups = pitch / 32; the bytes past the last group are
 * not defined).  A value is code * 2^e with scale byte e + 127:
 *   POS_CKPT_INT8   code = int8 in [-127, 127], e the smallest with
 *                   max|x| <= 127 * 2^e, at most 121;
 *   POS_CKPT_E4M3   code = float8 e4m3, e the smallest with
 *                   max|x| <= 448 * 2^e, at most 119;
 * e is at least -110 (a group of smaller magnitudes keeps what is left at
 * that e).  x / 2^e is exact and is rounded once, to the nearest code, ties
 * to even; only a group at the largest e saturates.  A group that holds an
 * infinity or a NaN has scale byte 255 and stands for NaNs.
 */
#define POS_CKPT_INT8 0
#define POS_CKPT_E4M3 1

/* Bytes of a checkpoint: *bytes (host) = rows * (pitch + scale bytes per
 * row).  POS_EINVAL: rows or cols < 0, cols above 2^31 - 33, a size of 2^62
 * or more, NULL. */
pos_status poseidon_ckpt_bytes(int64_t rows, int64_t cols, int64_t *bytes);

/*
 * Pack x [rows][cols] (rows ldx elements apart) of POS_BF16, POS_F16 or
 * POS_F32 into the checkpoint d_ckpt (16-byte aligned).
 * Errors: POS_EINVAL (NULL, negative sizes or stride, dtype or format,
 * alignment), POS_ECUDA.
 */
pos_status poseidon_ckpt_pack(const void *d_x, int32_t dtype, int64_t rows, int64_t cols,
                              int64_t ldx, int32_t format, void *d_ckpt, void *stream);

/*
 * The values of a checkpoint as y [rows][cols] (ldy >= cols elements apart).
 * They are exact in POS_BF16 and POS_F32; POS_F16 rounds to nearest even and
 * saturates at +-65504.
 */
pos_status poseidon_ckpt_unpack(const void *d_ckpt, int32_t format, int64_t rows, int64_t cols,
                                void *d_y, int32_t dtype, int64_t ldy, void *stream);

/*
 * Weight gradient of a linear layer y = x W^T, W [n][cols], from the
 * checkpoint of its input x [rows][cols] and the gradient dy [rows][n] of
 * its output:
 *   dw_out[i][j] = dw_in[i][j] + sum_r dy[r][i] * x[r][j]
 * d_dw_in is NULL (zeros) or has dw_out's layout; it may be dw_out itself,
 * which adds a micro-batch to the gradients of earlier ones, and must not
 * overlap it otherwise.  dtype is dy's: POS_BF16 or POS_F16; x is taken as
 * poseidon_ckpt_unpack gives it in that type.  Products are exact, sums are
 * kept in 32 bits, in an order that depends on the sizes and the GPU alone.
 * Scratch from the library's pool (stream-ordered): partial sums where the
 * rows are split, at most 64 MB; when dy is not 16-byte aligned (base and
 * ld_dy) or ld_dy < n, a copy of it, a block of at most 256 MB at a time.
 * Waits inside the kernel are bounded: two seconds, not counting time in which
 * the GPU ran something else.  One that ran out makes the gradients NaN.
 * Errors: POS_EINVAL (NULL, negative sizes or strides, ld_dw < cols, dtype,
 * format, rows, n or cols of 2^31 or more, alignment), POS_ENOMEM, POS_ECUDA.
 */
pos_status poseidon_ckpt_wgrad(const void *d_ckpt, int32_t format, const void *d_dy,
                               int32_t dtype, int64_t ld_dy, int64_t rows, int64_t n,
                               int64_t cols, const float *d_dw_in, float *d_dw_out,
                               int64_t ld_dw, void *stream);

/* How the first `rot` elements of a head are paired for the rotation. */
#define POS_ROT_HALF 0      /* (i, i + rot / 2) */
#define POS_ROT_ADJACENT 1  /* (2 i, 2 i + 1) */

/*
 * RMS norm of every query and key head with the position rotation in the
 * same pass.  For a head x [dim] of a token at position p:
 *   r = 1 / sqrt(mean(x^2) + eps),  u = x * r * w,
 *   (y_a, y_b) = (u_a c - u_b s, u_b c + u_a s) for the i-th pair (a, b),
 *   c = cos[p][i], s = sin[p][i]; elements from rot on keep u.
 * A token at a negative position is padding: its outputs and gradients are
 * zeros, whatever its inputs hold, and it adds nothing to the weights'
 * gradients.  A position >= n_pos makes the token's outputs and gradients
 * NaN.  Norms, rotation and sums are in 32 bits, rounded once on output.
 */
typedef struct pos_qk {
    int64_t tokens;
    int32_t heads_q, heads_k;   /* >= 0 */
    int32_t dim;                /* 1..256 */
    int32_t rot;                /* even, 0..dim */
    int32_t pairing;            /* POS_ROT_HALF or POS_ROT_ADJACENT */
    int32_t dtype;              /* of q, k, outputs and their gradients */
    int32_t format;             /* of the checkpoints */
    float eps;                  /* >= 0 */
    const float *w_q, *w_k;     /* [dim]; NULL = ones */
    const float *cos, *sin;     /* [n_pos][rot / 2] */
    int64_t n_pos;
    const int32_t *positions;   /* [tokens]; NULL = 0, 1, 2, ... */
} pos_qk;

/* A tensor [tokens][heads][dim] with contiguous heads. */
typedef struct pos_heads {
    void *data;
    int64_t token_stride, head_stride;
} pos_heads;

/*
 * Forward pass.  x, y: host arrays of two (queries, keys); y may be x itself
 * (the same pointers and strides).  rstd_q, rstd_k ([tokens][heads], float)
 * and ckpt_q, ckpt_k (16-byte aligned checkpoints of x as a matrix
 * [tokens * heads][dim]) are what the backward pass reads; each may be NULL.
 * Errors: POS_EINVAL (NULL, sizes, strides, rows of y that overlap, dtype,
 * pairing, format, a pointer off its elements), POS_ECUDA.
 */
pos_status poseidon_qk_forward(const pos_qk *qk, const pos_heads *x, const pos_heads *y,
                               float *rstd_q, float *rstd_k, void *ckpt_q, void *ckpt_k,
                               void *stream);

/*
 * Backward pass.  With g the gradient of y turned back, n = x * r, h = g * w:
 *   dx = r * (h - n * mean(h * n)),  dw = dw_in + sum over tokens, heads of g * n.
 * x (host array of two) or, where it is NULL, the checkpoints give x; rstd is
 * the forward pass's.  dy, dx: host arrays of two; dx may be dy itself.
 * d_dw ([2][dim], queries' then keys') may be NULL, d_dw_in (the same layout)
 * is NULL for zeros or may be d_dw itself.  The sums' order depends on the
 * sizes and the GPU alone.  Scratch from the library's pool: 8 * dim bytes for
 * each block of the grid (at most 8 per SM) when d_dw is not NULL.
 * Errors: POS_EINVAL (as above; neither x nor checkpoints, d_dw_in without
 * d_dw), POS_ENOMEM, POS_ECUDA.
 */
pos_status poseidon_qk_backward(const pos_qk *qk, const pos_heads *x, const void *ckpt_q,
                                const void *ckpt_k, const float *rstd_q, const float *rstd_k,
                                const pos_heads *dy, const pos_heads *dx, const float *d_dw_in,
                                float *d_dw, void *stream);

/*
 * Dropout whose mask is computed where it is needed and never stored: the backward
 * pass is the same call on the gradient.  Element (r, c) of a matrix is kept where
 * its 16 random bits, a whole number, are at least t = p * 65536 (rounded to nearest),
 * and then multiplied by 65536 / (65536 - t), so the mean is kept exactly.  The bits
 * are half word c % 8 (low halves first) of the four words that Philox-4x32 of ten
 * rounds gives for the counter (c / 8, r, low and high word of offset + *d_offset)
 * under the key (low and high word of seed).  One offset per tensor, layer and
 * micro-batch makes their masks independent.  d_offset is read when the kernel runs:
 * a captured graph whose program advances it draws new masks at every replay.
 * What a dropped element holds has no effect, a NaN neither.
 */
typedef struct pos_dropout {
    float p;                    /* 0..1; below 2^-17 nothing is dropped */
    uint64_t seed, offset;
    const uint64_t *d_offset;   /* device, 8-byte aligned; NULL = 0 */
} pos_dropout;

/*
 * y = residual + dropout(x), [rows][cols]; one rounding in 32 bits, one to y's type.
 * d_res (y's type) may be NULL: y = dropout(x).  x and y may have any two types.  y may
 * be x or d_res itself (the same pointer, stride and type) and must not overlap them
 * otherwise.
 * Errors: POS_EINVAL (NULL, p, rows or cols < 0 or of 2^31 - 8 or more, strides < 0 or
 * of 2^31 or more, ldy < cols, dtype, a pointer off its elements), POS_ECUDA.
 */
pos_status poseidon_dropout(const pos_dropout *drop, int64_t rows, int64_t cols, const void *d_x,
                            int32_t dtype, int64_t ldx, const void *d_res, int64_t ldr, void *d_y,
                            int32_t dtype_y, int64_t ldy, void *stream);

/*
 * The residual's addition and the RMS norm of the sum, row by row:
 *   h = residual + dropout(x)   rounded once in 32 bits, then to dtype_h,
 *   r = 1 / sqrt(mean(h^2) + eps),  y = h * r * w   of h as it is written,
 * sums in 32 bits.
 */
typedef struct pos_norm {
    int64_t rows;               /* 0..2^31 - 1 */
    int32_t cols;               /* 1..32768 */
    int32_t dtype;              /* of x, y and their gradients */
    int32_t dtype_h;            /* of the residual, h and their gradients: dtype or POS_F32 */
    int32_t format;             /* of the checkpoints */
    float eps;                  /* >= 0 */
    const float *w;             /* [cols]; NULL = ones */
    pos_dropout drop;           /* of x; p = 0: none */
} pos_norm;

/*
 * Forward pass.  d_res may be NULL (h = dropout(x)).  Each output may be NULL: h, y,
 * the checkpoints (16-byte aligned) of h, which the backward pass can read in h's
 * place, and of y, which poseidon_ckpt_wgrad reads (both as poseidon_ckpt_pack makes
 * them of the tensor written), rstd [rows] (r).  y is h r w rounded once to 32 bits,
 * but for the sum of the squares, and then to its type.  h may be d_res and y may be x
 * itself (the same pointers and strides); other overlaps are not allowed.
 * Errors: POS_EINVAL (NULL, sizes, strides, dtypes, format, eps, p, alignment),
 * POS_ECUDA.
 */
pos_status poseidon_norm_forward(const pos_norm *norm, const void *d_x, int64_t ldx,
                                 const void *d_res, int64_t ldr, void *d_h, int64_t ldh, void *d_y,
                                 int64_t ldy, void *d_ckpt_h, void *d_ckpt_y, float *d_rstd,
                                 void *stream);

/*
 * Backward pass.  With n = h * r (h, or where it is NULL its checkpoint, and the
 * forward pass's rstd) and a = dy * w:
 *   dh = dh_in + r * (a - n * mean(a * n)),  dx = dropout(dh),
 *   dw = dw_in + sum over the rows of dy * n,
 * dh_in the gradient that reaches h on other ways (NULL: zeros).  dh is the
 * gradient of the residual too.  dx is dropped from dh before its rounding.  dh, dx and
 * d_dw ([cols]) may be NULL; dh may be dh_in, dx may be dy and d_dw may be d_dw_in
 * itself.  The sums' order depends on the sizes and the GPU alone.  Scratch from the
 * library's pool where d_dw is not NULL: 4 * cols bytes for each block of the grid (what
 * the GPU holds at once, at most 16 an SM).
 * Errors: POS_EINVAL (as above; neither h nor its checkpoint, d_dw_in without d_dw),
 * POS_ENOMEM, POS_ECUDA.
 */
pos_status poseidon_norm_backward(const pos_norm *norm, const void *d_h, int64_t ldh,
                                  const void *d_ckpt_h, const float *d_rstd, const void *d_dy,
                                  int64_t lddy, const void *d_dh_in, int64_t lddh_in, void *d_dh,
                                  int64_t lddh, void *d_dx, int64_t lddx, const float *d_dw_in,
                                  float *d_dw, void *stream);

/*
 * Causal attention with grouped heads over packed sequences.  Token i of a sequence
 * sees its tokens j <= i; query head h reads key head h / (heads_q / heads_k):
 *   s_ij = scale * q_i k_j,  lse_i = log(sum_j exp(s_ij)),
 *   o_i = sum_j exp(s_ij - lse_i) v_j.
 * Sequence n is the tokens starts[n] .. starts[n + 1] - 1 and may be empty; what lies
 * before the first and behind the last is left as it was and may hold anything, and
 * so may later tokens and other sequences: an infinity or a NaN reaches only those
 * rows that see it.  A start below one before it counts as that one, one outside
 * 0..tokens as the nearest of these.
 */
typedef struct pos_attn {
    int64_t tokens;             /* below 2^31 - 512 */
    int32_t heads_q, heads_k;   /* 0..65536; heads_q a multiple of heads_k */
    int32_t dim;                /* 1..128 */
    int32_t dtype;              /* POS_BF16 or POS_F16 */
    float scale;                /* above 0 */
    int32_t sequences;          /* at most 2^24 */
    const int32_t *starts;      /* device [sequences + 1]; NULL = one sequence of all tokens */
} pos_attn;

/*
 * Forward pass.  x: host array of three (queries, keys, values), o: one; lse
 * [heads_q][tokens], which the backward pass reads, may be NULL.  o must not overlap x.
 * Scores and sums are in 32 bits; probabilities, relative to a reference within 2^8 of
 * the row's largest, are rounded to dtype for the product with the values, and o once
 * on output.
 * Scratch from the library's pool (stream-ordered): 16 bytes a tile of 256 tokens and
 * sequence where starts is not NULL; a copy of each of x that is off the 16-byte
 * alignment (base, strides and dim) or has a stride of 0.  Of a call's scratch the library
 * keeps up to 320 MB for later ones; more than that is given back when the stream, an
 * event or the device is next waited for.  Waits inside the kernels are
 * bounded as poseidon_ckpt_wgrad's are (POSEIDON_ATTN_WAIT_NS in the environment of the
 * process's first call, in nanoseconds, is another limit); where one ran out, every row
 * whose result is lost by that is NaN.
 * Errors: POS_EINVAL (NULL, sizes, heads, dim, dtype, scale, strides, rows of o that
 * overlap, a pointer off its elements), POS_ENOMEM, POS_ECUDA.
 */
pos_status poseidon_attn_forward(const pos_attn *attn, const pos_heads *x, const pos_heads *o,
                                 float *d_lse, void *stream);

/*
 * Backward pass.  lse and o are the forward pass's.  With p_ij = exp(s_ij - lse_i),
 * dp_ij = do_i v_j, D_i = sum_j p_ij dp_ij (which is do_i o_i, but for the rounding of o,
 * that the gradients are freed from) and ds_ij = p_ij (dp_ij - D_i):
 *   dq_i = scale * sum_j ds_ij k_j,  dk_j = scale * sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i,
 * the keys' and values' summed over the query heads of their group.  x, dx: host arrays of
 * three, o and d_o: one; dx must not overlap what is read.  Sums are in 32 bits, in an
 * order that the sizes and the GPU fix; p and ds are rounded to dtype for their products
 * (of a sequence's first 128 queries each is two values of dtype).
 * Scratch from the library's pool: 8 bytes a token and query head, in f16 4 a token and 8 a
 * sequence and key head, what the forward pass takes (16 bytes a tile of 128; a copy of d_o too where
 * it needs one) and, where there are few tiles of keys, 1 KB for each element of dim and
 * block that shares one (at most 8 blocks an SM).
 * Errors: as above (NULL lse; rows of dx that overlap).
 */
pos_status poseidon_attn_backward(const pos_attn *attn, const pos_heads *x, const pos_heads *o,
                                  const float *d_lse, const pos_heads *d_o, const pos_heads *dx,
                                  void *stream);

/* Message describing the last error of the calling thread ("" if none). */
const char *poseidon_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* POSEIDON_H */
