/*
 * reflex.h — C ABI of the REFLEX per-forward MoE hot path on one GB300
 * (sm_103a).  Library: paper_2608_01784_gb300/_build/libreflex.so.
 *
 * REFLEX (arxiv 2608.01784) splits token-choice MoE inference into expert
 * ranking (left to the default router) and expert-count allocation.  This
 * library implements both halves of one denoising forward:
 *
 *   reflex_allocate     the allocation rule k = Pi(S_t, K^Sigma) of Eq. 3,
 *                       realised by Refinement-Role Budgeting (Sec. 4.2,
 *                       Eq. 5) and Frontier-Guided Expert Reallocation
 *                       (Sec. 4.3, Eq. 6-9), clipped to [K_min, K_max].
 *   reflex_moe_forward  the variable-count MoE layer of Eq. 2: router scores,
 *                       TopK(r_i, k_i), normalised router weights, SwiGLU
 *                       experts on the selected token-expert pairs, weighted
 *                       sum (plus an optional always-on shared expert).
 *
 * Conventions shared by every call
 *   - All array arguments are DEVICE pointers unless stated otherwise; the
 *     caller owns them.  The library never allocates or frees device memory
 *     and never synchronises the stream, except reflex_moe_status and
 *     reflex_read_status, which synchronise to read an error word.
 *   - `stream` is a cudaStream_t passed as void* (NULL = legacy stream).  All
 *     work is enqueued asynchronously on it.
 *   - Row-major layouts.  Integer arrays are int32 unless stated.
 *   - Return value: a REFLEX_* status.  Host-side checks (null pointers,
 *     shapes, workspace size) return before anything is enqueued.  Checks
 *     that need device data (a count k_i out of range, too many active-block
 *     tokens) set bits in a device error word; read it with
 *     reflex_moe_status / reflex_read_status.
 */
#ifndef REFLEX_H
#define REFLEX_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ------------------------------------------------------- */
#define REFLEX_OK 0
#define REFLEX_EINVAL 1        /* null pointer, bad shape or parameter       */
#define REFLEX_EKRANGE 2       /* a count outside its allowed range          */
#define REFLEX_EWORKSPACE 3    /* workspace missing or smaller than needed   */
#define REFLEX_ECUDA 4         /* a CUDA runtime / launch error              */
#define REFLEX_ETIMEOUT 5      /* a bounded device wait expired              */
#define REFLEX_EUNSUPPORTED 6  /* shape not supported by the selected path   */
#define REFLEX_ECAPACITY 7     /* more active-block tokens than supported    */

/* ---- element types ------------------------------------------------------ */
#define REFLEX_DTYPE_F32 0     /* fp32 storage and fp32 arithmetic           */
#define REFLEX_DTYPE_BF16 1    /* bf16 storage, fp32 accumulation            */

/* ---- reflex_moe_forward flags ------------------------------------------ */
/* alpha renormalised over the selected experts (default reading of the
 * "normalized router weight" of Sec. 3.2); without it alpha is the softmax
 * over all E experts. */
#define REFLEX_FLAG_RENORM_TOPK 0x1u
/* bf16 only: run the expert GEMMs on the SIMT kernels instead of the
 * tcgen05/TMEM kernels (cross-checking; the fp32 path always uses SIMT). */
#define REFLEX_FLAG_SIMT_EXPERTS 0x2u
/* Residual connection for stacked layers: out = hidden + MoE(hidden), summed
 * in fp32 with the expert outputs and rounded once. */
#define REFLEX_FLAG_RESIDUAL 0x4u
/* bf16: compute every router score with the canonical fma chain.  Without
 * it (and with REFLEX_FLAG_RENORM_TOPK) the scores come from a tensor-core
 * GEMM and only the experts that could be selected are recomputed with the
 * chain: the selected experts, their weights and their scores are the same
 * bits either way (the screen's bound is stated with reflex_moe_forward);
 * only the record's other scores differ (tensor-core estimates). */
#define REFLEX_FLAG_EXACT_SCORES 0x8u
/* bf16 tcgen05 path, routed gate/up GEMM on CTA pairs (inter % 128 == 0, d %
 * 256 == 0, and expected rows per expert, T * k_max / (2 E), of at least 128;
 * fewer do, from 96, or 104 with d > 2048 and E >= 32, where the expected rows,
 * activations and outputs fit in 128 MB and no shared expert is given or T >=
 * 2048): the GEMM fetches its input rows from hidden itself through the pair
 * permutation, and DISPATCH only places the pairs (no copy of the rows in
 * pair order is written).  The outputs are the same bits as without the flag.
 * Elsewhere the flag changes nothing.  The fused dispatch is slower on GB300
 * (row copies by the GEMM's own warps do not keep up with the tensor cores:
 * the 32 x 1024-token LLaDA-MoE layer's gate/up GEMM 0.78 -> about 1.5 ms),
 * so it is off by default.  With stage selection the DISPATCH and EXPERT_UP
 * calls must agree on the flag. */
#define REFLEX_FLAG_GATHER_IN_GEMM 0x10u
/* Stage selection.  No stage bit = all five stages in order.  Stages read
 * what the previous stages left in the same workspace; running a stage whose
 * predecessors did not run on that workspace gives unspecified values (every
 * index read from the workspace is range-checked on the device, so no
 * out-of-bounds access results).  hidden must hold the same values at the
 * DISPATCH and EXPERT_UP stages of one forward (the shared expert reads it
 * at EXPERT_UP, and so do the routed experts with REFLEX_FLAG_GATHER_IN_GEMM)
 * and, with REFLEX_FLAG_RESIDUAL, at COMBINE. */
#define REFLEX_STAGE_ROUTE 0x100u       /* router scores, TopK, alpha        */
#define REFLEX_STAGE_DISPATCH 0x200u    /* pair counts, offsets, permutation */
#define REFLEX_STAGE_EXPERT_UP 0x400u   /* gate/up GEMM + SwiGLU (+ shared)  */
#define REFLEX_STAGE_EXPERT_DOWN 0x800u /* down GEMM (+ shared)              */
#define REFLEX_STAGE_COMBINE 0x1000u    /* weighted sum back to token order  */

/* ---- allocation hyper-parameters (Sec. 4.2-4.3; defaults in Sec. 5.1) --- */
typedef struct {
    int32_t k_min;      /* lower clip bound of every count, >= 1            */
    int32_t k_base;     /* K_base of Eq. 5                                  */
    int32_t k_max;      /* upper clip bound, >= k_min                       */
    int32_t delta_role; /* delta_role of Eq. 5 (0 = no role prior)          */
    int32_t delta_cur;  /* delta_cur of Eq. 9 (0 = no reallocation)         */
    float q;            /* outer-group fraction of Eq. 9, in (0, 1/2]       */
    float theta;        /* commitment threshold of Eq. 6                    */
    float w_cf;         /* commitment-frontier width of Eq. 6 and the
                           velocity clip, > 0                               */
    float v_ref;        /* velocity reference of Eq. 7                      */
    float tau;          /* gate temperature of Eq. 6-7, > 0                 */
    int32_t signal;     /* rank key of the Eq. 9 groups: REFLEX_SIGNAL_*    */
    int32_t role_shuffle; /* 1: permute each sequence's final counts among
                           its positions (Role-Shuffled RRB, App. C); the
                           multiset and sum of the counts are unchanged.
                           Sequences longer than 4096 tokens are left as
                           they are and flag REFLEX_ECAPACITY.              */
    uint64_t shuffle_seed; /* seed of the shuffle's splitmix64 stream       */
    int32_t count_rule; /* where the counts come from: REFLEX_RULE_*        */
    float rule_threshold; /* p of REFLEX_RULE_TOP_P, or the router-weight
                           threshold of REFLEX_RULE_EXPERT_THRESHOLD      */
} reflex_alloc_params;

/* Count rules.  REFLEX_RULE_REFLEX (0, the default) is the allocation of
 * Sec. 4.2-4.3 above.  The other two are the threshold-based comparison
 * methods of App. B, which take each token's count from its router scores
 * z_t instead of its refinement state (the paper runs them with the count
 * bounds [1, 12], i.e. k_min = 1, k_max = 12):
 *   TOP_P             the smallest prefix of the router-ranked experts
 *                     (scores descending, lower index first on ties) whose
 *                     cumulative routing mass reaches rule_threshold;
 *   EXPERT_THRESHOLD  the number of experts whose routing mass exceeds
 *                     rule_threshold;
 * either clipped to [k_min, min(k_max, E)].  The routing mass is the
 * softmax of z_t over all E experts, and the decision is taken in fp32 in
 * this order, so that the counts are reproducible bit for bit:
 *   m = max_e z_e;  u_e = exp(z_e - m) (the library's Cody-Waite exp, the
 *   one of the FPS sigmoids);  S = the sum of the u_e, lane l of 32 adding
 *   u_l, u_{l+32}, ... in ascending order, then the 32 lane sums combined by
 *   s_l <- s_l + s_{l xor o} for o = 16, 8, 4, 2, 1;
 *   TOP_P: c_j = c_{j-1} + u_(j) over the ranks j = 1, 2, ... (c_0 = 0),
 *   k = the smallest j with c_j / S >= rule_threshold;
 *   EXPERT_THRESHOLD: k = #{e : u_e / S > rule_threshold}.
 * The score rules read every router score, so a forward that takes its
 * counts from them computes every score with the canonical chain (as with
 * REFLEX_FLAG_EXACT_SCORES). */
#define REFLEX_RULE_REFLEX 0
#define REFLEX_RULE_TOP_P 1
#define REFLEX_RULE_EXPERT_THRESHOLD 2

/* Rank keys for the FGER groups (Sec. 4.3; signal ablation of App. C).  The
 * top floor(q |J_h|) tokens by (key desc, position asc) gain delta_cur, the
 * bottom ones lose it.
 *   FPS          S = F * P (Eq. 8), the REFLEX default
 *   FRONTIER     F alone (Eq. 6)
 *   PROGRESS     P alone (Eq. 7; 1 with fewer than two observations)
 *   CONFIDENCE   c^{t-1}
 *   UNCERTAINTY  1 - c^{t-1} (fp32)
 * RRB Only and FGER Only (Sec. 5.3) are parameter settings: delta_cur = 0 and
 * delta_role = 0 respectively. */
#define REFLEX_SIGNAL_FPS 0
#define REFLEX_SIGNAL_FRONTIER 1
#define REFLEX_SIGNAL_PROGRESS 2
#define REFLEX_SIGNAL_CONFIDENCE 3
#define REFLEX_SIGNAL_UNCERTAINTY 4

/* Role shuffle.  Token i of a sequence gets the key
 *   key_i = high 32 bits of splitmix64 output number i + 1 for shuffle_seed
 * (splitmix64: state_n = seed + n * 0x9e3779b97f4a7c15, output = the
 * Stafford "mix13" finaliser of state_n, Steele, Lea and Flood 2014), i the
 * token's index in the batch; with r_i the rank of (key_i, i) in ascending
 * order within the sequence, token i receives the count the unshuffled
 * allocation gives to the sequence's r_i-th position. */

/* Fills the Sec. 5.1 defaults: k_base 8, delta_role 4, delta_cur 2, q 0.25,
 * theta 0.9, w_cf 0.30 (LLaDA-MoE; 0.25 for LLaDA2.0-mini), v_ref 0.01,
 * tau 0.05, the clip [k_min, k_max] = [2, 12], signal FPS, no shuffle,
 * count rule REFLEX (rule_threshold 0). */
void reflex_default_params(reflex_alloc_params* p);

/*
 * reflex_allocate — per-token expert counts k_i for one denoising forward
 * (Eq. 3 realised by Eq. 5 and Eq. 9, Sec. 4.2-4.3).
 *
 *   router_scores  [T, E] fp32.  REFLEX's rule does not read it (the router
 *                  only ranks experts, Sec. 3.3) and it may be NULL; the
 *                  score rules (p->count_rule TOP_P or EXPERT_THRESHOLD)
 *                  take the counts from it alone (E experts per row), and
 *                  then every state array below may be NULL.
 *   conf_prev1     [T] fp32  c_i^{t-1}, the latest confidence observation.
 *   conf_prev2     [T] fp32  c_i^{t-2}; read only where hist_len >= 2.
 *   hist_len       [T] u8    number of past observations (0, 1, >= 2).
 *   masked         [T] u8    1 = position is [MASK] (member of M_t).
 *   block_id       [T] int32 b(i): 0 for prompt positions, 1..Q for target
 *                            blocks.
 *   seq_offsets    [B+1]     token range of each sequence; seq_offsets[0] = 0,
 *                            seq_offsets[B] = T, non-decreasing.
 *   active_block   [B]       a_t of each sequence, >= 1.
 *   p              HOST pointer to the hyper-parameters.
 *   k_out          [T] int32 output counts, each in [k_min, k_max].
 *   k_sum_out      [1] int64 nullable: sum of k_out (the realised budget).
 *   dev_status     [1] int32 nullable device error word; cleared by this
 *                  call, then OR-ed with error bits (see reflex_read_status).
 * Tokens of the active block that are masked and have at least one
 * observation form J_h and are ranked by the Frontier-Progress Score (ties:
 * lower position first); at most 4096 such tokens per sequence (more sets
 * REFLEX_ECAPACITY in dev_status and leaves them at K_cur, clipped).
 * Host errors: REFLEX_EINVAL for null required pointers, T < 0, B < 1, or
 * parameters violating 1 <= k_min <= k_max, k_base >= 1, delta_* >= 0,
 * 0 < q <= 0.5, w_cf > 0, tau > 0, an unknown count_rule, or (score rules)
 * a missing router_scores, E outside [1, 1024] or a non-finite
 * rule_threshold.  Counts below k_min (or above k_max) produced by Eq. 5 /
 * Eq. 9 are clipped.
 */
int reflex_allocate(const float* router_scores, const float* conf_prev1,
                    const float* conf_prev2, const uint8_t* hist_len,
                    const uint8_t* masked, const int32_t* block_id,
                    const int32_t* seq_offsets, const int32_t* active_block,
                    int32_t T, int32_t B, int32_t E,
                    const reflex_alloc_params* p, int32_t* k_out,
                    int64_t* k_sum_out, int32_t* dev_status, void* stream);

/*
 * reflex_update_state — refinement-state update after one denoising forward
 * of block-wise inference (Sec. 3.1, Eq. 1): commits, confidence history and
 * active-block advance, in place, for the next forward's reflex_allocate.
 *
 * Per sequence s with a = active_block[s] (1 <= a <= num_blocks[s]) and J =
 * the masked positions of block a:
 *   - C = {i in J : conf_new[i] >= theta_commit} is committed (masked -> 0);
 *     if C is empty and J is not, the most confident member of J (lower
 *     position on ties) is committed instead;
 *   - every position masked during the forward shifts its history:
 *     conf_prev2 <- conf_prev1, conf_prev1 <- conf_new, hist_len <-
 *     min(hist_len + 1, 2);
 *   - when no position of block a is left masked, active_block[s] = a + 1.
 * A sequence with active_block[s] > num_blocks[s] is finished and untouched.
 *
 *   conf_new        [T] fp32  c^t of the forward (read where masked).
 *   conf_prev1/2    [T] fp32  in/out, as in reflex_allocate.
 *   hist_len        [T] u8    in/out.
 *   masked          [T] u8    in/out.
 *   block_id        [T] int32, seq_offsets [B+1]: as in reflex_allocate.
 *   active_block    [B] int32 in/out.
 *   num_blocks      [B] int32 Q of each sequence (its last target block).
 *   theta_commit    commitment threshold of Eq. 1 (Sec. 5.1: 0.9).
 *   committed_out   [B] int32 nullable: positions committed in each sequence.
 *   dev_status      [1] int32 nullable; error bits are OR-ed in (not cleared).
 * Device buffers, one CTA per sequence; returns REFLEX_EINVAL for null
 * pointers, T < 0, B < 1 or a non-finite theta_commit.
 */
int reflex_update_state(const float* conf_new, float* conf_prev1, float* conf_prev2,
                        uint8_t* hist_len, uint8_t* masked, const int32_t* block_id,
                        const int32_t* seq_offsets, int32_t* active_block,
                        const int32_t* num_blocks, int32_t T, int32_t B,
                        float theta_commit, int32_t* committed_out,
                        int32_t* dev_status, void* stream);

/* Device pointers into the workspace after a forward (the routing record). */
typedef struct {
    int32_t* ids;     /* [T, k_max] selected experts in router rank order,
                         -1 in slots j >= k_i                               */
    float* alpha;     /* [T, k_max] normalised router weights, 0 padded     */
    int32_t* counts;  /* [E] pairs per expert                               */
    int32_t* offsets; /* [E+1] first pair row of each expert                */
    int32_t* perm;    /* [sum k] pair rows: token * k_max + slot, ordered by
                         (expert, token)                                    */
    int32_t* row_of;  /* [T, k_max] pair row of (token, slot), -1 unused    */
    int32_t* totals;  /* [2] device: sum k (pairs), number of 128-row tiles */
    float* scores;    /* [T, E] router scores r_i (fp32), valid after the
                         ROUTE stage: the fma chain of reflex_moe_forward for
                         every expert that could be selected (all experts
                         with REFLEX_FLAG_EXACT_SCORES or fp32), tensor-core
                         estimates for the others                           */
} reflex_route_record;

/* Bytes of workspace reflex_moe_forward needs for these shapes (0 if the
 * shapes are invalid).  Sized for the worst case T * k_max pairs, so the
 * forward never reads back the realised sum of k.  Never decreases as T
 * grows (other shapes fixed): a workspace sized for T serves every smaller
 * batch. */
size_t reflex_moe_workspace_size(int32_t dtype, int32_t T, int32_t d,
                                 int32_t E, int32_t inter,
                                 int32_t shared_inter, int32_t k_max);

/*
 * reflex_moe_forward — the variable-count MoE layer, Eq. 2 (Sec. 3.2):
 *   out_i = sum_{e in TopK(r_i, k_i)} alpha_{i,e} E_e(h_i)  [+ shared(h_i)]
 * with r_i = h_i W_r^T (fp32; each score is the sequential fused
 * multiply-add chain over the hidden index from +0), TopK ties broken to the
 * lower expert index, and SwiGLU experts
 *   E_e(h) = (silu(h W_g,e^T) * (h W_u,e^T)) W_d,e^T.
 * The TopK is decided on the canonical chain's scores.  bf16 layers with
 * renormalised weights screen first: tensor-core scores z~ with an interval
 * z~ -/+ (gamma_d + 2^-12 + (s+1) 2^-24) ||h_i|| ||w_e|| + d 2^-125 (gamma_d
 * = d u / (1 - d u), u = 2^-24, s split-K slices) that holds both the chain's
 * score and the exact product; experts whose interval lies below the k_i-th
 * largest lower end cannot be selected, all others are recomputed with the
 * chain.  Where a norm or an estimate is not finite, or the product of the
 * norms is within a factor of four of the fp32 range, the interval is (-inf,
 * inf).  This assumes the tensor cores' fp32 accumulation errs by at most
 * 2^-12 sum_k |h_k w_k|; REFLEX_FLAG_EXACT_SCORES computes every score with
 * the chain instead.
 *
 *   dtype           REFLEX_DTYPE_F32 or REFLEX_DTYPE_BF16 (all float arrays).
 *   hidden          [T, d]
 *   w_router        [E, d]
 *   w_gate_up       [E, 2*inter, d]: rows [0, inter) gate, [inter, 2*inter) up
 *   w_down          [E, d, inter]
 *   shared_gate_up  [2*shared_inter, d], nullable (with shared_inter = 0)
 *   shared_down     [d, shared_inter]
 *   k               [T] int32 counts (from reflex_allocate or any rule);
 *                   each must lie in [1, min(k_max, E)] (else the device
 *                   error word gets REFLEX_EKRANGE and the count is clamped).
 *   flags           REFLEX_FLAG_* | REFLEX_STAGE_* (see above).
 *   workspace       >= reflex_moe_workspace_size(...) bytes, 256-B aligned.
 *   ws_bytes        the workspace's size in bytes; smaller than
 *                   reflex_moe_workspace_size(...) for this call's shapes:
 *                   REFLEX_EWORKSPACE, nothing enqueued.
 *   out             [T, d] output.
 *   rec             HOST struct, nullable: receives device pointers into the
 *                   workspace (no copy is made).
 * T == 0 launches no kernel; the workspace header (error word, totals) is
 * cleared in stream order, so reflex_moe_status reports this call.
 * Shape rules: T >= 0, d % 64 == 0, 1 <= E <= 1024, 1 <= k_max <= 32,
 * inter % 64 == 0, shared_inter % 64 == 0.  The bf16 tcgen05 path also needs
 * d % 256 == 0 and inter, shared_inter % 128 == 0 (else REFLEX_EUNSUPPORTED
 * unless REFLEX_FLAG_SIMT_EXPERTS is given).
 */
int reflex_moe_forward(int32_t dtype, const void* hidden, const void* w_router,
                       const void* w_gate_up, const void* w_down,
                       const void* shared_gate_up, const void* shared_down,
                       int32_t shared_inter, const int32_t* k, int32_t T,
                       int32_t d, int32_t E, int32_t inter, int32_t k_max,
                       uint32_t flags, void* workspace, size_t ws_bytes,
                       void* out, reflex_route_record* rec, void* stream);

/*
 * reflex_step — one denoising forward's hot path in one call: the per-token
 * counts of reflex_allocate (Eq. 5, Eq. 6-9, clip to [K_min, K_max]) for the
 * state arrays, then reflex_moe_forward with those counts (Eq. 2).  Every
 * output equals, bit for bit, that of reflex_allocate followed by
 * reflex_moe_forward on the same stream with the same arguments.  The
 * router scores do not depend on the counts, so the count kernel is launched
 * right behind the score kernel and runs beside it; the TopK selection waits
 * for both.
 *
 *   conf_prev1 .. active_block, B, p, k_out, k_sum_out: as for
 *                   reflex_allocate (T is the forward's T); alloc_status is
 *                   its device error word (nullable; stored or cleared by the
 *                   call, then OR-ed), separate from the forward's error word
 *                   in the workspace.
 *   dtype .. rec:   as for reflex_moe_forward; the counts read by the forward
 *                   are k_out (written by this call).
 * Ownership and errors: every pointer except rec and p is device memory owned
 * by the caller; nothing is allocated.  Any argument error of either half
 * returns its status before anything is launched.  The REFLEX_STAGE_* bits of
 * flags select the forward's stages as for reflex_moe_forward; the counts are
 * computed in every case.
 * With a score rule (p->count_rule TOP_P or EXPERT_THRESHOLD) the counts come
 * from the forward's own router scores: the TopK selection derives each k_i
 * from z_i (as reflex_allocate with those scores would), writes it to k_out
 * and selects with it; the state arrays are not read (they may be NULL), and
 * the ROUTE stage must be among the selected stages (else REFLEX_EINVAL).
 */
int reflex_step(const float* conf_prev1, const float* conf_prev2, const uint8_t* hist_len,
                const uint8_t* masked, const int32_t* block_id, const int32_t* seq_offsets,
                const int32_t* active_block, int32_t B, const reflex_alloc_params* p,
                int32_t* k_out, int64_t* k_sum_out, int32_t* alloc_status,
                int32_t dtype, const void* hidden, const void* w_router,
                const void* w_gate_up, const void* w_down, const void* shared_gate_up,
                const void* shared_down, int32_t shared_inter, int32_t T, int32_t d,
                int32_t E, int32_t inter, int32_t k_max, uint32_t flags, void* workspace,
                size_t ws_bytes, void* out, reflex_route_record* rec, void* stream);

/*
 * reflex_route_noalloc — the routing step of reflex_moe_forward (router
 * scores, TopK(r_i, k_i), router weights) for callers that cannot allocate
 * device memory: code inside a framework that owns the device allocator and
 * forbids side allocations, plugins limited to the buffers they are handed,
 * or processes where cudaMalloc is not allowed after start-up.  The paper has
 * no counterpart; it is a deployment convenience.
 *
 * The one scratch buffer of this step, the fp32 score matrix [T, E], lives
 * in a fixed array inside the library's device memory
 * (REFLEX_NOALLOC_MAX_SCORES floats = 4 MiB, held on every GPU that uses the
 * library until the process exits).  Nothing is allocated or freed.
 *   ids_out    [T, k_max] int32, alpha_out [T, k_max] fp32: same meaning and
 *              values as the ids / alpha of reflex_route_record.
 *   dev_status nullable device error word: cleared with a 4-byte memset in
 *              stream order before this call's kernels (also when T == 0),
 *              then OR-ed with error bits; read it with reflex_read_status.
 * Returns REFLEX_EWORKSPACE when T * E > REFLEX_NOALLOC_MAX_SCORES, and
 * REFLEX_EINVAL for the shape errors of reflex_moe_forward.  The first call
 * on each device looks up the array's address; make it before any stream
 * capture.  All calls share the array: calls whose GPU work overlaps in time
 * race on it and must be serialised.
 */
#define REFLEX_NOALLOC_MAX_SCORES (1 << 20)
int reflex_route_noalloc(int32_t dtype, const void* hidden,
                         const void* w_router, const int32_t* k, int32_t T,
                         int32_t d, int32_t E, int32_t k_max, uint32_t flags,
                         int32_t* ids_out, float* alpha_out,
                         int32_t* dev_status, void* stream);

/*
 * ---- 8-bit products -------------------------------------------------------
 * Values are held as e4m3 codes (OCP 8-bit floating point, largest 448) with
 * one fp32 scale for each block of 128 consecutive columns of a row
 * (activations) or for each 128 x 128 block (weights); the last block of a
 * row or column may be shorter.  A code c of scale s stands for c * s.
 */

/*
 * reflex_quantize_fp8 — rows [rows, cols] to codes and scales.  With a = the
 * largest magnitude of a block, at least 2^-100 (a NaN counts as largest):
 *   scale = a / 448,  code = e4m3(x * (448 * (1 / a)))
 * in fp32, each operation rounded to nearest even.  An infinity or a NaN makes
 * every value that its block stands for NaN.
 *   dtype       REFLEX_DTYPE_F32 or REFLEX_DTYPE_BF16 (of x).
 *   x           [rows, cols], row stride ldx >= cols elements, any alignment
 *               of the elements' own size.
 *   block_rows  1 (a scale per row and 128 columns) or 128 (per 128 x 128).
 *   codes       [rows, cols] bytes, row stride ldc >= cols.
 *   scales      [ceil(rows / block_rows), ceil(cols / 128)] fp32, row stride
 *               lds >= ceil(cols / 128).
 * rows == 0 or cols == 0 writes nothing.
 */
int reflex_quantize_fp8(int32_t dtype, const void* x, int64_t rows, int64_t cols,
                        int64_t ldx, int32_t block_rows, uint8_t* codes, int64_t ldc,
                        float* scales, int64_t lds, void* stream);

/*
 * reflex_matmul_fp8 — out = A B^T over codes:
 *   out[m, n] = sum_b sa[m, b] sb[n / 128, b] sum_{k in block b} A[m, k] B[n, k]
 * with fp32 sums; each block of K is summed by the tensor cores and scaled
 * once, by the product of both scales in fp32 (which has to be finite).
 *   a         [M, K] codes, row stride lda (a multiple of 16, >= K);
 *             a_scales [M, ceil(K / 128)], row stride ldas.
 *   b         [N, K] codes, row stride ldb (a multiple of 16, >= K);
 *             b_scales [ceil(N / 128), ceil(K / 128)], row stride ldbs.
 *   out_dtype REFLEX_DTYPE_F32 or REFLEX_DTYPE_BF16; out [M, N], row stride
 *             ldo >= N elements.
 *   dev_status nullable device error word, cleared by this call.
 * a and b start on 16-byte boundaries.  M == 0 computes nothing.  Any N, K
 * >= 1; the same bits for a row whatever M and the other rows are, as long as
 * the number of CTAs that share a tile's K stays the same (it is chosen from M,
 * N and K).  Sizes up to 2^30, and up to 2^30 tiles of 128 x 256 (else
 * REFLEX_EUNSUPPORTED).  Rows of out on 16-byte boundaries are stored fastest.
 */
int reflex_matmul_fp8(const uint8_t* a, int64_t lda, const float* a_scales, int64_t ldas,
                      const uint8_t* b, int64_t ldb, const float* b_scales, int64_t ldbs,
                      int32_t M, int32_t N, int32_t K, int32_t out_dtype, void* out,
                      int64_t ldo, int32_t* dev_status, void* stream);

/*
 * reflex_linear_fp8 — a dense layer in 8 bits: x [M, K] (fp32 or bf16, row
 * stride ldx) is quantised in rows as by reflex_quantize_fp8 and multiplied
 * with the codes w [N, K] and w_scales as by reflex_matmul_fp8.
 *   workspace  >= reflex_linear_fp8_workspace_size(M, K) bytes, 256-B aligned;
 *              its first word is the call's error word (reflex_moe_status).
 * A workspace sized for M rows serves every smaller batch.  One to four rows are
 * summed in another order than more, where that is faster (chosen from M, N, K).
 */
size_t reflex_linear_fp8_workspace_size(int32_t M, int32_t K);
int reflex_linear_fp8(int32_t dtype, const void* x, int64_t ldx, const uint8_t* w,
                      int64_t ldw, const float* w_scales, int64_t ldws, int32_t M,
                      int32_t N, int32_t K, int32_t out_dtype, void* out, int64_t ldo,
                      void* workspace, size_t ws_bytes, void* stream);

/*
 * reflex_experts_fp8 — the routed SwiGLU experts of Eq. 2 in 8 bits, for a
 * routing that the caller holds (the ids, alpha of a route record):
 *   out_t = sum_{j < k_t} alpha[t, j] E_{ids[t, j]}(h_t)   (+ h_t)
 * with h_t quantised in rows, the activation silu(g) u of each pair quantised
 * again in rows of 128 columns; the weighted sum is in fp32, of outputs that
 * tiles of many pairs store as bf16 and a few pairs keep in fp32.
 *   hidden         [T, d] bf16.
 *   ids, alpha     [T, k_max]: slots j < k[t] are read; an id outside [0, E)
 *                  there sets REFLEX_EINVAL in the error word and its pair
 *                  is left out, whatever its weight is.
 *   k              [T] int32 counts in [1, min(k_max, E)] (else REFLEX_EKRANGE
 *                  in the error word and the count is clamped).
 *   w_gate_up      [E, 2 inter, d] codes: gate rows, then up rows;
 *   gate_up_scales [E, 2, ceil(inter / 128), ceil(d / 128)]: the blocks of the
 *                  gate rows and of the up rows are counted by themselves.
 *   w_down         [E, d, inter] codes; down_scales [E, ceil(d / 128),
 *                  ceil(inter / 128)].
 *   flags          REFLEX_FLAG_RESIDUAL or 0.
 *   workspace      >= reflex_experts_fp8_workspace_size(...) bytes (0 for
 *                  shapes that are not supported), 256-B aligned; reads as
 *                  reflex_moe_forward's with reflex_moe_status.
 *   out            [T, d] bf16.
 * hidden, out and the codes start on 16-byte boundaries.  A few pairs (chosen
 * from T, k_max, d and inter) are summed in another order than more.  Shape
 * rules: d % 64 == 0, inter % 64 == 0, 1 <= E <= 1024, 1 <= k_max <= 32, T >= 0.
 */
size_t reflex_experts_fp8_workspace_size(int32_t T, int32_t d, int32_t E, int32_t inter,
                                         int32_t k_max);
int reflex_experts_fp8(const void* hidden, const int32_t* ids, const float* alpha,
                       const int32_t* k, const uint8_t* w_gate_up,
                       const float* gate_up_scales, const uint8_t* w_down,
                       const float* down_scales, int32_t T, int32_t d, int32_t E,
                       int32_t inter, int32_t k_max, uint32_t flags, void* workspace,
                       size_t ws_bytes, void* out, void* stream);

/*
 * reflex_sample — one token for each row of logits from given uniforms, with
 * its probability (the confidence that reflex_allocate and
 * reflex_update_state read).  Per row, with T, top_k, top_p, min_p its
 * settings and m its largest logit:
 *   1. weights w_i, about 2^31 exp((z_i - m) / T), integers:
 *      t = max((z_i - m) * c, -40), c = min(1.442695021629333 / T, FLT_MAX);
 *      n = t rounded to an integer (ties to even); f = t - n;
 *      p = 1 + f (c1 + f (c2 + f (c3 + f (c4 + f c5)))); w_i = floor(p 2^(n+31))
 *      in fp32, every operation rounded by itself, c1 .. c5 = 0.6931471824645996,
 *      0.2402234971523285, 0.055503811687231064, 0.00966636836528778,
 *      0.0013381302123889327 (to fp32);
 *   2. ranks by logit, higher first, lower index first on ties (-0 equals +0);
 *      top-k keeps the first top_k; top-p keeps of these the ones whose
 *      predecessors weigh less than top_p times all that top-k kept; min-p
 *      keeps those with w_i >= min_p 2^31;
 *   3. the token is the first, by index, at which the running weight of the
 *      kept tokens exceeds u times all of it (products and comparisons with
 *      top_p and u in fp64, where the sums are exact).
 * T == 0 takes the largest logit (lowest index on ties).  Sums of integers
 * have no order, so a row's token is the same whatever the batch.
 *   dtype        REFLEX_DTYPE_F32 or REFLEX_DTYPE_BF16 (of logits).
 *   logits       [rows, vocab], row stride ld >= vocab elements.  -inf and NaN
 *                are never sampled; with +inf, those tokens alone are, alike.
 *   temperature  [rows] fp32, >= 0 and finite; NULL: 1.
 *   top_k        [rows] int32, off at <= 0; NULL: off.
 *   top_p        [rows] fp32, > 0, off at >= 1; NULL: off.
 *   min_p        [rows] fp32, <= 1, off at <= 0; NULL: off.
 *   u            [rows] fp32, clamped to [0, 1 - 2^-24].
 *   masked       [rows] u8, nullable: rows with 0 are left out.
 *   tokens_out   [rows] int32.
 *   conf_out     [rows] fp32: exp(z_token - m) / sum_i exp(z_i - m), the softmax
 *                of the whole row at temperature 1, whatever the filters.
 *   dev_status   [1] int32 nullable device error word; bits are OR-ed in (not
 *                cleared): REFLEX_EINVAL for a row whose settings are outside
 *                the ranges above or NaN.
 * Such a row, a row that is left out and a row without a logit above -inf get
 * token -1 and confidence 0.  vocab up to 2^18 (else REFLEX_EUNSUPPORTED);
 * rows == 0 does nothing.
 */
int reflex_sample(int32_t dtype, const void* logits, int64_t ld, int32_t rows, int32_t vocab,
                  const float* temperature, const int32_t* top_k, const float* top_p,
                  const float* min_p, const float* u, const uint8_t* masked,
                  int32_t* tokens_out, float* conf_out, int32_t* dev_status, void* stream);

/*
 * ---- around the experts, with gradients -------------------------------------
 */

/*
 * reflex_block_norm — root-mean-square norms around a block, with its gate and
 * scale, on the residual stream.  With r(v) = 1 / sqrt(mean(v^2) + eps), per row:
 *   a = y r(y) w_after,   out = h + scale * gate * a,   norm = out r(out) w_before
 * in fp32 from the inputs to each output's one rounding (norm is taken from out
 * before that is rounded).
 *   dtype     REFLEX_DTYPE_F32 or REFLEX_DTYPE_BF16, of every tensor.
 *   h         [rows, d] the stream, row stride ldh >= d elements.
 *   y         [rows, d] the block's output (ldy), nullable: out = h.
 *   w_after   [d], nullable: a = y.
 *   gate      [rows, d] with row stride ldg >= d, or [d] with ldg == 0; nullable: 1.
 *   w_before  [d]; needed for norm.
 *   scale, eps  finite, eps >= 0.
 *   out, norm [rows, d] (ldo, ldn), either nullable.
 * w_after and gate need y.  An output may be h, y or a [rows, d] gate itself (the
 * same address and stride); else outputs overlap nothing.  Any d from 1 to 16384
 * (above: REFLEX_EUNSUPPORTED), any strides; rows on 16-byte boundaries with d a
 * multiple of 8 are fastest.  A row's bits do not depend on the other rows.
 */
int reflex_block_norm(int32_t dtype, const void* h, int64_t ldh, const void* y, int64_t ldy,
                      const void* w_after, const void* gate, int64_t ldg, const void* w_before,
                      float scale, float eps, int64_t rows, int32_t d, void* out, int64_t ldo,
                      void* norm, int64_t ldn, void* stream);

/*
 * reflex_block_norm_backward — its gradients, from d_out and d_norm, those of out
 * and of norm (one of them may be NULL; d_norm comes with w_before).
 *   d_h, d_y  [rows, d]; d_y comes with y.
 *   d_gate, d_w_after, d_w_before  of their inputs' shapes; nullable: not wanted.
 *             Those of a [d] input are sums over the rows, in fp32 and in an order
 *             that depends on rows, d and the GPU alone.
 *   workspace >= reflex_block_norm_workspace_size(rows, d) bytes (0 for widths that
 *             are not supported), 256-B aligned; one for more rows serves fewer of
 *             the same width.
 * An output may be an input of its own shape, as above.  rows == 0 leaves zeros in
 * the sums.
 */
size_t reflex_block_norm_workspace_size(int64_t rows, int32_t d);
int reflex_block_norm_backward(int32_t dtype, const void* h, int64_t ldh, const void* y,
                               int64_t ldy, const void* w_after, const void* gate, int64_t ldg,
                               const void* w_before, float scale, float eps, int64_t rows,
                               int32_t d, const void* d_out, int64_t ld_d_out,
                               const void* d_norm, int64_t ld_d_norm, void* d_h, int64_t ld_d_h,
                               void* d_y, int64_t ld_d_y, void* d_gate, int64_t ld_d_gate,
                               void* d_w_after, void* d_w_before, void* workspace,
                               size_t ws_bytes, void* stream);

/*
 * reflex_expert_plan — the rows of token-expert pairs in expert order, as in the
 * record of reflex_moe_forward, for a routing that the caller holds.  Pairs (t, j)
 * are numbered in order of (expert, token, slot).
 *   ids       [T, k_max]; without k a negative id marks an unused slot.
 *   k         [T] int32, nullable: slots j < k[t] are used.  A count outside
 *             [0, k_max] sets REFLEX_EKRANGE in the error word and is clamped.
 *   row_of    [T, k_max] the pair's row, -1 without one: unused slots, pairs whose
 *             id is outside [0, E) (REFLEX_EINVAL in the error word) and pairs past
 *             the first cap_rows rows (REFLEX_ECAPACITY).
 *   counts    [E], offsets [E + 1]: rows of expert e are offsets[e] .. offsets[e + 1]
 *             - 1 (before the cut at cap_rows).
 *   perm      [>= pairs] nullable: row -> t * k_max + j.
 *   dev_status nullable device error word, cleared by this call.
 *   workspace >= reflex_expert_plan_workspace_size(...) bytes (0 for shapes that are
 *             not supported), 256-B aligned; one for more tokens serves fewer.
 * An expert may come several times in a token.  Shape rules: 1 <= E <= 1024,
 * 1 <= k_max <= 32, 0 <= T * k_max <= 2^30.
 */
size_t reflex_expert_plan_workspace_size(int64_t T, int32_t E, int32_t k_max);
int reflex_expert_plan(const int32_t* ids, const int32_t* k, int64_t T, int32_t E, int32_t k_max,
                       int64_t cap_rows, int32_t* row_of, int32_t* counts, int32_t* offsets,
                       int32_t* perm, int32_t* dev_status, void* workspace, size_t ws_bytes,
                       void* stream);

/*
 * reflex_expert_rows — tokens to their experts: rows[row_of[t, j]] = x[t].
 *   x         [T, d] (ldx); rows [cap_rows, d] (ldr).  Rows without a pair are
 *             left as they are.  row_of outside [0, cap_rows) is an unused slot.
 * Its gradient is reflex_expert_combine with alpha == NULL and no residual.  In these
 * calls d is at most 2^30 (above: REFLEX_EUNSUPPORTED).
 */
int reflex_expert_rows(int32_t dtype, const void* x, int64_t ldx, const int32_t* row_of,
                       int64_t T, int32_t d, int32_t k_max, int64_t cap_rows, void* rows,
                       int64_t ldr, void* stream);

/*
 * reflex_expert_combine — and back: out[t] = sum_j alpha[t, j] rows[row_of[t, j]]
 * (+ residual[t]), summed in fp32 in the order of j and rounded once.
 *   alpha     [T, k_max] fp32, of used slots; NULL: 1.
 *   residual  [T, d] (ldres), nullable; out [T, d] (ldo), which may be residual.
 */
int reflex_expert_combine(int32_t dtype, const void* rows, int64_t ldr, const float* alpha,
                          const int32_t* row_of, const void* residual, int64_t ldres, int64_t T,
                          int32_t d, int32_t k_max, int64_t cap_rows, void* out, int64_t ldo,
                          void* stream);

/*
 * reflex_expert_combine_backward — its gradients (that of the residual is d_out):
 *   d_rows[row_of[t, j]] = alpha[t, j] d_out[t]   [cap_rows, d], nullable; rows
 *             without a pair are left as they are.  d_rows may be rows.
 *   d_alpha[t, j] = <d_out[t], rows[row_of[t, j]]>  [T, k_max] fp32, nullable; 0 in
 *             unused slots.
 */
int reflex_expert_combine_backward(int32_t dtype, const void* d_out, int64_t ld_d_out,
                                   const void* rows, int64_t ldr, const float* alpha,
                                   const int32_t* row_of, int64_t T, int32_t d, int32_t k_max,
                                   int64_t cap_rows, void* d_rows, int64_t ld_d_rows,
                                   float* d_alpha, void* stream);

/*
 * reflex_head_loss — softmax cross entropy of a vocabulary head, with no logits kept:
 *   z[r, v] = sum_k hidden[r, k] w[v, k],  lse[r] = log sum_v exp z[r, v],
 *   loss[r] = lse[r] - z[r, targets[r]]
 * for the rows with a target; loss and lse are 0 for the others, whose hidden row is
 * not read.  Sums, exponentials and logits are fp32.
 *   hidden    [rows, k] bf16, row stride ld_hidden >= k, any alignment of 2 bytes.
 *   w         [vocab, k] bf16, row stride ldw >= k: rows start on 16-byte boundaries
 *             (w and ldw * 2 are multiples of 16).
 *   targets   [rows] int32; a negative one leaves its row out, one >= vocab too, with
 *             REFLEX_EINVAL in the error word.
 *   loss, lse [rows] fp32.
 *   dev_status nullable device error word, cleared by this call.
 *   workspace >= reflex_head_loss_workspace_size(...) bytes (0 for shapes that are not
 *             supported), 256-B aligned.
 * Any sizes up to 2^24 rows, 2^24 columns of the vocabulary and k = 2^20 (above:
 * REFLEX_EUNSUPPORTED).  A row's results have the same bits on every run, whatever
 * the other rows are; up to 64 rows are summed in another order than more.  A row with
 * a logit that is not finite has no influence on others.
 */
size_t reflex_head_loss_workspace_size(int32_t rows, int32_t vocab, int32_t k);
int reflex_head_loss(const void* hidden, int64_t ld_hidden, const void* w, int64_t ldw,
                     const int32_t* targets, int32_t rows, int32_t vocab, int32_t k, float* loss,
                     float* lse, int32_t* dev_status, void* workspace, size_t ws_bytes,
                     void* stream);

/*
 * reflex_head_loss_backward — its gradients from grad[r], the gradient of loss[r] (that
 * of a mean is 1 / rows, of a weighted loss the weight), and the forward call's lse:
 *   G[r, v] = grad[r] (exp(z[r, v] - lse[r]) - [v == targets[r]])
 *   d_hidden = G w  [rows, k], zeros in rows left out;  d_w = G^T hidden  [vocab, k]
 * with sums in fp32, of terms of which G is rounded to bf16, but for those of the targets
 * (in d_w those of a token's first four rows), which are taken in fp32.  The logits are
 * computed again, a piece of the vocabulary at a time.
 *   lse, grad [rows] fp32, of rows with a target.
 *   d_hidden, d_w  fp32 or bf16 by their dtype argument, any strides; either may be
 *             NULL (not wanted).  Rows of d_w on 16-byte boundaries are stored fastest.
 *             d_hidden may be hidden; else they overlap nothing (REFLEX_EINVAL where one
 *             shares bytes with w or with the other, or crosses it with rows of another
 *             stride).
 *   workspace >= reflex_head_loss_backward_workspace_size(...) bytes (for these very
 *             sizes), 256-B aligned.
 * The rest as in reflex_head_loss; the same bits on every run.
 */
size_t reflex_head_loss_backward_workspace_size(int32_t rows, int32_t vocab, int32_t k);
int reflex_head_loss_backward(const void* hidden, int64_t ld_hidden, const void* w, int64_t ldw,
                              const int32_t* targets, const float* lse, const float* grad,
                              int32_t rows, int32_t vocab, int32_t k, int32_t d_hidden_dtype,
                              void* d_hidden, int64_t ld_d_hidden, int32_t d_w_dtype, void* d_w,
                              int64_t ld_d_w, int32_t* dev_status, void* workspace,
                              size_t ws_bytes, void* stream);

/* Synchronises `stream` and returns the status recorded in the workspace's
 * device error word by the last forward (REFLEX_OK if clean). */
int reflex_moe_status(const void* workspace, void* stream);

/* Same for a caller-owned device error word (e.g. reflex_allocate's). */
int reflex_read_status(const int32_t* dev_status, void* stream);

/* Bounded-wait self-test: launches one block that waits on an mbarrier no
 * one arrives at, with a limit of `limit_us` microseconds (1..100000), then
 * records REFLEX_ETIMEOUT in dev_status and returns.  Exercises the same
 * wait routine the tcgen05 pipeline uses; nothing hangs. */
int reflex_selftest_wait_timeout(int32_t* dev_status, uint32_t limit_us,
                                 void* stream);

/* Human-readable status. */
const char* reflex_status_string(int status);

/* Version of this ABI (major * 100 + minor). */
int reflex_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* REFLEX_H */
