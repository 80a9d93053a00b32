// internal.h — launchers shared between the kernel files and the C-ABI host
// code (reflex_abi.cu).  Not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

#include "common.cuh"

namespace rx {

// Lets a kernel have `bytes` of dynamic shared memory, asking the runtime once for each
// device (`done`, a bit a device): the call takes longer than the checks of a launch.
template <typename K>
inline cudaError_t allow_smem(K kernel, size_t bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint64_t bit = uint64_t{1} << (dev & 63);
  if (e != cudaSuccess || (done.load(std::memory_order_relaxed) & bit)) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           static_cast<int>(bytes));
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

struct AllocArgs {
  int k_min, k_base, k_max, delta_role, delta_cur;
  float q, theta, w_cf, v_ref, tau;
  int signal;             // rank key of the Eq. 9 groups (REFLEX_SIGNAL_*)
  int role_shuffle;       // permute each sequence's final counts
  uint64_t shuffle_seed;  // splitmix64 seed of the permutation keys
  int count_rule;         // REFLEX_RULE_*: 0 = this allocation, else a score rule
  float rule_threshold;   // p of Top-p / the expert-threshold router weight
};

// ---- allocation (budget.cu) -----------------------------------------------
// alongside: launched right after a kernel that writes none of the inputs
// (the router scores of the same forward) and, when B > 1, itself or the one
// in front of it clears err / k_sum; the counts then run next to that kernel,
// and the budget grid adds to the two words and completes only after it.
// Otherwise, when B > 1, the caller has cleared them.
cudaError_t launch_budget(const float* conf1, const float* conf2,
                          const uint8_t* hist_len, const uint8_t* masked,
                          const int32_t* block_id, const int32_t* seq_off,
                          const int32_t* active_block, int T, int B,
                          const AllocArgs& a, int32_t* k_out,
                          unsigned long long* k_sum, uint32_t* err,
                          cudaStream_t stream, bool alongside = false);
cudaError_t launch_wait_selftest(uint32_t* err, uint64_t limit_ns,
                                 cudaStream_t stream);

// ---- refinement-state update (state.cu) ------------------------------------
cudaError_t launch_update_state(const float* conf_new, float* conf1, float* conf2,
                                uint8_t* hist_len, uint8_t* masked, const int32_t* block_id,
                                const int32_t* seq_off, int32_t* active,
                                const int32_t* num_blocks, int T, int B, float theta,
                                int32_t* committed, uint32_t* err, cudaStream_t stream);

// ---- routing (router.cu) --------------------------------------------------
// z[T, E] = router scores (sequential fp32 fma chain over the hidden index).
// The first CTA also clears the zero words (the call's header or error word,
// the allocation's outputs), so no memset precedes the first kernel.  err
// (nullable) receives kErrTimeout if a bounded wait of a kernel expires.
// pf (optional): bytes the score kernel hands to the L2 as bulk prefetches
// while it computes (the next kernels' weights; HBM is otherwise idle then).
struct L2Prefetch {
  const void* base = nullptr;
  uint64_t bytes = 0;  // a multiple of 16
};
cudaError_t launch_router_logits(int dtype, const void* hidden,
                                 const void* w_router, int T, int d, int E,
                                 float* z, const ZeroWords& zero, uint32_t* err,
                                 int num_sms, cudaStream_t stream,
                                 const L2Prefetch& pf = L2Prefetch{});
// Screened routing (bf16, renormalised weights): nw[e] = ||w_e||_2 rounded up
// (first kernel of the forward; clears the zero words like the score kernels);
// then, from the tensor-core score slices z[s][t][e] (s < k_splits), the
// exact TopK, alpha and ids, with the canonical chain recomputed for every
// expert that could be selected (written back into z's first slice).
cudaError_t launch_router_wnorm(const __nv_bfloat16* w, int E, int d, float* nw,
                                const ZeroWords& zero, cudaStream_t stream);
cudaError_t launch_router_screen_select(const __nv_bfloat16* h, const __nv_bfloat16* w,
                                        float* z, int k_splits, int64_t split_stride,
                                        const float* nw, const int32_t* k, int T, int E,
                                        int d, int k_max, int32_t* ids, float* alpha,
                                        uint32_t* err, cudaStream_t stream);
// Tile width and K slices of the screen GEMM for T x E scores over d: slices
// double while the tile count stays within 152 (this GPU's SM count).
inline int screen_bn(int E) { return E <= 64 ? 64 : 128; }
inline int screen_splits(int T, int E, int d) {
  const int64_t mt = (T + 127) / 128, nt = (E + screen_bn(E) - 1) / screen_bn(E);
  const int nkb = d / 64;
  int s = 1;
  while (s < 16 && mt * nt * s * 2 <= 152 && nkb % (2 * s) == 0) s *= 2;
  return s;
}
// Rows of the workspace's score region for the screen GEMM's slices: s T,
// and never fewer than for a smaller batch (s falls as T adds tiles, and a
// workspace sized for a batch must serve every smaller one).  A batch of m
// full 128-row tiles has the most rows among those of m tiles; beyond 152
// tiles s = 1.
inline int64_t screen_z_rows(int T, int E, int d) {
  int64_t rows = static_cast<int64_t>(screen_splits(T, E, d)) * T;
  const int64_t mt = (T + 127) / 128;
  for (int64_t m = 1; m < mt && m <= 152; ++m) {
    const int64_t r = screen_splits(static_cast<int>(m * 128), E, d) * m * 128;
    if (r > rows) rows = r;
  }
  return rows;
}
// Batched screen for E <= 256 (bf16, renormalised weights): z holds the
// tensor-core estimates [T, E] (one K slice), hss the tokens' sums of
// squares, nw the experts' norms (wnorm_kernel); map_h / map_w are 2D maps of
// the hidden states [T, d] and the router weights [E, d] with boxes of 64
// columns and screen_batch_token_rows(E) / screen_batch_expert_rows(E) rows, not
// swizzled.  Writes ids / alpha and the candidates' exact scores into z.
// the box heights of map_h (tokens per CTA) and map_w for E experts
int screen_batch_token_rows(int E);
int screen_batch_expert_rows(int E);
cudaError_t launch_router_screen_batch(const CUtensorMap* map_h, const CUtensorMap* map_w,
                                       float* z, const float* hss, const float* nw,
                                       const int32_t* k, int T, int E, int d, int k_max,
                                       int32_t* ids, float* alpha, uint32_t* err,
                                       int num_sms, cudaStream_t stream);
// The counts from the router scores (count rules 1 = Top-p, 2 = expert
// threshold, threshold thr, clip [k_lo, min(k_hi, E)]) into k_out (and added
// to k_sum, nullable, which the caller cleared), then ids / alpha [T, k_max]
// as launch_router_select gives them for those counts; ids == nullptr:
// counts only.
cudaError_t launch_router_select_rule(const float* z, int T, int E, int k_hi, int k_lo,
                                      int rule, float thr, int k_max, bool renorm,
                                      int32_t* k_out, unsigned long long* k_sum,
                                      int32_t* ids, float* alpha, cudaStream_t stream);
// ids/alpha [T, k_max] from z and the counts k.
cudaError_t launch_router_select(const float* z, const int32_t* k, int T,
                                 int E, int k_max, bool renorm, int32_t* ids,
                                 float* alpha, uint32_t* err,
                                 cudaStream_t stream);

// ---- dispatch (dispatch.cu) -----------------------------------------------
struct DispatchBufs {
  int32_t* blk_count;  // [nblk, E]
  int32_t* blk_off;    // [nblk, E]
  int32_t* counts;     // [E]
  int32_t* offsets;    // [E+1]
  int32_t* mt_prefix;  // [E+1] 128-row tiles
  int32_t* mt2_prefix; // [E+1] 256-row tiles
  int32_t* perm;       // [T*k_max]
  int32_t* row_of;     // [T*k_max]
  int32_t* totals;     // header: total_pairs, total_mtiles, total_mtiles2
  uint32_t* err;
  uint32_t* blk_mask;  // [nblk, E, BLK / 32] token bits of each block and expert
  // a caller's routing: its weights [T*k_max], and the same with 0 in slots without a
  // row (clamped away or refused), as the combine takes them; null otherwise
  const float* alpha = nullptr;
  float* weights = nullptr;
};
constexpr int kDispatchBlock = 256;       // tokens per dispatch block, large batches
constexpr int kDispatchBlockSmall = 32;   // tokens per dispatch block up to 4096 tokens
constexpr int kDispatchSmallT = 4096;
inline int dispatch_block(int T) { return T <= kDispatchSmallT ? kDispatchBlockSmall : kDispatchBlock; }
// per-block count buffers sized for either block size (monotonic in T, so a
// workspace sized for a batch also fits every smaller one)
inline int64_t dispatch_blocks_alloc(int T) {
  const int ts = T < kDispatchSmallT ? T : kDispatchSmallT;
  return (ts + kDispatchBlockSmall - 1) / kDispatchBlockSmall +
         (T + kDispatchBlock - 1) / kDispatchBlock;
}
// The pair layout (counts, offsets, tile prefixes, perm, row_of) and the
// gathered rows X_perm[row_of[t, j]] = X[t] for j < k_t (x_perm nullptr:
// the layout only, for a consumer that gathers the rows itself).
// mask words for either block size (monotonic in T, like the block counts)
inline int64_t dispatch_mask_words_alloc(int T) {
  const int ts = T < kDispatchSmallT ? T : kDispatchSmallT;
  return (ts + kDispatchBlockSmall - 1) / kDispatchBlockSmall +
         static_cast<int64_t>(T + kDispatchBlock - 1) / kDispatchBlock * (kDispatchBlock / 32);
}
cudaError_t launch_dispatch_gather(int dtype, const void* hidden, const int32_t* ids,
                                   const int32_t* k, int T, int E, int k_max, int cap_rows,
                                   int d, const DispatchBufs& b, void* x_perm, int num_sms,
                                   cudaStream_t stream);

// ---- experts: SIMT grouped GEMMs (experts_simt.cu) ------------------------
// Grouped mode: rows [offsets[e], offsets[e+1]) use expert e; dense mode
// (offsets == nullptr): rows [0, dense_rows) use the single weight set.
struct GroupRows {
  const int32_t* offsets;    // [E+1] or nullptr
  const int32_t* mt_prefix;  // [E+1] prefix of 128-row tile counts
  const int32_t* mt2_prefix; // [E+1] prefix of 256-row tile counts
  const int32_t* totals;     // device total rows (grouped mode)
  int E;
  int dense_rows;
  int cap_rows;
};
cudaError_t launch_swiglu_simt(int dtype, const void* x, const void* w_gate_up,
                               int d, int inter, const GroupRows& g, void* act,
                               int num_sms, cudaStream_t stream);
cudaError_t launch_down_simt(int dtype, const void* act, const void* w_down,
                             int d, int inter, const GroupRows& g, void* y,
                             int num_sms, cudaStream_t stream);

// ---- experts: tcgen05 grouped GEMMs (experts_tc.cu) -----------------------
struct TcGemmArgs {
  const CUtensorMap* map_a;  // A [rows, K] bf16, box {64, 128}, 128B swizzle
  const CUtensorMap* map_b;  // B [groups * rows_per_group, K] bf16
  int K;                     // reduction length
  int n_total;               // output columns per group (SwiGLU: inter)
  int b_rows_per_group;      // SwiGLU: 2*inter, down: d
  int b_up_offset;           // SwiGLU: inter (row offset of up weights)
  GroupRows g;               // row groups
  void* out;                 // [rows, ldo] bf16
  int ldo;
  uint32_t* err;
  int num_sms;
  // SwiGLU, 1-SM kernel: map_b is the 3D map of tc_gate_up_3d (box {64,
  // bn / 2, 2}: a tile's gate and up rows in one copy) instead of a 2D map
  bool b_gate_up_3d = false;
  // SwiGLU, CTA-pair kernel: when set, A row r is row gather_perm[r] /
  // gather_kmax (row r's pair index over k_max) of the token rows gather_x
  // [gather_tokens, K], copied by four warps of the kernel; nullptr: map_x
  // holds the rows in pair order
  const int32_t* gather_perm = nullptr;
  const void* gather_x = nullptr;
  int gather_kmax = 0;
  int gather_tokens = 0;
  // CTA-pair kernels: 2D map of out [rows, ldo] with a {64, 32} box, 128-byte
  // swizzle; whole 32-row output chunks are written by TMA stores through it
  const CUtensorMap* map_out = nullptr;
  // CTA-pair kernels (instead of map_a): four maps of A with boxes of 32, 64,
  // 96 and 128 rows
  const CUtensorMap* map_x = nullptr;
  // 1-SM kernels, grouped rows: a dense problem (the shared expert) whose
  // tiles the same launch computes; map_b of the kind of this one, n_total a
  // multiple of the tile's columns
  const TcGemmArgs* shared = nullptr;
  // the kernel in front of this one in the stream waited for the dispatch
  // (the tile prefix) before it let this launch start: the first weights may
  // be requested before this kernel's own wait
  bool early_b = false;
  // CTA-pair kernels: weight tiles with one reader are loaded evict-first
  bool once = false;
};
// SwiGLU: out = silu(A Wg^T) * (A Wu^T).  Down: out = A Wd^T.  bn = tile
// width (128 or 256, from tc_pick_bn); the B tensor map's box must have
// tc_b_box_rows(swiglu, bn) rows.
cudaError_t launch_swiglu_tc(const TcGemmArgs& a, int bn, cudaStream_t stream);
cudaError_t launch_down_tc(const TcGemmArgs& a, int bn, cudaStream_t stream);
int tc_b_box_rows(bool swiglu, int bn);
// Router-score screen: out[ks][t][e] = sum over the ks-th of k_splits equal
// slices of k of A[t, k] B[e, k] (fp32 accumulators, dense rows t < T =
// a.g.dense_rows, columns e < n_valid, row stride a.ldo), bn in {64, 128, 256}
// (B tensor map box of bn rows); a.K / 64 must be a multiple of k_splits.
// defer_wait: launched right behind a kernel that writes none of its inputs
// or outputs (it then overlaps that kernel and waits for it before exiting).
// row_norms (nullable, k_splits == 1 only): the sum of squares of every A
// row (fp32, one per row), computed from the staged A tiles.
cudaError_t launch_scores_tc(const TcGemmArgs& a, int bn, int k_splits, float* out,
                             int64_t split_stride, int n_valid, bool defer_wait,
                             cudaStream_t stream, float* row_norms = nullptr);
// CTA-pair (2-SM, cta_group::2) variants: tiles of 256 weight rows x up to
// 256 token rows, cluster of two CTAs; needs map_x, map_out and
// GroupRows::mt2_prefix in grouped mode.  map_b: SwiGLU a 5D map {K, 16, 2,
// inter / 16, groups} of the gate/up weights with box {64, 16, 2, 4, 1}, down
// a 2D map with boxes of 128 rows.  n_total must be a multiple of 128
// (SwiGLU) or 256 (down).
cudaError_t launch_swiglu_tc_pair(const TcGemmArgs& a, cudaStream_t stream);
cudaError_t launch_down_tc_pair(const TcGemmArgs& a, cudaStream_t stream);
int tc_n_granule(bool swiglu, int bn);  // output columns per tile
// 0 when n_total is not a multiple of the smaller granule.
int tc_pick_bn(bool swiglu, int n_total, int64_t mtiles_est, int num_sms);

// ---- combine (combine.cu) -------------------------------------------------
// out[t] = sum_{j<k_t} alpha[t,j] * y[row_of[t,j]] (+ y_shared[t]) (+ resid[t]).
cudaError_t launch_combine(int dtype, const void* y, const void* y_shared,
                           const void* resid, const int32_t* row_of, const float* alpha,
                           const int32_t* k, int T, int d, int k_max,
                           int cap_rows, void* out, uint32_t* err, int num_sms,
                           cudaStream_t stream);

// ---- sampling (sample.cu) ---------------------------------------------------
struct SampleArgs {
  const void* logits;  // [rows, vocab], row stride ld
  int64_t ld;
  int rows, vocab;
  const float* temperature;  // nullable, like the next three and masked
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  const uint8_t* masked;
  int32_t* tokens;
  float* conf;
  uint32_t* err;
};
int sample_max_vocab();
cudaError_t launch_sample(int dtype, const SampleArgs& p, int num_sms, cudaStream_t stream);

// ---- norms around a block (block_norm.cu) -------------------------------------
struct BlockNormArgs {
  int64_t rows;
  int d;
  int tpr, depth;  // set by the launcher: threads that share a row, rows of the ring
  float scale, eps;
  const void* h;
  int64_t ldh;
  const void* y;  // nullable
  int64_t ldy;
  const void* w_after;  // nullable
  const void* gate;     // nullable; ldg == 0: one row for all
  int64_t ldg;
  const void* w_before;  // nullable
  void* out;             // forward
  int64_t ldo;
  void* norm;
  int64_t ldn;
  const void* d_out;  // backward; nullable
  int64_t ld_d_out;
  const void* d_norm;
  int64_t ld_d_norm;
  void* d_h;
  int64_t ld_d_h;
  void* d_y;
  int64_t ld_d_y;
  void* d_gate;  // nullable, like the next two
  int64_t ld_d_gate;
  void* d_w_after;
  void* d_w_before;
  float* partial;  // [3][block_norm_parts][d]: sums of the weights' gradients
};
int block_norm_max_width();
// sums of a weight's gradient before they are added up, at most
int64_t block_norm_parts(int64_t rows, int d, int sms);
cudaError_t launch_block_norm(int dtype, const BlockNormArgs& p, bool backward, int sms,
                              cudaStream_t s);

// ---- tokens to experts and back (expert_rows.cu) --------------------------------
// CTAs of a plan of so many pairs or fewer
int64_t expert_plan_blocks_most(int64_t pairs, int sms);
cudaError_t launch_expert_plan(const int32_t* ids, const int32_t* k, int64_t T, int E, int k_max,
                               int cap_rows, int32_t* row_of, int32_t* counts, int32_t* offsets,
                               int32_t* perm, uint32_t* err, int32_t* blk_count, int sms,
                               cudaStream_t s);
struct ExpertRowsArgs {
  const int32_t* row_of;
  int64_t T;
  int d, k_max, cap_rows;
  const void* x;  // by token: tokens, residual (nullable), gradient of the output
  int64_t ldx;
  const void* rows;  // by pair
  int64_t ldr;
  const float* alpha;  // nullable in sums: 1
  void* out;           // what is written: rows, sums, gradient of the rows (nullable)
  int64_t ldo;
  float* d_alpha;  // nullable
};
cudaError_t launch_expert_rows(int dtype, const ExpertRowsArgs& p, int sms, cudaStream_t s);
cudaError_t launch_expert_combine(int dtype, const ExpertRowsArgs& p, bool backward, int sms,
                                  cudaStream_t s);

// ---- loss of a vocabulary head (head_loss.cu) --------------------------------------
constexpr int kHeadTile = 256;  // rows and columns of a tile of any of its products
constexpr int kHeadFewRows = 64;  // as many rows or fewer go past W, not W past them
constexpr int kHeadGroup = 32;  // tiles of rows that stay in L2 while the weights pass by

// The rows with a target in [0, vocab) to the front, zeros behind them up to whole
// tiles; what the other kernels read of each, its target's logit among it.  Clears the
// queue and sets the error word.
struct HeadRows {
  int64_t rows;
  int vocab, k;
  int tile;  // rows of a whole tile
  const int32_t* targets;
  const __nv_bfloat16* hidden;
  int64_t ld_hidden;
  const float* lse;   // nullable, with row_lse
  const float* grad;  // nullable, with row_grad
  __nv_bfloat16* packed;
  int64_t ld_packed;
  int* row;     // [rows] packed row -> row
  int* target;  // [rows up to whole tiles], like the next two
  float* row_lse;
  float* row_grad;
  const __nv_bfloat16* w;
  int64_t ldw;
  float* z_target;     // forward
  float* target_term;  // backward
  int* place;  // [rows] nullable: row -> packed row or -1
  int* live;
  uint32_t* queue;
  int n_queue;
  float* loss_out;  // nullable: zeros for the rows left out
  float* lse_out;
  uint32_t* err;  // nullable
};
cudaError_t launch_head_rows(const HeadRows& p, int sms, cudaStream_t stream);
// Whether W goes past the rows, for a vocabulary in `pieces`.
inline bool head_few_rows(int64_t rows, int pieces) { return rows <= kHeadFewRows && pieces == 1; }
// Then: columns of a tile, rows of W in one (what the CTAs' rounds of 128 leave shared out
// evenly), and the CTAs, each of which leaves a maximum and a sum for every column.
inline int head_few_columns(int64_t rows) { return rows <= 32 ? 32 : kHeadFewRows; }
inline int head_few_tile_rows(int vocab, int sms) {
  const int rounds = (vocab + sms * (kHeadTile / 2) - 1) / (sms * (kHeadTile / 2));
  return (vocab + sms * rounds - 1) / (sms * rounds);
}
inline int head_few_ctas(int vocab, int sms) {
  const int rows = head_few_tile_rows(vocab, sms), tiles = (vocab + rows - 1) / rows;
  return tiles < sms ? tiles : sms;
}

struct HeadProblem {
  PFN_cuTensorMapEncodeTiled_v12000 encode;
  const __nv_bfloat16* packed;
  int64_t ld_packed;
  const void* w;
  int64_t ldw;
};
struct HeadTiles {
  int rows, vocab, k;
  int rows_up;  // rows up to whole tiles
  const int* live;
  const __nv_bfloat16* packed;
  int64_t ld_packed;
  const int* row;
  const int* target;
  const float* row_lse;
  const float* row_grad;
  const float* z_target;     // [rows_up] the target's logit
  const float* target_term;  // [rows_up] G's term of the row's target, in fp32
  // maximum and sum: [2 * tiles of the vocabulary][rows_up]; of few rows [head_few_ctas]
  // [head_few_columns]
  float2* stats;
  int64_t ld_stats;
  uint32_t* queue;
  uint32_t* err;
  void* dw;  // nullable
  int64_t ld_dw;
  int dw_f32;
  int ld_sums;
  // set by the launchers: the piece whose gradients are taken (vt tiles from column v0)
  // and the one whose G is made (vt_next from v_next)
  int vt, v0, vt_next, v_next;
  int kt, parts, part_blocks, hidden_first, dw_mapped;
};
// G in pieces of piece_tiles tiles of the vocabulary (two of them, or one if that is
// all), the sums of Dh in parts of part_blocks stages each.
struct HeadPieces {
  int piece_tiles, part_blocks, parts;
  __nv_bfloat16* g;
  float* sums;  // [parts][rows_up][ld_sums]; nullable: no gradient of the rows
};
cudaError_t launch_head_loss(const HeadProblem& h, HeadTiles p, float* loss, float* lse, int sms,
                             cudaStream_t stream);
cudaError_t launch_head_loss_backward(const HeadProblem& h, HeadTiles p, const HeadPieces& q,
                                      const int* place, int64_t rows, void* d_hidden,
                                      int64_t ld_d_hidden, bool d_hidden_f32, int sms,
                                      cudaStream_t stream);

}  // namespace rx
