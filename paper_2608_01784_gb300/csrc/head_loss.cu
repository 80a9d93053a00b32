// head_loss.cu — softmax cross entropy of a vocabulary head without its logits in
// memory, and its gradients, on the 5th-generation tensor cores:
//   z = h W^T,  lse[r] = log sum_v exp z[r, v],  loss[r] = lse[r] - z[r, target[r]]
//   G[r, v] = c[r] (exp(z[r, v] - lse[r]) - [v = target[r]]),  Dh = G W,  DW = G^T h
// for the rows r with a target, which lie packed in front (head_rows_kernel); c[r] is
// the gradient of loss[r].
//
// Every product is made of tiles of 256 x 256 by pairs of CTAs (cta_group::2, M = 256,
// two accumulators of 256 columns in all of TMEM), fed by TMA through a ring of six
// stages of 64 along the reduction:
//   loss    z tile -> each thread has a row of 128 columns in fp32, of which it leaves
//           the maximum and the sum of exponentials;
//   grad    z tile -> G in bf16, a piece of the vocabulary at a time (MN-major operands
//           of the next two, straight from row-major memory);
//   hidden  G W of a part of the piece, added in fp32 where the last piece left off;
//   weight  G^T h, stored as it is wanted.
// A launch of the backward pass holds the hidden and weight tiles of one piece and the
// grad tiles of the next, which do not depend on each other, so that a launch has but
// one tail; pairs take tiles from a queue, the long ones first.  Every tile is summed
// by one pair in one order, wherever it runs: results do not depend on timing.
//
// A row's logit of its target is the one that its loss and its largest term of G depend
// on most, so it is added up in fp32 by itself (head_rows_kernel) and stands in its tile
// instead of the tensor cores' sum.  G is rounded to bf16, by up to 2^-8 of each term, as
// the products take it; what that takes from the target's term is added in fp32 where the
// gradients are put together (to the weights of a token for its first four rows, behind
// which roundings average out).  999 x 50001 x 2048: gradients in bf16 are off by 1.66e-3
// of their norm, as much as their own rounding, and were by 2.37e-3 without; a few rows,
// or rows of one weight, by up to 4e-3.  z, the sums of exponentials and all accumulators
// are fp32.  exp(z - m) is taken as 2^((z - m) c), c = log2 e: the difference is exact
// where it matters, however large z and m are (z c - m c is off by the rounding of m c,
// 0.4 at m = 1e7).
//
// Bound: the tensor cores, in a loop of seconds under the card's power cap (1.37 kW).
// 8192 rows x 16384 x 2048: the loss 326 to 340 us, 1.65 PFLOP/s (cuBLAS's product alone
// 307 at its best, 316 in a loop); x 131072 with both gradients, 8 M V K operations, 11.2
// ms, 1.57 PFLOP/s.  The operands' way from L2 (13 TB/s) is not far: clusters of two pairs that send
// each other half of W's tile need a quarter less of it, but only 36 of them find room, and
// they were 5 % slower.  With small K the exponentials: a tile takes 3200 cycles for them,
// 2048 for its products at K = 256 (16384 x 32000: 306 us).
//
// Every wait on a barrier in shared memory is bounded (2 s); on expiry the CTA records
// the timeout in the error word, drains its loads and MMAs, frees TMEM and exits.
#include <algorithm>

#include "common.cuh"
#include "internal.h"
#include "tcgen05.cuh"
#include "tcgen05_pair.cuh"

namespace rx {
namespace {

constexpr int kTile = kHeadTile;      // rows and columns of a pair's tile
constexpr int BK = 64;                // of the reduction in a stage: 128 bytes
constexpr int kHalf = kTile / 2;      // rows of A and of B in a CTA
constexpr int kOperand = kHalf * 128;  // 16 KB
constexpr int kStages = 6;
constexpr int kStageBytes = 2 * kOperand;
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kStaging = 32 * 128;  // of an epilogue warp
constexpr int kOwn = 4;  // rows of a token whose term its weights' gradient has in fp32
constexpr int kJobs = 4;            // tiles that are known ahead
// Stages whose products the tensor cores add by themselves in a tile of logits.  They cut
// sums instead of rounding them, always downwards in magnitude: over the 2048 of a row
// that put 2.4e-5 on logits of 20, over 8192 1.4e-3 on logits of 40.  Sums of 512 are added
// in registers instead, to the nearest (error of a loss 2.2e-7 of it, of 256 1.1e-7; 8192 x
// 16384 x 2048: 329 us, of 256 360).  The same in both directions: the gradient takes z
// against the lse that the loss made of it, and of a sure row nothing must be left.
constexpr int kLogitChunk = 8;
constexpr int kSmemBytes = kStages * kStageBytes + kEpiWarps * kStaging + 512 + 1024;
static_assert(kSmemBytes <= 227 * 1024, "shared memory of one CTA");
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr uint64_t kDrainNs = 1000000000ull;
constexpr float kLargest = 3.402823466e+38f;  // of fp32
constexpr float kLog2e = 1.44269504088896341f;

// kind::f16, bf16 operands, fp32 accumulator, M = N = 256; bits 15 and 16: A, B MN-major.
constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) |
                            (static_cast<uint32_t>(kTile >> 3) << 17) |
                            (static_cast<uint32_t>(kTile >> 4) << 24);

// Shared-memory descriptor of an MN-major operand: boxes of 64 (M or N) x 64 (K), 128
// bytes a K row, with the 128-byte swizzle; 8 K rows are 1024 bytes, boxes 8 KB apart.
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr) {
  uint64_t desc = static_cast<uint64_t>((saddr >> 4) & 0x3FFFu);
  desc |= static_cast<uint64_t>(8192 >> 4) << 16;
  desc |= static_cast<uint64_t>(1024 >> 4) << 32;
  desc |= static_cast<uint64_t>(1) << 46;
  desc |= static_cast<uint64_t>(2) << 61;
  return desc;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// (a - m) log2 e and (b - m) log2 e, two at a time.
__device__ __forceinline__ float2 exponents(float a, float b, float m) {
  float2 e;
  asm("{\n\t.reg .b64 v, n, c;\n\t"
      "mov.b64 v, {%2, %3};\n\t"
      "mov.b64 n, {%4, %4};\n\t"
      "mov.b64 c, {%5, %5};\n\t"
      "add.rn.f32x2 v, v, n;\n\t"
      "mul.rn.f32x2 v, v, c;\n\t"
      "mov.b64 {%0, %1}, v;\n\t}"
      : "=f"(e.x), "=f"(e.y)
      : "f"(a), "f"(b), "f"(-m), "f"(kLog2e));
  return e;
}

// What rounding takes from a term of G (0 where that would not be a number).
__device__ __forceinline__ float lost_in_bf16(float x) {
  const float g = __bfloat162float(__float2bfloat16_rn(x));
  return fabsf(g) < INFINITY ? x - g : 0.f;
}

// A staged box added to global memory in fp32.
__device__ __forceinline__ void tma_add_2d(const CUtensorMap* map, uint32_t src, int c0, int c1) {
  asm volatile(
      "cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];"
      ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(src)
      : "memory");
}

// ---- rows that count ----------------------------------------------------------
constexpr int kRowsThreads = 256;
constexpr int kRowsAhead = 2;  // vectors of a thread that are on their way early

// Eight products of bf16, added in their order.
__device__ __forceinline__ float dot8(const uint4& a, const uint4& b) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s = __fmaf_rn(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), s);
    s = __fmaf_rn(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), s);
  }
  return s;
}
// The vector of a row from column c on, zeros behind its end.
__device__ __forceinline__ uint4 vector_at(const __nv_bfloat16* row, int c, int k, bool vec) {
  if (vec && c + 8 <= k) return *reinterpret_cast<const uint4*>(row + c);
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto* at = reinterpret_cast<const uint16_t*>(row) + c + 2 * i;
    const uint32_t lo = c + 2 * i < k ? at[0] : 0u, hi = c + 2 * i + 1 < k ? at[1] : 0u;
    v[i] = lo | hi << 16;
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// Each CTA counts the rows in front of its own by itself (the targets of a batch are
// few bytes), so that packing them takes one launch.  A row's logit of its target, which
// its loss and its largest term of G come from, is added up here, in fp32 and to the
// nearest: by eights of columns, a lane's one after another, then the lanes'.
__global__ void __launch_bounds__(kRowsThreads)
    head_rows_kernel(const HeadRows p, bool vec) {
  __shared__ int s_count[3][kRowsThreads / 32];
  __shared__ int s_at[kRowsThreads];
  __shared__ float s_dot[kRowsAhead * kRowsThreads];
  grid_dep_wait();
  grid_dep_launch();
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int64_t per = (p.rows + gridDim.x - 1) / gridDim.x;
  const int64_t lo = min(p.rows, blockIdx.x * per), hi = min(p.rows, lo + per);
  int before = 0, total = 0, wrong = 0;
  // a CTA's only row is on its way while it counts those in front
  const bool ahead = per == 1 && vec && p.k <= kRowsAhead * kRowsThreads * 8;
  uint4 row[kRowsAhead], row_w[kRowsAhead];
  const int target_lo = ahead && lo < hi ? p.targets[lo] : -1;
  if (target_lo >= 0 && target_lo < p.vocab)
#pragma unroll
    for (int i = 0; i < kRowsAhead; ++i) {
      const int c = (i * kRowsThreads + tid) * 8;
      if (c >= p.k) continue;
      row[i] = *reinterpret_cast<const uint4*>(p.hidden + lo * p.ld_hidden + c);
      row_w[i] = *reinterpret_cast<const uint4*>(p.w + target_lo * p.ldw + c);
    }
#pragma unroll 4
  for (int64_t r = tid; r < p.rows; r += kRowsThreads) {
    const int t = p.targets[r];
    const bool live = t >= 0 && t < p.vocab;
    total += live;
    before += live && r < lo;
    wrong |= t >= p.vocab;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    before += __shfl_xor_sync(0xffffffffu, before, o);
    total += __shfl_xor_sync(0xffffffffu, total, o);
    wrong |= __shfl_xor_sync(0xffffffffu, wrong, o);
  }
  if (lane == 0) {
    s_count[0][w] = before;
    s_count[1][w] = total;
    s_count[2][w] = wrong;
  }
  __syncthreads();
  before = total = wrong = 0;
  for (int i = 0; i < kRowsThreads / 32; ++i) {
    before += s_count[0][i];
    total += s_count[1][i];
    wrong |= s_count[2][i];
  }
  if (blockIdx.x == 0) {
    if (tid == 0) {
      *p.live = total;
      if (p.err != nullptr) *p.err = wrong ? kErrIndex : 0u;
    }
    for (int i = tid; i < p.n_queue; i += kRowsThreads) p.queue[i] = 0u;
  }
  // a warp: a row, and its share of the target's logit; zeros from nullptr
  auto copy_row = [&](int64_t at, const __nv_bfloat16* from, const __nv_bfloat16* w) {
    __nv_bfloat16* to = p.packed + at * p.ld_packed;
    float dot = 0.f;
#pragma unroll 2
    for (int c = lane * 8; c < p.k; c += 256) {
      uint4 h = make_uint4(0u, 0u, 0u, 0u);
      if (from != nullptr) {
        h = vector_at(from, c, p.k, vec);
        dot = __fadd_rn(dot, dot8(h, vector_at(w, c, p.k, true)));
      }
      *reinterpret_cast<uint4*>(to + c) = h;  // (rows hold whole vectors)
    }
    return dot;
  };
  auto target_done = [&](int64_t at, int64_t r, float dot) {  // a warp
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
    if (lane != 0) return;
    if (p.z_target != nullptr) p.z_target[at] = dot;
    if (p.target_term != nullptr) p.target_term[at] = p.grad[r] * expm1f(dot - p.lse[r]);
  };
  for (int64_t r0 = lo; r0 < hi; r0 += kRowsThreads) {
    const int64_t r = r0 + tid;
    const int t = r < hi ? p.targets[r] : -1;
    const bool live = t >= 0 && t < p.vocab;
    const uint32_t mask = __ballot_sync(0xffffffffu, live);
    __syncthreads();  // (earlier readers of both arrays)
    if (lane == 0) s_count[0][w] = __popc(mask);
    __syncthreads();
    int at = before + __popc(mask & ((1u << lane) - 1u));
    int in_chunk = 0;
    for (int i = 0; i < kRowsThreads / 32; ++i) {
      if (i < w) at += s_count[0][i];
      in_chunk += s_count[0][i];
    }
    before += in_chunk;
    s_at[tid] = live ? at : -1;
    if (r < hi) {
      if (p.place != nullptr) p.place[r] = live ? at : -1;
      if (live) {
        p.row[at] = static_cast<int>(r);
        p.target[at] = t;
        if (p.grad != nullptr) p.row_grad[at] = p.grad[r];
        if (p.lse != nullptr) p.row_lse[at] = p.lse[r];
      } else if (p.loss_out != nullptr) {
        p.loss_out[r] = 0.f;
        p.lse_out[r] = 0.f;
      }
    }
    __syncthreads();
    if (ahead) {
      const int64_t to = s_at[0];
      if (to < 0) break;
#pragma unroll
      for (int i = 0; i < kRowsAhead; ++i) {
        const int c = (i * kRowsThreads + tid) * 8;
        if (c < p.k) *reinterpret_cast<uint4*>(p.packed + to * p.ld_packed + c) = row[i];
        s_dot[i * kRowsThreads + tid] = c < p.k ? dot8(row[i], row_w[i]) : 0.f;
      }
      __syncthreads();
      if (w == 0) {
        float dot = 0.f;
        for (int c = lane; c * 8 < p.k; c += 32) dot = __fadd_rn(dot, s_dot[c]);
        target_done(to, r0, dot);
      }
      break;
    }
    const int n = static_cast<int>(min(static_cast<int64_t>(kRowsThreads), hi - r0));
    for (int i = w; i < n; i += kRowsThreads / 32)
      if (s_at[i] >= 0)
        target_done(s_at[i], r0 + i,
                    copy_row(s_at[i], p.hidden + (r0 + i) * p.ld_hidden,
                             p.w + p.targets[r0 + i] * p.ldw));
  }
  // rows of zeros up to whole tiles
  const int64_t most = static_cast<int64_t>(total + p.tile - 1) / p.tile * p.tile;
  for (int64_t i = total + static_cast<int64_t>(blockIdx.x) * (kRowsThreads / 32) + w; i < most;
       i += static_cast<int64_t>(gridDim.x) * (kRowsThreads / 32)) {
    copy_row(i, nullptr, nullptr);
    if (lane == 0) {
      if (p.z_target != nullptr) p.z_target[i] = 0.f;
      if (p.target_term != nullptr) p.target_term[i] = 0.f;
      p.target[i] = -1;
      if (p.grad != nullptr) p.row_grad[i] = 0.f;
      if (p.lse != nullptr) p.row_lse[i] = 0.f;
    }
  }
}

// ---- tiles --------------------------------------------------------------------
enum { kLoss = 0, kGrad = 1, kHidden = 2, kWeight = 3 };

struct Maps {
  CUtensorMap h_rows;   // packed rows, boxes of 64 columns x 128 rows
  CUtensorMap w_rows;   // W, the same
  CUtensorMap h_cols;   // packed rows, boxes of 64 x 64
  CUtensorMap w_cols;   // W, the same
  CUtensorMap g_rows;   // the piece of G that is read, 64 x 128
  CUtensorMap g_cols;   // the same, 64 x 64
  CUtensorMap g_out;    // the piece of G that is written, 64 columns x 32 rows
  CUtensorMap dw_out;   // gradient of W, 64 (fp32: 32) columns x 32 rows
  CUtensorMap dh_out;   // [splits x rows] fp32 sums, 32 x 32
};

struct __align__(16) Tile {
  int kind;      // -1: the end
  int row0;      // rows of the tile: packed rows, weight: rows of the piece
  int col0;      // columns: vocabulary (grad: in the piece) or hidden columns
  int part;      // hidden: which part of the piece
  int kb0, kb1;  // stages of the reduction
};

// How many tiles of each kind the launch has, for `live` rows.
struct Counts {
  int mt;         // tiles of rows
  int grad, hidden, weight;
  __device__ __forceinline__ int all() const { return grad + hidden + weight; }
};
__device__ __forceinline__ Counts count_tiles(const HeadTiles& p, int live, bool loss) {
  Counts c;
  c.mt = (live + kTile - 1) / kTile;
  c.grad = c.mt * p.vt_next;
  c.hidden = loss ? 0 : c.mt * p.kt * p.parts;
  c.weight = loss || p.dw == nullptr ? 0 : p.vt * p.kt;
  return c;
}

__device__ __forceinline__ Tile decode(const HeadTiles& p, const Counts& c, int live, bool loss,
                                       int j) {
  Tile t{};
  if (!loss) {
    // hidden tiles and weight tiles, the longer ones first; the parts and columns of a
    // panel of G next to one another
    const int first = p.hidden_first ? c.hidden : c.weight;
    const bool in_first = j < first;
    if (j < c.hidden + c.weight) {
      const int i = in_first ? j : j - first;
      t.kind = in_first == p.hidden_first ? kHidden : kWeight;
      t.col0 = i % p.kt * kTile;
      if (t.kind == kHidden) {
        t.part = i / p.kt % p.parts;
        t.row0 = i / p.kt / p.parts * kTile;
        t.kb0 = t.part * p.part_blocks;
        t.kb1 = min(t.kb0 + p.part_blocks, p.vt * (kTile / BK));
      } else {
        t.row0 = i / p.kt * kTile;
        t.kb1 = (live + BK - 1) / BK;
      }
      return t;
    }
    j -= c.hidden + c.weight;
  }
  t.kind = loss ? kLoss : kGrad;
  // groups of kHeadGroup tiles of rows stay in L2 while W passes by
  const int per = kHeadGroup * p.vt_next;
  const int m0 = j / per * kHeadGroup, r = j % per;
  const int gm = min(kHeadGroup, c.mt - m0);
  t.row0 = (m0 + r % gm) * kTile;
  t.col0 = r / gm * kTile;
  t.kb1 = (p.k + BK - 1) / BK;
  return t;
}

// Running maximum and sum of 2^((z - m) log2 e).
struct Stats {
  float m, s;
};
__device__ __forceinline__ float safe_max(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ void add_chunk(Stats& st, const float (&z)[32]) {
  float top[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) top[i] = fmaxf(fmaxf(z[i], z[i + 8]), fmaxf(z[i + 16], z[i + 24]));
#pragma unroll
  for (int i = 0; i < 4; ++i) top[i] = fmaxf(top[i], top[i + 4]);
  const float m = fmaxf(st.m, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
  const float ref = safe_max(m);
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    const float2 e = exponents(z[i], z[i + 1], ref);
    sum[i & 3] += exp2_fast(e.x);
    sum[(i + 1) & 3] += exp2_fast(e.y);
  }
  const float chunk = (sum[0] + sum[1]) + (sum[2] + sum[3]);
  st.s = __fmaf_rn(st.s, exp2_fast((st.m - ref) * kLog2e), chunk);
  st.m = m;
}

template <bool LOSS>
__global__ void __launch_bounds__(kThreads, 1)
    head_tiles_kernel(const __grid_constant__ Maps maps, const HeadTiles p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sa = smem;
  uint8_t* sb = smem + kStages * kOperand;
  uint8_t* staging = smem + kStages * kStageBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(staging + kEpiWarps * kStaging);
  uint64_t* full = bars;                     // leader's is the one used
  uint64_t* empty = full + kStages;          // per CTA
  uint64_t* acc_full = empty + kStages;      // [2] per CTA
  uint64_t* acc_empty = acc_full + 2;        // [2] leader's is the one used
  uint64_t* job_full = acc_empty + 2;        // [kJobs] per CTA: the tile's number is there
  uint64_t* job_empty = job_full + kJobs;    // [kJobs] leader's: everyone has read it
  uint64_t* drain = job_empty + kJobs;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  // [kJobs] tiles, decoded by the leader's producer
  Tile* s_job = reinterpret_cast<Tile*>(reinterpret_cast<uint8_t*>(bars) + 256);
  static_assert((2 * kStages + 4 + 2 * kJobs + 1) * 8 + 8 <= 256 && sizeof(Tile) == 32 &&
                    kJobs * sizeof(Tile) <= 256, "barriers and tiles");

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const bool leader = rank == 0;
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 2);  // an expect_tx of each CTA
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&acc_full[b], 1);
      mbar_init(&acc_empty[b], 2 * kEpiWarps);
    }
    for (int j = 0; j < kJobs; ++j) {
      mbar_init(&job_full[j], 1);
      // the epilogue warps of both CTAs, the MMA issuer, the peer's producer
      mbar_init(&job_empty[j], 2 * kEpiWarps + 2);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_map(&maps.h_rows);
    prefetch_map(&maps.w_rows);
  }
  cluster_sync_all();  // barriers of both CTAs initialised; the peer is running
  if (warp == 1) tmem_alloc_pair(smem_addr(tmem_slot), 2 * kTile);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  grid_dep_wait();
  grid_dep_launch();
  const int live = min(max(*p.live, 0), p.rows);
  const Counts counts = count_tiles(p, live, LOSS);
  const int njobs = counts.all();

  // The n-th tile of this pair; false on a timeout.
  auto next_job = [&](uint32_t n, Tile& t) {
    const int slot = n % kJobs;
    if (!mbar_wait_cluster(&job_full[slot], (n / kJobs) & 1u, abort_flag, kWaitNs)) return false;
    const int4 a = reinterpret_cast<const int4*>(&s_job[slot])[0];
    const int2 b = reinterpret_cast<const int2*>(&s_job[slot])[2];
    t = Tile{a.x, a.y, a.z, a.w, b.x, b.y};
    return true;
  };
  // The calling thread has read it (not the end, behind which no slot is written).  Relaxed:
  // a release would wait until the thread's stores of the last tile's results have reached
  // L2, and its fence alone takes the MMAs 3 %.  The slot is written again only behind this
  // arrival, which depends on words of both of next_job's loads (kb0 <= kb1 in every
  // tile), so that neither load can be under way still.
  auto job_read = [&](uint32_t n, const Tile& t) {
    if (t.kind >= 0 && t.kb0 <= t.kb1)
      mbar_arrive_cluster_relaxed(map_to_rank(smem_addr(&job_empty[n % kJobs]), 0));
  };
  auto give_up = [&](bool timeout) {
    if (timeout && !*abort_flag) set_err(p.err, kErrTimeout);
    *abort_flag = 1;
  };

  if (warp == 0 && lane == 0) {
    // ---------------- tiles and TMA loads ----------------
    int stage = 0;
    uint32_t phase = 0, issued_mask = 0, issued_phase = 0;
    bool ok = true;
    int next = pair < njobs ? pair : -1;  // leader
    for (uint32_t n = 0; ok; ++n) {
      Tile t{-1};
      if (leader) {
        if (next >= 0) t = decode(p, counts, live, LOSS, next);
        const int slot = n % kJobs;
        if (!mbar_wait_cluster(&job_empty[slot], ((n / kJobs) & 1u) ^ 1u, abort_flag, kWaitNs)) {
          ok = false;
          break;
        }
        for (uint32_t c = 0; c < 2; ++c) {
          const uint32_t there = map_to_rank(smem_addr(&s_job[slot]), c);
          asm volatile("st.shared::cluster.v4.s32 [%0], {%1, %2, %3, %4};" ::"r"(there),
                       "r"(t.kind), "r"(t.row0), "r"(t.col0), "r"(t.part)
                       : "memory");
          asm volatile("st.shared::cluster.v2.s32 [%0], {%1, %2};" ::"r"(there + 16), "r"(t.kb0),
                       "r"(t.kb1)
                       : "memory");
          mbar_arrive_cluster(map_to_rank(smem_addr(&job_full[slot]), c));
        }
      } else {
        if (!next_job(n, t)) {
          ok = false;
          break;
        }
        job_read(n, t);
      }
      if (t.kind < 0) break;
      const int ra = t.row0 + static_cast<int>(rank) * kHalf;
      const int rb = t.col0 + static_cast<int>(rank) * kHalf;
      // The next tile's number takes a microsecond (the MMAs of two stages and a half):
      // asked for eight stages before the end of a longer tile (8192 x 16384 x 2048: 350 ->
      // 344 us), not earlier, so that a long tile does not hold back one that is waiting.
      const int ask = t.kb1 - t.kb0 > 8 ? t.kb1 - 8 : max(t.kb0, t.kb1 - 1);
      auto fetch = [&] {
        if (!leader) return;
        const uint32_t q = atomicAdd(p.queue, 1u) + static_cast<uint32_t>(npairs);
        next = q < static_cast<uint32_t>(njobs) ? static_cast<int>(q) : -1;
      };
      if (t.kb0 >= t.kb1) fetch();
      for (int kb = t.kb0; kb < t.kb1; ++kb) {
        if (!mbar_wait(&empty[stage], phase ^ 1u, abort_flag, kWaitNs)) {
          ok = false;
          break;
        }
        const uint32_t fb = map_to_rank(smem_addr(&full[stage]), 0);
        if (leader) mbar_expect_tx(smem_addr(&full[stage]), kStageBytes);
        else mbar_expect_tx_cluster(fb, kStageBytes);
        const uint32_t a = smem_addr(sa + stage * kOperand), b = smem_addr(sb + stage * kOperand);
        const int k0 = kb * BK;
        if (LOSS || t.kind == kGrad) {
          tma_load_2d_pair(a, &maps.h_rows, k0, ra, fb);
          tma_load_2d_pair(b, &maps.w_rows, k0, p.v_next + rb, fb);
        } else if (t.kind == kHidden) {
          tma_load_2d_pair(a, &maps.g_rows, k0, ra, fb);
          tma_load_2d_pair(b, &maps.w_cols, rb, p.v0 + k0, fb);
          tma_load_2d_pair(b + kOperand / 2, &maps.w_cols, rb + 64, p.v0 + k0, fb);
        } else {
          tma_load_2d_pair(a, &maps.g_cols, ra, k0, fb);
          tma_load_2d_pair(a + kOperand / 2, &maps.g_cols, ra + 64, k0, fb);
          tma_load_2d_pair(b, &maps.h_cols, rb, k0, fb);
          tma_load_2d_pair(b + kOperand / 2, &maps.h_cols, rb + 64, k0, fb);
        }
        issued_mask |= 1u << stage;
        issued_phase = (issued_phase & ~(1u << stage)) | (phase << stage);
        if (++stage == kStages) {
          stage = 0;
          phase ^= 1u;
        }
        if (kb == ask) fetch();
      }
    }
    if (!ok) give_up(true);
    if (*abort_flag && leader) {
      // every issued load must land before the CTA may exit
      for (int s = 0; s < kStages; ++s)
        if (issued_mask & (1u << s))
          mbar_wait(&full[s], (issued_phase >> s) & 1u, nullptr, kDrainNs);
    }
  } else if (warp == 1 && lane == 0 && leader) {
    // ---------------- MMAs ----------------
    int stage = 0;
    uint32_t phase = 0;
    uint32_t acc_n = 0;
    bool ok = true, issued_any = false;
    for (uint32_t n = 0; ok; ++n) {
      Tile t;
      if (!next_job(n, t)) {
        ok = false;
        break;
      }
      if (t.kind < 0) break;
      job_read(n, t);
      const bool a_mn = !LOSS && t.kind == kWeight, b_mn = !LOSS && t.kind >= kHidden;
      const uint32_t idesc = kIdesc | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
      // 16 along the reduction: 32 bytes of a row, or 16 rows of 128 bytes
      const uint32_t a_step = a_mn ? 2048 >> 4 : 32 >> 4, b_step = b_mn ? 2048 >> 4 : 32 >> 4;
      int kb = t.kb0;
      do {  // (once for a tile without a reduction)
        const int ab = acc_n & 1, first = kb;
        const int last = LOSS || t.kind == kGrad ? min(t.kb1, kb + kLogitChunk) : t.kb1;
        if (!mbar_wait(&acc_empty[ab], ((acc_n >> 1) & 1u) ^ 1u, abort_flag, kWaitNs)) {
          ok = false;
          break;
        }
        ++acc_n;
        tc_fence_after();
        const uint32_t d = tmem_base + static_cast<uint32_t>(ab * kTile);
        for (; kb < last; ++kb) {
          if (!mbar_wait(&full[stage], phase, abort_flag, kWaitNs)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t a = smem_addr(sa + stage * kOperand), b = smem_addr(sb + stage * kOperand);
          const uint64_t da = a_mn ? desc_mn(a) : desc_sw128(a);
          const uint64_t db = b_mn ? desc_mn(b) : desc_sw128(b);
#pragma unroll
          for (int u = 0; u < BK / 16; ++u)
            mma_bf16_pair(d, da + u * a_step, db + u * b_step, idesc,
                          (kb > first || u > 0) ? 1u : 0u);
          issued_any = true;
          mma_commit_pair(smem_addr(&empty[stage]));
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (!ok) break;
        mma_commit_pair(smem_addr(&acc_full[ab]));
      } while (kb < t.kb1);
    }
    if (!ok) give_up(true);
    if (*abort_flag && issued_any) {
      mma_commit_pair(smem_addr(drain));
      mbar_wait(drain, 0, nullptr, kDrainNs);
    }
  } else if (warp >= 2) {
    // ---------------- epilogue ----------------
    const int quarter = warp & 3;
    const int half = (warp - 2) >> 2;  // columns 128 half .. of the tile
    uint8_t* stg = staging + (warp - 2) * kStaging;
    const uint32_t stg_s = smem_addr(stg);
    // 16-byte chunk c of this thread's row in the staged box
    auto chunk_at = [&](int c) { return stg_s + lane * 128 + ((c ^ (lane & 7)) << 4); };
    auto put = [&](int c, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(chunk_at(c)), "r"(x), "r"(y),
                   "r"(z), "r"(w)
                   : "memory");
    };
    // the store that last used the box has read it
    auto box_free = [&] {
      if (lane == 0) bulk_wait_read<0>();
      __syncwarp();
    };
    auto box_filled = [&] {
      fence_proxy_async_smem();
      __syncwarp();
    };
    uint32_t acc_n = 0;
    for (uint32_t n = 0;; ++n) {
      Tile t{-1};
      int ok = 1;
      if (lane == 0) ok = next_job(n, t) ? 1 : 0;
      ok = __shfl_sync(0xffffffffu, ok, 0);
      t.kind = __shfl_sync(0xffffffffu, t.kind, 0);
      t.row0 = __shfl_sync(0xffffffffu, t.row0, 0);
      t.col0 = __shfl_sync(0xffffffffu, t.col0, 0);
      t.part = __shfl_sync(0xffffffffu, t.part, 0);
      t.kb0 = __shfl_sync(0xffffffffu, t.kb0, 0);
      t.kb1 = __shfl_sync(0xffffffffu, t.kb1, 0);
      if (!ok) {
        if (lane == 0) give_up(true);
        break;
      }
      if (t.kind < 0) break;
      if (lane == 0) job_read(n, t);
      const int row = t.row0 + static_cast<int>(rank) * kHalf + quarter * 32 + lane;
      const int warp_row = row - lane;
      const int col0 = t.col0 + half * 128;
      int target = -1;
      bool counted = false;  // else its weight is 0, even against weights that are infinite
      float c_row = 0.f, lse = 0.f, of_target = 0.f;  // its logit, or its term of G
      if (LOSS || t.kind == kGrad) {
        target = p.target[row];  // (rows up to whole tiles have one)
        of_target = LOSS ? p.z_target[row] : p.target_term[row];
        if (!LOSS) {
          counted = target >= 0;
          target -= p.v_next;
          c_row = p.row_grad[row];
          lse = p.row_lse[row];
        }
      }
      // weight: rows whose target is this thread's, in their order, while the products run
      int own[kOwn], n_own = 0;
      if (!LOSS && t.kind == kWeight) {
        constexpr int kAhead = 8;
        const int v = p.v0 + row, v_warp = v - lane;
        uint32_t open = 0xffffffffu;  // lanes that have fewer than kOwn
        for (int r0 = 0; r0 < live && open != 0u; r0 += 32 * kAhead) {
          int at[kAhead];
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            const int r = r0 + 32 * u + lane;
            at[u] = r < live ? p.target[r] : -1;
          }
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            if (r0 + 32 * u >= live) break;
            const uint32_t to = static_cast<uint32_t>(at[u] - v_warp);
            uint32_t in = __ballot_sync(0xffffffffu, to < 32u && (open >> (to & 31u) & 1u));
            for (; in != 0u; in &= in - 1u) {
              const int j = __ffs(in) - 1;
              if (__shfl_sync(0xffffffffu, at[u], j) != v || n_own == kOwn) continue;
#pragma unroll
              for (int q = 0; q < kOwn; ++q)
                if (q == n_own) own[q] = r0 + 32 * u + j;
              ++n_own;
            }
          }
          open = __ballot_sync(0xffffffffu, n_own < kOwn);
        }
      }
      uint32_t tm = 0, release = 0;
      auto acc_ready = [&] {  // the next accumulator is complete
        const int ab = acc_n & 1;
        if (lane == 0)
          ok = mbar_wait(&acc_full[ab], (acc_n >> 1) & 1u, abort_flag, kWaitNs) ? 1 : 0;
        ok = __shfl_sync(0xffffffffu, ok, 0);
        ++acc_n;
        tc_fence_after();
        tm = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) +
             static_cast<uint32_t>(ab * kTile + half * 128);
        release = map_to_rank(smem_addr(&acc_empty[ab]), 0);
        return ok != 0;
      };
      if (!acc_ready()) {
        if (lane == 0) give_up(true);
        break;
      }
      auto hand_back = [&] {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_relaxed(release);
      };
      float z[32];
      auto load = [&](int c) {  // 32 columns from 32 c
        uint32_t r[32];
        tmem_ld32(tm + 32 * c, r);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 32; ++i) z[i] = __uint_as_float(r[i]);
        if (c == 3) hand_back();
      };
      // logits: a row of 128 columns, in parts of kLogitChunk stages
      if (LOSS || t.kind == kGrad) {
        float sum[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          load(c);
#pragma unroll
          for (int i = 0; i < 32; ++i) sum[c][i] = z[i];
        }
        for (int kb = t.kb0 + kLogitChunk; kb < t.kb1; kb += kLogitChunk) {
          if (!acc_ready()) break;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            load(c);
#pragma unroll
            for (int i = 0; i < 32; ++i) sum[c][i] += z[i];
          }
        }
        if (!ok) {
          if (lane == 0) give_up(true);
          break;
        }
        if (LOSS) {
          Stats st{-INFINITY, 0.f};
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int v = col0 + 32 * c;
            const uint32_t at = static_cast<uint32_t>(target - v);
            if (at < 32u)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                sum[c][i] = at == static_cast<uint32_t>(i) ? of_target : sum[c][i];
            if (v + 32 > p.vocab)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (v + i >= p.vocab) sum[c][i] = -INFINITY;
            if (v < p.vocab) add_chunk(st, sum[c]);
          }
          p.stats[static_cast<int64_t>(col0 / 128) * p.ld_stats + row] = make_float2(st.m, st.s);
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float (&g)[32] = sum[c];
            const int v = col0 + 32 * c;  // in the piece
            const uint32_t at = static_cast<uint32_t>(target - v);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const float2 e = exponents(g[i], g[i + 1], lse);
              g[i] = c_row * exp2_fast(e.x);
              g[i + 1] = c_row * exp2_fast(e.y);
            }
            const int left = counted ? p.vocab - (p.v_next + v) : 0;
            if (left < 32)  // zeros behind the last column
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (i >= left) g[i] = 0.f;
            if (at < 32u)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                g[i] = at == static_cast<uint32_t>(i) ? of_target : g[i];
            if ((c & 1) == 0) box_free();
#pragma unroll
            for (int q = 0; q < 4; ++q)
              put((c & 1) * 4 + q, pack_bf16(g[8 * q], g[8 * q + 1]),
                  pack_bf16(g[8 * q + 2], g[8 * q + 3]), pack_bf16(g[8 * q + 4], g[8 * q + 5]),
                  pack_bf16(g[8 * q + 6], g[8 * q + 7]));
            if (c & 1) {
              box_filled();
              if (lane == 0) {
                tma_store_2d(&maps.g_out, stg_s, v - 32, warp_row);
                bulk_commit();
              }
            }
          }
        }
      } else if (t.kind == kHidden) {
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          load(c);
          if (col0 + 32 * c >= p.ld_sums || warp_row >= live) continue;
          box_free();
#pragma unroll
          for (int q = 0; q < 8; ++q)
            put(q, __float_as_uint(z[4 * q]), __float_as_uint(z[4 * q + 1]),
                __float_as_uint(z[4 * q + 2]), __float_as_uint(z[4 * q + 3]));
          box_filled();
          if (lane == 0) {
            const int at = t.part * p.rows_up + warp_row;
            if (p.v0 == 0) tma_store_2d(&maps.dh_out, stg_s, col0 + 32 * c, at);
            else tma_add_2d(&maps.dh_out, stg_s, col0 + 32 * c, at);
            bulk_commit();
          }
        }
      } else {
        // boxes of 128 bytes: 64 bf16 or 32 fp32 columns
        const int64_t out_row = static_cast<int64_t>(p.v0) + warp_row;
        const int rows = min(32, p.vocab - p.v0 - warp_row);
        auto flush = [&](int col, int cols) {
          const int n_cols = min(cols, p.k - col);
          if (rows <= 0 || n_cols <= 0) return;
          const int es = p.dw_f32 ? 4 : 2;
          int done = 0;  // columns that the map covers
          if (p.dw_mapped) {
            done = min(n_cols, max(0, p.k / (16 / es) * (16 / es) - col));
            if (lane == 0) {
              if (done > 0) tma_store_2d(&maps.dw_out, stg_s, col, static_cast<int>(out_row));
              bulk_commit();
            }
          }
          if (done == n_cols) return;
          for (int i = lane; i < rows * (n_cols - done); i += 32) {
            const int r = i / (n_cols - done), x = done + i % (n_cols - done);
            const uint8_t* from = stg + r * 128 + (((x * es >> 4) ^ (r & 7)) << 4) + (x * es & 15);
            const int64_t to = (out_row + r) * p.ld_dw + col + x;
            if (p.dw_f32)
              static_cast<float*>(p.dw)[to] = *reinterpret_cast<const float*>(from);
            else
              static_cast<uint16_t*>(p.dw)[to] = *reinterpret_cast<const uint16_t*>(from);
          }
          __syncwarp();
        };
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          load(c);
          if (t.kb1 == 0)  // no rows: nothing was added up
#pragma unroll
            for (int i = 0; i < 32; ++i) z[i] = 0.f;
          const int col = col0 + 32 * c;
#pragma unroll
          for (int q = 0; q < kOwn; ++q)
            if (q < n_own) {
              const float rest = lost_in_bf16(p.target_term[own[q]]);
              const __nv_bfloat16* from = p.packed + own[q] * p.ld_packed + col;
#pragma unroll
              for (int x = 0; x < 4; ++x)
                if (col + 8 * x < p.k) {
                  const uint4 h = *reinterpret_cast<const uint4*>(from + 8 * x);
                  const uint32_t w[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    float& lo = z[8 * x + 2 * i];
                    float& hi = z[8 * x + 2 * i + 1];
                    lo = __fmaf_rn(rest, __uint_as_float(w[i] << 16), lo);
                    hi = __fmaf_rn(rest, __uint_as_float(w[i] & 0xffff0000u), hi);
                  }
                }
            }
          if (p.dw_f32) {
            box_free();
#pragma unroll
            for (int q = 0; q < 8; ++q)
              put(q, __float_as_uint(z[4 * q]), __float_as_uint(z[4 * q + 1]),
                  __float_as_uint(z[4 * q + 2]), __float_as_uint(z[4 * q + 3]));
            box_filled();
            flush(col, 32);
            continue;
          }
          if ((c & 1) == 0) box_free();
#pragma unroll
          for (int q = 0; q < 4; ++q)
            put((c & 1) * 4 + q, pack_bf16(z[8 * q], z[8 * q + 1]),
                pack_bf16(z[8 * q + 2], z[8 * q + 3]), pack_bf16(z[8 * q + 4], z[8 * q + 5]),
                pack_bf16(z[8 * q + 6], z[8 * q + 7]));
          if (c & 1) {
            box_filled();
            flush(col - 32, 64);
          }
        }
      }
    }
    if (lane == 0) bulk_wait_all();  // every store written before exit
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // the pair's MMAs and TMEM reads are done in both CTAs
  tc_fence_after();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc_pair(tmem_base, 2 * kTile);
  }
}

// ---- few rows -------------------------------------------------------------------
// Up to NT (32 or 64) rows: W is what costs, so its rows are the tiles, up to 128 at a
// time by single CTAs (M = 128, N = NT; as many as give every CTA the same number of
// tiles), and stream through a ring of nine or ten stages at HBM's rate.  A thread has one
// row of W and NT logits.  Loss: it keeps a maximum and a sum for each of its columns over
// all of its tiles; the threads' are joined when the
// tiles are done, the CTAs' by the last of them, both in an order that depends neither on
// NT nor on the column: four groups of them, each from front to back, then the first two,
// the last two and both.  Gradient: G of the whole vocabulary, 64 bytes of a row by a
// warp.
// 32 x 65536 x 2048 with the packing of the rows: 57 us, W's bytes take 40; by pairs on 256
// rows 69 (as long as 256 of them take).
// Sums of 256 in the tensor cores, where larger calls have 512: with a row or two nothing
// averages out what they cut (losses off by up to 2.8e-6 of themselves at K = 4096, and by
// half of that here), and W's bytes hide most of it with eight accumulators to go round
// (32 x 65536 x 2048: 55.2 -> 56.7 us; of 128 61.7).
constexpr int kFewChunk = 4;
constexpr int kFewThreads = 192;  // TMA, MMA and four epilogue warps
template <int NT>
struct Few {
  static constexpr int kWBytes = kHalf * 128;
  static constexpr int kStageBytes = kWBytes + NT * 128;
  static constexpr int kStages = NT == 32 ? 10 : 9;
  static constexpr int kMisc = 512 + 4 * NT * 4;
  static constexpr int kSmem = kStages * kStageBytes + kMisc + 1024;
  static constexpr int kAcc = 8;  // accumulators
  static constexpr int kTmem = kAcc * NT;
  static_assert(kTmem <= 512, "columns of TMEM");
  static_assert(kSmem <= 227 * 1024, "shared memory of one CTA");
  static_assert(kHalf * NT * 8 <= kStages * kStageBytes, "the threads' sums go into the ring");
};

template <int NT, bool GRAD>
__global__ void __launch_bounds__(kFewThreads, 1)
    head_few_kernel(const __grid_constant__ CUtensorMap map_w,
                    const __grid_constant__ CUtensorMap map_h, const HeadTiles p, int tile_rows,
                    __nv_bfloat16* g_out, int64_t ld_g, float* loss, float* lse) {
  using F = Few<NT>;
  constexpr int kRing = F::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kRing * F::kStageBytes);
  uint64_t* full = bars;
  uint64_t* empty = full + kRing;
  uint64_t* acc_full = empty + kRing;
  uint64_t* acc_empty = acc_full + F::kAcc;
  uint64_t* drain = acc_empty + F::kAcc;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* s_last = reinterpret_cast<int*>(tmem_slot + 2);
  static_assert((2 * kRing + 2 * F::kAcc + 1) * 8 + 12 <= 512, "barriers");
  int* s_target = reinterpret_cast<int*>(reinterpret_cast<uint8_t*>(bars) + 512);
  float* s_of_target = reinterpret_cast<float*>(s_target + NT);
  float* s_lse = s_of_target + NT;
  float* s_grad = s_lse + NT;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int ntiles = (p.vocab + tile_rows - 1) / tile_rows;
  const uint32_t w_bytes = tile_rows * 128;
  const int nk = (p.k + BK - 1) / BK;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kRing; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < F::kAcc; ++b) {
      mbar_init(&acc_full[b], 1);
      mbar_init(&acc_empty[b], 4);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_map(&map_w);
    prefetch_map(&map_h);
  }
  __syncwarp();
  auto load_w = [&](int t, int kb, int s) {
    tma_load_2d(smem_addr(smem + s * F::kStageBytes), &map_w, kb * BK, t * tile_rows,
                smem_addr(&full[s]));
  };
  // The ring's first weights while the rows are still being packed: the kernel in front
  // (head_rows_kernel) waited for all before it when it let this one start, and writes
  // none of W.
  int early = 0;
  if (warp == 0 && lane == 0) {
    early = min(nk, kRing);  // (of the first tile)
    for (int s = 0; s < early; ++s) {
      mbar_expect_tx_only(smem_addr(&full[s]), w_bytes);
      load_w(blockIdx.x, s, s);
    }
  }
  if (warp == 1) tmem_alloc(smem_addr(tmem_slot), F::kTmem);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  grid_dep_wait();
  grid_dep_launch();
  for (int i = threadIdx.x; i < NT; i += kFewThreads) {
    s_target[i] = p.target[i];  // (rows up to whole tiles have one)
    s_of_target[i] = GRAD ? p.target_term[i] : p.z_target[i];
    if (GRAD) {
      s_lse[i] = p.row_lse[i];
      s_grad[i] = p.row_grad[i];
    }
  }
  __syncthreads();
  auto give_up = [&] {
    if (!*abort_flag) set_err(p.err, kErrTimeout);
    *abort_flag = 1;
  };

  if (warp == 0 && lane == 0) {
    // ---------------- TMA loads ----------------
    int stage = 0;
    uint32_t phase = 0, issued_mask = 0, issued_phase = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < ntiles && ok; t += gridDim.x) {
      for (int kb = 0; kb < nk; ++kb) {
        if (!mbar_wait(&empty[stage], phase ^ 1u, abort_flag, kWaitNs)) {
          ok = false;
          break;
        }
        const bool ahead = early > 0;
        mbar_expect_tx(smem_addr(&full[stage]), NT * 128 + (ahead ? 0u : w_bytes));
        if (ahead) --early;
        else load_w(t, kb, stage);
        tma_load_2d(smem_addr(smem + stage * F::kStageBytes + F::kWBytes), &map_h, kb * BK, 0,
                    smem_addr(&full[stage]));
        issued_mask |= 1u << stage;
        issued_phase = (issued_phase & ~(1u << stage)) | (phase << stage);
        if (++stage == kRing) {
          stage = 0;
          phase ^= 1u;
        }
      }
    }
    if (!ok) give_up();
    if (*abort_flag) {
      for (int i = 0; i < early; ++i) {  // the arrivals that are missing
        mbar_arrive1(smem_addr(&full[stage + i]));
        mbar_wait(&full[stage + i], 0, nullptr, kDrainNs);
      }
      for (int s = 0; s < kRing; ++s)
        if (issued_mask & (1u << s))
          mbar_wait(&full[s], (issued_phase >> s) & 1u, nullptr, kDrainNs);
    }
  } else if (warp == 1 && lane == 0) {
    // ---------------- MMAs ----------------
    constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) |
                               (static_cast<uint32_t>(NT >> 3) << 17) |
                               (static_cast<uint32_t>(kHalf >> 4) << 24);
    int stage = 0;
    uint32_t phase = 0, acc_n = 0;
    bool ok = true, issued_any = false;
    for (int t = blockIdx.x; t < ntiles && ok; t += gridDim.x) {
      for (int kb = 0; kb < nk && ok;) {
        const int ab = acc_n % F::kAcc, first = kb;
        const int last = min(nk, kb + kFewChunk);
        if (!mbar_wait(&acc_empty[ab], ((acc_n / F::kAcc) & 1u) ^ 1u, abort_flag, kWaitNs)) {
          ok = false;
          break;
        }
        ++acc_n;
        tc_fence_after();
        const uint32_t d = tmem_base + static_cast<uint32_t>(ab * NT);
        for (; kb < last; ++kb) {
          if (!mbar_wait(&full[stage], phase, abort_flag, kWaitNs)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t a = smem_addr(smem + stage * F::kStageBytes);
          const uint64_t da = desc_sw128(a), db = desc_sw128(a + F::kWBytes);
#pragma unroll
          for (int u = 0; u < BK / 16; ++u) {
            asm volatile(
                "{\n\t.reg .pred p;\n\t"
                "setp.ne.b32 p, %4, 0;\n\t"
                "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d),
                "l"(da + 2 * u), "l"(db + 2 * u), "r"(idesc),
                "r"(kb > first || u > 0 ? 1u : 0u)
                : "memory");
          }
          issued_any = true;
          mma_commit(smem_addr(&empty[stage]));
          if (++stage == kRing) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (ok) mma_commit(smem_addr(&acc_full[ab]));
      }
    }
    if (!ok) give_up();
    if (*abort_flag && issued_any) {
      mma_commit(smem_addr(drain));
      mbar_wait(drain, 0, nullptr, kDrainNs);
    }
  } else if (warp >= 2) {
    // ---------------- epilogue: a row of W each ----------------
    const int quarter = warp & 3, row = quarter * 32 + lane;
    float m[GRAD ? 1 : NT], sum[GRAD ? 1 : NT];
    if (!GRAD)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        m[j] = -kLargest;
        sum[j] = 0.f;
      }
    uint32_t acc_n = 0;
    int ok = 1;
    for (int t = blockIdx.x; t < ntiles && ok; t += gridDim.x) {
      float z[NT];
      for (int kb = 0; kb < nk; kb += kFewChunk) {
        const int ab = acc_n % F::kAcc;
        if (lane == 0)
          ok = mbar_wait(&acc_full[ab], (acc_n / F::kAcc) & 1u, abort_flag, kWaitNs) ? 1 : 0;
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
        ++acc_n;
        tc_fence_after();
        const uint32_t tm = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) +
                            static_cast<uint32_t>(ab * NT);
#pragma unroll
        for (int c = 0; c < NT / 32; ++c) {
          uint32_t r[32];
          tmem_ld32(tm + 32 * c, r);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; ++i)
            z[32 * c + i] = (kb > 0 ? z[32 * c + i] : 0.f) + __uint_as_float(r[i]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive1(smem_addr(&acc_empty[ab]));
      }
      if (!ok) {
        if (lane == 0) give_up();
        break;
      }
      const int v = t * tile_rows + row;
      const bool mine = row < tile_rows && v < p.vocab;  // (else it is not W's)
      if constexpr (GRAD) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          float x = s_grad[j] * exp2_fast((z[j] - s_lse[j]) * kLog2e);
          if (s_target[j] == v) x = s_of_target[j];
          if (s_target[j] < 0) x = 0.f;  // (W may be infinite)
          if (mine) g_out[j * ld_g + v] = __float2bfloat16_rn(x);
        }
      } else if (mine) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          if (s_target[j] == v) z[j] = s_of_target[j];
          // the larger one is the new maximum, which is finite for z = -inf too (exp 0)
          const float d = z[j] - m[j], e = exp2_fast(-fabsf(d) * kLog2e);
          sum[j] = d > 0.f ? __fmaf_rn(sum[j], e, 1.f) : sum[j] + e;
          m[j] = fmaxf(m[j], z[j]);
        }
      }
    }
    if (GRAD && blockIdx.x == 0)  // zeros up to whole tiles of the products that take G
      for (int v = p.vocab + row; v < (p.vocab + kTile - 1) / kTile * kTile; v += kHalf)
        for (int j = 0; j < NT; ++j) g_out[j * ld_g + v] = __float2bfloat16_rn(0.f);
    if constexpr (!GRAD) {
      // (all MMAs have read the ring: the last accumulator came after them)
      float2* part = reinterpret_cast<float2*>(smem);  // [NT][128]
      if (ok)
#pragma unroll
        for (int j = 0; j < NT; ++j) part[j * kHalf + (row ^ j)] = make_float2(m[j], sum[j]);
    }
  }
  __syncthreads();
  if constexpr (!GRAD) {
    auto merge = [](float2 a, float2 b) {
      const float mm = fmaxf(a.x, b.x), ref = safe_max(mm);
      return make_float2(mm, __fmaf_rn(a.y, exp2_fast((a.x - ref) * kLog2e),
                                       __fmul_rn(b.y, exp2_fast((b.x - ref) * kLog2e))));
    };
    // four groups by kShare lanes
    constexpr int kShare = 128 / NT;
    auto join = [&](auto of_group) {
      const int g = static_cast<int>(threadIdx.x) % kShare * (4 / kShare);
      float2 st = of_group(g);
      if (kShare == 2) st = merge(st, of_group(g + 1));
#pragma unroll
      for (int o = 1; o < kShare; o *= 2)
        st = merge(st, make_float2(__shfl_down_sync(0xffffffffu, st.x, o),
                                   __shfl_down_sync(0xffffffffu, st.y, o)));
      return st;
    };
    if (!*abort_flag) {
      // 128 threads' sums of a column by 128 / NT threads
      const float2* part = reinterpret_cast<const float2*>(smem);
      if (threadIdx.x < 128) {
        const int j = threadIdx.x / kShare, g = threadIdx.x % kShare;
        const float2 st = join([&](int group) {
          float2 a = make_float2(-INFINITY, 0.f);
          for (int i = 0; i < 32; ++i) a = merge(a, part[j * kHalf + ((group * 32 + i) ^ j)]);
          return a;
        });
        if (g == 0) p.stats[blockIdx.x * NT + j] = st;
      }
    }
    // the last CTA joins them all
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) *s_last = atomicAdd(p.queue, 1u) == gridDim.x - 1;
    __syncthreads();
    if (*s_last && threadIdx.x < 128) {
      __threadfence();
      const int live = min(max(*p.live, 0), p.rows);
      const int j = threadIdx.x / kShare, g = threadIdx.x % kShare;
      const float2 st = join([&](int group) {
        float2 a = make_float2(-INFINITY, 0.f);
#pragma unroll 8
        for (unsigned c = group; c < gridDim.x; c += 4) a = merge(a, __ldcg(p.stats + c * NT + j));
        return a;
      });
      if (g == 0 && j < live) {
        const float ln = logf(st.y), mm = safe_max(st.x);
        const int r = p.row[j];
        lse[r] = mm + ln;
        loss[r] = (mm - __ldcg(p.z_target + j)) + ln;
      }
    }
  }
  tc_fence_after();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc(tmem_base, F::kTmem);
  }
}

// ---- ends ---------------------------------------------------------------------
// The maxima and sums of a row's slices to its lse and loss: 32 rows x 32 groups of
// slices a CTA.
__global__ void __launch_bounds__(1024)
    head_loss_kernel(const float2* __restrict__ stats, int64_t ld_stats, int slices,
                     const int* __restrict__ live, const int* __restrict__ row,
                     const float* __restrict__ z_target, float* __restrict__ loss,
                     float* __restrict__ lse) {
  __shared__ float2 s_part[32][33];
  grid_dep_wait();
  grid_dep_launch();
  const int n = *live;
  if (blockIdx.x * 32 >= static_cast<unsigned>(n)) return;
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int64_t i = blockIdx.x * 32 + x;
  float2 st = make_float2(-INFINITY, 0.f);
  auto merge = [](float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x), ref = safe_max(m);
    return make_float2(m, a.y * exp2_fast((a.x - ref) * kLog2e) +
                              b.y * exp2_fast((b.x - ref) * kLog2e));
  };
  // (a NaN maximum is lost in fmaxf, its sum is not)
  for (int s = y; s < slices; s += 32) st = merge(st, stats[s * ld_stats + i]);
  s_part[y][x] = st;
  __syncthreads();
  if (y >= 1 || i >= n) return;
  for (int s = 1; s < 32; ++s) st = merge(st, s_part[s][x]);
  const float ln = logf(st.y), m = safe_max(st.x);
  const int r = row[i];
  lse[r] = m + ln;
  loss[r] = (m - z_target[i]) + ln;  // (m is often the target's own logit)
}

// Dh of the rows that count, the sums of its parts in their order and what rounding took
// from the target's term; zeros elsewhere.  A thread has four columns of a row (ld_sums
// is a multiple of 32, so they are there).
template <typename Te>
__global__ void __launch_bounds__(256)
    head_hidden_kernel(const float* __restrict__ sums, int64_t ld_sums, int64_t part_stride,
                       int parts, const int* __restrict__ place, const int* __restrict__ target,
                       const float* __restrict__ target_term,
                       const __nv_bfloat16* __restrict__ w, int64_t ldw, int64_t rows, int k,
                       Te* __restrict__ out, int64_t ldo, bool vec) {
  grid_dep_wait();
  grid_dep_launch();
  const int quads = (k + 3) / 4;
  const int64_t n = rows * quads;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t r = i / quads;
    const int c = static_cast<int>(i - r * quads) * 4;
    const int at = place[r];
    float f[4] = {0.f, 0.f, 0.f, 0.f};
    if (at >= 0) {
      const float* from = sums + at * ld_sums + c;
#pragma unroll 4
      for (int s = 0; s < parts; ++s) {
        const float4 v = *reinterpret_cast<const float4*>(from + s * part_stride);
        f[0] += v.x;
        f[1] += v.y;
        f[2] += v.z;
        f[3] += v.w;
      }
      const float rest = lost_in_bf16(target_term[at]);
      const __nv_bfloat16* row = w + target[at] * ldw + c;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = c + e < k ? to_f32(row[e]) : 0.f;
        if (fabsf(x) < INFINITY) f[e] = __fmaf_rn(rest, x, f[e]);
      }
    }
    Te* to = out + r * ldo + c;
    if (vec) {
      if constexpr (sizeof(Te) == 4) {
        *reinterpret_cast<float4*>(to) = make_float4(f[0], f[1], f[2], f[3]);
      } else {
        *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < k) to[e] = from_f32<Te>(f[e]);
    }
  }
}

bool box_map(CUtensorMap* m, PFN_cuTensorMapEncodeTiled_v12000 fn, const void* base, bool f32,
             int64_t rows, int64_t cols, int64_t ld, int box_cols, int box_rows) {
  const cuuint64_t es = f32 ? 4 : 2;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * es};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(box_cols),
                             static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t estr[2] = {1, 1};
  return fn(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
            const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool LOSS>
cudaError_t launch_tiles(const Maps& maps, const HeadTiles& p, int64_t jobs, int sms,
                         cudaStream_t stream) {
  auto kernel = head_tiles_kernel<LOSS>;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(kernel, kSmemBytes, done);
  if (e != cudaSuccess) return e;
  const int64_t pairs = jobs < sms / 2 ? jobs : sms / 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(2 * pairs));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, maps, p);
}

template <int NT, bool GRAD>
cudaError_t launch_few(const HeadProblem& h, const HeadTiles& p, void* g, int64_t ld_g,
                       float* loss, float* lse, int sms, cudaStream_t stream) {
  const int tile_rows = head_few_tile_rows(p.vocab, sms);
  CUtensorMap map_w, map_h;
  if (!box_map(&map_w, h.encode, h.w, false, p.vocab, p.k, h.ldw, BK, tile_rows) ||
      !box_map(&map_h, h.encode, h.packed, false, p.rows_up, p.k, h.ld_packed, BK, NT))
    return cudaErrorInvalidValue;
  auto kernel = head_few_kernel<NT, GRAD>;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(kernel, Few<NT>::kSmem, done);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(head_few_ctas(p.vocab, sms)), dim3(kFewThreads), Few<NT>::kSmem,
                    stream, map_w, map_h, p, tile_rows, static_cast<__nv_bfloat16*>(g), ld_g,
                    loss, lse);
}

}  // namespace

cudaError_t launch_head_rows(const HeadRows& p, int sms, cudaStream_t stream) {
  const bool vec = p.k % 8 == 0 && reinterpret_cast<uintptr_t>(p.hidden) % 16 == 0 &&
                   p.ld_hidden % 8 == 0;
  // (with rows of zeros to write, a few CTAs more than rows)
  const int64_t ctas = p.rows > 2 * sms ? 2 * sms : p.rows > 32 ? p.rows : 32;
  return launch_pdl(head_rows_kernel, dim3(static_cast<unsigned>(ctas)), dim3(kRowsThreads), 0,
                    stream, p, vec);
}

cudaError_t launch_head_loss(const HeadProblem& h, HeadTiles p, float* loss, float* lse, int sms,
                             cudaStream_t stream) {
  if (head_few_rows(p.rows, 1))
    return head_few_columns(p.rows) == 32
               ? launch_few<32, false>(h, p, nullptr, 0, loss, lse, sms, stream)
               : launch_few<64, false>(h, p, nullptr, 0, loss, lse, sms, stream);
  Maps maps;
  if (!box_map(&maps.h_rows, h.encode, h.packed, false, p.rows_up, p.k, h.ld_packed, BK, kHalf) ||
      !box_map(&maps.w_rows, h.encode, h.w, false, p.vocab, p.k, h.ldw, BK, kHalf))
    return cudaErrorInvalidValue;
  p.vt_next = static_cast<int>((static_cast<int64_t>(p.vocab) + kTile - 1) / kTile);
  p.v_next = 0;
  const int64_t mt = p.rows_up / kTile;
  cudaError_t e = launch_tiles<true>(maps, p, mt * p.vt_next, sms, stream);
  if (e != cudaSuccess) return e;
  return launch_pdl(head_loss_kernel, dim3(static_cast<unsigned>((p.rows + 31) / 32)), dim3(1024),
                    0, stream, static_cast<const float2*>(p.stats), p.ld_stats, 2 * p.vt_next,
                    p.live, p.row, p.z_target, loss, lse);
}

cudaError_t launch_head_loss_backward(const HeadProblem& h, HeadTiles p, const HeadPieces& q,
                                      const int* place, int64_t rows, void* d_hidden,
                                      int64_t ld_d_hidden, bool d_hidden_f32, int sms,
                                      cudaStream_t stream) {
  Maps maps;
  p.kt = (p.k + kTile - 1) / kTile;
  const int es = p.dw_f32 ? 4 : 2, unit = 16 / es;
  p.dw_mapped = reinterpret_cast<uintptr_t>(p.dw) % 16 == 0 && p.ld_dw % unit == 0 && p.k >= unit;
  p.dw_mapped = p.dw_mapped && p.dw != nullptr;
  if (!box_map(&maps.h_rows, h.encode, h.packed, false, p.rows_up, p.k, h.ld_packed, BK, kHalf) ||
      !box_map(&maps.h_cols, h.encode, h.packed, false, p.rows_up, p.k, h.ld_packed, 64, BK) ||
      !box_map(&maps.w_rows, h.encode, h.w, false, p.vocab, p.k, h.ldw, BK, kHalf) ||
      !box_map(&maps.w_cols, h.encode, h.w, false, p.vocab, p.k, h.ldw, 64, BK) ||
      (q.sums != nullptr &&
       !box_map(&maps.dh_out, h.encode, q.sums, true, static_cast<int64_t>(q.parts) * p.rows_up,
                p.ld_sums, p.ld_sums, 32, 32)) ||
      (p.dw_mapped && !box_map(&maps.dw_out, h.encode, p.dw, p.dw_f32, p.vocab, p.k / unit * unit,
                               p.ld_dw, 128 / es, 32)))
    return cudaErrorInvalidValue;
  const int64_t vt = (static_cast<int64_t>(p.vocab) + kTile - 1) / kTile;
  const int pieces = static_cast<int>((vt + q.piece_tiles - 1) / q.piece_tiles);
  const int64_t mt = p.rows_up / kTile;
  uint32_t* queue = p.queue;
  for (int i = 0; i <= pieces; ++i) {
    // hidden and weight tiles of piece i - 1, grad tiles of piece i
    const int64_t now = i > 0 ? std::min<int64_t>(q.piece_tiles, vt - (i - 1) * int64_t{q.piece_tiles}) : 0;
    const int64_t next = i < pieces ? std::min<int64_t>(q.piece_tiles, vt - i * int64_t{q.piece_tiles}) : 0;
    const int64_t ld_g = int64_t{q.piece_tiles} * kTile;
    const int64_t g_size = p.rows_up * ld_g;
    void* g_now = q.g + (pieces > 1 ? (i + 1) & 1 : 0) * g_size;
    void* g_next = q.g + (pieces > 1 ? i & 1 : 0) * g_size;
    if (!box_map(&maps.g_rows, h.encode, g_now, false, p.rows_up, ld_g, ld_g, BK, kHalf) ||
        !box_map(&maps.g_cols, h.encode, g_now, false, p.rows_up, ld_g, ld_g, 64, BK) ||
        !box_map(&maps.g_out, h.encode, g_next, false, p.rows_up, ld_g, ld_g, 64, 32))
      return cudaErrorInvalidValue;
    p.vt = static_cast<int>(now);
    p.v0 = (i - 1) * q.piece_tiles * kTile;
    p.vt_next = static_cast<int>(next);
    p.v_next = i * q.piece_tiles * kTile;
    const int blocks = p.vt * (kTile / BK);
    p.part_blocks = q.part_blocks;
    p.parts = q.sums != nullptr ? (blocks + q.part_blocks - 1) / q.part_blocks : 0;
    p.hidden_first = q.sums != nullptr && p.part_blocks * BK >= p.rows;
    p.queue = queue + i;
    if (i == 0 && head_few_rows(p.rows, pieces)) {
      // (64 rows: a whole stage of the products that take G)
      const cudaError_t e = launch_few<64, true>(h, p, g_next, ld_g, nullptr, nullptr, sms, stream);
      if (e != cudaSuccess) return e;
      continue;
    }
    const int64_t jobs = mt * next + mt * p.kt * p.parts + (p.dw != nullptr ? now * p.kt : 0);
    if (jobs == 0) continue;
    const cudaError_t e = launch_tiles<false>(maps, p, jobs, sms, stream);
    if (e != cudaSuccess) return e;
  }
  if (q.sums == nullptr) return cudaSuccess;
  const int64_t ctas = std::min<int64_t>((rows * ((p.k + 3) / 4) + 255) / 256, int64_t{sms} * 16);
  const int es_h = d_hidden_f32 ? 4 : 2;
  const auto* w = static_cast<const __nv_bfloat16*>(h.w);
  const bool vec = p.k % 4 == 0 && ld_d_hidden % 4 == 0 &&
                   reinterpret_cast<uintptr_t>(d_hidden) % (4 * es_h) == 0;
  // parts of the first piece; a shorter last piece adds to fewer of them
  const int64_t first = std::min<int64_t>(q.piece_tiles, vt) * (kTile / BK);
  const int parts = static_cast<int>((first + q.part_blocks - 1) / q.part_blocks);
  const int64_t stride = static_cast<int64_t>(p.rows_up) * p.ld_sums;
  if (d_hidden_f32)
    return launch_pdl(head_hidden_kernel<float>, dim3(static_cast<unsigned>(ctas)), dim3(256), 0,
                      stream, static_cast<const float*>(q.sums), p.ld_sums, stride, parts, place,
                      p.target, p.target_term, w, h.ldw, rows, p.k,
                      static_cast<float*>(d_hidden), ld_d_hidden, vec);
  return launch_pdl(head_hidden_kernel<__nv_bfloat16>, dim3(static_cast<unsigned>(ctas)),
                    dim3(256), 0, stream, static_cast<const float*>(q.sums), p.ld_sums, stride,
                    parts, place, p.target, p.target_term, w, h.ldw, rows, p.k,
                    static_cast<__nv_bfloat16*>(d_hidden), ld_d_hidden, vec);
}

}  // namespace rx
