// expert_rows.cu — tokens laid out by expert and summed back with their router
// weights, as calls of their own, and the gradients of both:
//   plan      the row of every pair (t, j) in the order (expert, token, slot)
//   rows      rows[row_of[t, j]] = x[t];        backward  Dx[t] = sum_j Drows[row_of[t, j]]
//   combine   out[t] = sum_j alpha[t, j] y[row_of[t, j]] (+ residual[t]);
//             backward  Dy[row] = alpha Dout[t],  Dalpha[t, j] = <Dout[t], y[row]>
// The plan is a stable counting sort without atomics whose order matters: each warp
// takes a run of pairs, 32 at a time; lanes of equal experts find one another
// (match.any), the lowest of them keeps the warp's count of that expert, and a lane's
// place is that count plus the equal lanes below it.  The same expert may come more
// than once in a token.  The copies and sums are bound by bytes; every one of them
// walks the tokens and reaches the pair rows through row_of, so a token's row crosses
// HBM once.  Unused slots contribute nothing, whatever their weights are; rows behind
// the last pair are neither read nor written.
#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "internal.h"

namespace rx {
namespace {

constexpr int kPlanWarps = 16;
constexpr int kPlanThreads = 32 * kPlanWarps;
constexpr int kPlanExperts = 1024;  // at most
constexpr int kPlanPairs = 2 * kPlanThreads;  // pairs of a CTA, at least

// The expert of pair i, -1 for an unused or refused slot.
struct Pairs {
  const int32_t* ids;
  const int32_t* k;
  int64_t n;
  int E, k_max;
  __device__ __forceinline__ int expert(int64_t i, uint32_t* err) const {
    if (i >= n) return -1;
    if (k != nullptr) {
      const int64_t t = i / k_max;
      const int kt = k[t];
      if (kt < 0 || kt > k_max) set_err(err, kErrKRange);
      if (static_cast<int>(i - t * k_max) >= kt) return -1;  // (k_max slots at most)
    }
    const int e = ids[i];
    if (e >= 0 && e < E) return e;
    // without counts, a negative id is an unused slot
    if (e >= E || k != nullptr) set_err(err, kErrIndex);
    return -1;
  }
};

// Adds the pairs [lo, hi) of this warp to its counts of experts.
__device__ __forceinline__ void count_pairs(const Pairs& p, int64_t lo, int64_t hi, int32_t* count,
                                            uint32_t* err) {
  const int lane = threadIdx.x & 31;
  for (int64_t i = lo; i < hi; i += 32) {
    const int e = i + lane < hi ? p.expert(i + lane, err) : -1;
    const uint32_t same = __match_any_sync(0xffffffffu, e);
    if (e >= 0 && (same & ((1u << lane) - 1u)) == 0u) count[e] += __popc(same);
    __syncwarp();
  }
}

__global__ void __launch_bounds__(kPlanThreads)
    plan_count_kernel(const Pairs p, int64_t per_warp, int32_t* __restrict__ blk_count,
                      uint32_t* err) {
  extern __shared__ int32_t s_count[];  // [kPlanWarps][E]
  grid_dep_wait();
  grid_dep_launch();
  // (the placing kernel reports what is wrong with a pair)
  if (blockIdx.x == 0 && threadIdx.x == 0 && err != nullptr) *err = 0u;
  for (int i = threadIdx.x; i < kPlanWarps * p.E; i += kPlanThreads) s_count[i] = 0;
  __syncthreads();
  const int w = threadIdx.x >> 5;
  const int64_t lo = (static_cast<int64_t>(blockIdx.x) * kPlanWarps + w) * per_warp;
  count_pairs(p, lo, min(lo + per_warp, p.n), s_count + w * p.E, nullptr);
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += kPlanThreads) {
    int c = 0;
    for (int i = 0; i < kPlanWarps; ++i) c += s_count[i * p.E + e];
    blk_count[static_cast<int64_t>(blockIdx.x) * p.E + e] = c;
  }
}

// Exclusive scan over E <= kPlanExperts values in shared memory, two to a thread; returns the sum.
__device__ int scan_experts(int32_t* v, int E, int32_t* s_warp) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int i = 2 * threadIdx.x;
  const int a = i < E ? v[i] : 0, b = i + 1 < E ? v[i + 1] : 0;
  int x = a + b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += u;
  }
  if (lane == 31) s_warp[w] = x;
  __syncthreads();
  int below = 0, total = 0;
  for (int j = 0; j < kPlanWarps; ++j) {
    if (j < w) below += s_warp[j];
    total += s_warp[j];
  }
  const int excl = below + x - a - b;
  if (i < E) v[i] = excl;
  if (i + 1 < E) v[i + 1] = excl + a;
  __syncthreads();
  return total;
}

// nblk == 1: the only kernel of the plan, which then counts for itself.
__global__ void __launch_bounds__(kPlanThreads)
    plan_place_kernel(const Pairs p, int64_t per_warp, int nblk,
                      const int32_t* __restrict__ blk_count, int cap_rows,
                      int32_t* __restrict__ row_of, int32_t* __restrict__ counts,
                      int32_t* __restrict__ offsets, int32_t* __restrict__ perm, uint32_t* err) {
  extern __shared__ int32_t s_count[];  // [kPlanWarps][E], then [E] totals, [E] of earlier CTAs
  __shared__ int32_t s_warp[kPlanWarps];
  const int E = p.E;
  int32_t* s_total = s_count + kPlanWarps * E;
  int32_t* s_before = s_total + E;
  grid_dep_wait();
  grid_dep_launch();
  if (nblk == 1 && threadIdx.x == 0 && err != nullptr) *err = 0u;
  for (int i = threadIdx.x; i < (kPlanWarps + 2) * E; i += kPlanThreads) s_count[i] = 0;
  __syncthreads();
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t lo = (static_cast<int64_t>(blockIdx.x) * kPlanWarps + w) * per_warp;
  const int64_t hi = min(lo + per_warp, p.n);
  count_pairs(p, lo, hi, s_count + w * E, nullptr);
  if (nblk > 1) {
    // all CTAs' counts, `share` threads to an expert
    int share = 1;
    while (2 * share * E <= kPlanThreads) share *= 2;
    for (int i = threadIdx.x; i < share * E; i += kPlanThreads) {
      const int e = i % E, g = i / E;
      int all = 0, before = 0;
#pragma unroll 16
      for (int b = g; b < nblk; b += share) {
        const int c = blk_count[static_cast<int64_t>(b) * E + e];
        all += c;
        before += b < static_cast<int>(blockIdx.x) ? c : 0;
      }
      atomicAdd(&s_total[e], all);  // whole numbers: any order
      atomicAdd(&s_before[e], before);
    }
    __syncthreads();
  } else {
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kPlanThreads)
      for (int i = 0; i < kPlanWarps; ++i) s_total[e] += s_count[i * E + e];
    __syncthreads();
  }
  if (blockIdx.x == 0)
    for (int e = threadIdx.x; e < E; e += kPlanThreads) counts[e] = s_total[e];
  __syncthreads();
  const int total = scan_experts(s_total, E, s_warp);
  if (blockIdx.x == 0) {
    for (int e = threadIdx.x; e < E; e += kPlanThreads) offsets[e] = s_total[e];
    if (threadIdx.x == 0) offsets[E] = total;
  }
  // counts of this CTA's warps to the first row of each warp
  for (int e = threadIdx.x; e < E; e += kPlanThreads) {
    int at = s_total[e] + s_before[e];
    for (int i = 0; i < kPlanWarps; ++i) {
      const int c = s_count[i * E + e];
      s_count[i * E + e] = at;
      at += c;
    }
  }
  __syncthreads();
  int32_t* place = s_count + w * E;
  for (int64_t i = lo; i < hi; i += 32) {
    const int e = i + lane < hi ? p.expert(i + lane, err) : -1;
    const uint32_t same = __match_any_sync(0xffffffffu, e);
    const uint32_t below = same & ((1u << lane) - 1u);
    int row = e >= 0 ? place[e] + __popc(below) : -1;
    __syncwarp();
    if (e >= 0 && below == 0u) place[e] += __popc(same);
    __syncwarp();
    if (row >= cap_rows) {
      set_err(err, kErrCapacity);
      row = -1;
    }
    if (i + lane < hi) row_of[i + lane] = row;
    if (row >= 0 && perm != nullptr) perm[row] = static_cast<int32_t>(i + lane);
  }
}

// ---- copies and sums ---------------------------------------------------------
constexpr int kThreads = 256;

// A lane's share of several turns over a row, as stored: units of UB bytes one warp
// apart, 16-byte vectors, or, where rows or columns do not allow it, words or elements
// (and then eight elements in more units, as a unit is all that a load brings).
// Words matter to bf16 rows of an even width: 65536 tokens of 150, one slot, combine
// 44 us by elements and 30 by words, 16384 of 1004, four slots, 71 and 44, and their
// gradients 83 and 63.
template <typename Te, int UB, int kVecs16>
struct Share {
  static constexpr int kEach = UB / static_cast<int>(sizeof(Te));
  static constexpr int kVecs = UB == 16 ? kVecs16 : 8 / kEach;
  static constexpr int kSpan = 32 * kEach * kVecs;  // columns of a warp
  static constexpr int kElems = kEach * kVecs;
  // (as words: elements of two bytes by themselves would take a register each)
  using Unit = std::conditional_t<UB == 16, uint4, std::conditional_t<UB == 4, uint32_t, Te>>;
  Unit u[kVecs];
  static __device__ __forceinline__ int col(int c0, int i) {
    return c0 + (i * 32 + static_cast<int>(threadIdx.x & 31)) * kEach;
  }
  __device__ __forceinline__ void load(const Te* row, int c0, int d) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (col(c0, i) < d) u[i] = *reinterpret_cast<const Unit*>(row + col(c0, i));
  }
  // (elements past the row are not set)
  __device__ __forceinline__ float at(int i, int e) const {
    uint32_t w;
    if constexpr (UB == 2) {
      return to_f32(u[i]);
    } else if constexpr (UB == 4) {
      w = u[i];
    } else {
      const uint32_t q[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
      w = q[sizeof(Te) == 4 ? e : e >> 1];
    }
    if constexpr (sizeof(Te) == 4) return __uint_as_float(w);
    return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
  }
  // unit i, kEach floats
  static __device__ __forceinline__ void store(Te* row, int c0, int d, int i, const float* f) {
    if (col(c0, i) >= d) return;
    Te* to = row + col(c0, i);
    if constexpr (kEach == 1) *to = from_f32<Te>(f[0]);
    else if constexpr (kEach == 2)
      *reinterpret_cast<__nv_bfloat162*>(to) = __floats2bfloat162_rn(f[0], f[1]);
    else if constexpr (sizeof(Te) == 2) store8(to, f);
    else *reinterpret_cast<float4*>(to) = make_float4(f[0], f[1], f[2], f[3]);
  }
};

// The used slots of token t, in order: lane i gets the i-th one's row and slot.
__device__ __forceinline__ int used_slots(const int32_t* row_of, int64_t t, int k_max,
                                          int cap_rows, int lane, int& row, int& slot) {
  int r = -1;
  if (lane < k_max) r = row_of[t * k_max + lane];
  const bool used = r >= 0 && r < cap_rows;
  const uint32_t mask = __ballot_sync(0xffffffffu, used);
  slot = lane;
  if ((mask & (mask + 1u)) != 0u) {  // gaps between them
    slot = __fns(mask, 0, lane + 1);  // -1 past the last one
    if (slot < 0 || slot > 31) slot = 0;
  }
  row = __shfl_sync(0xffffffffu, r, slot);
  return __popc(mask);
}

// x[t] to each of its rows: a warp per token and `turns` spans of columns, which stay
// in registers as stored.
template <typename V>
__global__ void __launch_bounds__(kThreads)
    rows_kernel(const V* __restrict__ x, int64_t ldx, const int32_t* __restrict__ row_of,
                int64_t T, int d, int k_max, int cap_rows, V* __restrict__ rows, int64_t ldr,
                int segments) {
  constexpr int kVecs = 8;  // of a lane and segment
  grid_dep_wait();
  grid_dep_launch();
  const int lane = threadIdx.x & 31;
  const int64_t units = T * segments;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
       u < units; u += step) {
    const int64_t t = u / segments;
    const int c0 = static_cast<int>(u - t * segments) * (32 * kVecs) + lane;
    int r = -1;
    if (lane < k_max) r = row_of[t * k_max + lane];
    if (r >= cap_rows) r = -1;
    V v[kVecs];
    const V* src = x + t * ldx;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (c0 + 32 * i < d) v[i] = __ldg(src + c0 + 32 * i);
    uint32_t used = __ballot_sync(0xffffffffu, r >= 0);
    while (used != 0u) {
      const int j = __ffs(used) - 1;
      used &= used - 1u;
      V* dst = rows + __shfl_sync(0xffffffffu, r, j) * ldr;
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
        if (c0 + 32 * i < d) dst[c0 + 32 * i] = v[i];
    }
  }
}

// A warp for a token and a few turns of its columns, four pair rows under way
// together.  alpha == nullptr: weight 1.
constexpr int kCombineVecs = 2;
constexpr int kBatch = 4;
template <typename Te, int UB>
__global__ void __launch_bounds__(kThreads, 3)
    combine_rows_kernel(const Te* __restrict__ rows, int64_t ldr,
                        const int32_t* __restrict__ row_of, const float* __restrict__ alpha,
                        const Te* residual, int64_t ldres, int64_t T, int d, int k_max,
                        int cap_rows, Te* out, int64_t ldo, int segments) {
  using S = Share<Te, UB, kCombineVecs>;
  grid_dep_wait();
  grid_dep_launch();
  const int lane = threadIdx.x & 31;
  const int64_t units = T * segments;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
       u < units; u += step) {
    const int64_t t = u / segments;
    const int c0 = static_cast<int>(u - t * segments) * S::kSpan;
    S res;
    if (residual != nullptr) res.load(residual + t * ldres, c0, d);
    int row, slot;
    float my_a = 1.f;
    if (alpha != nullptr && lane < k_max) my_a = alpha[t * k_max + lane];
    const int n = used_slots(row_of, t, k_max, cap_rows, lane, row, slot);
    my_a = __shfl_sync(0xffffffffu, my_a, slot);
    float acc[S::kElems];
#pragma unroll
    for (int i = 0; i < S::kElems; ++i) acc[i] = 0.f;
    for (int j0 = 0; j0 < n; j0 += kBatch) {
      S y[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int r = __shfl_sync(0xffffffffu, row, (j0 + b) & 31);
        if (j0 + b < n) y[b].load(rows + r * ldr, c0, d);
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const float a = __shfl_sync(0xffffffffu, my_a, (j0 + b) & 31);
        if (j0 + b < n)
#pragma unroll
          for (int i = 0; i < S::kVecs; ++i)
#pragma unroll
            for (int e = 0; e < S::kEach; ++e)
              acc[i * S::kEach + e] = __fmaf_rn(a, y[b].at(i, e), acc[i * S::kEach + e]);
      }
    }
#pragma unroll
    for (int i = 0; i < S::kVecs; ++i) {
      if (residual != nullptr)
#pragma unroll
        for (int e = 0; e < S::kEach; ++e) acc[i * S::kEach + e] += res.at(i, e);
      S::store(out + t * ldo, c0, d, i, acc + i * S::kEach);
    }
  }
}

// A warp for a pair, its whole rows under way (up to 1024 columns of bf16 at a time);
// the warps of a token run next to one another and read its gradient from L1 or L2.
constexpr int kGradVecs = 4;
template <typename Te, int UB>
__global__ void __launch_bounds__(kThreads, 4)
    combine_backward_kernel(const Te* __restrict__ d_out, int64_t ldd, const Te* rows, int64_t ldr,
                            const int32_t* __restrict__ row_of, const float* __restrict__ alpha,
                            int64_t T, int d, int k_max, int cap_rows, Te* d_rows, int64_t lddr,
                            float* __restrict__ d_alpha) {
  using S = Share<Te, UB, kGradVecs>;
  grid_dep_wait();
  grid_dep_launch();
  const int lane = threadIdx.x & 31;
  const int64_t pairs = T * k_max;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
       u < pairs; u += step) {
    const int r = row_of[u];
    if (r < 0 || r >= cap_rows) {
      if (lane == 0 && d_alpha != nullptr) d_alpha[u] = 0.f;
      continue;
    }
    const Te* go = d_out + u / k_max * ldd;
    const Te* y = rows + r * ldr;
    Te* dy = d_rows + r * lddr;
    const float a = alpha[u];
    float dot = 0.f;
    for (int c0 = 0; c0 < d; c0 += S::kSpan) {
      S g, f;
      g.load(go, c0, d);
      if (d_alpha != nullptr) f.load(y, c0, d);
      if (d_alpha != nullptr)
#pragma unroll
        for (int i = 0; i < S::kVecs; ++i)
          if (S::col(c0, i) < d)
#pragma unroll
            for (int e = 0; e < S::kEach; ++e) dot = __fmaf_rn(g.at(i, e), f.at(i, e), dot);
      if (d_rows != nullptr)
#pragma unroll
        for (int i = 0; i < S::kVecs; ++i) {
          float o[S::kEach];
#pragma unroll
          for (int e = 0; e < S::kEach; ++e) o[e] = a * g.at(i, e);
          S::store(dy, c0, d, i, o);
        }
    }
    if (d_alpha == nullptr) continue;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
    if (lane == 0) d_alpha[u] = dot;
  }
}

bool on(int bytes, const void* p, int64_t ld, int es) {
  return p == nullptr || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * es % bytes == 0);
}
unsigned warps_grid(int64_t warps, int sms) {
  const int64_t need = (warps + kThreads / 32 - 1) / (kThreads / 32);
  const int64_t most = static_cast<int64_t>(sms) * 32;
  return static_cast<unsigned>(need < most ? need : most);
}

template <typename V>
cudaError_t launch_rows(const ExpertRowsArgs& p, const void* x, int64_t ldx, void* rows,
                        int64_t ldr, int d, int sms, cudaStream_t s) {
  const int segments = (d + 255) / 256;
  return launch_pdl(rows_kernel<V>, dim3(warps_grid(p.T * segments, sms)), dim3(kThreads), 0, s,
                    static_cast<const V*>(x), ldx, p.row_of, p.T, d, p.k_max, p.cap_rows,
                    static_cast<V*>(rows), ldr, segments);
}

template <typename Te, int UB>
cudaError_t launch_combine_rows(const ExpertRowsArgs& p, int sms, cudaStream_t s) {
  constexpr int kSpan = Share<Te, UB, kCombineVecs>::kSpan;
  const int segments = (p.d + kSpan - 1) / kSpan;
  return launch_pdl(combine_rows_kernel<Te, UB>, dim3(warps_grid(p.T * segments, sms)),
                    dim3(kThreads), 0, s, static_cast<const Te*>(p.rows), p.ldr, p.row_of, p.alpha,
                    static_cast<const Te*>(p.x), p.ldx, p.T, p.d, p.k_max, p.cap_rows,
                    static_cast<Te*>(p.out), p.ldo, segments);
}

template <typename Te, int UB>
cudaError_t launch_combine_backward(const ExpertRowsArgs& p, int sms, cudaStream_t s) {
  return launch_pdl(combine_backward_kernel<Te, UB>, dim3(warps_grid(p.T * p.k_max, sms)),
                    dim3(kThreads), 0, s, static_cast<const Te*>(p.x), p.ldx,
                    static_cast<const Te*>(p.rows), p.ldr, p.row_of, p.alpha, p.T, p.d, p.k_max,
                    p.cap_rows, static_cast<Te*>(p.out), p.ldo, p.d_alpha);
}

// pairs of a warp and CTAs of the plan
int64_t plan_per_warp(int64_t n, int sms) {
  const int64_t want = (n + sms - 1) / sms;
  const int64_t per = want > kPlanPairs ? want : kPlanPairs;
  return (per + kPlanThreads - 1) / kPlanThreads * 32;
}

}  // namespace

int64_t expert_plan_blocks_most(int64_t n, int sms) {
  const int64_t blocks = (n + kPlanPairs - 1) / kPlanPairs;
  return blocks < 1 ? 1 : blocks < sms ? blocks : sms;
}

cudaError_t launch_expert_plan(const int32_t* ids, const int32_t* k, int64_t T, int E, int k_max,
                               int cap_rows, int32_t* row_of, int32_t* counts, int32_t* offsets,
                               int32_t* perm, uint32_t* err, int32_t* blk_count, int sms,
                               cudaStream_t s) {
  const Pairs p{ids, k, T * k_max, E, k_max};
  const int64_t per_warp = plan_per_warp(p.n, sms);
  // (no tokens: one CTA all the same, for counts of zero)
  const int nblk = static_cast<int>(std::max<int64_t>(
      1, (p.n + per_warp * kPlanWarps - 1) / (per_warp * kPlanWarps)));
  const size_t count_smem = static_cast<size_t>(kPlanWarps) * E * 4;
  const size_t place_smem = count_smem + 2 * static_cast<size_t>(E) * 4;
  cudaError_t e;
  if (place_smem > 48 * 1024) {
    // as much as any plan needs, so that no call lowers what another is about to launch with
    static std::atomic<uint64_t> count_done{0}, place_done{0};
    e = allow_smem(plan_count_kernel, size_t{kPlanWarps} * kPlanExperts * 4, count_done);
    if (e == cudaSuccess)
      e = allow_smem(plan_place_kernel, size_t{kPlanWarps + 2} * kPlanExperts * 4, place_done);
    if (e != cudaSuccess) return e;
  }
  if (nblk > 1) {
    e = launch_pdl(plan_count_kernel, dim3(nblk), dim3(kPlanThreads), count_smem, s, p, per_warp,
                   blk_count, err);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(plan_place_kernel, dim3(nblk), dim3(kPlanThreads), place_smem, s, p, per_warp,
                    nblk, static_cast<const int32_t*>(blk_count), cap_rows, row_of, counts,
                    offsets, perm, err);
}

cudaError_t launch_expert_rows(int dtype, const ExpertRowsArgs& p, int sms, cudaStream_t s) {
  const int es = dtype == 0 ? 4 : 2;
  const int64_t row = int64_t{p.d} * es;  // bytes
  auto rows_on = [&](int bytes) {
    return row % bytes == 0 && on(bytes, p.x, p.ldx, es) && on(bytes, p.out, p.ldo, es);
  };
  if (rows_on(16))
    return launch_rows<uint4>(p, p.x, p.ldx * es / 16, p.out, p.ldo * es / 16,
                              static_cast<int>(row / 16), sms, s);
  if (rows_on(4))
    return launch_rows<uint32_t>(p, p.x, p.ldx * es / 4, p.out, p.ldo * es / 4,
                                 static_cast<int>(row / 4), sms, s);
  return launch_rows<unsigned short>(p, p.x, p.ldx, p.out, p.ldo, p.d, sms, s);
}

cudaError_t launch_expert_combine(int dtype, const ExpertRowsArgs& p, bool backward, int sms,
                                  cudaStream_t s) {
  const int es = dtype == 0 ? 4 : 2;
  const int64_t row = int64_t{p.d} * es;  // bytes
  auto rows_on = [&](int bytes) {
    return row % bytes == 0 && on(bytes, p.x, p.ldx, es) && on(bytes, p.rows, p.ldr, es) &&
           on(bytes, p.out, p.ldo, es);
  };
  auto go = [&](auto combine, auto gradient) {
    return backward ? gradient(p, sms, s) : combine(p, sms, s);
  };
  using Bf = __nv_bfloat16;
  if (dtype == 0)
    return rows_on(16) ? go(launch_combine_rows<float, 16>, launch_combine_backward<float, 16>)
                       : go(launch_combine_rows<float, 4>, launch_combine_backward<float, 4>);
  return rows_on(16)  ? go(launch_combine_rows<Bf, 16>, launch_combine_backward<Bf, 16>)
         : rows_on(4) ? go(launch_combine_rows<Bf, 4>, launch_combine_backward<Bf, 4>)
                      : go(launch_combine_rows<Bf, 2>, launch_combine_backward<Bf, 2>);
}

}  // namespace rx
