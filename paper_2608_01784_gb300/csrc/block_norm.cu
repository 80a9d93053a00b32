// block_norm.cu — root-mean-square norms around a block, fused with the block's
// way back into the residual stream, and the gradients:
//   r(v) = 1 / sqrt(mean(v^2) + eps)
//   a = y r(y) w_after,  o = h + s g a,  n = o r(o) w_before
// (without w_after a = y, without a gate g = 1, without y o = h), and backward,
// with Do, Dn the gradients of o and n, v = Dn w_before, u = s O g w_after:
//   O  = Do + r(o) (v - o r(o)^2 mean(v o))          Dh = O
//   Dg = s O a                                       Dw_before = sum_t Dn o r(o)
//   Dy = r(y) (u - y r(y)^2 mean(u y))               Dw_after  = sum_t s O g y r(y)
// (with one gate for all rows Dg = s w_after S and Dw_after = s g S, S = sum_t O y r(y)).
// One pass: a row stays in the registers of the threads that share it, and two
// (backward: three) sums over the row are all that they exchange.  Everything between
// loads and stores is fp32; o is normalised before it is rounded, so n is rounded once,
// and the backward pass computes it again from h and y instead of reading the rounded
// o.  Bytes bound it, 4 rows of h's size forward and 6 backward, as long as a row takes
// few instructions: with options and row sizes looked up for each row, 500 and 735
// instructions for 8 elements a thread outweighed the arithmetic and the bytes.
// 32768 x 2048 bf16, us: forward 149 -> 88 (6.1 TB/s), backward 263 -> 146 (5.5 TB/s, with
// 5 us for the weights' sums); fp32 6.0 to 6.5 TB/s both ways.  Odd widths of bf16, without
// vectors or copies ahead, reach 2.2 to 2.8 TB/s; rows wider than 4096 backward 1.5 to 3,
// because their sums leave the registers.
#include <type_traits>

#include "common.cuh"
#include "internal.h"

namespace rx {
namespace {

constexpr int kMaxThreads = 512;
constexpr int kMaxEach = 32;  // elements of a row in a thread
constexpr int kMaxWidth = kMaxThreads * kMaxEach;

// ---- pairs of fp32 in one register pair: one instruction for both ---------------
struct F2 {
  uint64_t v;
};
__device__ __forceinline__ F2 f2(uint32_t lo, uint32_t hi) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ F2 f2(float x) { return f2(__float_as_uint(x), __float_as_uint(x)); }
__device__ __forceinline__ float2 parts(F2 a) {
  uint32_t lo, hi;
  asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(a.v));
  return make_float2(__uint_as_float(lo), __uint_as_float(hi));
}
__device__ __forceinline__ float total(F2 a) {
  const float2 p = parts(a);
  return p.x + p.y;
}
__device__ __forceinline__ F2 mul(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 add(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

// ---- a row shared by `tpr` threads -------------------------------------------
// Thread `lt` holds N elements, 16-byte vectors or elements v tpr + lt of the row, so
// that a warp's accesses are consecutive.  A CTA has one row at a time (TPR threads, 64
// to 512), or (TPR == 0) each of its warps one row or several narrow ones, which the
// warp walks together: past the last row, d is 0.
template <typename Te, bool VEC>
struct RowShare {
  static constexpr int kUnit = VEC ? 16 / static_cast<int>(sizeof(Te)) : 1;
  int d, tpr, lt;
  __device__ __forceinline__ int col(int i) const {
    return (i / kUnit * tpr + lt) * kUnit + i % kUnit;
  }
};

// A thread's elements as stored; of two bytes, two to a word.
template <typename Te, int N>
struct Raw {
  static constexpr int kWords = N * static_cast<int>(sizeof(Te)) / 4;
  static constexpr int kVecs = kWords / 4;  // 16 bytes
  static constexpr int kPerVec = 16 / static_cast<int>(sizeof(Te));
  uint32_t w[kWords];
  __device__ __forceinline__ F2 pair(int i) const {  // elements 2 i, 2 i + 1
    if constexpr (sizeof(Te) == 4) return f2(w[2 * i], w[2 * i + 1]);
    return f2(w[i] << 16, w[i] & 0xffff0000u);
  }
};

// PLAIN: nothing in this kernel writes the row.
template <bool PLAIN, typename Te, bool VEC, int N>
__device__ __forceinline__ void fetch(const RowShare<Te, VEC>& s, const Te* row, Raw<Te, N>& r) {
  if constexpr (VEC) {
#pragma unroll
    for (int q = 0; q < Raw<Te, N>::kVecs; ++q) {
      const int c = s.col(q * Raw<Te, N>::kPerVec);
      const uint4* at = reinterpret_cast<const uint4*>(row + c);
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (c < s.d) x = PLAIN ? __ldg(at) : *at;
      r.w[4 * q] = x.x;
      r.w[4 * q + 1] = x.y;
      r.w[4 * q + 2] = x.z;
      r.w[4 * q + 3] = x.w;
    }
  } else if constexpr (sizeof(Te) == 4) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      r.w[i] = s.col(i) < s.d ? reinterpret_cast<const uint32_t*>(row)[s.col(i)] : 0u;
  } else {
    uint16_t e[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
      e[i] = s.col(i) < s.d ? reinterpret_cast<const uint16_t*>(row)[s.col(i)] : 0;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) r.w[i] = e[2 * i] | static_cast<uint32_t>(e[2 * i + 1]) << 16;
  }
}

template <typename Te, bool VEC, int N>
__device__ __forceinline__ void put(const RowShare<Te, VEC>& s, Te* row, const F2 (&x)[N / 2]) {
  if constexpr (VEC) {
#pragma unroll
    for (int v = 0; v < N / s.kUnit; ++v) {
      const int c = s.col(s.kUnit * v);
      if (c >= s.d) continue;
      float f[s.kUnit];
#pragma unroll
      for (int i = 0; i < s.kUnit / 2; ++i) {
        const float2 p = parts(x[s.kUnit / 2 * v + i]);
        f[2 * i] = p.x;
        f[2 * i + 1] = p.y;
      }
      if constexpr (sizeof(Te) == 2) store8(row + c, f);
      else *reinterpret_cast<float4*>(row + c) = make_float4(f[0], f[1], f[2], f[3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float2 p = parts(x[i]);
      if (s.col(2 * i) < s.d) row[s.col(2 * i)] = from_f32<Te>(p.x);
      if (s.col(2 * i + 1) < s.d) row[s.col(2 * i + 1)] = from_f32<Te>(p.y);
    }
  }
}

// Sums of K values over the threads of a row, the same bits in all of them: within
// warps, then warp by warp through shared memory.  Warps leave their sums in one of two
// places in turn: a place is written again only after the barrier behind the next sum,
// which every thread reaches when it has read it.
template <int TPR>
struct RowSum {
  static constexpr int kWarps = TPR / 32;
  static constexpr int kPlaces = TPR ? 2 * 2 * kWarps : 4;
  float* place;
  int tpr, turn;
  template <int K>
  __device__ __forceinline__ void operator()(float (&x)[K]) {
    if constexpr (TPR == 0) {
      for (int o = tpr >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int n = 0; n < K; ++n) x[n] += __shfl_xor_sync(0xffffffffu, x[n], o);
    } else {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int n = 0; n < K; ++n) x[n] += __shfl_xor_sync(0xffffffffu, x[n], o);
      float* at = place + turn * (2 * kWarps);
      turn ^= 1;
      if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int n = 0; n < K; ++n) at[n * kWarps + (threadIdx.x >> 5)] = x[n];
      __syncthreads();
#pragma unroll
      for (int n = 0; n < K; ++n) {
        if constexpr (kWarps == 2) {
          const float2 v = *reinterpret_cast<const float2*>(at + 2 * n);
          x[n] = v.x + v.y;
        } else {
          x[n] = 0.f;
#pragma unroll
          for (int q = 0; q < kWarps / 4; ++q) {
            const float4 v = *reinterpret_cast<const float4*>(at + n * kWarps + 4 * q);
            x[n] += (v.x + v.y) + (v.z + v.w);
          }
        }
      }
    }
  }
};

// Tensors that a row is made of.
__host__ __device__ constexpr int ring_tensors(bool backward, bool token_gate) {
  return (backward ? 4 : 2) + token_gate;
}
constexpr int cta_threads(int TPR) { return TPR ? TPR : 256; }

// The rows of one thread group, one after another; tensors by pointer (nullptr: not
// there).  Each thread copies its own elements into its own places of a ring of `depth`
// rows (16 bytes at a time, element by element 4) and reads them back itself, so
// nothing but its own copies has to be waited for.  Elements of two bytes cannot be
// copied that way, and two of the widest fp32 rows do not fit: they are loaded when the
// row's turn comes.
constexpr int kRingBytes = 200 * 1024;  // of an SM
template <typename Te, bool VEC, int N, int TPR, bool BACK, bool TGATE>
struct Rows {
  using R = Raw<Te, N>;
  using S = RowShare<Te, VEC>;
  static constexpr int kThreads = cta_threads(TPR);
  static constexpr int kCount = ring_tensors(BACK, TGATE);
  static constexpr int kRowBytes = R::kWords * 4 * kThreads;
  static constexpr bool kRing = (VEC || sizeof(Te) == 4) && 2 * kCount * kRowBytes <= kRingBytes;
  static constexpr int kCopies = VEC ? R::kVecs : R::kWords;
  static constexpr int kCopy = VEC ? 16 : 4;  // bytes
  const Te* p[kCount];  // h, y, (d_out, d_norm), (gate): the next row to ask for
  int64_t ld[kCount];   // from one of this group's rows to its next
  int64_t left;         // rows behind the next one to ask for
  int64_t step;
  int d, depth;
  uint32_t base, slot;  // this thread's first place; the one whose turn it is

  __device__ __forceinline__ void set(int i, const void* t, int64_t stride, int64_t first) {
    p[i] = t ? static_cast<const Te*>(t) + first * stride : nullptr;
    ld[i] = step * stride;
  }
  __device__ __forceinline__ void request(uint32_t to, const S& s) {
    const bool live = left > 0;
    if (TPR == 0 || live) {
#pragma unroll
      for (int i = 0; i < kCount; ++i) {
        if (p[i] == nullptr) continue;
#pragma unroll
        for (int q = 0; q < kCopies; ++q) {  // (zeros, and no read, where there is nothing)
          const int c = s.col(q * S::kUnit);
          const bool in = live && c < d;
          const uint32_t at = to + i * kRowBytes + q * kThreads * kCopy;
          const Te* from = p[i] + c;
          if constexpr (VEC)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(from),
                         "r"(in ? 16 : 0)
                         : "memory");
          else
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(at), "l"(from),
                         "r"(in ? 4 : 0)
                         : "memory");
        }
        p[i] += ld[i];
      }
      left -= step;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ __forceinline__ void start(const S& s, uint8_t* smem) {
    if constexpr (kRing) {
      base = slot = smem_addr(smem) + threadIdx.x * kCopy;
      for (int i = 0; i < depth - 1; ++i) request(base + i * kCount * kRowBytes, s);
    }
  }
  // the next row has arrived
  __device__ __forceinline__ void wait() const {
    if constexpr (kRing) {
      if (depth == 3) asm volatile("cp.async.wait_group 1;" ::: "memory");
      else asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
  }
  // its tensor i
  __device__ __forceinline__ void read(int i, const S& s, R& r) const {
    if constexpr (!kRing) {
      fetch<false>(s, p[i], r);
    } else if constexpr (VEC) {
#pragma unroll
      for (int q = 0; q < R::kVecs; ++q)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r.w[4 * q]), "=r"(r.w[4 * q + 1]), "=r"(r.w[4 * q + 2]),
                       "=r"(r.w[4 * q + 3])
                     : "r"(slot + i * kRowBytes + q * kThreads * 16)
                     : "memory");
    } else {
#pragma unroll
      for (int q = 0; q < R::kWords; ++q)
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r.w[q])
                     : "r"(slot + i * kRowBytes + q * kThreads * 4)
                     : "memory");
    }
  }
  // this row is in registers: asks for the one `depth` - 1 after it, in the place of the
  // one before it
  __device__ __forceinline__ void ask(const S& s) {
    if constexpr (kRing) {
      constexpr uint32_t kSlot = kCount * kRowBytes;
      const uint32_t last = base + (depth - 1) * kSlot;
      request(slot == base ? last : slot - kSlot, s);
      slot = slot == last ? base : slot + kSlot;
    } else {
#pragma unroll
      for (int i = 0; i < kCount; ++i)
        if (p[i] != nullptr) p[i] += ld[i];
    }
  }
  // copies past the last row (zeros) land before the CTA exits
  __device__ __forceinline__ void drain() const {
    if constexpr (kRing) asm volatile("cp.async.wait_all;" ::: "memory");
  }
};

// Where a thread stands.
template <typename Te, bool VEC, int TPR>
struct Place {
  RowShare<Te, VEC> s;
  RowSum<TPR> sum;
  int64_t first, step;
  int in_warp;  // which of the rows of its warp
  __device__ __forceinline__ Place(const BlockNormArgs& p, float* s_sum) {
    const int tpr = TPR ? TPR : p.tpr;
    const int groups = cta_threads(TPR) / tpr, sub = threadIdx.x / tpr;
    s = RowShare<Te, VEC>{p.d, tpr, static_cast<int>(threadIdx.x) % tpr};
    sum = RowSum<TPR>{s_sum, tpr, 0};
    step = static_cast<int64_t>(gridDim.x) * groups;
    first = static_cast<int64_t>(blockIdx.x) * groups + sub;
    in_warp = TPR ? 0 : static_cast<int>(threadIdx.x & 31) / tpr;
  }
};

// A weight's share of a thread: in registers for all rows where there is room, else
// fetched (from L1) for each.
template <typename Te, bool VEC, int N>
struct Weight {
  static constexpr bool kKeep = N <= 8;
  const Te* w;
  F2 v[kKeep ? N / 2 : 1];
  Raw<Te, kKeep ? 8 : N> raw;
  __device__ __forceinline__ Weight(const void* p, const RowShare<Te, VEC>& s)
      : w(static_cast<const Te*>(p)) {
    if constexpr (kKeep) {
      if (w == nullptr) return;
      Raw<Te, N> r;
      fetch<true>(s, w, r);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) v[i] = r.pair(i);
    }
  }
  __device__ __forceinline__ explicit operator bool() const { return w != nullptr; }
  __device__ __forceinline__ void get(const RowShare<Te, VEC>& s) {
    if constexpr (!kKeep) fetch<true>(s, w, raw);
  }
  __device__ __forceinline__ F2 pair(int i) const {
    if constexpr (kKeep) return v[i];
    else return raw.pair(i);
  }
};

// scale * w_after * gate by columns, 1 for what is not there.
template <typename Te, bool VEC, int N>
struct Factor {
  Weight<Te, VEC, N> w, g;
  float scale;
  __device__ __forceinline__ Factor(const void* pw, const void* pg, float sc,
                                    const RowShare<Te, VEC>& s)
      : w(pw, s), g(pg, s), scale(sc) {
    if constexpr (Weight<Te, VEC, N>::kKeep) {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) w.v[i] = product(i);
    }
  }
  __device__ __forceinline__ F2 product(int i) const {
    F2 c = f2(scale);
    if (w) c = mul(c, w.pair(i));
    if (g) c = mul(c, g.pair(i));
    return c;
  }
  __device__ __forceinline__ void get(const RowShare<Te, VEC>& s) {
    if (w) w.get(s);
    if (g) g.get(s);
  }
  __device__ __forceinline__ F2 pair(int i) const {
    if constexpr (Weight<Te, VEC, N>::kKeep) return w.v[i];
    else return product(i);
  }
};

template <typename Te, bool VEC, int N, int TPR, bool TGATE>
__global__ void __launch_bounds__(cta_threads(TPR), 512 / cta_threads(TPR))
    norm_kernel(const BlockNormArgs p) {
  extern __shared__ __align__(16) uint8_t s_ring[];
  __shared__ __align__(16) float s_sum[RowSum<TPR>::kPlaces];
  Place<Te, VEC, TPR> at(p, s_sum);
  RowShare<Te, VEC>& s = at.s;
  const float inv_d = 1.f / static_cast<float>(p.d);
  const F2 scale = f2(p.scale);
  Rows<Te, VEC, N, TPR, false, TGATE> in{};
  in.step = at.step;
  in.left = p.rows - at.first;
  in.d = p.d;
  in.depth = p.depth;
  in.set(0, p.h, p.ldh, at.first);
  in.set(1, p.y, p.ldy, at.first);
  if (TGATE) in.set(in.kCount - 1, p.gate, p.ldg, at.first);
  grid_dep_wait();
  grid_dep_launch();
  in.start(s, s_ring);
  Weight<Te, VEC, N> w_after(p.w_after, s), w_before(p.w_before, s), gate(TGATE ? nullptr : p.gate, s);
  for (int64_t t = at.first; t - at.in_warp < p.rows; t += at.step) {
    if (TPR == 0 && t >= p.rows) s.d = 0;
    in.wait();
    F2 o[N / 2];
    if (p.y) {
      Raw<Te, N> y;
      in.read(1, s, y);
      F2 ry = f2(1.f);
      if (w_after) {
        F2 q2 = f2(0.f);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) q2 = fma(y.pair(i), y.pair(i), q2);
        float q[1] = {total(q2)};
        w_after.get(s);
        at.sum(q);
        ry = f2(rsqrtf(__fmaf_rn(q[0], inv_d, p.eps)));
      }
#pragma unroll
      for (int i = 0; i < N / 2; ++i) o[i] = y.pair(i);
      if (w_after)
#pragma unroll
        for (int i = 0; i < N / 2; ++i) o[i] = mul(mul(o[i], ry), w_after.pair(i));
      if (TGATE) {
        Raw<Te, N> g;
        in.read(in.kCount - 1, s, g);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) o[i] = mul(o[i], g.pair(i));
      } else if (gate) {
        gate.get(s);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) o[i] = mul(o[i], gate.pair(i));
      }
      Raw<Te, N> h;
      in.read(0, s, h);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) o[i] = fma(scale, o[i], h.pair(i));
    } else {
      Raw<Te, N> h;
      in.read(0, s, h);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) o[i] = h.pair(i);
    }
    in.ask(s);
    if (p.out) put<Te, VEC, N>(s, static_cast<Te*>(p.out) + t * p.ldo, o);
    if (w_before) {
      F2 q2 = f2(0.f);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) q2 = fma(o[i], o[i], q2);
      float q[1] = {total(q2)};
      w_before.get(s);
      at.sum(q);
      const F2 ro = f2(rsqrtf(__fmaf_rn(q[0], inv_d, p.eps)));
#pragma unroll
      for (int i = 0; i < N / 2; ++i) o[i] = mul(mul(o[i], ro), w_before.pair(i));
      put<Te, VEC, N>(s, static_cast<Te*>(p.norm) + t * p.ldn, o);
    }
  }
  in.drain();
}

template <typename Te, bool VEC, int N, int TPR, bool TGATE>
__global__ void __launch_bounds__(cta_threads(TPR), 512 / cta_threads(TPR))
    norm_backward_kernel(const BlockNormArgs p) {
  extern __shared__ __align__(16) uint8_t s_ring[];
  __shared__ __align__(16) float s_sum[RowSum<TPR>::kPlaces];
  __shared__ float s_cols[TPR ? 1 : 32 * N];  // columns of rows that a warp holds
  Place<Te, VEC, TPR> at(p, s_sum);
  RowShare<Te, VEC>& s = at.s;
  const float inv_d = 1.f / static_cast<float>(p.d);
  Rows<Te, VEC, N, TPR, true, TGATE> in{};
  in.step = at.step;
  in.left = p.rows - at.first;
  in.d = p.d;
  in.depth = p.depth;
  in.set(0, p.w_before ? p.h : nullptr, p.ldh, at.first);  // (else not needed)
  in.set(1, p.y, p.ldy, at.first);
  in.set(2, p.d_out, p.ld_d_out, at.first);
  in.set(3, p.d_norm, p.ld_d_norm, at.first);
  if (TGATE) in.set(in.kCount - 1, p.gate, p.ldg, at.first);
  grid_dep_wait();
  grid_dep_launch();
  in.start(s, s_ring);
  Weight<Te, VEC, N> w_before(p.w_before, s);
  Factor<Te, VEC, N> factor(p.w_after, TGATE ? nullptr : p.gate, p.scale, s);
  // this thread's columns of the weights' gradients, over all of its rows
  F2 sum_a[N / 2], sum_b[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) sum_a[i] = sum_b[i] = f2(0.f);
  for (int64_t t = at.first; t - at.in_warp < p.rows; t += at.step) {
    // a row of zeros behind the last one stays out of the sums: with eps = 0 its r is infinite
    const bool live = TPR != 0 || t < p.rows;
    if (!live) s.d = 0;
    in.wait();
    Raw<Te, N> y_raw, g;
    F2 y[N / 2];  // y r(y)
    float ry = 1.f;
    if (p.y) {
      in.read(1, s, y_raw);
      if (TGATE) in.read(in.kCount - 1, s, g);
      factor.get(s);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) y[i] = y_raw.pair(i);
      if (p.w_after) {
        F2 q2 = f2(0.f);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) q2 = fma(y[i], y[i], q2);
        float q[1] = {total(q2)};
        at.sum(q);
        ry = live ? rsqrtf(__fmaf_rn(q[0], inv_d, p.eps)) : 0.f;
        const F2 r = f2(ry);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) y[i] = mul(y[i], r);
      }
    }
    // O, the gradient of o through both of its uses
    F2 grad[N / 2];
    if (w_before) {
      F2 qo = f2(0.f), qv = f2(0.f);
      Raw<Te, N> dn;
      in.read(3, s, dn);
      w_before.get(s);
      {
        Raw<Te, N> h;
        in.read(0, s, h);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          F2 o = h.pair(i);
          if (p.y) o = fma(y[i], TGATE ? mul(factor.pair(i), g.pair(i)) : factor.pair(i), o);
          qo = fma(o, o, qo);
          qv = fma(mul(dn.pair(i), w_before.pair(i)), o, qv);
          grad[i] = o;
        }
      }
      float q[2] = {total(qo), total(qv)};
      at.sum(q);
      const float ro1 = live ? rsqrtf(__fmaf_rn(q[0], inv_d, p.eps)) : 0.f;
      const F2 ro = f2(ro1), m = f2(-(q[1] * inv_d * ro1 * ro1));
      Raw<Te, N> d_out;
      if (p.d_out) in.read(2, s, d_out);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const F2 o = grad[i], dn2 = dn.pair(i);
        sum_b[i] = fma(dn2, mul(o, ro), sum_b[i]);
        grad[i] = fma(ro, fma(o, m, mul(dn2, w_before.pair(i))),
                      p.d_out ? d_out.pair(i) : f2(0.f));
      }
    } else {
      Raw<Te, N> d_out;
      in.read(2, s, d_out);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) grad[i] = d_out.pair(i);
    }
    in.ask(s);
    put<Te, VEC, N>(s, static_cast<Te*>(p.d_h) + t * p.ld_d_h, grad);
    if (!p.y) continue;
    F2 q2 = f2(0.f), dg[TGATE ? N / 2 : 1];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      F2 u = mul(grad[i], factor.pair(i));
      if (TGATE) {
        dg[i] = mul(u, y[i]);
        u = mul(u, g.pair(i));
        sum_a[i] = fma(mul(grad[i], g.pair(i)), y[i], sum_a[i]);
      } else {
        sum_a[i] = fma(grad[i], y[i], sum_a[i]);
      }
      grad[i] = u;
      q2 = fma(u, y[i], q2);
    }
    if constexpr (TGATE)
      if (p.d_gate) put<Te, VEC, N>(s, static_cast<Te*>(p.d_gate) + t * p.ld_d_gate, dg);
    if (p.w_after) {
      float q[1] = {total(q2)};
      at.sum(q);
      const F2 r = f2(ry), m = f2(-(q[0] * inv_d));
#pragma unroll
      for (int i = 0; i < N / 2; ++i) grad[i] = mul(r, fma(y[i], m, grad[i]));
    }
    put<Te, VEC, N>(s, static_cast<Te*>(p.d_y) + t * p.ld_d_y, grad);
  }
  in.drain();
  // [3][gridDim.x][d]: this CTA's sums, of one row after another in a thread, then of
  // the rows of a warp, then warp by warp
  const bool want[3] = {p.d_w_after != nullptr, p.d_gate != nullptr && !TGATE,
                        p.d_w_before != nullptr};
  constexpr int kSlots = TPR ? 1 : cta_threads(TPR) / 32;
  const int slot = TPR ? 0 : threadIdx.x / 32;
  s.d = p.d;
#pragma unroll
  for (int which = 0; which < 3; ++which) {
    if (!want[which]) continue;
    // what the sum is multiplied by: scale and the other one of gate and w_after
    Factor<Te, VEC, N> rest(which == 1 ? p.w_after : nullptr,
                            which == 0 && !TGATE ? p.gate : nullptr, p.scale, s);
    rest.get(s);
    float f[N];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float2 x2 = parts(which == 2 ? sum_b[i] : mul(sum_a[i], rest.pair(i)));
      f[2 * i] = x2.x;
      f[2 * i + 1] = x2.y;
    }
    if constexpr (TPR == 0)
      for (int o = 16; o >= p.tpr; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] += __shfl_xor_sync(0xffffffffu, f[i], o);
    float* to = p.partial + (static_cast<int64_t>(which) * gridDim.x + blockIdx.x) * p.d;
    for (int turn = 0; turn < kSlots; ++turn) {
      if (TPR == 0) __syncthreads();
      if (slot != turn || at.in_warp != 0) continue;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = s.col(i);
        if (c >= p.d) continue;
        float v = f[i];
        if (turn > 0) v += s_cols[TPR ? 0 : c];
        if (turn + 1 < kSlots) s_cols[TPR ? 0 : c] = v;
        else to[c] = v;
      }
    }
  }
}

// The weights' gradients: column sums of the parts, in their order, eight slices of
// them to a CTA and the slices one after another.
constexpr int kSlices = 8;
template <typename Te>
__global__ void __launch_bounds__(32 * kSlices)
    norm_weights_kernel(const float* __restrict__ partial, int64_t parts, int d, Te* d_w_after,
                        Te* d_gate, Te* d_w_before) {
  __shared__ float s_part[kSlices][32];
  Te* out = blockIdx.y == 0 ? d_w_after : blockIdx.y == 1 ? d_gate : d_w_before;
  grid_dep_wait();
  grid_dep_launch();
  if (out == nullptr) return;
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  const int64_t per = (parts + kSlices - 1) / kSlices;
  const int64_t lo = slice * per, hi = lo + per < parts ? lo + per : parts;
  float sum = 0.f;
  if (c < d) {
    const float* at = partial + blockIdx.y * parts * d + c;
#pragma unroll 8
    for (int64_t i = lo; i < hi; ++i) sum += at[i * d];
  }
  s_part[slice][lane] = sum;
  __syncthreads();
  if (slice == 0 && c < d) {
    for (int i = 1; i < kSlices; ++i) sum += s_part[i][lane];
    out[c] = from_f32<Te>(sum);
  }
}

bool vector_rows(const void* p, int64_t ld, int es) {
  return p == nullptr || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * es % 16 == 0);
}

// Threads that share a row of d elements, `each` of them a thread.
int threads_per_row(int d, int each) {
  int tpr = 1;
  while (tpr < kMaxThreads && tpr * each < d) tpr *= 2;
  return tpr;
}
// Elements of a thread: forward 64 bytes of vectors, of which addresses and sums are a
// small part; backward and element by element 8, because more of them (with the sums of
// three weights' gradients) leave the registers.  More in rows that 512 threads do not
// hold otherwise.
constexpr int elements_first(bool backward, bool vec, int es) {
  return backward || !vec ? 8 : 64 / es;
}
int elements_each(int d, int each) {
  while (each * kMaxThreads < d) each *= 2;
  return each;
}
int cta_of(int tpr) { return tpr <= 32 ? 256 : tpr; }
int64_t norm_grid(int64_t rows, int tpr, int per_sm, int sms) {
  const int groups = cta_of(tpr) / tpr;
  const int64_t need = (rows + groups - 1) / groups;
  const int64_t most = static_cast<int64_t>(sms) * per_sm;
  return need < most ? need : most;
}
// CTAs of an SM that registers leave room for (as the launch bounds ask for)
int ctas_of_sm(int tpr) { return 512 / cta_of(tpr); }

template <typename Te, bool VEC, int N, int TPR, bool BACK, bool TGATE>
cudaError_t launch_norm(BlockNormArgs p, int sms, cudaStream_t s, int64_t* grid) {
  using In = Rows<Te, VEC, N, TPR, BACK, TGATE>;
  constexpr int kThreads = cta_threads(TPR);
  int per_sm = 512 / kThreads;
  size_t smem = 0;
  if (In::kRing) {
    constexpr size_t kRow = static_cast<size_t>(In::kCount) * In::kRowBytes;
    if (2 * kRow * per_sm > kRingBytes) per_sm = kRingBytes / (2 * kRow);
    p.depth = 3 * kRow * per_sm <= kRingBytes ? 3 : 2;
    smem = kRow * p.depth;
  }
  void (*kernel)(const BlockNormArgs);
  if constexpr (BACK) kernel = norm_backward_kernel<Te, VEC, N, TPR, TGATE>;
  else kernel = norm_kernel<Te, VEC, N, TPR, TGATE>;
  if (smem > 32 * 1024) {
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = allow_smem(kernel, kRingBytes, done);
    if (e != cudaSuccess) return e;
  }
  *grid = norm_grid(p.rows, p.tpr, per_sm, sms);
  return launch_pdl(kernel, dim3(static_cast<unsigned>(*grid)), dim3(kThreads), smem, s, p);
}
template <typename Te, bool VEC, int N, bool BACK, bool TGATE>
cudaError_t launch_norm_threads(const BlockNormArgs& p, int sms, cudaStream_t s, int64_t* grid) {
  switch (p.tpr) {
    case 64: return launch_norm<Te, VEC, N, 64, BACK, TGATE>(p, sms, s, grid);
    case 128: return launch_norm<Te, VEC, N, 128, BACK, TGATE>(p, sms, s, grid);
    case 256: return launch_norm<Te, VEC, N, 256, BACK, TGATE>(p, sms, s, grid);
    case 512: return launch_norm<Te, VEC, N, 512, BACK, TGATE>(p, sms, s, grid);
    default: return launch_norm<Te, VEC, N, 0, BACK, TGATE>(p, sms, s, grid);
  }
}
template <typename Te, bool VEC, bool BACK, bool TGATE>
cudaError_t launch_norm_each(BlockNormArgs p, int sms, cudaStream_t s, int64_t* grid) {
  constexpr int kFirst = elements_first(BACK, VEC, sizeof(Te));
  const int each = elements_each(p.d, kFirst);
  p.tpr = threads_per_row(p.d, each);
  if (each == kFirst) return launch_norm_threads<Te, VEC, kFirst, BACK, TGATE>(p, sms, s, grid);
  if constexpr (kFirst < 16)
    if (each == 16) return launch_norm<Te, VEC, 16, 512, BACK, TGATE>(p, sms, s, grid);
  return launch_norm<Te, VEC, 32, 512, BACK, TGATE>(p, sms, s, grid);
}
template <typename Te, bool VEC, bool TGATE>
cudaError_t launch_norm_way(const BlockNormArgs& p, bool backward, int sms, cudaStream_t s,
                            int64_t* grid) {
  return backward ? launch_norm_each<Te, VEC, true, TGATE>(p, sms, s, grid)
                  : launch_norm_each<Te, VEC, false, TGATE>(p, sms, s, grid);
}
template <typename Te>
cudaError_t launch_norm_typed(BlockNormArgs p, bool backward, int sms, cudaStream_t s) {
  constexpr int es = sizeof(Te);
  bool vec = p.d % (16 / es) == 0;
  vec = vec && vector_rows(p.h, p.ldh, es) && vector_rows(p.y, p.ldy, es) &&
        vector_rows(p.gate, p.ldg, es) && vector_rows(p.w_after, 0, es) &&
        vector_rows(p.w_before, 0, es) && vector_rows(p.out, p.ldo, es) &&
        vector_rows(p.norm, p.ldn, es) && vector_rows(p.d_out, p.ld_d_out, es) &&
        vector_rows(p.d_norm, p.ld_d_norm, es) && vector_rows(p.d_h, p.ld_d_h, es) &&
        vector_rows(p.d_y, p.ld_d_y, es) && vector_rows(p.d_gate, p.ld_d_gate, es);
  int64_t parts = 0;  // CTAs that leave sums
  if (p.rows > 0) {
    cudaError_t e;
    if (p.ldg)
      e = vec ? launch_norm_way<Te, true, true>(p, backward, sms, s, &parts)
              : launch_norm_way<Te, false, true>(p, backward, sms, s, &parts);
    else
      e = vec ? launch_norm_way<Te, true, false>(p, backward, sms, s, &parts)
              : launch_norm_way<Te, false, false>(p, backward, sms, s, &parts);
    if (e != cudaSuccess || !backward) return e;
  }
  if (!backward) return cudaSuccess;
  Te* dg = p.ldg ? nullptr : static_cast<Te*>(p.d_gate);
  if (p.d_w_after == nullptr && dg == nullptr && p.d_w_before == nullptr) return cudaSuccess;
  return launch_pdl(norm_weights_kernel<Te>, dim3((p.d + 31) / 32, 3), dim3(32 * kSlices), 0, s,
                    static_cast<const float*>(p.partial), parts, p.d,
                    static_cast<Te*>(p.d_w_after), dg, static_cast<Te*>(p.d_w_before));
}

}  // namespace

int block_norm_max_width() { return kMaxWidth; }

int64_t block_norm_parts(int64_t rows, int d, int sms) {
  const int tpr = threads_per_row(d, elements_each(d, elements_first(true, true, 4)));
  return norm_grid(rows, tpr, ctas_of_sm(tpr), sms);
}

cudaError_t launch_block_norm(int dtype, const BlockNormArgs& p, bool backward, int sms,
                              cudaStream_t s) {
  return dtype == 0 ? launch_norm_typed<float>(p, backward, sms, s)
                    : launch_norm_typed<__nv_bfloat16>(p, backward, sms, s);
}

}  // namespace rx
