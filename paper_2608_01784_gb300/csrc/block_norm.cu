// block_norm.cu — root-mean-square norms around a block, fused with the block's
// way back into the residual stream, and the gradients:
//   r(v) = 1 / sqrt(mean(v^2) + eps)
//   a = y r(y) w_after,  o = h + s g a,  n = o r(o) w_before
// (without w_after a = y, without a gate g = 1, without y o = h), and backward,
// with Do, Dn the gradients of o and n, v = Dn w_before, u = s O g w_after:
//   O  = Do + r(o) (v - o r(o)^2 mean(v o))          Dh = O
//   Dg = s O a                                       Dw_before = sum_t Dn o r(o)
//   Dy = r(y) (u - y r(y)^2 mean(u y))               Dw_after  = sum_t s O g y r(y)
// One pass: a row stays in the registers of the threads that share it, and two
// (backward: three) sums over the row are all that they exchange.  Everything
// between loads and stores is fp32; o is normalised before it is rounded, so n is
// rounded once, and the backward pass computes it again from h and y instead of
// reading the rounded o.  Bytes bound it: 4 rows of h's size forward, 6 backward.
#include "common.cuh"
#include "internal.h"

namespace rx {
namespace {

constexpr int kMaxThreads = 512;
constexpr int VE = 8;  // elements of a thread's vector
constexpr int kSharedCols = 128 * VE;  // of rows that share a CTA of 256 threads

// ---- a row shared by `tpr` threads -------------------------------------------
// Thread `lt` holds NV vectors: vectorised, vector v is elements (v tpr + lt) 8 ..
// + 7; element by element, its element i is (8 v + i) tpr + lt, so that a warp's
// accesses are consecutive either way.  A warp has one row or a part of one, or (up
// to 128 columns) several, which it walks together: past the last row, d is 0.
template <typename Te, bool VEC, int NV>
struct RowShare {
  int d, tpr, lt;
  __device__ __forceinline__ int col(int v, int i) const {
    return VEC ? (v * tpr + lt) * VE + i : (v * VE + i) * tpr + lt;
  }
};

// Elements as stored: rows that are fetched a turn ahead wait in this form.
template <typename Te, int NV>
struct alignas(16) Raw {
  Te e[NV * VE];
};

template <typename Te, bool VEC, int NV>
__device__ __forceinline__ void fetch(const RowShare<Te, VEC, NV>& s, const Te* row,
                                      Raw<Te, NV>& r) {
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if constexpr (VEC) {
      uint4* dst = reinterpret_cast<uint4*>(&r.e[v * VE]);
      const bool in = s.col(v, 0) < s.d;
#pragma unroll
      for (int q = 0; q < static_cast<int>(sizeof(Te) * VE / 16); ++q)
        dst[q] = in ? *(reinterpret_cast<const uint4*>(row + s.col(v, 0)) + q)
                    : make_uint4(0u, 0u, 0u, 0u);
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i)
        r.e[v * VE + i] = s.col(v, i) < s.d ? row[s.col(v, i)] : from_f32<Te>(0.f);
    }
  }
}

template <typename Te, bool VEC, int NV>
__device__ __forceinline__ void put(const RowShare<Te, VEC, NV>& s, Te* row, const float* f) {
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if constexpr (VEC) {
      if (s.col(v, 0) < s.d) store8(row + s.col(v, 0), f + v * VE);
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i)
        if (s.col(v, i) < s.d) row[s.col(v, i)] = from_f32<Te>(f[v * VE + i]);
    }
  }
}

// Sums of N values over the threads of a row, the same bits in all of them.  Warps
// leave their sums in one of two places in turn: a place is written again only after
// the barrier behind the next sum, which every thread reaches when it has read it.
template <int N>
__device__ __forceinline__ void row_sum(float (&x)[N], int tpr, int lt, int bar, float* place,
                                        int& turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < tpr)
#pragma unroll
      for (int n = 0; n < N; ++n) x[n] += __shfl_xor_sync(0xffffffffu, x[n], o);
  if (tpr <= 32) return;
  float* at = place + turn * 32;
  turn ^= 1;
  const int warps = tpr >> 5;
  if ((lt & 31) == 0)
#pragma unroll
    for (int n = 0; n < N; ++n) at[n * 16 + (lt >> 5)] = x[n];
  asm volatile("barrier.cta.sync %0, %1;" ::"r"(bar), "r"(tpr) : "memory");
#pragma unroll
  for (int n = 0; n < N; ++n) x[n] = 0.f;
  for (int w = 0; w < warps; ++w)
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] += at[n * 16 + w];
}

template <typename Te, bool VEC, int NV>
__global__ void __launch_bounds__(kMaxThreads)
    norm_kernel(const BlockNormArgs p) {
  constexpr int n = NV * VE;
  __shared__ float s_sum[kMaxThreads / 64][2 * 32];
  const int tpr = p.tpr, sub = threadIdx.x / tpr;
  RowShare<Te, VEC, NV> s{p.d, tpr, static_cast<int>(threadIdx.x) % tpr};
  float* place = s_sum[tpr > 32 ? sub : 0];
  int turn = 0;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (blockDim.x / tpr);
  int64_t t = static_cast<int64_t>(blockIdx.x) * (blockDim.x / tpr) + sub;
  const int in_warp = tpr < 32 ? static_cast<int>(threadIdx.x & 31) / tpr : 0;
  const Te* h = static_cast<const Te*>(p.h);
  const Te* y = static_cast<const Te*>(p.y);
  const Te* gate = static_cast<const Te*>(p.gate);
  const float inv_d = 1.f / static_cast<float>(p.d);
  grid_dep_wait();
  grid_dep_launch();
  Raw<Te, NV> wa, wb, g, hr, yr;
  if (p.w_after) fetch(s, static_cast<const Te*>(p.w_after), wa);
  if (p.w_before) fetch(s, static_cast<const Te*>(p.w_before), wb);
  if (gate && !p.ldg) fetch(s, gate, g);
  if (t >= p.rows) s.d = 0;
  fetch(s, h + t * p.ldh, hr);
  if (y) fetch(s, y + t * p.ldy, yr);
  for (; t - in_warp < p.rows; t += step) {
    if (gate && p.ldg) fetch(s, gate + t * p.ldg, g);
    float o[n];
#pragma unroll
    for (int i = 0; i < n; ++i) o[i] = to_f32(hr.e[i]);
    if (y) {
      float a[n];
      float ry = 1.f;
#pragma unroll
      for (int i = 0; i < n; ++i) a[i] = to_f32(yr.e[i]);
      if (p.w_after) {
        float q[1] = {0.f};
#pragma unroll
        for (int i = 0; i < n; ++i) q[0] = __fmaf_rn(a[i], a[i], q[0]);
        row_sum(q, tpr, s.lt, 1 + sub, place, turn);
        ry = rsqrtf(__fmaf_rn(q[0], inv_d, p.eps));
#pragma unroll
        for (int i = 0; i < n; ++i) a[i] = a[i] * ry * to_f32(wa.e[i]);
      }
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const float b = gate ? a[i] * to_f32(g.e[i]) : a[i];
        o[i] = __fmaf_rn(p.scale, b, o[i]);
      }
    }
    // the next row is on its way while this one is summed and stored
    const int64_t next = t + step;
    const RowShare<Te, VEC, NV> s_next{next < p.rows ? p.d : 0, tpr, s.lt};
    fetch(s_next, h + next * p.ldh, hr);
    if (y) fetch(s_next, y + next * p.ldy, yr);
    if (p.out) put(s, static_cast<Te*>(p.out) + t * p.ldo, o);
    if (p.w_before) {
      float q[1] = {0.f};
#pragma unroll
      for (int i = 0; i < n; ++i) q[0] = __fmaf_rn(o[i], o[i], q[0]);
      row_sum(q, tpr, s.lt, 1 + sub, place, turn);
      const float ro = rsqrtf(__fmaf_rn(q[0], inv_d, p.eps));
#pragma unroll
      for (int i = 0; i < n; ++i) o[i] = o[i] * ro * to_f32(wb.e[i]);
      put(s, static_cast<Te*>(p.norm) + t * p.ldn, o);
    }
    s.d = s_next.d;
  }
}

template <typename Te, bool VEC, int NV>
__global__ void __launch_bounds__(kMaxThreads)
    norm_backward_kernel(const BlockNormArgs p) {
  constexpr int n = NV * VE;
  __shared__ float s_sum[kMaxThreads / 64][2 * 32];
  __shared__ float s_cols[3][kSharedCols];
  const int tpr = p.tpr, sub = threadIdx.x / tpr;
  RowShare<Te, VEC, NV> s{p.d, tpr, static_cast<int>(threadIdx.x) % tpr};
  float* place = s_sum[tpr > 32 ? sub : 0];
  int turn = 0;
  const int in_warp = tpr < 32 ? static_cast<int>(threadIdx.x & 31) / tpr : 0;
  const int groups = blockDim.x / tpr;
  const int64_t step = static_cast<int64_t>(gridDim.x) * groups;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * groups + sub;
  const Te* h = static_cast<const Te*>(p.h);
  const Te* y = static_cast<const Te*>(p.y);
  const Te* gate = static_cast<const Te*>(p.gate);
  const float inv_d = 1.f / static_cast<float>(p.d);
  grid_dep_wait();
  grid_dep_launch();
  // this thread's columns of the weights' gradients, over all of its rows
  float sum_a[n], sum_g[n], sum_b[n];
#pragma unroll
  for (int i = 0; i < n; ++i) sum_a[i] = sum_g[i] = sum_b[i] = 0.f;
  Raw<Te, NV> wa, wb, g;
  if (p.w_after) fetch(s, static_cast<const Te*>(p.w_after), wa);
  if (p.w_before) fetch(s, static_cast<const Te*>(p.w_before), wb);
  if (gate && !p.ldg) fetch(s, gate, g);
  for (int64_t t = first; t - in_warp < p.rows; t += step) {
    if (t >= p.rows) s.d = 0;
    Raw<Te, NV> hr, yr, dor, dnr;
    fetch(s, h + t * p.ldh, hr);
    if (y) fetch(s, y + t * p.ldy, yr);
    if (p.d_out) fetch(s, static_cast<const Te*>(p.d_out) + t * p.ld_d_out, dor);
    if (p.w_before) fetch(s, static_cast<const Te*>(p.d_norm) + t * p.ld_d_norm, dnr);
    if (gate && p.ldg) fetch(s, gate + t * p.ldg, g);
    // o again, as the forward pass had it
    float ry = 1.f;
    if (p.w_after) {
      float q[1] = {0.f};
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const float f = to_f32(yr.e[i]);
        q[0] = __fmaf_rn(f, f, q[0]);
      }
      row_sum(q, tpr, s.lt, 1 + sub, place, turn);
      ry = rsqrtf(__fmaf_rn(q[0], inv_d, p.eps));
    }
    // O, from here on the gradient of o through both of its uses
    float grad[n];
#pragma unroll
    for (int i = 0; i < n; ++i) grad[i] = p.d_out ? to_f32(dor.e[i]) : 0.f;
    if (p.w_before) {
      float o[n], q[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < n; ++i) {
        o[i] = to_f32(hr.e[i]);
        if (y) {
          float a = to_f32(yr.e[i]);
          if (p.w_after) a = a * ry * to_f32(wa.e[i]);
          if (gate) a *= to_f32(g.e[i]);
          o[i] = __fmaf_rn(p.scale, a, o[i]);
        }
        q[0] = __fmaf_rn(o[i], o[i], q[0]);
        q[1] = __fmaf_rn(to_f32(dnr.e[i]) * to_f32(wb.e[i]), o[i], q[1]);
      }
      row_sum(q, tpr, s.lt, 1 + sub, place, turn);
      const float ro = rsqrtf(__fmaf_rn(q[0], inv_d, p.eps));
      const float m = q[1] * inv_d * ro * ro;
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const float dn = to_f32(dnr.e[i]);
        grad[i] = __fmaf_rn(ro, __fmaf_rn(-o[i], m, dn * to_f32(wb.e[i])), grad[i]);
        sum_b[i] = __fmaf_rn(dn, o[i] * ro, sum_b[i]);
      }
    }
    put(s, static_cast<Te*>(p.d_h) + t * p.ld_d_h, grad);
    if (!y) continue;
    float dg[n], q[1] = {0.f};
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float f = to_f32(yr.e[i]);
      const float hat = f * ry;
      const float w = p.w_after ? to_f32(wa.e[i]) : 1.f;
      float b = p.scale * grad[i];
      dg[i] = b * (hat * w);
      if (gate) b *= to_f32(g.e[i]);
      sum_a[i] = __fmaf_rn(b, hat, sum_a[i]);
      grad[i] = b * w;
      q[0] = __fmaf_rn(grad[i], f, q[0]);
    }
    if (gate && p.d_gate) {
      if (p.ldg) {
        put(s, static_cast<Te*>(p.d_gate) + t * p.ld_d_gate, dg);
      } else {
#pragma unroll
        for (int i = 0; i < n; ++i) sum_g[i] += dg[i];
      }
    }
    if (p.w_after) {
      row_sum(q, tpr, s.lt, 1 + sub, place, turn);
      const float m = q[0] * inv_d * ry * ry;
#pragma unroll
      for (int i = 0; i < n; ++i) grad[i] = ry * __fmaf_rn(-to_f32(yr.e[i]), m, grad[i]);
    }
    put(s, static_cast<Te*>(p.d_y) + t * p.ld_d_y, grad);
  }
  // [3][gridDim.x][d]: this CTA's sums, of one row after another in a thread, then of
  // the rows of a warp, then warp by warp
  s.d = p.d;
  const bool want[3] = {p.d_w_after != nullptr, p.d_gate != nullptr && !p.ldg,
                        p.d_w_before != nullptr};
  float* sums[3] = {sum_a, sum_g, sum_b};
  const int slots = tpr < 32 ? blockDim.x / 32 : groups;
  const int slot = tpr < 32 ? threadIdx.x / 32 : sub;
#pragma unroll
  for (int which = 0; which < 3; ++which) {
    if (!want[which]) continue;
    float* f = sums[which];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (o >= tpr)
#pragma unroll
        for (int i = 0; i < n; ++i) f[i] += __shfl_xor_sync(0xffffffffu, f[i], o);
    float* at = p.partial + (static_cast<int64_t>(which) * gridDim.x + blockIdx.x) * p.d;
    for (int turn_of = 0; turn_of < slots; ++turn_of) {
      if (turn_of > 0) __syncthreads();
      if (slot != turn_of || in_warp != 0) continue;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          const int c = s.col(v, i);
          if (c >= p.d) continue;
          float sum = f[v * VE + i];
          if (turn_of > 0) sum += s_cols[which][c];
          if (turn_of + 1 < slots) s_cols[which][c] = sum;
          else at[c] = sum;
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

// Threads that share a row: eight elements each, up to 512 threads.
int threads_per_row(int d) {
  int tpr = 1;
  while (tpr < kMaxThreads && tpr * VE < d) tpr *= 2;
  return tpr;
}
int block_threads(int tpr) { return tpr < 256 ? 256 : tpr; }
int64_t norm_grid(int64_t rows, int tpr, int per_sm, int sms) {
  const int groups = block_threads(tpr) / tpr;
  const int64_t need = (rows + groups - 1) / groups;
  const int64_t most = static_cast<int64_t>(sms) * per_sm;
  return need < most ? need : most;
}
// CTAs of 256 (512) threads an SM
int forward_ctas(int tpr) { return tpr <= 256 ? 8 : 4; }
int backward_ctas(int tpr) { return tpr <= 256 ? 4 : 2; }

template <typename Te, bool VEC, int NV>
cudaError_t launch_norm(const BlockNormArgs& p, bool backward, int sms, cudaStream_t s) {
  const int threads = block_threads(p.tpr);
  const int64_t grid =
      norm_grid(p.rows, p.tpr, backward ? backward_ctas(p.tpr) : forward_ctas(p.tpr), sms);
  if (backward)
    return launch_pdl(norm_backward_kernel<Te, VEC, NV>, dim3(static_cast<unsigned>(grid)),
                      dim3(threads), 0, s, p);
  return launch_pdl(norm_kernel<Te, VEC, NV>, dim3(static_cast<unsigned>(grid)), dim3(threads), 0,
                    s, p);
}
template <typename Te, bool VEC>
cudaError_t launch_norm_nv(const BlockNormArgs& p, bool backward, int sms, cudaStream_t s) {
  const int vecs = (p.d + p.tpr * VE - 1) / (p.tpr * VE);
  if (vecs <= 1) return launch_norm<Te, VEC, 1>(p, backward, sms, s);
  if (vecs <= 2) return launch_norm<Te, VEC, 2>(p, backward, sms, s);
  if (vecs <= 4) return launch_norm<Te, VEC, 4>(p, backward, sms, s);
  return cudaErrorInvalidValue;
}
template <typename Te>
cudaError_t launch_norm_typed(BlockNormArgs p, bool backward, int sms, cudaStream_t s) {
  constexpr int es = sizeof(Te);
  p.tpr = threads_per_row(p.d);
  bool vec = p.d % VE == 0;
  vec = vec && vector_rows(p.h, p.ldh, es) && vector_rows(p.y, p.ldy, es) &&
        vector_rows(p.gate, p.ldg, es) && vector_rows(p.w_after, 0, es) &&
        vector_rows(p.w_before, 0, es) && vector_rows(p.out, p.ldo, es) &&
        vector_rows(p.norm, p.ldn, es) && vector_rows(p.d_out, p.ld_d_out, es) &&
        vector_rows(p.d_norm, p.ld_d_norm, es) && vector_rows(p.d_h, p.ld_d_h, es) &&
        vector_rows(p.d_y, p.ld_d_y, es) && vector_rows(p.d_gate, p.ld_d_gate, es);
  int64_t parts = 0;
  if (p.rows > 0) {
    const cudaError_t e = vec ? launch_norm_nv<Te, true>(p, backward, sms, s)
                              : launch_norm_nv<Te, false>(p, backward, sms, s);
    if (e != cudaSuccess || !backward) return e;
    parts = block_norm_parts(p.rows, p.d, sms);
  }
  if (!backward) return cudaSuccess;
  Te* dg = p.ldg ? nullptr : static_cast<Te*>(p.d_gate);
  if (p.d_w_after == nullptr && dg == nullptr && p.d_w_before == nullptr) return cudaSuccess;
  return launch_pdl(norm_weights_kernel<Te>, dim3((p.d + 31) / 32, 3), dim3(32 * kSlices), 0, s,
                    static_cast<const float*>(p.partial), parts, p.d,
                    static_cast<Te*>(p.d_w_after), dg, static_cast<Te*>(p.d_w_before));
}

}  // namespace

int block_norm_max_width() { return kMaxThreads * VE * 4; }

int64_t block_norm_parts(int64_t rows, int d, int sms) {
  const int tpr = threads_per_row(d);
  return norm_grid(rows, tpr, backward_ctas(tpr), sms);
}

cudaError_t launch_block_norm(int dtype, const BlockNormArgs& p, bool backward, int sms,
                              cudaStream_t s) {
  return dtype == 0 ? launch_norm_typed<float>(p, backward, sms, s)
                    : launch_norm_typed<__nv_bfloat16>(p, backward, sms, s);
}

}  // namespace rx
