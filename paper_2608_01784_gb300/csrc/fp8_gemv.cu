// fp8_gemv.cu — 8-bit products of a few rows without the tensor cores: the dense
// layer of reflex_linear_fp8 for one to four rows in one launch, and the routed
// experts of reflex_experts_fp8 for a few pairs in two.
//
// Bound: the weights' bytes (65536 x 2048, one row: 25 us, 80 % of the measured
// copy rate) and, when they are few, launches and trips to HBM (4096 x 2048: 4.8 us,
// of which the bytes take 1.2, 3.7 with the weights in L2; twelve experts of 1024 for
// one token 25 us, 11).  Times are of replayed graphs.
// A warp takes four rows of the weights (experts: eight) at a time and 512 columns a
// step, 16 bytes of each row a lane, two steps in flight, and the rows of x are read
// from shared memory once for all of them.  Every CTA quantises its rows of x by
// itself (the codes of reflex_quantize_fp8 bit for bit): a launch more would take
// longer.  The 16 products of a lane lie in one block of K: the codes' products are
// summed in fp32 and scaled once by both scales, as the tiles do (a scale folded into
// x first would overflow for rows above 1e34), and the lanes' sums added at the end.
#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"

namespace rx {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kRows = 4;      // rows of W a warp has at work
constexpr int kChunk = 512;   // columns of a step
constexpr int kAhead = 2;     // steps whose loads are in flight

__device__ __forceinline__ float2 e4m3x2(uint32_t two) {
  const __half2_raw h =
      __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ void fma2(float2& acc, float2 a, float2 b) {
  uint64_t* d = reinterpret_cast<uint64_t*>(&acc);
  asm("fma.rn.f32x2 %0, %1, %2, %0;"
      : "+l"(*d)
      : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
}

// A row of x in shared memory: its codes as fp32, and behind them the scales of its
// blocks.  Element k: a lane's 16 columns as four vectors, each vector of all lanes in
// a row, so that no two lanes share a bank.
__host__ __device__ constexpr int row_floats(int chunks) { return chunks * (kChunk + kChunk / 128); }
__device__ __forceinline__ int place(int k) {
  return (k >> 9) * kChunk + ((k >> 2) & 3) * 128 + ((k >> 4) & 31) * 4 + (k & 3);
}

// 256 columns of a row (8 a lane, from c on) to codes and scales, 16 lanes a group of
// 128 as in the quantisation kernel.
template <typename Te>
__device__ __forceinline__ void quantise_pair(const Te* row, int c, int K, float* xs, int chunks) {
  float f[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    f[i] = c + i < K ? to_f32(row[c + i]) : 0.f;
    top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  const float a = fp8_amax(top), inv = fp8_inverse(a);
  if (c % 128 == 0) xs[chunks * kChunk + c / 128] = __fdiv_rn(a, kE4m3Max);
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const uint32_t q = e4m3x4(f[i] * inv, f[i + 1] * inv, f[i + 2] * inv, f[i + 3] * inv);
    const float2 lo = e4m3x2(q & 0xffffu), hi = e4m3x2(q >> 16);
    *reinterpret_cast<float4*>(xs + place(c + i)) = make_float4(lo.x, lo.y, hi.x, hi.y);
  }
}

template <typename Te, int M>
__global__ void __launch_bounds__(kThreads)
    linear_rows_kernel(const Te* __restrict__ x, int64_t ldx, const uint8_t* __restrict__ w,
                       int64_t ldw, const float* __restrict__ w_scales, int64_t ldws, int N,
                       int K, int out_f32, void* __restrict__ out, int64_t ldo, ZeroWords zero) {
  extern __shared__ __align__(16) float xs[];  // [M][row_floats(chunks)]
  grid_dep_wait();
  grid_dep_launch();
  if (blockIdx.x == 0) clear_words(zero);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int chunks = (K + kChunk - 1) / kChunk, ld = row_floats(chunks);
  const int pairs = chunks * kChunk / 256;
  for (int u = warp; u < M * pairs; u += kWarps) {
    const int m = u / pairs;
    quantise_pair(x + m * ldx, (u - m * pairs) * 256 + lane * 8, K, xs + m * ld, chunks);
  }
  __syncthreads();

  const int groups = (N + kRows - 1) / kRows, step = gridDim.x * kWarps;
  for (int g = blockIdx.x * kWarps + warp; g < groups; g += step) {
    const int n0 = g * kRows;
    const uint8_t* rows[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
      rows[r] = w + static_cast<int64_t>(min(n0 + r, N - 1)) * ldw + lane * 16;
    const float* sc = w_scales + (n0 >> 7) * ldws + (lane >> 3);
    float acc[kRows][M] = {};
    for (int c0 = 0; c0 < chunks; c0 += kAhead) {
      uint4 q[kAhead][kRows];
      float s[kAhead];
#pragma unroll
      for (int d = 0; d < kAhead; ++d) {
        const int k = (c0 + d) * kChunk + lane * 16;
        s[d] = 0.f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) q[d][r] = make_uint4(0u, 0u, 0u, 0u);
        if (k + 16 <= K) {
          s[d] = sc[(c0 + d) * (kChunk / 128)];
#pragma unroll
          for (int r = 0; r < kRows; ++r)
            q[d][r] = __ldcs(reinterpret_cast<const uint4*>(rows[r] + (c0 + d) * kChunk));
        } else if (k < K) {  // the row's end: what follows it is not its own
          s[d] = sc[(c0 + d) * (kChunk / 128)];
#pragma unroll
          for (int r = 0; r < kRows; ++r) {
            uint32_t v[4] = {};
            for (int i = 0; i < K - k; ++i)
              v[i >> 2] |= static_cast<uint32_t>(rows[r][(c0 + d) * kChunk + i]) << (8 * (i & 3));
            q[d][r] = make_uint4(v[0], v[1], v[2], v[3]);
          }
        }
      }
#pragma unroll
      for (int d = 0; d < kAhead; ++d) {
        if (c0 + d >= chunks) break;
        float2 sum[kRows][M] = {};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float4 xv[M];
#pragma unroll
          for (int m = 0; m < M; ++m)
            xv[m] = *reinterpret_cast<const float4*>(xs + m * ld + (c0 + d) * kChunk + j * 128 +
                                                     lane * 4);
#pragma unroll
          for (int r = 0; r < kRows; ++r) {
            const uint32_t word = j == 0 ? q[d][r].x : j == 1 ? q[d][r].y
                                          : j == 2 ? q[d][r].z : q[d][r].w;
            const float2 lo = e4m3x2(word & 0xffffu), hi = e4m3x2(word >> 16);
#pragma unroll
            for (int m = 0; m < M; ++m) {
              fma2(sum[r][m], lo, make_float2(xv[m].x, xv[m].y));
              fma2(sum[r][m], hi, make_float2(xv[m].z, xv[m].w));
            }
          }
        }
        const float* sx = xs + chunks * kChunk + (c0 + d) * (kChunk / 128) + (lane >> 3);
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const float both = s[d] * sx[m * ld];
#pragma unroll
          for (int r = 0; r < kRows; ++r)
            acc[r][m] = fmaf(sum[r][m].x + sum[r][m].y, both, acc[r][m]);
        }
      }
    }
    float mine = 0.f;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int m = 0; m < M; ++m) {
        float v = acc[r][m];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == r * M + m) mine = v;
      }
    const int n = n0 + lane / M, m = lane % M;
    if (lane < kRows * M && n < N) {
      if (out_f32) static_cast<float*>(out)[m * ldo + n] = mine;
      else static_cast<__nv_bfloat16*>(out)[m * ldo + n] = __float2bfloat16_rn(mine);
    }
  }
}

// ---- routed experts, few pairs ------------------------------------------------
// kAhead steps of R rows of a matrix, K a multiple of 16: their loads, then their
// products with xs.
template <int R>
struct Steps {
  uint4 q[kAhead][R];
  float s[kAhead][R / 4];  // scales of the first rows of each four (blocks of 128)
};
template <int R>
__device__ __forceinline__ void load_steps(Steps<R>& v, const uint8_t* const (&rows)[R],
                                           const float* const (&sc)[R / 4], int c0, int K) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int a = 0; a < kAhead; ++a) {
    const bool in = (c0 + a) * kChunk + lane * 16 < K;
#pragma unroll
    for (int g = 0; g < R / 4; ++g) v.s[a][g] = in ? sc[g][(c0 + a) * (kChunk / 128)] : 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
      v.q[a][r] = in ? __ldcs(reinterpret_cast<const uint4*>(rows[r] + (c0 + a) * kChunk))
                     : make_uint4(0u, 0u, 0u, 0u);
  }
}
template <int R>
__device__ __forceinline__ void add_steps(const Steps<R>& v, const float* xs, int c0, int chunks,
                                          float (&acc)[R]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int a = 0; a < kAhead; ++a) {
    if (c0 + a >= chunks) break;
    float2 sum[R] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 x =
          *reinterpret_cast<const float4*>(xs + (c0 + a) * kChunk + j * 128 + lane * 4);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const uint4& q = v.q[a][r];
        const uint32_t word = j == 0 ? q.x : j == 1 ? q.y : j == 2 ? q.z : q.w;
        fma2(sum[r], e4m3x2(word & 0xffffu), make_float2(x.x, x.y));
        fma2(sum[r], e4m3x2(word >> 16), make_float2(x.z, x.w));
      }
    }
    const float sx = xs[chunks * kChunk + (c0 + a) * (kChunk / 128) + (lane >> 3)];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = fmaf(sum[r].x + sum[r].y, v.s[a][r / 4] * sx, acc[r]);
  }
}
template <int R>
__device__ __forceinline__ void sum_lanes(float (&acc)[R]) {
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], o);
}

// act of one slot (token, j): a warp takes four columns (four gate and four up rows).
// Every CTA quantises its token.
__global__ void __launch_bounds__(kThreads) experts_up_rows_kernel(const Fp8ExpertsRows p) {
  extern __shared__ __align__(16) float xs[];
  grid_dep_wait();
  grid_dep_launch();
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    clear_words(p.zero);
    __syncthreads();
    for (int i = threadIdx.x; i < p.T * p.k_max; i += kThreads) {
      const int t = i / p.k_max, j = i - t * p.k_max, k = p.k[t];
      if (k < 1 || k > p.k_most) set_err(p.err, kErrKRange);
      if (j < min(max(k, 1), p.k_most) && (p.ids[i] < 0 || p.ids[i] >= p.E))
        set_err(p.err, kErrIndex);
    }
  }
  const int slot = blockIdx.y, t = slot / p.k_max;
  const int e = p.ids[slot];
  if (slot - t * p.k_max >= min(max(p.k[t], 1), p.k_most) || e < 0 || e >= p.E) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int col = blockIdx.x * (4 * kWarps) + warp * 4;
  const bool on = col < p.inter;  // inter is a multiple of 64
  const int chunks = (p.d + kChunk - 1) / kChunk;
  const int kb = (p.d + 127) / 128, ib = (p.inter + 127) / 128;
  const uint8_t* rows[8];
  const float* sc[2];
  Steps<8> v;
  if (on) {
#pragma unroll
    for (int r = 0; r < 8; ++r)
      rows[r] = p.w_gate_up +
                ((2 * static_cast<int64_t>(e) + (r >> 2)) * p.inter + col + (r & 3)) * p.d +
                lane * 16;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      sc[h] = p.gate_up_scales +
              ((2 * static_cast<int64_t>(e) + h) * ib + col / 128) * kb + (lane >> 3);
    load_steps(v, rows, sc, 0, p.d);
  }
  for (int u = warp; u < chunks * kChunk / 256; u += kWarps)
    quantise_pair(p.hidden + static_cast<int64_t>(t) * p.d, u * 256 + lane * 8, p.d, xs, chunks);
  __syncthreads();
  if (!on) return;
  float acc[8] = {};
  for (int c0 = 0; c0 < chunks; c0 += kAhead) {
    if (c0 > 0) load_steps(v, rows, sc, c0, p.d);
    add_steps(v, xs, c0, chunks, acc);
  }
  sum_lanes(acc);
  float mine = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane == i) mine = swiglu(acc[i], acc[4 + i]);
  if (lane < 4) p.act[static_cast<int64_t>(slot) * p.inter + col + lane] = mine;
}

// out of one token, eight columns a CTA: a warp takes a slot's product (its act
// quantised by the warp itself), and the slots are added in order.  The products stay
// in fp32 until the sum is rounded: they never leave the CTA.
__global__ void __launch_bounds__(kThreads) experts_down_rows_kernel(const Fp8ExpertsRows p) {
  extern __shared__ __align__(16) float xs[];  // [kWarps][row_floats(chunks)]
  __shared__ float y[32][8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = blockIdx.y, n0 = blockIdx.x * 8;
  const int chunks = (p.inter + kChunk - 1) / kChunk;
  const int ib = (p.inter + 127) / 128, db = (p.d + 127) / 128;
  const int kt = min(max(p.k[t], 1), p.k_most);
  float* my_xs = xs + warp * row_floats(chunks);
  const int32_t* ids = p.ids + t * p.k_max;
  bool waited = false;
  for (int j = warp; j < kt; j += kWarps) {
    const int e = ids[j];
    if (e < 0 || e >= p.E) {
      if (lane < 8) y[j][lane] = 0.f;
      continue;
    }
    const uint8_t* rows[8];
    const float* sc[2];
#pragma unroll
    for (int r = 0; r < 8; ++r)
      rows[r] = p.w_down + (static_cast<int64_t>(e) * p.d + n0 + r) * p.inter + lane * 16;
    sc[0] = sc[1] = p.down_scales + (static_cast<int64_t>(e) * db + n0 / 128) * ib + (lane >> 3);
    Steps<8> v;
    load_steps(v, rows, sc, 0, p.inter);
    // (k, ids, the weights and their scales are older than the launch before, which
    // allowed this one after its own wait: only act waits for it)
    if (!waited) grid_dep_wait();
    waited = true;
    const float* act = p.act + (static_cast<int64_t>(t) * p.k_max + j) * p.inter;
    for (int u = 0; u < chunks * kChunk / 256; ++u)
      quantise_pair(act, u * 256 + lane * 8, p.inter, my_xs, chunks);
    __syncwarp();
    float acc[8] = {};
    for (int c0 = 0; c0 < chunks; c0 += kAhead) {
      if (c0 > 0) load_steps(v, rows, sc, c0, p.inter);
      add_steps(v, my_xs, c0, chunks, acc);
    }
    sum_lanes(acc);
    __syncwarp();
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (lane == r) y[j][r] = acc[r];
  }
  if (!waited) grid_dep_wait();
  grid_dep_launch();
  __syncthreads();
  if (threadIdx.x < 8) {
    float sum = 0.f;
    for (int j = 0; j < kt; ++j) {
      const int e = ids[j];
      if (e >= 0 && e < p.E) sum = fmaf(p.alpha[t * p.k_max + j], y[j][threadIdx.x], sum);
    }
    const int64_t at = static_cast<int64_t>(t) * p.d + n0 + threadIdx.x;
    if (p.residual) sum += __bfloat162float(p.hidden[at]);
    p.out[at] = __float2bfloat16_rn(sum);
  }
}

template <typename Te, int M>
cudaError_t launch_m(const Te* x, const Fp8LinearRows& p, int num_sms, cudaStream_t stream) {
  auto kernel = linear_rows_kernel<Te, M>;
  const int chunks = (p.K + kChunk - 1) / kChunk;
  const size_t smem = static_cast<size_t>(M) * row_floats(chunks) * sizeof(float);
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(
        kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
  }
  // as many CTAs as three an SM give the same number of rounds
  const int groups = (p.N + kRows - 1) / kRows, per_round = 3 * num_sms * kWarps;
  const int rounds = (groups + per_round - 1) / per_round;
  const int grid = (groups + rounds * kWarps - 1) / (rounds * kWarps);
  return launch_pdl(kernel, dim3(grid), dim3(kThreads), smem, stream, x, p.ldx, p.w, p.ldw,
                    p.w_scales, p.ldws, p.N, p.K, p.out_f32, p.out, p.ldo, p.zero);
}

template <typename Te>
cudaError_t launch_typed(const Te* x, const Fp8LinearRows& p, int num_sms, cudaStream_t stream) {
  switch (p.M) {
    case 1: return launch_m<Te, 1>(x, p, num_sms, stream);
    case 2: return launch_m<Te, 2>(x, p, num_sms, stream);
    case 3: return launch_m<Te, 3>(x, p, num_sms, stream);
    default: return launch_m<Te, 4>(x, p, num_sms, stream);
  }
}

template <typename K>
cudaError_t launch_wide(K kernel, dim3 grid, size_t smem, const Fp8ExpertsRows& p,
                        cudaStream_t stream) {
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(
        kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(kernel, grid, dim3(kThreads), smem, stream, p);
}

size_t row_bytes(int cols) {
  return static_cast<size_t>((cols + kChunk - 1) / kChunk) * row_floats(1) * sizeof(float);
}

}  // namespace

// Two launches instead of six pay while the slots' weights, read again for every
// slot, are few.  Layer in us, every slot in use, here | tiles:
//   d 2048, inter 1024, k_max 12: 1 token (12 slots, 75 MB) 25 | 35, 2 45 | 57,
//   3 (226 MB) 64 | 59, 4 82 | 61; k_max 8: 3 (151 MB) 44 | 55, 4 (201 MB) 55 | 57;
//   d 2048, inter 512, k_max 12: 1 16 | 32, 4 (151 MB) 50 | 56, 6 (226 MB) 67 | 63;
//   d 1024, inter 512, k_max 8: 1 9 | 26, 8 (101 MB) 34 | 35, 16 (201 MB) 60 | 38;
//   d 256, inter 128, k_max 4: 1 6 | 20, 32 (128 slots) 19 | 21.
// Both kernels' rows lie in shared memory.
bool experts_rows_fit(int T, int k_max, int d, int inter) {
  const int64_t slots = static_cast<int64_t>(T) * k_max;
  return slots <= kFp8ExpertsRowsSlots && slots * 3 * d * inter <= (int64_t{160} << 20) &&
         row_bytes(d) <= 130 * 1024 && row_bytes(inter) * kWarps <= 130 * 1024;
}

cudaError_t launch_experts_rows(const Fp8ExpertsRows& p, cudaStream_t stream) {
  const dim3 up((p.inter + 4 * kWarps - 1) / (4 * kWarps), p.T * p.k_max);
  const cudaError_t e = launch_wide(experts_up_rows_kernel, up, row_bytes(p.d), p, stream);
  if (e != cudaSuccess) return e;
  return launch_wide(experts_down_rows_kernel, dim3(p.d / 8, p.T), row_bytes(p.inter) * kWarps, p,
                     stream);
}

// x fits in shared memory, and the products of each of up to four rows by
// themselves take no longer than the tensor cores' tiles of 128 (us, here |
// quantisation and tiles; weights from HBM): 4096 x 2048 at M = 1..4 4.8, 5.8, 6.8,
// 8.0 | 11.8 to 12.1; 4096 x 4096 at 4 13.7 | 14.9; 65536 x 2048 at 1, 2, 4 25, 34,
// 56 | 28.
bool linear_rows_fit(int M, int N, int K) {
  return M <= 4 && static_cast<int64_t>(M) * ((static_cast<int64_t>(K) + kChunk - 1) / kChunk *
                                              kChunk) <= 16384 &&
         (M == 1 || static_cast<int64_t>(M) * N * K <= (1 << 26));
}

cudaError_t launch_linear_rows(int dtype, const void* x, const Fp8LinearRows& p, int num_sms,
                               cudaStream_t stream) {
  if (dtype == 0) return launch_typed(static_cast<const float*>(x), p, num_sms, stream);
  return launch_typed(static_cast<const __nv_bfloat16*>(x), p, num_sms, stream);
}

}  // namespace rx
