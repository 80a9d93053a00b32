// fp8_gemv.cu — the dense layer of reflex_linear_fp8 for one to four rows:
// x quantised, then multiplied with e4m3 weights, in one launch.
//
// Bound: the weights' bytes (65536 x 2048, one row: 27 us, 73 % of the measured
// copy rate; 4096 x 2048: 4.8 us, of which the bytes take 1.2 and one launch, one
// trip to HBM and the quantisation the rest).  A warp takes four rows of the weights at a time and 512 columns a step,
// 16 bytes of each row a lane, so a step has 2 KB in flight and x is read from
// shared memory once for four rows.  Every CTA quantises x by itself (the codes
// of reflex_quantize_fp8 bit for bit): a second launch would take longer.  The 16
// products of a lane lie in one block of K: they are summed in fp32, scaled once
// by the weights' scale (x's scale is in x), and the lanes' sums added at the end.
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

// Element k of a row of x in shared memory: a lane's 16 columns as four vectors,
// each vector of all lanes in a row, so that no two lanes share a bank.
__device__ __forceinline__ int place(int k) {
  return (k >> 9) * kChunk + ((k >> 2) & 3) * 128 + ((k >> 4) & 31) * 4 + (k & 3);
}

template <typename Te, int M>
__global__ void __launch_bounds__(kThreads)
    linear_rows_kernel(const Te* __restrict__ x, int64_t ldx, const uint8_t* __restrict__ w,
                       int64_t ldw, const float* __restrict__ w_scales, int64_t ldws, int N,
                       int K, int out_f32, void* __restrict__ out, int64_t ldo, ZeroWords zero) {
  extern __shared__ __align__(16) float xs[];  // [M][chunks * kChunk], see place()
  grid_dep_wait();
  grid_dep_launch();
  if (blockIdx.x == 0) clear_words(zero);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int chunks = (K + kChunk - 1) / kChunk, row_floats = chunks * kChunk;
  // x: 16 lanes a group of 128, as the quantisation kernel
  const int pairs = row_floats / 256;
  for (int u = warp; u < M * pairs; u += kWarps) {
    const int m = u / pairs, c = (u - m * pairs) * 256 + lane * 8;
    const Te* row = x + m * ldx;
    float f[8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      f[i] = c + i < K ? to_f32(row[c + i]) : 0.f;
      top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float a = fp8_amax(top), inv = fp8_inverse(a), s = __fdiv_rn(a, kE4m3Max);
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const uint32_t q = e4m3x4(f[i] * inv, f[i + 1] * inv, f[i + 2] * inv, f[i + 3] * inv);
      const float2 lo = e4m3x2(q & 0xffffu), hi = e4m3x2(q >> 16);
      *reinterpret_cast<float4*>(xs + m * row_floats + place(c + i)) =
          make_float4(lo.x * s, lo.y * s, hi.x * s, hi.y * s);
    }
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
            xv[m] = *reinterpret_cast<const float4*>(xs + m * row_floats + (c0 + d) * kChunk +
                                                     j * 128 + lane * 4);
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
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
          for (int m = 0; m < M; ++m)
            acc[r][m] = fmaf(sum[r][m].x + sum[r][m].y, s[d], acc[r][m]);
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

template <typename Te, int M>
cudaError_t launch_m(const Te* x, const Fp8LinearRows& p, int num_sms, cudaStream_t stream) {
  auto kernel = linear_rows_kernel<Te, M>;
  const int chunks = (p.K + kChunk - 1) / kChunk;
  const size_t smem = static_cast<size_t>(M) * chunks * kChunk * sizeof(float);
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

}  // namespace

// x fits in shared memory, and the products of each of up to four rows by
// themselves take no longer than the tensor cores' tiles of 128 (us, here |
// quantisation and tiles): 4096 x 2048 at M = 1..4 4.8, 5.8, 6.7, 7.9 | 11.4;
// 4096 x 4096 at 4 13.7 | 14.1; 65536 x 2048 at 1, 2, 4 27, 35, 57 | 30.
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
