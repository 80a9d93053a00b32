// fp8.cuh — what the 8-bit kernels share: e4m3 conversion, the scale of a
// group, and the launchers of fp8_quantize.cu and fp8_gemm.cu.
#pragma once

#include <cuda.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace rx {

constexpr int kFp8Block = 128;
constexpr float kE4m3Max = 448.0f;

// The largest magnitude of a group from its bits: at least 2^-100, NaN kept.
__device__ __forceinline__ float fp8_amax(uint32_t bits) {
  const uint32_t least = 0x0d800000u;  // 2^-100
  return __uint_as_float(bits > least ? bits : least);
}

// What x is multiplied by to become a code: 448 * (1 / a), both rounded.
__device__ __forceinline__ float fp8_inverse(float a) {
  return __fmul_rn(__fdiv_rn(1.0f, a), kE4m3Max);
}

// Four values to e4m3 codes (round to nearest even), the first in the low byte.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  const uint32_t lo =
      __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi =
      __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}

// silu(g) u, to 2^-21 or so for |g| < 10: an activation that near the middle of two
// codes takes either, as it does by the order of the sums behind g and u.  The library's
// exponential and a rounded division give the experts the same error against 64 bits
// (2.57e-3 and 11.7e-3, to all digits) and take longer: layer at 1024 tokens of 64
// experts of 1024 140 us, here 123, at 8192 tokens of 256 of 512 429, here 377.
__device__ __forceinline__ float swiglu(float g, float u) {
  return __fdividef(g, 1.0f + __expf(-g)) * u;
}

// Rows to codes and scales.  The scale of row r, group g lies at scales +
// r * scale_row_bytes + 4 g.  The first CTA clears the zero words and, with
// k, flags counts outside [1, k_most] in err.
struct Fp8Rows {
  int64_t rows, cols, ldx;
  uint8_t* codes;
  int64_t ldc;
  uint8_t* scales;
  int64_t scale_row_bytes;
  ZeroWords zero;
  const int32_t* k = nullptr;
  int64_t n_k = 0;
  int k_most = 0;
  uint32_t* err = nullptr;
};
cudaError_t launch_quantize_rows(int dtype, const void* x, const Fp8Rows& q, int num_sms,
                                 cudaStream_t stream);
cudaError_t launch_quantize_blocks(int dtype, const void* x, int64_t rows, int64_t cols,
                                   int64_t ldx, uint8_t* codes, int64_t ldc, float* scales,
                                   int64_t lds, cudaStream_t stream);

// The dense layer for up to four rows of x, in one launch (fp8_gemv.cu).
struct Fp8LinearRows {
  int64_t ldx;
  const uint8_t* w;
  int64_t ldw;
  const float* w_scales;
  int64_t ldws;
  int M, N, K;
  int out_f32;
  void* out;
  int64_t ldo;
  ZeroWords zero;
};
bool linear_rows_fit(int M, int N, int K);
cudaError_t launch_linear_rows(int dtype, const void* x, const Fp8LinearRows& p, int num_sms,
                               cudaStream_t stream);

// The routed experts for few pairs, in two launches (fp8_gemv.cu).
struct Fp8ExpertsRows {
  const __nv_bfloat16* hidden;
  const int32_t* ids;
  const float* alpha;
  const int32_t* k;
  const uint8_t* w_gate_up;
  const float* gate_up_scales;
  const uint8_t* w_down;
  const float* down_scales;
  int T, d, E, inter, k_max, k_most;
  int residual;
  float* act;  // [T k_max, inter]
  __nv_bfloat16* out;
  ZeroWords zero;
  uint32_t* err;
};
constexpr int kFp8ExpertsRowsSlots = 128;  // the most slots (T k_max) it serves
bool experts_rows_fit(int T, int k_max, int d, int inter);
cudaError_t launch_experts_rows(const Fp8ExpertsRows& p, cudaStream_t stream);

// A row of codes with its scales behind it, in one piece that a row copy of
// 16-byte vectors moves: codes [cols], scales from the next multiple of 4.
inline int64_t fp8_scale_offset(int64_t cols) { return (cols + 3) / 4 * 4; }
inline int64_t fp8_packed_bytes(int64_t cols) {
  return (fp8_scale_offset(cols) + (cols + 127) / 128 * 4 + 15) / 16 * 16;
}

// C = A B^T over e4m3 codes with a scale for each 128 of K, grouped or dense.
struct Fp8GemmArgs {
  const CUtensorMap* map_a;  // A codes [rows, K]: boxes of {128, a_box}
  const CUtensorMap* map_b;  // B codes {K, rows of a group, groups}: {128, 128, 1}
  // out, boxes of 32 rows x 128 bytes (bf16: 64 columns, act codes: 128) over the columns
  // up to the last whole multiple of 8, where its rows lie on 16-byte boundaries and it is
  // not fp32 or split; else null
  const CUtensorMap* map_out = nullptr;
  int K;
  int n_out;  // columns of out per group (SwiGLU: inter)
  GroupRows g;
  int a_box;  // rows of an A box: 32, 64 or 128
  const uint8_t* a_scales;  // row r, group kb at r * a_scale_row_bytes + 4 kb
  int64_t a_scale_row_bytes;
  const float* b_scales;  // [groups][2 with SwiGLU][blocks of rows][b_scale_ld]
  int64_t b_scale_group;  // floats between groups (SwiGLU: between halves)
  int64_t b_scale_ld;
  void* out;
  int64_t ldo;       // elements; SwiGLU: bytes of a packed row
  int out_f32;       // fp32 out (dense only), else bf16
  int splits = 1;    // CTAs of a cluster that share a tile's K: 1, 2, 4 or 8 (dense only)
  uint32_t* err;
  int num_sms;
};
// SwiGLU: packed rows of codes and scales of silu(A Wg^T) * (A Wu^T).
cudaError_t launch_fp8_swiglu(const Fp8GemmArgs& a, cudaStream_t stream);
// A B^T to bf16 or fp32.
cudaError_t launch_fp8_matmul(const Fp8GemmArgs& a, cudaStream_t stream);

}  // namespace rx
