// fp8_quantize.cu — e4m3 codes with one fp32 scale for each block of 128.
//
// Rows (activations): the 128 columns of a group share a scale; blocks
// (weights): 128 rows x 128 columns do.  With a = the largest magnitude of
// the group, at least 2^-100,
//   scale = a / 448,   code = e4m3(x * (448 * (1 / a)))      (448: the largest e4m3)
// in fp32 IEEE operations, rounded to nearest even, so that the codes are the
// same bits wherever these operations are written out.  The product with the
// reciprocal instead of a division costs at most one rounding of x; the floor
// of a keeps the reciprocal finite and gives a group of zeros zero codes.  An
// infinity or a NaN makes every value that its group stands for NaN (the
// scale is infinite or NaN), as it would in the unquantised product.
//
// Bound: HBM (2 or 4 bytes in, 1 out per element).  16 lanes hold a group in
// registers (8 consecutive elements each, one 16-byte vector in bf16), so one
// pass over the data serves the maximum and the conversion.  32768 x 2048 bf16:
// 36 us, 84 % of the measured copy rate, fp32 52 us, 97 %; bf16 83 us with the division
// in every lane and one pair of groups in flight.  32 x 2048: 2.3 us, one launch in a
// replayed graph.  In 128 x 128 blocks 65536 x 2048 bf16 89 us (the bytes 59), fp32
// 118 (99).
#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"

namespace rx {
namespace {

constexpr int kThreads = 256;
constexpr int kUnits = 4;  // groups that a half of a warp has in flight

// 8 elements from column c on; those at or past cols are 0.
template <typename Te>
__device__ __forceinline__ void load_elems(const Te* row, int64_t c, int64_t cols, bool vec,
                                           float (&f)[8]) {
  if (vec && c + 8 <= cols) {
    load8(row + c, f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = c + i < cols ? to_f32(row[c + i]) : 0.f;
  }
}

// Magnitudes compare as unsigned integers; a NaN's are the largest.
__device__ __forceinline__ uint32_t amax_bits(const float (&f)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
  return m;
}

__device__ __forceinline__ void store_codes(uint8_t* row, int64_t c, int64_t cols, bool vec,
                                            const float (&f)[8], float inv) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = e4m3x4(f[4 * i] * inv, f[4 * i + 1] * inv, f[4 * i + 2] * inv, f[4 * i + 3] * inv);
  if (vec && c + 8 <= cols) {
    *reinterpret_cast<uint2*>(row + c) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) row[c + i] = static_cast<uint8_t>(w[i >> 2] >> (8 * (i & 3)));
  }
}

// 8 elements as loaded, their largest magnitude as fp32 bits, and their values.
template <typename Te>
struct Raw8;
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* row, int c, int cols, bool vec) {
    if (vec && c + 8 <= cols) {
      a = __ldcs(reinterpret_cast<const float4*>(row + c));
      b = __ldcs(reinterpret_cast<const float4*>(row + c) + 1);
    } else {
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = c + i < cols ? row[c + i] : 0.f;
      a = make_float4(f[0], f[1], f[2], f[3]);
      b = make_float4(f[4], f[5], f[6], f[7]);
    }
  }
  __device__ __forceinline__ uint32_t amax() const {
    const float f[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    return amax_bits(f);
  }
  __device__ __forceinline__ void widen(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};
template <>
struct Raw8<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* row, int c, int cols, bool vec) {
    if (vec && c + 8 <= cols) {
      v = __ldcs(reinterpret_cast<const uint4*>(row + c));
    } else {
      uint32_t e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        e[i] = c + i < cols ? reinterpret_cast<const uint16_t*>(row)[c + i] : 0u;
      v = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    }
  }
  __device__ __forceinline__ uint32_t amax() const {
    // magnitudes without their signs order as 16-bit integers, a NaN last
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu),
                                __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    return max(m << 16, m & 0xffff0000u);
  }
  __device__ __forceinline__ void widen(float (&f)[8]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};

// A warp takes 2 kUnits groups at a time: their loads in flight together (16 lanes a
// group), then a lane per group divides for the 16 that hold it.  kPacked: of
// several rows, one group after another, where a row has few.
template <typename Te, bool kPacked>
__global__ void __launch_bounds__(kThreads)
    quantize_rows_kernel(const Te* __restrict__ x, int64_t rows, int cols, int64_t ldx,
                         uint8_t* __restrict__ codes, int64_t ldc, uint8_t* __restrict__ scales,
                         int64_t scale_row_bytes, int vec_x, int vec_c, uint32_t groups,
                         ZeroWords zero, const int32_t* __restrict__ k, int64_t n_k, int k_most,
                         uint32_t* err) {
  grid_dep_wait();
  grid_dep_launch();
  if (blockIdx.x == 0 && (zero.n > 0 || k != nullptr)) {
    clear_words(zero);
    if (k != nullptr) {  // the counts of the call that these rows belong to
      __syncthreads();
      bool bad = false;
      for (int64_t i = threadIdx.x; i < n_k; i += kThreads) bad |= k[i] < 1 || k[i] > k_most;
      if (bad) set_err(err, kErrKRange);
    }
  }
  const int lane = threadIdx.x & 31, half = lane >> 4;
  constexpr int kGroups = 2 * kUnits;
  const uint32_t chunks = (groups + kGroups - 1) / kGroups;  // of a row
  const int64_t total = rows * groups;
  const int64_t units = kPacked ? (total + kGroups - 1) / kGroups : rows * chunks;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
       u < units; u += step) {
    // the unit's first group, and its groups
    const int64_t first = kPacked ? u * kGroups : u;
    const uint32_t per_row = kPacked ? groups : chunks;
    const int64_t r0 = (kPacked ? total : units) <= 0xffffffffll
                           ? static_cast<uint32_t>(first) / per_row : first / per_row;
    const uint32_t g0 = static_cast<uint32_t>(first - r0 * per_row) * (kPacked ? 1 : kGroups);
    const int left = static_cast<int>(
        min(static_cast<int64_t>(kGroups), kPacked ? total - first : int64_t{groups} - g0));
    auto locate = [&](int n, int64_t& r, uint32_t& g) {
      const uint32_t over = kPacked ? (g0 + n) / groups : 0u;
      g = g0 + n - over * groups;
      r = r0 + over;
    };
    Raw8<Te> raw[kUnits];
    int64_t row[kUnits];
    int col[kUnits];
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      uint32_t g;
      locate(2 * i + half, row[i], g);
      col[i] = static_cast<int>(g) * 128 + (lane & 15) * 8;
      if (2 * i + half < left) raw[i].load(x + row[i] * ldx, col[i], cols, vec_x != 0);
    }
    // the magnitude of the n-th group ends up in lane n
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      uint32_t m = 0;
      if (2 * i + half < left) m = raw[i].amax();
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      const uint32_t other = __shfl_xor_sync(0xffffffffu, m, 16);
      if ((lane >> 1) == i) mine = (lane & 1) == half ? m : other;
    }
    const float a = fp8_amax(mine), inv = fp8_inverse(a);
    if (lane < left) {
      int64_t r;
      uint32_t g;
      locate(lane, r, g);
      *reinterpret_cast<float*>(scales + r * scale_row_bytes + static_cast<int64_t>(g) * 4) =
          __fdiv_rn(a, kE4m3Max);
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const float by = __shfl_sync(0xffffffffu, inv, 2 * i + half);
      if (2 * i + half >= left) continue;
      float f[8];
      raw[i].widen(f);
      store_codes(codes + row[i] * ldc, col[i], cols, vec_c != 0, f, by);
    }
  }
}

// One CTA per 128 x 128 block (weights, laid out once): the block is read
// twice, the second time from L2.
template <typename Te>
__global__ void __launch_bounds__(kThreads)
    quantize_blocks_kernel(const Te* __restrict__ x, int64_t rows, int64_t cols, int64_t ldx,
                           uint8_t* __restrict__ codes, int64_t ldc, float* __restrict__ scales,
                           int64_t lds, int vec_x, int vec_c) {
  __shared__ uint32_t s_max[kThreads / 32];
  grid_dep_wait();
  grid_dep_launch();
  const int64_t kb = (cols + 127) / 128;
  const int64_t br = blockIdx.x / kb, bc = blockIdx.x % kb;
  const int64_t c = bc * 128 + (threadIdx.x & 15) * 8;
  const int64_t r0 = br * 128 + (threadIdx.x >> 4), r1 = min(rows, br * 128 + 128);
  uint32_t m = 0;
  for (int64_t r = r0; r < r1; r += kThreads / 16) {
    float f[8];
    load_elems(x + r * ldx, c, cols, vec_x != 0, f);
    m = max(m, amax_bits(f));
  }
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) m = max(m, s_max[i]);
  const float a = fp8_amax(m), inv = fp8_inverse(a);
  for (int64_t r = r0; r < r1; r += kThreads / 16) {
    float f[8];
    load_elems(x + r * ldx, c, cols, vec_x != 0, f);
    store_codes(codes + r * ldc, c, cols, vec_c != 0, f, inv);
  }
  if (threadIdx.x == 0) scales[br * lds + bc] = __fdiv_rn(a, kE4m3Max);
}

template <typename Te>
bool aligned_rows(const Te* x, int64_t ld) {
  constexpr int64_t kVec = sizeof(Te) == 1 ? 8 : 16;
  return reinterpret_cast<uintptr_t>(x) % kVec == 0 &&
         ld * static_cast<int64_t>(sizeof(Te)) % kVec == 0;
}

template <typename Te>
cudaError_t rows_typed(const Te* x, const Fp8Rows& q, int num_sms, cudaStream_t stream) {
  const int64_t groups = (q.cols + 127) / 128;
  // (30 million bf16 in rows of 64, 128, 256 and 384: packed 57, 21, 21 and 21 us, a
  // row a warp 150, 80, 36 and 35; in rows of 513 and 1000 packed 40 and 25, here 38
  // and 20)
  const bool packed = groups <= kUnits;
  const int64_t units = packed ? (q.rows * groups + 2 * kUnits - 1) / (2 * kUnits)
                               : q.rows * ((groups + 2 * kUnits - 1) / (2 * kUnits));
  const int64_t grid = (units + kThreads / 32 - 1) / (kThreads / 32);
  return launch_pdl(packed ? quantize_rows_kernel<Te, true> : quantize_rows_kernel<Te, false>,
                    dim3(static_cast<unsigned>(std::min<int64_t>(grid, 16 * num_sms))),
                    dim3(kThreads), 0, stream, x, q.rows, static_cast<int>(q.cols), q.ldx,
                    q.codes, q.ldc, q.scales, q.scale_row_bytes,
                    static_cast<int>(aligned_rows(x, q.ldx)),
                    static_cast<int>(aligned_rows(q.codes, q.ldc)),
                    static_cast<uint32_t>(groups), q.zero, q.k, q.n_k, q.k_most, q.err);
}

template <typename Te>
cudaError_t blocks_typed(const Te* x, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes,
                         int64_t ldc, float* scales, int64_t lds, cudaStream_t stream) {
  const int64_t blocks = ((rows + 127) / 128) * ((cols + 127) / 128);
  return launch_pdl(quantize_blocks_kernel<Te>, dim3(static_cast<unsigned>(blocks)),
                    dim3(kThreads), 0, stream, x, rows, cols, ldx, codes, ldc, scales, lds,
                    static_cast<int>(aligned_rows(x, ldx)),
                    static_cast<int>(aligned_rows(codes, ldc)));
}

}  // namespace

cudaError_t launch_quantize_rows(int dtype, const void* x, const Fp8Rows& q, int num_sms,
                                 cudaStream_t stream) {
  if (dtype == 0) return rows_typed(static_cast<const float*>(x), q, num_sms, stream);
  return rows_typed(static_cast<const __nv_bfloat16*>(x), q, num_sms, stream);
}

cudaError_t launch_quantize_blocks(int dtype, const void* x, int64_t rows, int64_t cols,
                                   int64_t ldx, uint8_t* codes, int64_t ldc, float* scales,
                                   int64_t lds, cudaStream_t stream) {
  if (dtype == 0)
    return blocks_typed(static_cast<const float*>(x), rows, cols, ldx, codes, ldc, scales, lds,
                        stream);
  return blocks_typed(static_cast<const __nv_bfloat16*>(x), rows, cols, ldx, codes, ldc, scales,
                      lds, stream);
}

}  // namespace rx
