// fp8_abi.cu — C entry points of the 8-bit path and of sampling: argument
// checks, workspace carving, tensor maps and the launch sequences of one
// quantisation, one product and one layer of routed experts.
#include <cudaTypedefs.h>

#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"
#include "reflex.h"

namespace rx {
PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder();
int device_sms();
}  // namespace rx

namespace {

using rx::WsHeader;

constexpr size_t kAlign = 256;
size_t up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
int64_t blocks(int64_t n) { return (n + 127) / 128; }
int64_t blocks2(int64_t n) { return (n + 255) / 256; }

#define RX_CUDA(x)                                  \
  do {                                              \
    if ((x) != cudaSuccess) return REFLEX_ECUDA;    \
  } while (0)

bool dtype_ok(int32_t t) { return t == REFLEX_DTYPE_F32 || t == REFLEX_DTYPE_BF16; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// Codes {cols, rows, groups} (groups == 0: a 2D map), boxes of 128 bytes of
// `box_rows` rows, 128-byte swizzle, zero fill past the edges.
bool code_map(CUtensorMap* m, const void* base, int64_t groups, int64_t rows, int64_t cols,
              int64_t ld, int64_t group_bytes, int box_rows) {
  auto fn = rx::tensor_map_encoder();
  if (fn == nullptr) return false;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows),
                              static_cast<cuuint64_t>(groups)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld),
                                 static_cast<cuuint64_t>(group_bytes)};
  const cuuint32_t box[3] = {128, static_cast<cuuint32_t>(box_rows), 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, groups > 0 ? 3 : 2, const_cast<void*>(base), dims,
            strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Rows of out as the kernel stores them, 32 x 128 bytes at a time with the same
// swizzle; rows of whole 16-byte vectors.
bool out_map(CUtensorMap* m, void* base, bool bf16, int64_t rows, int64_t cols, int64_t row_bytes) {
  auto fn = rx::tensor_map_encoder();
  if (fn == nullptr) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(row_bytes)};
  const cuuint32_t box[2] = {bf16 ? 64u : 128u, 32};
  const cuuint32_t estr[2] = {1, 1};
  return fn(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base,
            dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// CTAs of a cluster that share a tile's K, where the tiles leave SMs free.  Adding
// the parts costs some 3 us for each 32 rows of a tile, a block of K 0.5 us, so taller
// tiles are split at a longer K only (N x K, one CTA a tile | split, us):
//   M =   8, 4096 x 2048: 13 | 12 by 4, 20 by 8;   1024 x 8192: 34 | 18 by 4, 14 by 8
//   M =  64, 512 x 2048: 14 | 14;  512 x 3200: 20 | 16;  512 x 8000: 38 | 20
//   M = 128, 512 x 3200: 21 | 24;  512 x 5120: 28 | 25;  512 x 8000: 39 | 28
//   M = 256, 8192 x 8000: 43 | 51 by 2;   M = 300, 2048 x 5120: 29 | 29 by 4
// Clusters of eight find room at once in half of the SMs only: more wait for a
// second round, the 20 by 8 above.
int pick_splits(int64_t M, int64_t tiles, int64_t nkb, int sms) {
  int s = 1;
  while (s < 8 && nkb >= 4 * s && tiles * s * 2 <= (s < 4 ? sms : sms / 2)) s *= 2;
  // the blocks that a CTA is spared, against 8.5 for each 32 rows
  const int64_t quarters = std::min<int64_t>(4, (M + 31) / 32);
  return M > 32 && 2 * nkb * (s - 1) < 17 * quarters * s ? 1 : s;
}

int matmul(const uint8_t* a, int64_t lda, const uint8_t* a_scales, int64_t a_scale_row_bytes,
           const uint8_t* b, int64_t ldb, const float* b_scales, int64_t ldbs, int32_t M,
           int32_t N, int32_t K, int32_t out_dtype, void* out, int64_t ldo, uint32_t* err,
           cudaStream_t s) {
  const int sms = rx::device_sms();
  CUtensorMap ma, mb;
  const int a_box = M >= 128 ? 128 : M > 32 ? 64 : 32;
  if (!code_map(&ma, a, 0, M, K, lda, 0, a_box) ||
      !code_map(&mb, b, 1, N, K, ldb, ldb * static_cast<int64_t>(N), 128))
    return REFLEX_ECUDA;
  rx::Fp8GemmArgs g{};
  g.map_a = &ma;
  g.map_b = &mb;
  g.K = K;
  g.n_out = N;
  g.g = rx::GroupRows{nullptr, nullptr, nullptr, nullptr, 1, M, M};
  g.a_box = a_box;
  g.a_scales = a_scales;
  g.a_scale_row_bytes = a_scale_row_bytes;
  g.b_scales = b_scales;
  g.b_scale_ld = ldbs;
  g.out = out;
  g.ldo = ldo;
  g.out_f32 = out_dtype == REFLEX_DTYPE_F32;
  g.splits = pick_splits(M, blocks(M) * blocks2(N), blocks(K), sms);
  g.err = err;
  g.num_sms = sms;
  CUtensorMap mo;
  if (g.splits == 1 && !g.out_f32 && aligned(out, 16) && ldo % 8 == 0 && N >= 8) {
    if (!out_map(&mo, out, true, M, N / 8 * 8, ldo * 2)) return REFLEX_ECUDA;
    g.map_out = &mo;
  }
  RX_CUDA(rx::launch_fp8_matmul(g, s));
  return REFLEX_OK;
}

// Sizes that the kernels' 32-bit counts of tiles and columns hold.
bool product_fits(int64_t M, int64_t N, int64_t K) {
  constexpr int64_t most = int64_t{1} << 30;
  return M <= most && N <= most && K <= most && blocks(M) * blocks2(N) <= most;
}
// Rows, columns and strides of a product that the kernels and maps can take.
bool product_ok(int64_t M, int64_t N, int64_t K, int64_t ldb, int64_t ldbs, int32_t out_dtype,
                int64_t ldo) {
  return M >= 0 && N >= 1 && K >= 1 && ldb >= K && ldb % 16 == 0 && ldbs >= blocks(K) &&
         dtype_ok(out_dtype) && ldo >= N;
}

struct LinearLayout {
  size_t hdr, rows, total;
  int64_t row_bytes;
};
LinearLayout linear_layout(int64_t M, int64_t K) {
  LinearLayout L{};
  L.row_bytes = rx::fp8_packed_bytes(K);
  L.hdr = 0;
  L.rows = up(sizeof(WsHeader));
  L.total = L.rows + up(static_cast<size_t>(M) * L.row_bytes);
  return L;
}

struct ExpertsLayout {
  size_t hdr, x, blk_count, blk_mask, blk_off, counts, offsets, mt_prefix, mt2_prefix, perm,
      row_of, weights, xperm, act, y, act_rows, total;
  int64_t cap, x_bytes, act_bytes;
};
ExpertsLayout experts_layout(int32_t T, int32_t d, int32_t E, int32_t inter, int32_t k_max) {
  ExpertsLayout L{};
  L.cap = static_cast<int64_t>(T) * k_max;
  L.x_bytes = rx::fp8_packed_bytes(d);
  L.act_bytes = rx::fp8_packed_bytes(inter);
  const int64_t nblk = rx::dispatch_blocks_alloc(T);
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += up(bytes);
    return at;
  };
  L.hdr = take(sizeof(WsHeader));
  L.x = take(static_cast<size_t>(T) * L.x_bytes);
  L.blk_count = take(static_cast<size_t>(nblk) * E * 4);
  L.blk_mask = take(static_cast<size_t>(rx::dispatch_mask_words_alloc(T)) * E * 4);
  L.blk_off = take(static_cast<size_t>(nblk) * E * 4);
  L.counts = take(static_cast<size_t>(E) * 4);
  L.offsets = take(static_cast<size_t>(E + 1) * 4);
  L.mt_prefix = take(static_cast<size_t>(E + 1) * 4);
  L.mt2_prefix = take(static_cast<size_t>(E + 1) * 4);
  L.perm = take(L.cap * 4);
  L.row_of = take(L.cap * 4);
  L.weights = take(L.cap * 4);
  L.xperm = take(L.cap * L.x_bytes);
  L.act = take(L.cap * L.act_bytes);
  // Tiles leave the pairs' outputs in memory as bf16, in which the layer's output is
  // rounded anyway; fp32 ones take twice the bytes through two kernels and bring the
  // error against 64 bits down by 1 % (k_max 12, d 2048, bf16 | fp32; relative error, us):
  //   64 x 1024, 32 tokens 2.62e-3, 83 | 2.60e-3, 89; 1024 tokens 2.57e-3, 123 | 2.55e-3, 140;
  //   256 x 512, 8192 tokens 11.7e-3, 377 | 11.6e-3, 489.
  L.y = take(L.cap * d * 2);
  L.act_rows = take(std::min<int64_t>(L.cap, rx::kFp8ExpertsRowsSlots) * inter * 4);
  L.total = o;
  return L;
}
bool experts_ok(int32_t T, int32_t d, int32_t E, int32_t inter, int32_t k_max) {
  return T >= 0 && d > 0 && d % 64 == 0 && E >= 1 && E <= 1024 && inter > 0 && inter % 64 == 0 &&
         k_max >= 1 && k_max <= 32 && static_cast<int64_t>(T) * k_max <= (int64_t{1} << 30);
}

}  // namespace

extern "C" {

int reflex_quantize_fp8(int32_t dtype, const void* x, int64_t rows, int64_t cols, int64_t ldx,
                        int32_t block_rows, uint8_t* codes, int64_t ldc, float* scales,
                        int64_t lds, void* stream) {
  if (!dtype_ok(dtype) || rows < 0 || cols < 0 || (block_rows != 1 && block_rows != 128))
    return REFLEX_EINVAL;
  if (rows == 0 || cols == 0) return REFLEX_OK;
  if (cols > (1 << 30)) return REFLEX_EUNSUPPORTED;
  if (x == nullptr || codes == nullptr || scales == nullptr || ldx < cols || ldc < cols ||
      lds < blocks(cols))
    return REFLEX_EINVAL;
  if (!aligned(x, dtype == REFLEX_DTYPE_F32 ? 4 : 2) || !aligned(scales, 4)) return REFLEX_EINVAL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (block_rows == 128) {
    if (blocks(rows) * blocks(cols) > 0x7fffffff) return REFLEX_EUNSUPPORTED;
    RX_CUDA(rx::launch_quantize_blocks(dtype, x, rows, cols, ldx, codes, ldc, scales, lds, s));
    return REFLEX_OK;
  }
  rx::Fp8Rows q{rows, cols, ldx, codes, ldc, reinterpret_cast<uint8_t*>(scales), lds * 4, {}};
  RX_CUDA(rx::launch_quantize_rows(dtype, x, q, rx::device_sms(), s));
  return REFLEX_OK;
}

int reflex_matmul_fp8(const uint8_t* a, int64_t lda, const float* a_scales, int64_t ldas,
                      const uint8_t* b, int64_t ldb, const float* b_scales, int64_t ldbs,
                      int32_t M, int32_t N, int32_t K, int32_t out_dtype, void* out, int64_t ldo,
                      int32_t* dev_status, void* stream) {
  if (!product_ok(M, N, K, ldb, ldbs, out_dtype, ldo)) return REFLEX_EINVAL;
  if (!product_fits(M, N, K)) return REFLEX_EUNSUPPORTED;
  if (M > 0) {
    if (a == nullptr || a_scales == nullptr || b == nullptr || b_scales == nullptr ||
        out == nullptr || lda < K || lda % 16 != 0 || ldas < blocks(K))
      return REFLEX_EINVAL;
    if (!aligned(a, 16) || !aligned(b, 16) || !aligned(a_scales, 4) || !aligned(b_scales, 4) ||
        !aligned(out, out_dtype == REFLEX_DTYPE_F32 ? 4 : 2))
      return REFLEX_EINVAL;
  }
  if (!aligned(dev_status, 4)) return REFLEX_EINVAL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dev_status != nullptr) RX_CUDA(cudaMemsetAsync(dev_status, 0, sizeof(int32_t), s));
  if (M == 0) return REFLEX_OK;
  return matmul(a, lda, reinterpret_cast<const uint8_t*>(a_scales), ldas * 4, b, ldb, b_scales,
                ldbs, M, N, K, out_dtype, out, ldo, reinterpret_cast<uint32_t*>(dev_status), s);
}

size_t reflex_linear_fp8_workspace_size(int32_t M, int32_t K) {
  if (M < 0 || K < 1) return 0;
  return linear_layout(M, K).total;
}

int reflex_linear_fp8(int32_t dtype, const void* x, int64_t ldx, const uint8_t* w, int64_t ldw,
                      const float* w_scales, int64_t ldws, int32_t M, int32_t N, int32_t K,
                      int32_t out_dtype, void* out, int64_t ldo, void* workspace,
                      size_t ws_bytes, void* stream) {
  if (!dtype_ok(dtype) || !product_ok(M, N, K, ldw, ldws, out_dtype, ldo) || ldx < K)
    return REFLEX_EINVAL;
  if (!product_fits(M, N, K)) return REFLEX_EUNSUPPORTED;
  const LinearLayout L = linear_layout(M, K);
  if (workspace == nullptr || ws_bytes < L.total || !aligned(workspace, kAlign))
    return REFLEX_EWORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  WsHeader* hdr = reinterpret_cast<WsHeader*>(ws + L.hdr);
  if (M == 0) {
    RX_CUDA(cudaMemsetAsync(hdr, 0, sizeof(WsHeader), s));
    return REFLEX_OK;
  }
  if (x == nullptr || w == nullptr || w_scales == nullptr || out == nullptr) return REFLEX_EINVAL;
  if (!aligned(x, dtype == REFLEX_DTYPE_F32 ? 4 : 2) || !aligned(w, 16) ||
      !aligned(w_scales, 4) || !aligned(out, out_dtype == REFLEX_DTYPE_F32 ? 4 : 2))
    return REFLEX_EINVAL;
  rx::ZeroWords zero;
  zero.words = reinterpret_cast<uint32_t*>(hdr);
  zero.n = static_cast<int>(sizeof(WsHeader) / 4);
  if (rx::linear_rows_fit(M, N, K)) {
    const rx::Fp8LinearRows p{ldx, w, ldw, w_scales, ldws, M, N, K,
                              out_dtype == REFLEX_DTYPE_F32, out, ldo, zero};
    RX_CUDA(rx::launch_linear_rows(dtype, x, p, rx::device_sms(), s));
    return REFLEX_OK;
  }
  if (rx::tensor_map_encoder() == nullptr) return REFLEX_ECUDA;
  uint8_t* rows = ws + L.rows;
  uint8_t* scales = rows + rx::fp8_scale_offset(K);
  const rx::Fp8Rows q{M, K, ldx, rows, L.row_bytes, scales, L.row_bytes, zero};
  RX_CUDA(rx::launch_quantize_rows(dtype, x, q, rx::device_sms(), s));
  return matmul(rows, L.row_bytes, scales, L.row_bytes, w, ldw, w_scales, ldws, M, N, K,
                out_dtype, out, ldo, &hdr->err, s);
}

size_t reflex_experts_fp8_workspace_size(int32_t T, int32_t d, int32_t E, int32_t inter,
                                         int32_t k_max) {
  return experts_ok(T, d, E, inter, k_max) ? experts_layout(T, d, E, inter, k_max).total : 0;
}

int reflex_experts_fp8(const void* hidden, const int32_t* ids, const float* alpha,
                       const int32_t* k, const uint8_t* w_gate_up, const float* gate_up_scales,
                       const uint8_t* w_down, const float* down_scales, int32_t T, int32_t d,
                       int32_t E, int32_t inter, int32_t k_max, uint32_t flags, void* workspace,
                       size_t ws_bytes, void* out, void* stream) {
  if (!experts_ok(T, d, E, inter, k_max) || (flags & ~REFLEX_FLAG_RESIDUAL)) return REFLEX_EINVAL;
  const ExpertsLayout L = experts_layout(T, d, E, inter, k_max);
  if (workspace == nullptr || ws_bytes < L.total || !aligned(workspace, kAlign))
    return REFLEX_EWORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  WsHeader* hdr = reinterpret_cast<WsHeader*>(ws + L.hdr);
  if (T == 0) {
    RX_CUDA(cudaMemsetAsync(hdr, 0, sizeof(WsHeader), s));
    return REFLEX_OK;
  }
  if (hidden == nullptr || ids == nullptr || alpha == nullptr || k == nullptr ||
      w_gate_up == nullptr || gate_up_scales == nullptr || w_down == nullptr ||
      down_scales == nullptr || out == nullptr)
    return REFLEX_EINVAL;
  if (!aligned(hidden, 16) || !aligned(out, 16) || !aligned(w_gate_up, 16) ||
      !aligned(w_down, 16) || !aligned(ids, 4) || !aligned(alpha, 4) || !aligned(k, 4) ||
      !aligned(gate_up_scales, 4) || !aligned(down_scales, 4))
    return REFLEX_EINVAL;
  rx::ZeroWords zero;
  zero.words = reinterpret_cast<uint32_t*>(hdr);
  zero.n = static_cast<int>(sizeof(WsHeader) / 4);
  const int k_most = k_max < E ? k_max : E;
  if (rx::experts_rows_fit(T, k_max, d, inter)) {
    const rx::Fp8ExpertsRows p{static_cast<const __nv_bfloat16*>(hidden), ids, alpha, k, w_gate_up,
                               gate_up_scales, w_down, down_scales, T, d, E, inter, k_max, k_most,
                               (flags & REFLEX_FLAG_RESIDUAL) != 0,
                               reinterpret_cast<float*>(ws + L.act_rows),
                               static_cast<__nv_bfloat16*>(out), zero, &hdr->err};
    RX_CUDA(rx::launch_experts_rows(p, s));
    return REFLEX_OK;
  }
  if (rx::tensor_map_encoder() == nullptr) return REFLEX_ECUDA;
  const int sms = rx::device_sms();
  const int cap = static_cast<int>(L.cap);
  auto I32 = [&](size_t off) { return reinterpret_cast<int32_t*>(ws + off); };
  uint32_t* err = &hdr->err;

  // rows to codes once per token; the dispatch copies packed rows, half of
  // the bytes of bf16 ones
  rx::Fp8Rows q{T, d, d, ws + L.x, L.x_bytes, ws + L.x + rx::fp8_scale_offset(d), L.x_bytes, {}};
  q.zero = zero;
  q.k = k;
  q.n_k = T;
  q.k_most = k_most;
  q.err = err;
  RX_CUDA(rx::launch_quantize_rows(REFLEX_DTYPE_BF16, hidden, q, sms, s));
  rx::DispatchBufs b{I32(L.blk_count), I32(L.blk_off),    I32(L.counts), I32(L.offsets),
                     I32(L.mt_prefix), I32(L.mt2_prefix), I32(L.perm),   I32(L.row_of),
                     &hdr->total_pairs, err, reinterpret_cast<uint32_t*>(ws + L.blk_mask),
                     alpha, reinterpret_cast<float*>(ws + L.weights)};
  RX_CUDA(rx::launch_dispatch_gather(REFLEX_DTYPE_BF16, ws + L.x, ids, k, T, E, k_max, cap,
                                     static_cast<int>(L.x_bytes / 2), b, ws + L.xperm, sms, s));

  CUtensorMap ma1, mb1, mo1, ma2, mb2, mo2;
  constexpr int kBox = 32;
  if (!code_map(&ma1, ws + L.xperm, 0, cap, d, L.x_bytes, 0, kBox) ||
      !code_map(&mb1, w_gate_up, 2 * static_cast<int64_t>(E), inter, d, d,
                static_cast<int64_t>(inter) * d, 128) ||
      !code_map(&ma2, ws + L.act, 0, cap, inter, L.act_bytes, 0, kBox) ||
      !code_map(&mb2, w_down, E, d, inter, inter, static_cast<int64_t>(d) * inter, 128) ||
      !out_map(&mo1, ws + L.act, false, cap, inter, L.act_bytes) ||
      !out_map(&mo2, ws + L.y, true, cap, d, static_cast<int64_t>(d) * 2))
    return REFLEX_ECUDA;
  rx::Fp8GemmArgs g{};
  g.g = rx::GroupRows{I32(L.offsets), I32(L.mt_prefix), I32(L.mt2_prefix), &hdr->total_pairs,
                      E, 0, cap};
  g.a_box = kBox;
  g.err = err;
  g.num_sms = sms;
  rx::Fp8GemmArgs up_args = g;
  up_args.map_a = &ma1;
  up_args.map_b = &mb1;
  up_args.map_out = &mo1;
  up_args.K = d;
  up_args.n_out = inter;
  up_args.a_scales = ws + L.xperm + rx::fp8_scale_offset(d);
  up_args.a_scale_row_bytes = L.x_bytes;
  up_args.b_scales = gate_up_scales;
  up_args.b_scale_group = blocks(inter) * blocks(d);
  up_args.b_scale_ld = blocks(d);
  up_args.out = ws + L.act;
  up_args.ldo = L.act_bytes;
  RX_CUDA(rx::launch_fp8_swiglu(up_args, s));
  rx::Fp8GemmArgs dn = g;
  dn.map_a = &ma2;
  dn.map_b = &mb2;
  dn.map_out = &mo2;
  dn.K = inter;
  dn.n_out = d;
  dn.a_scales = ws + L.act + rx::fp8_scale_offset(inter);
  dn.a_scale_row_bytes = L.act_bytes;
  dn.b_scales = down_scales;
  dn.b_scale_group = blocks(d) * blocks(inter);
  dn.b_scale_ld = blocks(inter);
  dn.out = ws + L.y;
  dn.ldo = d;
  RX_CUDA(rx::launch_fp8_matmul(dn, s));
  const void* resid = (flags & REFLEX_FLAG_RESIDUAL) ? hidden : nullptr;
  RX_CUDA(rx::launch_combine(REFLEX_DTYPE_BF16, ws + L.y, nullptr, resid, I32(L.row_of),
                             reinterpret_cast<const float*>(ws + L.weights), k, T, d, k_max, cap,
                             out, err, sms, s));
  return REFLEX_OK;
}

int reflex_sample(int32_t dtype, const void* logits, int64_t ld, int32_t rows, int32_t vocab,
                  const float* temperature, const int32_t* top_k, const float* top_p,
                  const float* min_p, const float* u, const uint8_t* masked, int32_t* tokens_out,
                  float* conf_out, int32_t* dev_status, void* stream) {
  if (!dtype_ok(dtype) || rows < 0 || vocab < 1 || ld < vocab) return REFLEX_EINVAL;
  if (vocab > rx::sample_max_vocab() || rows > (1 << 27)) return REFLEX_EUNSUPPORTED;
  if (rows == 0) return REFLEX_OK;
  if (logits == nullptr || u == nullptr || tokens_out == nullptr || conf_out == nullptr ||
      !aligned(logits, dtype == REFLEX_DTYPE_F32 ? 4 : 2))
    return REFLEX_EINVAL;
  for (const void* words : {static_cast<const void*>(temperature), static_cast<const void*>(top_k),
                            static_cast<const void*>(top_p), static_cast<const void*>(min_p),
                            static_cast<const void*>(u), static_cast<const void*>(tokens_out),
                            static_cast<const void*>(conf_out),
                            static_cast<const void*>(dev_status)})
    if (!aligned(words, 4)) return REFLEX_EINVAL;
  const rx::SampleArgs a{logits, ld, rows,   vocab,      temperature, top_k, top_p,
                         min_p,  u,  masked, tokens_out, conf_out,
                         reinterpret_cast<uint32_t*>(dev_status)};
  RX_CUDA(rx::launch_sample(dtype, a, rx::device_sms(), static_cast<cudaStream_t>(stream)));
  return REFLEX_OK;
}

}  // extern "C"
