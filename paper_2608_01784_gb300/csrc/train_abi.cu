// train_abi.cu — C entry points of what stands around the experts, with gradients:
// norms around a block, tokens to experts and back, the loss of a vocabulary head.
// Argument checks and workspace carving; the kernels are in block_norm.cu,
// expert_rows.cu and head_loss.cu.
#include <limits.h>

#include <algorithm>
#include <cmath>

#include "common.cuh"
#include "internal.h"
#include "reflex.h"

namespace rx {
PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder();
int device_sms();
}  // namespace rx

namespace {

constexpr size_t kAlign = 256;
size_t up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

#define RX_CUDA(x)                                  \
  do {                                              \
    if ((x) != cudaSuccess) return REFLEX_ECUDA;    \
  } while (0)

bool dtype_ok(int32_t t) { return t == REFLEX_DTYPE_F32 || t == REFLEX_DTYPE_BF16; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// A matrix argument: a pointer on its element's boundary and rows that hold `cols`.
struct Matrix {
  const void* p;
  int64_t ld;
};
bool matrix_ok(const Matrix& m, int64_t cols, size_t es) {
  return m.p != nullptr && aligned(m.p, es) && m.ld >= cols;
}

// Whether two matrices share bytes. Rows of one pitch may lie between one another (halves
// of wider rows); ranges of different pitches that cross count as shared.
bool overlap(const Matrix& a, int64_t rows_a, size_t es_a, const Matrix& b, int64_t rows_b,
             size_t es_b, int64_t cols) {
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  const uint64_t pitch_a = a.ld * es_a, pitch_b = b.ld * es_b;
  const uint64_t row_a = cols * es_a, row_b = cols * es_b;
  if (pa + (rows_a - 1) * pitch_a + row_a <= pb || pb + (rows_b - 1) * pitch_b + row_b <= pa)
    return false;
  if (pitch_a != pitch_b) return true;
  const uint64_t off = pb >= pa ? (pb - pa) % pitch_a : (pitch_a - (pa - pb) % pitch_a) % pitch_a;
  return off < row_a || off + row_b > pitch_a;
}

bool norm_ok(int32_t dtype, const Matrix& h, const Matrix& y, const void* w_after,
             const Matrix& gate, const void* w_before, float scale, float eps, int64_t rows,
             int32_t d) {
  if (!dtype_ok(dtype) || rows < 0 || d < 1 || !std::isfinite(scale) || !(eps >= 0.f) ||
      !std::isfinite(eps))
    return false;
  const size_t es = dtype == REFLEX_DTYPE_F32 ? 4 : 2;
  // what scales the block's output needs one
  if (rows > 0 && y.p == nullptr && (w_after != nullptr || gate.p != nullptr)) return false;
  if (rows > 0 && !matrix_ok(h, d, es)) return false;
  if (rows > 0 && y.p != nullptr && !matrix_ok(y, d, es)) return false;
  if (gate.p != nullptr && ((gate.ld != 0 && gate.ld < d) || !aligned(gate.p, es))) return false;
  return aligned(w_after, es) && aligned(w_before, es);
}

bool plan_ok(int64_t T, int32_t E, int32_t k_max) {
  return T >= 0 && E >= 1 && E <= 1024 && k_max >= 1 && k_max <= 32 &&
         T <= (int64_t{1} << 30) / k_max;
}
constexpr int32_t kRowMost = 1 << 30;  // columns of a row: what lies a few steps on fits 31 bits
bool rows_ok(int32_t dtype, int64_t T, int32_t d, int32_t k_max, int64_t cap_rows) {
  return dtype_ok(dtype) && d >= 1 && plan_ok(T, 1, k_max) && cap_rows >= 0 &&
         cap_rows <= INT32_MAX;
}

using rx::kHeadTile;
constexpr int32_t kHeadMost = 1 << 24;  // rows, and columns of the vocabulary

int64_t tiles(int64_t n) { return (n + kHeadTile - 1) / kHeadTile; }
bool head_size_ok(int32_t rows, int32_t vocab, int32_t k) {
  return rows >= 0 && vocab >= 1 && k >= 1;
}
bool head_size_fits(int32_t rows, int32_t vocab, int32_t k) {
  return rows <= kHeadMost && vocab <= kHeadMost && k <= (1 << 20) &&
         tiles(rows) * tiles(vocab) <= (1 << 30);
}
bool head_ok(const void* hidden, int64_t ld_hidden, const void* w, int64_t ldw,
             const int32_t* targets, int32_t rows, int32_t vocab, int32_t k) {
  if (!head_size_ok(rows, vocab, k) || w == nullptr || !aligned(w, 16) || ldw < k || ldw % 8 != 0)
    return false;
  return rows == 0 || (matrix_ok({hidden, ld_hidden}, k, 2) && targets != nullptr &&
                       aligned(targets, 4));
}

// What both directions keep of the rows that count.
struct HeadLayout {
  size_t live, queue, row, target, packed, z_target, stats;  // forward
  size_t row_lse, row_grad, target_term, place, g, sums;     // backward
  size_t total;
  int64_t rows_up, ld_packed, ld_sums;
  int n_queue, piece_tiles, pieces, part_blocks, parts;
};
struct Carve {
  size_t at = 0;
  size_t operator()(size_t bytes) {
    const size_t here = at;
    at += up(bytes);
    return here;
  }
};
HeadLayout head_layout(int64_t rows, int64_t vocab, int64_t k, bool backward) {
  HeadLayout L{};
  L.rows_up = tiles(rows) * kHeadTile;
  L.ld_packed = (k + 7) / 8 * 8;
  L.ld_sums = (k + 31) / 32 * 32;
  L.n_queue = L.pieces = 1;
  const int64_t vt = tiles(vocab);
  if (backward) {
    // pieces of G of up to 512 MB, two of them: 8192 rows x 131072 x 2048 11.11 ms in pieces of
    // 128 MB, 10.95 of 256, 10.85 of 512 (fewer launches, each with a tail; pieces that fit
    // the L2, 32 and 64 MB, take longer)
    const int64_t column = std::max<int64_t>(1, L.rows_up) * kHeadTile * 2;  // of tiles: bytes
    const int64_t most = std::max<int64_t>(1, (int64_t{512} << 20) / column);
    L.piece_tiles = static_cast<int>(std::min(most, vt));
    L.pieces = static_cast<int>((vt + L.piece_tiles - 1) / L.piece_tiles);
    L.n_queue = L.pieces + 1;
    // parts of Dh: enough tiles for all pairs of SMs, so that none is long for the launch
    const int64_t mt = tiles(rows), kt = tiles(k), blocks = L.piece_tiles * (kHeadTile / 64);
    const int64_t want = std::min<int64_t>((100 + mt * kt - 1) / std::max<int64_t>(1, mt * kt), 64);
    L.part_blocks = static_cast<int>((blocks + want - 1) / want);
    L.parts = static_cast<int>((blocks + L.part_blocks - 1) / L.part_blocks);
  }
  Carve take;
  L.live = take(sizeof(int));
  L.queue = take(static_cast<size_t>(L.n_queue) * 4);
  L.row = take(rows * 4);
  L.target = take(L.rows_up * 4);
  L.packed = take(L.rows_up * L.ld_packed * 2);
  if (!backward) {
    L.z_target = take(L.rows_up * 4);
    const int64_t stats = rx::head_few_rows(rows, L.pieces)
                              ? int64_t{rx::head_few_ctas(static_cast<int>(vocab), rx::device_sms())} *
                                    rx::head_few_columns(rows)
                              : 2 * vt * L.rows_up;
    L.stats = take(stats * sizeof(float2));
  } else {
    L.row_lse = take(L.rows_up * 4);
    L.row_grad = take(L.rows_up * 4);
    L.target_term = take(L.rows_up * 4);
    L.place = take(rows * 4);
    const int buffers = L.piece_tiles < vt ? 2 : 1;
    L.g = take(buffers * L.rows_up * L.piece_tiles * kHeadTile * 2);
    L.sums = take(L.parts * L.rows_up * L.ld_sums * 4);
  }
  L.total = take.at;
  return L;
}
template <typename T>
T* at(void* ws, size_t offset) {
  return reinterpret_cast<T*>(static_cast<uint8_t*>(ws) + offset);
}
rx::HeadRows head_rows(const HeadLayout& L, void* ws, const void* hidden, int64_t ld_hidden,
                       const void* w, int64_t ldw, const int32_t* targets, int32_t rows,
                       int32_t vocab, int32_t k, int32_t* dev_status) {
  rx::HeadRows r{};
  r.w = static_cast<const __nv_bfloat16*>(w);
  r.ldw = ldw;
  r.rows = rows;
  r.vocab = vocab;
  r.k = k;
  r.targets = targets;
  r.hidden = static_cast<const __nv_bfloat16*>(hidden);
  r.ld_hidden = ld_hidden;
  r.packed = at<__nv_bfloat16>(ws, L.packed);
  r.ld_packed = L.ld_packed;
  r.row = at<int>(ws, L.row);
  r.target = at<int>(ws, L.target);
  r.live = at<int>(ws, L.live);
  r.queue = at<uint32_t>(ws, L.queue);
  r.n_queue = L.n_queue;
  r.err = reinterpret_cast<uint32_t*>(dev_status);
  // (the products of a few rows take 64 at a time)
  r.tile = rx::head_few_rows(rows, L.pieces) ? rx::kHeadFewRows : kHeadTile;
  return r;
}
rx::HeadTiles head_tiles(const HeadLayout& L, const rx::HeadRows& r) {
  rx::HeadTiles t{};
  t.rows = static_cast<int>(r.rows);
  t.vocab = r.vocab;
  t.k = r.k;
  t.rows_up = static_cast<int>(L.rows_up);
  t.live = r.live;
  t.packed = r.packed;
  t.ld_packed = r.ld_packed;
  t.row = r.row;
  t.target = r.target;
  t.queue = r.queue;
  t.err = r.err;
  return t;
}

}  // namespace

extern "C" {

int reflex_block_norm(int32_t dtype, const void* h, int64_t ldh, const void* y, int64_t ldy,
                      const void* w_after, const void* gate, int64_t ldg, const void* w_before,
                      float scale, float eps, int64_t rows, int32_t d, void* out, int64_t ldo,
                      void* norm, int64_t ldn, void* stream) {
  if (!norm_ok(dtype, {h, ldh}, {y, ldy}, w_after, {gate, ldg}, w_before, scale, eps, rows, d) ||
      (norm != nullptr && w_before == nullptr) ||
      (rows > 0 && out == nullptr && norm == nullptr))
    return REFLEX_EINVAL;
  const size_t es = dtype == REFLEX_DTYPE_F32 ? 4 : 2;
  if ((out != nullptr && !matrix_ok({out, ldo}, d, es)) ||
      (norm != nullptr && !matrix_ok({norm, ldn}, d, es)))
    return REFLEX_EINVAL;
  if (d > rx::block_norm_max_width()) return REFLEX_EUNSUPPORTED;
  if (rows == 0) return REFLEX_OK;
  rx::BlockNormArgs a{};
  a.rows = rows;
  a.d = d;
  a.scale = scale;
  a.eps = eps;
  a.h = h;
  a.ldh = ldh;
  a.y = y;
  a.ldy = ldy;
  a.w_after = w_after;
  a.gate = gate;
  a.ldg = ldg;
  a.w_before = norm != nullptr ? w_before : nullptr;
  a.out = out;
  a.ldo = ldo;
  a.norm = norm;
  a.ldn = ldn;
  RX_CUDA(rx::launch_block_norm(dtype, a, false, rx::device_sms(),
                                static_cast<cudaStream_t>(stream)));
  return REFLEX_OK;
}

size_t reflex_block_norm_workspace_size(int64_t rows, int32_t d) {
  if (rows < 0 || d < 1 || d > rx::block_norm_max_width()) return 0;
  const int64_t parts = std::max<int64_t>(1, rx::block_norm_parts(rows, d, rx::device_sms()));
  return up(3 * static_cast<size_t>(parts) * d * sizeof(float));
}

int reflex_block_norm_backward(int32_t dtype, const void* h, int64_t ldh, const void* y,
                               int64_t ldy, const void* w_after, const void* gate, int64_t ldg,
                               const void* w_before, float scale, float eps, int64_t rows,
                               int32_t d, const void* d_out, int64_t ld_d_out,
                               const void* d_norm, int64_t ld_d_norm, void* d_h, int64_t ld_d_h,
                               void* d_y, int64_t ld_d_y, void* d_gate, int64_t ld_d_gate,
                               void* d_w_after, void* d_w_before, void* workspace,
                               size_t ws_bytes, void* stream) {
  if (!norm_ok(dtype, {h, ldh}, {y, ldy}, w_after, {gate, ldg}, w_before, scale, eps, rows, d) ||
      (rows > 0 && ((d_norm != nullptr) != (w_before != nullptr) ||
                    (d_out == nullptr && d_norm == nullptr))) ||
      (d_w_after != nullptr && w_after == nullptr) || (d_gate != nullptr && gate == nullptr) ||
      (d_w_before != nullptr && w_before == nullptr))
    return REFLEX_EINVAL;
  const size_t es = dtype == REFLEX_DTYPE_F32 ? 4 : 2;
  if (rows > 0 && (!matrix_ok({d_h, ld_d_h}, d, es) ||
                   (d_out != nullptr && !matrix_ok({d_out, ld_d_out}, d, es)) ||
                   (d_norm != nullptr && !matrix_ok({d_norm, ld_d_norm}, d, es)) ||
                   (y != nullptr && !matrix_ok({d_y, ld_d_y}, d, es)) ||
                   (d_gate != nullptr && ldg != 0 && ld_d_gate < d)))
    return REFLEX_EINVAL;
  if (!aligned(d_gate, es) || !aligned(d_w_after, es) || !aligned(d_w_before, es))
    return REFLEX_EINVAL;
  if (d > rx::block_norm_max_width()) return REFLEX_EUNSUPPORTED;
  if (workspace == nullptr || ws_bytes < reflex_block_norm_workspace_size(rows, d) ||
      !aligned(workspace, kAlign))
    return REFLEX_EWORKSPACE;
  rx::BlockNormArgs a{};
  a.rows = rows;
  a.d = d;
  a.scale = scale;
  a.eps = eps;
  a.h = h;
  a.ldh = ldh;
  a.y = y;
  a.ldy = ldy;
  a.w_after = w_after;
  a.gate = gate;
  a.ldg = ldg;
  a.w_before = w_before;
  a.d_out = d_out;
  a.ld_d_out = ld_d_out;
  a.d_norm = d_norm;
  a.ld_d_norm = ld_d_norm;
  a.d_h = d_h;
  a.ld_d_h = ld_d_h;
  a.d_y = d_y;
  a.ld_d_y = ld_d_y;
  a.d_gate = d_gate;
  a.ld_d_gate = ld_d_gate;
  a.d_w_after = d_w_after;
  a.d_w_before = d_w_before;
  a.partial = static_cast<float*>(workspace);
  RX_CUDA(rx::launch_block_norm(dtype, a, true, rx::device_sms(),
                                static_cast<cudaStream_t>(stream)));
  return REFLEX_OK;
}

size_t reflex_expert_plan_workspace_size(int64_t T, int32_t E, int32_t k_max) {
  if (!plan_ok(T, E, k_max)) return 0;
  return up(static_cast<size_t>(rx::expert_plan_blocks_most(T * k_max, rx::device_sms())) * E * 4);
}

int reflex_expert_plan(const int32_t* ids, const int32_t* k, int64_t T, int32_t E, int32_t k_max,
                       int64_t cap_rows, int32_t* row_of, int32_t* counts, int32_t* offsets,
                       int32_t* perm, int32_t* dev_status, void* workspace, size_t ws_bytes,
                       void* stream) {
  if (!plan_ok(T, E, k_max) || cap_rows < 0) return REFLEX_EINVAL;
  if (counts == nullptr || offsets == nullptr || (T > 0 && (ids == nullptr || row_of == nullptr)))
    return REFLEX_EINVAL;
  for (const void* p : {static_cast<const void*>(ids), static_cast<const void*>(k),
                        static_cast<const void*>(row_of), static_cast<const void*>(counts),
                        static_cast<const void*>(offsets), static_cast<const void*>(perm),
                        static_cast<const void*>(dev_status)})
    if (!aligned(p, 4)) return REFLEX_EINVAL;
  if (workspace == nullptr || ws_bytes < reflex_expert_plan_workspace_size(T, E, k_max) ||
      !aligned(workspace, kAlign))
    return REFLEX_EWORKSPACE;
  const int cap = static_cast<int>(std::min<int64_t>(cap_rows, INT32_MAX));
  RX_CUDA(rx::launch_expert_plan(ids, k, T, E, k_max, cap, row_of, counts, offsets, perm,
                                 reinterpret_cast<uint32_t*>(dev_status),
                                 static_cast<int32_t*>(workspace), rx::device_sms(),
                                 static_cast<cudaStream_t>(stream)));
  return REFLEX_OK;
}

int reflex_expert_rows(int32_t dtype, const void* x, int64_t ldx, const int32_t* row_of,
                       int64_t T, int32_t d, int32_t k_max, int64_t cap_rows, void* rows,
                       int64_t ldr, void* stream) {
  if (!rows_ok(dtype, T, d, k_max, cap_rows)) return REFLEX_EINVAL;
  if (T == 0 || cap_rows == 0) return REFLEX_OK;
  if (d > kRowMost) return REFLEX_EUNSUPPORTED;
  const size_t es = dtype == REFLEX_DTYPE_F32 ? 4 : 2;
  if (!matrix_ok({x, ldx}, d, es) || !matrix_ok({rows, ldr}, d, es) || row_of == nullptr ||
      !aligned(row_of, 4))
    return REFLEX_EINVAL;
  rx::ExpertRowsArgs a{};
  a.row_of = row_of;
  a.T = T;
  a.d = d;
  a.k_max = k_max;
  a.cap_rows = static_cast<int>(cap_rows);
  a.x = x;
  a.ldx = ldx;
  a.out = rows;
  a.ldo = ldr;
  RX_CUDA(rx::launch_expert_rows(dtype, a, rx::device_sms(), static_cast<cudaStream_t>(stream)));
  return REFLEX_OK;
}

int reflex_expert_combine(int32_t dtype, const void* rows, int64_t ldr, const float* alpha,
                          const int32_t* row_of, const void* residual, int64_t ldres, int64_t T,
                          int32_t d, int32_t k_max, int64_t cap_rows, void* out, int64_t ldo,
                          void* stream) {
  if (!rows_ok(dtype, T, d, k_max, cap_rows)) return REFLEX_EINVAL;
  if (T == 0) return REFLEX_OK;
  if (d > kRowMost) return REFLEX_EUNSUPPORTED;
  const size_t es = dtype == REFLEX_DTYPE_F32 ? 4 : 2;
  if (!matrix_ok({out, ldo}, d, es) || (cap_rows > 0 && !matrix_ok({rows, ldr}, d, es)) ||
      (residual != nullptr && !matrix_ok({residual, ldres}, d, es)) || row_of == nullptr ||
      !aligned(row_of, 4) || !aligned(alpha, 4))
    return REFLEX_EINVAL;
  rx::ExpertRowsArgs a{};
  a.row_of = row_of;
  a.T = T;
  a.d = d;
  a.k_max = k_max;
  a.cap_rows = static_cast<int>(cap_rows);
  a.x = residual;
  a.ldx = ldres;
  a.rows = rows;
  a.ldr = ldr;
  a.alpha = alpha;
  a.out = out;
  a.ldo = ldo;
  RX_CUDA(rx::launch_expert_combine(dtype, a, false, rx::device_sms(),
                                    static_cast<cudaStream_t>(stream)));
  return REFLEX_OK;
}

int reflex_expert_combine_backward(int32_t dtype, const void* d_out, int64_t ld_d_out,
                                   const void* rows, int64_t ldr, const float* alpha,
                                   const int32_t* row_of, int64_t T, int32_t d, int32_t k_max,
                                   int64_t cap_rows, void* d_rows, int64_t ld_d_rows,
                                   float* d_alpha, void* stream) {
  if (!rows_ok(dtype, T, d, k_max, cap_rows)) return REFLEX_EINVAL;
  if (T == 0) return REFLEX_OK;
  if (d > kRowMost) return REFLEX_EUNSUPPORTED;
  const size_t es = dtype == REFLEX_DTYPE_F32 ? 4 : 2;
  if (!matrix_ok({d_out, ld_d_out}, d, es) || alpha == nullptr || row_of == nullptr ||
      (d_rows == nullptr && d_alpha == nullptr) || !aligned(row_of, 4) || !aligned(alpha, 4) ||
      !aligned(d_alpha, 4))
    return REFLEX_EINVAL;
  if (cap_rows > 0 && ((d_rows != nullptr && !matrix_ok({d_rows, ld_d_rows}, d, es)) ||
                       (d_alpha != nullptr && !matrix_ok({rows, ldr}, d, es))))
    return REFLEX_EINVAL;
  rx::ExpertRowsArgs a{};
  a.row_of = row_of;
  a.T = T;
  a.d = d;
  a.k_max = k_max;
  a.cap_rows = static_cast<int>(cap_rows);
  a.x = d_out;
  a.ldx = ld_d_out;
  a.rows = rows;
  a.ldr = ldr;
  a.alpha = alpha;
  a.out = d_rows;
  a.ldo = ld_d_rows;
  a.d_alpha = d_alpha;
  RX_CUDA(rx::launch_expert_combine(dtype, a, true, rx::device_sms(),
                                    static_cast<cudaStream_t>(stream)));
  return REFLEX_OK;
}

size_t reflex_head_loss_workspace_size(int32_t rows, int32_t vocab, int32_t k) {
  if (!head_size_ok(rows, vocab, k) || !head_size_fits(rows, vocab, k)) return 0;
  return head_layout(rows, vocab, k, false).total;
}

int reflex_head_loss(const void* hidden, int64_t ld_hidden, const void* w, int64_t ldw,
                     const int32_t* targets, int32_t rows, int32_t vocab, int32_t k, float* loss,
                     float* lse, int32_t* dev_status, void* workspace, size_t ws_bytes,
                     void* stream) {
  if (!head_ok(hidden, ld_hidden, w, ldw, targets, rows, vocab, k) || !aligned(dev_status, 4) ||
      (rows > 0 && (loss == nullptr || lse == nullptr)) || !aligned(loss, 4) || !aligned(lse, 4))
    return REFLEX_EINVAL;
  if (!head_size_fits(rows, vocab, k)) return REFLEX_EUNSUPPORTED;
  const HeadLayout L = head_layout(rows, vocab, k, false);
  if (workspace == nullptr || ws_bytes < L.total || !aligned(workspace, kAlign))
    return REFLEX_EWORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    if (dev_status != nullptr) RX_CUDA(cudaMemsetAsync(dev_status, 0, sizeof(int32_t), s));
    return REFLEX_OK;
  }
  const auto encode = rx::tensor_map_encoder();
  if (encode == nullptr) return REFLEX_ECUDA;
  const int sms = rx::device_sms();
  rx::HeadRows r =
      head_rows(L, workspace, hidden, ld_hidden, w, ldw, targets, rows, vocab, k, dev_status);
  r.z_target = at<float>(workspace, L.z_target);
  r.loss_out = loss;
  r.lse_out = lse;
  RX_CUDA(rx::launch_head_rows(r, sms, s));
  rx::HeadTiles t = head_tiles(L, r);
  t.z_target = r.z_target;
  t.stats = at<float2>(workspace, L.stats);
  t.ld_stats = L.rows_up;
  RX_CUDA(rx::launch_head_loss({encode, r.packed, L.ld_packed, w, ldw}, t, loss, lse, sms, s));
  return REFLEX_OK;
}

size_t reflex_head_loss_backward_workspace_size(int32_t rows, int32_t vocab, int32_t k) {
  if (!head_size_ok(rows, vocab, k) || !head_size_fits(rows, vocab, k)) return 0;
  return head_layout(rows, vocab, k, true).total;
}

int reflex_head_loss_backward(const void* hidden, int64_t ld_hidden, const void* w, int64_t ldw,
                              const int32_t* targets, const float* lse, const float* grad,
                              int32_t rows, int32_t vocab, int32_t k, int32_t d_hidden_dtype,
                              void* d_hidden, int64_t ld_d_hidden, int32_t d_w_dtype, void* d_w,
                              int64_t ld_d_w, int32_t* dev_status, void* workspace,
                              size_t ws_bytes, void* stream) {
  if (!head_ok(hidden, ld_hidden, w, ldw, targets, rows, vocab, k) || !aligned(dev_status, 4) ||
      (rows > 0 && (lse == nullptr || grad == nullptr)) || !aligned(lse, 4) || !aligned(grad, 4) ||
      (rows > 0 && d_hidden == nullptr && d_w == nullptr))
    return REFLEX_EINVAL;
  if (!dtype_ok(d_hidden_dtype) || !dtype_ok(d_w_dtype)) return REFLEX_EINVAL;
  const size_t es_h = d_hidden_dtype == REFLEX_DTYPE_F32 ? 4 : 2;
  const size_t es_w = d_w_dtype == REFLEX_DTYPE_F32 ? 4 : 2;
  if ((d_hidden != nullptr && !matrix_ok({d_hidden, ld_d_hidden}, k, es_h)) ||
      (d_w != nullptr && !matrix_ok({d_w, ld_d_w}, k, es_w)))
    return REFLEX_EINVAL;
  if (!head_size_fits(rows, vocab, k)) return REFLEX_EUNSUPPORTED;
  const HeadLayout L = head_layout(rows, vocab, k, true);
  if (workspace == nullptr || ws_bytes < L.total || !aligned(workspace, kAlign))
    return REFLEX_EWORKSPACE;
  // (the weights are still read while either gradient is written)
  const Matrix weights{w, ldw}, dw{d_w, ld_d_w}, dh{rows > 0 ? d_hidden : nullptr, ld_d_hidden};
  if ((d_w != nullptr && overlap(weights, vocab, 2, dw, vocab, es_w, k)) ||
      (dh.p != nullptr && overlap(weights, vocab, 2, dh, rows, es_h, k)) ||
      (d_w != nullptr && dh.p != nullptr && overlap(dw, vocab, es_w, dh, rows, es_h, k)))
    return REFLEX_EINVAL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    if (dev_status != nullptr) RX_CUDA(cudaMemsetAsync(dev_status, 0, sizeof(int32_t), s));
    if (d_w != nullptr)
      RX_CUDA(cudaMemset2DAsync(d_w, ld_d_w * es_w, 0, k * es_w, vocab, s));
    return REFLEX_OK;
  }
  const auto encode = rx::tensor_map_encoder();
  if (encode == nullptr) return REFLEX_ECUDA;
  const int sms = rx::device_sms();
  rx::HeadRows r =
      head_rows(L, workspace, hidden, ld_hidden, w, ldw, targets, rows, vocab, k, dev_status);
  r.lse = lse;
  r.grad = grad;
  r.row_lse = at<float>(workspace, L.row_lse);
  r.row_grad = at<float>(workspace, L.row_grad);
  r.target_term = at<float>(workspace, L.target_term);
  r.place = at<int>(workspace, L.place);
  RX_CUDA(rx::launch_head_rows(r, sms, s));
  rx::HeadTiles t = head_tiles(L, r);
  t.row_lse = r.row_lse;
  t.row_grad = r.row_grad;
  t.target_term = r.target_term;
  t.dw = d_w;
  t.ld_dw = ld_d_w;
  t.dw_f32 = d_w_dtype == REFLEX_DTYPE_F32;
  t.ld_sums = static_cast<int>(L.ld_sums);
  const rx::HeadPieces q{L.piece_tiles, L.part_blocks, L.parts,
                         at<__nv_bfloat16>(workspace, L.g),
                         d_hidden != nullptr ? at<float>(workspace, L.sums) : nullptr};
  RX_CUDA(rx::launch_head_loss_backward({encode, r.packed, L.ld_packed, w, ldw}, t, q, r.place,
                                        rows, d_hidden, ld_d_hidden,
                                        d_hidden_dtype == REFLEX_DTYPE_F32, sms, s));
  return REFLEX_OK;
}

}  // extern "C"
