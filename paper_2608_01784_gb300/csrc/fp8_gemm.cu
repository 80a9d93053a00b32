// fp8_gemm.cu — products of e4m3 codes with one fp32 scale for each block of
// 128, on the 5th-generation tensor cores, dense or grouped by expert.
//
//   D[r, c] = sum_kb sa[r, kb] * sb[c / 128, kb] * sum_{k in kb} A[r, k] B[c, k]
//   matmul: out = D (bf16 or fp32);
//   SwiGLU: act = silu(D gate) * (D up), quantised again: codes and a scale
//           for each 128 columns of act, the next product's A.
//
// The tensor cores sum one block of K (128) at a time: four
// tcgen05.mma.kind::f8f6f4 of K = 32 into a fresh TMEM accumulator.  Its
// products by the two scales are added to fp32 accumulators in registers,
// because neither scale is constant along K and neither need be a power of
// two.  Two TMEM accumulators of 256 columns (all 512) alternate, so that the
// MMAs of the next block run while the last one is read.
//
// Tiles: 128 rows of A x 256 rows of B (SwiGLU: 128 gate rows and the matching
// 128 up rows, hence whole groups of act columns in one CTA), taken from a grid of
// one CTA an SM.
//   warp 0      TMA producer: ring of three 48 KB stages, 128-byte swizzle;
//   warp 1      allocates TMEM, issues the MMAs;
//   warp 2      the tiles and their scales, up to 16 blocks of K ahead;
//   warp 3      TMA stores of finished tiles (bf16, act codes), which lie staged in
//               64 KB while the next tile is summed;
//   warps 4-11  two warpgroups, each thread one row and 64 + 64 columns (64
//               of either 128-row half of B): 128 accumulators in registers.
// Split tiles (few tiles, long K, dense only): the CTAs of a cluster take a part
// of K each and add their accumulators through distributed shared memory, 32 rows
// at a time in rank order, so the sums do not depend on timing.
//
// Bound: for many rows the sums in registers, and close behind them the codes'
// way from L2.  The MMAs of a block take 520 cycles; the eight warps that read it
// back (128 KB), scale it and hand the accumulator on take about 1000, of which the
// reads and FMAs by themselves are 340 and the rest are latencies of two barriers,
// of the scales' reads and of TMEM that two warps a scheduler cannot hide.
// 8192 x 8192 x 8192: 452 us, 2.43 PFLOP/s, on one card, 485 on the one that these
// were timed on: with a quarter of the MMAs 475, without the sums 426, without these
// and the loads of B 358, so no one of them is the limit by itself.  Sixteen warps of 64
// accumulators took 552 us (the same latencies by twice the warps); CTA pairs on a
// tile of 256 rows, accumulators of 128 columns, scalar FMAs and reading the next
// block's scales ahead were no faster as they were tried.  fp32 out (stored by the
// summing warps): 483 us where bf16 takes 452.  For few rows the weights' bytes:
// 32 x 50000 x 2048 30 us, of which the bytes take 16.
//
// Short K (512 in a down product) shows what a tile costs besides its blocks: finding
// it takes some 2000 cycles (warps 0 and 2 do it ahead) and storing it 8000 by one
// warp's vectors, 900 to 3000 by TMA.  61,000 pairs of 256 experts, d = 2048, inter
// = 512: layer 458 us without these two, 385 with.
//
// Every wait on a barrier in shared memory is bounded (2 s); on expiry the CTA records
// the timeout in the error word, drains its loads and MMAs, frees TMEM and exits.  The
// two barriers of a cluster (its CTAs run together; each comes to the last one past
// bounded waits alone) have no limit.
#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"
#include "tcgen05.cuh"

namespace rx {
namespace {

constexpr int BM = 128;
constexpr int BN = 256;
constexpr int kHalfB = BN / 2 * 128;  // 128 rows of B
constexpr int kABytes = BM * 128;
constexpr int kBBytes = 2 * kHalfB;
constexpr int kStages = 3;
// a staged tile, boxes of 128 rows x 128 bytes with the swizzle of the stages: bf16
// four of them, act codes one; else 32 rows x 256 fp32, or 4 KB a warp
constexpr int kBoxOut = BM * 128;
constexpr int kStageOut = 4 * kBoxOut;
constexpr int kScaleChunk = 16;  // blocks of K whose scales are fetched together
constexpr int kScaleBytes = 2 * kScaleChunk * (BM + 2) * 4;
constexpr int kIndexInts = 320;
constexpr int kBarBytes = 256;
constexpr int kSmemBytes = kStages * (kABytes + kBBytes) + kStageOut + kScaleBytes + kBarBytes +
                           kIndexInts * 4 + 1024;
static_assert(kSmemBytes <= 227 * 1024, "shared memory of one CTA");
// 384 x 168 registers at launch = 128 x 56 + 256 x 224 after the split
constexpr int kThreads = 384;
constexpr int kFirstPromoter = 4;
constexpr int kPromoters = 8;
constexpr int kGroupM = 32;  // m-tiles whose rows stay in L2 across the n-tiles
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr uint64_t kDrainNs = 1000000000ull;

enum { kSwiGLU = 0, kMatmul = 1 };

struct Params {
  int nkb;
  int n_out;
  int n_tiles;
  GroupRows g;
  int max_mtiles;
  int a_box;
  const uint8_t* a_scales;
  int64_t a_scale_row_bytes;
  const float* b_scales;
  int64_t b_scale_group;
  int64_t b_scale_ld;
  void* out;
  int64_t ldo;
  int out_f32;
  int staged;   // out goes through shared memory and map_out
  int out_vec;  // rows of out start on 16-byte boundaries
  int64_t scale_offset;  // SwiGLU: the scales' place in a packed row
  int splits;
  uint32_t* err;
};

// kind::f8f6f4: e4m3 A and B (types 0), fp32 accumulator, both K-major.
constexpr uint32_t kIdesc = (1u << 4) | (static_cast<uint32_t>(BN >> 3) << 17) |
                            (static_cast<uint32_t>(BM >> 4) << 24);
__device__ __forceinline__ void mma_e4m3(uint32_t tmem_d, uint64_t da, uint64_t db,
                                         uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(tmem_d),
      "l"(da), "l"(db), "r"(kIdesc), "r"(accumulate)
      : "memory");
}

// One lane of a converged warp.
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t e;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}\n"
      : "=r"(e));
  return e;
}

// Two fp32 in one 64-bit register: one FMA instruction for both.
__device__ __forceinline__ uint64_t pack2(uint32_t lo, uint32_t hi) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(lo), "r"(hi));
  return v;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  uint32_t lo, hi;
  asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(v));
  return make_float2(__uint_as_float(lo), __uint_as_float(hi));
}
// Waits for the TMEM loads in flight; r passes through, so that no use of it is
// moved in front of the wait.
__device__ __forceinline__ void tmem_ld_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]),
                 "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                 "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                 "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]),
                 "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]),
                 "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}
// acc += r * s, 32 columns of a row.
__device__ __forceinline__ void scaled_add(uint64_t* acc, const uint32_t (&r)[32], uint64_t s2) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint64_t x = pack2(r[2 * i], r[2 * i + 1]);
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc[i]) : "l"(x), "l"(s2));
  }
}

// A box of shared memory to global memory, clipped to the map's extents.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t from, int c0,
                                             int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map),
      "r"(from), "r"(c0), "r"(c1)
      : "memory");
}

// ---- clusters ---------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t saddr, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(saddr), "r"(rank));
  return a;
}
__device__ __forceinline__ void mbar_arrive_peer(uint32_t peer_bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(peer_bar)
               : "memory");
}
__device__ __forceinline__ float4 ld_peer4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();  // the barrier takes whole warps, whatever branch a lane comes from
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// mbar_wait for arrivals from the other CTAs of the cluster.
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t* bar, uint32_t parity,
                                                  const volatile int* abort) {
  const uint64_t t0 = global_ns();
  while (true) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}\n"
        : "=r"(ok)
        : "r"(smem_addr(bar)), "r"(parity)
        : "memory");
    if (ok) return true;
    if (*abort || global_ns() - t0 > kWaitNs) return false;
  }
}

// ---- tiles ------------------------------------------------------------------
struct __align__(16) Tile {
  int e, n, row0, rows;
};

// Tile counts per expert in shared memory where they fit; row offsets in L2.
__device__ __forceinline__ const int32_t* load_prefix(const Params& p, int32_t* cache) {
  if (p.g.offsets == nullptr || p.g.E + 1 > kIndexInts) return p.g.mt_prefix;
  for (int i = threadIdx.x; i <= p.g.E; i += kThreads) cache[i] = p.g.mt_prefix[i];
  return cache;  // the caller synchronises
}
__device__ __forceinline__ int tile_count(const Params& p, const int32_t* pref) {
  int mt = p.max_mtiles;
  if (p.g.offsets != nullptr) mt = max(0, min(pref[p.g.E], p.max_mtiles));
  return mt * p.n_tiles;
}
// Dense: n-tile by n-tile over kGroupM m-tiles at a time.  Grouped: expert,
// n-tile, m-tile, so CTAs at work at the same time share weights in L2.
// False: the workspace is inconsistent (in unsigned arithmetic whatever wraps
// fails one of the comparisons).
__device__ __forceinline__ bool decode_tile(const Params& p, const int32_t* pref, int t,
                                            Tile& o) {
  if (p.g.offsets == nullptr) {
    const int per = kGroupM * p.n_tiles;
    const int m0 = t / per * kGroupM, r = t % per;
    const int gm = min(kGroupM, p.max_mtiles - m0);
    o.e = 0;
    o.n = r / gm;
    o.row0 = (m0 + r % gm) * BM;
    o.rows = min(BM, p.g.dense_rows - o.row0);
    return true;
  }
  int lo = 0, hi = p.g.E;  // n_tiles * prefix[lo] <= t < n_tiles * prefix[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.n_tiles * pref[mid] <= t) lo = mid; else hi = mid;
  }
  const uint32_t first = pref[lo], last = pref[lo + 1];
  const uint32_t row_lo = p.g.offsets[lo], row_hi = p.g.offsets[lo + 1];
  const uint32_t mt_e = last - first, most = p.max_mtiles;
  if (mt_e - 1u >= most) return false;
  const uint32_t l = t - p.n_tiles * first, n = l / mt_e;
  const uint32_t row0 = row_lo + (l - n * mt_e) * BM;
  o.e = lo;
  o.n = n;
  o.row0 = row0;
  o.rows = min(static_cast<uint32_t>(BM), row_hi - row0);
  return n < static_cast<uint32_t>(p.n_tiles) && row_lo <= row0 && row0 < row_hi &&
         row_hi <= static_cast<uint32_t>(p.g.cap_rows);
}

// The scales of half h of a tile's columns by blocks of K.  A half past the last
// column has none: its columns are not stored.
__device__ __forceinline__ const float* b_scale_row(const Params& p, int mode, const Tile& tl,
                                                    int h) {
  if (mode == kSwiGLU)
    return p.b_scales + (2 * tl.e + h) * p.b_scale_group + tl.n * p.b_scale_ld;
  const int block = 2 * tl.n + (tl.n * BN + 128 < p.n_out ? h : 0);
  return p.b_scales + tl.e * p.b_scale_group + block * p.b_scale_ld;
}

template <int MODE, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1)
    fp8_gemm_kernel(const __grid_constant__ CUtensorMap map_a,
                    const __grid_constant__ CUtensorMap map_b,
                    const __grid_constant__ CUtensorMap map_out, const Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sa = smem;
  uint8_t* sb = smem + kStages * kABytes;
  uint8_t* patch = smem + kStages * (kABytes + kBBytes);
  float* sc_a = reinterpret_cast<float*>(patch + kStageOut);  // [2][kScaleChunk][BM]
  float* sc_b = sc_a + 2 * kScaleChunk * BM;                  // [2][kScaleChunk][2]
  uint64_t* bars = reinterpret_cast<uint64_t*>(patch + kStageOut + kScaleBytes);
  uint64_t* full = bars;                 // [kStages]
  uint64_t* empty = bars + kStages;      // [kStages]
  uint64_t* tfull = bars + 2 * kStages;  // [2] a TMEM accumulator is complete
  uint64_t* tempty = tfull + 2;          // [2] it has been read
  uint64_t* xbar = tempty + 2;           // [4] SwiGLU: row maxima of a quarter's two warps
  uint64_t* red_full = xbar + 4;         // split: every CTA's rows are in its patch
  uint64_t* red_empty = red_full + 1;    // split: every CTA has read them
  uint64_t* sfull = red_empty + 1;       // [2] a chunk of scales is in place
  uint64_t* sempty = sfull + 2;          // [2] it has been used
  uint64_t* ofull = sempty + 2;          // a tile of bf16 is staged
  uint64_t* oempty = ofull + 1;          // it has been stored
  uint64_t* drain = oempty + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  Tile* s_tile = reinterpret_cast<Tile*>(tmem_slot + 2);  // [2] whose scales these are
  Tile* o_tile = s_tile + 2;                              // the staged one
  static_assert(2 * kStages + 17 == 23 && 23 * 8 + 8 + 3 * 16 <= kBarBytes, "barriers");
  int32_t* cache = reinterpret_cast<int32_t*>(bars + kBarBytes / 8);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const int S = SPLIT ? p.splits : 1;
  const int rank = SPLIT ? static_cast<int>(cluster_rank()) : 0;
  const int t_first = blockIdx.x / S, t_step = gridDim.x / S;
  const int kb0 = SPLIT ? p.nkb * rank / S : 0, kb1 = SPLIT ? p.nkb * (rank + 1) / S : p.nkb;
  const bool staged = MODE == kSwiGLU || (!SPLIT && p.staged);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], kPromoters);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&sfull[b], 1);
      mbar_init(&sempty[b], kPromoters);
    }
    mbar_init(ofull, kPromoters);
    mbar_init(oempty, 1);
    for (int q = 0; q < 4; ++q) mbar_init(&xbar[q], 2);
    mbar_init(red_full, 2 * S);
    mbar_init(red_empty, kPromoters * S);
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_map(&map_a);
    prefetch_map(&map_b);
    if (staged) prefetch_map(&map_out);
  }
  if (warp == 1) tmem_alloc(smem_addr(tmem_slot), 2 * BN);
  tc_fence_before();
  if (SPLIT) cluster_sync();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  grid_dep_wait();
  grid_dep_launch();
  const int32_t* pref = load_prefix(p, cache);
  __syncthreads();
  const int ntiles = tile_count(p, pref);

  if (warp < kFirstPromoter) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0 && lane == 0) {
      // ---------------- TMA producer ----------------
      int stage = 0;
      uint32_t phase = 0, issued_mask = 0, issued_phase = 0;
      bool ok = true;
      Tile next;
      bool valid = t_first >= ntiles || decode_tile(p, pref, t_first, next);
      for (int t = t_first; t < ntiles && ok; t += t_step) {
        if (!valid) {
          set_err(p.err, kErrIndex);
          *abort_flag = 1;
          break;
        }
        const Tile tl = next;
        // rows of a box past the tile's last row are of no use: leave them out
        const int boxes = (tl.rows + p.a_box - 1) / p.a_box;
        const int c1 = MODE == kSwiGLU ? tl.n * 128 : tl.n * BN;
        const int c2 = MODE == kSwiGLU ? 2 * tl.e : tl.e;
        const bool second = MODE == kSwiGLU || c1 + 128 < p.n_out;
        const uint32_t bytes = boxes * p.a_box * 128 + (second ? 2 : 1) * kHalfB;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!mbar_wait(&empty[stage], phase ^ 1u, abort_flag, kWaitNs)) {
            ok = false;
            break;
          }
          const uint32_t fb = smem_addr(&full[stage]);
          mbar_expect_tx(fb, bytes);
          const uint32_t a_dst = smem_addr(sa + stage * kABytes);
          const uint32_t b_dst = smem_addr(sb + stage * kBBytes);
          tma_load_3d(b_dst, &map_b, kb * 128, c1, c2, fb);
          if (second)
            tma_load_3d(b_dst + kHalfB, &map_b, kb * 128, MODE == kSwiGLU ? c1 : c1 + 128,
                        MODE == kSwiGLU ? c2 + 1 : c2, fb);
          for (int i = 0; i < boxes; ++i)
            tma_load_2d(a_dst + i * p.a_box * 128, &map_a, kb * 128, tl.row0 + i * p.a_box, fb);
          issued_mask |= 1u << stage;
          issued_phase = (issued_phase & ~(1u << stage)) | (phase << stage);
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
          // (the ring is full: time for the next tile, some 2000 cycles)
          if (kb == min(kb0 + kStages, kb1) - 1 && t + t_step < ntiles)
            valid = decode_tile(p, pref, t + t_step, next);
        }
      }
      if (!ok) {
        set_err(p.err, kErrTimeout);
        *abort_flag = 1;
      }
      if (*abort_flag) {
        // every issued load must land before the CTA may exit
        for (int s = 0; s < kStages; ++s)
          if (issued_mask & (1u << s))
            mbar_wait(&full[s], (issued_phase >> s) & 1u, nullptr, kDrainNs);
      }
    } else if (warp == 1) {
      // ---------------- MMA issuer ----------------
      // The whole warp walks the loop, so that descriptors and addresses stay in
      // uniform registers, as tcgen05.mma takes them; one lane issues.
      const uint32_t elected = elect_one();
      int stage = 0;
      uint32_t phase = 0;
      uint32_t it = 0;
      bool ok = true, issued_any = false;
      const uint64_t da0 = desc_sw128(smem_addr(sa)), db0 = desc_sw128(smem_addr(sb));
      for (int t = t_first; t < ntiles && ok; t += t_step) {
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
          const int b = it & 1;
          ok = mbar_wait(&full[stage], phase, abort_flag, kWaitNs) &&
               mbar_wait(&tempty[b], ((it >> 1) & 1u) ^ 1u, abort_flag, kWaitNs);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          // (addresses count 16 bytes in a descriptor's low bits)
          const uint64_t da = da0 + static_cast<uint32_t>(stage * (kABytes >> 4));
          const uint64_t db = db0 + static_cast<uint32_t>(stage * (kBBytes >> 4));
          const uint32_t d = tmem_base + b * BN;
          if (elected) {
#pragma unroll
            for (int k = 0; k < 4; ++k) mma_e4m3(d, da + 2 * k, db + 2 * k, k > 0 ? 1u : 0u);
            mma_commit(smem_addr(&tfull[b]));
            mma_commit(smem_addr(&empty[stage]));
          }
          issued_any = true;
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      if (!ok && elected) {
        if (!*abort_flag) set_err(p.err, kErrTimeout);
        *abort_flag = 1;
      }
      __syncwarp();
      if (*abort_flag && issued_any && elected) {
        // MMAs in flight must finish before TMEM is freed
        mma_commit(smem_addr(drain));
        mbar_wait(drain, 0, nullptr, kDrainNs);
      }
    } else if (warp == 2) {
      // ---------------- scales ----------------
      // The scales of a row of A are fetched 16 blocks of K ahead, by themselves:
      // global loads in the warps that hand accumulators back delay the hand-over
      // by their latency (8192 x 8192 x 8192: some 30 us).
      uint32_t slot = 0, phase = 0;
      bool ok = true;
      for (int t = t_first; t < ntiles && ok; t += t_step) {
        Tile tl;
        if (!decode_tile(p, pref, t, tl)) break;
        const int rows = tl.rows;
        const float* b0 = b_scale_row(p, MODE, tl, 0);
        const float* b1 = b_scale_row(p, MODE, tl, 1);
        for (int c0 = kb0; c0 < kb1; c0 += kScaleChunk) {
          const int n = min(kScaleChunk, kb1 - c0);
          ok = __all_sync(0xffffffffu, mbar_wait(&sempty[slot], phase ^ 1u, abort_flag, kWaitNs));
          if (!ok) break;
          float* to = sc_a + slot * kScaleChunk * BM + lane;
          const uint8_t* from[BM / 32];
#pragma unroll
          for (int r = 0; r < BM / 32; ++r)
            from[r] = p.a_scales + c0 * 4 +
                      static_cast<int64_t>(tl.row0 + (r * 32 + lane < rows ? r * 32 + lane : 0)) *
                          p.a_scale_row_bytes;
          // (four loads in flight; eight spill)
#pragma unroll 1
          for (int i = 0; i < n; ++i) {
            float v[BM / 32];
#pragma unroll
            for (int r = 0; r < BM / 32; ++r) v[r] = reinterpret_cast<const float*>(from[r])[i];
#pragma unroll
            for (int r = 0; r < BM / 32; ++r) to[i * BM + r * 32] = v[r];
          }
          if (c0 == kb0 && lane == 0) s_tile[slot] = tl;
          if (lane < 2 * n)
            sc_b[slot * kScaleChunk * 2 + lane] = (lane & 1 ? b1 : b0)[c0 + (lane >> 1)];
          __syncwarp();
          if (lane == 0) mbar_arrive1(smem_addr(&sfull[slot]));
          slot ^= 1u;
          if (slot == 0) phase ^= 1u;
        }
      }
      if (!ok && lane == 0) {
        if (!*abort_flag) set_err(p.err, kErrTimeout);
        *abort_flag = 1;
      }
    } else if (warp == 3 && staged) {
      // ---------------- stores of staged tiles ----------------
      // (while the next tile is summed: boxes of 32 rows, of a group's last rows each
      // by itself, because another group's follow them)
      constexpr int kBoxes = MODE == kSwiGLU ? 1 : 4;  // of 128 bytes across
      constexpr int kEach = MODE == kSwiGLU ? 128 : 64;
      // the map ends with the last whole 16 bytes of a row: a box is clipped in units of
      // these, and would write over what follows the row
      const int whole_cols = p.n_out & ~7;
      uint32_t phase = 0;
      bool ok = true;
      for (int t = t_first; t < ntiles && ok; t += t_step, phase ^= 1u) {
        ok = __all_sync(0xffffffffu, mbar_wait(ofull, phase, abort_flag, kWaitNs));
        if (!ok) break;
        const Tile tl = *o_tile;
        const int col0 = tl.n * kBoxes * kEach;
        const int boxes = p.g.offsets == nullptr ? (tl.rows + 31) / 32 : tl.rows / 32;
        const int box = lane % kBoxes, first = lane / kBoxes * 32;
        if (lane < boxes * kBoxes && col0 + box * kEach < whole_cols)
          tma_store_2d(&map_out, smem_addr(patch + box * kBoxOut + first * 128),
                       col0 + box * kEach, tl.row0 + first);
        // (8 lanes across a box)
        const int r_box = (lane >> 3) % kBoxes, c = col0 + r_box * kEach + (lane & 7) * (kEach / 8);
        uint8_t* o = static_cast<uint8_t*>(p.out) +
                     (static_cast<int64_t>(tl.row0) * p.ldo + c) * (128 / kEach);
        if (c < p.n_out)  // (n_out of groups is a multiple of 64)
#pragma unroll 4
          for (int r = boxes * 32 + (lane >> 3) / kBoxes; r < tl.rows; r += 4 / kBoxes)
            *reinterpret_cast<uint4*>(o + r * p.ldo * (128 / kEach)) =
                *reinterpret_cast<const uint4*>(patch + r_box * kBoxOut + r * 128 +
                                                (((lane & 7) ^ (r & 7)) << 4));
        const int at = whole_cols - col0;  // the row's last columns, fewer than eight
        if (MODE == kMatmul && whole_cols < p.n_out && at < BN) {
          for (int r = lane; r < tl.rows; r += 32) {
            const uint16_t* from = reinterpret_cast<const uint16_t*>(
                patch + (at >> 6) * kBoxOut + r * 128 + (((at >> 3 & 7) ^ (r & 7)) << 4));
            uint16_t* to = static_cast<uint16_t*>(p.out) + (tl.row0 + r) * p.ldo + whole_cols;
            for (int j = 0; j < p.n_out - whole_cols; ++j) to[j] = from[j];
          }
        }
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive1(smem_addr(oempty));
      }
      asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
      if (!ok && lane == 0) {
        if (!*abort_flag) set_err(p.err, kErrTimeout);
        *abort_flag = 1;
      }
    }
  } else {
    // ---------------- sums and epilogue ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    const int quarter = warp & 3;          // TMEM lanes 32 * quarter ..
    const int wg = (warp - kFirstPromoter) >> 2;  // columns 64 wg .. of both halves
    const int pw = warp - kFirstPromoter;
    const int row = quarter * 32 + lane;
    uint8_t* my_patch = patch + pw * 4096;
    float* s_max = reinterpret_cast<float*>(patch + kBoxOut);  // SwiGLU: [2][2][128] row maxima
    uint32_t it = 0, red_phase = 0, sc_slot = 0, sc_phase = 0, o_phase = 0;
    uint32_t xt = 0;  // SwiGLU tiles that this quarter has had rows in
    bool ok = true;
    for (int t = t_first; t < ntiles && ok; t += t_step) {
      // the tile comes with its first scales (an invalid one does not: abort)
      ok = __all_sync(0xffffffffu, mbar_wait(&sfull[sc_slot], sc_phase, abort_flag, kWaitNs));
      if (!ok) break;
      const Tile tl = s_tile[sc_slot];
      const bool live = quarter * 32 < tl.rows;
      const bool store = row < tl.rows;
      uint64_t acc[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[i] = 0;
      auto scales_done = [&] {
        __syncwarp();
        if (lane == 0) mbar_arrive1(smem_addr(&sempty[sc_slot]));
        sc_slot ^= 1u;
        if (sc_slot == 0) sc_phase ^= 1u;
      };
      int in = 0;  // place in the chunk of scales
      for (int kb = kb0; kb < kb1; ++kb) {
        const int b = it & 1;
        if (kb > kb0 && ++in == kScaleChunk) {
          in = 0;
          scales_done();
          ok = __all_sync(0xffffffffu, mbar_wait(&sfull[sc_slot], sc_phase, abort_flag, kWaitNs));
          if (!ok) break;
        }
        const int at = sc_slot * kScaleChunk + in;
        const float sa_r = sc_a[at * BM + row];
        const float2 sb_r = *reinterpret_cast<const float2*>(sc_b + at * 2);
        const float s0 = sa_r * sb_r.x, s1 = sa_r * sb_r.y;
        ok = __all_sync(0xffffffffu, mbar_wait(&tfull[b], (it >> 1) & 1u, abort_flag, kWaitNs));
        if (!ok) break;
        const uint32_t ta = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) +
                            static_cast<uint32_t>(b * BN + wg * 64);
        const uint64_t p0 = pack2(__float_as_uint(s0), __float_as_uint(s0));
        const uint64_t p1 = pack2(__float_as_uint(s1), __float_as_uint(s1));
        uint32_t r[32];
        tc_fence_after();
        tmem_ld32(ta, r);
        tmem_ld_wait(r);
        scaled_add(acc, r, p0);
        tmem_ld32(ta + 32, r);
        tmem_ld_wait(r);
        scaled_add(acc + 16, r, p0);
        tmem_ld32(ta + 128, r);
        tmem_ld_wait(r);
        scaled_add(acc + 32, r, p1);
        tmem_ld32(ta + 160, r);
        tmem_ld_wait(r);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive1(smem_addr(&tempty[b]));
        ++it;
        scaled_add(acc + 48, r, p1);
      }
      if (!ok) break;
      scales_done();

      if (SPLIT) {
        // the cluster's accumulators, 32 rows at a time: rows i = rank, rank +
        // S, .. are this CTA's to add up and store, a warp a row
        float* red = reinterpret_cast<float*>(patch);
        for (int q = 0; q * 32 < tl.rows && ok; ++q, red_phase ^= 1u) {
          if (quarter == q) {
            ok = __all_sync(0xffffffffu, mbar_wait_cluster(red_empty, red_phase ^ 1u, abort_flag));
            if (!ok) break;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const float2 v0 = unpack2(acc[h * 32 + 2 * j]), v1 = unpack2(acc[h * 32 + 2 * j + 1]);
                const int chunk = (h * 32 + wg * 16 + j) ^ (lane & 7);
                *reinterpret_cast<float4*>(red + lane * BN + chunk * 4) =
                    make_float4(v0.x, v0.y, v1.x, v1.y);
              }
            __syncwarp();
            if (lane < S) mbar_arrive_peer(peer_addr(smem_addr(red_full), lane));
          }
          ok = __all_sync(0xffffffffu, mbar_wait_cluster(red_full, red_phase, abort_flag));
          if (!ok) break;
          for (int i = rank + S * pw; i < 32 && q * 32 + i < tl.rows; i += S * kPromoters) {
            // (all ranks' rows in flight, then summed in rank order)
            float v[2][4] = {};
            float4 x[8], y[8];
            const uint32_t at = smem_addr(red + i * BN);
#pragma unroll
            for (int s = 0; s < 8; ++s)
              if (s < S) {
                const uint32_t from = peer_addr(at, s);
                x[s] = ld_peer4(from + ((lane ^ (i & 7)) << 4));
                y[s] = ld_peer4(from + (((32 + lane) ^ (i & 7)) << 4));
              }
#pragma unroll
            for (int s = 0; s < 8; ++s)
              if (s < S) {
                v[0][0] += x[s].x; v[0][1] += x[s].y; v[0][2] += x[s].z; v[0][3] += x[s].w;
                v[1][0] += y[s].x; v[1][1] += y[s].y; v[1][2] += y[s].z; v[1][3] += y[s].w;
              }
            const int64_t r = tl.row0 + q * 32 + i;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int col = tl.n * BN + h * 128 + lane * 4;
              const bool whole = p.out_vec && col + 4 <= p.n_out;
              if (p.out_f32) {
                float* o = static_cast<float*>(p.out) + r * p.ldo + col;
                if (whole) {
                  *reinterpret_cast<float4*>(o) = make_float4(v[h][0], v[h][1], v[h][2], v[h][3]);
                } else {
#pragma unroll
                  for (int j = 0; j < 4; ++j)
                    if (col + j < p.n_out) o[j] = v[h][j];
                }
              } else {
                __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p.out) + r * p.ldo + col;
                if (whole) {
                  __nv_bfloat162 w[2] = {__floats2bfloat162_rn(v[h][0], v[h][1]),
                                         __floats2bfloat162_rn(v[h][2], v[h][3])};
                  *reinterpret_cast<uint2*>(o) = *reinterpret_cast<uint2*>(w);
                } else {
#pragma unroll
                  for (int j = 0; j < 4; ++j)
                    if (col + j < p.n_out) o[j] = __float2bfloat16_rn(v[h][j]);
                }
              }
            }
          }
          __syncwarp();
          if (lane < S) mbar_arrive_peer(peer_addr(smem_addr(red_empty), lane));
        }
        continue;
      }

      if (MODE == kSwiGLU && live) {
        // act in place of the gate sums, codes in place of the up sums
        uint32_t m = 0;
        const bool in = tl.n * 128 + wg * 64 < p.n_out;  // n_out is a multiple of 64
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const float2 g = unpack2(acc[i]), u = unpack2(acc[32 + i]);
          const float a0 = swiglu(g.x, u.x), a1 = swiglu(g.y, u.y);
          m = max(m, max(__float_as_uint(a0) & 0x7fffffffu, __float_as_uint(a1) & 0x7fffffffu));
          acc[i] = pack2(__float_as_uint(a0), __float_as_uint(a1));
        }
        if (!in) m = 0;
        // the row's maximum over both warps.  Two buffers: a warp that is a tile
        // ahead has seen the other's arrival for this tile, which follows its reads
        // of the tile before
        float* mine = s_max + (xt & 1) * 256;
        mine[wg * 128 + row] = __uint_as_float(m);
        __syncwarp();
        if (lane == 0) mbar_arrive1(smem_addr(&xbar[quarter]));
        ok = __all_sync(0xffffffffu, mbar_wait(&xbar[quarter], xt & 1, abort_flag, kWaitNs));
        ++xt;
        if (!ok) break;
        m = max(m, __float_as_uint(mine[(wg ^ 1) * 128 + row]));
        const float am = fp8_amax(m), inv = fp8_inverse(am);
        if (store && wg == 0)
          *reinterpret_cast<float*>(static_cast<uint8_t*>(p.out) +
                                    static_cast<int64_t>(tl.row0 + row) * p.ldo +
                                    p.scale_offset + tl.n * 4) = __fdiv_rn(am, kE4m3Max);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 x0 = unpack2(acc[4 * j]), x1 = unpack2(acc[4 * j + 1]);
          const float2 x2 = unpack2(acc[4 * j + 2]), x3 = unpack2(acc[4 * j + 3]);
          acc[32 + j] = pack2(e4m3x4(x0.x * inv, x0.y * inv, x1.x * inv, x1.y * inv),
                              e4m3x4(x2.x * inv, x2.y * inv, x3.x * inv, x3.y * inv));
        }
      }
      if (staged) {
        // hand the tile to the store warp
        ok = __all_sync(0xffffffffu, mbar_wait(oempty, o_phase ^ 1u, abort_flag, kWaitNs));
        if (!ok) break;
        o_phase ^= 1u;
        if (live && MODE == kSwiGLU) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<ulonglong2*>(patch + row * 128 + (((wg * 4 + j) ^ (row & 7)) << 4)) =
                make_ulonglong2(acc[32 + 2 * j], acc[33 + 2 * j]);
        } else if (live) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              uint32_t w[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float2 v = unpack2(acc[h * 32 + 4 * j + i]);
                __nv_bfloat162 b2 = __floats2bfloat162_rn(v.x, v.y);
                w[i] = *reinterpret_cast<uint32_t*>(&b2);
              }
              *reinterpret_cast<uint4*>(patch + (h * 2 + wg) * kBoxOut + row * 128 +
                                        ((j ^ (row & 7)) << 4)) =
                  make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        if (threadIdx.x == kFirstPromoter * 32) *o_tile = tl;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive1(smem_addr(ofull));
        continue;
      }

      if (!live) continue;
      {
        // fp32, or bf16 rows at any multiple of 2 bytes: 32 columns at a time through
        // a 32-row patch of 128-byte rows (16-byte chunks swizzled by the row), so
        // that a store instruction writes whole lines
        const int64_t row_base = tl.row0 + quarter * 32;
        const int rows = min(32, tl.rows - quarter * 32);
        auto at = [&](int r, int c) {
          return *reinterpret_cast<const float*>(my_patch + r * 128 + (((c >> 2) ^ (r & 7)) << 4) +
                                                 (c & 3) * 4);
        };
#pragma unroll
        for (int part = 0; part < 4; ++part) {
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 v0 = unpack2(acc[part * 16 + 2 * j]);
            const float2 v1 = unpack2(acc[part * 16 + 2 * j + 1]);
            *reinterpret_cast<float4*>(my_patch + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                make_float4(v0.x, v0.y, v1.x, v1.y);
          }
          __syncwarp();
          const int first = tl.n * BN + (part >> 1) * 128 + wg * 64 + (part & 1) * 32;
          const int cols = min(32, p.n_out - first);
          if (p.out_f32 && p.out_vec && cols == 32) {
            const int chunk = lane & 7;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int r = i * 4 + (lane >> 3);
              const float4 v =
                  *reinterpret_cast<const float4*>(my_patch + r * 128 + ((chunk ^ (r & 7)) << 4));
              if (r < rows)
                *reinterpret_cast<float4*>(static_cast<float*>(p.out) + (row_base + r) * p.ldo +
                                           first + chunk * 4) = v;
            }
          } else if (p.out_f32) {  // a lane a column
#pragma unroll 4
            for (int r = 0; r < rows; ++r)
              if (lane < cols)
                static_cast<float*>(p.out)[(row_base + r) * p.ldo + first + lane] = at(r, lane);
          } else {
            // two rows an instruction: words of two columns from the row's first 4-byte
            // boundary on, what is left in front and behind by itself
#pragma unroll 4
            for (int r = lane >> 4; r < rows; r += 2) {
              __nv_bfloat16* o =
                  static_cast<__nv_bfloat16*>(p.out) + (row_base + r) * p.ldo + first;
              const int odd = static_cast<int>(reinterpret_cast<uintptr_t>(o) >> 1 & 1);
              const int c = 2 * (lane & 15) + odd;
              if (c + 1 < cols)
                *reinterpret_cast<__nv_bfloat162*>(o + c) =
                    __floats2bfloat162_rn(at(r, c), at(r, c + 1));
              else if (c < cols)
                o[c] = __float2bfloat16_rn(at(r, c));
              if ((lane & 15) == 0 && odd && cols > 0) o[0] = __float2bfloat16_rn(at(r, 0));
            }
          }
        }
      }
    }
    if (!ok && lane == 0) {
      if (!*abort_flag) set_err(p.err, kErrTimeout);
      *abort_flag = 1;
    }
  }

  tc_fence_before();
  __syncwarp();
  if (SPLIT) cluster_sync();  // no CTA leaves while its rows are read
  __syncthreads();
  tc_fence_after();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc(tmem_base, 2 * BN);
  }
}

template <int MODE, bool SPLIT>
cudaError_t launch_impl(const Fp8GemmArgs& a, cudaStream_t stream) {
  auto kernel = fp8_gemm_kernel<MODE, SPLIT>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       kSmemBytes);
  if (e != cudaSuccess) return e;
  Params p{};
  static_assert(!(SPLIT && MODE == kSwiGLU), "only dense products are split");
  p.nkb = (a.K + 127) / 128;
  p.n_out = a.n_out;
  p.n_tiles = MODE == kSwiGLU ? (a.n_out + 127) / 128 : (a.n_out + BN - 1) / BN;
  p.g = a.g;
  p.max_mtiles = ((a.g.offsets != nullptr ? a.g.cap_rows : a.g.dense_rows) + BM - 1) / BM +
                 (a.g.offsets != nullptr ? a.g.E : 0);
  p.a_box = a.a_box;
  p.a_scales = a.a_scales;
  p.a_scale_row_bytes = a.a_scale_row_bytes;
  p.b_scales = a.b_scales;
  p.b_scale_group = a.b_scale_group;
  p.b_scale_ld = a.b_scale_ld;
  p.out = a.out;
  p.ldo = a.ldo;
  p.out_f32 = a.out_f32;
  p.staged = !SPLIT && a.map_out != nullptr;
  p.out_vec = reinterpret_cast<uintptr_t>(a.out) % 16 == 0 &&
              a.ldo * (a.out_f32 ? 4 : 2) % 16 == 0;
  p.scale_offset = fp8_scale_offset(a.n_out);
  p.splits = a.splits;
  p.err = a.err;
  const int64_t most = static_cast<int64_t>(p.max_mtiles) * p.n_tiles;
  const int per_tile = a.splits;
  const int64_t grid = std::max<int64_t>(1, std::min<int64_t>(a.num_sms / per_tile, most)) * per_tile;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {static_cast<unsigned>(per_tile), 1, 1};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = SPLIT ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, *a.map_a, *a.map_b,
                            p.staged ? *a.map_out : *a.map_a, p);
}

}  // namespace

cudaError_t launch_fp8_swiglu(const Fp8GemmArgs& a, cudaStream_t stream) {
  return launch_impl<kSwiGLU, false>(a, stream);
}
cudaError_t launch_fp8_matmul(const Fp8GemmArgs& a, cudaStream_t stream) {
  return a.splits > 1 ? launch_impl<kMatmul, true>(a, stream)
                      : launch_impl<kMatmul, false>(a, stream);
}

}  // namespace rx
