// sample.cu — one token per row of logits from given uniforms: temperature,
// top-k, top-p and min-p, with the chosen token's probability, the confidence
// that the refinement state takes.
//
// Every decision is taken on integers, so the token does not depend on how a
// row is split or in which order sums are formed.  With m the row's largest
// logit and c = log2(e) / T (fp32), each step one rounded fp32 operation,
//   t_i = max((z_i - m) * c, -40),  n_i = t_i to the nearest integer (ties to
//   even),  f_i = t_i - n_i,
//   p_i = 1 + f (c1 + f (c2 + f (c3 + f (c4 + f c5))))      (about 2^f)
//   w_i = floor(p_i * 2^(n_i + 31))                          (the weight)
// c1 .. c5 interpolate (2^f - 1) / f at the five Chebyshev nodes of [-1/2,
// 1/2]; p is within 3e-7 of 2^f.  Weights are 2^31 at the largest logit and 0
// from about 2^-31 of it down; sums of 2^18 of them fit 64 bits and are exact
// in a double, in which the comparisons with p * mass and u * mass are made.  The
// confidence is the library's exponential of the token over an fp32 sum of e^(z - m);
// the sum's terms, one a token, are hardware exponentials of a rounded exponent (each
// within 2^-22 and 2^-24 of its exponent; the terms that count are near the largest
// logit.  2048 rows of 131072 bf16, greedy 112 us, T = 0.7 206, top-k 50 228; with the
// library's 145, 255 and 260).
//
// Two shapes of one kernel.  Few rows, or short ones: a row is held in the shared
// memory of a cluster of 1 to 8 CTAs.  Many long rows: one CTA of 512 threads
// walks a row a few times, the first time from HBM, then from L2 (two CTAs an
// SM; a third of the cluster's barriers and none of its waits).
//
// Without top-k and top-p one pass forms the weights.  With them, a
// first pass counts the tokens by 32nds of an octave of weight; the counts (for
// top-p, times the middle weight of each bin) name the few bins that the last
// kept token, by logit, then index, can lie in.  A second pass collects those
// bins' tokens in a list (with everything above them where that is little; else
// it adds up the weights above) and, for top-p, all weights.  The cut is then
// found in the list, exactly, from histograms of the logits' bits, 128 bins at a
// time.  A row whose list overflows or misses the cut (many equal logits, top-p
// of a large top-k) takes the same search over all of its tokens.  Then one warp
// walks the 1024 tokens that u falls in.
//
// Bound: instruction issue, about 15 instructions a token for weights (fp32 in
// packed pairs), 8 for counts, against the 12 cycles that HBM gives an SM for 128
// bf16 tokens.  2048 rows of 131072 in bf16 (their bytes take 79 us): greedy 114 us,
// no filters 197, top-k 50 228, 5000 423, top-p 0.5 to 0.9999 between 410 and 525.  One
// such row: 24 us with every filter, a dozen of the cluster's barriers one after another.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "internal.h"

namespace rx {
namespace {

constexpr int kStep = 256;         // tokens of a warp's step: 8 consecutive ones a lane
constexpr int kSegSteps = 4;       // steps of a segment
constexpr int kFine = 1024;        // bins of 1/32 octave down to 2^-32
constexpr int kBins = 128;
constexpr int kMaxVocab = 1 << 18;

// kStream: a CTA walks a row in global memory; else a cluster holds it.
template <bool kStream>
struct Shape {
  static constexpr int kThreads = kStream ? 512 : 256;
  static constexpr int kWarps = kThreads / 32;
  static constexpr int kCtas = kStream ? 2 : 3;         // an SM
  static constexpr int kList = kStream ? 10240 : 2048;  // tokens of a CTA's list
  static constexpr int kMaxSegs = kStream ? 288 : 64;   // per CTA
};

struct Hist {  // masses in pieces of 11, 11 and 10 bits, at most 2^18 tokens each
  uint32_t count[kBins], m0[kBins], m1[kBins], m2[kBins];
};

// Tokens in reach of the cut: places in the slice, and the logits where the
// slice is not in shared memory.
template <bool kStream>
struct List {
  uint16_t place[Shape<false>::kList];
};
template <>
struct List<true> {
  uint32_t place[Shape<true>::kList];
  float z[Shape<true>::kList];
};

template <bool kStream>
struct Shared {
  using S = Shape<kStream>;
  uint32_t fine[kFine];  // tokens by weight
  Hist hist;
  List<kStream> list;
  unsigned long long seg_mass[S::kMaxSegs];  // weights of a segment's kept tokens ..
  uint32_t seg_lo[S::kMaxSegs], seg_hi[S::kMaxSegs];  // .. and of those from the list, in halves
  uint32_t seg_ties[S::kMaxSegs];
  // what the whole cluster reads, each written once before a cluster barrier
  float max, expsum;
  int first;                      // greedy: the first token of the largest logit
  uint32_t n_list;
  unsigned long long reach_mass;  // above the list
  unsigned long long mass;        // of all tokens
  unsigned long long whole_mass;  // the same, of the search over the whole row
  // the CTA's own
  unsigned long long warp_m[2][S::kWarps];
  unsigned long long above_mass, bin_mass;  // results of a search
  uint32_t above_count, bin_count, klo, khi;
  float warp_f[S::kWarps];
  uint32_t warp_c[S::kWarps];
  int bin[4];
  uint32_t at[4];
};
static_assert(sizeof(Shared<false>) <= 12 * 1024, "three CTAs of 56 KB slices an SM");
static_assert(sizeof(Shared<true>) <= 112 * 1024, "two CTAs an SM");

struct Args {
  const void* logits;
  int64_t ld;
  int vocab;
  int slice;  // tokens of a CTA
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  const uint8_t* masked;
  int32_t* tokens;
  float* conf;
  uint32_t* err;
};

// ---- clusters ---------------------------------------------------------------
__device__ __forceinline__ int cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return static_cast<int>(r);
}
__device__ __forceinline__ int cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return static_cast<int>(r);
}
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}
__device__ __forceinline__ uint32_t peer(const void* p, int rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
  return a;
}
// A word of another CTA's Shared (kStream: there is no other).
template <bool kStream>
__device__ __forceinline__ uint32_t peer_u32(const uint32_t* p, int rank) {
  if (kStream) return *p;
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(peer(p, rank)) : "memory");
  return v;
}
template <bool kStream>
__device__ __forceinline__ float peer_f32(const float* p, int rank) {
  return __uint_as_float(peer_u32<kStream>(reinterpret_cast<const uint32_t*>(p), rank));
}
template <bool kStream>
__device__ __forceinline__ unsigned long long peer_u64(const unsigned long long* p, int rank) {
  if (kStream) return *p;
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(peer(p, rank)) : "memory");
  return v;
}
template <bool kStream>
__device__ __forceinline__ uint4 peer_u32x4(const uint32_t* p, int rank) {
  if (kStream) return *reinterpret_cast<const uint4*>(p);
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(peer(p, rank))
               : "memory");
  return v;
}

// ---- the weights ------------------------------------------------------------
__device__ __forceinline__ uint64_t pk(float a, float b) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
  return v;
}
__device__ __forceinline__ void upk(uint64_t v, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

constexpr float kLog2e = 1.44269502162933349609375f;
constexpr float kTwo31 = 2147483648.0f;
// times 2^31: scaling by a power of two leaves every rounding as it is
constexpr float kC1 = 0.6931471824645996f * kTwo31, kC2 = 0.2402234971523285f * kTwo31,
                kC3 = 0.055503811687231064f * kTwo31, kC4 = 0.00966636836528778f * kTwo31,
                kC5 = 0.0013381302123889327f * kTwo31;
constexpr float kMagic = 12582912.0f;  // 1.5 * 2^23: adding it rounds to an integer

struct Pair {
  float t0, t1;      // exponents, at least -40
  float v0, v1;      // p 2^(n + 31)
  uint32_t w0, w1;   // weights
  uint64_t d;        // z - m
};
// Tokens with logits z (NaN: weight 0, as -inf).
__device__ __forceinline__ Pair weigh(float z0, float z1, float neg_m, float c) {
  Pair r;
  r.d = add2(pk(z0, z1), pk(neg_m, neg_m));
  upk(mul2(r.d, pk(c, c)), r.t0, r.t1);
  r.t0 = fmaxf(r.t0, -40.0f);
  r.t1 = fmaxf(r.t1, -40.0f);
  const uint64_t t = pk(r.t0, r.t1);
  const uint64_t tr = add2(t, pk(kMagic, kMagic));
  const uint64_t f = fma2(add2(tr, pk(-kMagic, -kMagic)), pk(-1.0f, -1.0f), t);
  uint64_t p = add2(mul2(pk(kC5, kC5), f), pk(kC4, kC4));
  p = add2(mul2(p, f), pk(kC3, kC3));
  p = add2(mul2(p, f), pk(kC2, kC2));
  p = add2(mul2(p, f), pk(kC1, kC1));
  p = add2(mul2(p, f), pk(kTwo31, kTwo31));
  float p0, p1, n0, n1;
  upk(p, p0, p1);
  upk(tr, n0, n1);
  // the low bits of tr are n: into the exponent
  r.v0 = __uint_as_float(__float_as_uint(p0) + (__float_as_uint(n0) << 23));
  r.v1 = __uint_as_float(__float_as_uint(p1) + (__float_as_uint(n1) << 23));
  r.w0 = __float2uint_rz(r.v0);
  r.w1 = __float2uint_rz(r.v1);
  return r;
}
__device__ __forceinline__ uint32_t weight_of(float z, float neg_m, float c) {
  return weigh(z, z, neg_m, c).w0;
}
__device__ __forceinline__ void add_wide(unsigned long long& sum, uint32_t w) {
  asm("mad.wide.u32 %0, %1, 1, %0;" : "+l"(sum) : "r"(w));
}
// -32 t to the nearest integer; kFine and more: not counted (t < -32, NaN).
__device__ __forceinline__ uint32_t fine_bin(float t) {
  return __float_as_uint(__fmaf_rn(t, -32.0f, kMagic)) - 0x4b400000u;
}

// ---- logits as ordered integers ---------------------------------------------
// bf16 logits use the upper 16 bits (keys of 16 bits).
template <typename Te>
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.0f);  // -0 ranks as +0
  const uint32_t k = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return sizeof(Te) == 2 ? k >> 16 : k;
}
template <typename Te>
__device__ __forceinline__ float key_value(uint32_t k) {
  if (sizeof(Te) == 2) k = (k << 16) | ((k & 0x8000u) ? 0u : 0xffffu);
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

__device__ __forceinline__ unsigned long long warp_sum(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum over the lanes below.
template <typename T>
__device__ __forceinline__ T warp_before(T v) {
  const int lane = threadIdx.x & 31;
  T x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x - v;
}

// Sums the cluster's histograms and finds the first bin at which the running
// count (from count0) reaches `want`, or the running mass (from mass0) does.
// Warp 0; the result goes to s.above_*, s.bin_*; returns the bin, or -1.
template <bool kStream>
__device__ int find_bin(Shared<kStream>& s, int C, bool by_count, unsigned long long want,
                        unsigned long long mass0, uint32_t count0) {
  const int lane = threadIdx.x & 31;
  uint32_t cnt[4] = {};
  unsigned long long mass[4] = {};
  for (int r = 0; r < C; ++r) {
    const uint4 n = peer_u32x4<kStream>(&s.hist.count[lane * 4], r),
                x = peer_u32x4<kStream>(&s.hist.m0[lane * 4], r),
                y = peer_u32x4<kStream>(&s.hist.m1[lane * 4], r),
                z = peer_u32x4<kStream>(&s.hist.m2[lane * 4], r);
    const uint32_t nn[4] = {n.x, n.y, n.z, n.w}, xx[4] = {x.x, x.y, x.z, x.w},
                   yy[4] = {y.x, y.y, y.z, y.w}, zz[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      cnt[i] += nn[i];
      mass[i] += xx[i] + (static_cast<unsigned long long>(yy[i]) << 11) +
                 (static_cast<unsigned long long>(zz[i]) << 22);
    }
  }
  uint32_t c = count0 + warp_before(cnt[0] + cnt[1] + cnt[2] + cnt[3]);
  unsigned long long m = mass0 + warp_before(mass[0] + mass[1] + mass[2] + mass[3]);
  int hit = -1;
  uint32_t bin_c = 0;
  unsigned long long bin_m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (hit >= 0) continue;
    if (cnt[i] > 0 && (by_count ? c + cnt[i] >= want : m + mass[i] >= want)) {
      hit = lane * 4 + i;
      bin_c = cnt[i];
      bin_m = mass[i];
    } else {
      c += cnt[i];
      m += mass[i];
    }
  }
  const uint32_t any = __ballot_sync(0xffffffffu, hit >= 0);
  if (any == 0) return -1;
  const int from = __ffs(any) - 1;
  if (lane == from) {
    s.above_count = c;
    s.above_mass = m;
    s.bin_count = bin_c;
    s.bin_mass = bin_m;
  }
  return __shfl_sync(0xffffffffu, hit, from);
}

// The smallest key in [lo, hi] with pred (false .. false true .. true), or hi
// + 1; a whole warp, 32 keys a round.
template <typename F>
__device__ uint32_t first_key(uint32_t lo, uint32_t hi, F pred) {
  const int lane = threadIdx.x & 31;
  unsigned long long a = lo, b = static_cast<unsigned long long>(hi) + 1;  // answer in [a, b]
  while (a < b) {
    const unsigned long long step = (b - a + 31) / 32;
    const unsigned long long k = a + lane * step;
    const uint32_t hits = __ballot_sync(0xffffffffu, k >= b || pred(static_cast<uint32_t>(k)));
    const int f = hits ? __ffs(hits) - 1 : 32;
    if (f == 0) return static_cast<uint32_t>(a);
    const unsigned long long na = a + (f - 1) * step + 1, nb = a + f * step;
    a = na;
    b = nb < b ? nb : b;
  }
  return static_cast<uint32_t>(a);
}

__device__ __forceinline__ void cp_async16(void* smem, const void* gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(smem)), "l"(gmem)
               : "memory");
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// The largest of m and 8 logits; NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max8(float m, const uint4 (&raw)[2]) {  // fp32
  const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w,
                         raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max_nan(m, __uint_as_float(w[j]));
  return m;
}
__device__ __forceinline__ float max8(float m, const uint4 (&raw)[1]) {  // bf16
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(raw);
  const __nv_bfloat162 x = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  return max_nan(m, max_nan(__low2float(x), __high2float(x)));
}
__device__ __forceinline__ void widen(const uint4 (&raw)[2], float (&z)[8]) {
  const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w,
                         raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
  for (int j = 0; j < 8; ++j) z[j] = __uint_as_float(w[j]);
}
__device__ __forceinline__ void widen(const uint4 (&raw)[1], float (&z)[8]) {
  const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    z[2 * j] = __uint_as_float(w[j] << 16);
    z[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
  }
}

enum { kListAll, kListReach, kWhole };   // where the cut is searched

struct Cut {  // kept: logits above `value`, and the first `ties` of those equal to it
  float value;
  uint32_t ties;
  unsigned long long mass;  // of what is kept
};

// One row, by the cluster or by the CTA.
template <typename Te, bool kStream>
__device__ __forceinline__ void sample_row(const Args& a, Shared<kStream>& s, Te* z_s, int C,
                                           int rank, int64_t row) {
  constexpr int kThreads = Shape<kStream>::kThreads, kWarps = Shape<kStream>::kWarps;
  constexpr int kList = Shape<kStream>::kList;
  constexpr int kVec = 16 / sizeof(Te), kRaw = 8 / kVec;  // a lane's step: kRaw vectors
  auto sync_all = [] {
    if (kStream) __syncthreads();
    else cluster_sync();
  };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool leader = rank == 0 && threadIdx.x == 0;

  // the row's settings; a row that is left out or refused costs no loads
  float temp = a.temperature ? a.temperature[row] : 1.0f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.0f;
  const float min_p = a.min_p ? a.min_p[row] : 0.0f;
  float u = a.u[row];
  const bool out = a.masked != nullptr && a.masked[row] == 0;
  const bool bad = !(temp >= 0.0f && temp <= FLT_MAX) || !(top_p > 0.0f) || !(min_p <= 1.0f) ||
                   !(u == u);
  if (out || bad) {
    if (leader) {
      a.tokens[row] = -1;
      a.conf[row] = 0.0f;
      if (!out) set_err(a.err, kErrIndex);
    }
    return;
  }
  u = fminf(fmaxf(u, 0.0f), 0.999999940395355224609375f);  // [0, 1 - 2^-24]
  const bool greedy = temp == 0.0f;
  if (greedy) temp = 1.0f;

  // ---- the CTA's tokens, and their largest logit ------------------------------
  // Positions are counted from the 16-byte boundary at or below the row's
  // start, so every vector of positions is one aligned load; positions outside
  // the row hold -inf.
  const Te* start = static_cast<const Te*>(a.logits) + row * a.ld;
  const int shift = static_cast<int>(reinterpret_cast<uintptr_t>(start) % 16 / sizeof(Te));
  const int lo = shift, hi = shift + a.vocab;  // positions of the row
  const Te* base = start - shift;
  const int pos0 = rank * a.slice;
  const int steps = a.slice / (kWarps * kStep);  // of each warp
  const int own = warp * steps * kStep + lane * 8;  // place of the lane's first token
  const int my_pos = pos0 + own;
  const float minus_inf = __int_as_float(0xff800000);
  bool fix = false, fix_inf = false;  // streamed rows with a NaN or +inf
  // 8 tokens from a place on, as they are
  auto fetch = [&](int place, uint4 (&raw)[kRaw]) {
#pragma unroll
    for (int v = 0; v < kRaw; ++v) {
      if (!kStream) {
        raw[v] = *reinterpret_cast<const uint4*>(z_s + place + v * kVec);
        continue;
      }
      const int q = place + v * kVec;
      if (q >= lo && q + kVec <= hi) {
        raw[v] = __ldg(reinterpret_cast<const uint4*>(base + q));
      } else {
        Te* e = reinterpret_cast<Te*>(&raw[v]);
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          e[j] = q + j >= lo && q + j < hi ? base[q + j] : from_f32<Te>(minus_inf);
      }
    }
  };
  // as fp32, without a NaN and with finite logits above -inf
  auto open = [&](const uint4 (&raw)[kRaw], float (&z)[8]) {
    widen(raw, z);
    if (kStream && fix) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        z[j] = z[j] == z[j] ? z[j] : minus_inf;
        if (fix_inf) z[j] = z[j] == -minus_inf ? 0.0f : minus_inf;
      }
    }
  };
  auto load = [&](int place, float (&z)[8]) {
    uint4 raw[kRaw];
    fetch(place, raw);
    open(raw, z);
  };
  // the warp's steps whose vectors all lie in the row (streamed: plain loads)
  const int in0 = pos0 + warp * steps * kStep < lo ? 1 : 0;
  const int in1 = min(steps, (hi - (pos0 + warp * steps * kStep)) / kStep);
  const uint4* my_vec = reinterpret_cast<const uint4*>(base + my_pos);
  constexpr int kStepVecs = kStep / kVec;
  // visit(i, z, raw) for the steps from i0 to i1 - 1, `kAhead` loads in flight
  // Streamed bf16: two.  With four the loops outgrow the instruction caches that two
  // CTAs in different rows' filters share (a quarter of the stalls; 2048 rows of
  // 131072 without filters 191 us, two 198, top-p 0.9 499, 471, 4096 mixed rows 417,
  // 331).
  constexpr int kAhead = kStream && sizeof(Te) == 2 ? 2 : 1;
  constexpr int kSample = kStream ? 32 / sizeof(Te) / 4 : 1;  // steps that top-k looks at first
  auto each_step = [&](int i0, int i1, auto visit) {
#pragma unroll 1
    for (int i = i0; i < i1; i += kAhead) {
      uint4 raw[kAhead][kRaw];
      if (kStream && i >= in0 && i + kAhead <= in1) {
        const uint4* at = my_vec + i * kStepVecs;
#pragma unroll
        for (int d = 0; d < kAhead; ++d)
#pragma unroll
          for (int v = 0; v < kRaw; ++v) raw[d][v] = __ldg(at + d * kStepVecs + v);
      } else {
#pragma unroll
        for (int d = 0; d < kAhead; ++d)
          if (d == 0 || i + d < i1) fetch(own + (i + d) * kStep, raw[d]);
      }
#pragma unroll
      for (int d = 0; d < kAhead; ++d) {
        if (d > 0 && i + d >= i1) break;
        float z[8];
        open(raw[d], z);
        visit(i + d, z, raw[d]);
      }
    }
  };
  if (!kStream) {
    for (int i = 0; i < steps; ++i) {
#pragma unroll
      for (int v = 0; v < kRaw; ++v) {
        const int q = my_pos + i * kStep + v * kVec;
        Te* to = z_s + own + i * kStep + v * kVec;
        if (q >= lo && q + kVec <= hi) {
          cp_async16(to, base + q);
        } else {
#pragma unroll
          for (int j = 0; j < kVec; ++j)
            to[j] = q + j >= lo && q + j < hi ? base[q + j] : from_f32<Te>(minus_inf);
        }
      }
    }
  }
  for (int i = threadIdx.x; i < kFine; i += kThreads) s.fine[i] = 0u;
  if (threadIdx.x == 0) {
    s.n_list = 0;
    s.first = 0x7fffffff;
  }
  float lane_max = minus_inf, m = minus_inf;
  int max_step = 0;  // the lane's first step with its largest logit
  if (!kStream) {
    cp_async_wait();  // a lane reads what it copied
#pragma unroll 4
    for (int i = 0; i < steps; ++i) {
      uint4 raw[kRaw];
      fetch(own + i * kStep, raw);
      const float x = max8(lane_max, raw);
      if (x > lane_max) max_step = i;
      lane_max = x;
    }
  } else {
    constexpr int kMaxAhead = 8 / kRaw;
    for (int i = 0; i < steps; i += kMaxAhead) {
      uint4 raw[kMaxAhead][kRaw];
      if (i >= in0 && i + kMaxAhead <= in1) {
        const uint4* at = my_vec + i * kStepVecs;
#pragma unroll
        for (int d = 0; d < kMaxAhead; ++d)
#pragma unroll
          for (int v = 0; v < kRaw; ++v) raw[d][v] = __ldg(at + d * kStepVecs + v);
      } else {
#pragma unroll
        for (int d = 0; d < kMaxAhead; ++d) fetch(own + min(i + d, steps - 1) * kStep, raw[d]);
      }
#pragma unroll
      for (int d = 0; d < kMaxAhead; ++d) {
        const float x = max8(lane_max, raw[d]);
        if (x > lane_max) max_step = i + d;
        lane_max = x;
      }
    }
  }
  auto block_max = [&] {
    float x = lane_max;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, o));
    if (lane == 0) s.warp_f[warp] = x;
    __syncthreads();
    x = s.warp_f[0];
    for (int w = 1; w < kWarps; ++w) x = max_nan(x, s.warp_f[w]);
    return x;
  };
  m = block_max();
  if (m != m) {  // NaN counts as -inf
    fix = kStream;
    lane_max = minus_inf;
    for (int i = 0; i < steps; ++i) {
      float z[8];
      load(own + i * kStep, z);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!kStream && z[j] != z[j])
          z_s[own + i * kStep + j] = from_f32<Te>(minus_inf);
        if (z[j] > lane_max) {
          lane_max = z[j];
          max_step = i;
        }
      }
    }
    __syncthreads();
    m = block_max();
  }
  if (threadIdx.x == 0) s.max = m;
  sync_all();
  for (int r = 0; r < C; ++r) m = fmaxf(m, peer_f32<kStream>(&s.max, r));
  if (!(m > minus_inf)) {  // nothing to sample from
    sync_all();
    if (leader) {
      a.tokens[row] = -1;
      a.conf[row] = 0.0f;
    }
    return;
  }
  if (m > FLT_MAX) {  // +inf: those tokens alone, alike
    if (!kStream) {
      for (int i = 0; i < steps; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          Te* at = z_s + own + i * kStep + j;
          *at = from_f32<Te>(to_f32(*at) == m ? 0.0f : minus_inf);
        }
    }
    fix = fix_inf = kStream;
    // (a lane without one has none of the largest logit now, whatever it had before)
    lane_max = lane_max == m ? 0.0f : minus_inf;
    m = 0.0f;
  }
  const float neg_m = -m;
  const float c = fminf(__fdiv_rn(kLog2e, temp), FLT_MAX);
  const bool by_k = !greedy && top_k > 0, by_p = !greedy && top_p < 1.0f;
  const bool cut_any = by_k || by_p;
  const uint32_t w_min =
      !greedy && min_p > 0.0f
          ? static_cast<uint32_t>(ceil(static_cast<double>(min_p) * 2147483648.0)) : 0u;

  // ---- one pass over the row ----------------------------------------------------
  const int segs = (steps + kSegSteps - 1) / kSegSteps;  // of each warp
  auto set_seg = [&](int g, unsigned long long w, uint32_t ties) {  // of the warp
    const int q = warp * segs + g;
    s.seg_mass[q] = w;
    s.seg_lo[q] = s.seg_hi[q] = 0;
    s.seg_ties[q] = ties;
  };
  const bool same_t = c == kLog2e;  // T = 1: the weights give the softmax
  float esum = 0.0f;
  uint64_t esum2 = 0;  // two partial sums
  auto add_exp = [&](uint64_t d) {
    float e0, e1;
    upk(mul2(d, pk(kLog2e, kLog2e)), e0, e1);
    esum2 = add2(esum2, pk(ex2(e0), ex2(e1)));
  };
  auto plain_pass = [&](auto same_c, auto min_c) {
    constexpr bool kSame = decltype(same_c)::value, kMin = decltype(min_c)::value;
    for (int g = 0; g < segs; ++g) {
      unsigned long long seg = 0;
      each_step(g * kSegSteps, min(steps, (g + 1) * kSegSteps), [&](int, const float (&z)[8], const uint4 (&)[kRaw]) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const Pair w = weigh(z[j], z[j + 1], neg_m, c);
          add_wide(seg, !kMin || w.w0 >= w_min ? w.w0 : 0u);
          add_wide(seg, !kMin || w.w1 >= w_min ? w.w1 : 0u);
          if (kSame) esum2 = add2(esum2, pk(w.v0, w.v1));
          else add_exp(w.d);
        }
      });
      seg = warp_sum(seg);
      if (lane == 0) set_seg(g, seg, 0);
    }
  };
  // Tokens of a step with logits from flo to fhi (`top`: of any) into the list.
  auto enlist = [&](bool top, float flo, float fhi, int i, const float (&z)[8],
                    const uint4 (&raw)[kRaw]) {
    uint32_t hits = 0;
    if (sizeof(Te) == 2 && !fix_inf) {  // two at a time; most steps have none
      const __nv_bfloat162 flo2 = __float2bfloat162_rn(flo), fhi2 = __float2bfloat162_rn(fhi);
      const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(raw);
      uint32_t in[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        in[j] = __hge2_mask(h[j], flo2);
        if (!top) in[j] &= __hle2_mask(h[j], fhi2);
      }
      if (in[0] | in[1] | in[2] | in[3]) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          hits |= (in[j] & 1u) << (2 * j) | (in[j] >> 31) << (2 * j + 1);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        hits |= static_cast<uint32_t>(z[j] >= flo && (top || z[j] <= fhi)) << j;
    }
    if (hits) {
      uint32_t at = atomicAdd(&s.n_list, static_cast<uint32_t>(__popc(hits)));
      const int place = own + i * kStep;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!(hits >> j & 1)) continue;
        if (at < kList) {
          s.list.place[at] = place + j;
          if constexpr (kStream) s.list.z[at] = z[j];
        }
        ++at;
      }
    }
  };
  const uint32_t kmax = key_of<Te>(m), kmin = key_of<Te>(minus_inf);
  auto bin_of_key = [&](uint32_t k) {  // falls as the key rises
    return fine_bin(__fmul_rn(__fadd_rn(key_value<Te>(k), neg_m), c));
  };
  bool listed_already = false;  // in the first pass (streamed, top-k of few)
  // The counts by bins, and the softmax's sum.
  auto count_pass = [&](auto same_c, int i0, int i1) {
    constexpr bool kSame = decltype(same_c)::value;
    each_step(i0, i1, [&](int, const float (&z)[8], const uint4 (&)[kRaw]) {
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const uint64_t d = add2(pk(z[j], z[j + 1]), pk(neg_m, neg_m));
        const uint64_t t = mul2(d, pk(c, c));
        if (kSame) {
          float e0, e1;
          upk(t, e0, e1);
          esum2 = add2(esum2, pk(ex2(e0), ex2(e1)));
        } else {
          add_exp(d);
        }
        float b0, b1;  // fine_bin of both
        upk(fma2(t, pk(-32.0f, -32.0f), pk(kMagic, kMagic)), b0, b1);
        const uint32_t n0 = __float_as_uint(b0) - 0x4b400000u, n1 = __float_as_uint(b1) - 0x4b400000u;
        if (n0 < kFine) atomicAdd(&s.fine[n0], 1u);
        if (n1 < kFine) atomicAdd(&s.fine[n1], 1u);
      }
    });
  };
  if (greedy) {
    each_step(0, steps, [&](int, const float (&z)[8], const uint4 (&)[kRaw]) {
#pragma unroll
      for (int j = 0; j < 8; j += 2) add_exp(add2(pk(z[j], z[j + 1]), pk(neg_m, neg_m)));
    });
    if (lane_max == m) {  // the lane's first token of the largest logit
      float z[8];
      load(own + max_step * kStep, z);
      int first = -1;
#pragma unroll
      for (int j = 7; j >= 0; --j)
        if (z[j] == m) first = j;
      if (first >= 0) atomicMin(&s.first, my_pos + max_step * kStep + first);
    }
  } else if (cut_any) {
    auto counts = [&](int i0, int i1) {
      if (same_t) count_pass(std::true_type(), i0, i1);
      else count_pass(std::false_type(), i0, i1);
    };
    if (kStream && by_k && steps >= 4 * kSample && top_k < a.vocab / 16 &&
        4 * top_k <= kList) {
      // Top-k of few: the counts of a sample (the first steps of every warp)
      // name the bins that hold three times as many tokens; these make the
      // list, and the other steps are not counted (2048 rows of 131072, top-k
      // 50: 313 us with counts, 228 us without).  Should the list be too short
      // all the same, or too long, the whole row is searched, so a quarter of the list
      // is the most that is asked for (top-k 3000 and 5000 there, 9000 and 15000 tokens
      // for 10240 places: 590 and 2910 us).
      counts(0, kSample);
      __syncthreads();
      if (warp == 0) {
        constexpr int kPer = kFine / 32;
        uint32_t n = 0;
        for (int i = 0; i < kPer; ++i) n += s.fine[lane * kPer + i];
        uint32_t upto = warp_before(n);
        const uint32_t want = 3u * top_k * kSample / steps + 48;
        uint32_t b = kFine - 1;
        for (int i = kPer - 1; i >= 0; --i) {  // the first bin at which `want` is reached
          if (upto + n >= want) b = lane * kPer + i;
          n -= s.fine[lane * kPer + i];
        }
        b = __reduce_min_sync(0xffffffffu, b);
        const uint32_t k = first_key(kmin, kmax, [&](uint32_t k) { return bin_of_key(k) <= b; });
        if (lane == 0) s.klo = k;
      }
      __syncthreads();
      const float flo = key_value<Te>(s.klo);
      each_step(kSample, steps, [&](int i, const float (&z)[8], const uint4 (&raw)[kRaw]) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) add_exp(add2(pk(z[j], z[j + 1]), pk(neg_m, neg_m)));
        enlist(true, flo, m, i, z, raw);
      });
      each_step(0, kSample, [&](int i, const float (&z)[8], const uint4 (&raw)[kRaw]) {
        enlist(true, flo, m, i, z, raw);
      });
      for (int g = lane; g < segs; g += 32) set_seg(g, 0, 0);
      listed_already = true;
    } else {
      counts(0, steps);
    }
  } else {
    if (w_min) {
      if (same_t) plain_pass(std::true_type(), std::true_type());
      else plain_pass(std::false_type(), std::true_type());
    } else {
      if (same_t) plain_pass(std::true_type(), std::false_type());
      else plain_pass(std::false_type(), std::false_type());
    }
  }
  {
    float e0, e1;
    upk(esum2, e0, e1);
    esum = warp_sum(e0 + e1);
    if (same_t && !cut_any && !greedy) esum *= 1.0f / kTwo31;
  }
  __syncthreads();  // block_max has read warp_f
  if (lane == 0) s.warp_f[warp] = esum;
  __syncthreads();
  if (threadIdx.x == 0) {
    float e = 0.0f;
    for (int w = 0; w < kWarps; ++w) e += s.warp_f[w];
    s.expsum = e;
  }
  sync_all();
  esum = 0.0f;
  for (int r = 0; r < C; ++r) esum += peer_f32<kStream>(&s.expsum, r);
  if (greedy) {
    int first = 0x7fffffff;
    for (int r = 0; r < C; ++r) first = min(first, static_cast<int>(peer_u32<kStream>(reinterpret_cast<const uint32_t*>(&s.first), r)));
    sync_all();
    if (leader) {
      a.tokens[row] = first - shift;
      a.conf[row] = 1.0f / esum;
    }
    return;
  }

  // ---- the last kept token of top-k and top-p ---------------------------------
  Cut cut{minus_inf, 0u, 0};
  int plan = kListAll;
  if (cut_any) {
    const uint32_t want_count = static_cast<uint32_t>(max(top_k, 0));
    uint32_t reach_lo = 0, reach_hi = 0, reach_count = 0;  // keys, and the tokens above
    auto keys_of_bins = [&](uint32_t b_hi, uint32_t b_lo) {
      // bins fall as logits rise; one warp finds either end
      if (warp == 0) {
        const uint32_t k = first_key(kmin, kmax, [&](uint32_t k) { return bin_of_key(k) <= b_lo; });
        if (lane == 0) s.klo = k;
      } else if (warp == 1) {
        const uint32_t k =
            b_hi == 0 ? kmax + 1
                      : first_key(kmin, kmax, [&](uint32_t k) { return bin_of_key(k) < b_hi; });
        if (lane == 0) s.khi = k - 1;
      }
      __syncthreads();
      reach_lo = s.klo;
      reach_hi = s.khi;
    };

    if (listed_already) {
      reach_lo = s.klo;
      reach_hi = kmax;
      if (s.n_list > kList || s.n_list < want_count) plan = kWhole;
      __syncthreads();
    } else {  // ---- the bins that the cut can lie in -----------------------------
      constexpr int kPer = kFine / kThreads;  // bins of a thread
      const int bin0 = threadIdx.x * kPer;
      uint32_t n[kPer] = {};
      for (int r = 0; r < C; ++r) {
        if constexpr (kPer == 4) {
          const uint4 v = peer_u32x4<kStream>(&s.fine[bin0], r);
          n[0] += v.x; n[1] += v.y; n[2] += v.z; n[3] += v.w;
        } else {
#pragma unroll
          for (int i = 0; i < kPer; ++i) n[i] = s.fine[bin0 + i];
        }
      }
      float w[kPer];  // the bins' middle weights, rounded down as every weight is
      float middle = exp2f(31.0f - static_cast<float>(threadIdx.x) * (kPer / 32.0f));
      uint32_t own_n = 0;
      float own_m = 0.0f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        w[i] = floorf(middle);
        middle *= 0.97857206208770013f;  // 2^(-1/32)
        own_n += n[i];
        own_m += n[i] * w[i];
      }
      uint32_t cnt = warp_before(own_n);
      float est = warp_before(own_m);
      if (lane == 31) {
        s.warp_c[warp] = cnt + own_n;
        s.warp_f[warp] = est + own_m;
      }
      if (threadIdx.x < 4) {
        // (top-p: a bin that rounding keeps from being named is the last one, below
        // which no weight counts)
        s.bin[threadIdx.x] = by_k ? kFine : kFine - 1;
        s.at[threadIdx.x] = 0;
      }
      __syncthreads();
      float whole = 0.0f;
      for (int i = 0; i < kWarps; ++i) {
        if (i < warp) {
          cnt += s.warp_c[i];
          est += s.warp_f[i];
        }
        whole += s.warp_f[i];
      }
      // top-p: a bin's weights are within 1.1 % of the middle one.  The cut is taken to
      // lie no earlier than the first bin up to which the sum may reach top_p of the
      // whole, and no later than the first at which it must, by the weights up to a
      // bin or by those behind it, of which 1 - top_p is left: next to top_p = 1 they
      // alone tell bins apart.  The second pair is closer, for rows whose first holds
      // too many tokens.  A pair that misses is found out by the search, which adds
      // the weights up exactly, and costs time alone.
      const float want = top_p * whole, rest = (1.0f - top_p) * whole;
      auto may = [&](float e, float off) {
        return e * (1.0f + off) >= want && (whole - e) * (1.0f - off) <= rest;
      };
      auto must = [&](float e, float off) {
        return e * (1.0f - off) >= want || (whole - e) * (1.0f + off) <= rest;
      };
      uint32_t c0 = cnt;
      float e0 = est;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        c0 += n[i];
        e0 += n[i] * w[i];
        if (n[i] == 0) continue;
        const int b = bin0 + i;
        if (by_k) {
          if (c0 >= want_count && c0 - n[i] < want_count) s.bin[0] = s.bin[1] = b;
        } else {
          // (a little less: the threads' running sums round differently)
          const float d0 = (e0 - n[i] * w[i]) * 0.9999f;
          if (may(e0, 0.012f) && !may(d0, 0.012f)) atomicMin(&s.bin[0], b);
          if (must(e0, 0.012f) && !must(d0, 0.012f)) atomicMin(&s.bin[1], b);
          if (may(e0, 0.003f) && !may(d0, 0.003f)) atomicMin(&s.bin[2], b);
          if (must(e0, 0.003f) && !must(d0, 0.003f)) atomicMin(&s.bin[3], b);
        }
      }
      __syncthreads();
      c0 = cnt;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int b = bin0 + i;
        if (b == s.bin[0]) s.at[0] = c0;
        if (b == s.bin[2]) s.at[2] = c0;
        c0 += n[i];
        if (b == s.bin[1]) s.at[1] = c0;
        if (b == s.bin[3]) s.at[3] = c0;
      }
      __syncthreads();
      const uint32_t room = static_cast<uint32_t>(kList * C) / 4 * 3;
      int b_hi = s.bin[0], b_lo = s.bin[1];
      uint32_t above = s.at[0], upto = s.at[1];
      if (b_lo < kFine && upto <= kList) {
        b_hi = 0;
        above = 0;
      } else {
        plan = kListReach;
        if (upto - above > room) {
          b_hi = s.bin[2];
          b_lo = s.bin[3];
          above = s.at[2];
          upto = s.at[3];
        }
        if (b_lo >= kFine || b_hi > b_lo || upto - above > room || (by_k && by_p)) plan = kWhole;
      }
      if (plan != kWhole) {
        reach_count = above;
        keys_of_bins(b_hi, b_lo);
      }
    }

    // weights of all tokens, of those above `from` that min-p keeps by segments,
    // and of the others above; visit(i, z) for every step
    auto weigh_pass = [&](auto min_c, float from, auto visit, unsigned long long* all_out,
                          unsigned long long* above_out) {
      constexpr bool kMin = decltype(min_c)::value;
      unsigned long long all = 0, above = 0;
      for (int g = 0; g < segs; ++g) {
        unsigned long long seg = 0;
        each_step(g * kSegSteps, min(steps, (g + 1) * kSegSteps), [&](int i, const float (&z)[8],
                                                                  const uint4 (&raw)[kRaw]) {
#pragma unroll
          for (int j = 0; j < 8; j += 2) {
            const Pair w = weigh(z[j], z[j + 1], neg_m, c);
            const uint32_t w0 = z[j] > from ? w.w0 : 0u, w1 = z[j + 1] > from ? w.w1 : 0u;
            add_wide(all, w.w0);
            add_wide(all, w.w1);
            if (kMin) {  // segments: what min-p keeps; above: the rest
              add_wide(seg, w0 >= w_min ? w0 : 0u);
              add_wide(seg, w1 >= w_min ? w1 : 0u);
              add_wide(above, w0 >= w_min ? 0u : w0);
              add_wide(above, w1 >= w_min ? 0u : w1);
            } else {
              add_wide(seg, w0);
              add_wide(seg, w1);
            }
          }
          visit(i, z, raw);
        });
        above += seg;
        seg = warp_sum(seg);
        if (lane == 0) set_seg(g, seg, 0);
      }
      all = warp_sum(all);
      above = warp_sum(above);
      if (lane == 0) {
        s.warp_m[0][warp] = all;
        s.warp_m[1][warp] = above;
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        all = above = 0;
        for (int w = 0; w < kWarps; ++w) {
          all += s.warp_m[0][w];
          above += s.warp_m[1][w];
        }
        *all_out = all;
        if (above_out) *above_out = above;
      }
    };

    unsigned long long total = 0, above_mass = 0;
    if (plan != kWhole && !listed_already) {
      // ---- the tokens in reach of the cut, and the weights above them ---------
      const float flo = key_value<Te>(reach_lo), fhi = key_value<Te>(reach_hi);
      auto put = [&](int i, const float (&z)[8], const uint4 (&raw)[kRaw]) {
        enlist(plan == kListAll, flo, fhi, i, z, raw);
      };
      if (plan == kListAll && by_k) {  // no weight but the listed ones counts
        if (lane_max >= flo) each_step(0, steps, put);
        for (int g = lane; g < segs; g += 32) set_seg(g, 0, 0);
      } else {
        if (w_min) weigh_pass(std::true_type(), fhi, put, &s.mass, &s.reach_mass);
        else weigh_pass(std::false_type(), fhi, put, &s.mass, &s.reach_mass);
      }
      sync_all();
      const bool weighed = plan == kListReach || !by_k;
      for (int r = 0; r < C; ++r) {
        if (peer_u32<kStream>(&s.n_list, r) > kList) plan = kWhole;
        if (weighed) {
          total += peer_u64<kStream>(&s.mass, r);
          above_mass += peer_u64<kStream>(&s.reach_mass, r);
        }
      }
    }

    // The search; false: the cut is not in the list.
    auto listed = [&](int i) {
      if constexpr (kStream) return s.list.z[i];
      else return to_f32(z_s[s.list.place[i]]);
    };
    auto search = [&]() {
      cut.mass = total;
      for (int which = 0; which < 2; ++which) {
        const bool count_rule = which == 0;
        if (count_rule ? !by_k : !by_p) continue;
        // sums are below 2^53: reaching p * mass is reaching it rounded up
        const unsigned long long want =
            count_rule ? want_count
                       : static_cast<unsigned long long>(
                             ceil(static_cast<double>(top_p) * static_cast<double>(cut.mass)));
        if (!count_rule && above_mass >= want) return false;
        uint32_t klo = reach_lo, khi = reach_hi;
        if (threadIdx.x == 0) {
          s.above_count = reach_count;
          s.above_mass = above_mass;
        }
        bool counted = false;
        while (klo < khi || !counted) {
          const uint32_t width = khi - klo;  // one less than the keys
          const int sh = max(0, 25 - __clz(width));
          // the cluster has read this histogram's last contents
          sync_all();
          for (int i = threadIdx.x; i < static_cast<int>(sizeof(Hist) / 4); i += kThreads)
            reinterpret_cast<uint32_t*>(&s.hist)[i] = 0u;
          __syncthreads();
          auto count_in = [&](float z) {
            const uint32_t k = key_of<Te>(z);
            if (k - klo > width) return;
            const uint32_t b = (khi - k) >> sh, w = weight_of(z, neg_m, c);
            atomicAdd(&s.hist.count[b], 1u);
            atomicAdd(&s.hist.m0[b], w & 0x7ffu);
            atomicAdd(&s.hist.m1[b], w >> 11 & 0x7ffu);
            atomicAdd(&s.hist.m2[b], w >> 22);
          };
          if (plan == kWhole) {
            const float flo = key_value<Te>(klo), fhi = key_value<Te>(khi);
            each_step(0, steps, [&](int, const float (&z)[8], const uint4 (&)[kRaw]) {
#pragma unroll
              for (int j = 0; j < 8; ++j)
                if (z[j] >= flo && z[j] <= fhi) count_in(z[j]);
            });
          } else {
            const int n = static_cast<int>(s.n_list);
            for (int i = threadIdx.x; i < n; i += kThreads) count_in(listed(i));
          }
          sync_all();
          counted = true;
          if (warp == 0) {
            const int b = find_bin<kStream>(s, C, count_rule, want, s.above_mass, s.above_count);
            if (lane == 0) {
              const uint32_t top = khi - (static_cast<uint32_t>(b < 0 ? 0 : b) << sh);
              s.khi = top;
              s.klo = b < 0 ? top : top - min(top - klo, (1u << sh) - 1u);
              if (b < 0) s.bin_count = 0;
            }
          }
          __syncthreads();
          klo = s.klo;
          khi = s.khi;
          if (s.bin_count == 0) break;
          __syncthreads();
        }
        if (s.bin_count == 0) {  // not reached: in the whole row, nothing is cut
          __syncthreads();
          if (plan != kWhole) return false;
          continue;
        }
        const unsigned long long w = s.bin_mass / s.bin_count, above = s.above_mass;
        const uint32_t ties = s.bin_count, above_count = s.above_count;
        __syncthreads();
        // the smallest r with r tokens of the cut's logit reaching what is asked for
        const unsigned long long r =
            count_rule ? want - above_count : (w ? (want - above + w - 1) / w : 1);
        cut.value = key_value<Te>(klo);
        cut.ties = static_cast<uint32_t>(r < ties ? r : ties);
        cut.mass = above + cut.ties * w;
      }
      return true;
    };
    if (plan == kWhole || !search()) {
      // ---- the same over every token ----------------------------------------------
      plan = kWhole;
      if (by_p) {
        weigh_pass(std::false_type(), m, [](int, const float (&)[8], const uint4 (&)[kRaw]) {}, &s.whole_mass, nullptr);
        sync_all();
        total = 0;
        for (int r = 0; r < C; ++r) total += peer_u64<kStream>(&s.whole_mass, r);
      }
      above_mass = 0;
      reach_count = 0;
      __syncthreads();
      keys_of_bins(0, kFine - 1);
      cut = Cut{minus_inf, 0u, 0};
      search();
    }
  }

  // ---- the kept mass of each segment ------------------------------------------
  const bool cut_used = cut.value > minus_inf;
  uint32_t w_tie = 0;
  if (cut_used) {
    w_tie = weight_of(cut.value, neg_m, c);
    if (w_tie < w_min) w_tie = 0;
  }
  if (cut_any) {
    __syncthreads();
    if (plan != kWhole) {
      const int n = static_cast<int>(s.n_list);
      for (int i = threadIdx.x; i < n; i += kThreads) {
        const int place = s.list.place[i], at = place / (steps * kStep);
        const int q = at * segs + (place - at * steps * kStep) / (kSegSteps * kStep);
        float z;
        if constexpr (kStream) z = s.list.z[i];
        else z = to_f32(z_s[place]);
        if (z > cut.value) {
          const uint32_t w = weight_of(z, neg_m, c);
          if (w >= w_min) {
            atomicAdd(&s.seg_lo[q], w & 0xffffu);
            atomicAdd(&s.seg_hi[q], w >> 16);
          }
        } else if (z == cut.value) {
          atomicAdd(&s.seg_ties[q], 1u);
        }
      }
    } else {
      for (int g = 0; g < segs; ++g) {
        unsigned long long seg = 0;
        uint32_t ties = 0;
        each_step(g * kSegSteps, min(steps, (g + 1) * kSegSteps), [&](int, const float (&z)[8], const uint4 (&)[kRaw]) {
#pragma unroll
          for (int j = 0; j < 8; j += 2) {
            const Pair p = weigh(z[j], z[j + 1], neg_m, c);
            add_wide(seg, z[j] > cut.value && p.w0 >= w_min ? p.w0 : 0u);
            add_wide(seg, z[j + 1] > cut.value && p.w1 >= w_min ? p.w1 : 0u);
            ties += (cut_used && z[j] == cut.value) + (cut_used && z[j + 1] == cut.value);
          }
        });
        seg = warp_sum(seg);
        ties = __reduce_add_sync(0xffffffffu, ties);
        if (lane == 0) set_seg(g, seg, ties);
      }
    }
  }
  if (cut_any) sync_all();

  // ---- the segment that u falls in, then the token -----------------------------
  if (warp == 0) {
    const int per_cta = kWarps * segs, all = per_cta * C;
    const int per_lane = (all + 31) / 32;  // segments, in order; at most 32
    auto seg_at = [&](int q, uint32_t& ties) {
      ties = 0;
      if (q >= all) return 0ull;
      const int r = q / per_cta, l = q - r * per_cta;
      ties = peer_u32<kStream>(&s.seg_ties[l], r);
      return peer_u64<kStream>(&s.seg_mass[l], r) + peer_u32<kStream>(&s.seg_lo[l], r) +
             (static_cast<unsigned long long>(peer_u32<kStream>(&s.seg_hi[l], r)) << 16);
    };
    // kept mass given the tokens equal to the cut before
    auto with_ties = [&](unsigned long long above, uint32_t before, uint32_t ties) {
      const uint32_t left = cut.ties > before ? cut.ties - before : 0u;
      return above + static_cast<unsigned long long>(min(left, ties)) * w_tie;
    };
    unsigned long long above = 0;
    uint32_t ties = 0;
    for (int i = 0; i < per_lane; ++i) {
      uint32_t n;
      above += seg_at(lane * per_lane + i, n);
      ties += n;
    }
    uint32_t before = warp_before(ties);
    unsigned long long kept = with_ties(above, before, ties);
    unsigned long long upto = warp_before(kept) + kept;
    // sums are integers below 2^53: exceeding u * mass is exceeding it rounded down
    const unsigned long long target = static_cast<unsigned long long>(
        static_cast<double>(u) * static_cast<double>(__shfl_sync(0xffffffffu, upto, 31)));
    // u < 1: some lane's running mass exceeds the target
    int f = __ffs(__ballot_sync(0xffffffffu, upto > target) | 1u << 31) - 1;
    unsigned long long run = __shfl_sync(0xffffffffu, upto - kept, f);
    uint32_t run_ties = __shfl_sync(0xffffffffu, before, f);
    // the lane's segments, one a lane
    above = seg_at(lane < per_lane ? f * per_lane + lane : all, ties);
    before = run_ties + warp_before(ties);
    kept = with_ties(above, before, ties);
    upto = run + warp_before(kept) + kept;
    const int q = f * per_lane;
    f = __ffs(__ballot_sync(0xffffffffu, upto > target) | 1u << 31) - 1;
    run = __shfl_sync(0xffffffffu, upto - kept, f);
    run_ties = __shfl_sync(0xffffffffu, before, f);
    const int found = min(q + f, all - 1);
    if (!kStream) cluster_arrive();  // the rest reads this CTA's memory alone
    if (found / per_cta == rank) {
      const int l = found % per_cta, w0 = l / segs, g = l % segs;
      uint4 raw[kSegSteps][kRaw];
#pragma unroll
      for (int i = 0; i < kSegSteps; ++i)
        fetch((w0 * steps + min(g * kSegSteps + i, steps - 1)) * kStep + lane * 8, raw[i]);
#pragma unroll
      for (int i = 0; i < kSegSteps; ++i) {
        if (g * kSegSteps + i >= steps) break;
        const int off = (w0 * steps + g * kSegSteps + i) * kStep + lane * 8;
        float z[8];
        open(raw[i], z);
        uint32_t w[8];
        ties = 0;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const Pair p = weigh(z[j], z[j + 1], neg_m, c);
          w[j] = z[j] > cut.value && p.w0 >= w_min ? p.w0 : 0u;
          w[j + 1] = z[j + 1] > cut.value && p.w1 >= w_min ? p.w1 : 0u;
          ties += (cut_used && z[j] == cut.value) + (cut_used && z[j + 1] == cut.value);
        }
        before = run_ties + warp_before(ties);
        run_ties = __shfl_sync(0xffffffffu, before + ties, 31);
        kept = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (cut_used && z[j] == cut.value) w[j] = before++ < cut.ties ? w_tie : 0u;
          kept += w[j];
        }
        upto = run + warp_before(kept) + kept;
        const uint32_t hit = __ballot_sync(0xffffffffu, upto > target);
        if (hit) {
          if (lane == __ffs(hit) - 1) {
            unsigned long long at = upto - kept;
            int pick = 7;
            float zt = z[7];
            bool done = false;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              at += w[j];
              if (!done && at > target) {
                done = true;
                pick = j;
                zt = z[j];
              }
            }
            a.tokens[row] = pos0 + off + pick - shift;
            a.conf[row] = expf(zt + neg_m) / esum;
          }
          break;
        }
        run = __shfl_sync(0xffffffffu, upto, 31);
      }
    }
  }
  if (!kStream) {
    if (warp != 0) cluster_arrive();
    cluster_wait();  // no CTA leaves while its sums are read
  }
}

template <typename Te, bool kStream>
__global__ void __launch_bounds__(Shape<kStream>::kThreads, Shape<kStream>::kCtas)
    sample_kernel(const Args a) {
  extern __shared__ __align__(16) uint8_t smem[];
  Shared<kStream>& s = *reinterpret_cast<Shared<kStream>*>(smem);
  Te* z_s = reinterpret_cast<Te*>(smem + (sizeof(s) + 15) / 16 * 16);  // a cluster's slice
  grid_dep_wait();
  grid_dep_launch();
  if constexpr (!kStream) {
    const int C = cluster_size();
    sample_row<Te, false>(a, s, z_s, C, cluster_rank(), blockIdx.x / C);
  } else {
    sample_row<Te, true>(a, s, z_s, 1, 0, blockIdx.x);
  }
}

template <typename Te, bool kStream>
cudaError_t launch_shape(const Args& a, int rows, int C, cudaStream_t stream) {
  auto kernel = sample_kernel<Te, kStream>;
  const size_t smem = (sizeof(Shared<kStream>) + 15) / 16 * 16 + (kStream ? 0 : a.slice * sizeof(Te));
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {static_cast<unsigned>(C), 1, 1};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(rows) * C);
  cfg.blockDim = dim3(Shape<kStream>::kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = C > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename Te>
cudaError_t launch_typed(Args a, int rows, int num_sms, cudaStream_t stream) {
  // positions that may precede a row in its first 16 bytes
  const bool whole = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 &&
                     (rows == 1 || a.ld * static_cast<int64_t>(sizeof(Te)) % 16 == 0);
  const int lead = whole ? 0 : 16 / static_cast<int>(sizeof(Te)) - 1;
  auto slice_of = [&](int C, int grain) {
    const int per = (a.vocab + lead + C - 1) / C;
    return (per + grain - 1) / grain * grain;
  };
  constexpr int kGrain = Shape<false>::kWarps * kStep;
  // CTAs a row: slices of at most 56 KB (three CTAs an SM), or what eight CTAs
  // give; more for few rows, as long as each has a step for every warp
  int C = 1;
  while (C < 8 && slice_of(C, kGrain) * sizeof(Te) > 56 * 1024) ++C;
  // A row that no CTA holds is streamed as soon as the rows fill half of the SMs
  // (rows of 131072 bf16 logits, cluster / stream in us, plain, top-k 50, top-p
  // 0.9: 32 rows 17, 26, 34 / 21, 27, 50; 76 rows 20, 29, 39 / 21, 27, 50; 100 rows
  // 28, 49, 60 / 22, 27, 49; 304 rows 59, 99, 131 / 34, 36, 75).
  if (C > 1 && 2 * static_cast<int64_t>(rows) >= num_sms) {
    a.slice = slice_of(1, Shape<true>::kWarps * kStep);
    return launch_shape<Te, true>(a, rows, 1, stream);
  }
  while (C < 8 && static_cast<int64_t>(rows) * C * 2 <= num_sms && slice_of(C, kGrain) > kGrain)
    C = std::min(8, C * 2);
  a.slice = slice_of(C, kGrain);
  return launch_shape<Te, false>(a, rows, C, stream);
}

}  // namespace

int sample_max_vocab() { return kMaxVocab; }

cudaError_t launch_sample(int dtype, const SampleArgs& p, int num_sms, cudaStream_t stream) {
  Args a{p.logits, p.ld,    p.vocab, 0,        p.temperature, p.top_k, p.top_p,
         p.min_p,  p.u,     p.masked, p.tokens, p.conf,        p.err};
  if (dtype == 0) return launch_typed<float>(a, p.rows, num_sms, stream);
  return launch_typed<__nv_bfloat16>(a, p.rows, num_sms, stream);
}

}  // namespace rx
