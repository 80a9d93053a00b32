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
// in a double, in which the comparisons with p * mass and u * mass are made.
//
// A row is held in shared memory by a cluster of 1 to 8 CTAs: it crosses HBM
// once, and what the filters need beyond one pass over the weights are cheap
// passes of comparisons.  The last kept token of top-k and of top-p (by logit,
// then index) is found from a histogram of the weights by eighths of an octave
// and, inside the bin that it falls in, by the logits' bits, 128 bins a pass.
// Then one warp walks the 1024 tokens that u falls in.
//
// Bound: the fp32 pipes (about 20 operations a token in packed pairs) close
// above HBM.
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace rx {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kStep = 256;         // tokens of a warp's step: 8 consecutive ones a lane
constexpr int kSegSteps = 4;       // steps of a segment
constexpr int kBins = 128;
constexpr int kCoarse = 96;        // level 0: eighths of an octave down to 2^-12, and the rest
constexpr int kMaxSegs = 64;       // per CTA
constexpr int kMaxVocab = 1 << 18;

struct Hist {  // of one pass; masses in two halves of 16 bits, at most 2^16 tokens each
  uint32_t count[kBins], lo[kBins], hi[kBins];
};

struct Shared {
  Hist hist[2];
  unsigned long long seg_mass[kMaxSegs];
  uint32_t seg_ties[kMaxSegs];
  unsigned long long mass;  // of the CTA's tokens
  uint32_t tail;            // its tokens in the last coarse bin
  float max, expsum;
  int first;                // greedy: its first token of the largest logit
  // results of a search
  unsigned long long above_mass, bin_mass;
  uint32_t above_count, bin_count, klo, khi;
  float warp_f[kWarps];
  unsigned long long warp_m[kWarps];
};

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
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer(const void* p, int rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ uint32_t ld_peer_u32(const void* p, int rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(peer(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ unsigned long long ld_peer_u64(const void* p, int rank) {
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(peer(p, rank)) : "memory");
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
__device__ __forceinline__ int coarse_bin(float t) {
  return t > -12.0f ? static_cast<int>(t * -8.0f) : kCoarse;
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

// Sums the cluster's histograms (and, at level 0, the rest of the mass and
// count in bin kCoarse) and finds the first bin at which the running count
// reaches want_count (by_count) or the running mass want_mass.  Warp 0 of
// each CTA; the result goes to s.above_*, s.bin_*; returns the bin, or -1.
__device__ int find_bin(Shared& s, const Hist& h, int C, bool level0, unsigned long long total,
                        bool by_count, unsigned long long want_count, double want_mass,
                        unsigned long long mass0, unsigned long long count0) {
  const int lane = threadIdx.x & 31;
  unsigned long long cnt[4], mass[4], my_c = 0, my_m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = lane * 4 + i;
    cnt[i] = mass[i] = 0;
    for (int r = 0; r < C; ++r) {
      cnt[i] += ld_peer_u32(&h.count[b], r);
      mass[i] += ld_peer_u32(&h.lo[b], r) +
                 (static_cast<unsigned long long>(ld_peer_u32(&h.hi[b], r)) << 16);
    }
    my_c += cnt[i];
    my_m += mass[i];
  }
  if (level0) {
    // what the coarse bins leave lies in the last one
    const unsigned long long rest = total - warp_sum(my_m);
    if (lane * 4 == kCoarse) {
      unsigned long long tail = 0;
      for (int r = 0; r < C; ++r) tail += ld_peer_u32(&s.tail, r);
      cnt[0] = tail;
      mass[0] = rest;
      my_c += tail;
      my_m += rest;
    }
  }
  unsigned long long c = my_c, m = my_m;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long pc = __shfl_up_sync(0xffffffffu, c, o);
    const unsigned long long pm = __shfl_up_sync(0xffffffffu, m, o);
    if (lane >= o) {
      c += pc;
      m += pm;
    }
  }
  c += count0 - my_c;
  m += mass0 - my_m;
  int hit = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool reached = by_count ? c + cnt[i] >= want_count
                                  : static_cast<double>(m + mass[i]) >= want_mass;
    if (hit < 0 && cnt[i] > 0 && reached) {
      hit = lane * 4 + i;
      my_c = cnt[i];
      my_m = mass[i];
    } else if (hit < 0) {
      c += cnt[i];
      m += mass[i];
    }
  }
  const uint32_t any = __ballot_sync(0xffffffffu, hit >= 0);
  if (any == 0) return -1;
  const int from = __ffs(any) - 1;
  if (lane == from) {
    s.above_count = static_cast<uint32_t>(c);
    s.above_mass = m;
    s.bin_count = static_cast<uint32_t>(my_c);
    s.bin_mass = my_m;
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

struct Cut {  // kept: logits above `value`, and the first `ties` of those equal to it
  float value;
  uint32_t ties;
  unsigned long long mass;  // of what is kept
};

template <typename Te>
__global__ void __launch_bounds__(kThreads, 3) sample_kernel(const Args a) {
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& s = *reinterpret_cast<Shared*>(smem);
  Te* z_s = reinterpret_cast<Te*>(smem + (sizeof(Shared) + 15) / 16 * 16);
  constexpr int kVec = 16 / sizeof(Te);
  const int C = cluster_size(), rank = cluster_rank();
  const int64_t row = blockIdx.x / C;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool leader = rank == 0 && threadIdx.x == 0;
  grid_dep_wait();
  grid_dep_launch();

  // the row's settings; a row that is left out or refused costs no loads
  float temp = a.temperature ? a.temperature[row] : 1.0f;
  const int top_k = a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.0f;
  const float min_p = a.min_p ? a.min_p[row] : 0.0f;
  float u = a.u[row];
  const bool out = a.masked != nullptr && a.masked[row] == 0;
  const bool bad = !(temp >= 0.0f && temp <= 3.4e38f) || !(top_p > 0.0f) || !(min_p <= 1.0f) ||
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

  // ---- the CTA's tokens into shared memory, their largest logit -------------
  // Positions are counted from the 16-byte boundary at or below the row's
  // start, so every vector of positions is one aligned load; positions outside
  // the row hold -inf.
  const Te* start = static_cast<const Te*>(a.logits) + row * a.ld;
  const int shift = static_cast<int>(reinterpret_cast<uintptr_t>(start) % 16 / sizeof(Te));
  const int lo = shift, hi = shift + a.vocab;  // positions of the row
  const Te* base = start - shift;
  const int pos0 = rank * a.slice;
  const int steps = a.slice / (kWarps * kStep);  // of each warp
  Te* mine = z_s + warp * steps * kStep + lane * 8;
  const int my_pos = pos0 + warp * steps * kStep + lane * 8;
  const float minus_inf = __int_as_float(0xff800000);
  float m = minus_inf;
  auto keep = [&](int i, const uint4 (&raw)[8 / kVec]) {
#pragma unroll
    for (int v = 0; v < 8 / kVec; ++v)
      *reinterpret_cast<uint4*>(mine + i * kStep + v * kVec) = raw[v];
    float z[8];
    load8(reinterpret_cast<const Te*>(raw), z);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, z[j]);  // a NaN is no maximum
  };
  const int first_pos = pos0 + warp * steps * kStep;
  const int whole =  // steps of the warp that lie in the row
      first_pos < lo ? 0 : max(0, min(steps, (hi - first_pos) / kStep));
#pragma unroll 4
  for (int i = 0; i < whole; ++i) {
    uint4 raw[8 / kVec];
#pragma unroll
    for (int v = 0; v < 8 / kVec; ++v)
      raw[v] = __ldcs(reinterpret_cast<const uint4*>(base + my_pos + i * kStep + v * kVec));
    keep(i, raw);
  }
  for (int i = whole; i < steps; ++i) {
    uint4 raw[8 / kVec];
#pragma unroll
    for (int v = 0; v < 8 / kVec; ++v) {
      const int q = my_pos + i * kStep + v * kVec;
      if (q >= lo && q + kVec <= hi) {
        raw[v] = __ldcs(reinterpret_cast<const uint4*>(base + q));
      } else {
        Te* e = reinterpret_cast<Te*>(&raw[v]);
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          e[j] = q + j >= lo && q + j < hi ? base[q + j] : from_f32<Te>(minus_inf);
      }
    }
    keep(i, raw);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) s.warp_f[warp] = m;
  for (int i = threadIdx.x; i < static_cast<int>(sizeof(s.hist) / 4); i += kThreads)
    reinterpret_cast<uint32_t*>(s.hist)[i] = 0u;
  if (threadIdx.x == 0) {
    s.tail = 0;
    s.first = 0x7fffffff;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, s.warp_f[w]);
    s.max = m;
  }
  cluster_sync();
  m = minus_inf;
  for (int r = 0; r < C; ++r) m = fmaxf(m, __uint_as_float(ld_peer_u32(&s.max, r)));
  if (!(m > minus_inf)) {  // nothing to sample from
    cluster_sync();
    if (leader) {
      a.tokens[row] = -1;
      a.conf[row] = 0.0f;
    }
    return;
  }
  if (m > 3.4028234e38f) {  // +inf: those tokens alone, alike
    for (int i = 0; i < steps; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float z = to_f32(mine[i * kStep + j]);
        mine[i * kStep + j] = from_f32<Te>(z == m ? 0.0f : minus_inf);
      }
    m = 0.0f;
  }
  const float neg_m = -m;
  const float c = fminf(__fdiv_rn(kLog2e, temp), 3.4028234e38f);
  const bool same_t = c == kLog2e;
  const bool by_k = !greedy && top_k > 0, by_p = !greedy && top_p < 1.0f;
  const bool cut_any = by_k || by_p, by_min = !greedy && min_p > 0.0f;

  // ---- one pass over the weights ----------------------------------------------
  const int segs = (steps + kSegSteps - 1) / kSegSteps;  // of each warp
  float esum = 0.0f;
  {
    unsigned long long mass = 0;
    uint32_t tail = 0;
    int first = 0x7fffffff;
    for (int g = 0; g < segs; ++g) {
      unsigned long long seg = 0;
      const int i1 = min(steps, (g + 1) * kSegSteps);
      for (int i = g * kSegSteps; i < i1; ++i) {
        float z[8];
        load8(mine + i * kStep, z);
        if (greedy) {
#pragma unroll
          for (int j = 7; j >= 0; --j)
            if (z[j] == m) first = min(first, my_pos + i * kStep + j);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            esum += ex2(fmaxf(__fmul_rn(__fadd_rn(z[j], neg_m), kLog2e), -126.0f));
          continue;
        }
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const Pair w = weigh(z[j], z[j + 1], neg_m, c);
          seg += w.w0;
          seg += w.w1;
          if (same_t) {
            esum += w.v0 + w.v1;
          } else {
            float d0, d1;
            upk(mul2(w.d, pk(kLog2e, kLog2e)), d0, d1);
            esum += ex2(fmaxf(d0, -126.0f)) + ex2(fmaxf(d1, -126.0f));
          }
          if (cut_any) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float t = h ? w.t1 : w.t0;
              const uint32_t ww = h ? w.w1 : w.w0;
              if (t > -12.0f) {
                const int b = coarse_bin(t);
                atomicAdd(&s.hist[0].count[b], 1u);
                atomicAdd(&s.hist[0].lo[b], ww & 0xffffu);
                atomicAdd(&s.hist[0].hi[b], ww >> 16);
              } else if (t > -32.0f) {
                ++tail;
              }
            }
          }
        }
      }
      if (!greedy) {
        seg = warp_sum(seg);
        mass += seg;
        if (lane == 0) {
          s.seg_mass[warp * segs + g] = seg;
          s.seg_ties[warp * segs + g] = 0;
        }
      }
    }
    if (same_t && !greedy) esum *= 1.0f / kTwo31;
    esum = warp_sum(esum);
    if (lane == 0) {
      s.warp_f[warp] = esum;
      s.warp_m[warp] = mass;
    }
    if (cut_any && tail) atomicAdd(&s.tail, tail);
    if (greedy && first != 0x7fffffff) atomicMin(&s.first, first);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    float e = 0.0f;
    unsigned long long t = 0;
    for (int w = 0; w < kWarps; ++w) {
      e += s.warp_f[w];
      t += s.warp_m[w];
    }
    s.expsum = e;
    s.mass = t;
  }
  cluster_sync();
  esum = 0.0f;
  unsigned long long total = 0;
  for (int r = 0; r < C; ++r) {
    esum += __uint_as_float(ld_peer_u32(&s.expsum, r));
    total += ld_peer_u64(&s.mass, r);
  }
  if (greedy) {
    int first = 0x7fffffff;
    for (int r = 0; r < C; ++r) first = min(first, static_cast<int>(ld_peer_u32(&s.first, r)));
    cluster_sync();
    if (leader) {
      a.tokens[row] = first - shift;
      a.conf[row] = 1.0f / esum;
    }
    return;
  }

  // ---- the last kept token of top-k and top-p ---------------------------------
  Cut cut{minus_inf, 0u, total};
  const unsigned long long want_count = static_cast<unsigned long long>(top_k);
  for (int which = 0; which < 2; ++which) {
    const bool count_rule = which == 0;
    if (count_rule ? !by_k : !by_p) continue;
    const double want_mass =
        count_rule ? 0.0 : static_cast<double>(top_p) * static_cast<double>(cut.mass);
    // level 0 is kept for the second search; deeper levels use the other one
    __syncthreads();
    if (warp == 0) {
      const int b = find_bin(s, s.hist[0], C, true, total, count_rule, want_count, want_mass, 0, 0);
      uint32_t klo = 1, khi = 0;  // none
      if (b >= 0) {
        // the bin's logits: keys from the first whose bin is at most b to the
        // last whose bin is not below b (bins fall as logits rise)
        const uint32_t kmax = key_of<Te>(m), kmin = key_of<Te>(minus_inf);
        auto bin_at = [&](uint32_t k) {
          const float t = fmaxf(__fmul_rn(__fadd_rn(key_value<Te>(k), neg_m), c), -40.0f);
          return t > -32.0f ? coarse_bin(t) : kCoarse + 1;
        };
        klo = first_key(kmin, kmax, [&](uint32_t k) { return bin_at(k) <= b; });
        khi = first_key(klo, kmax, [&](uint32_t k) { return bin_at(k) < b; }) - 1;
      }
      if (lane == 0) {
        s.klo = klo;
        s.khi = khi;
      }
    }
    __syncthreads();
    uint32_t klo = s.klo, khi = s.khi;
    if (klo > khi) continue;  // fewer tokens than asked for: nothing is cut
    while (klo < khi) {
      const uint32_t width = khi - klo;  // one less than the keys
      const int sh = max(0, 25 - __clz(width));
      Hist& h = s.hist[1];
      // the cluster has read this histogram's last contents
      cluster_sync();
      for (int i = threadIdx.x; i < static_cast<int>(sizeof(Hist) / 4); i += kThreads)
        reinterpret_cast<uint32_t*>(&h)[i] = 0u;
      __syncthreads();
      const float flo = key_value<Te>(klo), fhi = key_value<Te>(khi);
      for (int i = 0; i < steps; ++i) {
        float z[8];
        load8(mine + i * kStep, z);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (z[j] >= flo && z[j] <= fhi) {  // false for a NaN
            const uint32_t k = key_of<Te>(z[j]);
            if (k - klo > width) continue;  // a zero next to a bound at the other zero
            const uint32_t b = (khi - k) >> sh, ww = weight_of(z[j], neg_m, c);
            atomicAdd(&h.count[b], 1u);
            atomicAdd(&h.lo[b], ww & 0xffffu);
            atomicAdd(&h.hi[b], ww >> 16);
          }
      }
      cluster_sync();
      if (warp == 0) {
        const int b = find_bin(s, h, C, false, 0, count_rule, want_count, want_mass, s.above_mass,
                               s.above_count);
        if (lane == 0) {
          const uint32_t top = khi - (static_cast<uint32_t>(b < 0 ? 0 : b) << sh);
          s.khi = top;
          s.klo = b < 0 ? top : top - min(top - klo, (1u << sh) - 1u);
        }
      }
      __syncthreads();
      klo = s.klo;
      khi = s.khi;
      __syncthreads();
    }
    const float value = key_value<Te>(klo);
    const unsigned long long w = s.bin_mass / s.bin_count, above = s.above_mass;
    unsigned long long r;
    if (count_rule) {
      r = want_count - s.above_count;
    } else {
      // the smallest r >= 1 with above + r w >= want
      r = w ? static_cast<unsigned long long>((want_mass - static_cast<double>(above)) /
                                              static_cast<double>(w)) : 1;
      r = r > 2 ? r - 2 : 1;
      while (r < s.bin_count && static_cast<double>(above + r * w) < want_mass) ++r;
    }
    cut.value = value;
    cut.ties = static_cast<uint32_t>(r < s.bin_count ? r : s.bin_count);
    cut.mass = above + cut.ties * w;
  }

  // ---- the kept mass of each segment ------------------------------------------
  const uint32_t w_min = by_min ? static_cast<uint32_t>(ceil(static_cast<double>(min_p) *
                                                             2147483648.0)) : 0u;
  const bool cut_used = cut.value > minus_inf;
  uint32_t w_tie = 0;
  if (cut_used) {
    w_tie = weight_of(cut.value, neg_m, c);
    if (w_tie < w_min) w_tie = 0;
  }
  if (cut_used || by_min) {
    __syncthreads();
    for (int g = 0; g < segs; ++g) {
      unsigned long long seg = 0;
      uint32_t ties = 0;
      const int i1 = min(steps, (g + 1) * kSegSteps);
      for (int i = g * kSegSteps; i < i1; ++i) {
        float z[8];
        load8(mine + i * kStep, z);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (z[j] > cut.value) {
            const uint32_t w = weight_of(z[j], neg_m, c);
            seg += w >= w_min ? w : 0u;
          }
          ties += cut_used && z[j] == cut.value;
        }
      }
      seg = warp_sum(seg);
      ties = __reduce_add_sync(0xffffffffu, ties);
      if (lane == 0) {
        s.seg_mass[warp * segs + g] = seg;
        s.seg_ties[warp * segs + g] = ties;
      }
    }
  }
  cluster_sync();

  // ---- the segment that u falls in, then the token -----------------------------
  const int per_cta = kWarps * segs, all = per_cta * C;
  if (warp == 0) {
    unsigned long long kept = 0;
    // kept mass of segment q given the ties before it
    auto seg_at = [&](int q, uint32_t& ties) {
      const int r = q / per_cta, l = q % per_cta;
      ties = ld_peer_u32(&s.seg_ties[l], r);
      return ld_peer_u64(&s.seg_mass[l], r);
    };
    for (int round = 0; round < 2; ++round) {
      // round 0: the kept mass; round 1: the segment
      const double target = static_cast<double>(u) * static_cast<double>(kept);
      unsigned long long run = 0;
      uint32_t run_ties = 0;
      int found = -1;
      for (int q0 = 0; q0 < all && found < 0; q0 += 32) {
        uint32_t ties = 0;
        unsigned long long mass = q0 + lane < all ? seg_at(q0 + lane, ties) : 0;
        uint32_t before = ties;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t v = __shfl_up_sync(0xffffffffu, before, o);
          if (lane >= o) before += v;
        }
        const uint32_t tie_sum = __shfl_sync(0xffffffffu, before, 31);
        before += run_ties - ties;
        const uint32_t left = cut.ties > before ? cut.ties - before : 0u;
        mass += static_cast<unsigned long long>(min(left, ties)) * w_tie;
        unsigned long long incl = mass;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned long long v = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += v;
        }
        const unsigned long long sum = __shfl_sync(0xffffffffu, incl, 31);
        if (round == 1) {
          const uint32_t hit =
              __ballot_sync(0xffffffffu, static_cast<double>(run + incl) > target);
          if (hit) {
            const int f = __ffs(hit) - 1;
            found = q0 + f;
            run += __shfl_sync(0xffffffffu, incl - mass, f);
            run_ties = __shfl_sync(0xffffffffu, before, f);
            break;
          }
        }
        run += sum;
        run_ties += tie_sum;
      }
      if (round == 0) {
        kept = run;
      } else if (found >= 0 && found / per_cta == rank) {
        const int l = found % per_cta, w0 = l / segs, g = l % segs;
        const int i1 = min(steps, (g + 1) * kSegSteps);
        for (int i = g * kSegSteps; i < i1; ++i) {
          const int off = (w0 * steps + i) * kStep + lane * 8;
          float z[8];
          load8(z_s + off, z);
          uint32_t w[8], ties = 0;
          bool tie[8];
          unsigned long long mass = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t x = weight_of(z[j], neg_m, c);
            w[j] = z[j] > cut.value && x >= w_min ? x : 0u;
            tie[j] = cut_used && z[j] == cut.value;
            ties += tie[j];
          }
          uint32_t before = ties;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, before, o);
            if (lane >= o) before += v;
          }
          const uint32_t tie_sum = __shfl_sync(0xffffffffu, before, 31);
          before += run_ties - ties;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (tie[j]) w[j] = before++ < cut.ties ? w_tie : 0u;
            mass += w[j];
          }
          unsigned long long incl = mass;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
          }
          const uint32_t hit =
              __ballot_sync(0xffffffffu, static_cast<double>(run + incl) > target);
          if (hit) {
            if (lane == __ffs(hit) - 1) {
              unsigned long long at = run + incl - mass;
              int pick = 0;
              float zt = 0.0f;
              bool done = false;
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                at += w[j];
                if (!done && static_cast<double>(at) > target) {
                  done = true;
                  pick = j;
                  zt = z[j];
                }
              }
              a.tokens[row] = pos0 + off + pick - shift;
              a.conf[row] = ex2(fmaxf((zt + neg_m) * kLog2e, -126.0f)) / esum;
            }
            break;
          }
          run += __shfl_sync(0xffffffffu, incl, 31);
          run_ties += tie_sum;
        }
      }
    }
  }
  cluster_sync();  // no CTA leaves while its sums are read
}

template <typename Te>
cudaError_t launch_typed(Args a, int rows, int num_sms, cudaStream_t stream) {
  auto kernel = sample_kernel<Te>;
  constexpr size_t kHead = (sizeof(Shared) + 15) / 16 * 16;
  constexpr int kGrain = kWarps * kStep;
  auto slice_of = [&](int C) {  // 16 / sizeof(Te) - 1 positions may precede the row
    const int per = (a.vocab + 16 / static_cast<int>(sizeof(Te)) - 1 + C - 1) / C;
    return (per + kGrain - 1) / kGrain * kGrain;
  };
  // CTAs a row: slices of at most 70 KB, three to an SM; more for few rows,
  // as long as each has a whole step for every warp
  int C = 1;
  while (C < 8 && slice_of(C) * sizeof(Te) > 70 * 1024) C *= 2;
  while (C < 8 && static_cast<int64_t>(rows) * C * 2 <= num_sms && slice_of(C) > kGrain) C *= 2;
  a.slice = slice_of(C);
  const size_t smem = kHead + a.slice * sizeof(Te);
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
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = C > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
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
