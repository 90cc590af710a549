// Kernels over rows of logits: log-probability of one token per row, its entropy and gradients; a clipped policy loss
// and a loss on pairs of answers, each with its gradient with respect to the logits.
//
// With z = logits / tau, M the row's largest logit, k = log2(e) / tau and d_j = (logit_j - M) k (so p_j = 2^d_j / S):
//   S = sum 2^d_j,  T = sum 2^d_j d_j;   lse = M / tau + ln S,   log p_j = ln2 (d_j - log2 S),
//   H = -sum p ln p = ln2 (log2 S - T / S),
//   d(g log p_y + h H) / d logit_j = (g 1[j = y] - p_j (g + h H + h ln p_j)) / tau.
// All three sums are held as (M, S, T) triples that combine associatively, so a row is read once, in any split.
// M may be any reference in their place; where an exponent is formed by one fma, x k - fl(M k), the rounding of M k is
// corrected in the sums, and rows whose M k is large take the difference first.
//
// What bounds these kernels: a 16-bit logit is 2 bytes read (and 2 written), for which the memory takes 87 (174) cycles per
// SM and 1000 logits at the measured copy rate; an exponential for the sums and one for the gradient take 62 cycles each
// of the special-function unit (16 per clock and SM), and the arithmetic around them 5 and 3 instructions per logit in packed
// fp32 (two per instruction), 60 cycles in all at four instructions per clock.  So loads, exponentials and stores have to
// overlap throughout: bulk copies fetch ahead, several blocks share an SM, and one's barriers are another's arithmetic.
//
// Rows whose target is negative are ignored: their logits are not read (they may hold anything) and their gradient is
// zero.  A target beyond the vocabulary gives NaN.
#pragma once
#include "lists.cuh"

namespace tg {

struct TokenArgs {
  const char* z;         // logits
  char* dz;              // gradient, or null
  int64_t ldz, lddz;     // entries between rows
  const long long* y;    // targets
  int V;
  float k, inv_tau;      // log2(e) / tau, 1 / tau
  float k_lo, inv_lo;    // what their rounding to fp32 has left out: of k relative to it, of 1 / tau absolute
};

constexpr float TK_LN2 = 0.6931471805599453f;
// The special-function unit's 2^x comes out low on average: by 5e-8 below x = -2, 4.3e-8 from there to -0.7, 2.2e-8 above
// (measured on one B200, 2^24 exponents in each range; integers are exact).  EX2_LOW: what that makes of the sums of a warp or a
// block; EX2_LOW_SPLIT: where every thread has its own reference, so that most of a sum is near it or exact.
constexpr float TK_EX2_LOW = 4.8e-8f, TK_EX2_LOW_SPLIT = 2e-8f;
constexpr float TK_LOWEST = -3.402823466e38f;

__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float lg2(float x) { float r; asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// ---- granules: the 16 bytes of storage that a thread handles at a time ----
template <int KIND> struct Gran { static constexpr int E = KIND == LS_F32 ? 4 : 8, B = KIND == LS_F32 ? 4 : 2; };
template <int KIND> __device__ __forceinline__ uint32_t neg_inf_word() {
  return KIND == LS_F32 ? 0xff800000u : (KIND == LS_F16 ? 0xfc00fc00u : 0xff80ff80u);
}
// the pair q of a granule's entries (16-bit storage: q = 0..3, fp32: q = 0..1)
template <int KIND>
__device__ __forceinline__ float2 gpair(const uint4& v, int q) {
  if (KIND == LS_F32) return q == 0 ? make_float2(__uint_as_float(v.x), __uint_as_float(v.y)) : make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
  return widen2<KIND>(q == 0 ? v.x : q == 1 ? v.y : q == 2 ? v.z : v.w);
}
template <int KIND>
__device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {     // larger entries of two words; a NaN loses
  if (KIND == LS_F32) return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  if (KIND == LS_F16) { const __half2 r = __hmax2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b)); return *reinterpret_cast<const uint32_t*>(&r); }
  const __nv_bfloat162 r = __hmax2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
template <int KIND>
__device__ __forceinline__ uint32_t max_nan_word(uint32_t a, uint32_t b) {     // the same; a NaN stays (16-bit storage)
  if (KIND == LS_F16) { const __half2 r = __hmax2_nan(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b)); return *reinterpret_cast<const uint32_t*>(&r); }
  const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
template <int KIND>
__device__ __forceinline__ float max_of_word(uint32_t a) {
  if (KIND == LS_F32) return __uint_as_float(a);
  const float2 x = widen2<KIND>(a);
  return fmaxf(x.x, x.y);
}

// A row seen as granules: `mis` entries lie before it in its first granule.
template <int KIND>
struct Row {
  const char* base;      // 16-byte aligned address of the first granule
  int mis, V;
  __device__ __forceinline__ Row(const char* p, int V_) {
    const uint32_t o = (uint32_t)((uintptr_t)p & 15);
    base = p - o; mis = (int)(o / Gran<KIND>::B); V = V_;
  }
  __device__ __forceinline__ int granules() const { return (mis + V + Gran<KIND>::E - 1) / Gran<KIND>::E; }
  __device__ __forceinline__ bool whole(int g) const {          // all of granule g belongs to the row
    return (g > 0 || mis == 0) && (g + 1) * Gran<KIND>::E <= mis + V;
  }
  // an outer granule: entries outside the row read as -inf
  __device__ __noinline__ uint4 partial(int g) const {
    uint32_t w[4];
    for (int q = 0; q < 4; ++q) w[q] = neg_inf_word<KIND>();
    for (int i = 0; i < Gran<KIND>::E; ++i) {
      const int j = g * Gran<KIND>::E + i - mis;
      if (j < 0 || j >= V) continue;
      const char* p = base + ((int64_t)j + mis) * Gran<KIND>::B;
      if (KIND == LS_F32) w[i] = *reinterpret_cast<const uint32_t*>(p);
      else {
        const uint32_t h = *reinterpret_cast<const unsigned short*>(p);
        w[i >> 1] = (i & 1) ? (w[i >> 1] & 0xffffu) | (h << 16) : (w[i >> 1] & 0xffff0000u) | h;
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ uint4 load(int g) const {
    if (whole(g)) return ld_stream(reinterpret_cast<const uint4*>(base) + g);
    return partial(g);
  }
};

// ---- (M, S, T) ----
struct Triple { float m, s, t; };
// A factor of 2^d, d below this, is zero; times sums of up to 2^40 per entry it is still far from the end of the range.
constexpr float TK_FAR_BELOW = -1e4f;
// 2^d for d <= 0 without a mean error: the power of two nearest to it, times the first eight terms of exp(t ln 2), |t| <= 1/2
// (what is left out is below 6e-9).
__device__ __forceinline__ float exp2_even(float d) {
  const float i = rintf(d), t = (d - i) * TK_LN2;
  float p = 1.f / 5040.f;
  p = fmaf(p, t, 1.f / 720.f); p = fmaf(p, t, 1.f / 120.f); p = fmaf(p, t, 1.f / 24.f);
  p = fmaf(p, t, 1.f / 6.f); p = fmaf(p, t, 0.5f); p = fmaf(p, t, 1.f);
  return fmaf(p, t, 1.f) * ex2(i);
}
// Moves a triple to a larger maximum.  A part that has seen nothing but -inf has m = lowest, s = t = 0 and stays so.
// EVEN: where a sum is moved many times, the special-function unit's mean error in each factor would add up (to 5e-8 to 1.1e-7 in
// the log-probabilities of token_forward_kernel; 2e-8 where it is moved a few times).
template <bool EVEN = false>
__device__ __forceinline__ void rebase(Triple& a, float m, float k) {
  const float d = fmaxf((a.m - m) * k, TK_FAR_BELOW);
  const float f = EVEN ? exp2_even(d) : ex2(d);
  a.t = f * fmaf(a.s, d, a.t);
  a.s *= f;
  a.m = m;
}
// adds one logit
__device__ __forceinline__ void add_entry(Triple& a, float x, float k) {
  Triple b; b.m = fmaxf(x, TK_LOWEST); b.s = x == -INFINITY ? 0.f : x - x + 1.f; b.t = 0.f;      // NaN and inf give NaN
  const float m = fmaxf(a.m, b.m);
  rebase(a, m, k); rebase(b, m, k);
  a.s += b.s; a.t += b.t;
}
// adds a batch of granules whose maximum is not above a.m
template <int KIND, int NV>
__device__ __forceinline__ void accumulate(Triple& a, const uint4 (&v)[NV], float k) {
  const uint64_t nm = pk2(-a.m, -a.m), kk = pk2(k, k);
  uint64_t s2 = pk2(0.f, 0.f), t2 = s2;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int q = 0; q < Gran<KIND>::E / 2; ++q) {
      const float2 x = gpair<KIND>(v[i], q);
      const float2 d = upk2(mul2(add2(pk2(x.x, x.y), nm), kk));
      const uint64_t e = pk2(ex2(d.x), ex2(d.y));
      s2 = add2(s2, e);
      t2 = fma2(e, pk2(max_nan(d.x, -200.f), max_nan(d.y, -200.f)), t2);   // 0 * -inf is not wanted
    }
  const float2 s = upk2(s2), t = upk2(t2);
  a.s += s.x + s.y;
  a.t += t.x + t.y;
}
template <int KIND, int NV>
__device__ __forceinline__ float batch_max(const uint4 (&v)[NV]) {
  uint32_t m = v[0].x;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    m = max_word<KIND>(m, v[i].x); m = max_word<KIND>(m, v[i].y);
    m = max_word<KIND>(m, v[i].z); m = max_word<KIND>(m, v[i].w);
  }
  return fmaxf(max_of_word<KIND>(m), TK_LOWEST);      // also for a batch of NaN
}
__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// Combines the triples of the lanes; lanes from `width` on have none (m lowest, s and t 0).
template <bool EVEN = false>
__device__ __forceinline__ void warp_combine(Triple& a, float k, int width = 32) {
  rebase<EVEN>(a, warp_max(a.m), k);
  for (int o = 16; o; o >>= 1) {
    if (o >= width) continue;
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.t += __shfl_xor_sync(0xffffffffu, a.t, o);
  }
}

// ---- cluster of blocks that share a row ----
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_map(const void* smem, uint32_t rank) {
  uint32_t r; asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(smem)), "r"(rank)); return r;
}
__device__ __forceinline__ void cluster_st4(uint32_t addr, float a, float b, float c, float d) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
}

constexpr int TK_MAX_CLUSTER = 8;

// Combines the triples of all threads of the C blocks that share a row; the result is in every thread.  Each warp
// leaves its triple in the shared memory of each block, one barrier (over the cluster) follows, and each warp combines
// all of them, so that no second exchange is needed.  The caller has passed the cluster's start (cluster_wait after
// cluster_arrive_relaxed) where C > 1; nobody touches another block's memory after the barrier.
template <int THREADS>
__device__ __forceinline__ void row_combine(Triple& a, float k, int C, float4* sh) {
  constexpr int W = THREADS / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  warp_combine<true>(a, k);
  if (C == 1) {
    if (W == 1) return;
    if (lane == 0) sh[warp] = make_float4(a.m, a.s, a.t, 0.f);
    __syncthreads();
  } else {
    const int slot = (int)cluster_rank() * W + warp;
    if (lane < C) cluster_st4(cluster_map(sh + slot, (uint32_t)lane), a.m, a.s, a.t, 0.f);
    __syncwarp();
    cluster_arrive();
    cluster_wait();
  }
  a.m = TK_LOWEST; a.s = a.t = 0.f;
  for (int i = lane; i < C * W; i += 32) {
    const float4 o = sh[i];
    Triple b; b.m = o.x; b.s = o.y; b.t = o.z;
    const float m = fmaxf(a.m, b.m);
    rebase<true>(a, m, k); rebase<true>(b, m, k);
    a.s += b.s; a.t += b.t;
  }
  warp_combine<true>(a, k);
}

// What the sums say about one row.  The exponents were formed with k rounded to fp32, d (1 + k_lo) being the true ones: S is
// off by k_lo ln2 T to first order, the same way in every row, which the sums over an answer's tokens would show.
// The same holds for the special-function unit's mean error, `low`, of all but the largest entry, whose 2^0 is exact.  (Where M is
// a reference below the maximum, that entry's is not; the correction is then off by less than its own size, 5e-8.)
// ln S is formed as hi + lo, hi a multiple of a short ln 2, and log p with the part that its rounding to fp32 leaves out: the
// roundings of two numbers near 10 are more than half of the error of log p, and sums over an answer's tokens use both parts.
struct RowStat { float M, ls2, lse, logp, logp_lo, H; };
__device__ __forceinline__ RowStat row_stat(const Triple& a, float zy, const TokenArgs& p, float low = TK_EX2_LOW) {
  RowStat r;
  r.M = a.m;
  const float inv_s = 1.f / a.s, mean = TK_LN2 * (a.t * inv_s), drift = fmaf(p.k_lo, mean, low * (1.f - inv_s));
  float hi = 0.f, lo;
  if (a.s > 1e-30f && a.s < 1e30f) {
    uint32_t bits = __float_as_uint(a.s);
    float e = (float)((int)(bits >> 23) - 127), m = __uint_as_float((bits & 0x007fffffu) | 0x3f800000u);
    if (m > 1.5f) { m *= 0.5f; e += 1.f; }
    hi = e * 0.693115234375f;                                      // 2839 / 4096: exact
    lo = fmaf(e, 3.194618495e-05f, drift + logf(m));                // ln 2 - 2839 / 4096
  } else lo = logf(a.s);
  const float ls = hi + lo;
  r.ls2 = ls * 1.4426950408889634f;
  r.lse = fmaf(a.m, p.inv_tau, fmaf(a.m, p.inv_lo, ls));
  r.H = ls - mean;
  const float d = zy - a.m, q = d * p.inv_tau;
  r.logp_lo = 0.f;
  if (fabsf(q) < 1e30f) {
    const float db = d - zy, d_lo = (zy - (d - db)) + (-a.m - db);                            // zy - M = d + d_lo
    const float q_lo = fmaf(d, p.inv_tau, -q) + fmaf(d, p.inv_lo, d_lo * p.inv_tau);          // times 1 / tau = q + q_lo
    const float t = q - hi, tb = t - q, t_lo = (q - (t - tb)) + (-hi - tb);
    const float rest = (q_lo - lo) + t_lo;
    r.logp = t + rest;
    r.logp_lo = rest - (r.logp - t);
    if (r.logp_lo != r.logp_lo) r.logp_lo = 0.f;
  } else r.logp = q - ls;
  return r;
}
template <int KIND>
__device__ __forceinline__ float target_logit(const TokenArgs& p, int64_t row, long long y) {
  if (y >= p.V) return __int_as_float(0x7fc00000);      // NaN: reported, not read
  return ld_real<KIND>(p.z + (row * p.ldz + y) * Gran<KIND>::B);
}

// ---- gradient ----
// p_j (c0 + c1 L_j) with L_j = log2 p_j: c0 = -(g + h H) / tau, c1 = -h ln2 / tau, all times the loss scale.
struct GradCoef { float M, k, ls2, c0, c1; };
template <int KIND, bool ENT>
__device__ __forceinline__ uint4 grad_granule(const uint4& v, const GradCoef& gc) {
  const uint64_t nm = pk2(-gc.M, -gc.M), kk = pk2(gc.k, gc.k), nl = pk2(-gc.ls2, -gc.ls2), c0 = pk2(gc.c0, gc.c0), c1 = pk2(gc.c1, gc.c1);
  uint32_t w[4];
#pragma unroll
  for (int q = 0; q < Gran<KIND>::E / 2; ++q) {
    const float2 x = gpair<KIND>(v, q);
    const uint64_t L = fma2(add2(pk2(x.x, x.y), nm), kk, nl);
    const float2 l = upk2(L);
    uint64_t c = c0;
    if (ENT) c = fma2(pk2(max_nan(l.x, -200.f), max_nan(l.y, -200.f)), c1, c0);
    const float2 d = upk2(mul2(pk2(ex2(l.x), ex2(l.y)), c));
    if (KIND == LS_F32) { w[2 * q] = __float_as_uint(d.x); w[2 * q + 1] = __float_as_uint(d.y); }
    else w[q] = narrow2<KIND>(d.x, d.y);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int KIND, bool ENT>
__device__ __forceinline__ float grad_target(float zy, const GradCoef& gc, float g) {
  const float l = fmaf(zy - gc.M, gc.k, -gc.ls2);
  const float c = ENT ? fmaf(max_nan(l, -200.f), gc.c1, gc.c0) : gc.c0;
  return gc.c0 == 0.f && (!ENT || gc.c1 == 0.f) ? g : fmaf(ex2(l), c, g);      // (NaN times zero is not wanted)
}
// entry i of a granule
template <int KIND>
__device__ __forceinline__ void st_entry(char* p, const uint4& v, int i) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if (KIND == LS_F32) *reinterpret_cast<uint32_t*>(p) = w[i];
  else *reinterpret_cast<unsigned short*>(p) = (unsigned short)(w[i >> 1] >> (16 * (i & 1)));
}
// Stores granule g of the row's gradient.  `same`: gradient row and logits row lie alike relative to 16 bytes.
template <int KIND>
__device__ __noinline__ void store_entries(char* drow, int mis, int V, int g, uint4 v) {
#pragma unroll
  for (int i = 0; i < Gran<KIND>::E; ++i) {
    const int j = g * Gran<KIND>::E + i - mis;
    if (j >= 0 && j < V) st_entry<KIND>(drow + (int64_t)j * Gran<KIND>::B, v, i);
  }
}
template <int KIND>
__device__ __forceinline__ void store_granule(const Row<KIND>& r, char* drow, bool same, int g, const uint4& v) {
  if (same && r.whole(g)) st_stream(reinterpret_cast<uint4*>(drow - r.mis * Gran<KIND>::B) + g, v);
  else store_entries<KIND>(drow, r.mis, r.V, g, v);
}
// A gradient row of zeros, by `threads` threads.
template <int KIND>
__device__ __forceinline__ void zero_row(char* drow, int V, int tid, int threads) {
  constexpr int E = Gran<KIND>::E;
  const Row<KIND> d(drow, V);
  const int lo = d.mis ? 1 : 0, hi = (d.mis + V) / E;      // the whole granules
  uint4* at = reinterpret_cast<uint4*>(drow - d.mis * Gran<KIND>::B) + lo + tid;
  for (int g = lo + tid; g < hi; g += threads, at += threads) st_stream(at, make_uint4(0, 0, 0, 0));
  if (tid == 0 && lo) store_entries<KIND>(drow, d.mis, V, 0, make_uint4(0, 0, 0, 0));
  if (tid == 1 && hi >= lo && (d.mis + V) % E) store_entries<KIND>(drow, d.mis, V, hi, make_uint4(0, 0, 0, 0));
}
template <int KIND>
__device__ __forceinline__ bool same_alignment(const Row<KIND>& r, const char* drow) {
  return (int)((uintptr_t)drow & 15) == r.mis * Gran<KIND>::B;
}

// ---- clipped policy loss of one token ----
struct PolicyArgs {
  const float* old_logp; const float* ref_logp; const float* adv; const float* weight;   // ref_logp may be null
  float low, high;           // bounds of the ratio
  float kl_coef, ent_coef, grad_scale;
  float4* terms;                           // out: weighted policy, KL, entropy and clipping terms of each row
};
struct PolicyToken { float g, h; float4 terms; };
// r = exp(logp - old); the loss -min(r A, clip(r) A) has gradient -r A where the unclipped term is the smaller one or
// they are equal, and none elsewhere; kl = exp(u) - u - 1 with u = ref - logp has gradient 1 - exp(u).
// A weight of zero is a mask: whatever stands beside such a row (infinities, NaN, a ratio that overflows) does not count.
__device__ __forceinline__ PolicyToken policy_token(float logp, float H, float old, float ref, bool has_ref, float A, float w, const PolicyArgs& q) {
  PolicyToken o;
  if (w == 0.f) {
    o.g = o.h = 0.f; o.terms = make_float4(0.f, 0.f, 0.f, 0.f);
    return o;
  }
  const float r = expf(logp - old);
  const float free = A != 0.f ? r * A : 0.f;      // (0 also where the ratio overflows)
  const float bound = fminf(fmaxf(r, q.low), q.high) * A;
  const bool cut = free > bound;
  const float pg = cut ? -bound : -free;
  float kl = 0.f, dkl = 0.f;
  if (has_ref) {
    const float u = ref - logp, em = expm1f(u);
    kl = em < __int_as_float(0x7f800000) ? em - u : em;      // infinite, not NaN, where the policy forbids what the reference allows
    dkl = q.kl_coef != 0.f ? q.kl_coef * -em : 0.f;          // (an infinite KL that is only looked at)
  }
  o.g = w * ((cut ? 0.f : -free) + dkl);
  o.h = -q.ent_coef * w;
  o.terms = make_float4(w * pg, w * kl, w * H, cut ? w : 0.f);
  return o;
}

// ---------------------------------------------------------------------------------------------------------------
// Policy loss, forward and backward in one pass over device memory: a block works on one row at a time, reads it once for
// the sums and once more, from shared memory, for the gradient.
//
// The row's whole granules come in chunks of 128 granules per arithmetic warp, by bulk copies into a ring of N places that
// one further warp keeps full.  Chunks that stay for the second reading are released after it; where a row has more chunks
// than the ring has places, the ones too many go through it first, and again (from L2) at the end:
//   asked for:  e_1 .. e_x  r_1 .. r_n  e_1 .. e_x      released in the same order, so that the ring is a queue:
//   sums of     e_1 .. e_x  r_1 .. r_n
//   gradient of             r_1 .. r_n  e_1 .. e_x
// While the gradient frees places the next row's chunks arrive in them.  The up to E - 1 entries before the first and after
// the last whole granule are taken one by one by the first warp.
//
// Why a block and not a cluster per row: with the row in the registers of eight blocks the exchange of the sums (3,000 to
// 5,000 cycles between the last logit's arrival and the first gradient, most of it latency) was paid for every 32 KB
// instead of for every row; 8192 x 131072 bf16 logits took 0.95 ms so, and 1.2 ms with the rows fetched ahead.
constexpr int RW_MAX_WARPS = 16, RW_MAX_PLACES = 16, RW_JOBS = 4, RW_NV = 4;      // RW_NV: granules of a chunk per thread
struct RowGeom {
  int W, N;              // arithmetic warps, places of the ring
  int unit;              // rows that a block takes at a time
  int K, last;           // chunks of the longest row, granules before the last of them; others have at most one chunk less
  float reach, lowest;   // 200 / k; lowest value that the clamp may take in the storage type
  float slack;           // 40 / k
  int copies;            // of one row after which the fetching warp stops (for tests of what happens then), or 2^31 - 1
};

// A bounded wait that asks the hardware to keep the warp asleep for up to 20 us at a time: the other warps need the issue
// slots that frequent polling takes (more than half of all instructions on rows of 8000 logits).
// The bound, about half a second (a poll takes 4 us), is a constant: as a parameter it costs the policy loss 1 to 4 % (8192 x 131072
// bf16: 689 to 710 us instead of 683).
__device__ __forceinline__ bool mbar_wait_asleep(uint64_t* bar, uint32_t parity) {
  for (uint32_t i = 0; i < (1u << 17); ++i) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity), "r"(20000u) : "memory");
    if (ok) return true;
  }
  return false;
}

// Work distribution by the hardware's queue of blocks: a running block takes over one that has not been started.  The
// answer is 16 bytes in shared memory, counted on an mbarrier; once it was "none left", no further block may be asked for.
__device__ __forceinline__ void next_block_ask(uint4* answer, uint64_t* bar) {
  fence_async_smem();
  mbar_expect_tx(bar, 16);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(answer)), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ int next_block_get(const uint4* answer) {      // its index, or -1
  const ulonglong2 a = *reinterpret_cast<const ulonglong2*>(answer);
  uint32_t some, x;
  asm volatile(
      "{\n\t.reg .b128 r;\n\t.reg .pred p;\n\t"
      "mov.b128 r, {%2, %3};\n\t"
      "mov.b32 %1, 0;\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(some), "=r"(x) : "l"(a.x), "l"(a.y) : "memory");
  return some ? (int)x : -1;
}

__device__ __forceinline__ void bar_sync_n(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// Running sums of a warp relative to a reference that all its lanes share and that need not be the maximum: it is moved
// when a logit exceeds it by more than 2^40 (so the sums neither overflow nor lose anything).
struct WarpSums { float base, thr, nm, delta; uint32_t clamp; bool fast; uint64_t s2, t2; };
template <int KIND>
__device__ __forceinline__ void move_base(WarpSums& a, float top, const RowGeom& geo, float k) {
  top = warp_max(top);
  const float d = fmaxf(fmaf(a.base - top, k, -a.delta), TK_FAR_BELOW), f = ex2(d);
  const float2 s = upk2(a.s2), t = upk2(a.t2);
  a.s2 = pk2(s.x * f, s.y * f);
  a.t2 = pk2(f * fmaf(s.x, d, t.x), f * fmaf(s.y, d, t.y));
  a.base = top; a.thr = top + geo.slack;
  // One fma per exponent, d = x k - fl(base k), and -inf clamped before it is widened, where the reference lies within 2^12 of
  // zero in units of an exponent (2,839 at a temperature of one); else the difference first, for any temperature and any
  // logits.  Within the bound 2^delta is 1 +- 2^-13, and the clamp, which is rounded to the storage type, stays below
  // 2^-180 of the reference: a step of bfloat16 at |low| <= |top| + 200 / k is at most 34 / k.
  const float low = top - geo.reach;      // 2^-200 of the reference
  a.fast = fabsf(top * k) < 4096.f && low > geo.lowest;
  a.nm = a.fast ? -(top * k) : -top;
  a.delta = a.fast ? fmaf(top, k, a.nm) : 0.f;      // 2^(x k - fl(base k)) is 2^delta too large
  a.clamp = narrow2<KIND == LS_F32 ? LS_BF16 : KIND>(low, low);
}
template <int KIND, bool FAST>
__device__ __forceinline__ void add_granule(const uint4& v, uint32_t clamp, uint64_t nm, uint64_t kk, uint64_t& s2, uint64_t& t2) {
#pragma unroll
  for (int j = 0; j < Gran<KIND>::E / 2; ++j) {
    float2 x;
    if (KIND == LS_F32 || !FAST) x = gpair<KIND>(v, j);
    else x = widen2<KIND>(max_nan_word<KIND>(j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w, clamp));
    uint64_t d2 = FAST ? fma2(pk2(x.x, x.y), kk, nm) : mul2(add2(pk2(x.x, x.y), nm), kk);
    const float2 d = upk2(d2);
    const uint64_t e = pk2(ex2(d.x), ex2(d.y));
    s2 = add2(s2, e);
    if (KIND == LS_F32 || !FAST) d2 = pk2(max_nan(d.x, -200.f), max_nan(d.y, -200.f));      // 0 * -inf is not wanted
    t2 = fma2(e, d2, t2);
  }
}
// APART: the chunk's sums first, then to the others.  A lane of the forward kernel's blocks of four warps adds up to some thousand
// terms of a long row; one by one, small ones beside a large one would be lost (a mean error of 1e-7 in the log-probabilities of 131072
// logits).  With sixteen warps there are a quarter as many (3e-8 at most), and the same costs the policy loss 1.7 %.
template <int KIND, bool APART>
__device__ __forceinline__ void add_chunk(WarpSums& a, const uint4 (&v)[RW_NV], const RowGeom& geo, float k) {
  const float top = batch_max<KIND, RW_NV>(v);
  if (__any_sync(0xffffffffu, top > a.thr)) move_base<KIND>(a, top, geo, k);
  const uint64_t nm = pk2(a.nm, a.nm), kk = pk2(k, k);
  uint64_t s2 = APART ? pk2(0.f, 0.f) : a.s2, t2 = APART ? pk2(0.f, 0.f) : a.t2;
  if (a.fast) {
#pragma unroll
    for (int u = 0; u < RW_NV; ++u) add_granule<KIND, true>(v[u], a.clamp, nm, kk, s2, t2);
  } else {
#pragma unroll
    for (int u = 0; u < RW_NV; ++u) add_granule<KIND, false>(v[u], a.clamp, nm, kk, s2, t2);
  }
  a.s2 = APART ? add2(a.s2, s2) : s2;
  a.t2 = APART ? add2(a.t2, t2) : t2;
}

// What the row's sums give the gradient.  owner: the thread that writes the target's granule, or -1.
struct RowGrad { float M, nb, ls2, c0, c1, e0, e1, target, zy; int owner, fast; };
// c0, c1 are those of the loop over the granules, e0, e1 those of single entries (which take the difference first).
// 16-bit logits, |M k + log2 S| below 2^20: an exponent is one fma, L = x k + nb, nb being -(M k + log2 S) rounded.  The rounding,
// up to 2^-5 at that bound, is taken back here: p = 2^(L + off) = 2^off 2^L, in both coefficients.  fp32 logits, whose results
// are not rounded to fewer bits, rows further out and rows without a distribution take the difference first.
template <int KIND, bool ENT>
__device__ __forceinline__ void gradient_coef(RowGrad& h, float M, float ls2, float c0, float c1, float k) {
  h.M = M; h.ls2 = ls2; h.c0 = c0; h.c1 = c1;
  h.nb = fmaf(-M, k, -ls2);
  h.fast = KIND != LS_F32 && fabsf(h.nb) < 1048576.f;
  if (!h.fast) return;
  const float off = fmaf(-M, k, -h.nb) - ls2, f = ex2(off);
  if (ENT) h.c0 = fmaf(c1, off, c0);
  h.c0 *= f; h.c1 *= f;
}
// Coefficients of zero (a weight of zero, say) are to give zero whatever the logits are, so NaN too: such rows never are fast.
template <int KIND, bool ENT, bool FAST>
__device__ __forceinline__ uint4 row_gradient(const uint4& v, const RowGrad& h, float k) {
  const uint64_t kk = pk2(k, k), c0 = pk2(h.c0, h.c0), c1 = pk2(h.c1, h.c1);
  const bool none = !FAST && h.c0 == 0.f && (!ENT || h.c1 == 0.f);
  uint32_t w[4];
#pragma unroll
  for (int q = 0; q < Gran<KIND>::E / 2; ++q) {
    const float2 x = gpair<KIND>(v, q);
    const uint64_t x2 = pk2(x.x, x.y);
    const float2 l = upk2(FAST ? fma2(x2, kk, pk2(h.nb, h.nb)) : fma2(add2(x2, pk2(-h.M, -h.M)), kk, pk2(-h.ls2, -h.ls2)));
    uint64_t c = c0;
    if (ENT) c = fma2(pk2(max_nan(l.x, -200.f), max_nan(l.y, -200.f)), c1, c0);
    const float2 d = upk2(mul2(pk2(ex2(l.x), ex2(l.y)), c));
    if (KIND == LS_F32) { w[2 * q] = __float_as_uint(d.x); w[2 * q + 1] = __float_as_uint(d.y); }
    else w[q] = narrow2<KIND>(d.x, d.y);
  }
  if (none) { w[0] = w[1] = w[2] = w[3] = 0; }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Every wait on an mbarrier is bounded.  What happens when one runs out (nothing in normal operation leads there):
// * An arithmetic warp whose wait has run out stops work and goes to the barrier that the others reach next, their next row's or
//   the one at their end, having set `bad` for it.  All read `bad` behind that barrier and leave together, so nobody is left
//   waiting for a warp that is gone.  `bad` alternates between two places, since a warp may still read it behind one barrier when
//   another sets it for the next.
// * The fetching warp stops asking.  All warps meet when they have left their loops; the rows of every unit that the block has
//   taken and not finished then get NaN in all results.  At most seven units can be open: one in work, RW_JOBS handed on, one being
//   fetched, one just taken.
constexpr int RW_OPEN = 8;
struct RowBarriers {
  uint64_t full[RW_MAX_PLACES], empty[RW_MAX_PLACES], jfull[RW_JOBS], jempty[RW_JOBS], nbar;
  alignas(16) uint4 answer;
  longlong2 job[RW_JOBS];     // unit of rows (-1: no more), target of its first row
  int unit[RW_OPEN];          // the units that the block took last, the i-th at i modulo RW_OPEN
  int taken;                  // how many it has taken
  int done;                   // after a failure: how many all warps have finished
  volatile int bad[2], failed;
  __device__ __forceinline__ void init(int N, int W, int lane) {      // by one warp; a barrier of the block follows
    if (lane < N) { mbar_init(&full[lane], 1); mbar_init(&empty[lane], W); }
    if (lane < RW_JOBS) { mbar_init(&jfull[lane], 1); mbar_init(&jempty[lane], W); }
    if (lane == 31) {
      mbar_init(&nbar, 1);
      taken = 0; done = 0x7fffffff; bad[0] = bad[1] = failed = 0;
    }
    fence_mbar_init();
  }
};
static_assert((RW_JOBS & (RW_JOBS - 1)) == 0 && RW_OPEN >= RW_JOBS + 3, "job slots and open units");

// This warp has read a place of the ring.  The fence comes first because nothing else keeps the warp's shared loads, which
// may still be under way, before the asynchronous copy that the arrival lets into the place (without it, a few granules at
// the start of a chunk came out as those of the chunk N later, once in some thousand rows).
__device__ __forceinline__ void release_place(uint64_t* empty, int lane) {
  fence_async_smem();
  __syncwarp();
  if (lane == 0) mbar_arrive(empty);
}

// The fetching warp: takes units of rows, passes them on, and asks for the chunks of their live rows.  STAY: chunks stay
// for a second reading (n of them, see above); else each goes through the ring once.  LAST_FIRST: the units from the end.
// wanted(row): whether a row with a target is read at all.
template <int KIND, bool STAY, bool LAST_FIRST, typename F>
__device__ __forceinline__ void fetch_rows(const TokenArgs& p, int64_t rows, const RowGeom& geo, unsigned char* ring, RowBarriers& rb, int lane, int chunk, F wanted) {
  constexpr int E = Gran<KIND>::E, B = Gran<KIND>::B;
  const int N = geo.N;
  int s = 0, js = 0, taken = 0;
  uint32_t ph = 0, jph = 0, used = 0, nph = 0;
  bool ok = true, lost = false;
  int64_t block = blockIdx.x;
  for (;;) {
    const int64_t unit = LAST_FIRST ? (int64_t)gridDim.x - 1 - block : block;
    if (lane == 0) rb.unit[taken % RW_OPEN] = (int)unit;
    ++taken;
    if (!ok) break;
    if (lane == 0) next_block_ask(&rb.answer, &rb.nbar);
    const int64_t r0 = unit * geo.unit, mine = r0 + lane;
    const long long ym = lane < geo.unit && mine < rows ? p.y[mine] : -1;
    uint32_t live = __ballot_sync(0xffffffffu, ym >= 0 && wanted(mine));
    if (lane == 0) {
      ok = geo.copies > 0 && mbar_wait_asleep(&rb.jempty[js], jph ^ 1);
      if (ok) { rb.job[js] = make_longlong2(unit, ym); mbar_arrive(&rb.jfull[js]); }
      for (; live && ok; live &= live - 1) {
        const Row<KIND> r(p.z + (r0 + __ffs(live) - 1) * p.ldz * B, p.V);
        const int wa = r.mis ? 1 : 0, nw = max(0, (r.mis + p.V) / E - wa), K = geo.K - (nw <= geo.last), n = !STAY ? 0 : K <= N ? K : N - 2;
        const int all = STAY ? 2 * K - n : K, most = min(all, geo.copies);
        for (int j = 0; j < most && ok; ++j) {
          const int x = K - n, id = j < x ? n + j : (j < K ? j - x : n + j - K), at = id * chunk, len = min(chunk, nw - at);
          ok = mbar_wait_asleep(&rb.empty[s], ph ^ 1);
          if (!ok) break;
          mbar_expect_tx(&rb.full[s], (uint32_t)len * 16);
          bulk_g2s(ring + (size_t)s * chunk * 16, r.base + (size_t)(wa + at) * 16, (uint32_t)len * 16, &rb.full[s]);
          used |= 1u << s;
          if (++s == N) { s = 0; ph ^= 1; }
        }
        ok = ok && most == all;
      }
    }
    if (++js == RW_JOBS) { js = 0; jph ^= 1; }
    // (the answer is taken, after a failure too, before the block may end)
    const bool got = __all_sync(0xffffffffu, mbar_wait_asleep(&rb.nbar, nph));
    nph ^= 1;
    const int next = got ? next_block_get(&rb.answer) : -1;
    __syncwarp();
    ok = __shfl_sync(0xffffffffu, (int)(ok && got), 0) != 0;
    lost = !got;
    if (next < 0) break;
    block = next;
  }
  if (lane == 0) {
    if (ok) {
      ok = mbar_wait_asleep(&rb.jempty[js], jph ^ 1);
      if (ok) { rb.job[js] = make_longlong2(-1, 0); mbar_arrive(&rb.jfull[js]); }
    }
    // no copy is left in flight when the block ends: place i was last filled in phase ph (i < s) or the one before
    for (int i = 0; i < N; ++i)
      if (used >> i & 1) (void)mbar_wait_asleep(&rb.full[i], i < s ? ph : ph ^ 1);
    rb.taken = taken;
    if (lost) atomicMin(&rb.done, 0);      // a unit that this block may have been given and does not know of: NaN where it can
    if (!ok) rb.failed = 1;
  }
  __syncwarp();
}

struct ForwardArgs {
  float* logp; float* lse; float* entropy;      // out, may be null
  float* logp_lo;                               // out, may be null: what the rounding of logp has left out
  float2* stat;                                 // out, may be null: (M, log2 S) for a later gradient pass
  float* g;                                     // zeroed, may be null: gradient of rows that no later kernel gives one
  unsigned* ticket;                             // zeroed with it
};
// MODE: RW_FORWARD log-probabilities only (every chunk goes through the ring once, and the last warp's work on a row
// overlaps with the others' on the next), RW_POLICY the policy loss with its gradient, RW_ENTROPY with an entropy bonus.
enum { RW_FORWARD = 0, RW_POLICY = 1, RW_ENTROPY = 2 };
__device__ __forceinline__ void store_stat(const ForwardArgs& f, int64_t row, const RowStat& st) {
  if (f.logp) f.logp[row] = st.logp;
  if (f.lse) f.lse[row] = st.lse;
  if (f.logp_lo) f.logp_lo[row] = st.logp_lo;
  if (f.entropy) f.entropy[row] = st.H;
  if (f.stat) f.stat[row] = make_float2(st.M, st.ls2);
  if (f.g) f.g[row] = 0.f;
  if (f.ticket && row == 0) *f.ticket = 0;
}
// The end of a block: all its warps, the fetching one too, once they have left their loops.  After a failure the rows of the units
// that were not finished get NaN; `write(row, NaN)` sets what a row has besides its gradient.
template <int KIND, int W, typename F>
__device__ __noinline__ void row_block_failed(const RowBarriers& rb, const RowGeom& geo, const TokenArgs& p, int64_t rows, bool back, F write) {
  const float nan = __int_as_float(0x7fc00000);
  for (int i = max(rb.done, max(0, rb.taken - RW_OPEN)); i < rb.taken; ++i) {
    const int64_t r0 = (int64_t)rb.unit[i % RW_OPEN] * geo.unit, r1 = min((long long)(r0 + geo.unit), (long long)rows);
    for (int64_t row = r0; row < r1; ++row) {
      if (threadIdx.x == 0) write(row, nan);
      if (back)
        for (int j = (int)threadIdx.x; j < p.V; j += 32 * (W + 1)) st_real<KIND>(p.dz + (row * p.lddz + j) * Gran<KIND>::B, nan);
    }
  }
}
template <int KIND, int W, typename F>
__device__ __forceinline__ void row_block_end(const RowBarriers& rb, const RowGeom& geo, const TokenArgs& p, int64_t rows, bool back, F write) {
  __syncwarp();
  bar_sync_n(2, 32 * (W + 1));
  if (rb.failed) row_block_failed<KIND, W>(rb, geo, p, rows, back, write);
}
// 96 registers: 80 leave the scheduler too little to interleave (0.73 instead of 0.68 ms at 8192 x 131072 bf16), 128 too few
// warps (0.71 ms).  8192 x 131072 bf16 logits with gradient: 0.68 ms, 5.9 TB/s, after a cold start; 0.74 ms at the clocks that a
// second of it settles at, where the arithmetic weighs more.  Log-probabilities of 16384 x 32000: 0.174 ms, 6.0 TB/s.
template <int KIND, int MODE, int W>
__global__ void __maxnreg__(MODE == RW_FORWARD ? 64 : 96) token_row_kernel(const __grid_constant__ TokenArgs p, const __grid_constant__ PolicyArgs q, const __grid_constant__ ForwardArgs f,
                                                  int64_t rows, const __grid_constant__ RowGeom geo) {
  constexpr bool BACK = MODE != RW_FORWARD, ENT = MODE == RW_ENTROPY;
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ float4 sums[2][RW_MAX_WARPS];
  __shared__ __align__(16) RowGrad handed;
  __shared__ RowBarriers rb;
  constexpr int E = Gran<KIND>::E, B = Gran<KIND>::B;
  constexpr int threads = 32 * W, chunk = RW_NV * threads;
  const int N = geo.N, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == W) rb.init(N, W, lane);
  __syncthreads();
  griddep_wait();
  griddep_launch_dependents();
  const auto fail_row = [&](int64_t at, float nan) {
    RowStat none; none.logp = none.logp_lo = none.lse = none.H = none.M = none.ls2 = nan;
    store_stat(f, at, none);
    if (BACK) q.terms[at] = make_float4(nan, nan, nan, nan);
  };
  if (warp == W) {
    fetch_rows<KIND, BACK, false>(p, rows, geo, ring, rb, lane, chunk, [](int64_t) { return true; });
    row_block_end<KIND, W>(rb, geo, p, rows, BACK, fail_row);
    return;
  }
  int s = 0, jobs = 0;                // jobs: asked for so far, all but the last of them finished
  uint32_t ph = 0;
  bool ok = true, left = false;       // left: behind the barrier that all leave from

  // ---- the arithmetic warps ----
  const uint32_t ni = neg_inf_word<KIND>();
  const uint4* const places = reinterpret_cast<const uint4*>(ring);
  const int64_t zstep = p.ldz * B, dstep = p.lddz * B;
  const char* zrow = p.z;
  char* drow = p.dz;
  int64_t row = 0, row_end = 0;
  long long y_next = -1;
  int side = 0;      // of the double-buffered sums
  for (;; ++row, zrow += zstep, drow += dstep) {
    if (row == row_end) {      // the next unit of rows
      const int js = jobs % RW_JOBS;
      ok = __all_sync(0xffffffffu, mbar_wait_asleep(&rb.jfull[js], (uint32_t)(jobs / RW_JOBS) & 1));
      ++jobs;
      if (!ok) break;
      const longlong2 jb = rb.job[js];
      __syncwarp();
      if (lane == 0) mbar_arrive(&rb.jempty[js]);
      if (jb.x < 0) break;
      row = jb.x * geo.unit; row_end = min((long long)(row + geo.unit), (long long)rows);
      y_next = jb.y;
      zrow = p.z + row * zstep; drow = p.dz + row * dstep;
    }
    const long long y = y_next;
    if (row + 1 < row_end) y_next = p.y[row + 1];
    const Row<KIND> r(zrow, p.V);
    const bool same = same_alignment(r, drow);
    const int wa = r.mis ? 1 : 0, wb = (r.mis + p.V) / E, nw = max(0, wb - wa), K = geo.K - (nw <= geo.last), n = !BACK ? 0 : K <= N ? K : N - 2, x = K - n;
    const int tail = nw - (K - 1) * chunk;      // granules of the last chunk
    if (y < 0) {
      if (BACK) zero_row<KIND>(drow, p.V, tid, threads);
      if (tid == 0) {
        RowStat none; none.logp = none.logp_lo = none.lse = none.H = none.M = none.ls2 = 0.f;
        store_stat(f, row, none);
        if (BACK) q.terms[row] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      continue;
    }
    // the entries outside the whole granules: one per lane of the first warp at most
    int edge = -1;
    float xe = 0.f;
    if (warp == 0) {
      const int h = min(p.V, wa * E - r.mis * wa), t0 = max(h, wb * E - r.mis);
      if (lane < h) edge = lane;
      else if (lane >= 16 && t0 + lane - 16 < p.V) edge = t0 + lane - 16;
      if (edge >= 0) xe = ld_real<KIND>(r.base + (int64_t)(r.mis + edge) * B);
    }
    float zy = 0.f, old = 0.f, adv = 0.f, wt = 0.f, ref = 0.f;
    if (warp == W - 1) {
      zy = target_logit<KIND>(p, row, y);
      if (BACK) {
        old = q.old_logp[row]; adv = q.adv[row]; wt = q.weight[row];
        if (q.ref_logp) ref = q.ref_logp[row];
      }
    }
    // ---- sums ----
    WarpSums a;
    a.base = a.thr = TK_LOWEST; a.nm = -TK_LOWEST; a.delta = 0.f; a.clamp = ni; a.fast = false; a.s2 = a.t2 = pk2(0.f, 0.f);
    int rs = s;
    for (int j = 0; j < K; ++j) {
      ok = __all_sync(0xffffffffu, mbar_wait_asleep(&rb.full[s], ph));
      if (!ok) break;
      if (j == x) rs = s;
      const bool end = j == (x > 0 ? x : K) - 1;      // the row's last chunk
      const uint4* place = places + s * chunk + tid;
      uint4 v[RW_NV];
      if (!end || tail == chunk) {
#pragma unroll
        for (int u = 0; u < RW_NV; ++u) v[u] = place[u * threads];
      } else {
#pragma unroll
        for (int u = 0; u < RW_NV; ++u) {
          v[u] = make_uint4(ni, ni, ni, ni);
          if (tid + u * threads < tail) v[u] = place[u * threads];
        }
      }
      if (j < x) {
        release_place(&rb.empty[s], lane);
      }
      if (++s == N) { s = 0; ph ^= 1; }
      add_chunk<KIND, !BACK>(a, v, geo, p.k);
    }
    Triple c;
    {
      const float2 s2 = upk2(a.s2), t2 = upk2(a.t2);
      c.m = a.base; c.s = s2.x + s2.y; c.t = t2.x + t2.y;
      const float f = ex2(-a.delta);
      c.t = f * fmaf(c.s, -a.delta, c.t); c.s *= f;
      if (edge >= 0) add_entry(c, xe, p.k);
      warp_combine(c, p.k);
    }
    side ^= 1;
    if (lane == 0) {
      sums[side][warp] = make_float4(c.m, c.s, c.t, 0.f);
      if (!ok) rb.bad[side] = 1;
    }
    bar_sync_n(1, threads);
    const bool stop = rb.bad[side] != 0;
    if (warp == W - 1) {
      c.m = TK_LOWEST; c.s = c.t = 0.f;
      if (lane < W) { const float4 o = sums[side][lane]; c.m = o.x; c.s = o.y; c.t = o.z; }
      warp_combine(c, p.k, W);      // (lane 0 uses the result)
      const RowStat st = row_stat(c, zy, p);
      if (lane == 0) store_stat(f, row, st);
      if (BACK) {
      const PolicyToken o = policy_token(st.logp, st.H, old, ref, q.ref_logp != nullptr, adv, wt, q);
      if (lane == 0) {
        const float sc = q.grad_scale * p.inv_tau;
        RowGrad h;
        const float c0 = ENT && o.h != 0.f ? -fmaf(o.h, st.H, o.g) * sc : -o.g * sc, c1 = -o.h * TK_LN2 * sc;
        gradient_coef<KIND, ENT>(h, st.M, st.ls2, c0, c1, p.k);
        h.e0 = c0; h.e1 = c1;
        h.target = o.g * sc; h.zy = zy;
        // the thread that writes the target's granule (an edge entry: the lane that has it)
        const int l = y < p.V ? (r.mis + (int)y) / E - wa : -1;
        h.owner = l >= 0 && l < nw ? l % threads : -1;
        handed = h;
        q.terms[row] = o.terms;
      }
      __syncwarp();
      }
    }
    if (!BACK) {
      // (the next row's sums go to the other side, and nobody passes its barrier before the last warp has read this one's)
      if (stop) { ok = false; left = true; break; }
      continue;
    }
    bar_sync_n(1, threads);
    if (stop) { ok = false; left = true; break; }
    // ---- gradient ----
    const RowGrad h = handed;
    const bool fast = KIND != LS_F32 && h.fast;
    if (edge >= 0) {
      GradCoef gc; gc.M = h.M; gc.k = p.k; gc.ls2 = h.ls2; gc.c0 = h.e0; gc.c1 = h.e1;
      st_real<KIND>(drow + (int64_t)edge * B, grad_target<KIND, ENT>(xe, gc, edge == y ? h.target : 0.f));
    }
    uint4* dst = reinterpret_cast<uint4*>(drow - r.mis * B) + wa + tid;
    int at = rs;
    for (int j = 0; j < K; ++j, dst += chunk) {
      if (j >= n) {
        ok = __all_sync(0xffffffffu, mbar_wait_asleep(&rb.full[s], ph));
        if (!ok) break;
        at = s;
        if (++s == N) { s = 0; ph ^= 1; }
      }
      const uint4* place = places + at * chunk + tid;
      uint4 v[RW_NV];
      if (same && (j < K - 1 || tail == chunk)) {
#pragma unroll
        for (int u = 0; u < RW_NV; ++u) v[u] = place[u * threads];
        release_place(&rb.empty[at], lane);
#pragma unroll
        for (int u = 0; u < RW_NV; ++u)
          st_stream(dst + u * threads, fast ? row_gradient<KIND, ENT, true>(v[u], h, p.k) : row_gradient<KIND, ENT, false>(v[u], h, p.k));
      } else {
        const int len = j < K - 1 ? chunk : tail, g0 = wa + j * chunk;
#pragma unroll
        for (int u = 0; u < RW_NV; ++u)
          if (tid + u * threads < len) v[u] = place[u * threads];
        release_place(&rb.empty[at], lane);
#pragma unroll
        for (int u = 0; u < RW_NV; ++u)
          if (tid + u * threads < len) store_granule<KIND>(r, drow, same, g0 + tid + u * threads, fast ? row_gradient<KIND, ENT, true>(v[u], h, p.k) : row_gradient<KIND, ENT, false>(v[u], h, p.k));
      }
      if (++at == N) at = 0;
    }
    if (!ok) break;
    // the target's entry once more, by the thread that wrote its granule
    if (tid == h.owner) {
      GradCoef gc; gc.M = h.M; gc.k = p.k; gc.ls2 = h.ls2; gc.c0 = h.e0; gc.c1 = h.e1;
      st_real<KIND>(drow + y * B, grad_target<KIND, ENT>(h.zy, gc, h.target));
    }
  }
  if (!left) {
    side ^= 1;
    if (!ok && lane == 0) rb.bad[side] = 1;
    bar_sync_n(1, threads);
    if (rb.bad[side]) ok = false;
  }
  if (!ok && lane == 0) { atomicMin(&rb.done, jobs - 1); rb.failed = 1; }
  row_block_end<KIND, W>(rb, geo, p, rows, BACK, fail_row);
}

// Short rows (up to 16 KB): a warp takes one at a time, four granules per lane in a batch.  Nothing is shared, so the latency
// of a row's loads and of its scalar arithmetic is hidden by the SM's other warps alone (a block and its barriers for every
// row took 66 us instead of 23 us for 16384 rows of 1000 bf16 logits).  A row of more than one batch is read again for the
// gradient: up to about 7 KB from the L1 cache, which the 32 rows in work on an SM fit then (keeping it in 64 registers per lane
// leaves room for half as many warps: 64 us instead of 51 us for 12384 rows of 3001 bf16 logits, 41 us since the outer entries are
// taken one by each lane), longer ones mostly from memory (12384 rows of 8000: 306 MB read for 198 MB of logits, 94 us).
constexpr int SR_WARPS = 4, SR_NV = 4, SR_MAX_GRANULES = 1024;
template <int KIND, int MODE>
__global__ void __launch_bounds__(32 * SR_WARPS, 8) token_short_kernel(const __grid_constant__ TokenArgs p, const __grid_constant__ PolicyArgs q, const __grid_constant__ ForwardArgs f, int64_t rows) {
  constexpr bool BACK = MODE != RW_FORWARD, ENT = MODE == RW_ENTROPY;
  constexpr int E = Gran<KIND>::E, B = Gran<KIND>::B;
  const int lane = threadIdx.x & 31;
  griddep_wait();
  griddep_launch_dependents();
  const int64_t step = (int64_t)gridDim.x * SR_WARPS;
  int64_t row = (int64_t)blockIdx.x * SR_WARPS + (threadIdx.x >> 5);
  long long y_next = row < rows ? p.y[row] : -1;
  const uint32_t ni = neg_inf_word<KIND>();
  for (; row < rows; row += step) {
    const long long y = y_next;
    if (row + step < rows) y_next = p.y[row + step];
    const Row<KIND> r(p.z + row * p.ldz * B, p.V);
    const int wa = r.mis ? 1 : 0, wb = (r.mis + p.V) / E;      // the whole granules
    char* drow = p.dz + row * p.lddz * B;
    const bool same = same_alignment(r, drow);
    if (y < 0) {
      if (BACK) zero_row<KIND>(drow, p.V, lane, 32);
      if (lane == 0) {
        RowStat none; none.logp = none.logp_lo = none.lse = none.H = none.M = none.ls2 = 0.f;
        store_stat(f, row, none);
        if (BACK) q.terms[row] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      continue;
    }
    // the entries outside the whole granules: one per lane at most
    const int h = min(p.V, wa * E - r.mis * wa), t0 = max(h, wb * E - r.mis);
    const int edge = lane < h ? lane : (lane >= 16 && t0 + lane - 16 < p.V ? t0 + lane - 16 : -1);
    float xe = 0.f;
    if (edge >= 0) xe = ld_real<KIND>(r.base + (int64_t)(r.mis + edge) * B);
    const float zy = target_logit<KIND>(p, row, y);
    float old = 0.f, adv = 0.f, wt = 0.f, ref = 0.f;
    if (BACK) {
      old = q.old_logp[row]; adv = q.adv[row]; wt = q.weight[row];
      if (q.ref_logp) ref = q.ref_logp[row];
    }
    uint4 v[SR_NV];
    Triple a;
    a.m = TK_LOWEST; a.s = a.t = 0.f;
    const uint4* src = reinterpret_cast<const uint4*>(r.base);
    for (int g0 = wa + lane; g0 < wb; g0 += 32 * SR_NV) {
#pragma unroll
      for (int i = 0; i < SR_NV; ++i) {
        v[i] = make_uint4(ni, ni, ni, ni);
        if (g0 + 32 * i < wb) v[i] = src[g0 + 32 * i];      // (kept in the L1 cache)
      }
      rebase(a, fmaxf(a.m, batch_max<KIND, SR_NV>(v)), p.k);
      accumulate<KIND, SR_NV>(a, v, p.k);
    }
    if (edge >= 0) add_entry(a, xe, p.k);
    warp_combine(a, p.k);
    const RowStat st = row_stat(a, zy, p);
    if (lane == 0) store_stat(f, row, st);
    if (!BACK) continue;
    const PolicyToken o = policy_token(st.logp, st.H, old, ref, q.ref_logp != nullptr, adv, wt, q);
    if (lane == 0) q.terms[row] = o.terms;
    if (o.g == 0.f && (!ENT || o.h == 0.f)) {      // a gradient of zero, whatever the logits are
      __syncwarp();
      zero_row<KIND>(drow, p.V, lane, 32);
      continue;
    }
    const float sc = q.grad_scale * p.inv_tau;
    GradCoef gc; gc.M = st.M; gc.k = p.k; gc.ls2 = st.ls2;
    gc.c0 = -(ENT ? fmaf(o.h, st.H, o.g) : o.g) * sc; gc.c1 = -o.h * TK_LN2 * sc;
    const int gy = y < p.V ? (r.mis + (int)y) / E : -1;
    __syncwarp();      // every lane has read the target's logit before it is overwritten
    uint4* dst = reinterpret_cast<uint4*>(drow - r.mis * B);
    for (int g0 = wa + lane; g0 < wb; g0 += 32 * SR_NV) {
      if (wb - wa > 32 * SR_NV) {
#pragma unroll
        for (int i = 0; i < SR_NV; ++i)
          if (g0 + 32 * i < wb) v[i] = src[g0 + 32 * i];
      }
#pragma unroll
      for (int i = 0; i < SR_NV; ++i)
        if (g0 + 32 * i < wb) {
          const uint4 d = grad_granule<KIND, ENT>(v[i], gc);
          if (same) st_stream(dst + g0 + 32 * i, d); else store_entries<KIND>(drow, r.mis, p.V, g0 + 32 * i, d);
        }
    }
    if (edge >= 0) st_real<KIND>(drow + (int64_t)edge * B, grad_target<KIND, ENT>(xe, gc, edge == y ? o.g * sc : 0.f));
    if (gy >= wa && gy < wb && ((gy - wa) & 31) == lane) st_real<KIND>(drow + y * B, grad_target<KIND, ENT>(zy, gc, o.g * sc));
  }
}

// Deterministic sum of the rows' terms by one block: stats = loss, policy, KL, entropy, clipped weight.
__global__ void __launch_bounds__(1024) policy_sum_kernel(const float4* __restrict__ terms, int64_t rows, float kl_coef, float ent_coef, float* __restrict__ stats) {
  __shared__ double sh[4][32];
  griddep_wait();
  griddep_launch_dependents();
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for (int64_t i = threadIdx.x; i < rows; i += 4096) {
    float4 t[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) t[u] = i + 1024 * u < rows ? terms[i + 1024 * u] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int u = 0; u < 4; ++u) { s[0] += t[u].x; s[1] += t[u].y; s[2] += t[u].z; s[3] += t[u].w; }
  }
  for (int c = 0; c < 4; ++c) {
    for (int o = 16; o; o >>= 1) s[c] += __shfl_xor_sync(0xffffffffu, s[c], o);
    if ((threadIdx.x & 31) == 0) sh[c][threadIdx.x >> 5] = s[c];
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double t[4];
    for (int c = 0; c < 4; ++c) { t[c] = 0.0; for (int w = 0; w < 32; ++w) t[c] += sh[c][w]; }
    // (a term that is only looked at stays out of the loss, also an infinite one)
    stats[0] = (float)(t[0] + (kl_coef != 0.f ? (double)kl_coef * t[1] : 0.0) - (ent_coef != 0.f ? (double)ent_coef * t[2] : 0.0));
    for (int c = 0; c < 4; ++c) stats[1 + c] = (float)t[c];
  }
}

// ---------------------------------------------------------------------------------------------------------------
// Forward pass over a few rows: C blocks stream a row with running triples, so that four rows of 131072 bf16 logits keep 32 SMs
// busy (4.8 us, the launch included; what is read takes 0.2).  POLICY: the rows' loss terms too.
constexpr int TF_THREADS = 256;
template <int KIND, bool POLICY>
__global__ void __launch_bounds__(TF_THREADS, 4) token_forward_kernel(const __grid_constant__ TokenArgs p, const __grid_constant__ ForwardArgs f,
                                                                      const __grid_constant__ PolicyArgs q, int C) {
  constexpr int NV = 4;
  __shared__ float4 sh[TK_MAX_CLUSTER * (TF_THREADS / 32)];
  if (C > 1) cluster_arrive_relaxed();
  griddep_wait();
  griddep_launch_dependents();
  const int64_t row = blockIdx.x / C;
  const int rank = C > 1 ? (int)cluster_rank() : 0;
  const long long y = p.y[row];
  if (C > 1) cluster_wait();
  if (y < 0) {
    if (rank == 0 && threadIdx.x == 0) {
      RowStat none; none.logp = none.logp_lo = none.lse = none.H = none.M = none.ls2 = 0.f;
      store_stat(f, row, none);
      if (POLICY) q.terms[row] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    return;
  }
  const Row<KIND> r(p.z + row * p.ldz * Gran<KIND>::B, p.V);
  const int G = r.granules(), per = (G + C - 1) / C, g0 = rank * per, g1 = min(G, g0 + per);
  const float zy = target_logit<KIND>(p, row, y);
  const uint32_t ni = neg_inf_word<KIND>();
  Triple a; a.m = TK_LOWEST; a.s = a.t = 0.f;
  for (int gb = g0 + (int)threadIdx.x; gb < g1; gb += NV * TF_THREADS) {
    uint4 v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int g = gb + i * TF_THREADS;
      v[i] = make_uint4(ni, ni, ni, ni);
      if (g < g1) v[i] = r.load(g);
    }
    rebase<true>(a, fmaxf(a.m, batch_max<KIND, NV>(v)), p.k);
    accumulate<KIND, NV>(a, v, p.k);
  }
  row_combine<TF_THREADS>(a, p.k, C, sh);
  if (rank != 0 || threadIdx.x != 0) return;
  const RowStat st = row_stat(a, zy, p, TK_EX2_LOW_SPLIT);
  store_stat(f, row, st);
  if (POLICY) q.terms[row] = policy_token(st.logp, st.H, q.old_logp[row], q.ref_logp ? q.ref_logp[row] : 0.f, q.ref_logp != nullptr, q.adv[row], q.weight[row], q).terms;
}

// Gradient pass: short rows, one granule per thread and all rows one after the other; longer ones through the ring.  The
// rows are taken from the end: what the forward pass read last is still in the L2 cache.
struct BackwardArgs {
  const float* lse;          // of the forward call, or
  const float2* stat;        // (M, log2 S), more exact where lse is large
  const float* g;            // d loss / d logp
  const float* h;            // d loss / d entropy, or null
  const float* entropy;      // with h
  float scale;
};
// A row whose coefficients are zero has a gradient of zero whatever its logits are.
template <bool ENT>
__device__ __forceinline__ bool no_gradient(const BackwardArgs& b, int64_t row) { return b.g[row] == 0.f && (!ENT || b.h[row] == 0.f); }
constexpr int TB2_THREADS = 256;
template <int KIND, bool ENT>
__device__ __forceinline__ void backward_coef(const TokenArgs& p, const BackwardArgs& b, int64_t row, long long y, GradCoef& gc, float& target) {
  const float gg = b.g[row];
  float hh = 0.f, H = 0.f;
  if (ENT) { hh = b.h[row]; H = b.entropy[row]; }
  const float sc = b.scale * p.inv_tau;
  gc.k = p.k;
  if (b.stat) { const float2 s = b.stat[row]; gc.M = s.x; gc.ls2 = s.y; }
  else { gc.M = 0.f; gc.ls2 = b.lse[row] * 1.4426950408889634f; }
  gc.c0 = -(ENT ? fmaf(hh, H, gg) : gg) * sc; gc.c1 = -hh * TK_LN2 * sc;
  if (y >= p.V) gc.c0 = __int_as_float(0x7fc00000);
  target = gg * sc;
}
template <int KIND, bool ENT>
__global__ void __launch_bounds__(TB2_THREADS, 4) token_backward_short_kernel(const __grid_constant__ TokenArgs p, const __grid_constant__ BackwardArgs b, int64_t rows, uint32_t G) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t at = (int64_t)(gridDim.x - 1 - blockIdx.x) * TB2_THREADS + threadIdx.x, row = at / G;
  const int g = (int)(at - row * G);
  if (row >= rows) return;
  const long long y = p.y[row];
  const Row<KIND> r(p.z + row * p.ldz * Gran<KIND>::B, p.V);
  if (g >= r.granules()) return;
  char* drow = p.dz + row * p.lddz * Gran<KIND>::B;
  const bool same = same_alignment(r, drow);
  if (y < 0) { store_granule<KIND>(r, drow, same, g, make_uint4(0, 0, 0, 0)); return; }
  const uint4 v = r.load(g);
  GradCoef gc; float target;
  backward_coef<KIND, ENT>(p, b, row, y, gc, target);
  const bool mine = y < p.V && (r.mis + (int)y) / Gran<KIND>::E == g;
  float zy = 0.f;
  if (mine) zy = target_logit<KIND>(p, row, y);
  const bool none = no_gradient<ENT>(b, row);      // (looked at after the loads: 108 instead of 123 us for 12384 rows of 8000 bf16 logits)
  store_granule<KIND>(r, drow, same, g, none ? make_uint4(0, 0, 0, 0) : grad_granule<KIND, ENT>(v, gc));
  if (mine && !none) st_real<KIND>(drow + y * Gran<KIND>::B, grad_target<KIND, ENT>(zy, gc, target));
}

// Longer rows: 8192 x 32768 bf16 173 us, 6.2 TB/s of reading and writing (a block per piece of a row, loads and arithmetic one
// after the other: 195 us).
template <int KIND, bool ENT, int W>
__global__ void __maxnreg__(80) token_gradient_kernel(const __grid_constant__ TokenArgs p, const __grid_constant__ BackwardArgs b, int64_t rows, const __grid_constant__ RowGeom geo) {
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ RowBarriers rb;
  constexpr int E = Gran<KIND>::E, B = Gran<KIND>::B;
  constexpr int threads = 32 * W, chunk = RW_NV * threads;
  const int N = geo.N, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == W) rb.init(N, W, lane);
  __syncthreads();
  griddep_wait();
  griddep_launch_dependents();
  const auto fail_row = [](int64_t, float) {};
  if (warp == W) {
    fetch_rows<KIND, false, true>(p, rows, geo, ring, rb, lane, chunk, [&](int64_t at) { return !no_gradient<ENT>(b, at); });
    row_block_end<KIND, W>(rb, geo, p, rows, true, fail_row);
    return;
  }
  const uint4* const places = reinterpret_cast<const uint4*>(ring);
  const int64_t zstep = p.ldz * B, dstep = p.lddz * B;
  const char* zrow = p.z;
  char* drow = p.dz;
  int s = 0, jobs = 0;                // as in the row kernel
  uint32_t ph = 0;
  int64_t row = 0, row_end = 0;
  long long y_next = -1;
  GradCoef c_next; float t_next = 0.f;      // of the next row, asked for while this one is worked on
  c_next.M = c_next.k = c_next.ls2 = c_next.c0 = c_next.c1 = 0.f;
  bool ok = true;
  for (;; ++row, zrow += zstep, drow += dstep) {
    if (row == row_end) {      // the next unit of rows
      const int js = jobs % RW_JOBS;
      ok = __all_sync(0xffffffffu, mbar_wait_asleep(&rb.jfull[js], (uint32_t)(jobs / RW_JOBS) & 1));
      ++jobs;
      if (!ok) break;
      const longlong2 jb = rb.job[js];
      __syncwarp();
      if (lane == 0) mbar_arrive(&rb.jempty[js]);
      if (jb.x < 0) break;
      row = jb.x * geo.unit; row_end = min((long long)(row + geo.unit), (long long)rows);
      y_next = jb.y;
      zrow = p.z + row * zstep; drow = p.dz + row * dstep;
      if (y_next >= 0) backward_coef<KIND, ENT>(p, b, row, y_next, c_next, t_next);
    }
    const long long y = y_next;
    const GradCoef gc = c_next;
    const float target = t_next;
    if (row + 1 < row_end) {
      y_next = p.y[row + 1];
      backward_coef<KIND, ENT>(p, b, row + 1, y_next, c_next, t_next);      // (of an ignored row: read, not used)
    }
    const Row<KIND> r(zrow, p.V);
    const bool same = same_alignment(r, drow);
    if (y < 0 || no_gradient<ENT>(b, row)) {
      zero_row<KIND>(drow, p.V, tid, threads);
      continue;
    }
    const int wa = r.mis ? 1 : 0, wb = (r.mis + p.V) / E, nw = max(0, wb - wa), K = geo.K - (nw <= geo.last), tail = nw - (K - 1) * chunk;
    // the entries outside the whole granules, and the target's logit, by the threads that overwrite them
    if (warp == 0) {
      const int h = min(p.V, wa * E - r.mis * wa), t0 = max(h, wb * E - r.mis);
      const int edge = lane < h ? lane : (lane >= 16 && t0 + lane - 16 < p.V ? t0 + lane - 16 : -1);
      if (edge >= 0) st_real<KIND>(drow + (int64_t)edge * B, grad_target<KIND, ENT>(ld_real<KIND>(r.base + (int64_t)(r.mis + edge) * B), gc, edge == y ? target : 0.f));
    }
    const int ly = y < p.V ? (r.mis + (int)y) / E - wa : -1;
    const bool mine = ly >= 0 && ly < nw && (ly - tid) % threads == 0;
    float zy = 0.f;
    if (mine) zy = target_logit<KIND>(p, row, y);
    RowGrad h;
    gradient_coef<KIND, ENT>(h, gc.M, gc.ls2, gc.c0, gc.c1, p.k);
    const bool fast = KIND != LS_F32 && h.fast;
    uint4* dst = reinterpret_cast<uint4*>(drow - r.mis * B) + wa + tid;
    for (int j = 0; j < K; ++j, dst += chunk) {
      ok = __all_sync(0xffffffffu, mbar_wait_asleep(&rb.full[s], ph));
      if (!ok) break;
      const uint4* place = places + s * chunk + tid;
      uint4 v[RW_NV];
      if (same && (j < K - 1 || tail == chunk)) {
#pragma unroll
        for (int u = 0; u < RW_NV; ++u) v[u] = place[u * threads];
        release_place(&rb.empty[s], lane);
#pragma unroll
        for (int u = 0; u < RW_NV; ++u)
          st_stream(dst + u * threads, fast ? row_gradient<KIND, ENT, true>(v[u], h, p.k) : row_gradient<KIND, ENT, false>(v[u], h, p.k));
      } else {
        const int len = j < K - 1 ? chunk : tail, g0 = wa + j * chunk;
#pragma unroll
        for (int u = 0; u < RW_NV; ++u)
          if (tid + u * threads < len) v[u] = place[u * threads];
        release_place(&rb.empty[s], lane);
#pragma unroll
        for (int u = 0; u < RW_NV; ++u)
          if (tid + u * threads < len) store_granule<KIND>(r, drow, same, g0 + tid + u * threads, fast ? row_gradient<KIND, ENT, true>(v[u], h, p.k) : row_gradient<KIND, ENT, false>(v[u], h, p.k));
      }
      if (++s == N) { s = 0; ph ^= 1; }
    }
    if (!ok) break;
    if (mine) st_real<KIND>(drow + y * B, grad_target<KIND, ENT>(zy, gc, target));
  }
  if (!ok && lane == 0) { atomicMin(&rb.done, jobs - 1); rb.failed = 1; }
  row_block_end<KIND, W>(rb, geo, p, rows, true, fail_row);
}

// ---------------------------------------------------------------------------------------------------------------
// Pairs of answers.  R_s = beta * sum over the rows of answer s of (logp - ref), h = R_chosen - R_rejected,
// loss = -(1 - eps) log sigma(h) - eps log sigma(-h), averaged over the pairs; d loss / d logp = +-beta/B (sigma(h) - (1 - eps)).
struct PairArgs {
  const int* starts;          // 2 * pairs + 1 rows; answer s has rows [starts[s], starts[s + 1])
  const float* ref;
  const float* logp; const float* logp_lo;
  const long long* y;
  int64_t rows;
  int pairs;
  float beta, smoothing;
  float* g;                   // out: d loss / d logp of each row of the answers
  float* rewards;             // out: R_s
  double* terms;              // out: loss of each pair
  unsigned* ticket;           // 0; the last block to take one adds the terms up
  float* loss;
};
constexpr int TP_THREADS = 512;
__global__ void __launch_bounds__(TP_THREADS) pair_kernel(const __grid_constant__ PairArgs a) {
  __shared__ double sh[2][TP_THREADS / 32];
  __shared__ float coef;
  __shared__ int last;
  griddep_wait();
  griddep_launch_dependents();
  const int b = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int64_t at[4];
  double R[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    int64_t lo = a.starts[2 * b + c], hi = a.starts[2 * b + c + 1];      // bounds that make no sense never leave [0, rows]
    lo = lo < 0 ? 0 : (lo > a.rows ? a.rows : lo);
    hi = hi < lo ? lo : (hi > a.rows ? a.rows : hi);
    at[2 * c] = lo; at[2 * c + 1] = hi;
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    double s = 0.0;
    for (int64_t i = at[2 * c] + threadIdx.x; i < at[2 * c + 1]; i += TP_THREADS) {
      const float lp = a.logp[i], lo = a.logp_lo[i], rf = a.ref[i];
      s += a.y[i] >= 0 ? ((double)lp - (double)rf) + (double)lo : (double)lp;      // (an ignored row's is 0, or NaN after a failure)
    }
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    R[c] = s;
  }
  if (lane == 0) { sh[0][warp] = R[0]; sh[1][warp] = R[1]; }
  __syncthreads();
  if (threadIdx.x == 0) {
    R[0] = R[1] = 0.0;
    for (int w = 0; w < TP_THREADS / 32; ++w) { R[0] += sh[0][w]; R[1] += sh[1][w]; }
    R[0] *= (double)a.beta; R[1] *= (double)a.beta;
    const double h = R[0] - R[1], e = (double)a.smoothing;
    const double x = exp(-fabs(h)), tail = log1p(x);                     // -log sigma(z) = max(-z, 0) + tail
    // (h is infinite where a token of one answer has probability zero: a part that the smoothing leaves out stays out)
    a.terms[b] = h != h ? h : (e < 1.0 ? (1.0 - e) * (fmax(-h, 0.0) + tail) : 0.0) + (e > 0.0 ? e * (fmax(h, 0.0) + tail) : 0.0);
    a.rewards[2 * b] = (float)R[0]; a.rewards[2 * b + 1] = (float)R[1];
    const double right = h >= 0.0 ? 1.0 / (1.0 + x) : x / (1.0 + x);
    coef = (float)((double)a.beta * (right - (1.0 - e)) / (double)a.pairs);
    __threadfence();
    last = atomicAdd(a.ticket, 1u) == (unsigned)a.pairs - 1;
  }
  __syncthreads();
  if (a.g) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
      for (int64_t i = at[2 * c] + threadIdx.x; i < at[2 * c + 1]; i += TP_THREADS) a.g[i] = c == 0 ? coef : -coef;
  }
  if (!last) return;
  // every block's term is there; they are added in the order of the pairs whichever block is the last
  __threadfence();
  double s = 0.0;
  for (int i = threadIdx.x; i < a.pairs; i += TP_THREADS) s += __ldcg(a.terms + i);
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) sh[0][warp] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < TP_THREADS / 32; ++w) s += sh[0][w];
    *a.loss = (float)(s / (double)a.pairs);
  }
}

}  // namespace tg
