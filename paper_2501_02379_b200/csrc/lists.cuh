// Kernels over a list of tensors: gradient norm, clipping, AdamW.
//
// A list travels in the kernel's parameters (pointer, length and first chunk of each tensor), so a call copies nothing
// to the device, keeps nothing between calls and can be captured.  The tensors are cut into chunks, numbered through
// the whole list; block b of `grid` works on chunks [b total / grid, (b + 1) total / grid), a contiguous run whatever
// the sizes of the tensors, and finds the tensor of its first chunk by bisection.
#pragma once
#include "common.cuh"
#include "ptx.cuh"

namespace tg {

constexpr int LS_THREADS = 256;

// How the entries of a list of reals are stored (a complex tensor is a list of twice as many reals).
enum { LS_F32 = 0, LS_F16 = 1, LS_BF16 = 2 };

struct ListEntry {
  char* ptr;             // first entry
  uint64_t count;        // entries (reals), storage kind in the top two bits
};
__host__ __device__ __forceinline__ uint64_t list_count(uint64_t c) { return c & ((1ull << 62) - 1); }
__host__ __device__ __forceinline__ int list_kind(uint64_t c) { return (int)(c >> 62); }
__host__ __device__ __forceinline__ int list_log2_bytes(uint64_t c) { return list_kind(c) == LS_F32 ? 2 : 1; }

template <int CAP>
struct ListParams {
  int n;                 // tensors
  uint32_t gpc_log2;     // 16-byte granules per chunk, as a power of two
  uint32_t total;        // chunks
  uint32_t first[CAP + 1];   // first chunk of each tensor; first[n] = total
  ListEntry e[CAP];
};

// 16-byte granules that a tensor touches: the memory it lies in is cut at multiples of 16 bytes, so that whatever the
// alignment of its first entry all granules but the outer two are read and written by aligned 16-byte accesses.
__host__ __device__ __forceinline__ uint64_t list_granules(const ListEntry& e) {
  const uint64_t n = list_count(e.count);
  return n ? (((uint64_t)(uintptr_t)e.ptr & 15) + (n << list_log2_bytes(e.count)) + 15) >> 4 : 0;
}

// largest t with first[t] <= c (tensors without chunks share their successor's start and are skipped)
template <int CAP>
__device__ __forceinline__ int list_find(const ListParams<CAP>& p, uint32_t c) {
  int lo = 0, hi = p.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.first[mid] <= c) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void st_stream(uint4* p, uint4 v) {
  asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// one entry as fp32 (widening is exact)
template <int KIND>
__device__ __forceinline__ float ld_real(const char* p) {
  if (KIND == LS_F32) return *reinterpret_cast<const float*>(p);
  if (KIND == LS_F16) return __half2float(*reinterpret_cast<const __half*>(p));
  return __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(p));
}
template <int KIND>
__device__ __forceinline__ void st_real(char* p, float v) {
  if (KIND == LS_F32) *reinterpret_cast<float*>(p) = v;
  else if (KIND == LS_F16) *reinterpret_cast<__half*>(p) = __float2half_rn(v);
  else *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(v);
}
// the two entries of a 32-bit word of 16-bit storage
template <int KIND>
__device__ __forceinline__ float2 widen2(uint32_t w) {
  if (KIND == LS_F16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <int KIND>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {      // round to nearest even
  if (KIND == LS_F16) { const __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <int KIND>
__device__ __forceinline__ float sumsq_word(uint32_t w, float s) {
  if (KIND == LS_F32) { const float x = __uint_as_float(w); return fmaf(x, x, s); }
  const float2 x = widen2<KIND>(w);
  return fmaf(x.y, x.y, fmaf(x.x, x.x, s));
}
template <int KIND>
__device__ __forceinline__ float sumsq_batch(const uint4 (&v)[8]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    s = sumsq_word<KIND>(v[i].x, s); s = sumsq_word<KIND>(v[i].y, s);
    s = sumsq_word<KIND>(v[i].z, s); s = sumsq_word<KIND>(v[i].w, s);
  }
  return s;
}
template <int KIND>
__device__ __noinline__ double sumsq_words_double(const uint4* v, int n) {
  double acc = 0.0;
  for (int i = 0; i < n; ++i) {
    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
    for (int j = 0; j < 4; ++j) {
      if (KIND == LS_F32) { const double x = (double)__uint_as_float(w[j]); acc += x * x; }
      else { const float2 x = widen2<KIND>(w[j]); acc += (double)x.x * x.x + (double)x.y * x.y; }
    }
  }
  return acc;
}
template <int KIND>
__device__ __noinline__ double sumsq_entries(const char* p, uint32_t bytes) {
  double acc = 0.0;
  for (uint32_t b = 0; b < bytes; b += KIND == LS_F32 ? 4 : 2) { const double x = ld_real<KIND>(p + b); acc += x * x; }
  return acc;
}
__device__ __forceinline__ double sumsq_edge(int kind, const char* p, uint32_t bytes) {
  return kind == LS_F32 ? sumsq_entries<LS_F32>(p, bytes) : kind == LS_F16 ? sumsq_entries<LS_F16>(p, bytes) : sumsq_entries<LS_BF16>(p, bytes);
}

// Sum of squares of one chunk's share of a thread.  The up to 64 squares of one batch are added in fp32 and the batches
// in fp64: 2^-24 per term, and no loss in the long sum.  A batch whose fp32 sum leaves the range in which no square can
// have overflowed or been flushed (but is not all zeros) is added again in fp64, so gradients of 1e-30 or 1e30 count.
__device__ __forceinline__ double sumsq_chunk(const ListEntry& e, uint32_t chunk, uint32_t gpc_log2) {
  const int kind = list_kind(e.count);
  const uint32_t mis = (uint32_t)((uintptr_t)e.ptr & 15);
  const char* base = e.ptr - mis;
  const uint64_t end = mis + (list_count(e.count) << list_log2_bytes(e.count)), gfull = end >> 4, gall = (end + 15) >> 4;
  const uint64_t g0 = (uint64_t)chunk << gpc_log2;
  uint64_t g1 = g0 + (1ull << gpc_log2);
  const bool last = g1 >= gall;
  if (g1 > gfull) g1 = gfull;                                        // whole granules [first, g1) of the chunk
  const uint64_t first = g0 == 0 && mis != 0 ? 1 : g0;
  double acc = 0.0;
  for (uint64_t gb = first + threadIdx.x; gb < g1; gb += 8 * LS_THREADS) {
    const uint4* at = reinterpret_cast<const uint4*>(base) + gb;
    const uint32_t left = (uint32_t)(g1 - gb < 8 * LS_THREADS ? g1 - gb : 8 * LS_THREADS);
    uint4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = make_uint4(0, 0, 0, 0);
      if (i * LS_THREADS < left) v[i] = ld_stream(at + i * LS_THREADS);
    }
    const float s = kind == LS_F32 ? sumsq_batch<LS_F32>(v) : kind == LS_F16 ? sumsq_batch<LS_F16>(v) : sumsq_batch<LS_BF16>(v);
    if (s > 1e-20f && s < 1e38f) acc += (double)s;
    else {
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) any |= v[i].x | v[i].y | v[i].z | v[i].w;
      if (any) {
        uint4 w[8];      // a copy, so that the values of the usual case stay in registers
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = v[i];
        acc += kind == LS_F32 ? sumsq_words_double<LS_F32>(w, 8) : kind == LS_F16 ? sumsq_words_double<LS_F16>(w, 8) : sumsq_words_double<LS_BF16>(w, 8);
      }
    }
  }
  // the outer granules hold entries of other tensors too: entry by entry, by one thread each
  if (threadIdx.x == 0 && g0 == 0 && mis != 0) acc += sumsq_edge(kind, e.ptr, (uint32_t)((end < 16 ? end : 16) - mis));
  if (threadIdx.x == 32 && last && (end & 15) != 0 && !(gfull == 0 && mis != 0)) acc += sumsq_edge(kind, base + (gfull << 4), (uint32_t)(end & 15));
  return acc;
}

// Sum over the block; the result is valid in thread 0.  sh: 8 doubles.
__device__ __forceinline__ double block_sum(double v, double* sh) {
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
  if (threadIdx.x == 0)
    for (int w = 0; w < LS_THREADS / 32; ++w) t += sh[w];
  return t;
}

// Partial sums of squares.  Block b writes one per tensor t it has chunks of, at slot b + t: along the list each next
// (block, tensor) pair has a larger b + t, so the slots are distinct and a tensor's slots are b0 + t .. b1 + t.  Slots that
// no pair has are set to zero by the block before them, so that all grid + n of them may be added up.
// Bound: one read of the gradients.  Eight 16-byte loads per thread are under way at a time (128 KB per SM, three times what
// the memory's latency needs); two fused multiply-adds per 16-bit pair are nowhere near the limit.  1.64 GB of complex64 and
// bf16 gradients: 242 us, 6.8 TB/s.
template <int CAP>
__global__ void __launch_bounds__(LS_THREADS, 4) list_sumsq_kernel(const __grid_constant__ ListParams<CAP> p, double* __restrict__ partial) {
  __shared__ double sh[LS_THREADS / 32];
  griddep_wait();
  griddep_launch_dependents();
  uint32_t c = (uint32_t)((uint64_t)blockIdx.x * p.total / gridDim.x);
  const uint32_t c1 = (uint32_t)((uint64_t)(blockIdx.x + 1) * p.total / gridDim.x);
  if (c >= c1) return;
  int t = list_find(p, c);
  if (blockIdx.x == 0)
    for (int i = (int)threadIdx.x; i < t; i += LS_THREADS) partial[i] = 0.0;
  while (c < c1) {
    while (p.first[t + 1] <= c) ++t;
    const ListEntry e = p.e[t];
    const uint32_t stop = p.first[t + 1] < c1 ? p.first[t + 1] : c1;
    double acc = 0.0;
    for (; c < stop; ++c) acc += sumsq_chunk(e, c - p.first[t], p.gpc_log2);
    const double sum = block_sum(acc, sh);
    if (threadIdx.x == 0) partial[blockIdx.x + t] = sum;
    // up to the next pair's slot
    int next = t + 1;
    uint32_t slot = blockIdx.x;
    if (c >= c1) ++slot;                                     // the next block's first tensor, or the end of the slots
    if (c < p.total) { next = t; while (p.first[next + 1] <= c) ++next; } else { next = p.n; }
    for (uint32_t i = blockIdx.x + t + 1 + threadIdx.x; i < slot + next; i += LS_THREADS) partial[i] = 0.0;
  }
}

// The coefficient that brings a global norm down to max_norm.
__device__ __forceinline__ float clip_coefficient(float norm, float max_norm) {
  const float c = max_norm < __int_as_float(0x7f800000) ? max_norm / (norm + 1e-6f) : 1.f;
  return c < 1.f || c != c ? c : 1.f;
}
// The tensors' norms, and after the last slice of a long list the global norm and the coefficient, by one block.
// out[0] norm, out[1] coefficient, out[2 + i] norm of tensor i.  slice_sum[s] keeps the sums of the slices so far.
struct NormArgs {
  const double* partial;
  uint32_t grid;         // of the kernel that wrote them
  int base, slice, last;
  double* slice_sum;
  float max_norm;
  float* out;
};
// All partial sums of one slice, in a fixed order; valid in every thread.  sh: 8 doubles.
__device__ __forceinline__ double norm_sum(const double* __restrict__ partial, uint32_t slots, double* sh) {
  double s = 0.0;
  for (uint32_t i = threadIdx.x; i < slots; i += LS_THREADS) s += partial[i];
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < LS_THREADS / 32; ++w) s += sh[w];
  return s;
}
// One tensor's norm per warp, all at once (they are latency and nothing else), and by the first block the global results.
template <int CAP>
__device__ __forceinline__ void write_norms(const ListParams<CAP>& p, const NormArgs& a, uint32_t block, double* sh) {
  const int t = (int)block * (LS_THREADS / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (t < p.n) {
    const uint32_t f0 = p.first[t], f1 = p.first[t + 1];
    double s = 0.0;
    if (f1 > f0) {      // the blocks of chunks f0 and f1 - 1
      const uint32_t b0 = (uint32_t)((((uint64_t)f0 + 1) * a.grid - 1) / p.total), b1 = (uint32_t)(((uint64_t)f1 * a.grid - 1) / p.total);
      for (uint32_t b = b0 + lane; b <= b1; b += 32) s += a.partial[b + t];
      for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    }
    if (lane == 0) a.out[2 + a.base + t] = (float)sqrt(s);
  }
  if (block != 0) return;
  double s = a.grid > 0 ? norm_sum(a.partial, a.grid + p.n - 1, sh) : 0.0;
  if (threadIdx.x != 0) return;
  if (!a.last) { a.slice_sum[a.slice] = s; return; }
  for (int i = 0; i < a.slice; ++i) s += a.slice_sum[i];
  const float norm = (float)sqrt(s);
  a.out[0] = norm;
  a.out[1] = clip_coefficient(norm, a.max_norm);
}
template <int CAP>
__global__ void __launch_bounds__(LS_THREADS) list_norm_kernel(const __grid_constant__ ListParams<CAP> p, const __grid_constant__ NormArgs a) {
  __shared__ double sh[LS_THREADS / 32];
  griddep_wait();
  griddep_launch_dependents();
  write_norms<CAP>(p, a, blockIdx.x, sh);
}

// x <- c x for one chunk: every entry is multiplied in fp32 and rounded once to its storage type.
template <int KIND>
__device__ __forceinline__ uint32_t scale_word(uint32_t w, float c) {
  if (KIND == LS_F32) return __float_as_uint(__uint_as_float(w) * c);
  const float2 x = widen2<KIND>(w);
  return narrow2<KIND>(x.x * c, x.y * c);
}
template <int KIND>
__device__ __forceinline__ uint4 scale_granule(uint4 v, float c) {
  return make_uint4(scale_word<KIND>(v.x, c), scale_word<KIND>(v.y, c), scale_word<KIND>(v.z, c), scale_word<KIND>(v.w, c));
}
template <int KIND>
__device__ __noinline__ void scale_entries(char* p, uint32_t bytes, float c) {
  for (uint32_t b = 0; b < bytes; b += KIND == LS_F32 ? 4 : 2) st_real<KIND>(p + b, ld_real<KIND>(p + b) * c);
}
__device__ __forceinline__ void scale_edge(int kind, char* p, uint32_t bytes, float c) {
  if (kind == LS_F32) scale_entries<LS_F32>(p, bytes, c);
  else if (kind == LS_F16) scale_entries<LS_F16>(p, bytes, c);
  else scale_entries<LS_BF16>(p, bytes, c);
}
__device__ __forceinline__ void scale_chunk(const ListEntry& e, uint32_t chunk, uint32_t gpc_log2, float c) {
  const int kind = list_kind(e.count);
  const uint32_t mis = (uint32_t)((uintptr_t)e.ptr & 15);
  char* base = e.ptr - mis;
  const uint64_t end = mis + (list_count(e.count) << list_log2_bytes(e.count)), gfull = end >> 4, gall = (end + 15) >> 4;
  const uint64_t g0 = (uint64_t)chunk << gpc_log2;
  uint64_t g1 = g0 + (1ull << gpc_log2);
  const bool last = g1 >= gall;
  if (g1 > gfull) g1 = gfull;                                        // whole granules [first, g1) of the chunk
  const uint64_t first = g0 == 0 && mis != 0 ? 1 : g0;
  for (uint64_t gb = first + threadIdx.x; gb < g1; gb += 8 * LS_THREADS) {
    uint4* at = reinterpret_cast<uint4*>(base) + gb;
    const uint32_t left = (uint32_t)(g1 - gb < 8 * LS_THREADS ? g1 - gb : 8 * LS_THREADS);
    uint4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i * LS_THREADS < left) v[i] = ld_stream(at + i * LS_THREADS);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i] = kind == LS_F32 ? scale_granule<LS_F32>(v[i], c) : kind == LS_F16 ? scale_granule<LS_F16>(v[i], c) : scale_granule<LS_BF16>(v[i], c);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i * LS_THREADS < left) st_stream(at + i * LS_THREADS, v[i]);
  }
  // the outer granules hold entries of other tensors too: entry by entry, by one thread each
  if (threadIdx.x == 0 && g0 == 0 && mis != 0) scale_edge(kind, e.ptr, (uint32_t)((end < 16 ? end : 16) - mis), c);
  if (threadIdx.x == 32 && last && (end & 15) != 0 && !(gfull == 0 && mis != 0)) scale_edge(kind, base + (gfull << 4), (uint32_t)(end & 15), c);
}

// Scales every tensor by the coefficient.  A coefficient of 1 leaves every entry as it is, so nothing is read or written
// then.  WRITE: the list is one slice, and this kernel forms the norm itself, each block for itself, from the partial sums,
// while some further blocks write the results: a launch less on the way.
template <int CAP, bool WRITE>
__global__ void __launch_bounds__(LS_THREADS, 4) list_scale_kernel(const __grid_constant__ ListParams<CAP> p, const __grid_constant__ NormArgs a) {
  __shared__ double sh[LS_THREADS / 32];
  griddep_wait();
  griddep_launch_dependents();
  const uint32_t writers = WRITE ? (p.n + LS_THREADS / 32 - 1) / (LS_THREADS / 32) : 0, blocks = gridDim.x - writers;
  float s;
  if (WRITE) {
    if (blockIdx.x < writers) { write_norms<CAP>(p, a, blockIdx.x, sh); return; }
    s = clip_coefficient((float)sqrt(norm_sum(a.partial, a.grid + p.n - 1, sh)), a.max_norm);
  } else {
    s = a.out[1];
  }
  if (s == 1.f) return;
  // back to front: what the norm's pass read last is still in the caches
  const uint32_t b = gridDim.x - 1 - blockIdx.x;
  const uint32_t lo = (uint32_t)((uint64_t)b * p.total / blocks);
  uint32_t c = (uint32_t)((uint64_t)(b + 1) * p.total / blocks);
  if (lo >= c) return;
  int t = list_find(p, c - 1);
  while (c > lo) {
    --c;
    while (p.first[t] > c) --t;
    const ListEntry e = p.e[t];
    scale_chunk(e, c - p.first[t], p.gpc_log2, s);
  }
}

// ---------------------------------------------------------------------------------------------------------------
// AdamW over a list.  m <- b1 m + (1 - b1) c g, v <- b2 v + (1 - b2) |c g|^2,
// w <- (1 - lr wd) w - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps), everything in fp32.  For complex tensors
// |.| is the modulus and v has one real per complex entry, as in the optimizer's compressed space.
// Each entry is read and written once (28 bytes per entry for fp32 weights and for 16-bit ones with masters); memory bandwidth
// is the bound: 135 M bf16 weights with masters 591 us, 6.4 TB/s.  Two vectors of four entries per thread are loaded before
// the first is worked on (one: 670 us; four: 694 us, half the blocks).
struct AdamwScalars {
  float beta1, beta2, omb1, omb2;   // decay rates and 1 - beta
  float step_size;                  // lr / (1 - beta1^t)
  float inv_sqrt_c2;                // 1 / sqrt(1 - beta2^t)
  float eps, keep;                  // keep = 1 - lr * weight decay
  const float* gscale;              // device scalar c, or null (1)
};
struct AdamwEntry {
  char* w;               // weights in their storage type
  const char* g;         // gradients, same type
  float* m;
  float* v;
  float* master;         // fp32 weights of 16-bit ones, or null
  uint64_t count;        // entries (complex ones for LS_C64)
};
constexpr int LS_C64 = 3;
template <int CAP>
struct AdamwParams {
  int n;
  uint32_t epc_log2;     // entries per chunk, a power of two and at least 4
  uint32_t total;
  uint32_t first[CAP + 1];
  uint8_t head[CAP];     // entries before the first one at which all arrays can be accessed 4 entries (2 complex) at a
                         // time, or 255 where there is none
  AdamwEntry e[CAP];
};

__device__ __forceinline__ float adamw_real(float w, float g, float& m, float& v, const AdamwScalars& a) {
  m = a.beta1 * m + a.omb1 * g;
  v = a.beta2 * v + a.omb2 * (g * g);
  return a.keep * w - a.step_size * m / (sqrtf(v) * a.inv_sqrt_c2 + a.eps);
}
__device__ __forceinline__ void adamw_complex(float& wr, float& wi, float gr, float gi, float& mr, float& mi, float& v, const AdamwScalars& a) {
  mr = a.beta1 * mr + a.omb1 * gr;
  mi = a.beta1 * mi + a.omb1 * gi;
  v = a.beta2 * v + a.omb2 * (gr * gr + gi * gi);
  const float r = a.step_size / (sqrtf(v) * a.inv_sqrt_c2 + a.eps);
  wr = a.keep * wr - r * mr;
  wi = a.keep * wi - r * mi;
}

template <int KIND>
__device__ __forceinline__ void adamw_one(const AdamwEntry& e, uint64_t i, float c, const AdamwScalars& a) {
  if (KIND == LS_C64) {
    float* w = reinterpret_cast<float*>(e.w) + 2 * i;
    const float* g = reinterpret_cast<const float*>(e.g) + 2 * i;
    float wr = w[0], wi = w[1], mr = e.m[2 * i], mi = e.m[2 * i + 1], v = e.v[i];
    adamw_complex(wr, wi, g[0] * c, g[1] * c, mr, mi, v, a);
    w[0] = wr; w[1] = wi; e.m[2 * i] = mr; e.m[2 * i + 1] = mi; e.v[i] = v;
    return;
  }
  constexpr int K = KIND == LS_C64 ? LS_F32 : KIND;
  constexpr int B = K == LS_F32 ? 4 : 2;
  float m = e.m[i], v = e.v[i];
  const float old = e.master ? e.master[i] : ld_real<K>(e.w + B * i);
  const float w = adamw_real(old, ld_real<K>(e.g + B * i) * c, m, v, a);
  e.m[i] = m; e.v[i] = v;
  if (e.master) e.master[i] = w;
  st_real<K>(e.w + B * i, w);
}

__device__ __forceinline__ float4 f4(uint4 u) { return make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)); }
__device__ __forceinline__ uint4 u4(float4 f) { return make_uint4(__float_as_uint(f.x), __float_as_uint(f.y), __float_as_uint(f.z), __float_as_uint(f.w)); }
__device__ __forceinline__ float4 ld_f4(const float* p) { return f4(ld_stream(reinterpret_cast<const uint4*>(p))); }
__device__ __forceinline__ void st_f4(float* p, float4 v) { st_stream(reinterpret_cast<uint4*>(p), u4(v)); }
// four entries of storage KIND at an address that is a multiple of their size
template <int KIND>
__device__ __forceinline__ float4 ld_four(const char* p) {
  if (KIND == LS_F32) return ld_f4(reinterpret_cast<const float*>(p));
  uint2 u;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(u.x), "=r"(u.y) : "l"(p));
  const float2 a = widen2<KIND>(u.x), b = widen2<KIND>(u.y);
  return make_float4(a.x, a.y, b.x, b.y);
}
template <int KIND>
__device__ __forceinline__ void st_four(char* p, float4 v) {
  if (KIND == LS_F32) { st_f4(reinterpret_cast<float*>(p), v); return; }
  asm volatile("st.global.L1::no_allocate.v2.u32 [%0], {%1,%2};" ::"l"(p), "r"(narrow2<KIND>(v.x, v.y)), "r"(narrow2<KIND>(v.z, v.w)) : "memory");
}

// Entries [i0, i1) of one tensor by the block; `head` as in AdamwParams.
template <int KIND, bool MASTER>
__device__ __forceinline__ void adamw_chunk(const AdamwEntry& e, uint64_t i0, uint64_t i1, int head, float c, const AdamwScalars& a) {
  if (head == 255) {
    for (uint64_t i = i0 + threadIdx.x; i < i1; i += LS_THREADS) adamw_one<KIND>(e, i, c, a);
    return;
  }
  // the chunk's vectors start at `head` past a multiple of the vector length; the entries outside are done one by one
  constexpr int VL = KIND == LS_C64 ? 2 : 4;
  uint64_t a0 = i0 + head, a1;
  if (a0 > i1) a0 = i1;
  a1 = a0 + (i1 - a0) / VL * VL;
  constexpr int U = 2;
  for (uint64_t ib = a0 + (uint64_t)threadIdx.x * VL; ib < a1; ib += (uint64_t)U * LS_THREADS * VL) {
    if (KIND == LS_C64) {
      float4 w[U], g[U], m[U]; float2 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint64_t i = ib + (uint64_t)u * LS_THREADS * VL;
        if (i < a1) {
          g[u] = ld_f4(reinterpret_cast<const float*>(e.g) + 2 * i);
          m[u] = ld_f4(e.m + 2 * i);
          w[u] = ld_f4(reinterpret_cast<const float*>(e.w) + 2 * i);
          v[u] = *reinterpret_cast<const float2*>(e.v + i);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint64_t i = ib + (uint64_t)u * LS_THREADS * VL;
        if (i < a1) {
          adamw_complex(w[u].x, w[u].y, g[u].x * c, g[u].y * c, m[u].x, m[u].y, v[u].x, a);
          adamw_complex(w[u].z, w[u].w, g[u].z * c, g[u].w * c, m[u].z, m[u].w, v[u].y, a);
          st_f4(reinterpret_cast<float*>(e.w) + 2 * i, w[u]);
          st_f4(e.m + 2 * i, m[u]);
          *reinterpret_cast<float2*>(e.v + i) = v[u];
        }
      }
    } else {
      constexpr int K = KIND == LS_C64 ? LS_F32 : KIND;
      constexpr int B = K == LS_F32 ? 4 : 2;
      float4 w[U], g[U], m[U], v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint64_t i = ib + (uint64_t)u * LS_THREADS * VL;
        if (i < a1) {
          g[u] = ld_four<K>(e.g + B * i);
          m[u] = ld_f4(e.m + i);
          v[u] = ld_f4(e.v + i);
          w[u] = MASTER ? ld_f4(e.master + i) : ld_four<K>(e.w + B * i);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint64_t i = ib + (uint64_t)u * LS_THREADS * VL;
        if (i < a1) {
          w[u].x = adamw_real(w[u].x, g[u].x * c, m[u].x, v[u].x, a);
          w[u].y = adamw_real(w[u].y, g[u].y * c, m[u].y, v[u].y, a);
          w[u].z = adamw_real(w[u].z, g[u].z * c, m[u].z, v[u].z, a);
          w[u].w = adamw_real(w[u].w, g[u].w * c, m[u].w, v[u].w, a);
          st_f4(e.m + i, m[u]);
          st_f4(e.v + i, v[u]);
          if (MASTER) st_f4(e.master + i, w[u]);
          st_four<K>(e.w + B * i, w[u]);
        }
      }
    }
  }
  for (uint64_t i = i0 + threadIdx.x; i < a0; i += LS_THREADS) adamw_one<KIND>(e, i, c, a);
  for (uint64_t i = a1 + threadIdx.x; i < i1; i += LS_THREADS) adamw_one<KIND>(e, i, c, a);
}

// All tensors of one launch have the same storage, so that each has its own registers and no branch in the loop.
template <int KIND, bool MASTER, int CAP>
__global__ void __launch_bounds__(LS_THREADS, 4) list_adamw_kernel(const __grid_constant__ AdamwParams<CAP> p, const __grid_constant__ AdamwScalars a) {
  griddep_wait();
  griddep_launch_dependents();
  const float c = a.gscale ? *a.gscale : 1.f;
  uint32_t k = (uint32_t)((uint64_t)blockIdx.x * p.total / gridDim.x);
  const uint32_t k1 = (uint32_t)((uint64_t)(blockIdx.x + 1) * p.total / gridDim.x);
  if (k >= k1) return;
  int lo = 0, hi = p.n;
  while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (p.first[mid] <= k) lo = mid; else hi = mid; }
  int t = lo;
  for (; k < k1; ++k) {
    while (p.first[t + 1] <= k) ++t;
    const AdamwEntry& e = p.e[t];
    const uint64_t n = e.count;
    // chunk boundaries lie `head` past multiples of the chunk length, so that every chunk but the first starts with a vector
    const int head = p.head[t], shift = head == 255 ? 0 : head;
    const uint32_t j = k - p.first[t], last = p.first[t + 1] - p.first[t] - 1;
    const uint64_t i0 = j == 0 ? 0 : ((uint64_t)j << p.epc_log2) + shift;
    uint64_t i1 = j == last ? n : ((uint64_t)(j + 1) << p.epc_log2) + shift;
    if (i1 > n) i1 = n;
    if (i0 < i1) adamw_chunk<KIND, MASTER>(e, i0, i1, head == 255 ? 255 : (j == 0 ? head : 0), c, a);
  }
}

}  // namespace tg
