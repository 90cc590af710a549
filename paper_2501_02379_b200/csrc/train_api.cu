// Host side of the operators around the optimizer step: argument checks, launch shapes, workspace layout.
#include <cmath>
#include <cstring>

#include "../../include/tgrad.h"
#include "launch.cuh"
#include "lists.cuh"
#include "tokens.cuh"

using namespace tg;

namespace tg { std::atomic<int> g_copy_limit{kNoCopyLimit}; }

namespace {

#define TG_TRY(expr) do { tgrad_status s_ = (expr); if (s_ != TGRAD_OK) return s_; } while (0)

int sm_count() {
  int dev = 0, sm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sm < 1) return 148;
  return sm;
}
inline bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

// ---- lists ----
constexpr int kListSmall = 192, kListLarge = 1024;       // tensors per launch: 3.9 KB and 20 KB of kernel parameters
constexpr int kAdamwSmall = 64, kAdamwLarge = 512;       // 3.4 KB and 27 KB
constexpr uint32_t kMaxListBlocks = 2048;

// storage kind and reals per entry; false for a type that the lists do not take
bool list_type(int32_t dtype, int& kind, int& reals) {
  switch (dtype) {
    case TGRAD_C64: kind = LS_F32; reals = 2; return true;
    case TGRAD_C32H: kind = LS_F16; reals = 2; return true;
    case TGRAD_C32B: kind = LS_BF16; reals = 2; return true;
    case TGRAD_R32: kind = LS_F32; reals = 1; return true;
    case TGRAD_R16H: kind = LS_F16; reals = 1; return true;
    case TGRAD_R16B: kind = LS_BF16; reals = 1; return true;
  }
  return false;
}

tgrad_status check_list(const tgrad_tensor* list, int32_t n) {
  if (n < 0 || (n > 0 && !list)) return TGRAD_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    int kind, reals;
    if (!list_type(list[i].dtype, kind, reals)) return TGRAD_ERR_INVALID_ARG;
    if (list[i].numel < 0 || list[i].numel >= ((int64_t)1 << 48)) return TGRAD_ERR_INVALID_ARG;
    if (list[i].numel > 0 && (!list[i].d_data || misaligned(list[i].d_data, kind == LS_F32 ? 4 : 2))) return TGRAD_ERR_INVALID_ARG;
  }
  return TGRAD_OK;
}

size_t norm_bytes(int32_t n) {
  const int per = n < kListLarge ? n : kListLarge;
  return align_up((size_t)(kMaxListBlocks + per) * 8) + align_up((size_t)(n / kListLarge + 1) * 8);
}

// Fills the parameters for tensors [0, n) of `list`; returns the number of blocks (0: nothing in the list).
template <int CAP>
uint32_t fill_list(const tgrad_tensor* list, int n, int sm, ListParams<CAP>& p) {
  p.n = n;
  uint64_t granules = 0;
  for (int i = 0; i < n; ++i) {
    int kind = 0, reals = 1;
    list_type(list[i].dtype, kind, reals);
    p.e[i].ptr = static_cast<char*>(list[i].d_data);
    p.e[i].count = (uint64_t)list[i].numel * reals | ((uint64_t)kind << 62);
    granules += list_granules(p.e[i]);
  }
  // Chunks of 32 KB (eight 16-byte loads per thread in flight), down to 4 KB where there would be too few to give
  // every SM several blocks.
  uint32_t lg = 11;
  while (lg > 8 && (granules >> lg) < (uint64_t)sm * 8) --lg;
  while ((granules >> lg) > ((uint64_t)1 << 31)) ++lg;
  p.gpc_log2 = lg;
  uint64_t at = 0;
  for (int i = 0; i < n; ++i) {
    p.first[i] = (uint32_t)at;
    at += (list_granules(p.e[i]) + (1ull << lg) - 1) >> lg;
  }
  p.first[n] = p.total = (uint32_t)at;
  uint64_t grid = (uint64_t)sm * 4;
  if (grid > at) grid = at;
  return (uint32_t)(grid > kMaxListBlocks ? kMaxListBlocks : grid);
}

inline uint32_t norm_blocks(int n) { return (uint32_t)(n + LS_THREADS / 32 - 1) / (LS_THREADS / 32); }
// Blocks of the scaling pass: about six chunks for each, so that the hardware hands them out as SMs become free (973 MB:
// 464 us, 492 us with four blocks per SM), but no more than fill the GPU once where that is less, since each adds up the
// partial sums for itself (80 MB in 145 tensors: 25 us, 36 us with one chunk for each block).
inline uint32_t scale_blocks(uint32_t chunks, int sm) {
  const uint32_t few = (uint32_t)sm * 4, most = (uint32_t)sm * 32, want = chunks / 6;
  const uint32_t blocks = want < few ? few : (want > most ? most : want);
  return blocks < chunks ? blocks : chunks;
}
template <int CAP>
tgrad_status norm_slices(const tgrad_tensor* list, int32_t n, float max_norm, float* out, void* ws, bool clip, cudaStream_t st) {
  const int sm = sm_count(), per = n < kListLarge ? n : kListLarge;
  ListParams<CAP> p;
  NormArgs a;
  a.partial = static_cast<double*>(ws);
  a.slice_sum = reinterpret_cast<double*>(static_cast<char*>(ws) + align_up((size_t)(kMaxListBlocks + per) * 8));
  a.max_norm = max_norm; a.out = out;
  const bool one = n <= CAP;
  for (int base = 0, slice = 0; slice == 0 || base < n; base += CAP, ++slice) {
    const int cnt = n - base < CAP ? n - base : CAP;
    a.grid = fill_list<CAP>(list + base, cnt, sm, p);
    a.base = base; a.slice = slice; a.last = base + CAP >= n ? 1 : 0;
    if (a.grid > 0) {
      launch_chained(list_sumsq_kernel<CAP>, dim3(a.grid), dim3(LS_THREADS), 0, st, p, static_cast<double*>(ws));
      TG_LAUNCH_CHECK();
    }
    if (one && clip && a.grid > 0) {
      launch_chained(list_scale_kernel<CAP, true>, dim3(scale_blocks(p.total, sm) + norm_blocks(cnt)), dim3(LS_THREADS), 0, st, p, a);
      TG_LAUNCH_CHECK();
      return TGRAD_OK;
    }
    launch_chained(list_norm_kernel<CAP>, dim3(cnt ? norm_blocks(cnt) : 1), dim3(LS_THREADS), 0, st, p, a);
    TG_LAUNCH_CHECK();
  }
  if (!clip || one) return TGRAD_OK;
  for (int base = (n - 1) / CAP * CAP; base >= 0; base -= CAP) {
    const int cnt = n - base < CAP ? n - base : CAP;
    if (fill_list<CAP>(list + base, cnt, sm, p) == 0) continue;
    launch_chained(list_scale_kernel<CAP, false>, dim3(scale_blocks(p.total, sm)), dim3(LS_THREADS), 0, st, p, a);
    TG_LAUNCH_CHECK();
  }
  return TGRAD_OK;
}

tgrad_status norm_impl(const tgrad_tensor* grads, int32_t n, float max_norm, float* d_out, void* ws, size_t ws_bytes, bool clip, cudaStream_t st) {
  TG_TRY(check_list(grads, n));
  if (!(max_norm > 0.f) || !d_out || misaligned(d_out, 4) || !ws || misaligned(ws, 256)) return TGRAD_ERR_INVALID_ARG;
  if (ws_bytes < norm_bytes(n)) return TGRAD_ERR_BUFFER_TOO_SMALL;
  return n <= kListSmall ? norm_slices<kListSmall>(grads, n, max_norm, d_out, ws, clip, st) : norm_slices<kListLarge>(grads, n, max_norm, d_out, ws, clip, st);
}

// One launch per storage and CAP tensors.
template <int KIND, bool MASTER, int CAP>
tgrad_status adamw_slices(const tgrad_adamw_tensor* list, int32_t n, const AdamwScalars& a, cudaStream_t st) {
  constexpr int b = KIND == LS_C64 ? 8 : KIND == LS_F32 ? 4 : 2, vl = KIND == LS_C64 ? 2 : 4, mb = KIND == LS_C64 ? 8 : 4;
  const int32_t dtype = KIND == LS_C64 ? TGRAD_C64 : KIND == LS_F32 ? TGRAD_R32 : KIND == LS_F16 ? TGRAD_R16H : TGRAD_R16B;
  const int sm = sm_count();
  for (int i = 0; i < n;) {
    AdamwParams<CAP> p;
    p.n = 0;
    uint64_t entries = 0;
    for (; i < n && p.n < CAP; ++i) {
      const tgrad_adamw_tensor& t = list[i];
      if (t.dtype != dtype || (t.d_master != nullptr) != MASTER || t.numel == 0) continue;
      AdamwEntry& e = p.e[p.n];
      e.w = static_cast<char*>(t.d_weight); e.g = static_cast<const char*>(t.d_grad);
      e.m = static_cast<float*>(t.d_exp_avg); e.v = t.d_exp_avg_sq; e.master = t.d_master;
      e.count = (uint64_t)t.numel;
      p.head[p.n] = 255;
      for (int h = vl - 1; h >= 0; --h)
        if (!misaligned(e.w + h * b, vl * b) && !misaligned(e.g + h * b, vl * b) && !misaligned(reinterpret_cast<char*>(e.m) + h * mb, vl * mb) &&
            !misaligned(e.v + h, vl * 4) && (!MASTER || !misaligned(e.master + h, vl * 4)))
          p.head[p.n] = (uint8_t)h;
      entries += e.count;
      ++p.n;
    }
    if (p.n == 0) continue;
    // chunks of 4096 entries (two vectors of four per thread and turn), fewer where there would be too few of them
    uint32_t lg = 12;
    while (lg > 9 && (entries >> lg) < (uint64_t)sm * 8) --lg;
    while ((entries >> lg) > ((uint64_t)1 << 31)) ++lg;
    p.epc_log2 = lg;
    uint64_t at = 0;
    for (int t = 0; t < p.n; ++t) {
      p.first[t] = (uint32_t)at;
      at += (p.e[t].count + (1ull << lg) - 1) >> lg;
    }
    p.first[p.n] = p.total = (uint32_t)at;
    // many short blocks, handed out as SMs become free (135 M bf16 weights with masters: 594 us, 660 us with 8 per SM)
    uint64_t grid = (uint64_t)sm * 64;
    if (grid > at) grid = at;
    launch_chained(list_adamw_kernel<KIND, MASTER, CAP>, dim3((unsigned)grid), dim3(LS_THREADS), 0, st, p, a);
    TG_LAUNCH_CHECK();
  }
  return TGRAD_OK;
}
template <int KIND, bool MASTER>
tgrad_status adamw_kind(int count, const tgrad_adamw_tensor* list, int32_t n, const AdamwScalars& a, cudaStream_t st) {
  if (count == 0) return TGRAD_OK;
  return count <= kAdamwSmall ? adamw_slices<KIND, MASTER, kAdamwSmall>(list, n, a, st) : adamw_slices<KIND, MASTER, kAdamwLarge>(list, n, a, st);
}

// ---- rows of logits ----
int token_kind(int32_t dtype) { return dtype == TGRAD_R32 ? LS_F32 : dtype == TGRAD_R16H ? LS_F16 : dtype == TGRAD_R16B ? LS_BF16 : -1; }

tgrad_status check_logits(const tgrad_logits* in) {
  if (!in) return TGRAD_ERR_INVALID_ARG;
  const int kind = token_kind(in->dtype);
  if (kind < 0 || in->rows < 0 || in->vocab < 1 || in->vocab > ((int64_t)1 << 30)) return TGRAD_ERR_INVALID_ARG;
  if (in->rows > 1 && in->row_stride < in->vocab) return TGRAD_ERR_INVALID_ARG;
  if (!(in->temperature > 0.0) || !(in->temperature < 1e30) || !(in->temperature > 1e-30)) return TGRAD_ERR_INVALID_ARG;
  if (in->rows > 0 && (!in->d_logits || misaligned(in->d_logits, kind == LS_F32 ? 4 : 2) || !in->d_targets || misaligned(in->d_targets, 8))) return TGRAD_ERR_INVALID_ARG;
  if (in->rows >= ((int64_t)1 << 31) / TK_MAX_CLUSTER) return TGRAD_ERR_UNSUPPORTED;
  return TGRAD_OK;
}
tgrad_status check_dlogits(const tgrad_logits* in, const void* d, int64_t stride) {
  if (in->rows > 0 && (!d || misaligned(d, token_kind(in->dtype) == LS_F32 ? 4 : 2))) return TGRAD_ERR_INVALID_ARG;
  if (in->rows > 1 && stride < in->vocab) return TGRAD_ERR_INVALID_ARG;
  // the gradient may take the logits' place, entry by entry, and must not overlap them in another way
  if (d == in->d_logits && in->rows > 1 && stride != in->row_stride) return TGRAD_ERR_INVALID_ARG;
  return TGRAD_OK;
}
inline bool bad_floats(const void* p, bool wanted) { return wanted ? (!p || misaligned(p, 4)) : misaligned(p, 4); }

TokenArgs token_args(const tgrad_logits* in, void* d_dlogits, int64_t stride) {
  TokenArgs a;
  a.z = static_cast<const char*>(in->d_logits); a.dz = static_cast<char*>(d_dlogits);
  a.ldz = in->row_stride; a.lddz = stride; a.y = reinterpret_cast<const long long*>(in->d_targets); a.V = (int)in->vocab;
  const double inv = 1.0 / in->temperature, k = 1.4426950408889634 / in->temperature;
  a.inv_tau = (float)inv; a.inv_lo = (float)(inv - (double)a.inv_tau);
  a.k = (float)k; a.k_lo = (float)((k - (double)a.k) / k);
  return a;
}
// most granules that a row of these logits touches: rows whose stride is a multiple of 16 bytes all lie alike
inline int64_t max_granules(const tgrad_logits* in) {
  const int kind = token_kind(in->dtype), b = kind == LS_F32 ? 4 : 2, e = 16 / b;
  const int64_t mis = (int64_t)(reinterpret_cast<uintptr_t>(in->d_logits) & 15) / b;
  if (in->rows <= 1 || in->row_stride * b % 16 == 0) return (mis + in->vocab + e - 1) / e;
  return (in->vocab + 2 * (e - 1)) / e;
}

template <bool POLICY>
tgrad_status launch_forward(int kind, const tgrad_logits* in, const TokenArgs& a, const ForwardArgs& f, const PolicyArgs& q, cudaStream_t st) {
  // blocks per row: one while the rows alone fill the GPU, more (of at least one batch of loads each) where they do not
  const int sm = sm_count();
  const int64_t g = max_granules(in);
  int C = 1;
  while (C < TK_MAX_CLUSTER && in->rows * C < (int64_t)4 * sm && g > (int64_t)C * TF_THREADS * 4) C *= 2;
  const dim3 grid((unsigned)(in->rows * C));
  if (kind == LS_F32) launch_cluster(token_forward_kernel<LS_F32, POLICY>, grid, dim3(TF_THREADS), 0, C, st, a, f, q, C);
  else if (kind == LS_F16) launch_cluster(token_forward_kernel<LS_F16, POLICY>, grid, dim3(TF_THREADS), 0, C, st, a, f, q, C);
  else launch_cluster(token_forward_kernel<LS_BF16, POLICY>, grid, dim3(TF_THREADS), 0, C, st, a, f, q, C);
  TG_LAUNCH_CHECK();
  return TGRAD_OK;
}

// The one-pass policy kernel: shared memory of an SM for the rings of its blocks, 16 arithmetic warps for all of them at most.
constexpr size_t kRingBytes = 224 * 1024;
// Dynamic shared memory beyond the default, once per kernel and device.
template <typename F>
tgrad_status allow_shared(F kern, size_t bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return TGRAD_ERR_CUDA;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return TGRAD_OK;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return TGRAD_ERR_CUDA;
  if (dev < 64) done.fetch_or(bit, std::memory_order_release);
  return TGRAD_OK;
}
// Rows that a warp takes alone: short ones where there are enough of them for every SM to have eight warps busy, and always
// those of one batch (the pairs loss on 250 rows of 8191 fp16 logits: 13.3 us with more warps on each row, 18.1 us with one).
bool one_warp_each(const tgrad_logits* in) {
  const int64_t g = max_granules(in);
  return g <= 32 * SR_NV || (g <= SR_MAX_GRANULES && in->rows >= (int64_t)sm_count() * 8);
}
template <int KIND, int MODE>
tgrad_status launch_short(const tgrad_logits* in, const TokenArgs& a, const PolicyArgs& q, const ForwardArgs& f, cudaStream_t st) {
  int64_t grid = (in->rows + SR_WARPS - 1) / SR_WARPS;
  const int64_t most = (int64_t)sm_count() * 8;
  if (grid > most) grid = most;
  launch_chained(token_short_kernel<KIND, MODE>, dim3((unsigned)grid), dim3(32 * SR_WARPS), 0, st, a, q, f, in->rows);
  TG_LAUNCH_CHECK();
  return TGRAD_OK;
}
// Ring of a kernel on rows: `stay`, a row is read twice; else blocks of four warps, `blocks` of them to an SM.
RowGeom row_geom(const tgrad_logits* in, float k, bool stay, int blocks, int64_t* grid) {
  const int sm = sm_count();
  const int64_t G = max_granules(in), bytes = G * 16;
  RowGeom g; memset(&g, 0, sizeof(g));
  // The smallest blocks in whose rings at least half of a row stays: more of them share an SM, and one computes while
  // another waits at its barriers.  Measured with 4 / 8 / 16 warps (4 / 2 / 1 blocks per SM): rows of 16 KB 114 / 147 / - us,
  // 64 KB 203 / 221 / - us, 100 KB 320 / 347 / 426 us, 128 KB 228 / 201 / 219 us, 200 KB 366 / 304 / 322 us, 256 KB 877 / 795 / 678 us.
  // A row for each SM at most: all of an SM's warps on it.
  int per_sm = blocks;
  g.W = 4;
  if (stay && in->rows <= sm) { g.W = RW_MAX_WARPS; per_sm = 1; }
  while (stay && g.W < RW_MAX_WARPS && bytes > 2 * (int64_t)(kRingBytes / per_sm)) { g.W *= 2; per_sm /= 2; }
  const size_t chunk = (size_t)g.W * 32 * RW_NV * 16;
  const int64_t places = (int64_t)((kRingBytes + 2560 - 2560 * per_sm) / per_sm / chunk);      // a block's own shared memory: 2.5 KB
  const int64_t per = (int64_t)g.W * 32 * RW_NV;
  g.K = (int)((G + per - 1) / per); g.last = (int)((g.K - 1) * per);
  g.N = (int)(places > RW_MAX_PLACES ? RW_MAX_PLACES : places);
  g.copies = tg::g_copy_limit.load(std::memory_order_relaxed);
  g.reach = 200.f / k; g.slack = 40.f / k; g.lowest = token_kind(in->dtype) == LS_F16 ? -65000.f : -1e38f;
  // units of about 64 KB of logits, at most a warp's width of rows, and several for every block
  int64_t unit = (64 << 10) / bytes;
  if (unit > 32) unit = 32;
  const int64_t fair = in->rows / ((int64_t)sm * per_sm * 4);
  if (unit > fair) unit = fair;
  g.unit = (int)(unit < 1 ? 1 : unit);
  *grid = (in->rows + g.unit - 1) / g.unit;
  return g;
}
inline size_t ring_bytes(const RowGeom& g) { return (size_t)g.W * 32 * RW_NV * 16 * g.N; }

template <int KIND, int MODE, int W>
tgrad_status launch_row_warps(const RowGeom& g, int64_t grid, const tgrad_logits* in, const TokenArgs& a, const PolicyArgs& q, const ForwardArgs& f, cudaStream_t st) {
  auto kern = token_row_kernel<KIND, MODE, W>;
  static std::atomic<uint64_t> done{0};
  TG_TRY(allow_shared(kern, kRingBytes, done));
  launch_chained(kern, dim3((unsigned)grid), dim3(32 * (W + 1)), ring_bytes(g), st, a, q, f, in->rows, g);
  TG_LAUNCH_CHECK();
  return TGRAD_OK;
}
template <int KIND, int MODE>
tgrad_status launch_row(const tgrad_logits* in, const TokenArgs& a, const PolicyArgs& q, const ForwardArgs& f, cudaStream_t st) {
  if (one_warp_each(in)) return launch_short<KIND, MODE>(in, a, q, f, st);
  int64_t grid;
  const RowGeom g = row_geom(in, a.k, MODE != RW_FORWARD, MODE == RW_FORWARD ? 6 : 4, &grid);
  if constexpr (MODE == RW_FORWARD) {
    return launch_row_warps<KIND, MODE, 4>(g, grid, in, a, q, f, st);
  } else {
    return g.W == 4 ? launch_row_warps<KIND, MODE, 4>(g, grid, in, a, q, f, st)
           : g.W == 8 ? launch_row_warps<KIND, MODE, 8>(g, grid, in, a, q, f, st) : launch_row_warps<KIND, MODE, 16>(g, grid, in, a, q, f, st);
  }
}
template <int KIND, bool ENT>
tgrad_status launch_gradient(const tgrad_logits* in, const TokenArgs& a, const BackwardArgs& b, cudaStream_t st) {
  const int64_t G = max_granules(in);
  if (G <= SR_MAX_GRANULES) {
    const int64_t blocks = (in->rows * G + TB2_THREADS - 1) / TB2_THREADS;
    if (blocks >= ((int64_t)1 << 31)) return TGRAD_ERR_UNSUPPORTED;
    launch_chained(token_backward_short_kernel<KIND, ENT>, dim3((unsigned)blocks), dim3(TB2_THREADS), 0, st, a, b, in->rows, (uint32_t)G);
  } else {
    int64_t grid;
    const RowGeom g = row_geom(in, a.k, false, 4, &grid);
    auto kern = token_gradient_kernel<KIND, ENT, 4>;
    static std::atomic<uint64_t> done{0};
    TG_TRY(allow_shared(kern, kRingBytes, done));
    launch_chained(kern, dim3((unsigned)grid), dim3(32 * 5), ring_bytes(g), st, a, b, in->rows, g);
  }
  TG_LAUNCH_CHECK();
  return TGRAD_OK;
}
template <bool ENT>
tgrad_status launch_backward(int kind, const tgrad_logits* in, const TokenArgs& a, const BackwardArgs& b, cudaStream_t st) {
  return kind == LS_F32 ? launch_gradient<LS_F32, ENT>(in, a, b, st)
         : kind == LS_F16 ? launch_gradient<LS_F16, ENT>(in, a, b, st) : launch_gradient<LS_BF16, ENT>(in, a, b, st);
}
template <int MODE>
tgrad_status launch_row_kind(const tgrad_logits* in, const TokenArgs& a, const PolicyArgs& q, const ForwardArgs& f, cudaStream_t st) {
  const int kind = token_kind(in->dtype);
  return kind == LS_F32 ? launch_row<LS_F32, MODE>(in, a, q, f, st)
         : kind == LS_F16 ? launch_row<LS_F16, MODE>(in, a, q, f, st) : launch_row<LS_BF16, MODE>(in, a, q, f, st);
}
// Log-probabilities: several blocks on each of a few rows, the ring where the rows alone keep every block busy.
tgrad_status launch_logprob(const tgrad_logits* in, const TokenArgs& a, const ForwardArgs& f, cudaStream_t st) {
  PolicyArgs q; memset(&q, 0, sizeof(q));
  if (in->rows >= (int64_t)sm_count() * 8 || one_warp_each(in)) return launch_row_kind<RW_FORWARD>(in, a, q, f, st);
  return launch_forward<false>(token_kind(in->dtype), in, a, f, q, st);
}

size_t policy_bytes(int64_t rows) { return align_up((size_t)rows * 16); }
size_t preference_bytes(int64_t rows, int64_t pairs) { return align_up((size_t)rows * 8) + 2 * align_up((size_t)rows * 4) + align_up((size_t)pairs * 8) + 256; }

}  // namespace

extern "C" {

tgrad_status tgrad_set_copy_limit(int32_t copies) {
  tg::g_copy_limit.store(copies < 0 ? kNoCopyLimit : copies, std::memory_order_relaxed);
  return TGRAD_OK;
}

tgrad_status tgrad_grad_norm_bytes(int32_t n, size_t* workspace_bytes) {
  if (n < 0 || !workspace_bytes) return TGRAD_ERR_INVALID_ARG;
  *workspace_bytes = norm_bytes(n);
  return TGRAD_OK;
}
tgrad_status tgrad_grad_norm(const tgrad_tensor* grads, int32_t n, float max_norm, float* d_out, void* d_workspace,
                             size_t workspace_bytes, void* cuda_stream) {
  return norm_impl(grads, n, max_norm, d_out, d_workspace, workspace_bytes, false, static_cast<cudaStream_t>(cuda_stream));
}
tgrad_status tgrad_clip_grads(const tgrad_tensor* grads, int32_t n, float max_norm, float* d_out, void* d_workspace,
                              size_t workspace_bytes, void* cuda_stream) {
  return norm_impl(grads, n, max_norm, d_out, d_workspace, workspace_bytes, true, static_cast<cudaStream_t>(cuda_stream));
}

tgrad_status tgrad_adamw_step(const tgrad_adamw_tensor* list, int32_t n, const tgrad_adamw_config* c, void* cuda_stream) {
  if (n < 0 || (n > 0 && !list) || !c) return TGRAD_ERR_INVALID_ARG;
  if (!(c->beta1 >= 0.0 && c->beta1 < 1.0) || !(c->beta2 >= 0.0 && c->beta2 < 1.0) || !(c->eps >= 0.0) || c->step < 1 ||
      !std::isfinite(c->lr) || !std::isfinite(c->weight_decay) || misaligned(c->d_grad_scale, 4)) return TGRAD_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const tgrad_adamw_tensor& t = list[i];
    const bool c64 = t.dtype == TGRAD_C64, half = t.dtype == TGRAD_R16H || t.dtype == TGRAD_R16B;
    if (t.dtype == TGRAD_C32H || t.dtype == TGRAD_C32B) return TGRAD_ERR_UNSUPPORTED;
    if (!c64 && !half && t.dtype != TGRAD_R32) return TGRAD_ERR_INVALID_ARG;
    if (t.d_master && !half) return TGRAD_ERR_INVALID_ARG;
    if (t.numel < 0 || t.numel >= ((int64_t)1 << 48)) return TGRAD_ERR_INVALID_ARG;
    if (t.numel == 0) continue;
    const uintptr_t al = half ? 2 : 4;
    if (!t.d_weight || !t.d_grad || !t.d_exp_avg || !t.d_exp_avg_sq) return TGRAD_ERR_INVALID_ARG;
    if (misaligned(t.d_weight, al) || misaligned(t.d_grad, al) || misaligned(t.d_exp_avg, 4) || misaligned(t.d_exp_avg_sq, 4) || misaligned(t.d_master, 4))
      return TGRAD_ERR_INVALID_ARG;
  }
  AdamwScalars a;
  const double c1 = 1.0 - std::pow(c->beta1, (double)c->step), c2 = 1.0 - std::pow(c->beta2, (double)c->step);
  a.beta1 = (float)c->beta1; a.beta2 = (float)c->beta2; a.omb1 = (float)(1.0 - c->beta1); a.omb2 = (float)(1.0 - c->beta2);
  a.step_size = (float)(c->lr / c1); a.inv_sqrt_c2 = (float)(1.0 / std::sqrt(c2));
  a.eps = (float)c->eps; a.keep = (float)(1.0 - c->lr * c->weight_decay);
  a.gscale = c->d_grad_scale;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  int count[6] = {0, 0, 0, 0, 0, 0};
  for (int i = 0; i < n; ++i)
    if (list[i].numel > 0) ++count[list[i].dtype == TGRAD_C64 ? 0 : list[i].dtype == TGRAD_R32 ? 1 : (list[i].dtype == TGRAD_R16H ? 2 : 4) + (list[i].d_master ? 1 : 0)];
  TG_TRY((adamw_kind<LS_C64, false>(count[0], list, n, a, st)));
  TG_TRY((adamw_kind<LS_F32, false>(count[1], list, n, a, st)));
  TG_TRY((adamw_kind<LS_F16, false>(count[2], list, n, a, st)));
  TG_TRY((adamw_kind<LS_F16, true>(count[3], list, n, a, st)));
  TG_TRY((adamw_kind<LS_BF16, false>(count[4], list, n, a, st)));
  return adamw_kind<LS_BF16, true>(count[5], list, n, a, st);
}

tgrad_status tgrad_token_logprob(const tgrad_logits* in, float* d_logp, float* d_lse, float* d_entropy, void* cuda_stream) {
  TG_TRY(check_logits(in));
  if (bad_floats(d_logp, false) || bad_floats(d_lse, false) || bad_floats(d_entropy, false)) return TGRAD_ERR_INVALID_ARG;
  if (in->rows == 0) return TGRAD_OK;
  ForwardArgs f; memset(&f, 0, sizeof(f));
  f.logp = d_logp; f.lse = d_lse; f.entropy = d_entropy;
  return launch_logprob(in, token_args(in, nullptr, 0), f, static_cast<cudaStream_t>(cuda_stream));
}

tgrad_status tgrad_token_logprob_backward(const tgrad_logits* in, const float* d_lse, const float* d_entropy, const float* d_grad_logp,
                                          const float* d_grad_entropy, void* d_dlogits, int64_t dlogits_stride, void* cuda_stream) {
  TG_TRY(check_logits(in));
  TG_TRY(check_dlogits(in, d_dlogits, dlogits_stride));
  const bool any = in->rows > 0;
  if (bad_floats(d_lse, any) || bad_floats(d_grad_logp, any) || bad_floats(d_grad_entropy, false) || bad_floats(d_entropy, any && d_grad_entropy)) return TGRAD_ERR_INVALID_ARG;
  if (!any) return TGRAD_OK;
  BackwardArgs b; memset(&b, 0, sizeof(b));
  b.lse = d_lse; b.entropy = d_entropy; b.g = d_grad_logp; b.h = d_grad_entropy; b.scale = 1.f;
  const TokenArgs a = token_args(in, d_dlogits, dlogits_stride);
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return d_grad_entropy ? launch_backward<true>(token_kind(in->dtype), in, a, b, st) : launch_backward<false>(token_kind(in->dtype), in, a, b, st);
}

tgrad_status tgrad_policy_loss_bytes(int64_t rows, size_t* workspace_bytes) {
  if (rows < 0 || !workspace_bytes) return TGRAD_ERR_INVALID_ARG;
  *workspace_bytes = policy_bytes(rows) + 256;
  return TGRAD_OK;
}
tgrad_status tgrad_policy_loss(const tgrad_logits* in, const tgrad_policy_args* c, void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
  TG_TRY(check_logits(in));
  if (!c) return TGRAD_ERR_INVALID_ARG;
  const bool any = in->rows > 0;
  if (bad_floats(c->d_old_logp, any) || bad_floats(c->d_advantages, any) || bad_floats(c->d_weights, any) || bad_floats(c->d_ref_logp, false) ||
      bad_floats(c->d_stats, true) || bad_floats(c->d_logp, false) || bad_floats(c->d_entropy, false)) return TGRAD_ERR_INVALID_ARG;
  if (c->d_dlogits) TG_TRY(check_dlogits(in, c->d_dlogits, c->dlogits_stride));
  if (!(c->clip_low >= 0.f && c->clip_low <= 1.f) || !(c->clip_high >= 0.f) || !std::isfinite(c->kl_coef) || !std::isfinite(c->entropy_coef) || !std::isfinite(c->grad_scale))
    return TGRAD_ERR_INVALID_ARG;
  if (!d_workspace || misaligned(d_workspace, 256)) return TGRAD_ERR_INVALID_ARG;
  if (workspace_bytes < policy_bytes(in->rows)) return TGRAD_ERR_BUFFER_TOO_SMALL;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* ws = static_cast<char*>(d_workspace);
  PolicyArgs q; memset(&q, 0, sizeof(q));
  q.old_logp = c->d_old_logp; q.ref_logp = c->d_ref_logp; q.adv = c->d_advantages; q.weight = c->d_weights;
  q.low = 1.f - c->clip_low; q.high = 1.f + c->clip_high; q.kl_coef = c->kl_coef; q.ent_coef = c->entropy_coef; q.grad_scale = c->grad_scale;
  q.terms = reinterpret_cast<float4*>(ws);
  if (any) {
    const TokenArgs a = token_args(in, c->d_dlogits, c->dlogits_stride);
    ForwardArgs f; memset(&f, 0, sizeof(f));
    f.logp = c->d_logp; f.entropy = c->d_entropy;
    if (!c->d_dlogits) TG_TRY(launch_forward<true>(token_kind(in->dtype), in, a, f, q, st));
    else if (c->entropy_coef != 0.f) TG_TRY(launch_row_kind<RW_ENTROPY>(in, a, q, f, st));
    else TG_TRY(launch_row_kind<RW_POLICY>(in, a, q, f, st));
  }
  launch_chained(policy_sum_kernel, dim3(1), dim3(1024), 0, st, q.terms, in->rows, c->kl_coef, c->entropy_coef, c->d_stats);
  TG_LAUNCH_CHECK();
  return TGRAD_OK;
}

tgrad_status tgrad_preference_loss_bytes(int64_t rows, int32_t pairs, size_t* workspace_bytes) {
  if (rows < 0 || pairs < 0 || !workspace_bytes) return TGRAD_ERR_INVALID_ARG;
  *workspace_bytes = preference_bytes(rows, pairs) + 256;
  return TGRAD_OK;
}
tgrad_status tgrad_preference_loss(const tgrad_logits* in, const tgrad_preference_args* c, void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
  TG_TRY(check_logits(in));
  if (!c || c->pairs < 0) return TGRAD_ERR_INVALID_ARG;
  const bool any = in->rows > 0;
  if (bad_floats(c->d_ref_logp, any) || bad_floats(c->d_logp, any) || bad_floats(c->d_loss, true) || bad_floats(c->d_rewards, c->pairs > 0) ||
      !c->d_starts || misaligned(c->d_starts, 4)) return TGRAD_ERR_INVALID_ARG;
  if (c->d_dlogits) TG_TRY(check_dlogits(in, c->d_dlogits, c->dlogits_stride));
  if (!std::isfinite(c->beta) || !(c->label_smoothing >= 0.f && c->label_smoothing <= 1.f) || !std::isfinite(c->grad_scale)) return TGRAD_ERR_INVALID_ARG;
  if (!d_workspace || misaligned(d_workspace, 256)) return TGRAD_ERR_INVALID_ARG;
  if (workspace_bytes < preference_bytes(in->rows, c->pairs)) return TGRAD_ERR_BUFFER_TOO_SMALL;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* ws = static_cast<char*>(d_workspace);
  float2* stat = reinterpret_cast<float2*>(ws);
  float* g = reinterpret_cast<float*>(ws + align_up((size_t)in->rows * 8));
  float* logp_lo = reinterpret_cast<float*>(ws + align_up((size_t)in->rows * 8) + align_up((size_t)in->rows * 4));
  double* terms = reinterpret_cast<double*>(ws + align_up((size_t)in->rows * 8) + 2 * align_up((size_t)in->rows * 4));
  unsigned* ticket = reinterpret_cast<unsigned*>(reinterpret_cast<char*>(terms) + align_up((size_t)c->pairs * 8));
  const int kind = token_kind(in->dtype);
  const TokenArgs a = token_args(in, c->d_dlogits, c->dlogits_stride);
  if (any) {
    ForwardArgs f; memset(&f, 0, sizeof(f));
    f.logp = c->d_logp; f.stat = stat; f.logp_lo = logp_lo;
    f.g = c->d_dlogits ? g : nullptr; f.ticket = ticket;
    TG_TRY(launch_logprob(in, a, f, st));
  }
  else if (cudaMemsetAsync(ticket, 0, sizeof(*ticket), st) != cudaSuccess) return TGRAD_ERR_CUDA;
  if (c->pairs > 0) {
    PairArgs p; memset(&p, 0, sizeof(p));
    p.starts = c->d_starts; p.ref = c->d_ref_logp; p.logp = c->d_logp; p.logp_lo = logp_lo; p.y = reinterpret_cast<const long long*>(in->d_targets);
    p.rows = in->rows; p.pairs = c->pairs; p.beta = c->beta; p.smoothing = c->label_smoothing;
    p.g = c->d_dlogits ? g : nullptr; p.rewards = c->d_rewards; p.terms = terms; p.ticket = ticket; p.loss = c->d_loss;
    launch_chained(pair_kernel, dim3((unsigned)c->pairs), dim3(TP_THREADS), 0, st, p);
    TG_LAUNCH_CHECK();
  } else if (cudaMemsetAsync(c->d_loss, 0, sizeof(float), st) != cudaSuccess) return TGRAD_ERR_CUDA;
  if (any && c->d_dlogits) {
    BackwardArgs b; memset(&b, 0, sizeof(b));
    b.stat = stat; b.g = g; b.scale = c->grad_scale;
    TG_TRY(launch_backward<false>(kind, in, a, b, st));
  }
  return TGRAD_OK;
}

}  // extern "C"
