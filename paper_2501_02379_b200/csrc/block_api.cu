// Host side of the operators of a trained block: argument checks, launch shapes, workspace layout.
#include <cmath>
#include <cstring>

#include "../../include/tgrad.h"
#include "launch.cuh"
#include "norms.cuh"
#include "packed.cuh"
#include "wgrad.cuh"

using namespace tg;

namespace {

#define TG_TRY(expr) do { tgrad_status s_ = (expr); if (s_ != TGRAD_OK) return s_; } while (0)

int sm_count() {
  int dev = 0, sm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sm < 1) return 148;
  return sm;
}
inline bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }
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

int kind_of(int32_t dtype) { return dtype == TGRAD_R32 ? LS_F32 : dtype == TGRAD_R16H ? LS_F16 : dtype == TGRAD_R16B ? LS_BF16 : -1; }
inline int bytes_of(int kind) { return kind == LS_F32 ? 4 : 2; }

// Rows as the kernels take them; al: what divides the address of every row's first entry.
RowsOf rows_of(const tgrad_rows& r, int64_t rows, int kind) {
  const int b = bytes_of(kind);
  RowsOf t;
  t.p = static_cast<char*>(r.d_data); t.ld = rows > 1 ? r.row_stride : 0;
  uint64_t bits = reinterpret_cast<uintptr_t>(t.p) | (uint64_t)(t.ld * b);
  t.al = bits & 1 ? 1 : bits & 2 ? 2 : bits & 4 ? 4 : bits & 8 ? 8 : 16;
  return t;
}
RowsOf vector_of(const void* p, int kind) { tgrad_rows r; r.d_data = const_cast<void*>(p); r.row_stride = 0; return rows_of(r, 1, kind); }
// Whether a matrix's address and stride are none that can be used.  `wanted`: it has to be there.
bool bad_rows(const tgrad_rows& r, int64_t rows, int64_t width, int kind, bool wanted) {
  if (rows == 0) return false;
  if (!r.d_data) return wanted;
  return misaligned(r.d_data, bytes_of(kind)) || (rows > 1 && (r.row_stride < width || r.row_stride >= ((int64_t)1 << 40)));
}

// ---- packed ----
inline int64_t blocks_of(int64_t width) { return (width + 31) / 32; }
inline int64_t exp_stride(int64_t width) { return (blocks_of(width) + 3) / 4 * 4; }
tgrad_status check_shape(int64_t rows, int64_t width) {
  if (rows < 0 || width < 1 || width > ((int64_t)1 << 30) || rows >= ((int64_t)1 << 40)) return TGRAD_ERR_INVALID_ARG;
  if (rows > (((int64_t)1 << 48) - 1) / blocks_of(width)) return TGRAD_ERR_INVALID_ARG;
  return TGRAD_OK;
}
inline bool bad_packed(const void* p, int64_t rows, bool wanted) { return rows > 0 && (p ? misaligned(p, 16) : wanted); }
PackedRows packed_of(const void* p, int64_t rows, int64_t width) {
  PackedRows t;
  t.blocks = (int)blocks_of(width); t.exp_stride = (int)exp_stride(width);
  t.codes = static_cast<unsigned char*>(const_cast<void*>(p)); t.exps = p ? t.codes + rows * 32 * t.blocks : nullptr;
  return t;
}
ItemWalk walk_of(int64_t rows, int64_t width) {
  ItemWalk k;
  k.per_row = (int)(4 * blocks_of(width)); k.items = rows * k.per_row; k.rows = rows; k.width = (int)width;
  uint32_t l = 2;
  while (((int64_t)1 << l) < k.per_row) ++l;
  k.magic = (uint32_t)((((uint64_t)1 << (31 + l)) + k.per_row - 1) / k.per_row); k.shift = l - 1;
  return k;
}
// Entries per thread: several vectors in flight where there is enough work for that.
template <typename... KA, typename... AA>
tgrad_status launch_items(void (*kern)(KA...), int per_thread, const ItemWalk& k, cudaStream_t st, AA&&... args) {
  const int64_t grid = (k.items + PK_THREADS * per_thread - 1) / (PK_THREADS * per_thread);
  if (grid >= ((int64_t)1 << 31)) return TGRAD_ERR_UNSUPPORTED;
  launch_chained(kern, dim3((unsigned)grid), dim3(PK_THREADS), 0, st, static_cast<AA&&>(args)..., k);
  TG_LAUNCH_CHECK();
  return TGRAD_OK;
}
inline bool many(const ItemWalk& k) { return k.items >= (int64_t)148 * 8 * PK_THREADS; }

template <int KIND>
tgrad_status pack_kind(const RowsOf& x, const PackedRows& p, const ItemWalk& k, cudaStream_t st) {
  // (one vector a thread: 16384 x 8192 bf16 88 us, 97 with two, 122 with four; threads to switch between count for more than loads of one thread)
  if (x.al == 16 && k.width % 8 == 0) return launch_items(pack_kernel<KIND, true, 1>, 1, k, st, x, p);
  return launch_items(pack_kernel<KIND, false, 1>, 1, k, st, x, p);
}
template <int KIND>
tgrad_status unpack_kind(const RowsOf& x, const PackedRows& p, const ItemWalk& k, cudaStream_t st) {
  if (x.al == 16 && k.width % 8 == 0) return many(k) ? launch_items(unpack_kernel<KIND, true, 4>, 4, k, st, p, x) : launch_items(unpack_kernel<KIND, true, 1>, 1, k, st, p, x);
  return many(k) ? launch_items(unpack_kernel<KIND, false, 2>, 2, k, st, p, x) : launch_items(unpack_kernel<KIND, false, 1>, 1, k, st, p, x);
}

// ---- gated activation ----
template <int KIND, int ACT, bool GATED>
tgrad_status gated_launch(const GatedArgs& g, const ItemWalk& k, bool aligned, bool backward, cudaStream_t st) {
  if (!backward) return aligned ? launch_items(gated_kernel<KIND, ACT, GATED, true, 1>, 1, k, st, g) : launch_items(gated_kernel<KIND, ACT, GATED, false, 1>, 1, k, st, g);
  return aligned ? launch_items(gated_backward_kernel<KIND, ACT, GATED, true, 1>, 1, k, st, g) : launch_items(gated_backward_kernel<KIND, ACT, GATED, false, 1>, 1, k, st, g);
}
template <int KIND, int ACT>
tgrad_status gated_act(const GatedArgs& g, const ItemWalk& k, bool gated, bool aligned, bool backward, cudaStream_t st) {
  return gated ? gated_launch<KIND, ACT, true>(g, k, aligned, backward, st) : gated_launch<KIND, ACT, false>(g, k, aligned, backward, st);
}
template <int KIND>
tgrad_status gated_kind(int act, const GatedArgs& g, const ItemWalk& k, bool gated, bool aligned, bool backward, cudaStream_t st) {
  return act == TGRAD_ACT_SILU ? gated_act<KIND, ACT_SILU>(g, k, gated, aligned, backward, st)
         : act == TGRAD_ACT_GELU ? gated_act<KIND, ACT_GELU>(g, k, gated, aligned, backward, st) : gated_act<KIND, ACT_GELU_TANH>(g, k, gated, aligned, backward, st);
}
tgrad_status gated_impl(const tgrad_gated_args* c, bool backward, cudaStream_t st) {
  if (!c) return TGRAD_ERR_INVALID_ARG;
  const int kind = kind_of(c->dtype);
  if (kind < 0 || c->act < TGRAD_ACT_SILU || c->act > TGRAD_ACT_GELU_TANH) return TGRAD_ERR_INVALID_ARG;
  TG_TRY(check_shape(c->rows, c->width));
  const bool gated = backward ? c->d_packed_u != nullptr : c->u.d_data != nullptr;
  if (bad_rows(c->a, c->rows, c->width, kind, true) || bad_rows(c->u, c->rows, c->width, kind, gated) || bad_rows(c->y, c->rows, c->width, kind, true)) return TGRAD_ERR_INVALID_ARG;
  if (bad_packed(c->d_packed_a, c->rows, backward) || bad_packed(c->d_packed_u, c->rows, gated && c->d_packed_a) || bad_packed(c->d_packed_y, c->rows, false)) return TGRAD_ERR_INVALID_ARG;
  if (!gated && (c->u.d_data || c->d_packed_u)) return TGRAD_ERR_INVALID_ARG;
  if (!backward && ((c->d_packed_u && !c->d_packed_a) || c->d_packed_y)) return TGRAD_ERR_INVALID_ARG;
  if (c->rows == 0) return TGRAD_OK;
  GatedArgs g; memset(&g, 0, sizeof(g));
  const RowsOf a = rows_of(c->a, c->rows, kind), u = rows_of(c->u, c->rows, kind), y = rows_of(c->y, c->rows, kind);
  if (backward) { g.da = a; g.du = u; g.dy = y; } else { g.a = a; g.u = u; g.y = y; }
  g.pa = packed_of(c->d_packed_a, c->rows, c->width); g.pu = packed_of(c->d_packed_u, c->rows, c->width); g.py = packed_of(c->d_packed_y, c->rows, c->width);
  const ItemWalk k = walk_of(c->rows, c->width);
  const bool aligned = a.al == 16 && y.al == 16 && (!gated || u.al == 16) && c->width % 8 == 0;
  return kind == LS_F32 ? gated_kind<LS_F32>(c->act, g, k, gated, aligned, backward, st)
         : kind == LS_F16 ? gated_kind<LS_F16>(c->act, g, k, gated, aligned, backward, st) : gated_kind<LS_BF16>(c->act, g, k, gated, aligned, backward, st);
}

// ---- norms ----
constexpr size_t kNormShared = 224 * 1024;

tgrad_status check_norm(const tgrad_norm_config* c, bool block) {
  if (!c) return TGRAD_ERR_INVALID_ARG;
  const int kind = kind_of(c->dtype), pk = kind_of(c->param_dtype);
  if (kind < 0 || (pk != LS_F32 && pk != kind) || c->rows < 0 || c->width < 1) return TGRAD_ERR_INVALID_ARG;
  if (c->width > 16384 || c->rows >= ((int64_t)1 << 31)) return TGRAD_ERR_UNSUPPORTED;
  if (!std::isfinite(c->scale) || !(c->eps >= 0.f) || !std::isfinite(c->eps) || c->groups < 0) return TGRAD_ERR_INVALID_ARG;
  if (!c->layer && (c->d_bias || c->d_post_bias)) return TGRAD_ERR_INVALID_ARG;
  if ((!block || !c->post) && (c->d_post_weight || c->d_post_bias)) return TGRAD_ERR_INVALID_ARG;
  if (!block && c->groups) return TGRAD_ERR_INVALID_ARG;
  const int b = bytes_of(pk);
  if (misaligned(c->d_weight, b) || misaligned(c->d_bias, b) || misaligned(c->d_post_weight, b) || misaligned(c->d_post_bias, b)) return TGRAD_ERR_INVALID_ARG;
  if (c->groups) {
    if (!c->gate.d_data || bad_rows(c->gate, c->groups, c->width, pk, true)) return TGRAD_ERR_INVALID_ARG;
    if (!c->d_starts && c->rows % c->groups != 0) return TGRAD_ERR_INVALID_ARG;
    if (misaligned(c->d_starts, 4)) return TGRAD_ERR_INVALID_ARG;
  } else if (c->d_starts || c->gate.d_data) return TGRAD_ERR_INVALID_ARG;
  return TGRAD_OK;
}

ResNormArgs norm_args(const tgrad_norm_config* c, bool block) {
  ResNormArgs a; memset(&a, 0, sizeof(a));
  const int pk = kind_of(c->param_dtype);
  a.rows = c->rows; a.width = (int)c->width; a.blocks = (int)blocks_of(c->width); a.pf32 = pk == LS_F32;
  a.mode = !block ? NM_NONE : c->post ? NM_POST : NM_PLAIN;
  a.w = vector_of(c->d_weight, pk); a.b = vector_of(c->d_bias, pk); a.pw = vector_of(c->d_post_weight, pk); a.pb = vector_of(c->d_post_bias, pk);
  a.gate = rows_of(c->gate, c->groups, pk); a.starts = c->d_starts;
  a.groups = c->groups ? c->groups : 1;
  a.rows_per = c->groups && c->rows >= c->groups ? c->rows / c->groups : 1;
  a.gate_rows = c->groups > 1 && !c->d_starts && c->groups == c->rows;
  a.scale = c->scale; a.eps = c->eps;
  return a;
}

struct NormPlan { int V, tpr, teams, shared_params, stages, grid, combine; int64_t chunk, slots; size_t smem; };
// Threads on a row, row groups of a block, rows fetched ahead.  tensors: matrices that a row is read from.
NormPlan norm_plan(const tgrad_norm_config* c, int tensors, bool backward, int sm) {
  NormPlan p;
  const int kind = kind_of(c->dtype), nv = (int)(4 * blocks_of(c->width)), most = backward ? 512 : 1024;
  // One vector of 8 entries a thread where there are few rows (all of a block's warps on one), two where rows keep every SM busy; four where
  // a row is too long for that.
  p.V = nv <= 32 || (c->rows <= sm && nv <= most) ? 1 : nv <= 2 * most ? 2 : 4;
  p.tpr = (nv + 32 * p.V - 1) / (32 * p.V) * 32;
  p.teams = most / p.tpr;
  if (p.tpr > 32 && p.teams > 15) p.teams = 15;      // one named barrier each
  const int64_t fair = (c->rows + sm - 1) / sm;
  if (p.teams > fair) p.teams = (int)(fair < 1 ? 1 : fair);
  const bool single = !c->d_starts && (c->groups <= 1 || c->groups == c->rows);
  p.combine = backward && single;
  const int64_t all = (int64_t)sm * p.teams;
  p.chunk = (c->rows + all - 1) / all;
  if (p.chunk > 256) p.chunk = 256;                  // longer sums in fp32 would lose more than 1e-6
  if (p.chunk < 1) p.chunk = 1;
  int64_t groups = (c->rows + p.chunk - 1) / p.chunk;
  int64_t grid = backward ? (groups + p.teams - 1) / p.teams : (fair + p.teams - 1) / p.teams * sm;
  if (!backward) { const int64_t need = (c->rows + p.teams - 1) / p.teams; grid = need < sm ? need : sm; }
  p.grid = (int)(grid < 1 ? 1 : grid);
  p.slots = p.combine ? p.grid : (int64_t)p.grid * p.teams;
  const size_t stage = (size_t)tensors * p.V * (kind == LS_F32 ? 2 : 1) * p.tpr * p.teams * 16, params = (size_t)64 * nv;
  const int ahead = backward ? 3 : NM_MAX_STAGES;
  const int64_t each = backward ? p.chunk : (c->rows + (int64_t)p.grid * p.teams - 1) / ((int64_t)p.grid * p.teams);
  // weights in shared memory where a block has several rows of them to serve and two rows still fit beside
  p.shared_params = each * p.teams > 2 && kNormShared >= NM_RED_BYTES + params + 2 * stage;
  const size_t room = kNormShared - NM_RED_BYTES - (p.shared_params ? params : 0);
  p.stages = (int)(room / stage);
  if (p.stages > ahead) p.stages = ahead;
  if (p.stages > each) p.stages = (int)each;
  if (!backward && p.stages < 1) p.stages = 1;       // (a row of two matrices always fits)
  size_t ring = (size_t)p.stages * stage;
  const size_t join = p.combine ? (size_t)p.teams * 128 * blocks_of(c->width) : 0;
  if (ring < join) ring = join;
  p.smem = NM_RED_BYTES + (p.shared_params ? params : 0) + ring;
  return p;
}
// Whether the kernels for aligned rows of whole vectors take a call, and with which ring.
bool norm_fast(NormPlan& p, const ResNormArgs& a, int kind, bool backward) {
  if (p.V > 2 || a.width % 8 != 0 || a.gate_rows || a.mode == NM_PLAIN) return false;
  if (backward && (a.mode != NM_POST || !a.dx.p || a.px.codes)) return false;
  const RowsOf* rows[6] = {&a.x, &a.f, &a.dh, &a.dx, &a.out0, &a.out1};
  for (const RowsOf* r : rows)
    if (r->p && r->al != 16) return false;
  const int64_t each = backward ? p.chunk : (a.rows + (int64_t)p.grid * p.teams - 1) / ((int64_t)p.grid * p.teams);
  if (each * p.teams <= 2) return false;             // filling shared memory with the weights would not pay
  const size_t row = (size_t)a.width * bytes_of(kind), fixed = NM_RED_BYTES + NM_BARS + 256 * (size_t)a.blocks;
  const size_t stage = p.teams * (backward ? 3 * row + (a.pf.codes ? 32 * (size_t)a.blocks : row) : (a.mode == NM_NONE ? 1 : 2) * row);
  if (fixed + stage > kNormShared) return false;
  int64_t stages = (int64_t)((kNormShared - fixed) / stage);
  if (stages > NM_MAX_STAGES) stages = NM_MAX_STAGES;
  if (stages > each) stages = each;
  p.stages = (int)stages;
  const size_t join = p.combine ? (size_t)p.teams * 128 * a.blocks : 0, ring = stages * stage;
  p.smem = fixed + (ring < join ? join : ring);
  return p.smem <= kNormShared;
}
template <int KIND, bool LN, int V>
tgrad_status norm_fast_launch(const NormPlan& p, ResNormArgs& a, bool backward, cudaStream_t st) {
  static std::atomic<uint64_t> done[3];
  const int which = !backward ? 0 : a.pf.codes ? 1 : 2;
  void (*kern)(ResNormArgs) = which == 0 ? norm_forward_fast_kernel<KIND, LN, V> : which == 1 ? norm_backward_fast_kernel<KIND, LN, V, true> : norm_backward_fast_kernel<KIND, LN, V, false>;
  TG_TRY(allow_shared(kern, kNormShared, done[which]));
  a.stages = p.stages; a.copies = g_copy_limit.load(std::memory_order_relaxed);
  launch_chained(kern, dim3(p.grid), dim3(p.tpr * p.teams), p.smem, st, a);
  TG_LAUNCH_CHECK();
  return TGRAD_OK;
}
template <int KIND, bool LN, int V>
tgrad_status norm_launch(const NormPlan& p, ResNormArgs& a, bool backward, cudaStream_t st) {
  if constexpr (V <= 2) {
    NormPlan fast = p;
    if (norm_fast(fast, a, KIND, backward)) return norm_fast_launch<KIND, LN, V>(fast, a, backward, st);
  }
  if (backward) {
    static std::atomic<uint64_t> done{0};
    TG_TRY(allow_shared(norm_backward_kernel<KIND, LN, V>, kNormShared, done));
    launch_chained(norm_backward_kernel<KIND, LN, V>, dim3(p.grid), dim3(p.tpr * p.teams), p.smem, st, a);
  } else if constexpr (V < 4) {
    static std::atomic<uint64_t> done{0};
    TG_TRY(allow_shared(norm_forward_kernel<KIND, LN, V>, kNormShared, done));
    launch_chained(norm_forward_kernel<KIND, LN, V>, dim3(p.grid), dim3(p.tpr * p.teams), p.smem, st, a);
  }
  TG_LAUNCH_CHECK();
  return TGRAD_OK;
}
template <int KIND, bool LN>
tgrad_status norm_vectors(const NormPlan& p, ResNormArgs& a, bool backward, cudaStream_t st) {
  return p.V == 1 ? norm_launch<KIND, LN, 1>(p, a, backward, st) : p.V == 2 ? norm_launch<KIND, LN, 2>(p, a, backward, st) : norm_launch<KIND, LN, 4>(p, a, backward, st);
}
tgrad_status norm_kind(int kind, bool layer, const NormPlan& p, ResNormArgs& a, bool backward, cudaStream_t st) {
  a.tpr = p.tpr; a.stages = p.stages; a.shared_params = p.shared_params; a.chunk = p.chunk; a.combine = p.combine;
  a.part_stride = 32 * (int64_t)a.blocks;
  if (layer) return kind == LS_F32 ? norm_vectors<LS_F32, true>(p, a, backward, st) : kind == LS_F16 ? norm_vectors<LS_F16, true>(p, a, backward, st) : norm_vectors<LS_BF16, true>(p, a, backward, st);
  return kind == LS_F32 ? norm_vectors<LS_F32, false>(p, a, backward, st) : kind == LS_F16 ? norm_vectors<LS_F16, false>(p, a, backward, st) : norm_vectors<LS_BF16, false>(p, a, backward, st);
}
template <int KIND, bool LN>
tgrad_status sums_launch(const NormSums& s, cudaStream_t st) {
  const unsigned columns = (unsigned)((s.width + 31) / 32);
  const bool groups = s.dpw.p || s.dpb.p || (s.dgate.p && !s.per_row);      // any sum over t is wanted
  const unsigned parts = !groups ? 1u : s.groups < 1024 ? 1u + s.groups : 1024u;
  NormSums a = s;
  if (!groups) a.groups = 0;
  launch_chained(norm_sums_kernel<KIND, LN>, dim3(columns, parts), dim3(32, NF_Y), 0, st, a);
  TG_LAUNCH_CHECK();
  if (groups && s.groups > 1 && (s.dpw.p || s.dpb.p)) {
    launch_chained(norm_groups_kernel<KIND, LN>, dim3(columns), dim3(32, NF_Y), 0, st, a);
    TG_LAUNCH_CHECK();
  }
  return TGRAD_OK;
}
size_t norm_part_bytes(const tgrad_norm_config* c, const NormPlan& p) {
  const bool single = !c->d_starts && (c->groups <= 1 || c->groups == c->rows);
  return align_up((size_t)(2 * p.slots + (single ? 1 : 2 * (int64_t)c->groups)) * (c->layer ? 2 : 1) * 32 * blocks_of(c->width) * 4);
}

// ---- weight gradient ----
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled() {
  static EncodeTiledFn fn = []() -> EncodeTiledFn {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

struct WgradPlan { int terms, tn, tiles_n, tiles_k, whole, splits, clusters; int64_t steps, per_split; bool copy; int64_t ld; size_t parts_bytes, partial_bytes; };
WgradPlan wgrad_plan(const tgrad_weight_grad_args* c, int sm) {
  WgradPlan p;
  const int kind = kind_of(c->dtype);
  p.terms = kind == LS_F32 ? 3 : 1;
  p.copy = kind == LS_F32 || misaligned(c->dy.d_data, 16) || (c->rows > 1 && c->dy.row_stride % 8 != 0);
  p.ld = p.copy ? (c->out + 7) / 8 * 8 : c->rows > 1 ? c->dy.row_stride : (c->out + 7) / 8 * 8;
  p.tn = kind_of(c->out_dtype) == LS_F32 ? 128 : 256;      // columns of x of a tile: the sums of fp32 results have to fit in registers
  p.tiles_n = (int)((c->out + WG_TILE_N - 1) / WG_TILE_N); p.tiles_k = (int)((c->width + p.tn - 1) / p.tn);
  const int tokens = p.tn == 128 ? WgGeom<128>::TOKENS : WgGeom<256>::TOKENS;
  p.steps = (c->rows + tokens - 1) / tokens * p.terms;
  // Whole tiles for all full rounds of the clusters (two SMs each); what is left is split along the tokens, in parts of 512 at least, as many as
  // keep the clusters busy for one round.
  const int64_t tiles = (int64_t)p.tiles_n * p.tiles_k, clusters = sm / 2 < 1 ? 1 : sm / 2;
  int64_t rest = tiles % clusters, splits = rest ? clusters / rest : 1;
  if (splits > p.steps * tokens / 512) splits = p.steps * tokens / 512;
  if (splits < 2) { splits = 1; rest = 0; }
  p.per_split = (p.steps + splits - 1) / splits;
  p.splits = (int)(p.per_split ? (p.steps + p.per_split - 1) / p.per_split : 1);
  if (p.splits < 2) { p.splits = 1; rest = 0; }
  p.whole = (int)(tiles - rest);
  const int64_t units = p.whole + rest * p.splits;
  p.clusters = (int)(units < clusters ? units : clusters);
  p.parts_bytes = p.copy ? align_up((size_t)p.terms * c->rows * p.ld * 2) : 0;
  p.partial_bytes = p.splits > 1 ? align_up((size_t)p.splits * rest * WG_TILE_N * p.tn * 4) : 0;
  return p;
}
template <bool F16, int TN>
tgrad_status wgrad_launch(const WgradPlan& p, const CUtensorMap& map_dy, const CUtensorMap& map_codes, const WgradArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  TG_TRY(allow_shared(wgrad_kernel<F16, TN>, WgGeom<TN>::SMEM, done));
  launch_cluster(wgrad_kernel<F16, TN>, dim3((unsigned)(2 * p.clusters)), dim3(WgGeom<TN>::THREADS), WgGeom<TN>::SMEM, 2, st, map_dy, map_codes, a);
  TG_LAUNCH_CHECK();
  if (p.splits > 1) {
    const int64_t threads = ((int64_t)p.tiles_n * p.tiles_k - p.whole) * WG_TILE_N * (TN / 8);
    launch_chained(wgrad_sum_kernel<TN>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, a);
    TG_LAUNCH_CHECK();
  }
  return TGRAD_OK;
}
tgrad_status check_wgrad(const tgrad_weight_grad_args* c) {
  if (!c) return TGRAD_ERR_INVALID_ARG;
  const int kind = kind_of(c->dtype), to = kind_of(c->out_dtype);
  if (kind < 0 || (to != kind && to != LS_F32) || c->rows < 0 || c->out < 1 || c->width < 1) return TGRAD_ERR_INVALID_ARG;
  if (c->out > ((int64_t)1 << 24) || c->width > ((int64_t)1 << 24) || c->rows >= ((int64_t)1 << 31)) return TGRAD_ERR_UNSUPPORTED;
  if ((c->out + 255) / 256 * ((c->width + 127) / 128) >= ((int64_t)1 << 24)) return TGRAD_ERR_UNSUPPORTED;
  if (bad_rows(c->dy, c->rows, c->out, kind, true) || bad_packed(c->d_packed, c->rows, true)) return TGRAD_ERR_INVALID_ARG;
  if (!c->d_weight.d_data || bad_rows(c->d_weight, c->out, c->width, to, true)) return TGRAD_ERR_INVALID_ARG;
  return TGRAD_OK;
}

}  // namespace

extern "C" {

tgrad_status tgrad_packed_bytes(int64_t rows, int64_t width, size_t* bytes) {
  if (!bytes) return TGRAD_ERR_INVALID_ARG;
  TG_TRY(check_shape(rows, width));
  *bytes = (size_t)rows * (32 * blocks_of(width) + exp_stride(width));
  return TGRAD_OK;
}
tgrad_status tgrad_act_pack(const tgrad_rows* x, int64_t rows, int64_t width, int32_t dtype, void* d_packed, void* cuda_stream) {
  const int kind = kind_of(dtype);
  if (kind < 0 || !x) return TGRAD_ERR_INVALID_ARG;
  TG_TRY(check_shape(rows, width));
  if (bad_rows(*x, rows, width, kind, true) || bad_packed(d_packed, rows, true)) return TGRAD_ERR_INVALID_ARG;
  if (rows == 0) return TGRAD_OK;
  const RowsOf t = rows_of(*x, rows, kind);
  const PackedRows p = packed_of(d_packed, rows, width);
  const ItemWalk k = walk_of(rows, width);
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return kind == LS_F32 ? pack_kind<LS_F32>(t, p, k, st) : kind == LS_F16 ? pack_kind<LS_F16>(t, p, k, st) : pack_kind<LS_BF16>(t, p, k, st);
}
tgrad_status tgrad_act_unpack(const void* d_packed, int64_t rows, int64_t width, int32_t dtype, const tgrad_rows* x, void* cuda_stream) {
  const int kind = kind_of(dtype);
  if (kind < 0 || !x) return TGRAD_ERR_INVALID_ARG;
  TG_TRY(check_shape(rows, width));
  if (bad_rows(*x, rows, width, kind, true) || bad_packed(d_packed, rows, true)) return TGRAD_ERR_INVALID_ARG;
  if (rows == 0) return TGRAD_OK;
  const RowsOf t = rows_of(*x, rows, kind);
  const PackedRows p = packed_of(d_packed, rows, width);
  const ItemWalk k = walk_of(rows, width);
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return kind == LS_F32 ? unpack_kind<LS_F32>(t, p, k, st) : kind == LS_F16 ? unpack_kind<LS_F16>(t, p, k, st) : unpack_kind<LS_BF16>(t, p, k, st);
}

tgrad_status tgrad_gated_act(const tgrad_gated_args* args, void* cuda_stream) { return gated_impl(args, false, static_cast<cudaStream_t>(cuda_stream)); }
tgrad_status tgrad_gated_act_backward(const tgrad_gated_args* args, void* cuda_stream) { return gated_impl(args, true, static_cast<cudaStream_t>(cuda_stream)); }

tgrad_status tgrad_residual_norm(const tgrad_norm_config* c, const tgrad_norm_forward* io, void* cuda_stream) {
  if (!io) return TGRAD_ERR_INVALID_ARG;
  const bool block = io->f.d_data != nullptr;
  TG_TRY(check_norm(c, block || (c && c->rows == 0)));
  const int kind = kind_of(c->dtype);
  if (bad_rows(io->x, c->rows, c->width, kind, true) || bad_rows(io->f, c->rows, c->width, kind, false) || bad_rows(io->out_x, c->rows, c->width, kind, false) ||
      bad_rows(io->out_h, c->rows, c->width, kind, true)) return TGRAD_ERR_INVALID_ARG;
  if (bad_packed(io->d_packed_x, c->rows, false) || bad_packed(io->d_packed_f, c->rows, false) || bad_packed(io->d_packed_h, c->rows, false)) return TGRAD_ERR_INVALID_ARG;
  if ((io->d_packed_f && !block && c->rows > 0) || misaligned(io->d_stats, 4)) return TGRAD_ERR_INVALID_ARG;
  if (c->rows == 0) return TGRAD_OK;
  ResNormArgs a = norm_args(c, block);
  a.x = rows_of(io->x, c->rows, kind); a.f = rows_of(io->f, c->rows, kind);
  a.out0 = rows_of(io->out_x, c->rows, kind); a.out1 = rows_of(io->out_h, c->rows, kind);
  a.px = packed_of(io->d_packed_x, c->rows, c->width); a.pf = packed_of(io->d_packed_f, c->rows, c->width); a.ph = packed_of(io->d_packed_h, c->rows, c->width);
  a.stats = io->d_stats;
  const NormPlan p = norm_plan(c, block ? 2 : 1, false, sm_count());
  return norm_kind(kind, c->layer != 0, p, a, false, static_cast<cudaStream_t>(cuda_stream));
}

tgrad_status tgrad_residual_norm_backward_bytes(const tgrad_norm_config* c, size_t* workspace_bytes) {
  if (!workspace_bytes) return TGRAD_ERR_INVALID_ARG;
  TG_TRY(check_norm(c, true));
  *workspace_bytes = norm_part_bytes(c, norm_plan(c, 4, true, sm_count()));
  return TGRAD_OK;
}
tgrad_status tgrad_residual_norm_backward(const tgrad_norm_config* c, const tgrad_norm_backward* io, void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!io) return TGRAD_ERR_INVALID_ARG;
  const bool block = io->f.d_data != nullptr || io->d_packed_f != nullptr;
  TG_TRY(check_norm(c, block || (c && c->rows == 0)));
  const int kind = kind_of(c->dtype), pk = kind_of(c->param_dtype);
  if (bad_rows(io->grad_h, c->rows, c->width, kind, true) || bad_rows(io->grad_x, c->rows, c->width, kind, false) ||
      bad_rows(io->x, c->rows, c->width, kind, !io->d_packed_x) || bad_rows(io->f, c->rows, c->width, kind, false) ||
      bad_rows(io->dx, c->rows, c->width, kind, true) || bad_rows(io->df, c->rows, c->width, kind, block)) return TGRAD_ERR_INVALID_ARG;
  if (bad_packed(io->d_packed_x, c->rows, false) || bad_packed(io->d_packed_f, c->rows, false)) return TGRAD_ERR_INVALID_ARG;
  if ((io->x.d_data && io->d_packed_x) || (io->f.d_data && io->d_packed_f)) return TGRAD_ERR_INVALID_ARG;
  if (c->rows > 0 && (!io->d_stats || misaligned(io->d_stats, 4))) return TGRAD_ERR_INVALID_ARG;
  const int b = bytes_of(pk);
  if (misaligned(io->d_dweight, b) || misaligned(io->d_dbias, b) || misaligned(io->d_dpost_weight, b) || misaligned(io->d_dpost_bias, b)) return TGRAD_ERR_INVALID_ARG;
  if (!c->layer && (io->d_dbias || io->d_dpost_bias)) return TGRAD_ERR_INVALID_ARG;
  if (io->dgate.d_data && (!c->groups || bad_rows(io->dgate, c->groups, c->width, pk, true))) return TGRAD_ERR_INVALID_ARG;
  if ((io->d_dpost_weight || io->d_dpost_bias) && c->rows > 0 && (!block || !c->post)) return TGRAD_ERR_INVALID_ARG;
  if (!d_workspace || misaligned(d_workspace, 256)) return TGRAD_ERR_INVALID_ARG;
  const NormPlan p = norm_plan(c, 2 + (io->grad_x.d_data ? 1 : 0) + (block ? 1 : 0), true, sm_count());
  if (workspace_bytes < norm_part_bytes(c, p)) return TGRAD_ERR_BUFFER_TOO_SMALL;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  ResNormArgs a = norm_args(c, block);
  a.x = rows_of(io->x, c->rows, kind); a.f = rows_of(io->f, c->rows, kind); a.dh = rows_of(io->grad_h, c->rows, kind); a.dx = rows_of(io->grad_x, c->rows, kind);
  a.out0 = rows_of(io->dx, c->rows, kind); a.out1 = rows_of(io->df, c->rows, kind);
  a.px = packed_of(io->d_packed_x, c->rows, c->width); a.pf = packed_of(io->d_packed_f, c->rows, c->width);
  a.stats = const_cast<float*>(io->d_stats);
  a.dgate = rows_of(io->dgate, c->groups, pk);
  const bool sums = io->d_dweight || io->d_dbias || io->d_dpost_weight || io->d_dpost_bias || (io->dgate.d_data && !a.gate_rows);
  a.part = sums ? static_cast<float*>(d_workspace) : nullptr;
  if (c->rows > 0) TG_TRY(norm_kind(kind, c->layer != 0, p, a, true, st));
  if (!sums) return TGRAD_OK;
  NormSums s; memset(&s, 0, sizeof(s));
  s.part = static_cast<float*>(d_workspace); s.slots = c->rows > 0 ? p.slots : 0; s.part_stride = 32 * blocks_of(c->width);
  s.chunk = p.combine ? 0 : p.chunk; s.rows = c->rows; s.rows_per = a.rows_per; s.starts = c->d_starts;
  s.groups = a.gate_rows ? 1 : a.groups; s.width = a.width; s.pf32 = a.pf32; s.per_row = a.gate_rows; s.post = a.mode == NM_POST;
  s.pw = a.pw; s.pb = a.pb; s.gate = a.gate;
  s.dw = vector_of(io->d_dweight, pk); s.db = vector_of(io->d_dbias, pk); s.dpw = vector_of(io->d_dpost_weight, pk); s.dpb = vector_of(io->d_dpost_bias, pk);
  s.dgate = a.dgate;
  if (c->layer) return kind == LS_F32 ? sums_launch<LS_F32, true>(s, st) : kind == LS_F16 ? sums_launch<LS_F16, true>(s, st) : sums_launch<LS_BF16, true>(s, st);
  return kind == LS_F32 ? sums_launch<LS_F32, false>(s, st) : kind == LS_F16 ? sums_launch<LS_F16, false>(s, st) : sums_launch<LS_BF16, false>(s, st);
}

tgrad_status tgrad_weight_grad_bytes(const tgrad_weight_grad_args* c, size_t* workspace_bytes) {
  if (!workspace_bytes) return TGRAD_ERR_INVALID_ARG;
  TG_TRY(check_wgrad(c));
  const WgradPlan p = wgrad_plan(c, sm_count());
  *workspace_bytes = p.parts_bytes + p.partial_bytes;
  return TGRAD_OK;
}
tgrad_status tgrad_weight_grad(const tgrad_weight_grad_args* c, void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
  TG_TRY(check_wgrad(c));
  const int sm = sm_count();
  const WgradPlan p = wgrad_plan(c, sm);
  const size_t need = p.parts_bytes + p.partial_bytes;
  if (need > 0 && (!d_workspace || misaligned(d_workspace, 256))) return TGRAD_ERR_INVALID_ARG;
  if (workspace_bytes < need) return TGRAD_ERR_BUFFER_TOO_SMALL;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int kind = kind_of(c->dtype), to = kind_of(c->out_dtype);
  WgradArgs a; memset(&a, 0, sizeof(a));
  a.tokens = c->rows; a.terms = p.terms; a.N = (int)c->out; a.K = (int)c->width; a.tiles_n = p.tiles_n; a.tiles_k = p.tiles_k;
  a.out = rows_of(c->d_weight, c->out, to); a.out_kind = to; a.accumulate = c->accumulate != 0;
  if (c->rows == 0) {      // nothing to add: zeros, or what is there
    if (c->accumulate) return TGRAD_OK;
    const size_t row = (size_t)c->width * bytes_of(to);
    return cudaMemset2DAsync(c->d_weight.d_data, c->out > 1 ? (size_t)c->d_weight.row_stride * bytes_of(to) : row, 0, row, (size_t)c->out, st) == cudaSuccess ? TGRAD_OK : TGRAD_ERR_CUDA;
  }
  EncodeTiledFn enc = encode_tiled();
  if (!enc) return TGRAD_ERR_CUDA;
  const void* dy = c->dy.d_data;
  if (p.copy) {
    const RowsOf r = rows_of(c->dy, c->rows, kind);
    const int64_t grid = (c->rows * (p.ld / 8) + 255) / 256;
    if (grid >= ((int64_t)1 << 31)) return TGRAD_ERR_UNSUPPORTED;
    uint16_t* parts = static_cast<uint16_t*>(d_workspace);
    if (kind == LS_F32) launch_chained(wgrad_parts_kernel<LS_F32>, dim3((unsigned)grid), dim3(256), 0, st, r, c->rows, a.N, (int)p.ld, parts);
    else if (kind == LS_F16) launch_chained(wgrad_parts_kernel<LS_F16>, dim3((unsigned)grid), dim3(256), 0, st, r, c->rows, a.N, (int)p.ld, parts);
    else launch_chained(wgrad_parts_kernel<LS_BF16>, dim3((unsigned)grid), dim3(256), 0, st, r, c->rows, a.N, (int)p.ld, parts);
    TG_LAUNCH_CHECK();
    dy = parts;
  }
  const PackedRows x = packed_of(c->d_packed, c->rows, c->width);
  a.exps = x.exps; a.exp_words = x.exp_stride / 4;
  a.whole = p.whole; a.splits = p.splits; a.steps = p.steps; a.per_split = p.per_split;
  // fp32 results leave tensor memory after every 32 instructions (4 steps of 128 tokens; 16 where the entries are fp32), 16-bit ones once
  a.group = kind == LS_F32 ? 2 : to == LS_F32 ? 4 : 0x7fffffff;
  a.copies = g_copy_limit.load(std::memory_order_relaxed);
  a.partial = p.splits > 1 ? reinterpret_cast<float*>(static_cast<char*>(d_workspace) + p.parts_bytes) : nullptr;
  const bool f16 = kind == LS_F16;
  CUtensorMap map_dy, map_codes;
  const cuuint32_t one[3] = {1, 1, 1}, tokens = p.tn == 128 ? WgGeom<128>::TOKENS : WgGeom<256>::TOKENS;
  {
    const cuuint64_t dims[3] = {(cuuint64_t)(p.copy ? p.ld : c->out), (cuuint64_t)c->rows, (cuuint64_t)p.terms};
    const cuuint64_t strides[2] = {(cuuint64_t)p.ld * 2, (cuuint64_t)p.ld * 2 * c->rows};
    const cuuint32_t box[3] = {64, tokens, 1};
    if (enc(&map_dy, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(dy), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) return TGRAD_ERR_CUDA;
  }
  {
    const cuuint64_t dims[3] = {(cuuint64_t)(32 * x.blocks), (cuuint64_t)c->rows, 1};
    const cuuint64_t strides[2] = {(cuuint64_t)(32 * x.blocks), (cuuint64_t)(32 * x.blocks) * c->rows};
    const cuuint32_t box[3] = {(cuuint32_t)p.tn / 2, tokens, 1};
    if (enc(&map_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, x.codes, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) return TGRAD_ERR_CUDA;
  }
  if (f16) TG_TRY(to == LS_F32 ? (wgrad_launch<true, 128>(p, map_dy, map_codes, a, st)) : (wgrad_launch<true, 256>(p, map_dy, map_codes, a, st)));
  else TG_TRY(to == LS_F32 ? (wgrad_launch<false, 128>(p, map_dy, map_codes, a, st)) : (wgrad_launch<false, 256>(p, map_dy, map_codes, a, st)));
  return TGRAD_OK;
}

}  // extern "C"
