// Host side of the norms around a block: argument checks, launch shapes, workspace layout.
#include "block_host.cuh"
#include "norms.cuh"

using namespace tg;

namespace {

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

}  // namespace

extern "C" {

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

}  // extern "C"
