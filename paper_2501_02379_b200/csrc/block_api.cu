// Host side of packing, the gated activation and the weight gradient: argument checks, launch shapes, workspace layout.
#include "block_host.cuh"
#include "wgrad.cuh"

using namespace tg;

namespace {

ItemWalk walk_of(int64_t rows, int64_t width) {
  ItemWalk k;
  k.per_row = (int)(4 * blocks_of(width)); k.items = rows * k.per_row; k.width = (int)width;
  uint32_t l = 2;
  while (((int64_t)1 << l) < k.per_row) ++l;
  k.magic = (uint32_t)((((uint64_t)1 << (31 + l)) + k.per_row - 1) / k.per_row); k.shift = l - 1;
  return k;
}
template <typename... KA, typename... AA>
tgrad_status launch_items(void (*kern)(KA...), int per_thread, const ItemWalk& k, cudaStream_t st, AA&&... args) {      // per_thread: vectors
  const int64_t grid = (k.items + PK_THREADS * per_thread - 1) / (PK_THREADS * per_thread);
  if (grid >= ((int64_t)1 << 31)) return TGRAD_ERR_UNSUPPORTED;
  launch_chained(kern, dim3((unsigned)grid), dim3(PK_THREADS), 0, st, static_cast<AA&&>(args)..., k);
  TG_LAUNCH_CHECK();
  return TGRAD_OK;
}
// Reading back: several vectors a thread in flight where every SM has its threads all the same.
inline bool many(const ItemWalk& k) { return k.items >= (int64_t)sm_count() * 8 * PK_THREADS; }

template <int KIND>
tgrad_status pack_kind(const RowsOf& x, const PackedRows& p, const ItemWalk& k, cudaStream_t st) {
  if (x.al == 16 && k.width % 8 == 0) return launch_items(pack_kernel<KIND, true>, 1, k, st, x, p);
  return launch_items(pack_kernel<KIND, false>, 1, k, st, x, p);
}
template <int KIND>
tgrad_status unpack_kind(const RowsOf& x, const PackedRows& p, const ItemWalk& k, cudaStream_t st) {
  if (x.al == 16 && k.width % 8 == 0) return many(k) ? launch_items(unpack_kernel<KIND, true, 4>, 4, k, st, p, x) : launch_items(unpack_kernel<KIND, true, 1>, 1, k, st, p, x);
  return many(k) ? launch_items(unpack_kernel<KIND, false, 2>, 2, k, st, p, x) : launch_items(unpack_kernel<KIND, false, 1>, 1, k, st, p, x);
}

// ---- gated activation ----
template <int KIND, int ACT, bool GATED>
tgrad_status gated_launch(const GatedArgs& g, const ItemWalk& k, bool aligned, bool backward, cudaStream_t st) {
  if (!backward) return aligned ? launch_items(gated_kernel<KIND, ACT, GATED, true>, 1, k, st, g) : launch_items(gated_kernel<KIND, ACT, GATED, false>, 1, k, st, g);
  return aligned ? launch_items(gated_backward_kernel<KIND, ACT, GATED, true>, 1, k, st, g) : launch_items(gated_backward_kernel<KIND, ACT, GATED, false>, 1, k, st, g);
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
template <bool F16, int TN, bool RUNNING>
tgrad_status wgrad_product(const WgradPlan& p, const CUtensorMap& map_dy, const CUtensorMap& map_codes, const WgradArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  TG_TRY(allow_shared(wgrad_kernel<F16, TN, RUNNING>, WgGeom<TN>::SMEM, done));
  launch_cluster(wgrad_kernel<F16, TN, RUNNING>, dim3((unsigned)(2 * p.clusters)), dim3(WgGeom<TN>::THREADS), WgGeom<TN>::SMEM, 2, st, map_dy, map_codes, a);
  TG_LAUNCH_CHECK();
  return TGRAD_OK;
}
template <bool F16, int TN>
tgrad_status wgrad_launch(const WgradPlan& p, const CUtensorMap& map_dy, const CUtensorMap& map_codes, const WgradArgs& a, cudaStream_t st) {
  // running sums where some unit has more steps than a group
  if (TN == 256 && (p.whole > 0 ? p.steps : p.per_split) > a.group) TG_TRY((wgrad_product<F16, TN, TN == 256>(p, map_dy, map_codes, a, st)));
  else TG_TRY((wgrad_product<F16, TN, false>(p, map_dy, map_codes, a, st)));
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
  // Instructions of 16 tokens whose sums the tensor core forms, cutting off at most 2^-22 at each: 32 for fp32 results (4 steps of 128 tokens; 16
  // where the entries are fp32), 256 for 16-bit ones (64 steps of 64), an eighth of half an ulp of fp16.
  a.group = kind == LS_F32 ? 2 : p.tn == 128 ? 4 : 64;
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
