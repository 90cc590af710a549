// Norms around a block of a model, with the block's gate and the scale of the residual stream, forward and backward.
//
// With n(v) = (v - m) r w + b of a row, r = 1 / sqrt(mean (v - m)^2 + eps), m = mean v (layer norm) or 0 (RMS norm, without b):
//   x' = scale x + gate * n_post(f),    h = n_pre(x').
// Backward, with v^ = (v - m) r and J(d, v^, r) = r (d - v^ mean(d v^) - mean d) (the last term for layer norm only):
//   t = dx' + J(dh w, x'^, r_pre),   dx = scale t,   df = J(gate t w_post, f^, r_post),
//   dw = sum dh x'^,  db = sum dh,  dw_post = sum gate t f^,  db_post = sum gate t,  dgate = sum t (f^ w_post + b_post),
// the sums over the rows that share the parameter.  Rows that share a gate need S1 = sum t f^ and S0 = sum t only: the parameters are
// factors of these, so one pair of sums per column serves dw_post, db_post and dgate.
//
// Bound by memory: every input is read once, every output written once.  A row belongs to `tpr` threads of a block, each holding V vectors
// of 8 entries; the blocks stay, one per SM, and walk over the rows.  What a thread will read it copies itself into places of
// its own in shared memory (cp.async), some rows ahead, so the copies need no barrier and no registers, and the memory is busy
// while a row waits in its reductions.  Column sums stay in registers over all rows of a thread's chunk and are added up in a fixed
// order by a second launch.
// Measured at 16384 x 8192 bf16 at burst clocks: forward 176 us (164 at the copy rate; 204 with f kept in 8 bits, 185), backward 265 us (246) from f in
// storage, 272 us (226) from f in 8 bits.
#pragma once
#include "packed.cuh"

namespace tg {

constexpr int NM_MAX_STAGES = 4;
enum { NM_NONE = 0, NM_PLAIN = 1, NM_POST = 2 };      // no block, a block's output as it is, the same normalised

struct ResNormArgs {
  RowsOf x, f;               // forward: stream and block output; backward: x' and f as kept in storage
  RowsOf dh, dx;             // backward: gradients of h and of x' (p null: none)
  RowsOf out0, out1;         // forward: x' (p null: not wanted) and h; backward: dx and df
  PackedRows px, pf, ph;     // forward: kept copies to write (codes null: not wanted); backward: x' and f given packed (codes null: not)
  RowsOf w, b, pw, gate, pb; // parameters; p null: 1 (weights, gate) or 0 (biases).  gate: a row for each group
  RowsOf dgate;              // backward, a gate for each row: its gradient
  const int* starts;         // groups + 1 first rows, or null: groups of rows_per rows
  int64_t rows, rows_per;
  int groups;
  int gate_rows;             // 1: a gate for each row
  int mode, width, blocks;   // blocks of 32 entries of a row
  int pf32;                  // parameters are fp32 (else of the storage type)
  int shared_params;         // weights (with a single gate row folded in) are held in shared memory
  float scale, eps;
  float* stats;              // [2 or 4][rows]: 1 / deviation of f and x', then their means
  int tpr, stages;
  int copies;                // for tests: rows that a team copies at most
  int64_t chunk;             // backward: rows of a row group
  float* part;               // backward: column sums
  int64_t part_stride;       // floats of a slot's row: 32 blocks
  int combine;               // backward: the row groups of a block are added up first
};

// ---- parameters ----
template <int KIND>
__device__ __forceinline__ void param8(const RowsOf& t, int pf32, int64_t row, int c, int n, float fill, float (&v)[8]) {
  if (!t.p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fill;
  } else if (KIND == LS_F32 || pf32) {
    const float* p = reinterpret_cast<const float*>(t.p) + row * t.ld + c;
    if (n == 8 && t.al == 16) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? __ldg(p + i) : 0.f;
    }
  } else {
    const char* p = t.p + (row * t.ld + c) * 2;
    if (n == 8 && t.al == 16) {
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
      const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { const float2 d = widen2<KIND>(u[i]); v[2 * i] = d.x; v[2 * i + 1] = d.y; }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? ld_real<KIND>(p + 2 * i) : 0.f;
    }
  }
}
template <int KIND>
__device__ __forceinline__ void store_param(const RowsOf& t, int pf32, int64_t row, int c, float v) {
  if (KIND == LS_F32 || pf32) reinterpret_cast<float*>(t.p)[row * t.ld + c] = v;
  else st_real<KIND>(t.p + (row * t.ld + c) * 2, v);
}

// ---- a thread's places in shared memory ----
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async8u(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4u(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void sts32(uint32_t dst, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst), "r"(v) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v; asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory"); return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v; asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory"); return v;
}
__device__ __forceinline__ void bulk_g2s_at(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {      // bulk_g2s to a shared address
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) { uint32_t v; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory"); return v; }

// 8 entries, in planes of 16 bytes per thread (fp32: two of them)
template <int KIND> struct NmPlanes { static constexpr int n = KIND == LS_F32 ? 2 : 1; };
template <int KIND>
__device__ __forceinline__ void fetch8(uint32_t dst, uint32_t plane, const RowsOf& t, int64_t row, int c, int n) {
  constexpr int B = KIND == LS_F32 ? 4 : 2, E = 4 / B;      // entries of a word
  const char* p = t.p + (row * t.ld + c) * B;
  if (n == 8 && t.al == 16) {
#pragma unroll
    for (int i = 0; i < B / 2; ++i) cp_async16(dst + i * plane, p + 16 * i);
  } else {
#pragma unroll
    for (int i = 0; i < 2 * B; ++i) {
      const uint32_t at = dst + (i >> 2) * plane + (i & 3) * 4;
      if (t.al >= 4 && E * i + E <= n) cp_async4u(at, p + 4 * i);
      else {
        uint32_t v = 0;
        if (E == 2) {
          if (2 * i < n) v = *reinterpret_cast<const unsigned short*>(p + 4 * i);
          if (2 * i + 1 < n) v |= (uint32_t)*reinterpret_cast<const unsigned short*>(p + 4 * i + 2) << 16;
        }
        sts32(at, v);
      }
    }
  }
}
template <int KIND>
__device__ __forceinline__ void take8(uint32_t src, uint32_t plane, float (&v)[8]) {
  const uint4 a = lds128(src);
  if (KIND == LS_F32) {
    const uint4 b = lds128(src + plane);
    const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(u[i]);
  } else {
    const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 d = widen2<KIND>(u[i]); v[2 * i] = d.x; v[2 * i + 1] = d.y; }
  }
}
// packed entries: 8 bytes of codes and the word that holds the block's byte
__device__ __forceinline__ void fetch8_packed(uint32_t dst, const PackedRows& t, int64_t row, int v) {
  const unsigned char *codes = t.codes + row * t.blocks * 32, *exps = t.exps + row * t.exp_stride;
  cp_async8u(dst, codes + (uint32_t)v * 8u);
  cp_async4u(dst + 8, exps + (uint32_t)((v >> 2) & ~3));
}
__device__ __forceinline__ void take8_packed(uint32_t src, int v, float (&out)[8]) {
  const uint4 q = lds128(src);
  unpack8(make_uint2(q.x, q.y), (q.z >> (8 * ((v >> 2) & 3))) & 255u, out);
}

// ---- sums over a row ----
struct RowTeam {
  float2* red;               // two buffers of 32
  int warps, warp, lane, id, turn;
  __device__ __forceinline__ void sync() const {
    if (warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(warps * 32) : "memory");
  }
  // sums of a and b (TWO) over the team, the same bits in every thread
  template <bool TWO>
  __device__ __forceinline__ float2 sum(float a, float b) {
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) { a += __shfl_xor_sync(0xffffffffu, a, m); if (TWO) b += __shfl_xor_sync(0xffffffffu, b, m); }
    if (warps == 1) return make_float2(a, b);
    float2* r = red + (turn ^= 32);
    if (lane == 0) { if (TWO) r[warp] = make_float2(a, b); else r[warp].x = a; }
    sync();
    a = lane < warps ? r[lane].x : 0.f;
    if (TWO) b = lane < warps ? r[lane].y : 0.f;
    if (warps > 16) { a += __shfl_xor_sync(0xffffffffu, a, 16); if (TWO) b += __shfl_xor_sync(0xffffffffu, b, 16); }
#pragma unroll
    for (int m = 8; m > 0; m >>= 1) { a += __shfl_xor_sync(0xffffffffu, a, m); if (TWO) b += __shfl_xor_sync(0xffffffffu, b, m); }
    if (warps <= 16) { a = __shfl_sync(0xffffffffu, a, 0); if (TWO) b = __shfl_sync(0xffffffffu, b, 0); }      // (lanes 16 to 31 have summed zeros)
    return make_float2(a, b);
  }
};

// the group that a row belongs to; -1: none
__device__ __forceinline__ int group_of(const ResNormArgs& A, int64_t row) {
  if (A.gate_rows) return (int)row;
  if (!A.starts) return A.groups == 1 ? 0 : (int)(row / A.rows_per);
  int lo = -1, hi = A.groups;            // starts[lo] <= row < starts[hi]
  while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (__ldg(A.starts + mid) <= row) lo = mid; else hi = mid; }
  return lo >= 0 && row < __ldg(A.starts + lo + 1) ? lo : -1;
}

__device__ __forceinline__ void wait_stages(int ahead) {      // all copies but those of the last `ahead` rows have landed
  if (ahead <= 0) cp_async_wait<0>();
  else if (ahead == 1) cp_async_wait<1>();
  else if (ahead == 2) cp_async_wait<2>();
  else cp_async_wait<3>();
}

// weights in shared memory: planes of 4 floats for each half of a vector, w first, then w_post (times the gate where there is one for all rows)
template <int KIND>
__device__ __forceinline__ void fill_params(const ResNormArgs& A, float4* ps) {
  const int nv = 4 * A.blocks;
  for (int v = threadIdx.x; v < nv; v += blockDim.x) {
    const int n = max(0, min(8, A.width - 8 * v));
    float a[8], g[8];
    param8<KIND>(A.w, A.pf32, 0, 8 * v, n, 1.f, a);
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = i < n ? a[i] : 0.f;      // (0 where there is no entry, also without weights)
    ps[v] = make_float4(a[0], a[1], a[2], a[3]); ps[nv + v] = make_float4(a[4], a[5], a[6], a[7]);
    param8<KIND>(A.pw, A.pf32, 0, 8 * v, n, 1.f, a);
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = i < n ? a[i] : 0.f;
    if (A.groups == 1 && !A.starts && !A.gate_rows) {
      param8<KIND>(A.gate, A.pf32, 0, 8 * v, n, 1.f, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] *= g[i];
    }
    ps[2 * nv + v] = make_float4(a[0], a[1], a[2], a[3]); ps[3 * nv + v] = make_float4(a[4], a[5], a[6], a[7]);
  }
}
__device__ __forceinline__ void shared8(const float4* ps, int nv, int which, int v, float (&out)[8]) {
  const float4 a = ps[2 * which * nv + v], b = ps[(2 * which + 1) * nv + v];
  out[0] = a.x; out[1] = a.y; out[2] = a.z; out[3] = a.w; out[4] = b.x; out[5] = b.y; out[6] = b.z; out[7] = b.w;
}

constexpr int NM_RED_BYTES = 32 * 64 * 8;      // 32 teams at most, two buffers of 32 pairs each

// Mean and 1 / deviation of the entries that `take(j, v)` gives.
template <bool LN, int V, typename Take>
__device__ __forceinline__ void row_stats(RowTeam& team, const int (&n)[V], float inv, float eps, Take take, float& mean, float& rstd) {
  mean = 0.f;
  if (LN) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float v[8]; take(j, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];           // (entries that do not exist are 0)
    }
    mean = team.sum<false>(s, 0.f).x * inv;
  }
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    float v[8]; take(j, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) { const float d = LN && i >= n[j] ? 0.f : v[i] - mean; s = fmaf(d, d, s); }
  }
  rstd = rsqrtf(fmaf(team.sum<false>(s, 0.f).x, inv, eps));
}

template <int KIND, bool LN, int V>
__global__ void __launch_bounds__(1024, 1) norm_forward_kernel(const ResNormArgs A) {
  extern __shared__ __align__(16) unsigned char nm_smem[];
  griddep_chain();
  const int nv = 4 * A.blocks, teams = blockDim.x / A.tpr, mine = threadIdx.x / A.tpr, t = threadIdx.x - mine * A.tpr;
  RowTeam team{reinterpret_cast<float2*>(nm_smem) + mine * 64, A.tpr >> 5, t >> 5, (int)(threadIdx.x & 31), mine + 1, 0};
  float4* ps = reinterpret_cast<float4*>(nm_smem + NM_RED_BYTES);
  if (A.shared_params) { fill_params<KIND>(A, ps); __syncthreads(); }
  const uint32_t plane = blockDim.x * 16;
  constexpr int P = NmPlanes<KIND>::n * V;
  const uint32_t base = smem_u32(nm_smem) + NM_RED_BYTES + (A.shared_params ? 64 * nv : 0) + threadIdx.x * 16;
  int at[V], n[V];
#pragma unroll
  for (int j = 0; j < V; ++j) { at[j] = t + j * A.tpr; n[j] = max(0, min(8, A.width - 8 * at[j])); }
  const int64_t first = (int64_t)blockIdx.x * teams + mine, step = (int64_t)gridDim.x * teams;
  const int S = A.stages, per = A.mode == NM_NONE ? 1 : 2;
  auto slot = [&](int s, int tensor, int j) { return base + (uint32_t)((s * per + tensor) * P + j * NmPlanes<KIND>::n) * plane; };
  auto issue = [&](int s, int64_t row) {
    if (row < A.rows) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        fetch8<KIND>(slot(s, 0, j), plane, A.x, row, 8 * at[j], n[j]);
        if (A.mode != NM_NONE) fetch8<KIND>(slot(s, 1, j), plane, A.f, row, 8 * at[j], n[j]);
      }
    }
    cp_async_commit();
  };
  for (int s = 0; s < S; ++s) issue(s, first + s * step);
  const float inv = 1.f / (float)A.width;
  int s = 0;
  for (int64_t row = first; row < A.rows; row += step) {
    wait_stages(S - 1);
    float x[V][8];
#pragma unroll
    for (int j = 0; j < V; ++j) take8<KIND>(slot(s, 0, j), plane, x[j]);
    if (A.mode != NM_NONE) {
      const int g = group_of(A, row);
      float m0 = 0.f, r0 = 1.f;
      if (A.mode == NM_POST)
        row_stats<LN, V>(team, n, inv, A.eps, [&](int j, float (&v)[8]) { take8<KIND>(slot(s, 1, j), plane, v); }, m0, r0);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float f[8], p[8], q[8];
        take8<KIND>(slot(s, 1, j), plane, f);
        if (A.pf.codes) {
          uint32_t byte;
          const uint2 w = pack8(f, byte);
          if (at[j] < nv) store_packed(A.pf, row, at[j], row * nv + at[j], w, byte);
        }
        const bool folded = A.shared_params && A.groups == 1 && !A.starts && !A.gate_rows;
        if (A.shared_params && at[j] < nv) shared8(ps, nv, 1, at[j], p); else param8<KIND>(A.pw, A.pf32, 0, 8 * at[j], n[j], 1.f, p);
        if (!folded) param8<KIND>(A.gate, A.pf32, max(g, 0), 8 * at[j], n[j], 1.f, q);
        float b[8];
        if (LN && A.pb.p) {
          param8<KIND>(A.pb, A.pf32, 0, 8 * at[j], n[j], 0.f, b);
          if (folded && A.gate.p) param8<KIND>(A.gate, A.pf32, 0, 8 * at[j], n[j], 1.f, q);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float d = (f[i] - m0) * r0 * p[i];
          if (LN && A.pb.p) d += folded && A.gate.p ? b[i] * q[i] : b[i];
          if (!folded) d *= q[i];
          x[j][i] = g >= 0 ? fmaf(A.scale, x[j][i], d) : A.scale * x[j][i];      // (a row of no group: whatever stands in f)
        }
      }
      if (A.stats && t == 0) { A.stats[row] = r0; if (LN) A.stats[2 * A.rows + row] = m0; }
    } else {
      if (A.stats && t == 0) { A.stats[row] = 1.f; if (LN) A.stats[2 * A.rows + row] = 0.f; }
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] *= A.scale;
    }
    issue(s, row + S * step);                       // the row's places are read: the next one that will stand there
    s = s + 1 == S ? 0 : s + 1;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (LN || A.b.p || n[j] < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = i < n[j] ? x[j][i] : 0.f;
      }
      if (A.out0.p) store8_any<KIND>(A.out0, row, 8 * at[j], n[j], x[j], true);
      if (A.px.codes) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = x[j][i];
        round8<KIND>(v);
        uint32_t byte;
        const uint2 w = pack8(v, byte);
        if (at[j] < nv) store_packed(A.px, row, at[j], row * nv + at[j], w, byte);
      }
    }
    float m1, r1;
    row_stats<LN, V>(team, n, inv, A.eps, [&](int j, float (&v)[8]) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = x[j][i];
    }, m1, r1);
    if (A.stats && t == 0) { A.stats[A.rows + row] = r1; if (LN) A.stats[3 * A.rows + row] = m1; }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float p[8], b[8];
      if (A.shared_params && at[j] < nv) shared8(ps, nv, 0, at[j], p); else param8<KIND>(A.w, A.pf32, 0, 8 * at[j], n[j], 1.f, p);
      if (LN) param8<KIND>(A.b, A.pf32, 0, 8 * at[j], n[j], 0.f, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[j][i] = (x[j][i] - m1) * r1 * p[i];
        if (LN) x[j][i] += b[i];
        if (i >= n[j]) x[j][i] = 0.f;
      }
      store8_any<KIND>(A.out1, row, 8 * at[j], n[j], x[j], true);
      if (A.ph.codes) {
        round8<KIND>(x[j]);
        uint32_t byte;
        const uint2 w = pack8(x[j], byte);
        if (at[j] < nv) store_packed(A.ph, row, at[j], row * nv + at[j], w, byte);
      }
    }
  }
  cp_async_wait<0>();
}

// Slot of the column sums: those of dh (and dh x'^) at [slot], those of t (and t f^) at [slots + slot + group], so that row groups
// that see several sequences, and sequences that several row groups see, have places of their own.
template <int KIND, bool LN, int V>
__global__ void __launch_bounds__(512, 1) norm_backward_kernel(const ResNormArgs A) {
  extern __shared__ __align__(16) unsigned char nm_smem[];
  griddep_chain();
  const int nv = 4 * A.blocks, teams = blockDim.x / A.tpr, mine = threadIdx.x / A.tpr, t = threadIdx.x - mine * A.tpr;
  RowTeam team{reinterpret_cast<float2*>(nm_smem) + mine * 64, A.tpr >> 5, t >> 5, (int)(threadIdx.x & 31), mine + 1, 0};
  float4* ps = reinterpret_cast<float4*>(nm_smem + NM_RED_BYTES);
  if (A.shared_params) { fill_params<KIND>(A, ps); __syncthreads(); }
  const uint32_t plane = blockDim.x * 16;
  constexpr int P = NmPlanes<KIND>::n * V;
  const uint32_t ring = NM_RED_BYTES + (A.shared_params ? 64 * nv : 0);
  const uint32_t base = smem_u32(nm_smem) + ring + threadIdx.x * 16;
  int at[V], n[V];
#pragma unroll
  for (int j = 0; j < V; ++j) { at[j] = t + j * A.tpr; n[j] = max(0, min(8, A.width - 8 * at[j])); }
  const int64_t team_id = (int64_t)blockIdx.x * teams + mine;
  const int64_t first = team_id * A.chunk, last = min(first + A.chunk, A.rows);
  const int S = A.stages;
  const int per = 2 + (A.dx.p ? 1 : 0) + (A.mode != NM_NONE ? 1 : 0);
  auto slot = [&](int s, int tensor, int j) { return base + (uint32_t)((s * per + tensor) * P + j * NmPlanes<KIND>::n) * plane; };
  const int T_DX = 2, T_F = A.dx.p ? 3 : 2;
  auto issue = [&](int s, int64_t row) {
    if (S > 0 && row < last) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        fetch8<KIND>(slot(s, 0, j), plane, A.dh, row, 8 * at[j], n[j]);
        if (A.px.codes) { if (at[j] < nv) fetch8_packed(slot(s, 1, j), A.px, row, at[j]); }
        else fetch8<KIND>(slot(s, 1, j), plane, A.x, row, 8 * at[j], n[j]);
        if (A.dx.p) fetch8<KIND>(slot(s, T_DX, j), plane, A.dx, row, 8 * at[j], n[j]);
        if (A.mode != NM_NONE) {
          if (A.pf.codes) { if (at[j] < nv) fetch8_packed(slot(s, T_F, j), A.pf, row, at[j]); }
          else fetch8<KIND>(slot(s, T_F, j), plane, A.f, row, 8 * at[j], n[j]);
        }
      }
    }
    cp_async_commit();
  };
  // a tensor's entries: from the thread's places, or (no room for a row there) from memory
  auto dense = [&](int s, int tensor, const RowsOf& m, int64_t row, int j, float (&v)[8]) {
    if (S > 0) take8<KIND>(slot(s, tensor, j), plane, v); else load8<KIND, false>(m, row, 8 * at[j], n[j], v);
  };
  auto kept = [&](int s, int tensor, const PackedRows& p, const RowsOf& m, int64_t row, int j, float (&v)[8]) {
    if (!p.codes) dense(s, tensor, m, row, j, v);
    else if (at[j] >= nv) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    } else if (S > 0) take8_packed(slot(s, tensor, j), at[j], v);
    else unpack8(ld_codes(p.codes + (row * nv + at[j]) * 8), p.exps[row * p.exp_stride + (at[j] >> 2)], v);
  };
  float sw[V][8], sb[LN ? V : 1][8], s1[V][8], s0[LN ? V : 1][8];
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) { sw[j][i] = s1[j][i] = 0.f; if (LN) sb[j][i] = s0[j][i] = 0.f; }
  const int nw = LN ? 2 : 1;
  const int64_t slots = A.combine ? gridDim.x : (int64_t)gridDim.x * teams;
  auto flush = [&](float* to, float (&a)[V][8], bool clear) {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (at[j] < nv) {
        reinterpret_cast<float4*>(to + 8 * at[j])[0] = make_float4(a[j][0], a[j][1], a[j][2], a[j][3]);
        reinterpret_cast<float4*>(to + 8 * at[j])[1] = make_float4(a[j][4], a[j][5], a[j][6], a[j][7]);
        if (clear) {
#pragma unroll
          for (int i = 0; i < 8; ++i) a[j][i] = 0.f;
        }
      }
  };
  auto slot_w = [&](int64_t k, int which) { return A.part + (k * nw + which) * A.part_stride; };
  auto slot_s = [&](int64_t k, int which) { return A.part + ((slots + k) * nw + which) * A.part_stride; };
  for (int s = 0; s < S; ++s) issue(s, first + s);
  const float inv = 1.f / (float)A.width;
  const bool folded = A.shared_params && A.groups == 1 && !A.starts && !A.gate_rows;
  int s = 0, group = -1;
  float4 next = make_float4(1.f, 1.f, 0.f, 0.f);       // the statistics of a row, read a row ahead
  auto read_stats = [&](int64_t row) {
    if (row >= last) return;
    next.y = A.stats[A.rows + row];
    if (LN) next.w = A.stats[3 * A.rows + row];
    if (A.mode == NM_POST) { next.x = A.stats[row]; if (LN) next.z = A.stats[2 * A.rows + row]; }
  };
  read_stats(first);
  for (int64_t row = first; row < last; ++row) {
    wait_stages(S - 1);
    const float r0 = next.x, r1 = next.y, m0 = next.z, m1 = next.w;
    read_stats(row + 1);
    float sum_u = 0.f, sum_d = 0.f;
    float tt[V][8];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float d[8], u[8], p[8];
      dense(s, 0, A.dh, row, j, d);
      kept(s, 1, A.px, A.x, row, j, u);
      if (A.shared_params && at[j] < nv) shared8(ps, nv, 0, at[j], p); else param8<KIND>(A.w, A.pf32, 0, 8 * at[j], n[j], 1.f, p);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float xh = (u[i] - m1) * r1;
        sw[j][i] = fmaf(d[i], xh, sw[j][i]);
        if (LN) sb[j][i] += d[i];
        const float e = d[i] * p[i];
        tt[j][i] = e;
        sum_u = fmaf(e, xh, sum_u);
        if (LN) sum_d += e;
      }
    }
    float2 c = team.sum<LN>(sum_u, sum_d);
    c.x *= inv; c.y *= inv;
    int g = -1;
    if (A.mode != NM_NONE) {
      g = group_of(A, row);
      if (!A.combine && !A.gate_rows && g != group) {            // another sequence: its own column sums
        if (group >= 0) { flush(slot_s(team_id + group, 0), s1, true); if (LN) flush(slot_s(team_id + group, 1), reinterpret_cast<float (&)[V][8]>(s0), true); }
        group = g;
      }
    }
    sum_u = sum_d = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float u[8], v[8];
      kept(s, 1, A.px, A.x, row, j, u);
      if (A.dx.p) dense(s, T_DX, A.dx, row, j, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float xh = (u[i] - m1) * r1;
        float e = fmaf(-xh, c.x, tt[j][i]);
        if (LN) e -= c.y;
        tt[j][i] = A.dx.p ? fmaf(r1, e, v[i]) : r1 * e;
        v[i] = A.scale * tt[j][i];
      }
      store8_any<KIND>(A.out0, row, 8 * at[j], n[j], v, true);
      if (A.mode != NM_NONE && g >= 0) {
        float f[8], p[8], q[8];
        kept(s, T_F, A.pf, A.f, row, j, f);
        if (A.shared_params && at[j] < nv) shared8(ps, nv, 1, at[j], p); else param8<KIND>(A.pw, A.pf32, 0, 8 * at[j], n[j], 1.f, p);
        if (!folded) param8<KIND>(A.gate, A.pf32, g, 8 * at[j], n[j], 1.f, q);
        if (A.gate_rows && A.dgate.p) {
          float b[8];
          param8<KIND>(A.pw, A.pf32, 0, 8 * at[j], n[j], 1.f, u);
          param8<KIND>(A.pb, A.pf32, 0, 8 * at[j], n[j], 0.f, b);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i < n[j]) store_param<KIND>(A.dgate, A.pf32, row, 8 * at[j] + i, tt[j][i] * fmaf((f[i] - m0) * r0, u[i], b[i]));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float fh = (f[i] - m0) * r0;
          const float d = folded ? tt[j][i] : tt[j][i] * q[i];
          const float to = A.gate_rows ? d : tt[j][i];
          s1[j][i] = fmaf(to, fh, s1[j][i]);
          if (LN) s0[j][i] += i < n[j] ? to : 0.f;
          const float e = i < n[j] ? d * p[i] : 0.f;
          tt[j][i] = e;
          sum_u = fmaf(e, fh, sum_u);
          if (LN) sum_d += e;
        }
      }
    }
    if (A.mode != NM_NONE) {
      c = make_float2(0.f, 0.f);
      if (A.mode == NM_POST) { c = team.sum<LN>(sum_u, sum_d); c.x *= inv; c.y *= inv; }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float f[8];
        if (A.mode == NM_POST) kept(s, T_F, A.pf, A.f, row, j, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (A.mode == NM_POST) {
            const float fh = (f[i] - m0) * r0;
            float e = fmaf(-fh, c.x, tt[j][i]);
            if (LN) e -= c.y;
            tt[j][i] = r0 * e;
          }
          if (g < 0) tt[j][i] = 0.f;
        }
        store8_any<KIND>(A.out1, row, 8 * at[j], n[j], tt[j], true);
      }
    }
    if (S > 0) { issue(s, row + S); s = s + 1 == S ? 0 : s + 1; }
  }
  cp_async_wait<0>();
  if (!A.part) return;
  if (A.combine) {
    // the block's teams, one kind of sum after the other, through the ring's memory
    float* buf = reinterpret_cast<float*>(nm_smem + ring);
    auto join = [&](float* to, float (&a)[V][8]) {
      __syncthreads();
      flush(buf + (int64_t)mine * A.part_stride, a, false);
      __syncthreads();
      for (int c = threadIdx.x; c < A.part_stride; c += blockDim.x) {
        float v = 0.f;
        for (int k = 0; k < teams; ++k) v += buf[(int64_t)k * A.part_stride + c];
        to[c] = v;
      }
    };
    join(slot_w(blockIdx.x, 0), sw);
    if (LN) join(slot_w(blockIdx.x, 1), reinterpret_cast<float (&)[V][8]>(sb));
    if (A.mode != NM_NONE) {
      join(slot_s(blockIdx.x, 0), s1);
      if (LN) join(slot_s(blockIdx.x, 1), reinterpret_cast<float (&)[V][8]>(s0));
    }
    return;
  }
  flush(slot_w(team_id, 0), sw, false);
  if (LN) flush(slot_w(team_id, 1), reinterpret_cast<float (&)[V][8]>(sb), false);
  if (A.mode != NM_NONE && group >= 0) {
    flush(slot_s(team_id + group, 0), s1, false);
    if (LN) flush(slot_s(team_id + group, 1), reinterpret_cast<float (&)[V][8]>(s0), false);
  }
}

// ---- the same for what large models run: every row at a multiple of 16 bytes, a width of whole vectors of 8, weights in shared memory ----
// Per entry the backward kernel takes 42 instructions instead of the general one's 97: rows come by bulk copies that one thread of a row's
// team issues some rows ahead, into places that are free once the team's next barrier, which the reductions have anyway, is passed; pairs of fp32 in
// one instruction; no tests per entry; what a reduction separates is kept in registers instead of being read and widened again.
// A wait for a copy is bounded; one that ran out turns what its warp makes of the team's further rows to NaN (x', means, kept copies, gradients and
// column sums), and by the sums over a row all that follows from these.

constexpr uint32_t NM_WAIT_POLLS = 1u << 20;
constexpr uint64_t NM_WAIT_NS = 500000000ull;
static __device__ __noinline__ bool nm_wait_long(uint64_t* bar, uint32_t parity) {
  uint64_t start = 0;
  for (uint32_t i = 0; i < NM_WAIT_POLLS; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((i & 15) == 15) {
      uint64_t now;
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
      if (start == 0) start = now;
      else if (now - start > NM_WAIT_NS) break;
    }
  }
  return false;
}
// A team's places for rows.  poison: NaN once a copy has not come, -0 before, which changes nothing that it is added to.
struct NmRing {
  uint64_t* bars;
  int stages, at = 0;
  int copied = 0;
  uint32_t parity = 0, failed = 0;      // failed: 1 + the place and parity whose copy did not come
  float poison = -0.f;
  __device__ __forceinline__ void wait() {                 // whole warps, which give up together
    if (failed != 0 || __all_sync(0xffffffffu, mbar_try_wait(&bars[at], parity))) return;
    const bool ok = nm_wait_long(&bars[at], parity);
    __syncwarp();
    if (__all_sync(0xffffffffu, ok)) return;
    poison = __int_as_float(0x7fffffff);
    failed = 1 + 2 * at + parity;
  }
  __device__ __forceinline__ void next() { if (++at == stages) { at = 0; parity ^= 1; } }
};
// After a wait that ran out nothing more is copied; what is under way has to land before shared memory is given up.
static __device__ __noinline__ void nm_settle(uint64_t* bars, int stages, uint32_t failed) {
  for (int k = 0; k < stages; ++k) {
    const int s = ((int)(failed - 1) >> 1) + k;
    nm_wait_long(&bars[s % stages], ((failed - 1) ^ (uint32_t)(s >= stages)) & 1u);
  }
}

template <int KIND> __device__ __forceinline__ const char* row_of(const RowsOf& t, int64_t row) { return t.p + row * t.ld * (KIND == LS_F32 ? 4 : 2); }
// the pairs of vector v of a row that starts at `row`
template <int KIND>
__device__ __forceinline__ void take_pairs(uint32_t row, uint32_t v, uint64_t (&out)[4]) {
  if (KIND == LS_F32) {
    const uint4 a = lds128(row + v * 32), b = lds128(row + v * 32 + 16);
    out[0] = pk2(__uint_as_float(a.x), __uint_as_float(a.y)); out[1] = pk2(__uint_as_float(a.z), __uint_as_float(a.w));
    out[2] = pk2(__uint_as_float(b.x), __uint_as_float(b.y)); out[3] = pk2(__uint_as_float(b.z), __uint_as_float(b.w));
  } else {
    const uint4 a = lds128(row + v * 16);
    float2 f = widen2<KIND>(a.x); out[0] = pk2(f.x, f.y);
    f = widen2<KIND>(a.y); out[1] = pk2(f.x, f.y);
    f = widen2<KIND>(a.z); out[2] = pk2(f.x, f.y);
    f = widen2<KIND>(a.w); out[3] = pk2(f.x, f.y);
  }
}
// the same of a packed row, times r
__device__ __forceinline__ void take_packed(uint32_t row, uint32_t v, uint32_t byte, float r, uint64_t (&out)[4]) {
  const uint2 q = lds64(row + v * 8);
  const float s = __uint_as_float(byte << 23) * r;      // (a power of two: no rounding but that of the products)
  const uint64_t scale = pk2(s, s), off = pk2(-8388736.f, -8388736.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = (i < 2 ? q.x : q.y) ^ 0x80808080u;
    const uint64_t c = pk2(__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 + 2 * (i & 1))), __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7441 + 2 * (i & 1))));
    out[i] = mul2(add2(c, off), scale);
  }
}
template <int KIND>
__device__ __forceinline__ void store_pairs(const char* row, uint32_t v, const uint64_t (&x)[4]) {
  const float2 a = upk2(x[0]), b = upk2(x[1]), d = upk2(x[2]), e = upk2(x[3]);
  uint4* p = reinterpret_cast<uint4*>(const_cast<char*>(row) + v * (KIND == LS_F32 ? 32u : 16u));
  if (KIND == LS_F32) {
    st_stream(p, make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y)));
    st_stream(p + 1, make_uint4(__float_as_uint(d.x), __float_as_uint(d.y), __float_as_uint(e.x), __float_as_uint(e.y)));
  } else st_stream(p, make_uint4(narrow2<KIND>(a.x, a.y), narrow2<KIND>(b.x, b.y), narrow2<KIND>(d.x, d.y), narrow2<KIND>(e.x, e.y)));
}
// kept copy of 4 pairs, as rounded to the storage type; whole warps
template <int KIND>
__device__ __forceinline__ void keep_pairs(const PackedRows& t, int64_t row, int v, int nv, const uint64_t (&x)[4], bool rounded) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 q = upk2(x[i]); f[2 * i] = q.x; f[2 * i + 1] = q.y; }
  if (!rounded) round8<KIND>(f);
  uint32_t byte;
  const uint2 w = pack8(f, byte);
  if (v < nv) store_packed(t, row, v, row * nv + v, w, byte);
}
__device__ __forceinline__ void shared_pairs(uint32_t ps, uint32_t nv, int which, uint32_t v, uint64_t (&out)[4]) {
  const uint4 a = lds128(ps + (2 * which * nv + v) * 16), b = lds128(ps + ((2 * which + 1) * nv + v) * 16);
  out[0] = pk2(__uint_as_float(a.x), __uint_as_float(a.y)); out[1] = pk2(__uint_as_float(a.z), __uint_as_float(a.w));
  out[2] = pk2(__uint_as_float(b.x), __uint_as_float(b.y)); out[3] = pk2(__uint_as_float(b.z), __uint_as_float(b.w));
}
template <int KIND>
__device__ __forceinline__ void param_pairs(const RowsOf& t, int pf32, int64_t row, int c, int n, float fill, uint64_t (&out)[4]) {
  float v[8];
  param8<KIND>(t, pf32, row, c, n, fill, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = pk2(v[2 * i], v[2 * i + 1]);
}
__device__ __forceinline__ float sum_pair(uint64_t v) { const float2 f = upk2(v); return f.x + f.y; }
__device__ __forceinline__ void zero_pairs(uint64_t (&v)[4]) { v[0] = v[1] = v[2] = v[3] = pk2(0.f, 0.f); }

// Shared memory of a team: NM_MAX_STAGES barriers; then, behind all teams' and the weights, its ring of rows.
constexpr int NM_BARS = 32 * NM_MAX_STAGES * 8;

template <int KIND, bool LN, int V>
__global__ void __launch_bounds__(1024, 1) norm_forward_fast_kernel(const ResNormArgs A) {
  extern __shared__ __align__(16) unsigned char nm_smem[];
  const int nv = 4 * A.blocks, nd = A.width >> 3, teams = blockDim.x / A.tpr;
  const int mine = __shfl_sync(0xffffffffu, threadIdx.x / A.tpr, 0), t = threadIdx.x - mine * A.tpr;      // (known to the compiler as the warp's: rows' addresses are)
  RowTeam team{reinterpret_cast<float2*>(nm_smem) + mine * 64, A.tpr >> 5, t >> 5, (int)(threadIdx.x & 31), mine + 1, 0};
  uint64_t* bars = reinterpret_cast<uint64_t*>(nm_smem + NM_RED_BYTES) + mine * NM_MAX_STAGES;
  const int S = A.stages, per = A.mode == NM_NONE ? 1 : 2;
  if (t == 0) {
    for (int s = 0; s < S; ++s) mbar_init(&bars[s], 1);
    fence_mbar_init();
  }
  griddep_chain();
  fill_params<KIND>(A, reinterpret_cast<float4*>(nm_smem + NM_RED_BYTES + NM_BARS));
  __syncthreads();
  const uint32_t bytes = (uint32_t)A.width * (KIND == LS_F32 ? 4 : 2), ps = smem_u32(nm_smem) + NM_RED_BYTES + NM_BARS;
  const uint32_t places = ps + 64 * nv + (uint32_t)(mine * S * per) * bytes;
  NmRing ring{bars, S};
  const int64_t first = (int64_t)blockIdx.x * teams + mine, step = (int64_t)gridDim.x * teams;
  const bool folded = A.groups == 1 && !A.starts;
  auto issue = [&](int s, int64_t row) {                 // one thread
    if (row >= A.rows || ring.failed || ring.copied++ >= A.copies) return;
    mbar_expect_tx(&bars[s], bytes * per);
    const uint32_t to = places + (uint32_t)(s * per) * bytes;
    bulk_g2s_at(to, row_of<KIND>(A.x, row), bytes, &bars[s]);
    if (A.mode != NM_NONE) bulk_g2s_at(to + bytes, row_of<KIND>(A.f, row), bytes, &bars[s]);
  };
  if (t == 0)
    for (int s = 0; s < S; ++s) issue(s, first + s * step);
  const float inv = 1.f / (float)A.width;
  const uint64_t zero = pk2(0.f, 0.f);
  // mean and 1 / deviation of V vectors, which leave without the mean
  auto stats = [&](uint64_t (&v)[V][4], float& mean, float& rstd) {
    mean = 0.f;
    if (LN) {
      uint64_t s = zero;
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) s = add2(s, v[j][i]);
      mean = team.sum<false>(sum_pair(s), 0.f).x * inv;
      const uint64_t m = pk2(-mean, -mean);
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (t + j * A.tpr < nd) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[j][i] = add2(v[j][i], m);
        }
    }
    uint64_t s = zero, r = zero;
#pragma unroll
    for (int j = 0; j < V; ++j) { s = fma2(v[j][0], v[j][0], s); r = fma2(v[j][1], v[j][1], r); s = fma2(v[j][2], v[j][2], s); r = fma2(v[j][3], v[j][3], r); }
    rstd = rsqrtf(fmaf(team.sum<false>(sum_pair(add2(s, r)), 0.f).x, inv, A.eps));
  };
  for (int64_t row = first; row < A.rows; row += step) {
    ring.wait();
    const uint32_t from = places + (uint32_t)(ring.at * per) * bytes;
    const uint64_t scale = pk2(A.scale + ring.poison, A.scale + ring.poison), lost = pk2(ring.poison, ring.poison);      // (a scale that is NaN makes x' so)
    uint64_t x[V][4];
    float mean, rstd;
    if (A.mode != NM_NONE) {
      uint64_t f[V][4];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = t + j * A.tpr;
        if (v < nd) take_pairs<KIND>(from + bytes, v, f[j]); else zero_pairs(f[j]);
        f[j][0] = add2(f[j][0], lost);                     // one NaN: the whole kept block, and by the sums the row
        if (A.pf.codes) keep_pairs<KIND>(A.pf, row, v, nv, f[j], true);
      }
      stats(f, mean, rstd);
      if (A.stats && t == 0) { A.stats[row] = rstd; if (LN) A.stats[2 * A.rows + row] = mean; }
      const int g = folded ? 0 : group_of(A, row);
      const uint64_t r = pk2(rstd, rstd);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = t + j * A.tpr;
        if (v >= nd) { zero_pairs(x[j]); continue; }
        uint64_t p[4], q[4], b[4];
        take_pairs<KIND>(from, v, x[j]);
        shared_pairs(ps, nv, 1, v, p);
        if (LN && A.pb.p) {
          param_pairs<KIND>(A.pb, A.pf32, 0, 8 * v, 8, 0.f, b);
          if (folded && A.gate.p) {
            param_pairs<KIND>(A.gate, A.pf32, 0, 8 * v, 8, 1.f, q);
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = mul2(b[i], q[i]);
          }
        }
        if (folded) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint64_t d = mul2(f[j][i], r);
            x[j][i] = fma2(scale, x[j][i], LN && A.pb.p ? fma2(d, p[i], b[i]) : mul2(d, p[i]));
          }
        } else {
          param_pairs<KIND>(A.gate, A.pf32, max(g, 0), 8 * v, 8, 1.f, q);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint64_t d = mul2(mul2(f[j][i], r), p[i]);
            if (LN && A.pb.p) d = add2(d, b[i]);
            x[j][i] = g < 0 ? mul2(scale, x[j][i]) : fma2(scale, x[j][i], mul2(d, q[i]));      // (a row of no group: whatever stands in f)
          }
        }
      }
    } else {
      if (A.stats && t == 0) { A.stats[row] = 1.f; if (LN) A.stats[2 * A.rows + row] = 0.f; }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = t + j * A.tpr;
        if (v >= nd) { zero_pairs(x[j]); continue; }
        take_pairs<KIND>(from, v, x[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[j][i] = mul2(scale, x[j][i]);
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int v = t + j * A.tpr;
      if (A.out0.p && v < nd) store_pairs<KIND>(row_of<KIND>(A.out0, row), v, x[j]);
      if (A.px.codes) keep_pairs<KIND>(A.px, row, v, nv, x[j], false);
    }
    stats(x, mean, rstd);
    if (A.tpr == 32) __syncwarp();                         // (a team of several warps has passed a barrier in the sum above)
    if (t == 0) issue(ring.at, row + S * step);                  // the row's places have been read: the next one that will stand there
    ring.next();
    if (A.stats && t == 0) { A.stats[A.rows + row] = rstd; if (LN) A.stats[3 * A.rows + row] = mean; }
    const uint64_t r = pk2(rstd, rstd);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int v = t + j * A.tpr;
      if (v < nd) {
        uint64_t p[4], b[4];
        shared_pairs(ps, nv, 0, v, p);
        if (LN && A.b.p) {
          param_pairs<KIND>(A.b, A.pf32, 0, 8 * v, 8, 0.f, b);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[j][i] = fma2(mul2(x[j][i], r), p[i], b[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[j][i] = mul2(mul2(x[j][i], r), p[i]);
        }
        store_pairs<KIND>(row_of<KIND>(A.out1, row), v, x[j]);
      }
      if (A.ph.codes) keep_pairs<KIND>(A.ph, row, v, nv, x[j], false);
    }
  }
  if (t == 0 && ring.failed) nm_settle(ring.bars, S, ring.failed);
}

// Backward with a normalised block and a gradient of x'; x' in storage, f packed (PF) or in storage.
template <int KIND, bool LN, int V, bool PF>
__global__ void __launch_bounds__(512, 1) norm_backward_fast_kernel(const ResNormArgs A) {
  extern __shared__ __align__(16) unsigned char nm_smem[];
  const int nv = 4 * A.blocks, nd = A.width >> 3, teams = blockDim.x / A.tpr;
  const int mine = __shfl_sync(0xffffffffu, threadIdx.x / A.tpr, 0), t = threadIdx.x - mine * A.tpr;
  RowTeam team{reinterpret_cast<float2*>(nm_smem) + mine * 64, A.tpr >> 5, t >> 5, (int)(threadIdx.x & 31), mine + 1, 0};
  uint64_t* bars = reinterpret_cast<uint64_t*>(nm_smem + NM_RED_BYTES) + mine * NM_MAX_STAGES;
  const int S = A.stages;
  if (t == 0) {
    for (int s = 0; s < S; ++s) mbar_init(&bars[s], 1);
    fence_mbar_init();
  }
  griddep_chain();
  fill_params<KIND>(A, reinterpret_cast<float4*>(nm_smem + NM_RED_BYTES + NM_BARS));
  __syncthreads();
  const uint32_t bytes = (uint32_t)A.width * (KIND == LS_F32 ? 4 : 2), f_bytes = PF ? 32u * A.blocks : bytes, stage = 3 * bytes + f_bytes;
  const uint32_t ps = smem_u32(nm_smem) + NM_RED_BYTES + NM_BARS, places = ps + 64 * nv + (uint32_t)(mine * S) * stage;
  NmRing ring{bars, S};
  const int64_t team_id = (int64_t)blockIdx.x * teams + mine;
  const int64_t first = team_id * A.chunk, last = min(first + A.chunk, A.rows);
  const bool folded = A.groups == 1 && !A.starts;
  auto issue = [&](int s, int64_t row) {                 // one thread
    if (row >= last || ring.failed || ring.copied++ >= A.copies) return;
    mbar_expect_tx(&bars[s], stage);
    const uint32_t to = places + (uint32_t)s * stage;
    bulk_g2s_at(to, row_of<KIND>(A.dh, row), bytes, &bars[s]);
    bulk_g2s_at(to + bytes, row_of<KIND>(A.x, row), bytes, &bars[s]);
    bulk_g2s_at(to + 2 * bytes, row_of<KIND>(A.dx, row), bytes, &bars[s]);
    bulk_g2s_at(to + 3 * bytes, PF ? reinterpret_cast<const char*>(A.pf.codes) + row * f_bytes : row_of<KIND>(A.f, row), f_bytes, &bars[s]);
  };
  if (t == 0)
    for (int s = 0; s < S; ++s) issue(s, first + s);
  // what comes by plain loads, a row ahead: the statistics and (PF) the bytes of this thread's blocks
  float4 next = make_float4(1.f, 1.f, 0.f, 0.f);
  uint32_t next_byte[V];
  auto ahead = [&](int64_t row) {
    if (row >= last) return;
    next.x = A.stats[row]; next.y = A.stats[A.rows + row];
    if (LN) { next.z = A.stats[2 * A.rows + row]; next.w = A.stats[3 * A.rows + row]; }
    if (PF) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (t + j * A.tpr < nd) next_byte[j] = A.pf.exps[row * A.pf.exp_stride + ((t + j * A.tpr) >> 2)];
    }
  };
  ahead(first);
  const uint64_t zero = pk2(0.f, 0.f), scale = pk2(A.scale, A.scale);
  uint64_t sw[V][4], s1[V][4], sb[LN ? V : 1][4], s0[LN ? V : 1][4];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    zero_pairs(sw[j]); zero_pairs(s1[j]);
    if (LN) { zero_pairs(sb[LN ? j : 0]); zero_pairs(s0[LN ? j : 0]); }
  }
  const int nw = LN ? 2 : 1;
  const int64_t slots = A.combine ? gridDim.x : (int64_t)gridDim.x * teams;
  auto flush = [&](float* to, const uint64_t (&a)[4], int j) {
    const int v = t + j * A.tpr;
    if (v >= nv) return;
    const float2 f0 = upk2(a[0]), f1 = upk2(a[1]), f2 = upk2(a[2]), f3 = upk2(a[3]);
    reinterpret_cast<float4*>(to + 8 * v)[0] = make_float4(f0.x, f0.y, f1.x, f1.y);
    reinterpret_cast<float4*>(to + 8 * v)[1] = make_float4(f2.x, f2.y, f3.x, f3.y);
  };
  auto slot_w = [&](int64_t k, int which) { return A.part + (k * nw + which) * A.part_stride; };
  auto slot_s = [&](int64_t k, int which) { return A.part + ((slots + k) * nw + which) * A.part_stride; };
  const float inv = 1.f / (float)A.width;
  int group = folded ? 0 : -1;
  for (int64_t row = first; row < last; ++row) {
    const float r0 = next.x, m0 = next.z, m1 = next.w;
    float r1 = next.y;
    uint32_t byte[V];
#pragma unroll
    for (int j = 0; j < V; ++j) byte[j] = next_byte[j];
    ahead(row + 1);
    ring.wait();
    r1 += ring.poison;
    const uint32_t from = places + (uint32_t)ring.at * stage;
    uint64_t e[V][4], u[V][4], su = zero, sd = zero;
    {
      const uint64_t m = pk2(-m1, -m1), r = pk2(r1, r1);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = t + j * A.tpr;
        if (v >= nd) { zero_pairs(e[j]); zero_pairs(u[j]); continue; }
        uint64_t d[4], w[4];
        take_pairs<KIND>(from, v, d);
        take_pairs<KIND>(from + bytes, v, u[j]);
        shared_pairs(ps, nv, 0, v, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[j][i] = mul2(LN ? add2(u[j][i], m) : u[j][i], r);
          sw[j][i] = fma2(d[i], u[j][i], sw[j][i]);
          if (LN) sb[LN ? j : 0][i] = add2(sb[LN ? j : 0][i], d[i]);
          e[j][i] = mul2(d[i], w[i]);
          su = fma2(e[j][i], u[j][i], su);
          if (LN) sd = add2(sd, e[j][i]);
        }
      }
    }
    float2 c = team.sum<LN>(sum_pair(su), LN ? sum_pair(sd) : 0.f);
    int g = 0;
    if (!folded) {
      g = group_of(A, row);
      if (g != group) {                                  // another sequence: its own column sums
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (group >= 0) { flush(slot_s(team_id + group, 0), s1[j], j); if (LN) flush(slot_s(team_id + group, 1), s0[LN ? j : 0], j); }
          zero_pairs(s1[j]);
          if (LN) zero_pairs(s0[LN ? j : 0]);
        }
        group = g;
      }
    }
    {
      // t = dx' + r1 (e - u mean(e u) - mean e)
      const uint64_t cu = pk2(-inv * c.x, -inv * c.x), cd = pk2(-inv * c.y, -inv * c.y), r = pk2(r1, r1), m = pk2(-m0, -m0), q0 = pk2(r0, r0);
      su = sd = zero;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = t + j * A.tpr;
        if (v >= nd) continue;
        uint64_t x[4], p[4];
        take_pairs<KIND>(from + 2 * bytes, v, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint64_t k = fma2(u[j][i], cu, e[j][i]);
          if (LN) k = add2(k, cd);
          e[j][i] = fma2(r, k, x[i]);
          x[i] = mul2(scale, e[j][i]);
        }
        store_pairs<KIND>(row_of<KIND>(A.out0, row), v, x);
        if (PF) take_packed(from + 3 * bytes, v, byte[j], LN ? 1.f : r0, u[j]);
        else take_pairs<KIND>(from + 3 * bytes, v, u[j]);
        if (LN || !PF) {
#pragma unroll
          for (int i = 0; i < 4; ++i) u[j][i] = mul2(LN ? add2(u[j][i], m) : u[j][i], q0);
        }
        shared_pairs(ps, nv, 1, v, p);
        if (!folded) {
          uint64_t q[4];
          param_pairs<KIND>(A.gate, A.pf32, max(g, 0), 8 * v, 8, 1.f, q);
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] = mul2(p[i], q[i]);
          if (g < 0) { zero_pairs(u[j]); zero_pairs(e[j]); zero_pairs(p); }      // a row of no group: whatever stands in f
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s1[j][i] = fma2(e[j][i], u[j][i], s1[j][i]);
          if (LN) s0[LN ? j : 0][i] = add2(s0[LN ? j : 0][i], e[j][i]);
          e[j][i] = mul2(e[j][i], p[i]);
          su = fma2(e[j][i], u[j][i], su);
          if (LN) sd = add2(sd, e[j][i]);
        }
      }
    }
    c = team.sum<LN>(sum_pair(su), LN ? sum_pair(sd) : 0.f);
    if (A.tpr == 32) __syncwarp();
    if (t == 0) issue(ring.at, row + S);                         // the row's places have been read
    ring.next();
    {
      const float r = g < 0 ? 0.f : r0;
      const uint64_t fu = pk2(-inv * c.x, -inv * c.x), fd = pk2(-inv * c.y, -inv * c.y), f = pk2(r, r);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int v = t + j * A.tpr;
        if (v >= nd) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint64_t k = fma2(u[j][i], fu, e[j][i]);
          if (LN) k = add2(k, fd);
          e[j][i] = mul2(f, k);
        }
        store_pairs<KIND>(row_of<KIND>(A.out1, row), v, e[j]);
      }
    }
  }
  if (t == 0 && ring.failed) nm_settle(ring.bars, S, ring.failed);
  if (!A.part) return;
  if (LN) {                                              // (of the column sums only these have been formed without 1 / deviation)
    const uint64_t p = pk2(ring.poison, ring.poison);
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) sb[LN ? j : 0][i] = add2(sb[LN ? j : 0][i], p);
  }
  if (A.combine && teams > 1) {
    // the block's teams, one kind of sum after the other, through the ring's memory
    float* buf = reinterpret_cast<float*>(nm_smem + NM_RED_BYTES + NM_BARS + 64 * nv);
    auto join = [&](float* to, const uint64_t (&a)[V][4]) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < V; ++j) flush(buf + (int64_t)mine * A.part_stride, a[j], j);
      __syncthreads();
      for (int c = threadIdx.x; c < A.part_stride; c += blockDim.x) {
        float v = 0.f;
        for (int k = 0; k < teams; ++k) v += buf[(int64_t)k * A.part_stride + c];
        to[c] = v;
      }
    };
    join(slot_w(blockIdx.x, 0), sw);
    if constexpr (LN) join(slot_w(blockIdx.x, 1), sb);
    join(slot_s(blockIdx.x, 0), s1);
    if constexpr (LN) join(slot_s(blockIdx.x, 1), s0);
    return;
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    flush(slot_w(team_id, 0), sw[j], j);
    if (LN) flush(slot_w(team_id, 1), sb[LN ? j : 0], j);
    if (group >= 0) {
      flush(slot_s(team_id + group, 0), s1[j], j);
      if (LN) flush(slot_s(team_id + group, 1), s0[LN ? j : 0], j);
    }
  }
}

// Column sums of the slots, in a fixed order: 32 columns a block, NF_Y threads on each.  Blocks (x, 0) add up dw and db, blocks (x, 1 + g) the
// sums of group g.  Several groups: their sums go behind the slots, and a second launch multiplies them by the gates and adds them.
constexpr int NF_Y = 16;
struct NormSums {
  float* part;
  int64_t slots, part_stride, chunk, rows, rows_per;
  const int* starts;
  int groups, width, pf32, per_row, post;   // per_row: the sums hold gate * t already; post: the block's output is normalised
  RowsOf pw, pb, gate;                      // parameters
  RowsOf dw, db, dpw, dpb, dgate;           // their gradients; p null: not wanted
};
template <int KIND>
__device__ __forceinline__ float sums_param(const RowsOf& t, int pf32, int64_t row, int c, float fill) {
  if (!t.p) return fill;
  return KIND == LS_F32 || pf32 ? reinterpret_cast<const float*>(t.p)[row * t.ld + c] : ld_real<KIND>(t.p + (row * t.ld + c) * 2);
}
// where the sums of group g stand
__device__ __forceinline__ float* sums_of_group(const NormSums& A, int nw, int64_t g) { return A.part + (2 * A.slots + A.groups + g) * nw * A.part_stride; }

// the rows of group g: [r0, r1), none where r0 >= r1
__device__ __forceinline__ void rows_of_group(const NormSums& A, int64_t g, int64_t& r0, int64_t& r1) {
  r0 = 0; r1 = A.rows;
  if (A.starts) { r0 = max((int64_t)A.starts[g], (int64_t)0); r1 = min((int64_t)A.starts[g + 1], A.rows); }
  else if (A.groups > 1) { r0 = g * A.rows_per; r1 = min(r0 + A.rows_per, A.rows); }      // (no rows at all: no group has any)
}

template <int KIND, bool LN>
__global__ void __launch_bounds__(32 * NF_Y) norm_sums_kernel(const NormSums A) {
  __shared__ float2 red[NF_Y][33];
  griddep_chain();
  const int x = threadIdx.x, y = threadIdx.y, c = blockIdx.x * 32 + x, nw = LN ? 2 : 1;
  const bool live = c < A.width;
  for (int64_t part = blockIdx.y; part <= A.groups; part += gridDim.y) {
    const int64_t g = part - 1;
    int64_t at = 0, k0 = 0, k1 = A.slots - 1;             // slots at + [k0, k1]
    bool none = false;                                    // a group without rows
    if (g >= 0) {
      at = A.slots + (A.per_row ? 0 : g);
      int64_t r0, r1;
      rows_of_group(A, g, r0, r1);
      none = r0 >= r1;
      if (none) k1 = -1;
      else if (A.chunk) { k0 = r0 / A.chunk; k1 = (r1 - 1) / A.chunk; }      // (chunk 0: combined sums, one group)
    }
    float2 v = make_float2(0.f, 0.f);
    if (live) {
      const float* p = A.part + (at + k0 + y) * nw * A.part_stride + c;
#pragma unroll 8
      for (int64_t k = k0 + y; k <= k1; k += NF_Y, p += (int64_t)NF_Y * nw * A.part_stride) {
        v.x += p[0];
        if (LN) v.y += p[A.part_stride];
      }
    }
    red[y][x] = v;
    __syncthreads();
    if (y == 0 && live) {
      for (int k = 1; k < NF_Y; ++k) { v.x += red[k][x].x; v.y += red[k][x].y; }
      if (g < 0) {
        if (A.dw.p) store_param<KIND>(A.dw, A.pf32, 0, c, v.x);
        if (A.db.p) store_param<KIND>(A.db, A.pf32, 0, c, v.y);
      } else {
        if (A.dgate.p && !A.per_row) {
          const float pw = A.post ? sums_param<KIND>(A.pw, A.pf32, 0, c, 1.f) : 1.f, pb = LN && A.post ? sums_param<KIND>(A.pb, A.pf32, 0, c, 0.f) : 0.f;
          store_param<KIND>(A.dgate, A.pf32, g, c, none ? 0.f : fmaf(v.x, pw, v.y * pb));
        }
        if (A.groups == 1) {
          const float gate = A.per_row || none ? 1.f : sums_param<KIND>(A.gate, A.pf32, 0, c, 1.f);
          if (A.dpw.p) store_param<KIND>(A.dpw, A.pf32, 0, c, gate * v.x);
          if (A.dpb.p) store_param<KIND>(A.dpb, A.pf32, 0, c, gate * v.y);
        } else {
          float* to = sums_of_group(A, nw, g) + c;
          to[0] = v.x;
          if (LN) to[A.part_stride] = v.y;
        }
      }
    }
    __syncthreads();
  }
}
template <int KIND, bool LN>
__global__ void __launch_bounds__(32 * NF_Y) norm_groups_kernel(const NormSums A) {
  __shared__ float2 red[NF_Y][33];
  griddep_chain();
  const int x = threadIdx.x, y = threadIdx.y, c = blockIdx.x * 32 + x, nw = LN ? 2 : 1;
  float2 v = make_float2(0.f, 0.f);
  if (c < A.width) {
#pragma unroll 4
    for (int64_t g = y; g < A.groups; g += NF_Y) {
      int64_t r0, r1;
      rows_of_group(A, g, r0, r1);
      const float gate = r0 < r1 ? sums_param<KIND>(A.gate, A.pf32, g, c, 1.f) : 0.f;      // (one that no row has may be anything)
      const float* p = sums_of_group(A, nw, g) + c;
      v.x = fmaf(gate, p[0], v.x);
      if (LN) v.y = fmaf(gate, p[A.part_stride], v.y);
    }
  }
  red[y][x] = v;
  __syncthreads();
  if (y == 0 && c < A.width) {
    for (int k = 1; k < NF_Y; ++k) { v.x += red[k][x].x; v.y += red[k][x].y; }
    if (A.dpw.p) store_param<KIND>(A.dpw, A.pf32, 0, c, v.x);
    if (A.dpb.p) store_param<KIND>(A.dpb, A.pf32, 0, c, v.y);
  }
}

}  // namespace tg
