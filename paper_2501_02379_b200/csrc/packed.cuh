// Activations in 8 bits: packing, unpacking, and the gated activation that keeps its inputs packed.
//
// Format.  A block of 32 entries of a row shares a power of two: with E = floor(log2 max |x|) over the block and
// e = max(E - 6, -126),
//   code = clamp(round(x 2^-e), -127, 127) (round to nearest even),   x^ = code 2^e,
// and the block's byte is e + 127.  So |x - x^| <= 2^e / 2, half of 1/64 of a power of two that the largest entry reaches (up to
// 2^e for an entry within 1/256 of the next one, where the code is clamped).  Byte 0: a block of zeros.  Byte 255: a block with an entry
// that is not finite; its codes are 0 and 0 * 2^128 = 0 * infinity makes every entry read back as NaN, without a test.
// A power of two and not max / 127: the quotient, the codes and x^ are exact, so the codes do not depend on how they are computed, and
// x^ (7 bits) is itself a bfloat16, or an fp16 number where x was one: a tensor core multiplies by x^ without a rounding.
// Memory: rows of 32 B codes each (B blocks, the last one filled with zeros), then rows of B bytes, padded with zeros to a
// multiple of 4.
//
// A thread takes 8 entries (16 bytes of 16-bit storage, 8 bytes of codes), four neighbours a block.  Reading back is bound by memory
// (16384 x 8192 bf16: 62 us, 62 at the copy rate); packing by issue slots, 73 % busy, beside memory (84 us for 62), and so is the gated
// activation (16384 x 14336 bf16 silu at burst clocks: forward 394 us for 290, backward 330 us for 290; 781 us for both at sustained ones).
#pragma once
#include "lists.cuh"

namespace tg {

// Rows of a dense tensor: `al` bytes (2, 4, 8 or 16) divide the address of every row's first entry.
struct RowsOf {
  char* p;
  int64_t ld;            // entries from one row to the next
  int al;
};
struct PackedRows {
  unsigned char* codes;  // 32 * blocks bytes a row
  unsigned char* exps;   // exp_stride bytes a row
  int blocks, exp_stride;
};

// Blocks of an SM that the registers of the 16-bit kernels have to leave room for: threads to switch between are worth a few spilled registers
// (12000 x 2730 fp16, rows at odd words: gated activation 67 us, 81 without the bound; backward 60 and 79).
constexpr int PK_THREADS = 256, PK_BLOCKS = 8, PK_BLOCKS_ODD = 6;

// 8 entries of a row from entry c on, of which n (0..8) exist; the others are 0.  ALIGNED: al is 16 and n is 8 or 0.
template <int KIND, bool ALIGNED>
__device__ __forceinline__ void load8(const RowsOf& t, int64_t row, int c, int n, float (&v)[8]) {
  constexpr int B = KIND == LS_F32 ? 4 : 2;
  const char* p = t.p + (row * t.ld + c) * B;
  if (n == 8 && (ALIGNED || t.al >= 4)) {
    uint32_t w[8];
    if (ALIGNED || t.al == 16) {
#pragma unroll
      for (int i = 0; i < B / 2; ++i) {
        const uint4 q = ld_stream(reinterpret_cast<const uint4*>(p) + i);
        w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
      }
    } else if (t.al == 8) {
#pragma unroll
      for (int i = 0; i < B; ++i) { const uint2 q = reinterpret_cast<const uint2*>(p)[i]; w[2 * i] = q.x; w[2 * i + 1] = q.y; }
    } else {
#pragma unroll
      for (int i = 0; i < 2 * B; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (KIND == LS_F32) v[i] = __uint_as_float(w[i]);
      else if ((i & 1) == 0) { const float2 q = widen2<KIND>(w[i / 2]); v[i] = q.x; v[i + 1] = q.y; }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? ld_real<KIND>(p + i * B) : 0.f;
  }
}
template <int KIND, bool ALIGNED>
__device__ __forceinline__ void store8(const RowsOf& t, int64_t row, int c, int n, const float (&v)[8]) {
  constexpr int B = KIND == LS_F32 ? 4 : 2;
  char* p = t.p + (row * t.ld + c) * B;
  if (n == 8 && (ALIGNED || t.al >= 4)) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (KIND == LS_F32) w[i] = __float_as_uint(v[i]);
      else if ((i & 1) == 0) w[i / 2] = narrow2<KIND>(v[i], v[i + 1]);
    }
    if (ALIGNED || t.al == 16) {
#pragma unroll
      for (int i = 0; i < B / 2; ++i) st_stream(reinterpret_cast<uint4*>(p) + i, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
    } else if (t.al == 8) {
#pragma unroll
      for (int i = 0; i < B; ++i) reinterpret_cast<uint2*>(p)[i] = make_uint2(w[2 * i], w[2 * i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < 2 * B; ++i) reinterpret_cast<uint32_t*>(p)[i] = w[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) st_real<KIND>(p + i * B, v[i]);
  }
}
// 16 bytes from byte 16 - m of w on, m in [4 K, 4 K + 4) and even
template <int K>
__device__ __forceinline__ void shifted4(const uint32_t (&w)[8], int m, uint32_t (&o)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = m & 2 ? __funnelshift_r(w[3 + i - K], w[4 + i - K], 16) : w[4 + i - K];
}
// store8 for rows of any alignment, by a whole warp.  Where its lanes hold neighbouring vectors of one row (`same`), the aligned 16 bytes that two
// neighbours share are put together from both, so that nearly all is written 16 bytes at a time: 16-bit entries one by one took six times as long
// (16384 x 8191 bf16 read back from codes: 364 us).
template <int KIND>
__device__ __forceinline__ void store8_any(const RowsOf& t, int64_t row, int c, int n, const float (&v)[8], bool same) {
  if (KIND == LS_F32 || t.al >= 4 || !same) { store8<KIND, false>(t, row, c, n, v); return; }
  uint16_t* p = reinterpret_cast<uint16_t*>(t.p) + row * t.ld + c;
  const int m = __shfl_sync(0xffffffffu, (int)(reinterpret_cast<uintptr_t>(p) & 15), 0);      // bytes, the same for all lanes
  uint32_t w[8];                                                                              // the neighbour's words, then this lane's
#pragma unroll
  for (int i = 0; i < 4; ++i) { w[4 + i] = narrow2<KIND>(v[2 * i], v[2 * i + 1]); w[i] = __shfl_up_sync(0xffffffffu, w[4 + i], 1); }
  const bool full = n == 8;
  const int lane = threadIdx.x & 31;
  const uint32_t all = __ballot_sync(0xffffffffu, full);
  const bool before = lane > 0 && (all >> (lane - 1) & 1), behind = lane < 31 && (all >> (lane + 1) & 1);
  if (full && before) {
    uint32_t o[4];
    if (m < 4) shifted4<0>(w, m, o); else if (m < 8) shifted4<1>(w, m, o); else if (m < 12) shifted4<2>(w, m, o); else shifted4<3>(w, m, o);
    st_stream(reinterpret_cast<uint4*>(p - m / 2), make_uint4(o[0], o[1], o[2], o[3]));
  }
  // what no pair of neighbours covers: the first lane's head, the last full one's tail, a row's last entries
  const int from = full && before ? 8 - m / 2 : 0, to = full && behind ? 8 - m / 2 : n;
  if (from < to) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= from && i < to) p[i] = (uint16_t)(w[4 + i / 2] >> (16 * (i & 1)));
  }
}
// rounded to the storage type and back
template <int KIND>
__device__ __forceinline__ void round8(float (&v)[8]) {
  if (KIND != LS_F32) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) { const float2 q = widen2<KIND>(narrow2<KIND>(v[i], v[i + 1])); v[i] = q.x; v[i + 1] = q.y; }
  }
}

// Codes of 8 entries; the four threads of a block of 32 (lanes 4 i to 4 i + 3) call it together, with the whole warp.
// The integer of v 2^-e stands in the low bits of v 2^-e + 1.5 * 2^23.  Only a block whose largest entry is within 1/256 of the next power of two
// can have codes beyond 127; the test for that is one for the warp, so that the usual path has no clamp per entry.
__device__ __forceinline__ uint2 pack8(const float (&v)[8], uint32_t& byte) {
  float m = fabsf(v[0]);
#pragma unroll
  for (int i = 1; i < 8; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(fabsf(v[i])));
  uint32_t top = __float_as_uint(m);                     // as integers from here: NaN above infinity above the rest
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const int e = (int)(top >> 23);
  byte = e == 255 ? 255u : (top == 0 ? 0u : (uint32_t)max(e - 6, 1));
  const float up = __uint_as_float((254u - (e == 255 ? 1u : byte)) << 23);              // 2^(127 - byte)
  uint32_t q[8];
  if (__any_sync(0xffffffffu, (top & 0x7fffffu) >= 0x7f0000u)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = __float_as_uint(fminf(fmaxf(v[i] * up, -127.f), 127.f) + 12582912.f);
  } else {
    const uint64_t u2 = pk2(up, up), magic = pk2(12582912.f, 12582912.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = upk2(fma2(pk2(v[2 * i], v[2 * i + 1]), u2, magic));
      q[2 * i] = __float_as_uint(f.x); q[2 * i + 1] = __float_as_uint(f.y);
    }
  }
  uint2 w;
  w.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
  w.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
  if (e == 255) w = make_uint2(0u, 0u);
  return w;
}
__device__ __forceinline__ void unpack8(uint2 w, uint32_t byte, float (&v)[8]) {
  const float s = __uint_as_float(byte << 23);
  const uint64_t scale = pk2(s, s), off = pk2(-8388736.f, -8388736.f);                  // 2^23 + 128
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = (i < 2 ? w.x : w.y) ^ 0x80808080u;                               // code + 128
    const uint64_t c = pk2(__uint_as_float(__byte_perm(x, 0x4b000000u, 0x7440 + 2 * (i & 1))), __uint_as_float(__byte_perm(x, 0x4b000000u, 0x7441 + 2 * (i & 1))));
    const float2 f = upk2(mul2(add2(c, off), scale));
    v[2 * i] = f.x; v[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint2 ld_codes(const unsigned char* p) {
  uint2 v;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

// An item is 8 entries of a row, numbered through the rows: item i has its codes at byte 8 i.
struct ItemWalk {
  int64_t items;         // rows * per_row
  int width, per_row;    // items of a row: 4 * blocks
  uint32_t magic, shift; // i / per_row = (i magic) >> (32 + shift) for i < 2^31: with l = ceil(log2 per_row), magic = ceil(2^(31 + l) / per_row), shift = l - 1
};
__device__ __forceinline__ void item_place(const ItemWalk& k, int64_t i, int64_t& row, int& v) {
  if (k.items <= 0x7fffffffll) { const uint32_t r = __umulhi((uint32_t)i, k.magic) >> k.shift; row = r; v = (int)((uint32_t)i - r * (uint32_t)k.per_row); }
  else { row = i / k.per_row; v = (int)(i - row * k.per_row); }
}
__device__ __forceinline__ bool one_row(int64_t row) { return __all_sync(0xffffffffu, row == __shfl_sync(0xffffffffu, row, 0)); }
// entries of item v of a row that exist
__device__ __forceinline__ int item_count(const ItemWalk& k, int v) { return max(0, min(8, k.width - 8 * v)); }

__device__ __forceinline__ void store_packed(const PackedRows& t, int64_t row, int v, int64_t item, uint2 codes, uint32_t byte) {
  asm volatile("st.global.L1::no_allocate.v2.u32 [%0], {%1,%2};" ::"l"(t.codes + item * 8), "r"(codes.x), "r"(codes.y) : "memory");
  if ((v & 3) == 0) {
    unsigned char* e = t.exps + row * t.exp_stride;
    e[v >> 2] = (unsigned char)byte;
    if ((v >> 2) == t.blocks - 1)
      for (int k = t.blocks; k < t.exp_stride; ++k) e[k] = 0;
  }
}

// (one vector a thread: 16384 x 8192 bf16 88 us, 97 with two, 122 with four; threads to switch between count for more than loads of one thread)
template <int KIND, bool ALIGNED>
__global__ void __launch_bounds__(PK_THREADS, KIND != LS_F32 ? (ALIGNED ? PK_BLOCKS : PK_BLOCKS_ODD) : 1) pack_kernel(const RowsOf x, const PackedRows out, const ItemWalk k) {
  griddep_chain();
  const int64_t i = (int64_t)blockIdx.x * PK_THREADS + threadIdx.x;
  float v[8];
  int64_t row;
  int at;
  item_place(k, min(i, k.items - 1), row, at);
  load8<KIND, ALIGNED>(x, row, 8 * at, i < k.items ? item_count(k, at) : 0, v);
  uint32_t byte;
  const uint2 w = pack8(v, byte);
  if (i < k.items) store_packed(out, row, at, i, w, byte);
}

template <int KIND, bool ALIGNED, int U>
__global__ void __launch_bounds__(PK_THREADS) unpack_kernel(const PackedRows in, const RowsOf x, const ItemWalk k) {
  griddep_chain();
  const int64_t first = (int64_t)blockIdx.x * (PK_THREADS * U) + threadIdx.x;
  uint2 w[U];
  uint32_t byte[U];
  int64_t row[U];
  int at[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int64_t i = min(first + j * PK_THREADS, k.items - 1);
    item_place(k, i, row[j], at[j]);
    w[j] = ld_codes(in.codes + i * 8);
    byte[j] = in.exps[row[j] * in.exp_stride + (at[j] >> 2)];
  }
#pragma unroll
  for (int j = 0; j < U; ++j) {
    float v[8];
    unpack8(w[j], byte[j], v);
    const int n = first + j * PK_THREADS < k.items ? item_count(k, at[j]) : 0;
    if (ALIGNED) store8<KIND, true>(x, row[j], 8 * at[j], n, v);
    else store8_any<KIND>(x, row[j], 8 * at[j], n, v, one_row(row[j]));
  }
}

// ---- gated activation ----
// y = act(a) u.  With p the activation's gate (the logistic function of z(a), or the normal distribution at a for GELU), act(a) = a p and
//   act'(a) = p + a p (1 - p) z'(a),   act'(a) = p + a exp(-a^2 / 2) / sqrt(2 pi)  for GELU;
// the tanh form of GELU is a p with z = 2 sqrt(2 / pi) (a + 0.044715 a^3), since (1 + tanh w) / 2 = 1 / (1 + exp(-2 w)).  With
// t = exp(-|z|) the logistic function is 1 / (1 + t) or t / (1 + t) and p (1 - p) = t / (1 + t)^2: nothing cancels or overflows.
enum { ACT_SILU = 0, ACT_GELU = 1, ACT_GELU_TANH = 2 };

// p; s: act'(a)
template <int ACT>
__device__ __forceinline__ float act_gate(float a, float& s) {
  if (ACT == ACT_GELU) {
    const float p = 0.5f * erfcf(a * -0.70710678118654752f);
    s = fmaf(a * 0.3989422804014327f, __expf(-0.5f * a * a), p);
    return p;
  }
  const float z = ACT == ACT_SILU ? a : 1.5957691216057308f * fmaf(0.044715f * a * a, a, a);
  float r;
  const float t = __expf(-fabsf(z));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + t));      // of a number from 1 to 2
  const float tr = t * r, q = tr * r;
  const float p = z < 0.f ? tr : r;
  if (ACT == ACT_SILU) s = fmaf(a, q, p);
  else s = q == 0.f ? p : fmaf(a * q, 1.5957691216057308f * fmaf(0.134145f * a, a, 1.f), p);      // far out z' overflows where q is 0
  return p;
}

struct GatedArgs {
  RowsOf a, u, y;            // forward; u.p null: y = act(a)
  RowsOf dy, da, du;         // backward
  PackedRows pa, pu, py;     // kept inputs; py.codes null: not wanted
};

template <int KIND, int ACT, bool GATED, bool ALIGNED>
__global__ void __launch_bounds__(PK_THREADS, KIND != LS_F32 ? (ALIGNED ? PK_BLOCKS : PK_BLOCKS_ODD) : 1) gated_kernel(const GatedArgs g, const ItemWalk k) {
  griddep_chain();
  const int64_t i = (int64_t)blockIdx.x * PK_THREADS + threadIdx.x;
  float a[8], u[8];
  int64_t row;
  int at;
  item_place(k, min(i, k.items - 1), row, at);
  const int n = i < k.items ? item_count(k, at) : 0;
  load8<KIND, ALIGNED>(g.a, row, 8 * at, n, a);
  if (GATED) load8<KIND, ALIGNED>(g.u, row, 8 * at, n, u);
  if (g.pa.codes) {
    uint32_t byte;
    uint2 w = pack8(a, byte);
    if (i < k.items) store_packed(g.pa, row, at, i, w, byte);
    if (GATED) {
      w = pack8(u, byte);
      if (i < k.items) store_packed(g.pu, row, at, i, w, byte);
    }
  }
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float s;
    y[e] = a[e] * act_gate<ACT>(a[e], s);
    if (GATED) y[e] *= u[e];
  }
  if (ALIGNED) store8<KIND, true>(g.y, row, 8 * at, n, y);
  else store8_any<KIND>(g.y, row, 8 * at, n, y, one_row(row));
}

template <int KIND, int ACT, bool GATED, bool ALIGNED>
__global__ void __launch_bounds__(PK_THREADS, KIND != LS_F32 ? (ALIGNED ? PK_BLOCKS : PK_BLOCKS_ODD) : 1) gated_backward_kernel(const GatedArgs g, const ItemWalk k) {
  griddep_chain();
  const int64_t item = (int64_t)blockIdx.x * PK_THREADS + threadIdx.x, i = min(item, k.items - 1);
  float dy[8], a[8], u[8], f[8];
  int64_t row;
  int at;
  item_place(k, i, row, at);
  const uint2 wa = ld_codes(g.pa.codes + i * 8);
  const uint32_t ba = g.pa.exps[row * g.pa.exp_stride + (at >> 2)];
  uint2 wu;
  uint32_t bu;
  if (GATED) {
    wu = ld_codes(g.pu.codes + i * 8);
    bu = g.pu.exps[row * g.pu.exp_stride + (at >> 2)];
  }
  load8<KIND, ALIGNED>(g.dy, row, 8 * at, item_count(k, at), dy);
  const int n = item < k.items ? item_count(k, at) : 0;
  unpack8(wa, ba, a);
  if (GATED) unpack8(wu, bu, u);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float s;
    const float p = act_gate<ACT>(a[e], s);
    f[e] = a[e] * p;
    a[e] = GATED ? dy[e] * u[e] * s : dy[e] * s;
    if (GATED) { dy[e] *= f[e]; f[e] *= u[e]; }
  }
  if (ALIGNED) {
    store8<KIND, true>(g.da, row, 8 * at, n, a);
    if (GATED) store8<KIND, true>(g.du, row, 8 * at, n, dy);
  } else {
    const bool same = one_row(row);
    store8_any<KIND>(g.da, row, 8 * at, n, a, same);
    if (GATED) store8_any<KIND>(g.du, row, 8 * at, n, dy, same);
  }
  if (g.py.codes) {
    round8<KIND>(f);
    uint32_t byte;
    const uint2 w = pack8(f, byte);
    if (item < k.items) store_packed(g.py, row, at, item, w, byte);
  }
}

}  // namespace tg
