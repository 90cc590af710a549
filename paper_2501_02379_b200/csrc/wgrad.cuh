// Weight gradient of a linear layer whose input was kept in 8 bits:  dW[n][k] = sum over tokens m of dy[m][n] x^[m][k].
//
// A matrix product whose contraction runs over the rows of both operands, on the 5th-generation tensor cores: per tile of 128 columns of dy
// by 128 of x and step of 64 tokens,
//   * one thread loads dy's box (64 tokens of two times 64 entries, 128-byte swizzle) and the codes' (64 tokens of 128 bytes) by tiled TMA,
//     a warp the blocks' bytes (a word a token);
//   * four warps turn the codes into 16-bit numbers in the layout that the tensor core reads: x^ = code 2^e has 7 bits, so it is exact in
//     bfloat16, and in fp16 for what was packed from fp16; products are exact in fp32;
//   * one thread issues tcgen05.mma (both operands with the tile's columns contiguous), accumulators in tensor memory;
//   * eight warps move the sums out.  The tensor core adds with truncation, which would bias a long sum, so where the result is fp32 it leaves
//     tensor memory after every few steps and is added up in registers; a 16-bit result stays there for the whole sum.
// fp32 dy is split beforehand into three bfloat16 parts that add up to it exactly, which are three times as many steps into the same sums;
// 16-bit dy that TMA cannot address (rows that do not start at multiples of 16 bytes) is copied beforehand.
// Few tiles and many tokens: the tokens are split between blocks, whose sums a second launch adds in a fixed order.
// Every wait is bounded; one that ran out leaves NaN in the tiles that its block did not finish.
#pragma once
#include <cuda.h>
#include "norms.cuh"

namespace tg {

constexpr int WG_THREADS = 512;        // warp 0: TMA, 1: MMA issue, 2: the blocks' bytes, 3: tensor memory, 4-7: codes to numbers, 8-15: sums
constexpr int WG_TOKENS = 64, WG_TILE = 128;
constexpr int WG_BOX = 64 * 128;                                  // bytes of 64 tokens by 64 16-bit entries
constexpr int WG_A = 0, WG_B = 2 * WG_BOX, WG_CODES = 4 * WG_BOX, WG_EXPS = 5 * WG_BOX, WG_STAGE = 5 * WG_BOX + 1024;
constexpr int WG_STAGES = 5;
constexpr int WG_NUMBER_THREADS = 128, WG_SUM_THREADS = 256;
constexpr size_t WG_SMEM = (size_t)WG_STAGES * WG_STAGE + 1024;
constexpr uint32_t WG_WAIT_POLLS = 1u << 22;
constexpr uint64_t WG_WAIT_NS = 500000000ull;

struct WgradArgs {
  const unsigned char* exps;
  int exp_words;             // 4-byte words of bytes per token
  int64_t tokens;
  int terms;                 // parts of dy (3 for fp32)
  int N, K;
  int tiles_n, tiles_k, splits;
  int64_t steps, per_split;  // steps of the whole contraction and of a split
  int group;                 // steps between two moves of the sums
  RowsOf out;
  int out_kind, accumulate;
  float* partial;            // [splits][128 tiles_n][128 tiles_k]
};

__device__ __forceinline__ bool wg_wait(uint64_t* bar, uint32_t parity, volatile int* failed) {
  uint64_t start = 0;
  for (uint32_t i = 0; i < WG_WAIT_POLLS; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((i & 63) == 63) {
      if (*failed) return false;
      uint64_t now;
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
      if (start == 0) start = now;
      else if (now - start > WG_WAIT_NS) break;
    }
  }
  *failed = 1;
  return false;
}

// Descriptor of a tile whose columns are contiguous (128-byte swizzle): groups of 64 columns WG_BOX bytes apart, groups of 8 tokens 1,024.
__device__ __forceinline__ uint64_t umma_desc_mn128(uint32_t smem_addr) {
  uint64_t d = (uint64_t)((smem_addr & 0x3ffffu) >> 4);
  d |= (uint64_t)(WG_BOX >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// tile number -> place: bands of 8 tiles of dy's columns, so that the tiles in flight share their operands in the L2 cache
__device__ __forceinline__ void wg_tile(const WgradArgs& A, int tile, int& tn, int& tk) {
  const int per = 8 * A.tiles_k, band = tile / per, in = tile - band * per, height = min(8, A.tiles_n - 8 * band);
  tk = in / height;
  tn = 8 * band + (in - tk * height);
}

// 8 codes to 8 numbers, exact.  The low seven bits of a code stand as mantissa behind 128 (bfloat16 0x4300), the sign bit in the number
// that is taken from it (128, or 256 with the lowest exponent bit set).
template <bool F16>
__device__ __forceinline__ uint4 wg_numbers(uint2 w, uint32_t byte) {
  uint32_t r[4];
  if (F16) {
    float v[8];
    unpack8(w, byte, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = narrow2<LS_F16>(v[2 * i], v[2 * i + 1]);
  } else {
    const uint32_t s = byte * 0x00800080u;             // 2^e twice
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t t = __byte_perm(i < 2 ? w.x : w.y, 0u, i & 1 ? 0x4342 : 0x4140);
      const uint32_t m = (t & 0x007f007fu) | 0x43004300u, o = (t & 0x00800080u) | 0x43004300u;
      __nv_bfloat162 q = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&m), *reinterpret_cast<const __nv_bfloat162*>(&o));
      q = __hmul2(q, *reinterpret_cast<const __nv_bfloat162*>(&s));
      r[i] = *reinterpret_cast<const uint32_t*>(&q);
    }
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

template <int KIND>
__device__ __forceinline__ void wg_store(const WgradArgs& A, int64_t n, int k, const float* v) {
  float o[8];
  const int cnt = max(0, min(8, A.K - k));
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = v[i];
  if (A.accumulate) {
    float u[8];
    load8<KIND, false>(A.out, n, k, cnt, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] += u[i];
  }
  store8<KIND, false>(A.out, n, k, cnt, o);
}

template <bool F16>
__global__ void __launch_bounds__(WG_THREADS, 1) wgrad_kernel(const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_codes, const WgradArgs A) {
  extern __shared__ unsigned char wg_raw[];
  __shared__ __align__(8) uint64_t full[WG_STAGES], ready[WG_STAGES], empty[WG_STAGES], acc_full[2], acc_free[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int failed_s;
  volatile int* failed = &failed_s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t raw = smem_u32(wg_raw), stage0 = (raw + 1023u) & ~1023u;

  if (tid == 0) {
    for (int s = 0; s < WG_STAGES; ++s) { mbar_init(&full[s], 33); mbar_init(&ready[s], WG_NUMBER_THREADS); mbar_init(&empty[s], 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_free[b], WG_SUM_THREADS); }
    failed_s = 0;
    fence_mbar_init();
  }
  if (warp == 3) { tmem_alloc(&tmem_slot, 256); tmem_relinquish(); }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = tmem_slot;
  griddep_chain();

  const int tiles = A.tiles_n * A.tiles_k, units = tiles * A.splits;
  // what a unit (a tile and a part of the tokens) is
  auto steps_of = [&](int unit, int64_t& from) {
    const int64_t sp = unit / tiles;
    from = sp * A.per_split;
    return (uint32_t)max((int64_t)0, min(A.per_split, A.steps - from));
  };

  if (warp == 0) {
    if (lane == 0) {
      uint32_t g = 0;                                    // steps so far: stage g % STAGES, round g / STAGES
      for (int unit = blockIdx.x; unit < units && !*failed; unit += gridDim.x) {
        int tn, tk; wg_tile(A, unit % tiles, tn, tk);
        int64_t from; const uint32_t n = steps_of(unit, from);
        for (uint32_t it = 0; it < n; ++it, ++g) {
          const int s = g % WG_STAGES;
          if (!wg_wait(&empty[s], ((g / WG_STAGES) & 1) ^ 1, failed)) break;
          const int64_t step = from + it;
          const int chunk = (int)(step / A.terms), term = (int)(step - (int64_t)chunk * A.terms);
          const uint32_t at = stage0 + s * WG_STAGE;
          mbar_expect_tx(&full[s], 3 * WG_BOX);
          tma_load_3d(at + WG_A, &map_dy, tn * WG_TILE, chunk * WG_TOKENS, term, &full[s]);
          tma_load_3d(at + WG_A + WG_BOX, &map_dy, tn * WG_TILE + 64, chunk * WG_TOKENS, term, &full[s]);
          tma_load_3d(at + WG_CODES, &map_codes, tk * WG_TILE, chunk * WG_TOKENS, 0, &full[s]);
        }
      }
      // copies still under way must land before the block's shared memory is given up (only after a wait that ran out)
      if (*failed)
        for (uint32_t j = g > WG_STAGES ? g - WG_STAGES : 0; j < g; ++j) mbar_wait_bounded(&full[j % WG_STAGES], (j / WG_STAGES) & 1, 1u << 16);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      // fp32 accumulator, both operands with their columns contiguous (bits 15, 16), 128 x 128
      const uint32_t idesc = umma_idesc(F16 ? 0 : 1, WG_TILE) | (1u << 15) | (1u << 16);
      uint32_t g = 0, moves = 0;
      for (int unit = blockIdx.x; unit < units && !*failed; unit += gridDim.x) {
        int64_t from; const uint32_t n = steps_of(unit, from);
        uint32_t in_group = 0;
        for (uint32_t it = 0; it < n; ++it, ++g) {
          const uint32_t b = moves & 1;
          if (in_group == 0 && !wg_wait(&acc_free[b], ((moves >> 1) & 1) ^ 1, failed)) break;
          const int s = g % WG_STAGES;
          if (!wg_wait(&ready[s], (g / WG_STAGES) & 1, failed)) break;
          tc_fence_after_sync();
          const uint32_t at = stage0 + s * WG_STAGE;
          const uint64_t da = umma_desc_mn128(at + WG_A), db = umma_desc_mn128(at + WG_B);
#pragma unroll
          for (int ks = 0; ks < WG_TOKENS / 16; ++ks)      // 16 tokens: two groups of 8
            umma_ss<false>(tmem + b * WG_TILE, da + (uint64_t)(ks * 2048 >> 4), db + (uint64_t)(ks * 2048 >> 4), idesc, in_group != 0 || ks != 0);
          umma_commit(&empty[s]);
          if (++in_group == (uint32_t)A.group || it + 1 == n) { umma_commit(&acc_full[b]); in_group = 0; ++moves; }
        }
      }
    }
    __syncwarp();
  } else if (warp == 2) {
    uint32_t g = 0;
    for (int unit = blockIdx.x; unit < units && !*failed; unit += gridDim.x) {
      int tn, tk; wg_tile(A, unit % tiles, tn, tk);
      int64_t from; const uint32_t n = steps_of(unit, from);
      for (uint32_t it = 0; it < n; ++it, ++g) {
        const int s = g % WG_STAGES;
        if (!wg_wait(&empty[s], ((g / WG_STAGES) & 1) ^ 1, failed)) break;
        const int64_t m0 = (from + it) / A.terms * WG_TOKENS;
        unsigned char* to = wg_raw + (stage0 - raw) + s * WG_STAGE + WG_EXPS;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int64_t m = m0 + lane + 32 * h;
          const bool in = m < A.tokens && tk < A.exp_words;
          cp_async4(to + 4 * (lane + 32 * h), A.exps + (in ? (m * A.exp_words + tk) * 4 : 0), in ? 4 : 0);
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&full[s])) : "memory");
      }
    }
    cp_async_wait<0>();
  } else if (warp >= 4 && warp < 8) {
    const int w = tid - 128;
    const int q = w & 15, m_first = w >> 4;              // this thread: columns 8 q .. 8 q + 7 of tokens m_first + 8 i
    uint32_t g = 0;
    for (int unit = blockIdx.x; unit < units && !*failed; unit += gridDim.x) {
      int64_t from; const uint32_t n = steps_of(unit, from);
      for (uint32_t it = 0; it < n; ++it, ++g) {
        const int s = g % WG_STAGES;
        if (!wg_wait(&full[s], (g / WG_STAGES) & 1, failed)) break;
        const uint32_t at = stage0 + s * WG_STAGE;
        uint2 c[8];
        uint32_t e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int m = m_first + 8 * i;
          c[i] = lds64(at + WG_CODES + m * 128 + q * 8);
          e[i] = lds32(at + WG_EXPS + m * 4);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int m = m_first + 8 * i;
          const uint4 r = wg_numbers<F16>(c[i], (e[i] >> (8 * (q >> 2))) & 255u);
          const uint32_t to = at + WG_B + (q >> 3) * WG_BOX + m * 128 + (((q & 7) ^ (m & 7)) << 4);
          asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w) : "memory");
        }
        fence_async_smem();
        mbar_arrive(&ready[s]);
      }
    }
  } else if (warp >= 8) {
    const int quarter = warp & 3, half = (warp - 8) >> 2;  // tensor-memory lanes 32 * quarter .., columns 64 * half ..
    uint32_t moves = 0;
    for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
      int tn, tk; wg_tile(A, unit % tiles, tn, tk);
      int64_t from; const uint32_t n = steps_of(unit, from);
      const uint32_t groups = (n + A.group - 1) / A.group;
      float sum[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) sum[i] = 0.f;
      for (uint32_t k = 0; k < groups; ++k, ++moves) {
        const uint32_t b = moves & 1;
        const bool ok = wg_wait(&acc_full[b], (moves >> 1) & 1, failed);
        if (!__all_sync(0xffffffffu, ok)) {
#pragma unroll
          for (int i = 0; i < 64; ++i) sum[i] = __int_as_float(0x7fffffff);
          break;
        }
        tc_fence_after_sync();
        const uint32_t ta = tmem + b * WG_TILE + half * 64 + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          uint32_t r[16];
          tmem_ld16(ta + 16 * p, r);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[16 * p + i] += __uint_as_float(r[i]);
        }
        tc_fence_before_sync();
        mbar_arrive(&acc_free[b]);
      }
      const int64_t row = (int64_t)tn * WG_TILE + quarter * 32 + lane;
      const int col = tk * WG_TILE + half * 64;
      if (A.partial) {
        float4* p = reinterpret_cast<float4*>(A.partial + (((int64_t)(unit / tiles) * A.tiles_n * WG_TILE + row) * A.tiles_k) * WG_TILE + col);
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = make_float4(sum[4 * i], sum[4 * i + 1], sum[4 * i + 2], sum[4 * i + 3]);
      } else if (row < A.N) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (A.out_kind == LS_F32) wg_store<LS_F32>(A, row, col + 8 * i, sum + 8 * i);
          else if (A.out_kind == LS_F16) wg_store<LS_F16>(A, row, col + 8 * i, sum + 8 * i);
          else wg_store<LS_BF16>(A, row, col + 8 * i, sum + 8 * i);
        }
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 3) tmem_dealloc(tmem, 256);
}

// dW from the splits' sums: 8 entries a thread, the splits in order.
__global__ void __launch_bounds__(256) wgrad_sum_kernel(const WgradArgs A) {
  griddep_chain();
  const int per = (A.K + 7) / 8;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)A.N * per) return;
  const int64_t n = i / per;
  const int k = (int)(i - n * per) * 8;
  const int64_t ld = (int64_t)A.tiles_k * WG_TILE, size = (int64_t)A.tiles_n * WG_TILE * ld;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < A.splits; ++s) {
    const float4* p = reinterpret_cast<const float4*>(A.partial + s * size + n * ld + k);
    const float4 a = p[0], b = p[1];
    v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
  }
  if (A.out_kind == LS_F32) wg_store<LS_F32>(A, n, k, v);
  else if (A.out_kind == LS_F16) wg_store<LS_F16>(A, n, k, v);
  else wg_store<LS_BF16>(A, n, k, v);
}

// dy in parts that TMA can address: [terms][tokens][ld] 16-bit, ld a multiple of 8.  fp32 in three bfloat16 parts, each but the last one cut
// off behind its 8 bits, so that they add up to it exactly.
template <int KIND>
__global__ void __launch_bounds__(256) wgrad_parts_kernel(const RowsOf dy, int64_t tokens, int N, int ld, uint16_t* out) {
  griddep_chain();
  const int per = ld / 8;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= tokens * per) return;
  const int64_t m = i / per;
  const int c = (int)(i - m * per) * 8;
  float v[8];
  load8<KIND, false>(dy, m, c, max(0, min(8, N - c)), v);
  uint16_t* to = out + m * ld + c;
  if (KIND != LS_F32) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = narrow2<KIND>(v[2 * j], v[2 * j + 1]);
    *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
    return;
  }
  const int64_t part = tokens * ld;
#pragma unroll
  for (int term = 0; term < 3; ++term) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool finite = (__float_as_uint(v[j]) & 0x7f800000u) != 0x7f800000u;
      uint32_t h = __float_as_uint(v[j]) >> 16;
      if (!finite && (__float_as_uint(v[j]) & 0x7fffffu)) h = 0x7fff;
      if (term == 2 && finite) { const __nv_bfloat16 r = __float2bfloat16_rn(v[j]); h = *reinterpret_cast<const uint16_t*>(&r); }
      v[j] = finite ? v[j] - __uint_as_float(h << 16) : 0.f;      // (infinity and NaN stand in the first part alone)
      w[j >> 1] = j & 1 ? w[j >> 1] | (h << 16) : h;
    }
    *reinterpret_cast<uint4*>(to + term * part) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

}  // namespace tg
