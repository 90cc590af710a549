// Weight gradient of a linear layer whose input was kept in 8 bits:  dW[n][k] = sum over tokens m of dy[m][n] x^[m][k].
//
// A matrix product whose contraction runs over the rows of both operands, on the 5th-generation tensor cores.  Two blocks on neighbouring SMs
// (a cluster, tcgen05 with cta_group::2) share a tile of 256 columns of dy by TN of x; each holds 128 of dy's and TN / 2 of x's.  Per
// step of 64 tokens (128 where TN is 128), in each block:
//   * one thread loads dy's boxes (64 tokens of 64 entries, 128-byte swizzle) and the codes' (64 tokens) by tiled TMA, a warp the blocks'
//     bytes (a word a token);
//   * eight warps (four where TN is 128) turn the codes into 16-bit numbers in the layout that the tensor core reads: x^ = code 2^e has 7 bits, so it is exact in
//     bfloat16, and in fp16 for what was packed from fp16; products are exact in fp32.  Two such groups take steps in turn, so that one's
//     latencies are covered by the other's;
//   * in the first block one thread issues tcgen05.mma for both (operands with the tile's columns contiguous), accumulators in tensor memory;
//   * eight warps move the sums out.  The tensor core adds with truncation, which biases a long sum (by 1e-7 an instruction where the terms have one
//     sign: 7.8e-4 after 7500, more than half an ulp of fp16), so sums of a few steps leave it and are added in fp32: for an fp32 result after 32
//     instructions (16 where the entries are fp32), into registers (TN = 128: as many as fit); for a 16-bit result (TN = 256) after 256, into the
//     other half of tensor memory (1.7e-5 at most).  A 16-bit sum of 64 steps or fewer stays, and tensor memory holds a second tile meanwhile.
// Bound by the warps that turn codes into numbers: a group takes about 1,000 clocks for a step, 500 a step for the two, and the tensor
// cores of two SMs 512 for 64 x 256 x 256; measured 450 ns a step for 270 of tensor cores (8192 x 2048 x 4608 bf16: 116 us, 1,335 TFLOP/s,
// tensor pipe 73 % busy, the pipe of integer and logic instructions 65 %; to fp32 148 us; 16384 x 4096 x 14336: 1.72 ms at sustained clocks).  Two blocks and
// not one: each turns half of the columns into numbers, and a tile of 128 x 128 on one SM would have to read its operands from shared
// memory as fast as that allows (16384 x 4096 x 14336 that way: 3.57 ms).
// fp32 dy is split beforehand into three bfloat16 parts that add up to it exactly, which are three times as many steps into the same sums;
// 16-bit dy that TMA cannot address (rows that do not start at multiples of 16 bytes) is copied beforehand.
// The tiles behind the last full round of the clusters (all, where there are few): their tokens are split between clusters, whose sums a second
// launch adds in a fixed order.  (16384 x 4096 x 14336 has 896 tiles for 74 clusters: 12 rounds and 8 tiles.)
// Every wait is bounded; one that ran out leaves NaN in the tiles that its block did not finish.
#pragma once
#include <cuda.h>
#include "norms.cuh"

namespace tg {

constexpr int WG_TILE_N = 256;
// Warp 0: TMA, 1: MMA issue, 2: the blocks' bytes, 3: tensor memory, then two groups of NW that turn codes into numbers, then 8 for the sums.
// Rings of shared memory, for three lifetimes: dy's boxes from their copy to the end of the instructions that read them, codes from their copy
// until they are numbers (the first two of one depth, so that one barrier stands for both copies), numbers from then to the end of the instructions.
template <int TN> struct WgGeom {
  static constexpr int TOKENS = TN == 256 ? 64 : 128;             // of a step: 16 KB of numbers for a block either way
  static constexpr int BOX = TOKENS * 128;                        // bytes of a step's tokens by 64 16-bit entries
  static constexpr int H = TN / 2;                                // columns of x of a block
  static constexpr int NW = TN == 256 ? 8 : 4, THREADS = 32 * (4 + 2 * NW + 8);      // (with fp32 sums, 96 registers a thread)
  static constexpr int SA = TN == 256 ? 6 : 4, SB = TN == 256 ? 4 : 3;      // places for copies (dy's and codes'), for numbers
  static constexpr int A_BYTES = 2 * BOX, B_BYTES = H * TOKENS * 2, C_BYTES = H * TOKENS, E_BYTES = TOKENS * 4;
  static constexpr int B = SA * A_BYTES, C = B + SB * B_BYTES, E = C + SA * C_BYTES;      // dy's ring stands first
  static constexpr size_t SMEM = (size_t)E + SA * E_BYTES + 1024;
};
constexpr uint32_t WG_WAIT_POLLS = 1u << 22;
constexpr uint64_t WG_WAIT_NS = 500000000ull;

struct WgradArgs {
  const unsigned char* exps;
  int exp_words;             // 4-byte words of bytes per token
  int64_t tokens;
  int terms;                 // parts of dy (3 for fp32)
  int N, K;
  int tiles_n, tiles_k;
  int whole, splits;         // tiles whose sums one cluster forms; parts of the tokens of the others
  int64_t steps, per_split;  // steps of the whole contraction and of a part
  int group;                 // steps between two moves of the sums
  int copies;                // for tests: steps that a block copies at most
  RowsOf out;
  int out_kind, accumulate;
  float* partial;            // [splits][tiles - whole][256][TN]
};

// ---- two blocks as one ----
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// an arrival at the first block's barrier that stands where `bar` stands in this block.  (Without .release.cluster, which would have the
// thread wait until its writes are visible in the whole cluster: 600 instead of 1,020 TFLOP/s at 8192 x 2048 x 4608.  What the tensor core
// reads has been written in its own SM's shared memory and passed the proxy fence, which is what orders it.)
__device__ __forceinline__ void arrive_first(uint64_t* bar) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(smem_u32(bar)));
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(a) : "memory");
}
__device__ __forceinline__ void tmem_alloc2(uint32_t* smem_result, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(smem_result)), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc2(uint32_t taddr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
__device__ __forceinline__ void umma2_f16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, bool accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"((uint32_t)accumulate)
               : "memory");
}
// 16 consecutive columns of this thread's lane from registers.  Whole warp.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]),
      "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// both blocks' barriers that stand at `bar` get an arrival once every MMA issued so far has completed
__device__ __forceinline__ void umma2_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}

// Waits of whole warps: the result is the same in all lanes, and known to be by the compiler.  What one thread does for its block (copies,
// tensor-core instructions, their commits) stands in loops that whole warps run and is done by an elected lane: these instructions take
// their operands from registers of the warp, and in code that the compiler holds for divergent it moves each there by a loop of its own
// (measured with `if (lane == 0)` around the loops: 870 clocks for the instructions of a step).
static __device__ __noinline__ bool wg_wait_long(uint64_t* bar, uint32_t parity, volatile int* failed) {
  uint64_t start = 0;
  for (uint32_t i = 0; i < WG_WAIT_POLLS; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((i & 15) == 15) {
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
__device__ __forceinline__ bool wg_wait(uint64_t* bar, uint32_t parity, volatile int* failed) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  const bool ok = wg_wait_long(bar, parity, failed);
  __syncwarp();
  return __all_sync(0xffffffffu, ok);
}
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
// Place in a ring of N and the parity of its barriers.
template <int N>
struct WgRing {
  uint32_t at = 0, parity = 0;
  __device__ __forceinline__ void next(uint32_t by = 1) { if ((at += by) >= N) { at -= N; parity ^= 1; } }
};

// Descriptor of a tile whose columns are contiguous (128-byte swizzle): groups of 64 columns `box` bytes apart, groups of 8 tokens 1,024.
__device__ __forceinline__ uint64_t umma_desc_mn128(uint32_t smem_addr, uint32_t box) {
  uint64_t d = (uint64_t)((smem_addr & 0x3ffffu) >> 4);
  d |= (uint64_t)(box >> 4) << 16;
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
// that is taken from it (128, or 256 with the lowest exponent bit set).  byte: the block's, in both halves of the word.
template <bool F16>
__device__ __forceinline__ uint4 wg_numbers(uint2 w, uint32_t byte) {
  uint32_t r[4];
  if (F16) {
    float v[8];
    unpack8(w, byte & 255u, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = narrow2<LS_F16>(v[2 * i], v[2 * i + 1]);
  } else {
    const uint32_t s = byte << 7;                      // 2^e, twice
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

// RUNNING (TN = 256): a unit has more than one group, and half of tensor memory holds the running sums instead of a second accumulator.
template <bool F16, int TN, bool RUNNING>
__global__ void __launch_bounds__(WgGeom<TN>::THREADS, 1) wgrad_kernel(const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_codes, const WgradArgs A) {
  typedef WgGeom<TN> G;
  constexpr int SA = G::SA, SB = G::SB, NW = G::NW, ACC = RUNNING ? 1 : 2;      // ACC: accumulators in tensor memory
  constexpr int KIND = TN == 128 ? LS_F32 : F16 ? LS_F16 : LS_BF16;      // of the result
  extern __shared__ unsigned char wg_raw[];
  // (of ready and acc_free the first block's are used)
  __shared__ __align__(8) uint64_t full[SA], a_empty[SA], c_empty[SA], ready[SB], b_empty[SB], acc_full[ACC], acc_free[ACC];
  __shared__ uint32_t tmem_slot;
  __shared__ int failed_s;
  volatile int* failed = &failed_s;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const uint32_t raw = smem_u32(wg_raw), ring = (raw + 1023u) & ~1023u;

  if (tid == 0) {
    for (int s = 0; s < SA; ++s) { mbar_init(&full[s], 33); mbar_init(&a_empty[s], 1); mbar_init(&c_empty[s], NW); }
    for (int s = 0; s < SB; ++s) { mbar_init(&ready[s], 2 * NW); mbar_init(&b_empty[s], 1); }
    for (int b = 0; b < ACC; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_free[b], 2 * 8); }
    failed_s = 0;
    fence_mbar_init();
  }
  if (warp == 3) tmem_alloc2(&tmem_slot, 2 * TN);          // two accumulators, or one and the running sums
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync();
  tc_fence_after_sync();
  const uint32_t tmem = tmem_slot;
  griddep_chain();

  // A unit is a tile, or a part of the tokens of one of the tiles behind the last full round of the clusters.
  const int rest = A.tiles_n * A.tiles_k - A.whole, units = A.whole + rest * A.splits, clusters = gridDim.x >> 1, mine = blockIdx.x >> 1;
  auto tile_of = [&](int unit) { return unit < A.whole ? unit : A.whole + (unit - A.whole) % rest; };
  auto part_of = [&](int unit) { return unit < A.whole ? 0 : (unit - A.whole) / rest; };
  auto steps_of = [&](int unit, int64_t& from) {
    from = part_of(unit) * A.per_split;
    return (uint32_t)(unit < A.whole ? A.steps : max((int64_t)0, min(A.per_split, A.steps - from)));
  };
  bool ok = true;

  if (warp == 0) {
    WgRing<SA> a;
    uint32_t g = 0;
    for (int unit = mine; unit < units && ok; unit += clusters) {
      int tn, tk; wg_tile(A, tile_of(unit), tn, tk);
      const int n0 = tn * WG_TILE_N + (int)rank * 128, k0 = tk * TN + (int)rank * G::H;
      int64_t from; const uint32_t n = steps_of(unit, from);
      int m0 = (int)(from / A.terms) * G::TOKENS, term = (int)(from % A.terms);
      for (uint32_t it = 0; it < n; ++it, ++g, a.next()) {
        ok = wg_wait(&c_empty[a.at], a.parity ^ 1, failed) && wg_wait(&a_empty[a.at], a.parity ^ 1, failed);
        if (!ok) break;
        if (g < (uint32_t)A.copies && elect_one()) {
          const uint32_t at = ring + a.at * G::A_BYTES;
          mbar_expect_tx(&full[a.at], 2 * G::BOX + G::C_BYTES);
          tma_load_3d(ring + G::C + a.at * G::C_BYTES, &map_codes, k0, m0, 0, &full[a.at]);
          tma_load_3d(at, &map_dy, n0, m0, term, &full[a.at]);
          tma_load_3d(at + G::BOX, &map_dy, n0 + 64, m0, term, &full[a.at]);
        }
        __syncwarp();
        if (++term == A.terms) { term = 0; m0 += G::TOKENS; }
      }
    }
    // the tensor core's arrivals from the other block come in before this one ends, and so do copies after a wait that ran out
    for (uint32_t j = g > SA ? g - SA : 0; j < g && ok; ++j) ok = wg_wait(&a_empty[j % SA], (j / SA) & 1, failed);
    for (uint32_t j = g > SB ? g - SB : 0; j < g && ok; ++j) ok = wg_wait(&b_empty[j % SB], (j / SB) & 1, failed);
    if (!ok)
      for (uint32_t j = g > SA ? g - SA : 0; j < g; ++j) mbar_wait_bounded(&full[j % SA], (j / SA) & 1, 1u << 16);
  } else if (warp == 1) {
    if (rank == 0) {
      // fp32 accumulator, both operands with their columns contiguous (bits 15, 16), 256 rows
      const uint32_t idesc = (umma_idesc(F16 ? 0 : 1, TN) & 0x00ffffffu) | (16u << 24) | (1u << 15) | (1u << 16);
      const uint64_t da0 = umma_desc_mn128(ring, G::BOX), db0 = umma_desc_mn128(ring + G::B, G::BOX);
      WgRing<SA> a;
      WgRing<SB> b;
      WgRing<ACC> acc;
      for (int unit = mine; unit < units && ok; unit += clusters) {
        int64_t from; const uint32_t n = steps_of(unit, from);
        uint32_t in_group = 0;
        for (uint32_t it = 0; it < n; ++it, a.next(), b.next()) {
          ok = (in_group != 0 || wg_wait(&acc_free[acc.at], acc.parity ^ 1, failed)) && wg_wait(&ready[b.at], b.parity, failed);      // numbers and dy's boxes of both blocks
          if (!ok) break;
          tc_fence_after_sync();
          const bool last = in_group + 1 == (uint32_t)A.group || it + 1 == n;
          if (elect_one()) {
            const uint64_t da = da0 + (uint64_t)(a.at * (G::A_BYTES >> 4)), db = db0 + (uint64_t)(b.at * (G::B_BYTES >> 4));
#pragma unroll
            for (int ks = 0; ks < G::TOKENS / 16; ++ks)      // 16 tokens: two groups of 8
              umma2_f16(tmem + acc.at * TN, da + (uint64_t)(ks * 2048 >> 4), db + (uint64_t)(ks * 2048 >> 4), idesc, in_group != 0 || ks != 0);
            umma2_commit(&b_empty[b.at]);
            umma2_commit(&a_empty[a.at]);
            if (last) umma2_commit(&acc_full[acc.at]);
          }
          __syncwarp();
          if (last) { in_group = 0; acc.next(); } else ++in_group;
        }
      }
    }
  } else if (warp == 2) {
    WgRing<SA> a;
    for (int unit = mine; unit < units && ok; unit += clusters) {
      int tn, tk; wg_tile(A, tile_of(unit), tn, tk);
      const int word = (tk * TN + (int)rank * G::H) >> 7;
      int64_t from; const uint32_t n = steps_of(unit, from);
      int m0 = (int)(from / A.terms) * G::TOKENS, term = (int)(from % A.terms);
      for (uint32_t it = 0; it < n; ++it, a.next()) {
        ok = wg_wait(&c_empty[a.at], a.parity ^ 1, failed);
        if (!ok) break;
        unsigned char* to = wg_raw + (ring - raw) + G::E + a.at * G::E_BYTES;
#pragma unroll
        for (int h = 0; h < G::TOKENS / 32; ++h) {
          const int64_t m = (int64_t)m0 + lane + 32 * h;
          const bool in = m < A.tokens && word < A.exp_words;
          cp_async4(to + 4 * (lane + 32 * h), A.exps + (in ? (m * A.exp_words + word) * 4 : 0), in ? 4 : 0);
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&full[a.at])) : "memory");
        if (++term == A.terms) { term = 0; m0 += G::TOKENS; }
      }
    }
    cp_async_wait<0>();
  } else if (warp >= 4 && warp < 4 + 2 * NW) {
    constexpr int Q = G::H / 8, T = 32 * NW, PER = G::TOKENS * Q / T;      // vectors of 8 columns per token; threads of a group; vectors of a thread
    const int w = (tid - 128) % T, group = (warp - 4) / NW;
    const int q = w % Q, m_first = w / Q;                       // this thread: columns 8 q .. of tokens m_first + i T / Q
    const uint32_t pick = 0x4040u + 0x0101u * (uint32_t)((q >> 2) + (TN == 128 ? 2 * (int)rank : 0));      // the block's byte of a token's word
    // (T / Q is a multiple of 8: the swizzle of a thread's vectors is the same for all its tokens)
    const uint32_t from_c = ring + G::C + m_first * G::H + q * 8, from_e = ring + G::E + m_first * 4;
    const uint32_t to_b = ring + G::B + (q >> 3) * G::BOX + m_first * 128 + (((q & 7) ^ (m_first & 7)) << 4);
    WgRing<SA> a;
    WgRing<SB> b;
    a.at = b.at = group;                                        // this group's steps: every second one through all units
    uint32_t skip = group;
    for (int unit = mine; unit < units && ok; unit += clusters) {
      int64_t from; const uint32_t n = steps_of(unit, from);
      uint32_t it = skip;
      for (; it < n; it += 2, a.next(2), b.next(2)) {
        ok = wg_wait(&full[a.at], a.parity, failed);                // dy's boxes too: the arrival below stands for them as well
        if (!ok) break;
        uint2 code[PER];
        uint32_t e[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          code[i] = lds64(from_c + a.at * G::C_BYTES + i * (T / Q) * G::H);
          e[i] = lds32(from_e + a.at * G::E_BYTES + i * (T / Q) * 4);
        }
        uint4 r[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) r[i] = wg_numbers<F16>(code[i], __byte_perm(e[i], 0u, pick));
        __syncwarp();
        if (lane == 0) mbar_arrive(&c_empty[a.at]);
        ok = wg_wait(&b_empty[b.at], b.parity ^ 1, failed);
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < PER; ++i)
          asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to_b + b.at * G::B_BYTES + i * (T / Q) * 128), "r"(r[i].x), "r"(r[i].y), "r"(r[i].z), "r"(r[i].w) : "memory");
        fence_async_smem();
        __syncwarp();
        if (lane == 0) arrive_first(&ready[b.at]);
      }
      skip = it - n;
    }
  } else if (warp >= 4 + 2 * NW) {
    constexpr int W = TN / 2;                              // columns of a warp
    const int quarter = warp & 3, half = (warp - 4 - 2 * NW) >> 2; // tensor-memory lanes 32 * quarter .., columns W * half ..
    WgRing<ACC> acc;
    for (int unit = mine; unit < units; unit += clusters) {
      int tn, tk; wg_tile(A, tile_of(unit), tn, tk);
      int64_t from; const uint32_t n = steps_of(unit, from);
      const int64_t row = (int64_t)tn * WG_TILE_N + rank * 128 + quarter * 32 + lane;
      const int col = tk * TN + half * W;
      // 16 sums of a row: to the split's place, or rounded and stored
      auto put = [&](int c, const float (&v)[16]) {
        if (unit >= A.whole && A.splits > 1) {
          float4* p = reinterpret_cast<float4*>(A.partial + ((int64_t)(unit - A.whole) * WG_TILE_N + rank * 128 + quarter * 32 + lane) * TN + c - tk * TN);
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        } else if (row < A.N) {
#pragma unroll
          for (int i = 0; i < 2; ++i) wg_store<KIND>(A, row, c + 8 * i, v + 8 * i);
        }
      };
      const uint32_t lanes = tmem + half * W + ((uint32_t)(quarter * 32) << 16);
      if (TN == 128) {
        const uint32_t groups = (n + A.group - 1) / A.group;
        float sum[W / 16][16];
#pragma unroll
        for (int p = 0; p < W / 16; ++p)
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[p][i] = 0.f;
        for (uint32_t k = 0; k < groups && ok; ++k, acc.next()) {
          ok = wg_wait(&acc_full[acc.at], acc.parity, failed);
          if (!ok) break;
          tc_fence_after_sync();
#pragma unroll
          for (int p = 0; p < W / 16; ++p) {
            uint32_t r[16];
            tmem_ld16(lanes + acc.at * TN + 16 * p, r);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[p][i] += __uint_as_float(r[i]);
          }
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) arrive_first(&acc_free[acc.at]);
        }
#pragma unroll
        for (int p = 0; p < W / 16; ++p) {
          if (!ok) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[p][i] = __int_as_float(0x7fffffff);
          }
          put(col + 16 * p, sum[p]);
        }
      } else if (RUNNING) {
        // (the tensor core waits until a group's sums are added: at 8192 x 2048 x 4608 1.3 % of the time with 64 steps a group, 3 % with 32, 6 % with 16)
        const uint32_t groups = (n + A.group - 1) / A.group, sums = lanes + TN;      // these warps' alone
        for (uint32_t k = 0; k < groups && ok; ++k, acc.next()) {
          ok = wg_wait(&acc_full[acc.at], acc.parity, failed);
          if (!ok) break;
          tc_fence_after_sync();
#pragma unroll
          for (int p = 0; p < W / 16; ++p) {
            uint32_t r[16], s[16];
            float v[16];
            tmem_ld16(lanes + 16 * p, r);
            if (k != 0) tmem_ld16(sums + 16 * p, s);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = k != 0 ? __uint_as_float(s[i]) + __uint_as_float(r[i]) : __uint_as_float(r[i]);
            tmem_st16(sums + 16 * p, v);
          }
          tmem_wait_st();
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) arrive_first(&acc_free[acc.at]);
        }
#pragma unroll
        for (int p = 0; p < W / 16; ++p) {
          uint32_t r[16];
          tmem_ld16(sums + 16 * p, r);
          tmem_wait_ld();
          float v[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = ok ? __uint_as_float(r[i]) : __int_as_float(0x7fffffff);
          put(col + 16 * p, v);
        }
      } else {
        ok = ok && wg_wait(&acc_full[acc.at], acc.parity, failed);
        tc_fence_after_sync();
#pragma unroll
        for (int p = 0; p < W / 16; ++p) {
          uint32_t r[16];
          tmem_ld16(lanes + acc.at * TN + 16 * p, r);
          tmem_wait_ld();
          if (p == W / 16 - 1) {                           // all read: the tensor core may have the place back
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0 && ok) arrive_first(&acc_free[acc.at]);
          }
          float v[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = ok ? __uint_as_float(r[i]) : __int_as_float(0x7fffffff);
          put(col + 16 * p, v);
        }
        acc.next();
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync();                                          // no block ends while the other may still read from it or arrive at its barriers
  if (warp == 3) tmem_dealloc2(tmem, 2 * TN);
}

// The tiles whose tokens were split: 8 entries a thread, the parts in order.
template <int TN>
__global__ void __launch_bounds__(256) wgrad_sum_kernel(const WgradArgs A) {
  griddep_chain();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  constexpr int per = TN / 8;
  const int rest = A.tiles_n * A.tiles_k - A.whole, t = (int)(i / (WG_TILE_N * per)), in = (int)(i - (int64_t)t * WG_TILE_N * per), r = in / per, c = (in - r * per) * 8;
  if (t >= rest) return;
  int tn, tk; wg_tile(A, A.whole + t, tn, tk);
  const int64_t n = (int64_t)tn * WG_TILE_N + r;
  const int k = tk * TN + c;
  if (n >= A.N || k >= A.K) return;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < A.splits; ++s) {
    const float4* p = reinterpret_cast<const float4*>(A.partial + (((int64_t)s * rest + t) * WG_TILE_N + r) * TN + c);
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
