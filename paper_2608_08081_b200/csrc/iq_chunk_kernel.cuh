// Attention of any number of new tokens over the packed cache: tiles of 256 (token, query head) pairs of a KV head, shared by a pair of CTAs, one
// pass over the blocks that they see.
//
// A step of NB cached rows: S[pair][row] = Q K^T, Q the rotated queries as two binary16 terms, K the levels of the codes;
// t = S scale_K + log2(scale_V) - reference_pair in units of log2; p = 2^t; O[pair][coordinate] += p V, V the levels; l_pair += p / scale_V. The
// output is R^T O / l.
// A row's V scale is part of its exponent, so p is the row's weight in the OUTPUT, and the reference follows the largest of those: p
// goes to the tensor cores as two binary16 terms (22 bits, or 2^-25 of the reference), also where a row with most of the weight has next to no
// value. One term would add as much error as the binary16 output's own rounding (outputs 2.6e-4 - 2.8e-4 off in norm instead of 2.07e-4, which the rounding alone
// makes), and a token's precision would hang on whether enough others come with it to take this kernel; it took 5.0 ms for 6.0 with 4096 tokens behind 28 000 rows, 159
// us for 179 with 1000 behind 6000, half of the difference instructions, half products. The queries have two terms as well, as their
// error would grow with the scores: 2^-22 of an element, or 2^-25 where one power of two scales the CTA's 128 pairs to a largest element of 2^8 to 2^9.
// References are raised only when a weight passes 2^15: then sums and O are scaled, which waits for the values of the step before (a raised
// reference is the step's maximum; with it 5 log2 units lower, raises took 6 % of the time).
//
// Segments. The tensor core cuts its running sum towards zero with each product of 16 rows (measured: 1e-7 of the final sum, all in one direction), and
// weights below 2^-25 of the reference are left out of O though not of l: both would grow with the rows, to 8e-4 and up to 2^-8 of an output behind 128 K of them.
// So a piece is worked in segments of at most 8192 rows with references and sums of their own, joined in fp32 through each thread's own
// places of the workspace: some 5e-5 and at most 2^-12, however many rows there are.
//
// Work split. The two CTAs of a pair have 128 rows of Q, S and O each in their tensor memory, and half of the levels of a step each in shared memory: one
// product of both (cta_group::2, M = 256) reads the operand once from either, and each block is dequantised once for 256 pairs. Warps of a
// CTA: eight softmax, 16 rows each; four that make K levels, four V levels; one that issues the products of the pair; three that bring the next
// tile's queries. Softmax warps meet nobody in the loop over the steps. Items (sequence, KV head, tile) are laid end to end and cut into
// equal ranges, one per pair of CTAs; tiles that two or more pairs share are merged by a second launch.
//
// What bounds it. 4096 tokens behind 28 000 rows, 64/8 heads, 3 bits: 6.0 ms = 0.67 PFLOP/s of the 4 d a (pair, row) needs; the two terms of Q and of the
// weights make it 8 d, 1.35 PFLOP/s on the tensor pipe. A step of 128 rows takes the pipe 2048 cycles and a softmax warp some 3000, one instruction after the
// other (with one term to a weight 2600 - 2700: barrier 210, scores 250, exponents 850, exponentials and sums 1150, weights handed over 110, loop 150). Two buffers of
// scores and the trip from weights to the scores that take their place (2100 cycles with one term) keep the steps from overlapping further. The schedulers issue
// in 0.52 of the cycles, the special-function pipe is busy 0.31, shift/logic 0.35, the tensor pipe 0.60 (1000 tokens behind 6000 rows, 180 us, of
// which the beginning and end of a piece take 6 us each).
// Built and slower, with one term to a weight: one CTA to a tile (issue 0.55 of the cycles, half of it for levels: 5.9 ms for 5.1); four softmax warps to 32 rows, a quarter of the
// columns each, which meet once a step (3200 cycles a step); a fourth to three quarters of the exponentials as polynomials of degree 4 on the
// multiply-add pipe (215 us: 221, 228, 239); the next step's scores asked for before the weights are handed over (175 us: 185); the look at
// the references behind the exponentials, which then run beside the exponents (no gain). Code that is
// not at hand costs as much as any pipe: with a piece's rotations in long unrolled code and K and V levels in code of their own, 10 % of the
// instruction fetches missed (now 3.6 %) and 64 tokens behind 1000 rows took 29.9 us instead of 26.7.
#pragma once
#include <type_traits>

#include "iq_chunk_common.cuh"
#include "iq_format.cuh"
#include "iq_tile_mma.cuh"

namespace iq {

constexpr float CHUNK_LIMIT = 15.f;                   // log2 of the largest p ...
constexpr float CHUNK_START = 0.f;                    // ... and of the step's largest behind a raise
// Blocks of a segment (a power of two). 16, 32 and 64 blocks and no segments, with one term to a weight: 5.19, 5.18, 5.07 and 5.05 ms for 4096 tokens behind 28 000
// rows; 175, 166, 159 and 161 us for 1000 behind 6000.
constexpr int CHUNK_SEGMENT = 64;
constexpr float CHUNK_LEAST_SCALE = 8.67361738e-19f;  // 2^-60: V scales below it count as this

// (Off by 2^-22 of the logarithm, and by one unit in the last place. log2f and a division: 1 % more time.)
__device__ __forceinline__ float chunk_log2(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float chunk_inverse(float x) {
  float y;
  asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Layouts of the loads: 16x256b leaves rows lane / 4 and lane / 4 + 8 of 16 and columns 2 (lane % 4), + 1 of every 8 with a thread (so that it needs the
// factors of 16 columns, not of all), 16x128b takes back the same as pairs of binary16 values, one to a column.
__device__ __forceinline__ void chunk_ld_rows(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ void chunk_ld_rows(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ void chunk_st_rows(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void chunk_st_rows(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
               "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
__device__ __forceinline__ void chunk_st_pairs(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void chunk_st_pairs(uint32_t taddr, const uint32_t (&r)[4]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x2.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3])
               : "memory");
}
__device__ __forceinline__ void chunk_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr) : "memory");
}
// What two binary16 values have left of x and y, as two binary16 values. (A multiply-add that takes binary16 factors as they are: with conversions
// before it, 1 % more time.)
__device__ __forceinline__ uint32_t chunk_rest(uint32_t first, float x, float y) {
  float a, b;
  asm("{\n\t.reg .f16 u, v, m;\n\tmov.b16 m, 0xBC00;\n\tmov.b32 {u, v}, %2;\n\tfma.rn.f32.f16 %0, u, m, %3;\n\tfma.rn.f32.f16 %1, v, m, %4;\n\t}"
      : "=f"(a), "=f"(b)
      : "r"(first), "f"(x), "f"(y));
  return pack_half2(a, b);
}
// Values that a tcgen05.ld has left in registers are not used before the wait for it.
template <int C>
__device__ __forceinline__ void chunk_landed(uint32_t (&r)[C]) {
#pragma unroll
  for (int i = 0; i < C; i++) asm volatile("" : "+r"(r[i]));
}
// Unnormalised Walsh-Hadamard transform of 32 values of a thread.
__device__ __forceinline__ void chunk_wht32(float (&v)[32]) {
#pragma unroll
  for (int s = 1; s < 32; s <<= 1)
#pragma unroll
    for (int i = 0; i < 32; i++)
      if ((i & s) == 0) {
        const float x = v[i], y = v[i + s];
        v[i] = x + y;
        v[i + s] = x - y;
      }
}
// The 8 SO(4) blocks (or their transposes) of 32 consecutive coordinates; m: their matrices, in shared memory.
template <bool TRANSPOSE>
__device__ __forceinline__ void chunk_so4(const float4* m, float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const float4 a = m[4 * j], b = m[4 * j + 1], c = m[4 * j + 2], d = m[4 * j + 3];
    const float x0 = v[4 * j], x1 = v[4 * j + 1], x2 = v[4 * j + 2], x3 = v[4 * j + 3];
    if (TRANSPOSE) {
      v[4 * j] = a.x * x0 + b.x * x1 + c.x * x2 + d.x * x3;
      v[4 * j + 1] = a.y * x0 + b.y * x1 + c.y * x2 + d.y * x3;
      v[4 * j + 2] = a.z * x0 + b.z * x1 + c.z * x2 + d.z * x3;
      v[4 * j + 3] = a.w * x0 + b.w * x1 + c.w * x2 + d.w * x3;
    } else {
      v[4 * j] = a.x * x0 + a.y * x1 + a.z * x2 + a.w * x3;
      v[4 * j + 1] = b.x * x0 + b.y * x1 + b.z * x2 + b.w * x3;
      v[4 * j + 2] = c.x * x0 + c.y * x1 + c.z * x2 + c.w * x3;
      v[4 * j + 3] = d.x * x0 + d.y * x1 + d.z * x2 + d.w * x3;
    }
  }
}
__device__ __forceinline__ float chunk_sign(int a, int b) { return __popc(a & b) & 1 ? -1.f : 1.f; }

template <int D>
struct ChunkLayout {
  static constexpr int NB = D == 128 ? 128 : 64;   // cached rows of a step
  static constexpr int SUB = 128 / NB;             // steps of a block
  static constexpr int NC = 32, NI = NC / 8;       // columns of S that a softmax warp takes at a time (of its 16 rows); groups of 8
  static constexpr int PARTS = NB / NC;
  static constexpr int SETS = D / 32;              // runs of 32 coordinates
  static constexpr int SEGMENT = CHUNK_SEGMENT * SUB;  // steps of a segment (a power of two)
  static constexpr size_t KEPT = chunk_kept(D);
  // Warps: softmax, K levels, V levels, products (one, in the first CTA of a pair), queries on their way. Registers of a thread: 96 at
  // launch, 480 over the five groups of warps (two of them softmax, two levels): as many as none of them spills with (152, 64 and 48: 2 - 8 % slower).
  static constexpr int SOFTMAX_WARPS = 8, K_WARP = 8, V_WARP = 12, MMA_WARP = 16, QUERY_WARP = 17, THREADS = 640;
  static constexpr int SOFTMAX_REGS = 128, LEVEL_REGS = 72, MMA_REGS = 80;
  // tensor memory: Q (D = 128: both terms; 256: the first), two buffers of scores, O. The weights of NC columns go over their
  // scores: the first terms in the first half of the columns, two to a column, the second terms in the second.
  static constexpr int Q_COL = 0, S_COL = 128, O_COL = 512 - D;
  // shared memory: K and V levels of some steps (this CTA's half of them: rows of K, coordinates of V), the tile's queries as they came, the
  // second term of Q (D = 256), the rest
  static constexpr int STAGES = D == 128 ? 4 : 2, OPERAND = 16384;
  static constexpr int OFF_K = 0, OFF_V = STAGES * OPERAND, OFF_RAW = 2 * STAGES * OPERAND, OFF_Q = OFF_RAW + 128 * D * 2;
  static constexpr int OFF_S = OFF_Q + (D == 256 ? 128 * D * 2 : 0);
  static constexpr int COLUMNS = 2 * STAGES;       // steps whose columns' factors are kept: at least STAGES + 2
  // M = 256: 128 rows of each CTA of the pair
  static constexpr uint32_t IDESC_QK = (1u << 4) | (((uint32_t)NB >> 3) << 17) | ((256u >> 4) << 24);
  static constexpr uint32_t IDESC_PV = (1u << 4) | (((uint32_t)D >> 3) << 17) | ((256u >> 4) << 24);
};
template <int D>
struct ChunkShared {
  using L = ChunkLayout<D>;
  // In the first CTA, arrived at by both: k_full, v_full, p_full, q_ready. In the second: column_full. In each: the others.
  uint64_t column_full[L::COLUMNS];          // the factors of a step's columns
  uint64_t k_full[L::STAGES], k_empty[L::STAGES], v_full[L::STAGES], v_empty[L::STAGES];
  uint64_t s_full[2], p_full[2], o_done[2];  // of even and odd steps
  uint64_t q_ready, raw_full, raw_empty, drain;
  uint32_t tmem, failed;
  ChunkRange range;
  ChunkPiece piece[4];                    // pieces 0, 4, ..., 1, 5, ...: with their queries (no blocks: there are no more)
  uint32_t go[4];                         // whether there is such a piece: one thread's finding, so that all find the same
  alignas(16) float4 m[3][D];             // SO(4) matrices of the KV head of pieces 0, 3, ...
  // Factors of a step's rows: of two at a time the scales of S, then the log2 of the V scales; of each 1 / V scale.
  alignas(16) float4 column[L::COLUMNS][L::NB / 2];
  float weight[L::COLUMNS][L::NB];
  float row_sum[128], row_ref[128];       // at the end of a piece
  float warp_q[4][3];                     // the largest elements of a piece's queries
  const __half* query[128];               // where the queries of the tile's rows lie (nullptr: a row without a token)
};
template <int D>
constexpr int CHUNK_SMEM = ChunkLayout<D>::OFF_S + (int)sizeof(ChunkShared<D>) + 1024;
static_assert(CHUNK_SMEM<128> <= 232448 && CHUNK_SMEM<256> <= 232448, "shared memory");

// ---- the pair of CTAs
__device__ __forceinline__ uint32_t chunk_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// The address, among the pair's, of something at the same place in the shared memory of CTA `rank`.
__device__ __forceinline__ uint32_t chunk_at(const void* p, uint32_t rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
// (No generic write of one CTA is read by the other: levels and second terms are read by products, behind a proxy fence, the rest lies in tensor
// memory. The factors of a step's columns are passed on within each CTA: arrivals and waits at the pair's scope took 15 % more time, as a release
// there waits for every load and store of the thread.)
__device__ __forceinline__ void chunk_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void chunk_pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Completion of the products so far, at the barrier in the same place of both CTAs.
__device__ __forceinline__ void chunk_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
// D[256 rows: both CTAs' tensor memory] (+)= A B, B's rows half in either CTA's shared memory; A in tensor memory, or in shared memory.
__device__ __forceinline__ void chunk_mma(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem), "r"(a_tmem),
               "l"(bdesc), "r"(idesc), "r"(accumulate)
               : "memory");
}
__device__ __forceinline__ void chunk_mma_ss(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(adesc), "l"(bdesc),
               "r"(idesc), "r"(accumulate)
               : "memory");
}
// Bounded wait of a converged warp. A wait that gives up is noted in `failed` of both CTAs, and from then on no wait of theirs lasts: every
// thread goes on through the same loops and barriers over whatever is there, so that the pair ends together. Other warps may note it at any
// moment, so warps that share a barrier never go by their own reading of it: the query warps by the OR of all of theirs, the softmax warps by
// one thread's (`go`).
__device__ __forceinline__ void chunk_wait(uint64_t* bar, uint32_t parity, uint32_t limit, uint32_t* failed) {
  for (uint32_t i = 0; !mbar_try_wait(bar, parity); i++)
    if (i >= limit || *(volatile uint32_t*)failed) {
      *(volatile uint32_t*)failed = 1;
      asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(chunk_at(failed, chunk_rank() ^ 1)), "r"(1) : "memory");
      break;
    }
  __syncwarp();
}

// Address of the 16-byte chunk c of row r in an operand of rows of 128 bytes, 128-byte swizzle.
__device__ __forceinline__ uint8_t* chunk_swizzled(uint8_t* slab, int r, int c) { return slab + r * 128 + ((c ^ (r & 7)) << 4); }

// The steps of a CTA one after the other, for the warps that make its levels: where the step's block starts in the cache. A lane looks up the
// place of one step, 32 steps of a piece at a time.
struct ChunkSteps {
  ChunkWalk walk;
  ChunkPiece c;
  int j, steps;        // of the piece
  size_t place;        // of the lane's step, in the cache's rows
  size_t row0;         // of this step's block
  __device__ __forceinline__ void start(const ChunkParams& p, const ChunkRange& r) {
    walk.start(p, r);
    j = -1;
    steps = 0;
  }
  template <int SUB>
  __device__ __forceinline__ bool next(const ChunkParams& p, int lane, uint32_t* status) {
    if (++j >= steps) {
      do
        if (!walk.next(p, c)) { j = steps = 0; return false; }
      while (c.hi == c.lo);
      j = 0;
      steps = (c.hi - c.lo) * SUB;
    }
    if ((j & 31) == 0) {
      place = 0;
      if (j + lane < steps) place = cache_row(p.pm, c.b, c.g, c.x.block(c.lo + (j + lane) / SUB) * 128, status);
    }
    row0 = __shfl_sync(FULL, (unsigned long long)place, j & 31);
    return true;
  }
};
// 64 entries of packed levels as binary16 values, to row r of a slab of rows of 128 bytes.
template <int BITS>
__device__ __forceinline__ void chunk_levels(const uint32_t (&raw)[2 * BITS], const uint32_t (&lo)[4], const uint32_t (&hi)[4], LookupConst c, uint8_t* slab, int r) {
#pragma unroll
  for (int u = 0; u < 2; u++) {
    uint32_t x[16];
    dequant32_f16<BITS>(raw + u * BITS, lo, hi, c, x);
#pragma unroll
    for (int k = 0; k < 4; k++) *reinterpret_cast<uint4*>(chunk_swizzled(slab, r, 4 * u + k)) = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
  }
}
template <int BITS>
__device__ __forceinline__ void chunk_load(const uint8_t* src, uint32_t (&raw)[2 * BITS]) {
#pragma unroll
  for (int i = 0; i < BITS; i++) {
    const uint2 x = __ldg(reinterpret_cast<const uint2*>(src) + i);
    raw[2 * i] = x.x;
    raw[2 * i + 1] = x.y;
  }
}

template <int D, int BITS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(ChunkLayout<D>::THREADS, 1) chunk_kernel(const __grid_constant__ ChunkParams p) {
  using L = ChunkLayout<D>;
  constexpr int NB = L::NB, NC = L::NC, NI = L::NI, PARTS = L::PARTS, SUB = L::SUB, SETS = L::SETS, ST = L::STAGES;
  constexpr int P = PackedFormat<BITS>::row_bytes(D), R = PackedFormat<BITS>::V_RECORD_BYTES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);  // (the swizzle goes by the address)
  ChunkShared<D>& s = *reinterpret_cast<ChunkShared<D>*>(smem + L::OFF_S);
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);
  const int rank = (int)chunk_rank(), pair = blockIdx.x >> 1;

  if (tid == 0) {
    for (int i = 0; i < ST; i++) {
      mbar_init(&s.k_full[i], 8);
      mbar_init(&s.v_full[i], 8);
      mbar_init(&s.k_empty[i], 1);
      mbar_init(&s.v_empty[i], 1);
    }
    for (int i = 0; i < L::COLUMNS; i++) mbar_init(&s.column_full[i], NB / 32);
    for (int i = 0; i < 2; i++) {
      mbar_init(&s.s_full[i], 2);
      mbar_init(&s.o_done[i], 1);
      mbar_init(&s.p_full[i], 2 * L::SOFTMAX_WARPS);
    }
    mbar_init(&s.q_ready, 2 * L::SOFTMAX_WARPS);
    mbar_init(&s.raw_full, 3);
    mbar_init(&s.raw_empty, L::SOFTMAX_WARPS);
    mbar_init(&s.drain, 1);
    s.failed = 0;
    fence_mbar_init();
    fence_proxy_async();
  }
  if (warp == L::MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem)), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::);
  }
  grid_dependency_wait();
  if (warp == 0) {
    const ChunkRange r = chunk_range(p, pair, lane);
    if (lane == 0) s.range = r;
  }
  tc_fence_before();
  __syncthreads();
  chunk_pair_sync();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(FULL, s.tmem, 0);
  if (s.range.total == 0) {  // (a step whose sequences are all the other kernel's: nothing but the note for the merge)
    allow_dependent_launch();
    if (tid == 0 && rank == 0) p.cuts[pair].last = -1;
    if (warp == L::MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
    return;
  }
  uint32_t n = 0;  // steps so far

  if (warp >= L::MMA_WARP) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::MMA_REGS));
    ChunkWalk walk;
    ChunkPiece c;
    walk.start(p, s.range);
    uint32_t pieces = 0;
    if (warp >= L::QUERY_WARP) {
      // ================================================================ the queries of the next piece, as they are
      const int t = tid - 32 * L::QUERY_WARP, query_bar = 6;
      constexpr int CHUNKS = D / 8;  // of 16 bytes, of a row
      for (bool more = true; more;) {
        more = walk.next(p, c);
        if (more && c.hi == c.lo) {  // no token of the item sees a row
          for (int r = t; r < 128; r += 96) {
            const int at = c.t * CHUNK_ROWS + rank * 128 + r, tok = at / p.group;
            if (tok >= c.sq.n) break;
            const size_t out_row = ((size_t)c.sq.tok0 + tok) * p.n_q_heads + c.g * p.group + at - tok * p.group;
            for (int k = 0; k < CHUNKS; k++) reinterpret_cast<uint4*>(p.out + out_row * D)[k] = make_uint4(0u, 0u, 0u, 0u);
            if (p.lse) p.lse[out_row] = -INFINITY;
          }
          continue;
        }
        if (pieces > 0) chunk_wait(&s.raw_empty, (pieces - 1) & 1, p.wait_polls, &s.failed);
        // One finding for the three warps, which meet at barriers below (where a wait has given up, what is there may still be read).
        if (cta_bar_or_n(query_bar, 96, *(volatile uint32_t*)&s.failed != 0)) break;
        if (!more) c.hi = c.lo = 0;
        if (t == 0) s.piece[pieces & 3] = c;
        if (more) {
          const __half* const q = p.q + (p.token_start ? c.sq.tok0 * p.qs_t : c.b * p.qs_b);
          for (int r = t; r < 128; r += 96) {
            const int at = c.t * CHUNK_ROWS + rank * 128 + r, tok = at / p.group, head = c.g * p.group + at - tok * p.group;
            s.query[r] = tok < c.sq.n ? q + tok * p.qs_t + head * p.qs_h : nullptr;
          }
          cta_bar_sync_n(query_bar, 96);
#pragma unroll 4
          for (int i = t; i < 128 * CHUNKS; i += 96) {
            const int r = i / CHUNKS, k = i % CHUNKS;
            const __half* const row = s.query[r];
            const uint32_t dst = smem_u32(smem + L::OFF_RAW + r * (2 * D) + ((k ^ (r & 7)) << 4));
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(row ? row + 8 * k : p.q), "r"(row ? 16 : 0) : "memory");
          }
          if (t < D / 4) {
            float M[4][4];
            so4_matrix<float>(p.rot + ((size_t)c.g * (D / 4) + t) * 8, M);
            float4* const m = s.m[pieces % 3] + 4 * t;
#pragma unroll
            for (int i = 0; i < 4; i++) m[i] = make_float4(M[i][0], M[i][1], M[i][2], M[i][3]);
          }
          asm volatile("cp.async.wait_all;" ::: "memory");
          __half2 top = __float2half2_rn(0.f);  // of the elements that this thread brought
#pragma unroll 4
          for (int i = t; i < 128 * CHUNKS; i += 96) {
            const int r = i / CHUNKS, k = i % CHUNKS;
            const uint4 x = *reinterpret_cast<const uint4*>(smem + L::OFF_RAW + r * (2 * D) + ((k ^ (r & 7)) << 4));
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int k2 = 0; k2 < 4; k2++) {
              const uint32_t a = w[k2] & 0x7FFF7FFFu;
              const __half2 h = *reinterpret_cast<const __half2*>(&a);
              const uint32_t kept = a & ~__heq2_mask(h, __half2half2(__ushort_as_half(0x7C00)));  // (an infinite query is its own affair, as NaN)
              top = __hmax2(top, *reinterpret_cast<const __half2*>(&kept));
            }
          }
          const float most = warp_max(fmaxf(__low2float(top), __high2float(top)));
          if (lane == 0) s.warp_q[pieces & 3][warp - L::QUERY_WARP] = most;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.raw_full);
        cta_bar_sync_n(query_bar, 96);  // (the rows' places have been read)
        pieces++;
      }
      if (t == 0 && rank == 0) {  // (also where a wait gave up, whose pieces have not all been walked: the outputs are invalid, the places are not)
        if (walk.cut.last == 0) walk.cut.last = (int)min((long long)s.range.pairs - 1, unit_div(walk.cut_end * s.range.pairs - 1, s.range.total));
        p.cuts[pair] = walk.cut;
      }
    } else if (rank == 0) {
      // ================================================================ products, of both CTAs
      // (an operand further on in shared memory: its descriptor plus the distance in units of 16 bytes, which stays within the address's bits)
      const uint64_t k_desc = smem_desc_k128(smem_u32(smem + L::OFF_K)), v_desc = smem_desc_k128(smem_u32(smem + L::OFF_V));
      const uint64_t q_desc = smem_desc_k128(smem_u32(smem + L::OFF_Q));
      constexpr int ROLL = D == 256 ? 8 : 1;  // (a product of 64 columns takes half as long as the loop around four of them allows for)
      auto scores = [&](uint32_t i) {  // S = Q K^T of step i, whose levels are there; the second terms first
        const uint32_t o = i & 1, st = i % ST;
        const uint64_t b = k_desc + st * (L::OPERAND >> 4);
        const uint32_t d = tmem + L::S_COL + o * NB;
        if (elect_one()) {
#pragma unroll ROLL
          for (int k = 0; k < 2 * (D / 64); k++) {  // 64 coordinates: of the second terms, then of the first
            const int hi = k / (D / 64), slab = k % (D / 64);
            const uint64_t bs = b + slab * (NB / 2 * 128 >> 4);
#pragma unroll
            for (int i = 0; i < 4; i++) {
              if (D == 256 && !hi) chunk_mma_ss(d, q_desc + ((slab * 16384 + i * 32) >> 4), bs + (i * 32 >> 4), L::IDESC_QK, k + i != 0);
              else chunk_mma(d, tmem + L::Q_COL + (hi ? 0 : D / 2) + (4 * slab + i) * 8, bs + (i * 32 >> 4), L::IDESC_QK, k + i != 0);
            }
          }
          chunk_commit(&s.s_full[o]);
          chunk_commit(&s.k_empty[st]);
          mbar_arrive(&s.s_full[o]);  // (passes on the factors of the step's columns, which came with this CTA's levels)
        }
        __syncwarp();
      };
      auto values = [&](uint32_t i, bool first) {  // O += P V of step i, whose weights and levels are there
        const uint32_t o = i & 1, st = i % ST;
        const uint64_t b = v_desc + st * (L::OPERAND >> 4);
        if (elect_one()) {
#pragma unroll 1
          for (int k = 0; k < NB / 64; k++)  // 64 rows: two parts of weights
#pragma unroll
            for (int i = 0; i < 8; i++)  // 16 rows, their weights' second terms and then their first
              chunk_mma(tmem + L::O_COL, tmem + L::S_COL + o * NB + (2 * k + (i >> 2)) * NC + (i & 1 ? 0 : NC / 2) + (i >> 1 & 1) * 8, b + ((k * (D / 2 * 128) + (i >> 1) * 32) >> 4), L::IDESC_PV,
                        !(first && k + i == 0));
          chunk_commit(&s.o_done[o]);
          chunk_commit(&s.v_empty[st]);
        }
        __syncwarp();
      };
      auto wait_k = [&](uint32_t i) { chunk_wait(&s.k_full[i % ST], (i / ST) & 1, p.wait_polls, &s.failed); };
      auto wait_v = [&](uint32_t i) { chunk_wait(&s.v_full[i % ST], (i / ST) & 1, p.wait_polls, &s.failed); };
      while (walk.next(p, c)) {
        const int steps = (c.hi - c.lo) * SUB;
        if (steps == 0) continue;
        wait_k(n);
        if (steps > 1) wait_k(n + 1);
        chunk_wait(&s.q_ready, pieces & 1, p.wait_polls, &s.failed);
        pieces++;
        tc_fence_after();
        scores(n);
        if (steps > 1) scores(n + 1);
        // The scores of step n + 2 take the place of the weights of step n, so their products follow each other; the levels of both have been waited
        // for when the weights come.
        for (int j = 0; j < steps; j++, n++) {
          wait_v(n);
          if (j + 2 < steps) wait_k(n + 2);
          chunk_wait(&s.p_full[n & 1], (n >> 1) & 1, p.wait_polls, &s.failed);
          tc_fence_after();
          values(n, (j & (L::SEGMENT - 1)) == 0);
          if (j + 2 < steps) scores(n + 2);
        }
      }
    } else {
      // ================================================================ in the second CTA: the factors of a step's columns passed on beside its scores
      while (walk.next(p, c))
        for (int j = (c.hi - c.lo) * SUB; j > 0; j--, n++) {
          chunk_wait(&s.column_full[n % L::COLUMNS], (n / L::COLUMNS) & 1, p.wait_polls, &s.failed);
          if (n >= 2) chunk_wait(&s.s_full[n & 1], ((n >> 1) - 1) & 1, p.wait_polls, &s.failed);  // (one arrival to a phase)
          if (lane == 0) mbar_arrive(&s.s_full[n & 1]);
          __syncwarp();
        }
    }
  } else if (warp >= L::K_WARP) {
    // ================================================================ levels: of K, a thread 64 coordinates of a row, and the factors of the
    // rows; of V, 64 rows of a coordinate. One code for both: instructions that are not at hand are what a warp here waits for most.
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::LEVEL_REGS));
    const bool is_v = warp >= L::V_WARP;
    const int t = tid - 32 * (is_v ? L::V_WARP : L::K_WARP);
    constexpr int KR = NB / 2, VR = D / 2;  // rows of the CTA's operand: of K, coordinates of V
    const int r = is_v ? t % VR : t % KR, part = is_v ? t / VR : t / KR;
    const uint8_t* const src = is_v ? p.v_codes + (rank * VR + r) * R + part * (R / 2) : p.k_codes + (rank * KR + r) * P + part * (8 * BITS);
    const int sub_bytes = is_v ? R / 2 : NB * P;  // from a block's first step to its second
    uint8_t* const slab = smem + (is_v ? L::OFF_V + part * (VR * 128) : L::OFF_K + part * (KR * 128));
    uint64_t* const empty = is_v ? s.v_empty : s.k_empty;
    const uint32_t full = chunk_at(is_v ? s.v_full : s.k_full, 0);
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      lo[i] = is_v ? p.lut_v_lo[i] : p.lut_lo[i];
      hi[i] = is_v ? p.lut_v_hi[i] : p.lut_hi[i];
    }
    const bool factors = !is_v && t < NB;
    ChunkSteps steps;
    steps.start(p, s.range);
    uint32_t raw[2 * BITS];
    float ks = 0.f, vs = 0.f;
    auto load = [&]() {
      chunk_load<BITS>(src + steps.row0 * P + (SUB > 1 ? (steps.j & 1) * sub_bytes : 0), raw);
      if (factors) {
        const int first = SUB > 1 ? (steps.j & 1) * NB : 0, row = steps.c.x.block(steps.c.lo + steps.j / SUB) * 128 + first + t;
        ks = vs = 0.f;
        if (row < steps.c.x.end) {  // (rows that no token sees may hold anything)
          ks = load_scale(p.k_scales, steps.row0 + first + t, p.scale_f16);
          vs = load_scale(p.v_scales, steps.row0 + first + t, p.scale_f16);
        }
      }
    };
    uint32_t* const status = warp == L::K_WARP && rank == 0 ? p.status : nullptr;
    bool have = steps.next<SUB>(p, lane, status);
    if (have) load();
    while (have) {
      const uint32_t st = n % ST;
      if (n >= ST) chunk_wait(&empty[st], ((n / ST) - 1) & 1, p.wait_polls, &s.failed);
      if (factors) {
        float* const col = reinterpret_cast<float*>(&s.column[n % L::COLUMNS][t >> 1]) + (t & 1);
        vs = vs < CHUNK_LEAST_SCALE ? CHUNK_LEAST_SCALE : vs;
        col[0] = ks * p.score_unit;
        col[2] = chunk_log2(vs);
        s.weight[n % L::COLUMNS][t] = vs < INFINITY ? chunk_inverse(vs) : 1.f;  // (finite: tokens that do not see the row multiply it by 0)
      }
      chunk_levels<BITS>(raw, lo, hi, p.lookup, slab + st * L::OPERAND, r);
      have = steps.next<SUB>(p, lane, status);
      if (have) load();
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) {
        chunk_arrive(full + 8 * st);
        if (factors && rank == 1) mbar_arrive(&s.column_full[n % L::COLUMNS]);
      }
      n++;
    }
  } else {
    // ================================================================ queries, softmax, outputs
    // A warp has 16 rows and all columns of S: its references and sums are nobody else's, so it meets no other in the loop over the steps.
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::SOFTMAX_REGS));
    const int quad = warp & 3, half = warp >> 2;           // rows 32 quad + 16 half ...; half of the coordinates of rows 32 quad ...
    const uint32_t lanes = (uint32_t)quad << 21;           // the quarter of the tensor-memory lanes
    const uint32_t lanes16 = lanes + ((uint32_t)half << 20);
    const int pair_bar = 1 + quad, all_bar = 5;            // barriers: the two warps of a quarter; all
    const int row = 32 * quad + lane;                      // the thread's row where it has one
    const int row2 = 32 * quad + 16 * half + (lane >> 2);  // its two rows in the loop over the blocks: 8 apart
    const int first_row = rank * 128;                      // of the tile's
    const uint32_t q_ready = chunk_at(&s.q_ready, 0), p_full = chunk_at(s.p_full, 0);  // where the products are issued
    const int set0 = half * (SETS / 2), set1 = set0 + SETS / 2;
    // The rotated queries of piece `count`, q~ = M H q, a thread half of a row's coordinates. False: there is no such piece.
    float q_unit = 0.f;  // what a unit of a score is
    auto queries = [&](uint32_t count) {
      const float4* const m = s.m[count % 3];
      const uint8_t* const raw_row = smem + L::OFF_RAW + row * (2 * D);
      auto q = [&](int k) { return *reinterpret_cast<const uint4*>(raw_row + ((k ^ (row & 7)) << 4)); };  // 16 bytes of the thread's row
      chunk_wait(&s.raw_full, count & 1, p.wait_polls, &s.failed);
      if (tid == 0) s.go[count & 3] = *(volatile uint32_t*)&s.failed ? 0u : s.piece[count & 3].hi > s.piece[count & 3].lo;
      cta_bar_sync_n(all_bar, 32 * L::SOFTMAX_WARPS);
      if (!s.go[count & 3]) return false;
      const float qmax = fmaxf(fmaxf(s.warp_q[count & 3][0], s.warp_q[count & 3][1]), s.warp_q[count & 3][2]);
      const int e2 = qmax > 0.f ? 13 - ((int)(__float_as_uint(qmax) >> 23) - 126 + 4) : 0;  // |q~| <= sqrt(D) max |q|: at most 2^13
      const float q_scale = rsqrtf((float)D) * __uint_as_float((uint32_t)(127 + e2) << 23);
      q_unit = __uint_as_float((uint32_t)(127 - e2) << 23);
      // (A run at a time, in loops: a piece's beginning and end are long code that runs once, and the instructions' way from memory is most of its time.)
#pragma unroll 1
      for (int set = set0; set < set1; set++) {
        float v[32];
#pragma unroll
        for (int i = 0; i < 32; i++) v[i] = 0.f;
#pragma unroll 1
        for (int r = 0; r < SETS; r++) {
          const float sg = chunk_sign(set, r);
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const uint4 x = q(4 * r + i);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int k = 0; k < 4; k++) {
              const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
              v[8 * i + 2 * k] = fmaf(sg, f.x, v[8 * i + 2 * k]);
              v[8 * i + 2 * k + 1] = fmaf(sg, f.y, v[8 * i + 2 * k + 1]);
            }
          }
        }
        chunk_wht32(v);
        chunk_so4<false>(m + 32 * set, v);
        uint32_t hi[16], lo[16];
#pragma unroll
        for (int k = 0; k < 16; k++) {
          const float a0 = v[2 * k] * q_scale, a1 = v[2 * k + 1] * q_scale;
          hi[k] = pack_half2(a0, a1);
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi[k]));
          lo[k] = pack_half2(a0 - f.x, a1 - f.y);
        }
        tc_st16(tmem + lanes + L::Q_COL + set * 16, hi);
        if constexpr (D == 128) {
          tc_st16(tmem + lanes + L::Q_COL + D / 2 + set * 16, lo);
        } else {
          uint8_t* const slab = smem + L::OFF_Q + (set >> 1) * 16384;
#pragma unroll
          for (int k = 0; k < 4; k++)
            *reinterpret_cast<uint4*>(chunk_swizzled(slab, row, 4 * (set & 1) + k)) = make_uint4(lo[4 * k], lo[4 * k + 1], lo[4 * k + 2], lo[4 * k + 3]);
        }
      }
      tc_wait_st();
      if constexpr (D == 256) fence_proxy_async();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        chunk_arrive(q_ready);
        mbar_arrive(&s.raw_empty);
      }
      return true;
    };

    // What the segments of a piece before the present one have come to, in the thread's own places of the workspace: references and sums of its two
    // rows, then O. Its factors for what is there (`had`) and for the present segment, and their references and sums joined.
    float4* const kept = p.kept + (size_t)blockIdx.x * L::KEPT + tid;
    auto join = [&](bool first, const float (&ref)[2], const float (&sum)[2], float (&had)[2], float (&now)[2]) {
      const float4 x = first ? make_float4(-INFINITY, -INFINITY, 0.f, 0.f) : kept[0];
      float4 y;
      auto both = [](float r0, float l0, float r1, float l1, float& f0, float& f1, float& r, float& l) {
        r = fmaxf(r0, r1);
        f0 = r0 > -INFINITY ? ex2f(r0 - r) : 0.f;  // (nothing seen)
        f1 = r1 > -INFINITY ? ex2f(r1 - r) : 0.f;
        l = fmaf(l0, f0, l1 * f1);
      };
      both(x.x, x.z, ref[0], sum[0], had[0], now[0], y.x, y.z);
      both(x.y, x.w, ref[1], sum[1], had[1], now[1], y.y, y.w);
      return y;
    };
    // O so far = what is there and the present segment's, to the workspace, or (the last segment) back to tensor memory.
    auto join_values = [&](bool first, bool last, const float (&had)[2], const float (&now)[2]) {
#pragma unroll 1
      for (int x = 0; x < D; x += 32) {
        uint32_t o[16];
        float4 y[4];
#pragma unroll
        for (int i = 0; i < 4; i++) y[i] = first ? make_float4(0.f, 0.f, 0.f, 0.f) : kept[256 * (1 + x / 8 + i)];
        chunk_ld_rows(tmem + lanes16 + L::O_COL + x, o);
        tc_wait_ld();
        chunk_landed(o);
#pragma unroll
        for (int i = 0; i < 4; i++) {
          y[i].x = fmaf(__uint_as_float(o[4 * i]), now[0], y[i].x * had[0]);
          y[i].y = fmaf(__uint_as_float(o[4 * i + 1]), now[0], y[i].y * had[0]);
          y[i].z = fmaf(__uint_as_float(o[4 * i + 2]), now[1], y[i].z * had[1]);
          y[i].w = fmaf(__uint_as_float(o[4 * i + 3]), now[1], y[i].w * had[1]);
        }
        if (last) {
#pragma unroll
          for (int i = 0; i < 4; i++) {
            o[4 * i] = __float_as_uint(y[i].x);
            o[4 * i + 1] = __float_as_uint(y[i].y);
            o[4 * i + 2] = __float_as_uint(y[i].z);
            o[4 * i + 3] = __float_as_uint(y[i].w);
          }
          chunk_st_rows(tmem + lanes16 + L::O_COL + x, o);
        } else {
#pragma unroll
          for (int i = 0; i < 4; i++) kept[256 * (1 + x / 8 + i)] = y[i];
        }
      }
    };

    uint32_t pieces = 0;
    bool more = queries(0);
    while (more) {
      const ChunkPiece& c = s.piece[pieces & 3];
      const int steps = (c.hi - c.lo) * SUB;
      float neg_ref[2], limit[2];  // minus the reference; what an exponent may be beside it (-inf: the pair has seen no row of the segment)
      F32x2 l[2];
      auto segment = [&]() {
#pragma unroll
        for (int k = 0; k < 2; k++) {
          neg_ref[k] = 0.f;
          limit[k] = -INFINITY;
          l[k] = f32x2(0.f, 0.f);
        }
      };
      // References and sums of the segment.
      auto sums = [&](float (&ref)[2], float (&sum)[2]) {
#pragma unroll
        for (int k = 0; k < 2; k++) {
          ref[k] = limit[k] > -INFINITY ? -neg_ref[k] : -INFINITY;
          sum[k] = l[k].lo() + l[k].hi();
        }
      };
      segment();
      uint32_t whole_steps = 0;  // of 32 steps, those that all of the CTA's rows see whole: a lane looks at one
      auto first_of = [&](int j) { return c.x.block(c.lo + j / SUB) * 128 + (SUB > 1 ? (j & 1) * NB : 0); };  // a step's first row
      for (int j = 0; j < steps; j++, n++) {
        if ((j & 31) == 0) {
          const int at = c.t * CHUNK_ROWS + first_row;
          const int r = first_of(min(j + lane, steps - 1));
          const int first_pos = c.sq.ctx + at / p.group, last_from = p.window > 0 ? c.sq.ctx + (at + 127) / p.group - p.window + 1 : 0;
          whole_steps = __ballot_sync(FULL, r + NB <= c.x.end && (!p.causal || r + NB - 1 <= first_pos) && (r >= last_from || r + NB <= p.sinks));
        }
        const bool begins = (j & (L::SEGMENT - 1)) == 0;
        if (begins && j > 0) {  // ---- the segment that has ended is added to those before it
          float ref[2], sum[2], had[2], now[2];
          sums(ref, sum);
          const bool first = j == L::SEGMENT;
          const float4 y = join(first, ref, sum, had, now);
          kept[0] = y;
          chunk_wait(&s.o_done[(n - 1) & 1], ((n - 1) >> 1) & 1, p.wait_polls, &s.failed);
          tc_fence_after();
          join_values(first, false, had, now);
          segment();
        }
        const bool whole = whole_steps >> (j & 31) & 1u;
        const uint32_t s_col = tmem + lanes16 + L::S_COL + (n & 1) * NB;
        const float4* const col = &s.column[n % L::COLUMNS][lane & 3];
        const float* const wt = &s.weight[n % L::COLUMNS][2 * (lane & 3)];
        chunk_wait(&s.s_full[n & 1], (n >> 1) & 1, p.wait_polls, &s.failed);
        tc_fence_after();
        // ---- exponents; t[x][k][i]: row row2 + 8 k, columns NC x + 8 i + 2 (lane % 4) and the next
        F32x2 t[PARTS][2][NI];
        {
          uint32_t raw[PARTS][4 * NI];
#pragma unroll
          for (int x = 0; x < PARTS; x++) chunk_ld_rows(s_col + NC * x, raw[x]);
          tc_wait_ld();
#pragma unroll
          for (int x = 0; x < PARTS; x++) chunk_landed(raw[x]);
#pragma unroll
          for (int x = 0; x < PARTS; x++)
#pragma unroll
            for (int i = 0; i < NI; i++) {
              const float4 a = col[(NC * x + 8 * i) / 2];
              const F32x2 ks = mul2(f32x2(a.x, a.y), f32x2(q_unit, q_unit)), lv = f32x2(a.z, a.w);
#pragma unroll
              for (int k = 0; k < 2; k++)
                t[x][k][i] = add2(fma2(f32x2(__uint_as_float(raw[x][4 * i + 2 * k]), __uint_as_float(raw[x][4 * i + 2 * k + 1])), ks, lv), f32x2(neg_ref[k], neg_ref[k]));
            }
        }
        if (!whole) {  // rows are seen up to `last`, of those from `from` on and below the sinks
          const int row0 = first_of(j) + 2 * (lane & 3);
#pragma unroll
          for (int k = 0; k < 2; k++) {
            const int pos = c.sq.ctx + (c.t * CHUNK_ROWS + first_row + row2 + 8 * k) / p.group;
            const int last = p.causal ? min(pos, c.x.end - 1) : c.x.end - 1, from = p.window > 0 ? pos - p.window + 1 : 0;
            uint32_t seen = 0;  // bit 2 (NI x + i) + e: column NC x + 8 i + 2 (lane % 4) + e
#pragma unroll 1
            for (int i = PARTS * NI - 1; i >= 0; i--) {
              const int r = row0 + 8 * i;
              const bool a = r <= last && (r >= from || r < p.sinks), b = r + 1 <= last && (r + 1 >= from || r + 1 < p.sinks);
              seen = seen << 2 | (b ? 2u : 0u) | (a ? 1u : 0u);
            }
#pragma unroll
            for (int x = 0; x < PARTS; x++)
#pragma unroll
              for (int i = 0; i < NI; i++)
                t[x][k][i] = f32x2(seen >> (2 * (NI * x + i)) & 1u ? t[x][k][i].lo() : -INFINITY, seen >> (2 * (NI * x + i)) & 2u ? t[x][k][i].hi() : -INFINITY);
          }
        }
        float top[2];
#pragma unroll
        for (int k = 0; k < 2; k++) {
          top[k] = -INFINITY;
#pragma unroll
          for (int x = 0; x < PARTS; x++)
#pragma unroll
            for (int i = 0; i < NI; i++) top[k] = max3f(top[k], t[x][k][i].lo(), t[x][k][i].hi());
        }
        if (__builtin_expect(__any_sync(FULL, top[0] > limit[0] || top[1] > limit[1]), 0)) {
          // ---- new references for the rows that need one
          float factor[2];
#pragma unroll
          for (int k = 0; k < 2; k++) {
            float most = fmaxf(top[k], __shfl_xor_sync(FULL, top[k], 1));
            most = fmaxf(most, __shfl_xor_sync(FULL, most, 2));
            factor[k] = 1.f;
            if (most > limit[k]) {
              const float less = CHUNK_START - most;
              if (limit[k] > -INFINITY) factor[k] = ex2f(less);
              neg_ref[k] += less;
              limit[k] = CHUNK_LIMIT;
              l[k] = mul2(l[k], f32x2(factor[k], factor[k]));
#pragma unroll
              for (int x = 0; x < PARTS; x++)
#pragma unroll
                for (int i = 0; i < NI; i++) t[x][k][i] = add2(t[x][k][i], f32x2(less, less));
            }
          }
          if (!begins) {
            chunk_wait(&s.o_done[(n - 1) & 1], ((n - 1) >> 1) & 1, p.wait_polls, &s.failed);
            tc_fence_after();
#pragma unroll 1
            for (int x = 0; x < D; x += 16) {
              uint32_t o[8];
              chunk_ld_rows(tmem + lanes16 + L::O_COL + x, o);
              tc_wait_ld();
              chunk_landed(o);
#pragma unroll
              for (int i = 0; i < 8; i++) o[i] = __float_as_uint(__uint_as_float(o[i]) * (i & 2 ? factor[1] : factor[0]));
              chunk_st_rows(tmem + lanes16 + L::O_COL + x, o);
            }
          }
        }
        // ---- weights, over the scores, and their sums
#pragma unroll
        for (int x = 0; x < PARTS; x++) {
          uint32_t pk[2 * NI], rest[2 * NI];
#pragma unroll
          for (int i = 0; i < NI; i++) {
            const float2 a = *reinterpret_cast<const float2*>(wt + NC * x + 8 * i);
#pragma unroll
            for (int k = 0; k < 2; k++) {
              const F32x2 e = f32x2(ex2f(t[x][k][i].lo()), ex2f(t[x][k][i].hi()));
              l[k] = fma2(e, f32x2(a.x, a.y), l[k]);
              pk[2 * i + k] = pack_half2(e.lo(), e.hi());
              rest[2 * i + k] = chunk_rest(pk[2 * i + k], e.lo(), e.hi());
            }
          }
          chunk_st_pairs(s_col + NC * x, pk);
          chunk_st_pairs(s_col + NC * x + NC / 2, rest);
        }
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) chunk_arrive(p_full + 8 * (n & 1));
      }

      // ---- sums and references of the rows
      const bool joined = steps > L::SEGMENT;
      float had[2], now[2];
      {
        float ref[2], sum[2];
        sums(ref, sum);
        if (joined) {
          const float4 y = join(false, ref, sum, had, now);
          ref[0] = y.x;
          ref[1] = y.y;
          sum[0] = y.z;
          sum[1] = y.w;
        }
#pragma unroll
        for (int k = 0; k < 2; k++) {
          float all = sum[k];
          all += __shfl_xor_sync(FULL, all, 1);
          all += __shfl_xor_sync(FULL, all, 2);
          if ((lane & 3) == 0) {
            s.row_sum[row2 + 8 * k] = all;
            s.row_ref[row2 + 8 * k] = ref[k];
          }
        }
      }
      // ---- the next piece's queries come first: its first products run under this one's outputs
      more = queries(pieces + 1);
      const int at = c.t * CHUNK_ROWS + first_row + row, tok = at / p.group, head = c.g * p.group + at - tok * p.group;
      const bool valid = tok < c.sq.n;
      const size_t out_row = ((size_t)c.sq.tok0 + tok) * p.n_q_heads + head;
      cta_bar_sync_n(pair_bar, 64);
      const float sum = s.row_sum[row], ref = s.row_ref[row];
      chunk_wait(&s.o_done[(n - 1) & 1], ((n - 1) >> 1) & 1, p.wait_polls, &s.failed);
      tc_fence_after();
      if (joined) {
        join_values(false, true, had, now);
        tc_wait_st();
        tc_fence_before();
        cta_bar_sync_n(pair_bar, 64);
        tc_fence_after();
      }
      const uint32_t o_col = tmem + lanes + L::O_COL;
      if (c.slot >= 0) {
        // ---- a partial: eight rows of 32 bytes at a time (rows without a token included: nobody reads them)
        float* const dst = p.part_acc + ((size_t)c.slot * CHUNK_ROWS + first_row + row2) * D + 2 * (lane & 3);
#pragma unroll 2
        for (int x = 0; x < D; x += 32) {
          uint32_t o[16];
          chunk_ld_rows(tmem + lanes16 + L::O_COL + x, o);
          tc_wait_ld();
          chunk_landed(o);
#pragma unroll
          for (int i = 0; i < 4; i++)
#pragma unroll
            for (int k = 0; k < 2; k++)
              *reinterpret_cast<float2*>(dst + 8 * k * D + x + 8 * i) =
                  make_float2(__uint_as_float(o[4 * i + 2 * k]) * p.value_unit, __uint_as_float(o[4 * i + 2 * k + 1]) * p.value_unit);
        }
        if (half == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * ((size_t)c.slot * CHUNK_ROWS + first_row + row)) = make_float2(ref, sum);
      } else {
        // ---- o = H M^T o~ / l: runs of 32 coordinates in place, then across the runs
        const float4* const m = s.m[pieces % 3];
        const float unit = sum == 0.f ? 0.f : p.value_unit * rsqrtf((float)D) / sum;
#pragma unroll 1
        for (int set = set0; set < set1; set++) {
          uint32_t r[32];
          float v[32];
          tc_ld32(o_col + 32 * set, r);
          chunk_landed(r);
#pragma unroll
          for (int k = 0; k < 32; k++) v[k] = __uint_as_float(r[k]) * unit;
          chunk_so4<true>(m + 32 * set, v);
          chunk_wht32(v);
#pragma unroll
          for (int i = 0; i < 2; i++) {
            uint32_t y[16];
#pragma unroll
            for (int k = 0; k < 16; k++) y[k] = __float_as_uint(v[16 * i + k]);
            tc_st16(o_col + 32 * set + 16 * i, y);
          }
        }
        tc_wait_st();
        tc_fence_before();
        cta_bar_sync_n(pair_bar, 64);
        tc_fence_after();
        constexpr int XC = 8;  // columns of a run at a time
#pragma unroll 1
        for (int x = 0; x < 32; x += XC) {
          uint32_t u[SETS][XC];
#pragma unroll
          for (int r = 0; r < SETS; r++) chunk_ld8(o_col + 32 * r + x, u[r]);
          tc_wait_ld();
#pragma unroll
          for (int r = 0; r < SETS; r++) chunk_landed(u[r]);
#pragma unroll 1
          for (int set = set0; set < set1; set += 2) {
            float o[2][XC];
#pragma unroll
            for (int i = 0; i < XC; i++) { o[0][i] = __uint_as_float(u[0][i]); o[1][i] = __uint_as_float(u[1][i]); }
#pragma unroll
            for (int r = 2; r < SETS; r += 2) {
              const float sg = chunk_sign(set >> 1, r >> 1);
#pragma unroll
              for (int i = 0; i < XC; i++) {
                o[0][i] = fmaf(sg, __uint_as_float(u[r][i]), o[0][i]);
                o[1][i] = fmaf(sg, __uint_as_float(u[r + 1][i]), o[1][i]);
              }
            }
            if (valid) {
              uint4* const dst = reinterpret_cast<uint4*>(p.out + out_row * D + 32 * set + x);
#pragma unroll
              for (int i = 0; i < XC; i += 8) {
                auto both = [&](int k) { return pack_half2(o[0][k] + o[1][k], o[0][k + 1] + o[1][k + 1]); };
                auto less = [&](int k) { return pack_half2(o[0][k] - o[1][k], o[0][k + 1] - o[1][k + 1]); };
                dst[i / 8] = make_uint4(both(i), both(i + 2), both(i + 4), both(i + 6));
                dst[i / 8 + 4] = make_uint4(less(i), less(i + 2), less(i + 4), less(i + 6));
              }
            }
          }
        }
        if (valid && p.lse && half == 0) p.lse[out_row] = sum == 0.f ? -INFINITY : fmaf(ref, 0.6931471805599453f, logf(sum));
      }
      tc_fence_before();
      cta_bar_sync_n(pair_bar, 64);  // (the sums have been read, and O)
      pieces++;
    }
  }

  allow_dependent_launch();
  __syncthreads();
  if (*(volatile uint32_t*)&s.failed) {  // (set for both CTAs where one of their waits gave up)
    if (tid == 0 && p.status) atomicOr(&p.status[0], IQ_STATUS_WAIT_TIMEOUT);
    if (warp == L::MMA_WARP && rank == 0) {  // products may still be running: they are waited for, with a limit, before the memory goes
      if (elect_one())
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(&s.drain)) : "memory");
      __syncwarp();
      mbar_wait_bounded(&s.drain, 0u, DEC_WAIT_LIMIT);
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  chunk_pair_sync();  // (neither leaves while the other's products or signals need its memory)
  if (warp == L::MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
}

template <int D, int BITS>
static cudaError_t chunk_launch_one(const ChunkParams& p, cudaStream_t stream) {
  static bool configured[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  auto kern = chunk_kernel<D, BITS>;
  if (!configured[dev]) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, CHUNK_SMEM<D>);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  return launch_after_predecessor(kern, dim3(2 * p.pairs), dim3(ChunkLayout<D>::THREADS), CHUNK_SMEM<D>, stream, p);
}
template <int BITS>
static cudaError_t chunk_launch(const ChunkParams& p, int head_dim, cudaStream_t stream) {
  return head_dim == 128 ? chunk_launch_one<128, BITS>(p, stream) : chunk_launch_one<256, BITS>(p, stream);
}
cudaError_t launch_chunk_b2(const ChunkParams& p, int head_dim, cudaStream_t stream);
cudaError_t launch_chunk_b3(const ChunkParams& p, int head_dim, cudaStream_t stream);
cudaError_t launch_chunk_b4(const ChunkParams& p, int head_dim, cudaStream_t stream);

}  // namespace iq
