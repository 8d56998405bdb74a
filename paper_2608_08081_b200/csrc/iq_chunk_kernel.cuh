// Attention of any number of new tokens over the packed cache: tiles of 128 (token, query head) pairs of a KV head, one pass over the
// blocks that they see.
//
// A step of NB cached rows: S[pair][row] = Q K^T, Q the rotated queries as two binary16 terms, K the levels of the codes; w = S scale_K + log2(scale_V)
// in units of log2; p = 2^(w - reference_pair); O[pair][coordinate] += p V, V the levels; l_pair += p / scale_V. The output is R^T O / l.
// A row's V scale is part of its exponent, so p is the row's weight in the OUTPUT, and the reference follows the largest of those: p
// goes to the tensor cores as one binary16 value, whose 11 bits hold down to 2^-19 of it and which leaves out less than 2^-30 of it, also where
// a row with most of the weight has next to no value. One term's rounding is as much error as that of the binary16 output; the queries' would
// grow with the scores, so they have two (22 bits; of the tile's largest element, as one power of two scales all of them).
// References are raised only when a weight passes 2^15: then sums and O are scaled (a raised reference lies 5 log2 units below the block's
// maximum).
//
#pragma once
#include "iq_chunk_common.cuh"
#include "iq_format.cuh"
#include "iq_tile_mma.cuh"

namespace iq {

constexpr float CHUNK_LIMIT = 15.f;                // log2 of the largest p ...
constexpr float CHUNK_START = 5.f;                 // ... and of the block's largest behind a raise
constexpr float CHUNK_LEAST_SCALE = 8.67361738e-19f;  // 2^-60: V scales below it count as this

// Layouts of the loads: 16x256b leaves rows lane / 4 and lane / 4 + 8 of 16 and columns 2 (lane % 4), + 1 of every 8 with a thread (so that it needs the
// factors of 16 columns, not of all), 16x128b takes back the same as pairs of binary16 values, one to a column.
__device__ __forceinline__ void chunk_ld_rows(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
               : "r"(taddr) : "memory");
}
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
__device__ __forceinline__ void chunk_st_pairs(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
__device__ __forceinline__ void chunk_st_pairs(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// Values that a tcgen05.ld has left in registers are not used before the wait for it.
template <int C>
__device__ __forceinline__ void chunk_landed(uint32_t (&r)[C]) {
#pragma unroll
  for (int i = 0; i < C; i++) asm volatile("" : "+r"(r[i]));
}
// Unnormalised Walsh-Hadamard transform of 64 values of a thread.
__device__ __forceinline__ void chunk_wht64(float (&v)[64]) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1)
#pragma unroll
    for (int i = 0; i < 64; i++)
      if ((i & s) == 0) {
        const float x = v[i], y = v[i + s];
        v[i] = x + y;
        v[i + s] = x - y;
      }
}
// The 16 SO(4) blocks (or their transposes) of 64 consecutive coordinates; m: their matrices, in shared memory.
template <bool TRANSPOSE>
__device__ __forceinline__ void chunk_so4(const float4* m, float (&v)[64]) {
#pragma unroll
  for (int j = 0; j < 16; j++) {
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
  static constexpr int NB = D == 128 ? 128 : 64;   // cached rows of a step: K and V levels of a step are 32 KB each
  static constexpr int SUB = 128 / NB;             // steps of a block
  static constexpr int NC = NB / 2, NI = NC / 8;   // columns of S that a warp has; groups of 8
  static constexpr int SETS = D / 64;              // runs of 64 coordinates
  static constexpr int SOFTMAX_WARPS = 8, DEQUANT_WARP = 8, MMA_WARP = 12, THREADS = 512;
  // registers of a thread: 128 at launch, 512 over the four groups of warps (the last one's other three warps only wait)
  static constexpr int SOFTMAX_REGS = 168, DEQUANT_REGS = 104, MMA_REGS = 72;
  // tensor memory: Q (D = 128: both terms; 256: the first), two buffers of scores, O. The probabilities of a warp's columns go
  // over their scores, two to a column.
  static constexpr int Q_COL = 0, S_COL = 128, O_COL = 512 - D;
  // shared memory: two buffers each of K and V levels, the second term of Q (D = 256), the rest
  static constexpr int OPERAND = 32768;
  static constexpr int OFF_K = 0, OFF_V = 2 * OPERAND, OFF_Q = 4 * OPERAND;
  static constexpr int OFF_S = OFF_Q + (D == 256 ? 128 * D * 2 : 0);
  static constexpr uint32_t IDESC_QK = (1u << 4) | (((uint32_t)NB >> 3) << 17) | ((128u >> 4) << 24);
  static constexpr uint32_t IDESC_PV = (1u << 4) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
};
template <int D>
struct ChunkShared {
  using L = ChunkLayout<D>;
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];  // of even and odd steps
  uint64_t s_full[2], p_full[2], o_done[2], c_full[4], q_ready, drain;
  uint32_t tmem, failed;
  ChunkRange range;
  alignas(16) float4 m[2][D];             // SO(4) matrices of the KV head of even and odd pieces
  alignas(16) float column[4][3][L::NB];  // of a step's rows: scale of S, log2 of the V scale, 1 / V scale
  alignas(16) float row_max[2][128];      // of the halves of the columns; at the end of a piece: sums
  float row_ref[128];
  float warp_q[L::SOFTMAX_WARPS];
};
template <int D>
constexpr int CHUNK_SMEM = ChunkLayout<D>::OFF_S + (int)sizeof(ChunkShared<D>) + 1024;
static_assert(CHUNK_SMEM<128> <= 232448 && CHUNK_SMEM<256> <= 232448, "shared memory");

// Bounded wait of a converged warp. A wait that gives up is noted in `failed`, and from then on no wait of the CTA lasts: every thread
// goes on through the same loops and barriers over whatever is there, so that the CTA ends together.
__device__ __forceinline__ void chunk_wait(uint64_t* bar, uint32_t parity, uint32_t limit, uint32_t* failed) {
  for (uint32_t i = 0; !mbar_try_wait(bar, parity); i++)
    if (i >= limit || *(volatile uint32_t*)failed) { *(volatile uint32_t*)failed = 1; break; }
  __syncwarp();
}

// Address of the 16-byte chunk c of row r in an operand of rows of 128 bytes, 128-byte swizzle.
__device__ __forceinline__ uint8_t* chunk_swizzled(uint8_t* slab, int r, int c) { return slab + r * 128 + ((c ^ (r & 7)) << 4); }

// The packed words of a step that a dequantising thread loads: 128 entries of K (a row, or half of one), 128 of V (a record, or halves of two).
template <int D, int BITS>
struct ChunkRaw {
  uint32_t k[4 * BITS], v[4 * BITS];
  float ks, vs;
  __device__ __forceinline__ void load(const ChunkParams& p, size_t row0, int sub, int tid, bool seen) {
    constexpr int P = PackedFormat<BITS>::row_bytes(D), R = PackedFormat<BITS>::V_RECORD_BYTES;
    const int row = D == 128 ? tid : sub * 64 + (tid & 63);
    const uint4* kp = reinterpret_cast<const uint4*>(p.k_codes + (row0 + row) * P + (D == 128 ? 0 : (tid >> 6) * (P / 2)));
#pragma unroll
    for (int i = 0; i < BITS; i++) {
      const uint4 x = __ldg(kp + i);
      k[4 * i] = x.x; k[4 * i + 1] = x.y; k[4 * i + 2] = x.z; k[4 * i + 3] = x.w;
    }
    const uint8_t* vp = p.v_codes + row0 * P + tid * R;
    if constexpr (D == 128) {
#pragma unroll
      for (int i = 0; i < BITS; i++) {
        const uint4 x = __ldg(reinterpret_cast<const uint4*>(vp) + i);
        v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; h++)  // records tid and 128 + tid
#pragma unroll
        for (int i = 0; i < BITS; i++) {
          const uint2 x = __ldg(reinterpret_cast<const uint2*>(vp + h * 128 * R + sub * (R / 2)) + i);
          v[2 * BITS * h + 2 * i] = x.x; v[2 * BITS * h + 2 * i + 1] = x.y;
        }
    }
    ks = vs = 0.f;
    if (seen) {  // (rows that no token sees may hold anything)
      ks = load_scale(p.k_scales, row0 + row, p.scale_f16);
      vs = load_scale(p.v_scales, row0 + row, p.scale_f16);
    }
  }
};

template <int D, int BITS>
__global__ void __launch_bounds__(ChunkLayout<D>::THREADS, 1) chunk_kernel(const __grid_constant__ ChunkParams p) {
  using L = ChunkLayout<D>;
  constexpr int NB = L::NB, NC = L::NC, NI = L::NI, SUB = L::SUB, SETS = L::SETS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);  // (the swizzle goes by the address)
  ChunkShared<D>& s = *reinterpret_cast<ChunkShared<D>*>(smem + L::OFF_S);
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);

  if (tid == 0) {
    for (int i = 0; i < 2; i++) {
      mbar_init(&s.k_full[i], 4);
      mbar_init(&s.v_full[i], 4);
      mbar_init(&s.k_empty[i], 1);
      mbar_init(&s.v_empty[i], 1);
      mbar_init(&s.s_full[i], 1);
      mbar_init(&s.o_done[i], 1);
      mbar_init(&s.p_full[i], L::SOFTMAX_WARPS);
    }
    for (int i = 0; i < 4; i++) mbar_init(&s.c_full[i], 4);
    mbar_init(&s.q_ready, L::SOFTMAX_WARPS);
    mbar_init(&s.drain, 1);
    s.failed = 0;
    fence_mbar_init();
    fence_proxy_async();
  }
  if (warp == L::MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem)), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
  }
  grid_dependency_wait();
  if (warp == 0) {
    const ChunkRange r = chunk_range(p, lane);
    if (lane == 0) s.range = r;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(FULL, s.tmem, 0);
  ChunkWalk walk;
  ChunkPiece c;
  uint32_t n = 0;  // steps of the CTA so far

  if (warp >= L::MMA_WARP) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::MMA_REGS));
    if (warp == L::MMA_WARP) {
    walk.start(p, s.range);
    // ================================================================ products
    uint32_t pieces = 0;
    const uint32_t k_smem = smem_u32(smem + L::OFF_K), v_smem = smem_u32(smem + L::OFF_V), q_smem = smem_u32(smem + L::OFF_Q);
    auto values = [&](uint32_t i, bool first) {  // O += P V of step i
      const uint32_t o = i & 1, ph = (i >> 1) & 1;
      chunk_wait(&s.v_full[o], ph, p.wait_polls, &s.failed);
      chunk_wait(&s.p_full[o], ph, p.wait_polls, &s.failed);
      tc_fence_after();
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < NB / 16; k++) {
          const uint32_t a = tmem + L::S_COL + o * NB + (k / (NC / 16)) * NC + (k % (NC / 16)) * 8;
          const uint32_t b = v_smem + o * L::OPERAND + (k >> 2) * (D * 128) + (k & 3) * 32;
          tc_mma_f16(tmem + L::O_COL, a, smem_desc_k128(b), L::IDESC_PV, !(first && k == 0));
        }
        tc_commit(&s.v_empty[o]);
        tc_commit(&s.o_done[o]);
      }
      __syncwarp();
    };
    while (walk.next(p, c)) {
      const int steps = (c.hi - c.lo) * SUB;
      if (steps == 0) continue;
      chunk_wait(&s.q_ready, pieces & 1, p.wait_polls, &s.failed);
      pieces++;
      tc_fence_after();
      for (int j = 0; j < steps; j++, n++) {
        const uint32_t o = n & 1, ph = (n >> 1) & 1;
        chunk_wait(&s.k_full[o], ph, p.wait_polls, &s.failed);
        tc_fence_after();
        if (elect_one()) {  // the second terms first
#pragma unroll
          for (int k = 0; k < 2 * (D / 16); k++) {
            const int kk = k % (D / 16), hi = k / (D / 16);
            const uint64_t b = smem_desc_k128(k_smem + o * L::OPERAND + (kk >> 2) * (NB * 128) + (kk & 3) * 32);
            const uint32_t d = tmem + L::S_COL + o * NB;
            if (D == 256 && !hi) tc_mma_f16_ss(d, smem_desc_k128(q_smem + (kk >> 2) * 16384 + (kk & 3) * 32), b, L::IDESC_QK, k != 0);
            else tc_mma_f16(d, tmem + L::Q_COL + (hi ? 0 : D / 2) + kk * 8, b, L::IDESC_QK, k != 0);
          }
          tc_commit(&s.k_empty[o]);
          tc_commit(&s.s_full[o]);
        }
        __syncwarp();
        if (j > 0) values(n - 1, j == 1);
      }
      values(n - 1, steps == 1);
    }
    }
  } else if (warp >= L::DEQUANT_WARP) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::DEQUANT_REGS));
    walk.start(p, s.range);
    // ================================================================ levels of the codes
    const int t = tid - 32 * L::DEQUANT_WARP;
    // the step to load next, and where its block starts; the table is looked up a step before
    int v = 0, sub = 0;
    bool more = false, have = false, seen = false;
    size_t row0 = 0;
    int next_sub = 0;
    auto locate = [&]() {  // the next step, if there is one
      if (!more || v == c.hi) {
        do more = walk.next(p, c); while (more && c.hi == c.lo);
        v = c.lo;
        sub = 0;
      }
      have = more;
      if (!more) return;
      const int row = c.x.block(v) * 128;
      if (sub == 0) row0 = cache_row(p.pm, c.b, c.g, row, t == 0 ? p.status : nullptr);
      seen = row + (D == 128 ? t : sub * 64 + (t & 63)) < c.x.end;
      next_sub = sub;
      if (++sub == SUB) { sub = 0; v++; }
    };
    ChunkRaw<D, BITS> next;
    locate();
    if (have) next.load(p, row0, next_sub, t, seen);
    while (have) {
      const ChunkRaw<D, BITS> cur = next;
      locate();
      if (have) next.load(p, row0, next_sub, t, seen);
      const uint32_t o = n & 1;
      // ---- K
      if (n >= 2) chunk_wait(&s.k_empty[o], ((n >> 1) - 1) & 1, p.wait_polls, &s.failed);
      if (D == 128 || t < 64) {
        float* const col = &s.column[n & 3][0][t];
        const float vs = cur.vs < CHUNK_LEAST_SCALE ? CHUNK_LEAST_SCALE : cur.vs;
        col[0] = cur.ks * p.score_unit;
        col[NB] = log2f(vs);
        col[2 * NB] = 1.f / vs;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.c_full[n & 3]);
      uint8_t* const kd = smem + L::OFF_K + o * L::OPERAND;
#pragma unroll
      for (int u = 0; u < 4; u++) {
        uint32_t x[16];
        dequant32_f16<BITS>(cur.k + u * BITS, p.lut_lo, p.lut_hi, p.lookup, x);
        const int e = (D == 128 ? 0 : (t >> 6) * 128) + 32 * u, r = D == 128 ? t : t & 63;  // first coordinate
        uint8_t* const slab = kd + (e >> 6) * (NB * 128);
#pragma unroll
        for (int k = 0; k < 4; k++)
          *reinterpret_cast<uint4*>(chunk_swizzled(slab, r, ((e >> 3) & 7) + k)) = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.k_full[o]);
      // ---- V
      if (n >= 2) chunk_wait(&s.v_empty[o], ((n >> 1) - 1) & 1, p.wait_polls, &s.failed);
      uint8_t* const vd = smem + L::OFF_V + o * L::OPERAND;
#pragma unroll
      for (int u = 0; u < 4; u++) {
        uint32_t x[16];
        dequant32_f16<BITS>(cur.v + u * BITS, p.lut_v_lo, p.lut_v_hi, p.lookup, x);
        const int e = D == 128 ? 32 * u : 32 * (u & 1), r = D == 128 ? t : t + 128 * (u >> 1);  // first row, coordinate
        uint8_t* const slab = vd + (e >> 6) * (D * 128);
#pragma unroll
        for (int k = 0; k < 4; k++)
          *reinterpret_cast<uint4*>(chunk_swizzled(slab, r, ((e >> 3) & 7) + k)) = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.v_full[o]);
      n++;
    }
  } else {
    // ================================================================ queries, softmax, outputs
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::SOFTMAX_REGS));
    walk.start(p, s.range);
    const int quad = warp & 3, half = warp >> 2;           // rows 32 quad ..., half of the columns or coordinates
    const uint32_t lanes = (uint32_t)quad << 21;           // the quarter of the tensor-memory lanes
    const int pair_bar = 1 + quad, all_bar = 5;            // barriers: the two warps of the same rows; all
    const int row = 32 * quad + lane;                      // the thread's row where it has one
    const int row4 = 32 * quad + (lane >> 2);              // its four rows in the loop over the blocks: 8 apart
    uint32_t pieces = 0;
    while (walk.next(p, c)) {
      const int steps = (c.hi - c.lo) * SUB;
      const int tok = (c.t * CHUNK_ROWS + row) / p.group, head = c.g * p.group + (c.t * CHUNK_ROWS + row) - tok * p.group;
      const bool valid = tok < c.sq.n;
      const size_t out_row = ((size_t)c.sq.tok0 + tok) * p.n_q_heads + head;
      if (steps == 0) {  // the item's tokens see no row
        if (valid) {
          uint4* const dst = reinterpret_cast<uint4*>(p.out + out_row * D + half * (D / 2));
#pragma unroll 1
          for (int i = 0; i < D / 16; i++) dst[i] = make_uint4(0u, 0u, 0u, 0u);
          if (p.lse && half == 0) p.lse[out_row] = -INFINITY;
        }
        continue;
      }
      // ---- the rotated queries, q~ = M H q, a thread its half of a row's coordinates
      float4* const m = s.m[pieces & 1];
      const __half* const q = p.q + (p.token_start ? (c.sq.tok0 + tok) * p.qs_t : c.b * p.qs_b + tok * p.qs_t) + head * p.qs_h;
      float qmax = 0.f;
      {
        __half2 top = __float2half2_rn(0.f);
        if (valid) {
#pragma unroll
          for (int i = 0; i < D / 16; i++) {
            const uint4 x = *reinterpret_cast<const uint4*>(q + half * (D / 2) + 8 * i);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int k = 0; k < 4; k++) top = __hmax2(top, __habs2(*reinterpret_cast<const __half2*>(&w[k])));
          }
        }
        qmax = fminf(fmaxf(__low2float(top), __high2float(top)), 65504.f);  // (an infinite query is its own affair)
      }
      qmax = warp_max(qmax);
      if (lane == 0) s.warp_q[warp] = qmax;
      if (tid < D / 4) {
        float M[4][4];
        so4_matrix<float>(p.rot + ((size_t)c.g * (D / 4) + tid) * 8, M);
#pragma unroll
        for (int i = 0; i < 4; i++) m[4 * tid + i] = make_float4(M[i][0], M[i][1], M[i][2], M[i][3]);
      }
      cta_bar_sync_n(all_bar, 32 * L::SOFTMAX_WARPS);
#pragma unroll
      for (int k = 0; k < L::SOFTMAX_WARPS; k++) qmax = fmaxf(qmax, s.warp_q[k]);
      const int e2 = qmax > 0.f ? 13 - ((int)(__float_as_uint(qmax) >> 23) - 126 + 4) : 0;  // |q~| <= sqrt(D) max |q|: at most 2^13
      const float q_scale = rsqrtf((float)D) * __uint_as_float((uint32_t)(127 + e2) << 23);
      const float q_unit = __uint_as_float((uint32_t)(127 - e2) << 23);
#pragma unroll 1
      for (int set = half * (SETS / 2); set < (half + 1) * (SETS / 2); set++) {
        float v[64];
#pragma unroll
        for (int i = 0; i < 64; i++) v[i] = 0.f;
        if (valid) {
#pragma unroll 1
          for (int r = 0; r < SETS; r++) {
            const float sg = chunk_sign(set, r);
#pragma unroll
            for (int i = 0; i < 8; i++) {
              const uint4 x = *reinterpret_cast<const uint4*>(q + 64 * r + 8 * i);
              const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int k = 0; k < 4; k++) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
                v[8 * i + 2 * k] = fmaf(sg, f.x, v[8 * i + 2 * k]);
                v[8 * i + 2 * k + 1] = fmaf(sg, f.y, v[8 * i + 2 * k + 1]);
              }
            }
          }
        }
        chunk_wht64(v);
        chunk_so4<false>(m + 64 * set, v);
#pragma unroll
        for (int i = 0; i < 2; i++) {
          uint32_t hi[16], lo[16];
#pragma unroll
          for (int k = 0; k < 16; k++) {
            const float a0 = v[32 * i + 2 * k] * q_scale, a1 = v[32 * i + 2 * k + 1] * q_scale;
            hi[k] = pack_half2(a0, a1);
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi[k]));
            lo[k] = pack_half2(a0 - f.x, a1 - f.y);
          }
          tc_st16(tmem + lanes + L::Q_COL + set * 32 + 16 * i, hi);
          if constexpr (D == 128) {
            tc_st16(tmem + lanes + L::Q_COL + D / 2 + set * 32 + 16 * i, lo);
          } else {
            uint8_t* const slab = smem + L::OFF_Q + set * 16384;
#pragma unroll
            for (int k = 0; k < 4; k++)
              *reinterpret_cast<uint4*>(chunk_swizzled(slab, row, 4 * i + k)) = make_uint4(lo[4 * k], lo[4 * k + 1], lo[4 * k + 2], lo[4 * k + 3]);
          }
        }
      }
      tc_wait_st();
      if constexpr (D == 256) fence_proxy_async();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.q_ready);

      // ---- what the thread's four rows see of a masked step: rows up to `last`, of those from `from` on and below the sinks
      int last[4], from[4];
#pragma unroll
      for (int k = 0; k < 4; k++) {
        const int pos = c.sq.ctx + (c.t * CHUNK_ROWS + row4 + 8 * k) / p.group;
        last[k] = p.causal ? min(pos, c.x.end - 1) : c.x.end - 1;
        from[k] = p.window > 0 ? pos - p.window + 1 : 0;
      }
      const int first_pos = c.sq.ctx + c.x.t0, last_from = p.window > 0 ? c.sq.ctx + c.x.t1 - p.window + 1 : 0;
      float neg_ref[4], limit[4];  // -inf: no row seen so far
      F32x2 l[4];
#pragma unroll
      for (int k = 0; k < 4; k++) {
        neg_ref[k] = 0.f;
        limit[k] = -INFINITY;
        l[k] = f32x2(0.f, 0.f);
      }
      for (int j = 0; j < steps; j++, n++) {
        const int row0 = c.x.block(c.lo + j / SUB) * 128 + (j % SUB) * NB;
        const bool whole = row0 + NB <= c.x.end && (!p.causal || row0 + NB - 1 <= first_pos) && (row0 >= last_from || row0 + NB <= p.sinks);
        const uint32_t s_col = tmem + lanes + L::S_COL + (n & 1) * NB + half * NC;
        chunk_wait(&s.c_full[n & 3], (n >> 2) & 1, p.wait_polls, &s.failed);
        F32x2 ks[NI], lv[NI], rv[NI];
        {
          const float* const col = &s.column[n & 3][0][half * NC + 2 * (lane & 3)];
#pragma unroll
          for (int i = 0; i < NI; i++) {
            const float2 a = *reinterpret_cast<const float2*>(col + 8 * i), b = *reinterpret_cast<const float2*>(col + NB + 8 * i);
            const float2 d = *reinterpret_cast<const float2*>(col + 2 * NB + 8 * i);
            ks[i] = f32x2(a.x * q_unit, a.y * q_unit);
            lv[i] = f32x2(b.x, b.y);
            rv[i] = f32x2(d.x, d.y);
          }
        }
        chunk_wait(&s.s_full[n & 1], (n >> 1) & 1, p.wait_polls, &s.failed);
        tc_fence_after();
        uint32_t raw[2][4 * NI];
        chunk_ld_rows(s_col, raw[0]);
        chunk_ld_rows(s_col + (16u << 16), raw[1]);
        tc_wait_ld();
        chunk_landed(raw[0]);
        chunk_landed(raw[1]);
        // ---- exponents; w[k][i]: row row4 + 8 k, columns 8 i + 2 (lane % 4) and the next
        F32x2 w[4][NI];
        float top[4];
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
          for (int i = 0; i < NI; i++) {
            const int x = 4 * i + 2 * (k & 1);
            w[k][i] = fma2(f32x2(__uint_as_float(raw[k >> 1][x]), __uint_as_float(raw[k >> 1][x + 1])), ks[i], lv[i]);
          }
        if (!whole) {
#pragma unroll
          for (int k = 0; k < 4; k++)
#pragma unroll
            for (int i = 0; i < NI; i++) {
              const int r = row0 + half * NC + 8 * i + 2 * (lane & 3);
              const bool a = r <= last[k] && (r >= from[k] || r < p.sinks), b = r + 1 <= last[k] && (r + 1 >= from[k] || r + 1 < p.sinks);
              w[k][i] = f32x2(a ? w[k][i].lo() : -INFINITY, b ? w[k][i].hi() : -INFINITY);
            }
        }
        bool over = false;
#pragma unroll
        for (int k = 0; k < 4; k++) {
          top[k] = fmaxf(w[k][0].lo(), w[k][0].hi());
#pragma unroll
          for (int i = 1; i < NI; i++) top[k] = max3f(top[k], w[k][i].lo(), w[k][i].hi());
          over |= top[k] > limit[k];
        }
        if (__builtin_expect(cta_bar_or_n(pair_bar, 64, over), 0)) {
          // ---- new references for the rows that need one
#pragma unroll
          for (int k = 0; k < 4; k++) {
            top[k] = fmaxf(top[k], __shfl_xor_sync(FULL, top[k], 1));
            top[k] = fmaxf(top[k], __shfl_xor_sync(FULL, top[k], 2));
            if ((lane & 3) == 0) s.row_max[half][row4 + 8 * k] = top[k];
          }
          cta_bar_sync_n(pair_bar, 64);
          float factor[4];
#pragma unroll
          for (int k = 0; k < 4; k++) {
            const float t = fmaxf(top[k], s.row_max[half ^ 1][row4 + 8 * k]);
            factor[k] = 1.f;
            if (t > limit[k]) {
              const float ref = t - CHUNK_START;
              if (limit[k] > -INFINITY) factor[k] = ex2f(-neg_ref[k] - ref);
              neg_ref[k] = -ref;
              limit[k] = ref + CHUNK_LIMIT;
              l[k] = mul2(l[k], f32x2(factor[k], factor[k]));
            }
          }
          cta_bar_sync_n(pair_bar, 64);  // (row_max has been read)
          if (j > 0) {
            chunk_wait(&s.o_done[(n - 1) & 1], ((n - 1) >> 1) & 1, p.wait_polls, &s.failed);
            tc_fence_after();
#pragma unroll 1
            for (int x = 0; x < 2 * (D / 32); x++) {
              const uint32_t at = tmem + lanes + L::O_COL + half * (D / 2) + (x >> 1) * 16 + ((uint32_t)(x & 1) << 20);
              const float f0 = x & 1 ? factor[2] : factor[0], f1 = x & 1 ? factor[3] : factor[1];
              uint32_t o[8];
              chunk_ld_rows(at, o);
              tc_wait_ld();
              chunk_landed(o);
#pragma unroll
              for (int i = 0; i < 8; i++) o[i] = __float_as_uint(__uint_as_float(o[i]) * (i & 2 ? f1 : f0));
              chunk_st_rows(at, o);
            }
          }
        }
        // ---- weights
#pragma unroll
        for (int x = 0; x < 2; x++) {
          uint32_t pk[2 * NI];
#pragma unroll
          for (int i = 0; i < NI; i++)
#pragma unroll
            for (int y = 0; y < 2; y++) {
              const int k = 2 * x + y;
              const F32x2 t = add2(w[k][i], f32x2(neg_ref[k], neg_ref[k]));
              const float p0 = ex2f(t.lo()), p1 = ex2f(t.hi());
              F32x2 r = rv[i];
              if (!whole) r = f32x2(p0 == 0.f ? 0.f : r.lo(), p1 == 0.f ? 0.f : r.hi());  // (a row that is not seen may have any scale)
              l[k] = fma2(f32x2(p0, p1), r, l[k]);
              pk[2 * i + y] = pack_half2(p0, p1);
            }
          chunk_st_pairs(s_col + ((uint32_t)x << 20), pk);
        }
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.p_full[n & 1]);
      }

      // ---- sums and references of the rows
#pragma unroll
      for (int k = 0; k < 4; k++) {
        float sum = l[k].lo() + l[k].hi();
        sum += __shfl_xor_sync(FULL, sum, 1);
        sum += __shfl_xor_sync(FULL, sum, 2);
        if ((lane & 3) == 0) {
          s.row_max[half][row4 + 8 * k] = sum;
          if (half == 0) s.row_ref[row4 + 8 * k] = limit[k] > -INFINITY ? -neg_ref[k] : -INFINITY;
        }
      }
      cta_bar_sync_n(pair_bar, 64);
      const float sum = s.row_max[0][row] + s.row_max[1][row], ref = s.row_ref[row];
      chunk_wait(&s.o_done[(n - 1) & 1], ((n - 1) >> 1) & 1, p.wait_polls, &s.failed);
      tc_fence_after();
      const uint32_t o_col = tmem + lanes + L::O_COL;
      if (c.slot >= 0) {
        // ---- a partial
        float* const dst = p.part_acc + ((size_t)c.slot * CHUNK_ROWS + row) * D;
#pragma unroll 1
        for (int x = half * (D / 2); x < (half + 1) * (D / 2); x += 16) {
          float o[16];
          tc_ld16(o_col + x, o);
          if (valid) {
#pragma unroll
            for (int i = 0; i < 4; i++)
              *reinterpret_cast<float4*>(dst + x + 4 * i) =
                  make_float4(o[4 * i] * p.value_unit, o[4 * i + 1] * p.value_unit, o[4 * i + 2] * p.value_unit, o[4 * i + 3] * p.value_unit);
          }
        }
        if (half == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * ((size_t)c.slot * CHUNK_ROWS + row)) = make_float2(ref, sum);
      } else {
        // ---- o = H M^T o~ / l: runs of 64 coordinates in place, then across the runs
        const float unit = sum == 0.f ? 0.f : p.value_unit * rsqrtf((float)D) / sum;
#pragma unroll 1
        for (int set = half * (SETS / 2); set < (half + 1) * (SETS / 2); set++) {
          uint32_t r[32];
          float v[64];
#pragma unroll
          for (int i = 0; i < 2; i++) {
            tc_ld32(o_col + 64 * set + 32 * i, r);
            chunk_landed(r);
#pragma unroll
            for (int k = 0; k < 32; k++) v[32 * i + k] = __uint_as_float(r[k]) * unit;
          }
          chunk_so4<true>(m + 64 * set, v);
          chunk_wht64(v);
#pragma unroll
          for (int i = 0; i < 4; i++) {
            uint32_t y[16];
#pragma unroll
            for (int k = 0; k < 16; k++) y[k] = __float_as_uint(v[16 * i + k]);
            tc_st16(o_col + 64 * set + 16 * i, y);
          }
        }
        tc_wait_st();
        tc_fence_before();
        cta_bar_sync_n(pair_bar, 64);
        tc_fence_after();
#pragma unroll 1
        for (int x = 0; x < 64; x += 16) {
          float u[SETS][16];
#pragma unroll
          for (int r = 0; r < SETS; r++) tc_ld16(o_col + 64 * r + x, u[r]);
#pragma unroll 1
          for (int set = half * (SETS / 2); set < (half + 1) * (SETS / 2); set++) {
            float o[16];
#pragma unroll
            for (int i = 0; i < 16; i++) o[i] = u[0][i];
#pragma unroll
            for (int r = 1; r < SETS; r++) {
              const float sg = chunk_sign(set, r);
#pragma unroll
              for (int i = 0; i < 16; i++) o[i] = fmaf(sg, u[r][i], o[i]);
            }
            if (valid) {
              uint4* const dst = reinterpret_cast<uint4*>(p.out + out_row * D + 64 * set + x);
              dst[0] = make_uint4(pack_half2(o[0], o[1]), pack_half2(o[2], o[3]), pack_half2(o[4], o[5]), pack_half2(o[6], o[7]));
              dst[1] = make_uint4(pack_half2(o[8], o[9]), pack_half2(o[10], o[11]), pack_half2(o[12], o[13]), pack_half2(o[14], o[15]));
            }
          }
        }
        if (valid && p.lse && half == 0) p.lse[out_row] = sum == 0.f ? -INFINITY : fmaf(ref, 0.6931471805599453f, logf(sum));
      }
      tc_fence_before();
      cta_bar_sync_n(pair_bar, 64);  // (the sums have been read)
      pieces++;
    }
    if (tid == 0) {  // the item that a later CTA ends, for the merge
      long long* const info = p.cut_info + CHUNK_INFO * blockIdx.x;
      info[0] = walk.info_b;
      info[1] = ((long long)walk.info_g << 32) | (uint32_t)walk.info_t;
      info[2] = walk.info_at;
      info[3] = s.range.total;
    }
  }

  allow_dependent_launch();
  __syncthreads();
  if (*(volatile uint32_t*)&s.failed) {  // (nobody writes it any more)
    if (tid == 0 && p.status) atomicOr(&p.status[0], IQ_STATUS_WAIT_TIMEOUT);
    if (warp == L::MMA_WARP) {  // products may still be running: they are waited for, with a limit, before the tensor memory goes
      if (elect_one()) tc_commit(&s.drain);
      __syncwarp();
      mbar_wait_bounded(&s.drain, 0u, DEC_WAIT_LIMIT);
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == L::MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
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
  return launch_after_predecessor(kern, dim3(p.ctas), dim3(ChunkLayout<D>::THREADS), CHUNK_SMEM<D>, stream, p);
}
template <int BITS>
static cudaError_t chunk_launch(const ChunkParams& p, int head_dim, cudaStream_t stream) {
  return head_dim == 128 ? chunk_launch_one<128, BITS>(p, stream) : chunk_launch_one<256, BITS>(p, stream);
}
cudaError_t launch_chunk_b2(const ChunkParams& p, int head_dim, cudaStream_t stream);
cudaError_t launch_chunk_b3(const ChunkParams& p, int head_dim, cudaStream_t stream);
cudaError_t launch_chunk_b4(const ChunkParams& p, int head_dim, cudaStream_t stream);

}  // namespace iq
