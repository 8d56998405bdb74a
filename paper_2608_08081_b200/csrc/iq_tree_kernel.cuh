// Attention for drafted tokens over the packed cache: one pass over the blocks of a (sequence, KV head) for up to N (token, query head)
// pairs, the columns.
//
// A block of 128 rows: S[row][column] = A_K B_Q, A_K the levels of the K codes (binary16, exact: the integers of an 8-bit grid or the levels
// themselves), B_Q the rotated queries; t = S scale_row unit - reference_column in units of log2; p = 2^t; O[coordinate][column] += A_V B_P,
// A_V the levels of the V codes (bfloat16), B_P = p times the row's V scale. Both tiles are dequantised into tensor memory (the A operands),
// the queries and probabilities are shared memory (B). A column's sum of p stays with the row's thread until the piece ends; a reference
// that a score leaves behind is raised for all columns, and sums and O scaled. Products with both terms of an operand go to the same
// accumulator.
// q~ is two binary16 terms (22 bits): one term's 11 would be as much error again as the rounding of a binary16 output. p times the V scale
// is two bfloat16 terms, which leave out 2^-18 of it at most, however far it lies below the largest one: where a row takes 99 % of the
// weight and has next to no value the output is the other rows' (with binary16 terms it was off by 1 %). The integers of an 8-bit
// grid are bfloat16 values; other levels (11 bits) are sums of two, and their blocks have two tiles of V levels one after the other (16
// sequences of 16 K rows, 32 columns: 162 us, one tile 132).
//
// What bounds it: neither memory nor a pipe. 32 sequences of up to 32 K rows, 8 KV heads, 32 columns, 3 bits: 0.336 ms = 2.0 TB/s of packed
// rows and 0.23 PFLOP/s; the shift/logic pipe, which has the lookups (216 instructions for 128 codes), is busy half of the time, the
// tensor pipe a quarter, and the schedulers issue in 0.6 of the cycles: a warp has an instruction ready every five cycles or so, and
// the waits between the warpgroups (90 cycles each when there is nothing to wait for) come on top. By measurement (the same launch):
// every warp dequantising and taking half of the softmax 0.44 ms; dequantisation and softmax apart, one control warp 0.38; K, V, each
// product, loads and the search for work in warps of their own 0.37 (the search in one place: the loops then stay in the instruction
// cache, which half of the fetches missed before); two softmax groups 0.39; one CTA per SM with two blocks to a step and everything in
// pairs 0.35; two groups each for K and V 0.37; this one, pairs of everything and one wait per block, with two CTAs, 0.33 (the fp32 sums and
// bfloat16 terms, which came later, and a better share of the work: 0.336).
#pragma once
#include "iq_decode_common.cuh"
#include "iq_format.cuh"
#include "iq_tree_common.cuh"

namespace iq {

// Warpgroups of a CTA: one or two for the softmax (a thread to a cache row; two: half of the columns each), one that dequantises K (a thread
// to a row), one that dequantises V (a thread to a coordinate), and one of which a warp each issues the score products, issues the value
// products, loads, and finds the work.

// A score this far (log2) above its column's reference raises the references, to this far above the block's maximum. (fp32 and
// bfloat16 have room for more; further from the reference a score relative to it is rounded more coarsely.)
constexpr float TREE_RAISE = 16.f;
constexpr float TREE_HEADROOM = 2.f;
// The tensor core cuts its sums off, always towards zero: 3e-7 of the sum a block in the values of a piece (160 blocks: 4.9e-5 of the
// output). They are added up in fp32 in the piece's partial after every so many tiles of V levels. (Every 8: 32 columns and 220 blocks
// to a CTA 345 us, 16: 338, 32: 334, with shrinkage of 2e-6, 4e-6 and twice that.)
constexpr int TREE_FOLD = 16;

// The pieces of a CTA's range: runs of blocks of an item. One warp walks along the range and leaves the pieces in shared memory, up to
// TREE_BATCH at a time, the next ones while the others work on these.
struct TreePiece {
  TreeSeq sq;
  int b, g, tile, lo, hi;
  size_t item;
};
constexpr int TREE_BATCH = 16;
struct TreeBatch {
  int pieces, blocks;
  TreePiece piece[TREE_BATCH];
};

constexpr int TREE_STAGES = 6;  // at most
template <int N>
struct TreeShared {
  uint64_t full[TREE_STAGES], taken[TREE_STAGES], q_ready, drain;
  uint64_t k_ready[2], s_done[2], s_read[2], p_ready[2], o_done[2];  // of even and odd blocks
  uint64_t v_ready[2], v_used[2];  // of even and odd tiles of V levels
  uint32_t tmem, failed;
  uint32_t fresh[2];                // the values of an even or odd block start the accumulator anew
  alignas(16) float neg_ref[N];     // minus the reference of each column, log2 units
  alignas(16) float l_factor[N];    // of the last raise
  alignas(16) float warp_max[4][N];             // per quarter of the rows; at the end of a piece: sums
  float warp_q[16];
  int token[N];                     // the token of a column, counted from the tile's first
  TreeMasks<N> masks;
  TreeBatch batch[2];
};

template <int D, int BITS, int N>
struct TreeLayout {
  static constexpr int DJ = D / 128;
  static constexpr int P = PackedFormat<BITS>::row_bytes(D);
  static constexpr int TILE_BYTES = 128 * P;                   // K rows of a block, or V records
  static constexpr int BLOCK_BYTES = 2 * TILE_BYTES + 2 * 512; // with the scales
  static constexpr int CTAS = tree_ctas_per_sm(D, N);
  static constexpr int BQ_LBO = N * 16 + 16;                   // bytes between the 8-coordinate groups of B_Q (16 more than they take: no bank conflicts)
  static constexpr int BQ_TERM = D / 8 * BQ_LBO;
  static constexpr int BP_LBO = 128, BP_SBO = 2048;
  static constexpr int BP_TERM = N / 8 * BP_SBO;
  static constexpr int SHARED = (sizeof(TreeShared<N>) + 127) / 128 * 128;
  static constexpr int FIXED = SHARED + 2 * 2 * BP_TERM + 2 * BQ_TERM;  // the probabilities of two blocks, the queries; two terms each
  static constexpr int ROOM = (228 / CTAS - 1) * 1024;         // shared memory of a CTA
  static constexpr int FIT = (ROOM - FIXED) / BLOCK_BYTES;
  static constexpr int STAGES = FIT < TREE_STAGES ? FIT : TREE_STAGES;
  static constexpr int SMEM = FIXED + STAGES * BLOCK_BYTES;
  // Warpgroups of the softmax, columns of a thread. Every thread has some 150 instructions a block beside those of its columns, so four
  // groups are slower than two (64 columns, a sequence of 32 K rows: 132 us instead of 120).
  static constexpr int SW = CTAS == 2 ? 1 : 2, NC = N / SW;
  static constexpr int SOFTMAX = 128 * SW, THREADS = SOFTMAX + 3 * 128;
  static constexpr int K_WARP = 4 * SW, V_WARP = K_WARP + 4, QK_WARP = V_WARP + 4, PV_WARP = QK_WARP + 1, LOAD_WARP = QK_WARP + 2, WALK_WARP = QK_WARP + 3;
  // Registers of a thread where two CTAs share an SM: 64 at launch, 256 over the four groups; a softmax thread holds N sums and N scores.
  static constexpr int SOFTMAX_REGS = N == 16 ? 88 : 112, OTHER_REGS = N == 16 ? 56 : 48;
  // tensor memory: K tiles (binary16, two to a column), V tiles, scores, values; two of a kind where they
  // fit, so that the next one is made while this one is used
  static constexpr int COLS = 512 / CTAS, TILE_COLS = 64 * DJ;
  static constexpr int V_BUFS = 3 * TILE_COLS + N + DJ * N <= COLS ? 2 : 1;
  static constexpr int K_BUFS = (2 + V_BUFS) * TILE_COLS + N + DJ * N <= COLS ? 2 : 1;
  static constexpr int S_BUFS = (K_BUFS + V_BUFS) * TILE_COLS + 2 * N + DJ * N <= COLS ? 2 : 1;
  static constexpr int K_COL = 0, V_COL = K_BUFS * TILE_COLS, S_COL = V_COL + V_BUFS * TILE_COLS, O_COL = S_COL + S_BUFS * N;
  static_assert(O_COL + DJ * N <= COLS, "tensor memory");
  static_assert(STAGES >= 2 && SMEM <= ROOM, "shared memory");
  // fp32 result, M = 128; scores: binary16 operands, B_Q K-major; values: bfloat16 operands, B_P MN-major
  static constexpr uint32_t IDESC_Q = (1u << 4) | (((uint32_t)N >> 3) << 17) | ((128u >> 4) << 24);
  static constexpr uint32_t IDESC_P = IDESC_Q | (1u << 7) | (1u << 10) | (1u << 16);
};

// Bounded wait of a converged warp. A wait that gives up is noted in `failed`, and from then on no wait of the CTA lasts: every thread
// goes on through the same loops and barriers over whatever is there, so that the CTA ends together.
__device__ __forceinline__ void tree_wait(uint64_t* bar, uint32_t parity, uint32_t limit, uint32_t* failed);
// The wait for block n on a pair of barriers, one for even and one for odd blocks.
__device__ __forceinline__ void tree_wait2(uint64_t* bars, uint32_t n, uint32_t limit, uint32_t* failed) { tree_wait(bars + (n & 1), (n >> 1) & 1, limit, failed); }
__device__ __forceinline__ void tree_wait(uint64_t* bar, uint32_t parity, uint32_t limit, uint32_t* failed) {
  for (uint32_t i = 0; !mbar_try_wait(bar, parity); i++)
    if (i >= limit || *(volatile uint32_t*)failed) { *(volatile uint32_t*)failed = 1; break; }
  __syncwarp();
}

// The same answer for all lanes of a converged warp.
__device__ __forceinline__ bool tree_failed(const uint32_t* failed) { return __any_sync(FULL, *(const volatile uint32_t*)failed != 0); }

template <int C>
__device__ __forceinline__ void tree_ld(uint32_t taddr, float (&o)[C]) {
  static_assert(C == 8 || C == 16 || C == 32, "columns");
  uint32_t r[C];
  if constexpr (C == 8) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
  } else if constexpr (C == 16) {
    tc_ld16_issue(taddr, r);
  } else {
    uint32_t a[16], b[16];
    tc_ld16_issue(taddr, a);
    tc_ld16_issue(taddr + 16, b);
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; i++) { r[i] = a[i]; r[16 + i] = b[i]; }
  }
  if constexpr (C != 32) tc_wait_ld();
#pragma unroll
  for (int i = 0; i < C; i++) o[i] = __uint_as_float(r[i]);
}
// A pair of values as two bfloat16 terms each, 2^-18 of the value left out. The difference is a mixed-precision subtraction: without the
// shift and mask that would make fp32 values of the first terms (64 columns 186 us instead of 188).
__device__ __forceinline__ void tree_two_terms(float y0, float y1, uint32_t& first, uint32_t& second) {
  first = pack_bf162(y0, y1);
  float r0, r1;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tsub.rn.f32.bf16 %0, l, %3;\n\tsub.rn.f32.bf16 %1, h, %4;\n\t}" : "=f"(r0), "=f"(r1) : "r"(first), "f"(y0), "f"(y1));
  second = pack_bf162(-r0, -r1);
}

// 128 codes of a packed run in shared memory -> 64 columns of the thread's tensor-memory lane.
template <int BITS>
__device__ __forceinline__ void tree_dequant(const uint8_t* run, const uint32_t (&lo)[4], const uint32_t (&hi)[4], LookupConst c, uint32_t taddr) {
  uint32_t w[4 * BITS];
#pragma unroll
  for (int i = 0; i < BITS; i++) {
    const uint4 x = reinterpret_cast<const uint4*>(run)[i];
    w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
  }
#pragma unroll
  for (int u = 0; u < 4; u++) {
    uint32_t o[16];
    dequant32_f16<BITS>(w + u * BITS, lo, hi, c, o);
    tc_st16(taddr + 16 * u, o);
  }
}

// Sum over the warp's lanes of each of C values per lane, the lanes trading halves of their values: lane l ends with the sum of value
// l / (32 / C).
template <int C, int X = 16>
__device__ __forceinline__ float tree_reduce(const float (&v)[C], int lane) {
  if constexpr (C == 1) {
    float r = v[0];
#pragma unroll
    for (int x = X; x > 0; x >>= 1) r += __shfl_xor_sync(FULL, r, x);
    return r;
  } else {
    float h[C / 2];
    const bool up = lane & X;
#pragma unroll
    for (int i = 0; i < C / 2; i++) h[i] = (up ? v[i + C / 2] : v[i]) + __shfl_xor_sync(FULL, up ? v[i] : v[i + C / 2], X);
    return tree_reduce<C / 2, X / 2>(h, lane);
  }
}
__device__ __forceinline__ float tree_warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// The queries of a piece by W warps (this one is warp w): q~ = R q as two binary16 terms of the operand B_Q, times one power of two for
// all of the tile (|q~_i| <= sqrt(d) max |q|). Returns that power's exponent. Two barriers `bar` of `threads`.
template <int D, int BITS, int N>
__device__ __forceinline__ int tree_queries(const TreeParams& p, TreeShared<N>& s, uint8_t* bq, const TreePiece& c, int q0, int nq, int w, int W,
                                            int bar, int threads, int lane) {
  using L = TreeLayout<D, BITS, N>;
  constexpr int E = D / 32;
  auto load = [&](int n, uint32_t (&raw)[E / 2]) {
    const int t = (q0 + n) / p.group, h = c.g * p.group + (q0 + n) - t * p.group;
    const __half* q = p.q + (p.token_start ? c.sq.tok0 * p.qs_t : c.b * p.qs_b) + t * p.qs_t + h * p.qs_h + lane * E;
    if constexpr (E == 4) {
      const uint2 x = *reinterpret_cast<const uint2*>(q);
      raw[0] = x.x; raw[1] = x.y;
    } else {
      const uint4 x = *reinterpret_cast<const uint4*>(q);
      raw[0] = x.x; raw[1] = x.y; raw[E / 2 - 2] = x.z; raw[E / 2 - 1] = x.w;
    }
  };
  float qmax = 0.f;
#pragma unroll 4
  for (int n = w; n < nq; n += W) {
    uint32_t raw[E / 2];
    load(n, raw);
#pragma unroll
    for (int e = 0; e < E / 2; e++) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&raw[e]));
      qmax = fmaxf(qmax, fminf(fmaxf(fabsf(f.x), fabsf(f.y)), 65504.f));  // (an infinite query is its own affair)
    }
  }
  qmax = tree_warp_max(qmax);
  if (lane == 0) s.warp_q[w] = qmax;
  QuatPairs<E> qp;
  qp.load(p.rot + (size_t)c.g * (D / 4) * 8, lane);
  cta_bar_sync_n(bar, threads);
  for (int k = 0; k < W; k++) qmax = fmaxf(qmax, s.warp_q[k]);
  const int e2 = qmax > 0.f ? 13 - ((int)(__float_as_uint(qmax) >> 23) - 126 + 4) : 0;  // (sqrt(d) <= 2^4; at most 2^13)
  const float scale = rsqrtf((float)D) * __uint_as_float((uint32_t)(127 + e2) << 23);
#pragma unroll 2
  for (int n = w; n < N; n += W) {
    uint8_t* const dst = bq + (n >> 3) * 128 + (n & 7) * 16 + (E == 4 ? (lane >> 1) * L::BQ_LBO + (lane & 1) * 8 : lane * L::BQ_LBO);
    if (n >= nq) {
      if constexpr (E == 4) *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<uint2*>(dst + L::BQ_TERM) = make_uint2(0u, 0u);
      else *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<uint4*>(dst + L::BQ_TERM) = make_uint4(0u, 0u, 0u, 0u);
      continue;
    }
    uint32_t raw[E / 2];
    load(n, raw);
    float x[E];
#pragma unroll
    for (int e = 0; e < E / 2; e++) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&raw[e]));
      x[2 * e] = f.x; x[2 * e + 1] = f.y;
    }
    wht_warp<float, E>(x, lane);
    qp.template apply<false>(x);
    uint32_t hi[E / 2], lo[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; e++) {
      const float a0 = x[2 * e] * scale, a1 = x[2 * e + 1] * scale;
      hi[e] = pack_half2(a0, a1);
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi[e]));
      lo[e] = pack_half2(a0 - f.x, a1 - f.y);
    }
    if constexpr (E == 4) {
      *reinterpret_cast<uint2*>(dst) = make_uint2(hi[0], hi[1]);
      *reinterpret_cast<uint2*>(dst + L::BQ_TERM) = make_uint2(lo[0], lo[1]);
    } else {
      *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[E / 2 - 2], hi[E / 2 - 1]);
      *reinterpret_cast<uint4*>(dst + L::BQ_TERM) = make_uint4(lo[0], lo[1], lo[E / 2 - 2], lo[E / 2 - 1]);
    }
  }
  fence_proxy_async();
  cta_bar_sync_n(bar, threads);
  return e2;
}

template <int D, int BITS, int N>
__global__ void __launch_bounds__((TreeLayout<D, BITS, N>::THREADS), (TreeLayout<D, BITS, N>::CTAS)) tree_kernel(const __grid_constant__ TreeParams p) {
  using L = TreeLayout<D, BITS, N>;
  constexpr int DJ = L::DJ, NST = L::STAGES, NC = L::NC;
  extern __shared__ __align__(1024) uint8_t smem[];
  TreeShared<N>& s = *reinterpret_cast<TreeShared<N>*>(smem);
  uint8_t* const bp = smem + L::SHARED;
  uint8_t* const bq = bp + 2 * 2 * L::BP_TERM;
  uint8_t* const stages = bq + 2 * L::BQ_TERM;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);

  if (tid == 0) {
    for (int i = 0; i < NST; i++) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.taken[i], 1);
    }
    mbar_init(&s.q_ready, 4 * L::SW);
    for (int i = 0; i < 2; i++) {
      mbar_init(&s.k_ready[i], 4);
      mbar_init(&s.v_ready[i], 4);
      mbar_init(&s.v_used[i], 1);
      mbar_init(&s.o_done[i], 1);
      mbar_init(&s.p_ready[i], 4 * L::SW);
      mbar_init(&s.s_done[i], 1);
      mbar_init(&s.s_read[i], 4 * L::SW);
    }
    mbar_init(&s.drain, 2);
    s.failed = 0;
    fence_mbar_init();
    fence_proxy_async();
  }
  if (warp == L::QK_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem)), "r"(L::COLS));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
  }
  grid_dependency_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(FULL, s.tmem, 0);
  const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's quarter of the tensor-memory lanes
  uint32_t i = 0;  // blocks of the CTA so far
  // Batch k of pieces is there (false: an empty one, the range is done), and the one before it has been worked off by everybody.
  auto batch = [&](int k) {
    cta_bar_sync_n(3, L::THREADS);
    return s.batch[k & 1].pieces != 0;
  };

  if (warp >= L::QK_WARP) {
    if constexpr (L::CTAS == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::OTHER_REGS));
    if (warp == L::LOAD_WARP) {
      // ---- loads: block i into stage i % NST, when block i - NST has been taken
      const uint32_t sc_bytes = p.scale_f16 ? 256u : 512u;
      const size_t sc_size = p.scale_f16 ? 2 : 4;
      for (int k = 0; batch(k); k++) for (int j = 0; j < s.batch[k & 1].pieces; j++) {
        const TreePiece c = s.batch[k & 1].piece[j];
        for (int v = c.lo; v < c.hi && !tree_failed(&s.failed); v++, i++) {
          const int st = i % NST;
          const size_t row0 = tree_block_row(p, c.b, c.g, c.sq, v, lane == 0 ? p.status : nullptr);
          if (i >= NST) tree_wait(&s.taken[st], (i / NST - 1) & 1, p.wait_polls, &s.failed);
          if (tree_failed(&s.failed)) break;  // (a second load on a barrier that still expects the first is no use to anybody)
          if (elect_one()) {
            uint8_t* const dst = stages + st * L::BLOCK_BYTES;
            mbar_expect_tx(&s.full[st], 2 * L::TILE_BYTES + 2 * sc_bytes);
            bulk_g2s(dst, p.k_codes + row0 * L::P, L::TILE_BYTES, &s.full[st]);
            bulk_g2s(dst + 2 * L::TILE_BYTES, reinterpret_cast<const uint8_t*>(p.k_scales) + row0 * sc_size, sc_bytes, &s.full[st]);
            bulk_g2s(dst + L::TILE_BYTES, p.v_codes + row0 * L::P, L::TILE_BYTES, &s.full[st]);
            bulk_g2s(dst + 2 * L::TILE_BYTES + 512, reinterpret_cast<const uint8_t*>(p.v_scales) + row0 * sc_size, sc_bytes, &s.full[st]);
          }
          __syncwarp();
        }
      }
      // every copy that was asked for has landed (where no wait gave up: at once)
      for (uint32_t m = i > NST ? i - NST : 0; m < i; m++) mbar_wait_bounded(&s.full[m % NST], (m / NST) & 1, DEC_WAIT_LIMIT);
    } else if (warp == L::QK_WARP) {
      // ---- score products. (Those of a piece's first block wait for its queries, which wait for the piece before.)
      const uint64_t desc = smem_desc_mn(smem_u32(bq), L::BQ_LBO, 128);
      uint32_t pieces = 0;
      for (int k = 0; batch(k); k++) for (int j = 0; j < s.batch[k & 1].pieces; j++) {
        tree_wait(&s.q_ready, pieces & 1, p.wait_polls, &s.failed);
        pieces++;
        for (const uint32_t end = i + s.batch[k & 1].piece[j].hi - s.batch[k & 1].piece[j].lo; i < end; i++) {
          if (i >= L::S_BUFS) tree_wait2(s.s_read, i - L::S_BUFS, p.wait_polls, &s.failed);  // the scores before have been read
          // and the probabilities of the block before last: the softmax, which waits for the scores, need not ask
          if (i > 1) tree_wait2(s.o_done, i - 2, p.wait_polls, &s.failed);
          tree_wait2(s.k_ready, i, p.wait_polls, &s.failed);
          tc_fence_after();
          if (elect_one()) {
            const uint32_t d = tmem + L::S_COL + (L::S_BUFS == 2 ? (i & 1) * N : 0), a = tmem + L::K_COL + (L::K_BUFS == 2 ? (i & 1) * L::TILE_COLS : 0);
#pragma unroll 1
            for (int t = 0; t < 2 * DJ; t++) {  // terms of q~, halves of the coordinates: the second terms first, while there is little to cut off
              const uint32_t at = (t & (DJ - 1)) * 16 * L::BQ_LBO + (t < DJ ? L::BQ_TERM : 0);
#pragma unroll
              for (int m = 0; m < 8; m++)
                tc_mma_f16(d, a + (t & (DJ - 1)) * 64 + 8 * m, desc + ((at + 2 * m * L::BQ_LBO) >> 4), L::IDESC_Q, t || m);
            }
            tc_commit(&s.s_done[i & 1]);
          }
          __syncwarp();
        }
      }
    } else if (warp == L::PV_WARP) {
      // ---- value products
      const uint64_t desc = smem_desc_mn(smem_u32(bp), L::BP_LBO, L::BP_SBO);
      uint32_t tile = 0;  // of V levels so far
      for (int k = 0; batch(k); k++) for (int j = 0; j < s.batch[k & 1].pieces; j++) {
        for (const uint32_t end = i + s.batch[k & 1].piece[j].hi - s.batch[k & 1].piece[j].lo; i < end; i++) {
          tree_wait2(s.p_ready, i, p.wait_polls, &s.failed);
          const uint32_t more = !*(volatile uint32_t*)&s.fresh[i & 1];
#pragma unroll 1
          for (int y = 0; y < p.v_terms; y++, tile++) {  // terms of the levels; of the second one's products the smaller is left out
            tree_wait2(s.v_ready, tile, p.wait_polls, &s.failed);
            tc_fence_after();
            if (elect_one()) {
              const uint32_t a = tmem + L::V_COL + (L::V_BUFS == 2 ? (tile & 1) * L::TILE_COLS : 0);
#pragma unroll 1
              for (int t = 0; t < 2 * DJ; t += 1 + y) {  // terms of the probabilities, halves of the coordinates
                const uint32_t x = t >> 1, at = ((t & 1) + 2 * (i & 1)) * L::BP_TERM;
#pragma unroll
                for (int m = 0; m < 8; m++)
                  tc_mma_f16(tmem + L::O_COL + x * N, a + 64 * x + 8 * m, desc + ((at + 2 * m * L::BP_LBO) >> 4), L::IDESC_P, more || y || (t & 1) || m);
              }
              if (p.v_terms > 1) tc_commit(&s.v_used[tile & 1]);
              if (y + 1 == p.v_terms) {
                mbar_arrive(&s.taken[i % NST]);
                tc_commit(&s.o_done[i & 1]);
              }
            }
            __syncwarp();
          }
        }
      }
    }
    else if (warp == L::WALK_WARP) {
      // ---- the pieces
      const TreeRange range = tree_range<N>(p, lane);
      long long at = range.at, seq_at = range.seq_at;
      int b = range.b;
      TreeSeq sq;
      if (at < range.end) sq = tree_seq<N>(p, b);
      for (int k = 0;; k++) {
        TreeBatch& out = s.batch[k & 1];
        int count = 0, blocks = 0;
        while (count < TREE_BATCH && at < range.end) {
          if (at >= seq_at + sq.weight) { seq_at += sq.weight; sq = tree_seq<N>(p, ++b); continue; }
          const int len = sq.blocks + TREE_SEG_COST;
          const int m = (int)unit_div(at - seq_at, len);  // item of the sequence
          const long long item_at = seq_at + (long long)m * len;
          const int off = (int)(at - item_at), take = (int)min((long long)(len - off), range.end - at);
          const int lo = max(off - TREE_SEG_COST, 0), hi = max(off + take - TREE_SEG_COST, 0), g = m / sq.tiles, tile = m - g * sq.tiles;
          const size_t item = ((size_t)b * p.n_kv_heads + g) * p.tiles + tile;
          at += take;
          if (off == 0 && lane == 0) {  // the item starts here: which CTAs have its blocks
            int2 info = make_int2(0, 0);
            if (sq.blocks) {
              info.x = tree_cta_of(item_at + TREE_SEG_COST, range.total, range.ctas);
              info.y = tree_cta_of(item_at + len - 1, range.total, range.ctas) - info.x + 1;
            }
            p.item_info[item] = info;
          }
          if (lo < hi) {
            if (lane == 0) out.piece[count] = {sq, b, g, tile, lo, hi, item};
            count++;
            blocks += hi - lo;
          }
        }
        if (lane == 0) { out.pieces = count; out.blocks = blocks; }
        cta_bar_sync_n(3, L::THREADS);
        if (count == 0) break;
      }
    }
  } else if (warp >= L::K_WARP) {
    if constexpr (L::CTAS == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::OTHER_REGS));
    // ---- dequantisation. One loop for both sides, and its parts rolled up where they repeat: the code that the SM's warps run side by
    // side has to fit its instruction cache.
    const int r = tid & 127;
    const bool k_side = warp < L::V_WARP;
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int x = 0; x < 4; x++) {
      lo[x] = k_side ? p.lut_lo[x] : p.lut_v_lo[0][x];
      hi[x] = k_side ? p.lut_hi[x] : p.lut_v_hi[0][x];
    }
    const int terms = k_side ? 1 : p.v_terms;
    uint32_t n = 0;  // tiles so far
    const uint8_t* const run = stages + (k_side ? r * L::P : L::TILE_BYTES + r * (16 * BITS));
    const int next = k_side ? 16 * BITS : 128 * 16 * BITS;
    const uint32_t col = tmem + lanes + (k_side ? L::K_COL : L::V_COL), bufs = k_side ? L::K_BUFS : L::V_BUFS;
    uint64_t* const ready = k_side ? s.k_ready : s.v_ready;
    uint64_t* const used = k_side ? s.s_done : terms > 1 ? s.v_used : s.o_done;
    for (int k = 0; batch(k); k++) {
      if (k == 0) {  // a hand with the first piece's queries, while its first tiles come
        const TreePiece c = s.batch[0].piece[0];
        const int q0 = c.tile * N;
        tree_queries<D, BITS, N>(p, s, bq, c, q0, min(N, c.sq.tokens * p.group - q0), warp, 4 * L::SW + 8, 2, L::SOFTMAX + 256, lane);
      }
      for (const uint32_t end = i + s.batch[k & 1].blocks; i < end; i++) {
        const uint32_t st = i % NST;
        tree_wait(&s.full[st], (i / NST) & 1, p.wait_polls, &s.failed);
#pragma unroll 1
        for (int y = 0; y < terms; y++, n++) {
          if (terms > 1) {
#pragma unroll
            for (int x = 0; x < 4; x++) {
              lo[x] = p.lut_v_lo[y][x];
              hi[x] = p.lut_v_hi[y][x];
            }
          }
          if (n >= bufs) tree_wait2(used, n - bufs, p.wait_polls, &s.failed);  // the tile before is read no more
          tc_fence_after();
#pragma unroll 1
          for (int x = 0; x < DJ; x++)
            tree_dequant<BITS>(run + st * L::BLOCK_BYTES + x * next, lo, hi, p.lookup, col + (bufs == 2 ? (n & 1) * L::TILE_COLS : 0) + 64 * x);
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(ready + (n & 1));
        }
      }
    }
  } else {
    // ---- softmax
    if constexpr (L::CTAS == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::SOFTMAX_REGS));
    const int r = tid & 127, c0 = (warp >> 2) * NC;  // the thread's row, its first column
    const uint32_t o_col = tmem + lanes + L::O_COL + c0;
    uint8_t* const bp_row = bp + c0 / 8 * L::BP_SBO + (r & 7) * 16 + (r >> 3) * L::BP_LBO;
    for (int k = 0; batch(k); k++) for (int j = 0; j < s.batch[k & 1].pieces; j++) {
      const TreePiece c = s.batch[k & 1].piece[j];
      const int q0 = c.tile * N, nq = min(N, c.sq.tokens * p.group - q0), t0 = q0 / p.group;
      if (tid == 0) s.masks.from_max = 0;
      cta_bar_sync_n(1, L::SOFTMAX);  // the last piece's references have been read
      const bool first = i == 0;
      const int e2 = tree_queries<D, BITS, N>(p, s, bq, c, q0, nq, warp, 4 * L::SW + (first ? 8 : 0), 2, L::SOFTMAX + (first ? 256 : 0), lane);
      if (lane == 0) mbar_arrive(&s.q_ready);
      // (the first score products run meanwhile)
      tree_masks(p, s.masks, c.b, c.sq, t0, (q0 + nq - 1) / p.group - t0 + 1, tid, L::SOFTMAX);
      if (tid < N) {
        s.neg_ref[tid] = 1e30f;
        s.token[tid] = (q0 + tid) / p.group - t0;
      }
      cta_bar_sync_n(1, L::SOFTMAX);
      const float score_unit = p.score_unit * __uint_as_float((uint32_t)(127 - e2) << 23);

      float l[NC];
#pragma unroll
      for (int n = 0; n < NC; n++) l[n] = 0.f;
      // The values: those of the last `held` blocks in tensor memory, those before in the piece's partial.
      const size_t part = (c.item + blockIdx.x) * N;
      float* const part_row = p.part_acc + (part + c0) * D + r;
      const int fold = TREE_FOLD / p.v_terms;
      int held = 0;
      bool kept = false;
      // blocks that every token of the tile sees in full (those of the sinks are looked at row by row)
      const int from_max = s.masks.from_max, all_from = from_max ? max(c.sq.sink_blocks, ((from_max + 127) >> 7) - c.sq.skipped) : 0;
      const int all_to = (c.sq.ctx >> 7) - c.sq.skipped;
      for (int v = c.lo; v < c.hi; v++, i++) {
        const uint8_t* const st = stages + (i % NST) * L::BLOCK_BYTES + 2 * L::TILE_BYTES;
        const uint32_t s_col = tmem + lanes + L::S_COL + (L::S_BUFS == 2 ? (i & 1) * N : 0) + c0;
        const bool masked = v < all_from || v >= all_to;
        tree_wait2(s.s_done, i, p.wait_polls, &s.failed);  // (and with it the block's copies and the room for its probabilities: see the score products)
        tc_fence_after();
        const float ks = load_scale(st, r, p.scale_f16) * score_unit;
        float vs = load_scale(st + 512, r, p.scale_f16);
        uint32_t sees = 0xFFFFFFFFu;  // bit n: column c0 + n sees the row
        if (__builtin_expect(masked, 0)) {
          const int row = c.sq.block(v) * 128 + r;
          sees = 0;
#pragma unroll 1
          for (int m = 0; m < NC && c0 + m < nq; m++)
            if (tree_sees(s.masks, s.token[c0 + m], row, c.sq.ctx, c.sq.rows, p.sinks)) sees |= 1u << m;
          if (!sees) vs = 0.f;
        }

        // scores relative to the references; -inf where the token does not see the row
        float t[NC];
        auto relative = [&]() {
          tree_ld<NC>(s_col, t);
          const float4* ref = reinterpret_cast<const float4*>(s.neg_ref + c0);
#pragma unroll
          for (int m = 0; m < NC; m += 4) {
            const float4 f = ref[m / 4];
            const F32x2 a = fma2(f32x2(t[m], t[m + 1]), f32x2(ks, ks), f32x2(f.x, f.y)), b = fma2(f32x2(t[m + 2], t[m + 3]), f32x2(ks, ks), f32x2(f.z, f.w));
            t[m] = a.lo(); t[m + 1] = a.hi(); t[m + 2] = b.lo(); t[m + 3] = b.hi();
          }
          if (__builtin_expect(masked, 0)) {
#pragma unroll
            for (int m = 0; m < NC; m++)
              if (!(sees >> m & 1u)) t[m] = -INFINITY;
          }
        };
        relative();
        float top = fmaxf(t[0], t[1]);
#pragma unroll
        for (int m = 2; m < NC; m += 2) top = max3f(top, t[m], t[m + 1]);
        const bool raised = cta_bar_or_n(1, L::SOFTMAX, top > TREE_RAISE);
        if (__builtin_expect(raised, 0)) {
          // ---- new references: the maximum of each column over the block
#pragma unroll 1
          for (int n0 = 0; n0 < NC; n0 += 8) {
            float z[8], m[8];
            tree_ld<8>(s_col + n0, z);
#pragma unroll
            for (int x = 0; x < 8; x++) m[x] = tree_warp_max((sees >> (n0 + x) & 1u) ? z[x] * ks : -3e38f);
            if (lane == 0) {
              *reinterpret_cast<float4*>(&s.warp_max[warp & 3][c0 + n0]) = make_float4(m[0], m[1], m[2], m[3]);
              *reinterpret_cast<float4*>(&s.warp_max[warp & 3][c0 + n0 + 4]) = make_float4(m[4], m[5], m[6], m[7]);
            }
          }
          cta_bar_sync_n(1, L::SOFTMAX);
          if (tid < N) {
            const float m = fmaxf(fmaxf(s.warp_max[0][tid], s.warp_max[1][tid]), fmaxf(s.warp_max[2][tid], s.warp_max[3][tid]));
            const float old = -s.neg_ref[tid];
            const float ref = m > -2e38f ? fmaxf(old, m + TREE_HEADROOM) : old;
            s.neg_ref[tid] = -ref;
            s.l_factor[tid] = ex2f(old - ref);
          }
          cta_bar_sync_n(1, L::SOFTMAX);
#pragma unroll
          for (int m = 0; m < NC; m += 4) {
            const float4 f = *reinterpret_cast<const float4*>(s.l_factor + c0 + m);
            l[m] *= f.x; l[m + 1] *= f.y; l[m + 2] *= f.z; l[m + 3] *= f.w;
          }
          relative();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.s_read[i & 1]);
        // ---- probabilities, and times the V scale as two bfloat16 terms of the operand B_P
        uint8_t* const bp_block = bp_row + (i & 1) * 2 * L::BP_TERM;
#pragma unroll
        for (int n0 = 0; n0 < NC; n0 += 8) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int x = 0; x < 4; x++) {
            const int m = n0 + 2 * x;
            const float p0 = ex2f(t[m]), p1 = ex2f(t[m + 1]);
            const F32x2 ls = add2(f32x2(l[m], l[m + 1]), f32x2(p0, p1)), y = mul2(f32x2(p0, p1), f32x2(vs, vs));
            l[m] = ls.lo();
            l[m + 1] = ls.hi();
            tree_two_terms(y.lo(), y.hi(), hi[x], lo[x]);
          }
          uint8_t* const dst = bp_block + (n0 / 8) * L::BP_SBO;
          *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(dst + L::BP_TERM) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        if (__builtin_expect(masked && !(vs < INFINITY), 0)) {  // an infinite scale, and tokens that do not see its row: 0 instead of 0 times infinity
#pragma unroll 1
          for (int m = 0; m < NC; m++)
            if (!(sees >> m & 1u)) {
              uint8_t* const dst = bp_block + (m / 8) * L::BP_SBO + (m & 7) * 2;
              *reinterpret_cast<uint16_t*>(dst) = 0;
              *reinterpret_cast<uint16_t*>(dst + L::BP_TERM) = 0;
            }
        }
        fence_proxy_async();
        // ---- the values so far into the partial, to the new references. (Sixteen columns at a time where a thread has the registers.)
        constexpr int FC = L::CTAS == 2 ? 16 : 8;
        if (held && (raised || held == fold)) {
          tree_wait2(s.o_done, i - 1, p.wait_polls, &s.failed);
          tc_fence_after();
#pragma unroll 1
          for (int n0 = 0; n0 < DJ * NC; n0 += FC) {
            const int n1 = n0 & (NC - 1), h = n0 / NC;
            float* const dst = part_row + (size_t)n1 * D + 128 * h;
            float o[FC], old[FC];
#pragma unroll
            for (int x = 0; x < FC; x++) old[x] = kept ? dst[x * D] : 0.f;
            tree_ld<FC>(o_col + h * N + n1, o);
#pragma unroll
            for (int x = 0; x < FC; x++) o[x] += old[x];
            if (raised) {
#pragma unroll
              for (int x = 0; x < FC; x++) o[x] *= s.l_factor[c0 + n1 + x];
            }
#pragma unroll
            for (int x = 0; x < FC; x++) dst[x * D] = o[x];
          }
          kept = true;
          held = 0;
        }
        if (tid == 0) s.fresh[i & 1] = held == 0;
        held++;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.p_ready[i & 1]);
      }
      // ---- the piece's partial. Sums over the rows: in the warp, then over the four warps, in a fixed order.
      cta_bar_sync_n(1, L::SOFTMAX);  // (warp_max of a raise has been read)
      {
        const float sum = tree_reduce<NC>(l, lane);
        if (lane % (32 / NC) == 0) s.warp_max[warp & 3][c0 + lane / (32 / NC)] = sum;
      }
      cta_bar_sync_n(1, L::SOFTMAX);
      if (tid < nq) {
        const float sum = (s.warp_max[0][tid] + s.warp_max[1][tid]) + (s.warp_max[2][tid] + s.warp_max[3][tid]);
        *reinterpret_cast<float2*>(p.part_ml + 2 * (part + tid)) = make_float2(-s.neg_ref[tid], sum);
      }
      tree_wait2(s.o_done, i - 1, p.wait_polls, &s.failed);
      tc_fence_after();
#pragma unroll 1
      for (int h = 0; h < DJ; h++)
#pragma unroll 1
        for (int n0 = 0; n0 < NC && c0 + n0 < nq; n0 += 8) {
          float o[8];
          tree_ld<8>(o_col + h * N + n0, o);
          float* const dst = part_row + (size_t)n0 * D + 128 * h;
          if (kept) {
#pragma unroll
            for (int n = 0; n < 8; n++) o[n] += dst[n * D];
          }
#pragma unroll
          for (int n = 0; n < 8; n++)
            if (c0 + n0 + n < nq) dst[n * D] = o[n] * p.value_unit;
        }
      tc_fence_before();
    }
  }

  allow_dependent_launch();
  __syncthreads();
  if (*(volatile uint32_t*)&s.failed) {  // (nobody writes it any more)
    if (tid == 0 && p.status) atomicOr(&p.status[0], IQ_STATUS_WAIT_TIMEOUT);
    if (warp == L::QK_WARP || warp == L::PV_WARP) {  // MMAs may still be running: they are waited for, with a limit, before the tensor memory goes
      if (elect_one()) tc_commit(&s.drain);
      __syncwarp();
      mbar_wait_bounded(&s.drain, 0u, DEC_WAIT_LIMIT);
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == L::QK_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L::COLS));
}

template <int D, int BITS, int N>
static cudaError_t tree_launch_one(const TreeParams& p, cudaStream_t stream) {
  using L = TreeLayout<D, BITS, N>;
  static bool configured[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  auto kern = tree_kernel<D, BITS, N>;
  if (!configured[dev]) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  return launch_after_predecessor(kern, dim3(p.ctas), dim3(L::THREADS), L::SMEM, stream, p);
}
template <int BITS>
static cudaError_t tree_launch(const TreeParams& p, int head_dim, cudaStream_t stream) {
  if (head_dim == 128) return p.tile == 16 ? tree_launch_one<128, BITS, 16>(p, stream) : p.tile == 32 ? tree_launch_one<128, BITS, 32>(p, stream) : tree_launch_one<128, BITS, 64>(p, stream);
  return p.tile == 16 ? tree_launch_one<256, BITS, 16>(p, stream) : p.tile == 32 ? tree_launch_one<256, BITS, 32>(p, stream) : tree_launch_one<256, BITS, 64>(p, stream);
}
cudaError_t launch_tree_b2(const TreeParams& p, int head_dim, cudaStream_t stream);
cudaError_t launch_tree_b3(const TreeParams& p, int head_dim, cudaStream_t stream);
cudaError_t launch_tree_b4(const TreeParams& p, int head_dim, cudaStream_t stream);

}  // namespace iq
