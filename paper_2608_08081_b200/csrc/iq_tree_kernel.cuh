// Attention for drafted tokens over the packed cache: one pass over the blocks of a (sequence, KV head) for up to N (token, query head)
// pairs.
#pragma once
#include "iq_decode_common.cuh"
#include "iq_format.cuh"
#include "iq_tree_common.cuh"

namespace iq {

constexpr int TREE_COMPUTE = 256;                // two groups of four warps
constexpr int TREE_THREADS = TREE_COMPUTE + 32;  // and the control warp
constexpr float TREE_RAISE = 4.f;                // a score this far (log2) above its column's reference raises the references,
constexpr float TREE_HEADROOM = 3.f;             // to this far above the block's maximum
constexpr float TREE_P_UNIT = 1024.f;            // a probability of 1 of a row with the longest V scale as a binary16 operand

template <int N>
struct TreeShared {
  uint64_t full[4], k_ready, s_done, p_ready, o_done, drain;
  uint32_t tmem, failed;
  float neg_ref[N];                 // minus the reference of each column, log2 units
  float l_factor[N], o_factor[N];   // of the last raise
  float warp_max[4][N];             // per quarter of the rows; at the end of a piece: sums
  float warp_v[8], warp_q[8];
  int token[N];                     // the token of a column, counted from the tile's first
  TreeMasks<N> masks;
  long long scratch[TREE_THREADS / 32 + 2];
};

template <int D, int BITS, int N>
struct TreeLayout {
  static constexpr int DJ = D / 128;
  static constexpr int P = PackedFormat<BITS>::row_bytes(D);
  static constexpr int TILE_BYTES = 128 * P;                   // K rows of a block, or V records
  static constexpr int STAGE_BYTES = 2 * TILE_BYTES + 2 * 512;
  static constexpr int BQ_LBO = N * 16 + 16;                   // bytes between the 8-coordinate groups of B_Q (16 more than they take: no bank conflicts)
  static constexpr int BQ_TERM = D / 8 * BQ_LBO;
  static constexpr int BP_LBO = 128, BP_SBO = 2048;
  static constexpr int BP_TERM = N / 8 * BP_SBO;
  static constexpr int SHARED = (sizeof(TreeShared<N>) + 127) / 128 * 128;
  static constexpr int FIXED = SHARED + 2 * BP_TERM + 2 * BQ_TERM;
  static constexpr int CTAS = D == 128 ? 2 : 1;                // per SM
  static constexpr int ROOM = (228 / CTAS - 1) * 1024;         // shared memory of a CTA
  static constexpr int FIT = (ROOM - FIXED) / STAGE_BYTES;
  static constexpr int STAGES = FIT < 4 ? FIT : 4;
  static constexpr int SMEM = FIXED + STAGES * STAGE_BYTES;
  // tensor memory: K tile (binary16, two to a column), V tile, scores, values
  static constexpr int K_COL = 0, V_COL = D / 2, S_COL = V_COL + 64 * DJ, O_COL = S_COL + N;
  static constexpr int COLS = 512 / CTAS;
  static_assert(O_COL + DJ * N <= COLS, "tensor memory");
  static_assert(STAGES >= 2 && SMEM <= ROOM, "shared memory");
  // fp32 result, binary16 operands, M = 128; B_Q K-major, B_P MN-major
  static constexpr uint32_t IDESC_Q = (1u << 4) | (((uint32_t)N >> 3) << 17) | ((128u >> 4) << 24);
  static constexpr uint32_t IDESC_P = IDESC_Q | (1u << 16);
};

// The pieces of a CTA's range: runs of blocks of an item.
struct TreePiece {
  TreeSeq sq;
  int b, g, tile, lo, hi;
};
struct TreeWalk {
  long long at, seq_at;
  int b;
  __device__ __forceinline__ void start(const TreeRange& r) { at = r.at; seq_at = r.seq_at; b = r.b; }
  __device__ __forceinline__ size_t item(const TreeParams& p, const TreePiece& c) const { return ((size_t)c.b * p.n_kv_heads + c.g) * p.tiles + c.tile; }
  // The next piece with blocks; false: the range has no more. `write`: this thread notes the items that start in the range.
  __device__ __forceinline__ bool next(const TreeParams& p, const TreeRange& r, TreePiece& c, bool write) {
    while (at < r.end) {
      c.sq = tree_seq(p, b);
      if (at >= seq_at + c.sq.weight) { seq_at += c.sq.weight; b++; continue; }
      const int len = c.sq.blocks + TREE_SEG_COST;
      const int k = (int)((at - seq_at) / len);  // item of the sequence
      const long long item_at = seq_at + (long long)k * len;
      const int off = (int)(at - item_at), take = (int)min((long long)(len - off), r.end - at);
      c.b = b;
      c.g = k / c.sq.tiles;
      c.tile = k - c.g * c.sq.tiles;
      c.lo = max(off - TREE_SEG_COST, 0);
      c.hi = max(off + take - TREE_SEG_COST, 0);
      at += take;
      if (off == 0 && write) {
        int2 info = make_int2(0, 0);
        if (c.sq.blocks) {
          info.x = tree_cta_of(item_at + TREE_SEG_COST, r.total, r.ctas);
          info.y = tree_cta_of(item_at + len - 1, r.total, r.ctas) - info.x + 1;
        }
        p.item_info[item(p, c)] = info;
      }
      if (c.lo < c.hi) return true;
    }
    return false;
  }
};

// Bounded wait of a converged warp. A wait that gives up is noted in `failed`, and from then on no wait of the CTA lasts: every thread
// goes on through the same loops and barriers over whatever is there, so that the CTA ends together.
__device__ __forceinline__ void tree_wait(uint64_t* bar, uint32_t parity, uint32_t* failed) {
  for (uint32_t i = 0; !mbar_try_wait(bar, parity); i++)
    if (*(volatile uint32_t*)failed || i >= DEC_WAIT_LIMIT) { *(volatile uint32_t*)failed = 1; break; }
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
__device__ __forceinline__ void tree_st8(uint32_t taddr, const float (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])),
               "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])),
               "r"(__float_as_uint(v[7])) : "memory");
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

template <int D, int BITS, int N>
__global__ void __launch_bounds__(TREE_THREADS, (TreeLayout<D, BITS, N>::CTAS)) tree_kernel(const __grid_constant__ TreeParams p) {
  using L = TreeLayout<D, BITS, N>;
  constexpr int DJ = L::DJ, E = D / 32, NH = N / 2, NW = N / 8, NST = L::STAGES;
  extern __shared__ __align__(1024) uint8_t smem[];
  TreeShared<N>& s = *reinterpret_cast<TreeShared<N>*>(smem);
  uint8_t* const bp = smem + L::SHARED;
  uint8_t* const bq = bp + 2 * L::BP_TERM;
  uint8_t* const stages = bq + 2 * L::BQ_TERM;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);
  const bool control = warp == TREE_COMPUTE / 32;

  if (tid == 0) {
    for (int i = 0; i < NST; i++) mbar_init(&s.full[i], 1);
    mbar_init(&s.k_ready, 4);
    mbar_init(&s.s_done, 1);
    mbar_init(&s.p_ready, 8);
    mbar_init(&s.o_done, 1);
    mbar_init(&s.drain, 1);
    s.failed = 0;
    fence_mbar_init();
    fence_proxy_async();
  }
  if (control) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem)), "r"(L::COLS));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
  }
  grid_dependency_wait();
  tc_fence_before();
  const TreeRange range = tree_range<TREE_THREADS>(p, s.scratch);  // (its barriers also cover the set-up above)
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(FULL, s.tmem, 0);
  TreeWalk walk;
  walk.start(range);
  TreePiece c;
  uint32_t i = 0;  // blocks of the CTA so far

  if (control) {
    // ---- loads and products
    TreeWalk ahead;
    ahead.start(range);
    TreePiece a;
    bool more = ahead.next(p, range, a, false);
    int av = more ? a.lo : 0;
    uint32_t loads = 0;
    const uint32_t sc_bytes = p.scale_f16 ? 256u : 512u;
    const size_t sc_size = p.scale_f16 ? 2 : 4;
    auto load_next = [&]() {
      if (!more || tree_failed(&s.failed)) return;
      const int st = loads % NST;
      const size_t row0 = cache_row(p.pm, a.b, a.g, (long long)a.sq.block(av) * 128, lane == 0 ? p.status : nullptr);
      if (elect_one()) {
        uint8_t* const dst = stages + st * L::STAGE_BYTES;
        mbar_expect_tx(&s.full[st], 2 * L::TILE_BYTES + 2 * sc_bytes);
        bulk_g2s(dst, p.k_codes + row0 * L::P, L::TILE_BYTES, &s.full[st]);
        bulk_g2s(dst + 2 * L::TILE_BYTES, reinterpret_cast<const uint8_t*>(p.k_scales) + row0 * sc_size, sc_bytes, &s.full[st]);
        bulk_g2s(dst + L::TILE_BYTES, p.v_codes + row0 * L::P, L::TILE_BYTES, &s.full[st]);
        bulk_g2s(dst + 2 * L::TILE_BYTES + 512, reinterpret_cast<const uint8_t*>(p.v_scales) + row0 * sc_size, sc_bytes, &s.full[st]);
      }
      __syncwarp();
      loads++;
      if (++av == a.hi) {
        more = ahead.next(p, range, a, false);
        av = a.lo;
      }
    };
    for (int st = 0; st < NST; st++) load_next();
    const uint64_t desc_q = smem_desc_mn(smem_u32(bq), L::BQ_LBO, 128), desc_p = smem_desc_mn(smem_u32(bp), L::BP_LBO, L::BP_SBO);
    while (walk.next(p, range, c, false)) {
      for (int v = c.lo; v < c.hi; v++, i++) {
        tree_wait(&s.k_ready, i & 1, &s.failed);
        tc_fence_after();
        if (!tree_failed(&s.failed) && elect_one()) {
#pragma unroll
          for (int t = 0; t < 2; t++)
#pragma unroll
            for (int k = 0; k < D / 16; k++)
              tc_mma_f16(tmem + L::S_COL, tmem + L::K_COL + 8 * k, desc_q + ((t * L::BQ_TERM + 2 * k * L::BQ_LBO) >> 4), L::IDESC_Q, t || k);
          tc_commit(&s.s_done);
        }
        __syncwarp();
        tree_wait(&s.p_ready, i & 1, &s.failed);
        tc_fence_after();
        if (!tree_failed(&s.failed) && elect_one()) {
#pragma unroll
          for (int j = 0; j < DJ; j++)
#pragma unroll
            for (int t = 0; t < 2; t++)
#pragma unroll
              for (int k = 0; k < 8; k++)
                tc_mma_f16(tmem + L::O_COL + j * N, tmem + L::V_COL + 64 * j + 8 * k, desc_p + ((t * L::BP_TERM + 2 * k * L::BP_LBO) >> 4), L::IDESC_P,
                           v > c.lo || t || k);
          tc_commit(&s.o_done);
        }
        __syncwarp();
        load_next();
      }
    }
    // every copy that was asked for has landed (where no wait gave up: at once)
    for (uint32_t n = loads > NST ? loads - NST : 0; n < loads; n++) mbar_wait_bounded(&s.full[n % NST], (n / NST) & 1, DEC_WAIT_LIMIT);
  } else {
    const int wg = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's quarter of the tensor-memory lanes
    const uint32_t s_col = tmem + lanes + L::S_COL + wg * NH, o_col = tmem + lanes + L::O_COL + wg * NH;
    uint8_t* const bp_row = bp + wg * (NH / 8) * L::BP_SBO + (r & 7) * 16 + (r >> 3) * L::BP_LBO;
    while (walk.next(p, range, c, tid == 0)) {
      // ---- the piece's queries: q~ = R q as two binary16 terms, one power of two for all of the tile. |q~_i| <= sqrt(d) max |q|.
      const int q0 = c.tile * N, nq = min(N, c.sq.tokens * p.group - q0), t0 = q0 / p.group;
      cta_bar_sync_n(1, TREE_COMPUTE);  // the last piece's references have been read
      uint32_t raw[NW][E / 2];
      float qmax = 0.f;
#pragma unroll
      for (int k = 0; k < NW; k++) {
        const int n = warp * NW + k;
        if (n < nq) {
          const int t = (q0 + n) / p.group, h = c.g * p.group + (q0 + n) - t * p.group;
          const __half* q = p.q + c.b * p.qs_b + t * p.qs_t + h * p.qs_h + lane * E;
          if constexpr (E == 4) {
            const uint2 x = *reinterpret_cast<const uint2*>(q);
            raw[k][0] = x.x; raw[k][1] = x.y;
          } else {
            const uint4 x = *reinterpret_cast<const uint4*>(q);
            raw[k][0] = x.x; raw[k][1] = x.y; raw[k][E / 2 - 2] = x.z; raw[k][E / 2 - 1] = x.w;
          }
        } else {
#pragma unroll
          for (int e = 0; e < E / 2; e++) raw[k][e] = 0u;
        }
      }
#pragma unroll
      for (int k = 0; k < NW; k++)
#pragma unroll
        for (int e = 0; e < E / 2; e++) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&raw[k][e]));
          qmax = fmaxf(qmax, fminf(fmaxf(fabsf(f.x), fabsf(f.y)), 65504.f));  // (an infinite query is its own affair)
        }
      qmax = warp_max(qmax);
      if (lane == 0) s.warp_q[warp] = qmax;
      if (tid == 0) s.masks.from_max = 0;
      cta_bar_sync_n(1, TREE_COMPUTE);
#pragma unroll
      for (int k = 0; k < 8; k++) qmax = fmaxf(qmax, s.warp_q[k]);
      // the power of two that brings sqrt(d) max |q| to at most 2^13
      const int e2 = qmax > 0.f ? (int)(__float_as_uint(qmax) >> 23) - 126 + 4 : 13;  // (sqrt(d) <= 2^4)
      const float q_scale = __uint_as_float((uint32_t)(127 + 13 - e2) << 23), score_unit = p.score_unit * __uint_as_float((uint32_t)(127 - 13 + e2) << 23);
      tree_masks(p, s.masks, c.b, c.sq, t0, (q0 + nq - 1) / p.group - t0 + 1, tid, TREE_COMPUTE);
      if (tid < N) {
        s.neg_ref[tid] = 1e30f;
        s.token[tid] = (q0 + tid) / p.group - t0;
      }
      {
        QuatPairs<E> qp;
        qp.load(p.rot + (size_t)c.g * (D / 4) * 8, lane);
#pragma unroll
        for (int k = 0; k < NW; k++) {
          const int n = warp * NW + k;
          float x[E];
#pragma unroll
          for (int e = 0; e < E / 2; e++) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&raw[k][e]));
            x[2 * e] = f.x; x[2 * e + 1] = f.y;
          }
          wht_warp<float, E>(x, lane);
          qp.template apply<false>(x);
          uint32_t hi[E / 2], lo[E / 2];
#pragma unroll
          for (int e = 0; e < E / 2; e++) {
            const float a0 = x[2 * e] * (rsqrtf((float)D) * q_scale), a1 = x[2 * e + 1] * (rsqrtf((float)D) * q_scale);
            hi[e] = pack_half2(a0, a1);
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi[e]));
            lo[e] = pack_half2(a0 - f.x, a1 - f.y);
          }
          uint8_t* const dst = bq + (n >> 3) * 128 + (n & 7) * 16 + (E == 4 ? (lane >> 1) * L::BQ_LBO + (lane & 1) * 8 : lane * L::BQ_LBO);
          if constexpr (E == 4) {
            *reinterpret_cast<uint2*>(dst) = make_uint2(hi[0], hi[1]);
            *reinterpret_cast<uint2*>(dst + L::BQ_TERM) = make_uint2(lo[0], lo[1]);
          } else {
            *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[E / 2 - 2], hi[E / 2 - 1]);
            *reinterpret_cast<uint4*>(dst + L::BQ_TERM) = make_uint4(lo[0], lo[1], lo[E / 2 - 2], lo[E / 2 - 1]);
          }
        }
      }
      fence_proxy_async();
      cta_bar_sync_n(1, TREE_COMPUTE);

      float l[NH];
#pragma unroll
      for (int n = 0; n < NH; n++) l[n] = 0.f;
      float v_ref = 0.f;  // a power of two at least as large as every V scale so far
      for (int v = c.lo; v < c.hi; v++, i++) {
        const uint8_t* const st = stages + (i % NST) * L::STAGE_BYTES;
        tree_wait(&s.full[i % NST], (i / NST) & 1, &s.failed);
        if (wg == 0) {
#pragma unroll
          for (int j = 0; j < DJ; j++)
            tree_dequant<BITS>(st + r * L::P + j * (16 * BITS), p.lut_lo, p.lut_hi, p.lookup, tmem + lanes + L::K_COL + 64 * j);
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&s.k_ready);
        } else {
          if (i > 0) tree_wait(&s.o_done, (i - 1) & 1, &s.failed);
          tc_fence_after();
#pragma unroll
          for (int j = 0; j < DJ; j++)
            tree_dequant<BITS>(st + L::TILE_BYTES + (r + 128 * j) * (16 * BITS), p.lut_v_lo, p.lut_v_hi, p.lookup, tmem + lanes + L::V_COL + 64 * j);
          tc_wait_st();
        }
        const float ks = load_scale(st + 2 * L::TILE_BYTES, r, p.scale_f16) * score_unit;
        float vs = load_scale(st + 2 * L::TILE_BYTES + 512, r, p.scale_f16);
        const int row0 = c.sq.block(v) * 128, row = row0 + r;
        const bool masked = row0 + 128 > c.sq.ctx || !(row0 >= s.masks.from_max || row0 + 128 <= p.sinks);
        tree_wait(&s.s_done, i & 1, &s.failed);
        tc_fence_after();

        // scores relative to the references; -inf where the token does not see the row
        float t[NH];
        auto scores = [&]() {
          tree_ld<NH>(s_col, t);
          const float4* ref = reinterpret_cast<const float4*>(s.neg_ref + wg * NH);
#pragma unroll
          for (int n = 0; n < NH; n += 4) {
            const float4 f = ref[n / 4];
            t[n] = fmaf(t[n], ks, f.x);
            t[n + 1] = fmaf(t[n + 1], ks, f.y);
            t[n + 2] = fmaf(t[n + 2], ks, f.z);
            t[n + 3] = fmaf(t[n + 3], ks, f.w);
          }
        };
        uint32_t sees = 0xFFFFFFFFu;  // bit n: column n of this thread sees the row
        scores();
        if (masked) {
          sees = 0;
#pragma unroll
          for (int n = 0; n < NH; n++)
            if (wg * NH + n < nq && tree_sees(s.masks, s.token[wg * NH + n], row, c.sq.ctx, c.sq.rows, p.sinks)) sees |= 1u << n;
#pragma unroll
          for (int n = 0; n < NH; n++)
            if (!(sees >> n & 1u)) t[n] = -INFINITY;
          if (!sees) vs = 0.f;
        }
        float top = t[0];
#pragma unroll
        for (int n = 1; n + 1 < NH; n += 2) top = max3f(top, t[n], t[n + 1]);
        top = fmaxf(top, t[NH - 1]);
        const float vs_fin = vs < INFINITY ? vs : 0.f;  // (an infinite or undefined scale is its own row's affair)
        if (cta_bar_or_n(1, TREE_COMPUTE, top > TREE_RAISE || vs_fin > v_ref)) {
          // ---- new references: the maximum of each column over the block, and of the V scales
          const float vm = warp_max(vs_fin);
          if (lane == 0) s.warp_v[warp] = vm;
#pragma unroll
          for (int n0 = 0; n0 < NH; n0 += 8) {
            float z[8];
            tree_ld<8>(s_col + n0, z);
#pragma unroll
            for (int n = 0; n < 8; n++) {
              const float m = warp_max((sees >> (n0 + n) & 1u) ? z[n] * ks : -3e38f);
              if (lane == 0) s.warp_max[warp & 3][wg * NH + n0 + n] = m;
            }
          }
          cta_bar_sync_n(1, TREE_COMPUTE);
          float v_new = v_ref;
#pragma unroll
          for (int k = 0; k < 8; k++) v_new = fmaxf(v_new, s.warp_v[k]);
          // the power of two at or above it, not below 2^-100
          v_new = v_new > v_ref ? fmaxf(__uint_as_float((__float_as_uint(v_new) + 0x7FFFFFu) & 0x7F800000u), 7.888609e-31f) : v_ref;
          if (!(v_new < INFINITY)) v_new = 1.7014118e38f;  // 2^127
          if (tid < N) {
            const float m = fmaxf(fmaxf(s.warp_max[0][tid], s.warp_max[1][tid]), fmaxf(s.warp_max[2][tid], s.warp_max[3][tid]));
            const float old = -s.neg_ref[tid];
            const float ref = m > -2e38f ? fmaxf(old, m + TREE_HEADROOM) : old;
            const float f = ex2f(old - ref);
            s.neg_ref[tid] = -ref;
            s.l_factor[tid] = f;
            s.o_factor[tid] = v_new > 0.f ? f * (v_ref / v_new) : f;
          }
          cta_bar_sync_n(1, TREE_COMPUTE);
          v_ref = v_new;
#pragma unroll
          for (int n = 0; n < NH; n++) l[n] *= s.l_factor[wg * NH + n];
          if (v > c.lo) {
            tree_wait(&s.o_done, (i - 1) & 1, &s.failed);
            tc_fence_after();
#pragma unroll 1
            for (int j = 0; j < DJ; j++)
#pragma unroll 1
              for (int n0 = 0; n0 < NH; n0 += 8) {
                float o[8];
                tree_ld<8>(o_col + j * N + n0, o);
#pragma unroll
                for (int n = 0; n < 8; n++) o[n] *= s.o_factor[wg * NH + n0 + n];
                tree_st8(o_col + j * N + n0, o);
              }
            tc_wait_st();
          }
          scores();
#pragma unroll
          for (int n = 0; n < NH; n++)
            if (!(sees >> n & 1u)) t[n] = -INFINITY;
        }
        // ---- probabilities, and times the V scale as two binary16 terms of the operand B_P
        if (wg == 0 && i > 0) tree_wait(&s.o_done, (i - 1) & 1, &s.failed);
        const float vn = v_ref > 0.f ? vs * (TREE_P_UNIT / v_ref) : 0.f;
#pragma unroll
        for (int n0 = 0; n0 < NH; n0 += 8) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int k = 0; k < 4; k++) {
            const int n = n0 + 2 * k;
            const float p0 = ex2f(t[n]), p1 = ex2f(t[n + 1]);
            l[n] += p0;
            l[n + 1] += p1;
            float x0 = p0 * vn, x1 = p1 * vn;
            if (masked) {  // (0 times an infinite scale)
              if (!(sees >> n & 1u)) x0 = 0.f;
              if (!(sees >> (n + 1) & 1u)) x1 = 0.f;
            }
            hi[k] = pack_half2(x0, x1);
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi[k]));
            lo[k] = pack_half2(x0 - f.x, x1 - f.y);
          }
          uint8_t* const dst = bp_row + (n0 / 8) * L::BP_SBO;
          *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(dst + L::BP_TERM) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        fence_proxy_async();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.p_ready);
      }
      // ---- the piece's partial
      const size_t part = (walk.item(p, c) + blockIdx.x) * N;
      // sums over the rows: lane by lane in the warp, then over its four warps, in a fixed order
#pragma unroll
      for (int n = 0; n < NH; n++) {
        float x = l[n];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(FULL, x, o);
        if (lane == 0) s.warp_max[warp & 3][wg * NH + n] = x;
      }
      cta_bar_sync_n(1, TREE_COMPUTE);
      if (tid < nq) {
        const float sum = (s.warp_max[0][tid] + s.warp_max[1][tid]) + (s.warp_max[2][tid] + s.warp_max[3][tid]);
        *reinterpret_cast<float2*>(p.part_ml + 2 * (part + tid)) = make_float2(-s.neg_ref[tid], sum);
      }
      const float unit = p.value_unit * (v_ref / TREE_P_UNIT);
      tree_wait(&s.o_done, (i - 1) & 1, &s.failed);
      tc_fence_after();
#pragma unroll 1
      for (int j = 0; j < DJ; j++)
#pragma unroll 1
        for (int n0 = 0; n0 < NH; n0 += 8) {
          if (wg * NH + n0 >= nq) break;
          float o[8];
          tree_ld<8>(o_col + j * N + n0, o);
          float* const dst = p.part_acc + (part + wg * NH + n0) * D + 128 * j + r;
#pragma unroll
          for (int n = 0; n < 8; n++)
            if (wg * NH + n0 + n < nq) dst[n * D] = o[n] * unit;
        }
      tc_fence_before();
    }
  }

  allow_dependent_launch();
  __syncthreads();
  if (*(volatile uint32_t*)&s.failed) {  // (nobody writes it any more)
    if (tid == 0 && p.status) atomicOr(&p.status[0], IQ_STATUS_WAIT_TIMEOUT);
    if (control) {  // MMAs may still be running: they are waited for, with a limit, before the tensor memory goes
      if (elect_one()) tc_commit(&s.drain);
      __syncwarp();
      mbar_wait_bounded(&s.drain, 0u, DEC_WAIT_LIMIT);
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (control) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L::COLS));
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
  return launch_after_predecessor(kern, dim3(p.ctas), dim3(TREE_THREADS), L::SMEM, stream, p);
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
