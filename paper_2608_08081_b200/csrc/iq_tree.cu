// Attention for drafted tokens over the packed cache: the kernel over the blocks of all sequences, and the merge of its partials with
// the inverse rotation.
#include "iq_common.cuh"
#include "iq_decode_common.cuh"
#include "iq_format.cuh"
#include "iq_tree_common.cuh"

namespace iq {
namespace {

constexpr int TREE_THREADS = 256;
constexpr int TREE_TILE = 16;

template <int D>
struct TreeSmem {
  float q[TREE_TILE][D];
  float kv[128][D + 1];
  float pr[TREE_TILE][128];
  float m[TREE_TILE], l[TREE_TILE], alpha[TREE_TILE];
  TreeMasks<TREE_TILE> masks;
  long long scratch[TREE_THREADS / 32 + 4];
};

template <int BITS>
__device__ __forceinline__ float level_of(const uint32_t (&lo)[4], const uint32_t (&hi)[4], int code) {
  const uint32_t l = (lo[code >> 2] >> (8 * (code & 3))) & 0xFFu, h = (hi[code >> 2] >> (8 * (code & 3))) & 0xFFu;
  return __half2float(__ushort_as_half((unsigned short)(l | (h << 8))));
}

template <int D, int BITS>
__global__ void __launch_bounds__(TREE_THREADS) tree_kernel(const __grid_constant__ TreeParams p) {
  constexpr int N = TREE_TILE, E = D / 32, P = PackedFormat<BITS>::row_bytes(D);
  extern __shared__ __align__(16) uint8_t smem[];
  TreeSmem<D>& s = *reinterpret_cast<TreeSmem<D>*>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  grid_dependency_wait();
  const TreeRange range = tree_range<TREE_THREADS>(p, s.scratch);
  if (range.at >= range.end) return;
  int b = range.b;
  long long seq_at = range.seq_at, at = range.at;
  while (at < range.end) {
    const TreeSeq sq = tree_seq(p, b);
    const int len = sq.blocks + TREE_SEG_COST;
    const int k = sq.weight ? (int)((at - seq_at) / len) : 0;  // item of the sequence
    if (at >= seq_at + sq.weight) { seq_at += sq.weight; b++; continue; }
    const int g = k / sq.tiles, tile = k - g * sq.tiles;
    const long long item_at = seq_at + (long long)k * len;
    const int off = (int)(at - item_at), take = (int)min((long long)(len - off), range.end - at);
    const int lo = max(off - TREE_SEG_COST, 0), hi = max(off + take - TREE_SEG_COST, 0);
    const size_t item = ((size_t)b * p.n_kv_heads + g) * p.tiles + tile;
    if (off == 0 && tid == 0) {
      int2 info = make_int2(0, 0);
      if (sq.blocks) {
        info.x = tree_cta_of(item_at + TREE_SEG_COST, range.total, range.ctas);
        info.y = tree_cta_of(item_at + len - 1, range.total, range.ctas) - info.x + 1;
      }
      p.item_info[item] = info;
    }
    at += take;
    if (lo >= hi) continue;
    // ---- the piece: blocks [lo, hi) of the item
    const int q0 = tile * N, nq = min(N, sq.tokens * p.group - q0), t0 = q0 / p.group, nt = (q0 + nq - 1) / p.group - t0 + 1;
    __syncthreads();
    if (tid == 0) s.masks.from_max = 0;
    __syncthreads();
    tree_masks(p, s.masks, b, sq, t0, nt, tid, TREE_THREADS);
    for (int n = warp; n < N; n += TREE_THREADS / 32) {
      float v[E];
#pragma unroll
      for (int e = 0; e < E; e++) v[e] = 0.f;
      if (n < nq) {
        const int t = (q0 + n) / p.group, h = g * p.group + (q0 + n) % p.group;
        const __half* q = p.q + b * p.qs_b + t * p.qs_t + h * p.qs_h + lane * E;
#pragma unroll
        for (int e = 0; e < E; e++) v[e] = __half2float(q[e]);
        QuatPairs<E> qp;
        qp.load(p.rot + (size_t)g * (D / 4) * 8, lane);
        wht_warp<float, E>(v, lane);
        qp.template apply<false>(v);
      }
#pragma unroll
      for (int e = 0; e < E; e++) s.q[n][lane * E + e] = v[e] * rsqrtf((float)D) * p.score_unit;
      if (lane == 0) { s.m[n] = -1e30f; s.l[n] = 0.f; }
    }
    const int c = tid % D, half = tid / D;  // value pass: coordinate, first of the queries
    constexpr int NV = N * D / TREE_THREADS;
    float acc[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) acc[i] = 0.f;
    for (int v = lo; v < hi; v++) {
      const int blk = sq.block(v);
      const size_t row0 = cache_row(p.pm, b, g, (long long)blk * 128, p.status);
      __syncthreads();
      {
        const int r = tid & 127, h2 = tid >> 7;
        const uint32_t* w = reinterpret_cast<const uint32_t*>(p.k_codes + (row0 + r) * P);
        for (int i = h2 * (D / 2); i < (h2 + 1) * (D / 2); i++) s.kv[r][i] = level_of<BITS>(p.lut_lo, p.lut_hi, packed_code<BITS>(w, i));
      }
      __syncthreads();
      {
        const int r = tid & 127, n0 = (tid >> 7) * (N / 2), row = blk * 128 + r;
        const float ks = load_scale(p.k_scales, row0 + r, p.scale_f16);
        float z[N / 2];
#pragma unroll
        for (int n = 0; n < N / 2; n++) z[n] = 0.f;
        for (int i = 0; i < D; i++)
#pragma unroll
          for (int n = 0; n < N / 2; n++) z[n] = fmaf(s.q[n0 + n][i], s.kv[r][i], z[n]);
#pragma unroll
        for (int n = 0; n < N / 2; n++) {
          bool see = n0 + n < nq;
          if (see) see = tree_sees(s.masks, (q0 + n0 + n) / p.group - t0, row, sq.ctx, sq.rows, p.sinks);
          s.pr[n0 + n][r] = see ? z[n] * ks : -INFINITY;
        }
      }
      __syncthreads();
      for (int n = warp * (N / 8); n < (warp + 1) * (N / 8); n++) {
        float z[4], mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; i++) { z[i] = s.pr[n][lane + 32 * i]; mx = fmaxf(mx, z[i]); }
        mx = fmaxf(warp_max(mx), s.m[n]);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const bool see = z[i] != -INFINITY;
          const float e = see ? ex2f(z[i] - mx) : 0.f;
          sum += e;
          s.pr[n][lane + 32 * i] = see ? e * load_scale(p.v_scales, row0 + lane + 32 * i, p.scale_f16) : 0.f;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
        if (lane == 0) {
          s.alpha[n] = ex2f(s.m[n] - mx);
          s.l[n] = s.l[n] * s.alpha[n] + sum;
          s.m[n] = mx;
        }
      }
      for (int i = tid; i < D; i += TREE_THREADS) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(p.v_codes + row0 * P + (size_t)i * 16 * BITS);
        for (int r = 0; r < 128; r++) s.kv[r][i] = level_of<BITS>(p.lut_v_lo, p.lut_v_hi, packed_code<BITS>(w, r));
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; i++) acc[i] *= s.alpha[half * NV + i];
      for (int r = 0; r < 128; r++) {
        const float x = s.kv[r][c];
#pragma unroll
        for (int i = 0; i < NV; i++) acc[i] = fmaf(s.pr[half * NV + i][r], x, acc[i]);
      }
    }
    const size_t part = (item + blockIdx.x) * N;
#pragma unroll
    for (int i = 0; i < NV; i++) p.part_acc[(part + half * NV + i) * D + c] = acc[i] * p.value_unit;
    if (tid < N) {
      p.part_ml[2 * (part + tid)] = s.m[tid];
      p.part_ml[2 * (part + tid) + 1] = s.l[tid];
    }
  }
}

constexpr int MERGE_WARPS = 4;
// A warp to a (sequence, token, query head): its item's partials, one per CTA that had blocks of the item, then o = R^T o~.
template <int D>
__global__ void __launch_bounds__(MERGE_WARPS * 32) tree_merge_kernel(const __grid_constant__ TreeParams p) {
  constexpr int E = D / 32;
  grid_dependency_wait();
  allow_dependent_launch();
  const int lane = threadIdx.x & 31;
  const long long i = (long long)blockIdx.x * MERGE_WARPS + (threadIdx.x >> 5);
  const int h = (int)(i % p.n_q_heads);
  const long long bt = i / p.n_q_heads;
  const int t = (int)(bt % p.n_tokens_max);
  const int b = (int)(bt / p.n_tokens_max);
  if (b >= p.batch) return;
  if (p.n_tokens && t >= p.n_tokens[b]) return;
  const int g = h / p.group, n = t * p.group + h % p.group, tile = n / p.tile;
  const size_t item = ((size_t)b * p.n_kv_heads + g) * p.tiles + tile;
  QuatPairs<E> qp;
  qp.load(p.rot + (size_t)g * (D / 4) * 8, lane);
  const int2 info = p.item_info[item];
  const size_t first = (item + info.x) * p.tile + (n - tile * p.tile);
  float m = -INFINITY, l = 0.f, v[E];
#pragma unroll
  for (int e = 0; e < E; e++) v[e] = 0.f;
  for (int k = 0; k < info.y; k++) {
    const size_t o = first + (size_t)k * p.tile;
    const float mk = p.part_ml[2 * o], lk = p.part_ml[2 * o + 1];
    if (lk == 0.f) continue;
    const float mn = fmaxf(m, mk), wa = ex2f(m - mn), wk = ex2f(mk - mn);
#pragma unroll
    for (int e4 = 0; e4 < E / 4; e4++) {
      const float4 f = *reinterpret_cast<const float4*>(p.part_acc + o * D + lane * E + 4 * e4);
      v[4 * e4] = fmaf(wk, f.x, wa * v[4 * e4]);
      v[4 * e4 + 1] = fmaf(wk, f.y, wa * v[4 * e4 + 1]);
      v[4 * e4 + 2] = fmaf(wk, f.z, wa * v[4 * e4 + 2]);
      v[4 * e4 + 3] = fmaf(wk, f.w, wa * v[4 * e4 + 3]);
    }
    l = fmaf(lk, wk, wa * l);
    m = mn;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; e++) v[e] *= inv;
  qp.template apply<true>(v);
  wht_warp<float, E>(v, lane);
  const size_t o = ((size_t)b * p.n_tokens_max + t) * p.n_q_heads + h;
#pragma unroll
  for (int e = 0; e < E; e++) v[e] *= rsqrtf((float)D);
  if (p.out_is_fp16) {
    uint32_t* out = reinterpret_cast<uint32_t*>(reinterpret_cast<__half*>(p.out) + o * D + lane * E);
#pragma unroll
    for (int e = 0; e < E / 2; e++) out[e] = pack_half2(v[2 * e], v[2 * e + 1]);
  } else {
    float4* out = reinterpret_cast<float4*>(reinterpret_cast<float*>(p.out) + o * D + lane * E);
#pragma unroll
    for (int e = 0; e < E / 4; e++) out[e] = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
  }
  if (p.lse && lane == 0) p.lse[o] = l == 0.f ? -INFINITY : fmaf(m, 0.6931471805599453f, logf(l));
}

template <int D, int BITS>
cudaError_t launch(const TreeParams& p, cudaStream_t stream) {
  const size_t smem = sizeof(TreeSmem<D>);
  cudaError_t e = cudaFuncSetAttribute(tree_kernel<D, BITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_after_predecessor(tree_kernel<D, BITS>, dim3(p.ctas), dim3(TREE_THREADS), smem, stream, p);
}

}  // namespace

int tree_tile(int head_dim, int queries) { return TREE_TILE; }
int tree_ctas_per_sm(int head_dim, int tile) { return head_dim == 128 ? 2 : 1; }

cudaError_t launch_tree_attention(const TreeParams& p, int head_dim, cudaStream_t stream) {
  cudaError_t e;
  if (head_dim == 128) e = p.bits == 2 ? launch<128, 2>(p, stream) : p.bits == 3 ? launch<128, 3>(p, stream) : launch<128, 4>(p, stream);
  else e = p.bits == 2 ? launch<256, 2>(p, stream) : p.bits == 3 ? launch<256, 3>(p, stream) : launch<256, 4>(p, stream);
  if (e != cudaSuccess) return e;
  const long long heads = (long long)p.batch * p.n_tokens_max * p.n_q_heads;
  const dim3 grid((unsigned)((heads + MERGE_WARPS - 1) / MERGE_WARPS));
  return head_dim == 128 ? launch_after_predecessor(tree_merge_kernel<128>, grid, dim3(MERGE_WARPS * 32), 0, stream, p)
                         : launch_after_predecessor(tree_merge_kernel<256>, grid, dim3(MERGE_WARPS * 32), 0, stream, p);
}

}  // namespace iq
