// Attention of any number of new tokens over the packed cache: the kernel over the blocks of all tiles, and the merge of the tiles that
// two or more pairs of CTAs share.
#include "iq_chunk_kernel.cuh"

namespace iq {
namespace {

constexpr int CHUNK_MERGE_WARPS = 4;
// CTA (c, y): rows 4 y ... of the tile that begins in the range of pair c of the launch and ends in a later one, a warp to a row: the tile's
// partials, from consecutive pairs, then o = R^T o~. All that is read hangs on the pairs' notes alone, so it takes three trips to memory one after
// the other. (With the pieces worked out again from the lengths, two rows to a warp: 12 us for 8 tiles, 44 for 40 at head_dim 256; now 7 and 20.)
template <int D>
__global__ void __launch_bounds__(CHUNK_MERGE_WARPS * 32) chunk_merge_kernel(const __grid_constant__ ChunkParams p) {
  constexpr int E = D / 32, NF = 4;
  grid_dependency_wait();
  allow_dependent_launch();
  const int pair = blockIdx.x, lane = threadIdx.x & 31, row = blockIdx.y * CHUNK_MERGE_WARPS + (threadIdx.x >> 5);
  const ChunkCut cut = p.cuts[pair];
  if (cut.last < 0) return;
  const int tok = (cut.t * CHUNK_ROWS + row) / p.group, h = cut.g * p.group + (cut.t * CHUNK_ROWS + row) - tok * p.group;
  if (tok >= cut.n) return;
  QuatPairs<E> qp;
  qp.load(p.rot + (size_t)cut.g * (D / 4) * 8, lane);
  float m = -INFINITY, l = 0.f, v[E];
  bool any = false;
#pragma unroll
  for (int e = 0; e < E; e++) v[e] = 0.f;
  // partials of pairs k0 ..., 32 at a time, their rows requested NF at a time whether they are there or not (the workspace is)
  for (int k0 = pair; k0 <= cut.last; k0 += 32) {
    const int cnt = min(32, cut.last + 1 - k0), k = min(k0 + lane, cut.last);
    auto place = [&](int pr) { return (size_t)(2 * pr + (pr == pair ? 1 : 0)) * CHUNK_ROWS + row; };
    float4 f[NF][E / 4];
    auto request = [&](int i) {
#pragma unroll
      for (int y = 0; y < NF; y++) {
        const float* a = p.part_acc + place(k0 + min(i + y, cnt - 1)) * D + lane * E;
#pragma unroll
        for (int e4 = 0; e4 < E / 4; e4++) f[y][e4] = *reinterpret_cast<const float4*>(a + 4 * e4);
      }
    };
    request(0);
    const int partials = p.cuts[k].partials;
    float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * place(k));
    const bool there = lane < cnt && (partials & (k == pair ? 2 : 1));  // (a pair without a block of the tile left nothing)
    any |= __any_sync(FULL, there);
    if (!there || ml.y == 0.f) ml = make_float2(-INFINITY, 0.f);        // nothing seen (undefined sums count)
    const float top = fmaxf(m, warp_max(ml.x));
    const float w = ml.y == 0.f ? 0.f : ex2f(ml.x - top), old = l == 0.f ? 0.f : ex2f(m - top);
    float sum = ml.y * w;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
    l = fmaf(l, old, sum);
    m = top;
#pragma unroll
    for (int e = 0; e < E; e++) v[e] *= old;
    for (int i = 0; i < cnt; i += NF) {
      if (i) request(i);
#pragma unroll
      for (int y = 0; y < NF; y++) {
        const float wi = __shfl_sync(FULL, w, (i + y) & 31);
        if (i + y >= cnt || wi == 0.f) continue;
#pragma unroll
        for (int e4 = 0; e4 < E / 4; e4++) {
          v[4 * e4] = fmaf(wi, f[y][e4].x, v[4 * e4]);
          v[4 * e4 + 1] = fmaf(wi, f[y][e4].y, v[4 * e4 + 1]);
          v[4 * e4 + 2] = fmaf(wi, f[y][e4].z, v[4 * e4 + 2]);
          v[4 * e4 + 3] = fmaf(wi, f[y][e4].w, v[4 * e4 + 3]);
        }
      }
    }
  }
  if (!any) return;  // one pair had all blocks, and wrote the outputs
  const float unit = l == 0.f ? 0.f : rsqrtf((float)D) / l;
#pragma unroll
  for (int e = 0; e < E; e++) v[e] *= unit;
  qp.template apply<true>(v);
  wht_warp<float, E>(v, lane);
  const size_t o = ((size_t)cut.tok0 + tok) * p.n_q_heads + h;
  uint32_t* const out = reinterpret_cast<uint32_t*>(p.out + o * D + lane * E);
#pragma unroll
  for (int e = 0; e < E / 2; e++) out[e] = pack_half2(v[2 * e], v[2 * e + 1]);
  if (p.lse && lane == 0) p.lse[o] = l == 0.f ? -INFINITY : fmaf(m, 0.6931471805599453f, logf(l));
}

}  // namespace

cudaError_t launch_chunk_attention(const ChunkParams& p, int head_dim, cudaStream_t stream) {
  const cudaError_t e = p.bits == 2 ? launch_chunk_b2(p, head_dim, stream) : p.bits == 3 ? launch_chunk_b3(p, head_dim, stream) : launch_chunk_b4(p, head_dim, stream);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)p.pairs, CHUNK_ROWS / CHUNK_MERGE_WARPS);
  return head_dim == 128 ? launch_after_predecessor(chunk_merge_kernel<128>, grid, dim3(CHUNK_MERGE_WARPS * 32), 0, stream, p)
                         : launch_after_predecessor(chunk_merge_kernel<256>, grid, dim3(CHUNK_MERGE_WARPS * 32), 0, stream, p);
}

}  // namespace iq
