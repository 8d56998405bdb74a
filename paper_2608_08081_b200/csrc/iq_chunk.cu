// Attention of any number of new tokens over the packed cache: the kernel over the blocks of all tiles, and the merge of the tiles that
// two or more pairs of CTAs share.
#include "iq_chunk_kernel.cuh"

namespace iq {
namespace {

constexpr int CHUNK_MERGE_WARPS = 4, CHUNK_MERGE_ROWS = 8;  // rows of a tile that a CTA merges
// CTA (c, y): rows 8 y ... of the tile that begins in the range of pair c of the launch and ends in a later one. A warp to a row at a time: the
// tile's partials, from consecutive pairs, then o = R^T o~.
template <int D>
__global__ void __launch_bounds__(CHUNK_MERGE_WARPS * 32) chunk_merge_kernel(const __grid_constant__ ChunkParams p) {
  constexpr int E = D / 32;
  grid_dependency_wait();
  allow_dependent_launch();
  const int pair = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long* const info = p.cut_info + CHUNK_INFO * pair;
  const int b = (int)info[0];
  if (b < 0) return;
  const int g = (int)(info[1] >> 32), t = (int)(info[1] & 0xFFFFFFFFu);
  const long long item_at = info[2], total = info[3];
  const ChunkSeq sq = chunk_seq(p, b);
  const ChunkTile x = chunk_tile(p, sq, t);
  const long long units = chunk_units(p, sq, t);
  const int pairs = (int)max(1ll, min((long long)p.pairs, total / p.least_units));
  const int last = (int)min((long long)pairs - 1, chunk_div((item_at + units) * pairs - 1, total));  // the pair that ends the tile
  // blocks of the tile before the range of pair k
  auto before = [&](int k) { return chunk_blocks_before(p, chunk_cut(total, k, pairs) - item_at, units, x.blocks); };
  if (x.blocks == 0) return;
  {  // one of the pairs may have had all blocks, and written the outputs
    bool all = false;
    for (int k = pair + lane; k <= last; k += 32) all |= (k == pair ? 0 : before(k)) == 0 && (k == last ? x.blocks : before(k + 1)) == x.blocks;
    if (__any_sync(FULL, all)) return;
  }
  QuatPairs<E> qp;
  qp.load(p.rot + (size_t)g * (D / 4) * 8, lane);
  for (int row = blockIdx.y * CHUNK_MERGE_ROWS + warp; row < (blockIdx.y + 1) * CHUNK_MERGE_ROWS; row += CHUNK_MERGE_WARPS) {
    const int tok = (t * CHUNK_ROWS + row) / p.group, h = g * p.group + (t * CHUNK_ROWS + row) - tok * p.group;
    if (tok >= sq.n) return;
    float m = -INFINITY, l = 0.f, v[E];
#pragma unroll
    for (int e = 0; e < E; e++) v[e] = 0.f;
    for (int k0 = pair; k0 <= last; k0 += 32) {  // 32 partials at a time, their rows loaded eight at a time
      const int cnt = min(32, last + 1 - k0);
      const int k = k0 + lane;
      const bool mine = lane < cnt && (k == pair ? 0 : before(k)) < (k == last ? x.blocks : before(k + 1));  // (pairs without a block of the tile left nothing)
      const size_t slot_row = ((size_t)(2 * k + (k == pair ? 1 : 0))) * CHUNK_ROWS + row;
      float2 ml = make_float2(-INFINITY, 0.f);
      if (mine) ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * slot_row);
      if (ml.y == 0.f) ml.x = -INFINITY;  // nothing seen (undefined sums count)
      const float top = fmaxf(m, warp_max(ml.x));
      const float w = ml.y == 0.f ? 0.f : ex2f(ml.x - top), old = l == 0.f ? 0.f : ex2f(m - top);
      float sum = ml.y * w;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
      l = fmaf(l, old, sum);
      m = top;
#pragma unroll
      for (int e = 0; e < E; e++) v[e] *= old;
      constexpr int NF = 8;
      for (int i = 0; i < cnt; i += NF) {
        float4 f[NF][E / 4];
        float wi[NF];
#pragma unroll
        for (int y = 0; y < NF; y++) {
          wi[y] = __shfl_sync(FULL, w, (i + y) & 31);
          if (i + y >= cnt) wi[y] = 0.f;
          const int kk = k0 + i + y;
          const float* a = p.part_acc + ((size_t)(2 * kk + (kk == pair ? 1 : 0)) * CHUNK_ROWS + row) * D + lane * E;
          if (wi[y] != 0.f) {
#pragma unroll
            for (int e4 = 0; e4 < E / 4; e4++) f[y][e4] = *reinterpret_cast<const float4*>(a + 4 * e4);
          }
        }
#pragma unroll
        for (int y = 0; y < NF; y++) {
          if (wi[y] == 0.f) continue;
#pragma unroll
          for (int e4 = 0; e4 < E / 4; e4++) {
            v[4 * e4] = fmaf(wi[y], f[y][e4].x, v[4 * e4]);
            v[4 * e4 + 1] = fmaf(wi[y], f[y][e4].y, v[4 * e4 + 1]);
            v[4 * e4 + 2] = fmaf(wi[y], f[y][e4].z, v[4 * e4 + 2]);
            v[4 * e4 + 3] = fmaf(wi[y], f[y][e4].w, v[4 * e4 + 3]);
          }
        }
      }
    }
    const float unit = l == 0.f ? 0.f : rsqrtf((float)D) / l;
#pragma unroll
    for (int e = 0; e < E; e++) v[e] *= unit;
    qp.template apply<true>(v);
    wht_warp<float, E>(v, lane);
    const size_t o = ((size_t)sq.tok0 + tok) * p.n_q_heads + h;
    uint32_t* const out = reinterpret_cast<uint32_t*>(p.out + o * D + lane * E);
#pragma unroll
    for (int e = 0; e < E / 2; e++) out[e] = pack_half2(v[2 * e], v[2 * e + 1]);
    if (p.lse && lane == 0) p.lse[o] = l == 0.f ? -INFINITY : fmaf(m, 0.6931471805599453f, logf(l));
  }
}

}  // namespace

cudaError_t launch_chunk_attention(const ChunkParams& p, int head_dim, cudaStream_t stream) {
  const cudaError_t e = p.bits == 2 ? launch_chunk_b2(p, head_dim, stream) : p.bits == 3 ? launch_chunk_b3(p, head_dim, stream) : launch_chunk_b4(p, head_dim, stream);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)p.pairs, CHUNK_ROWS / CHUNK_MERGE_ROWS);
  return head_dim == 128 ? launch_after_predecessor(chunk_merge_kernel<128>, grid, dim3(CHUNK_MERGE_WARPS * 32), 0, stream, p)
                         : launch_after_predecessor(chunk_merge_kernel<256>, grid, dim3(CHUNK_MERGE_WARPS * 32), 0, stream, p);
}

}  // namespace iq
