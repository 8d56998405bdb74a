// Attention for drafted tokens over the packed cache: the kernel over the blocks of all sequences, and the merge of its partials with
// the inverse rotation.
#include "iq_tree_kernel.cuh"

namespace iq {
namespace {

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
  long long tok0;
  if (t >= tree_tokens(p, b, tok0)) return;
  const int g = h / p.group, n = t * p.group + h % p.group, tile = n / p.tile;
  const size_t item = ((size_t)b * p.n_kv_heads + g) * p.tiles + tile;
  QuatPairs<E> qp;
  qp.load(p.rot + (size_t)g * (D / 4) * 8, lane);
  const int2 info = p.item_info[item];
  const size_t first = (item + info.x) * p.tile + (n - tile * p.tile);
  // 32 partials at a time: a lane takes the (m, l) of one, the reference and the weights come from warp reductions, and their rows are
  // loaded eight at a time, whatever the weights (one after the other each costs a trip to memory: a window of 33 blocks over 17 CTAs 20.3 us, so 16.9)
  float m = -INFINITY, l = 0.f, v[E];
#pragma unroll
  for (int e = 0; e < E; e++) v[e] = 0.f;
  for (int k0 = 0; k0 < info.y; k0 += 32) {
    const int cnt = min(32, info.y - k0);
    const size_t row0 = first + (size_t)k0 * p.tile;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < cnt) ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * (row0 + (size_t)lane * p.tile));
    constexpr int NF = 8;
    float4 f[NF][E / 4];
    auto request = [&](int k) {
#pragma unroll
      for (int x = 0; x < NF; x++) {
        const float* a = p.part_acc + (row0 + (size_t)min(k + x, cnt - 1) * p.tile) * D + lane * E;
#pragma unroll
        for (int e4 = 0; e4 < E / 4; e4++) f[x][e4] = *reinterpret_cast<const float4*>(a + 4 * e4);
      }
    };
    request(0);
    if (ml.y == 0.f) ml.x = -INFINITY;  // nothing seen (undefined sums count)
    const float top = fmaxf(m, warp_max(ml.x));
    const float w = ml.y == 0.f ? 0.f : ex2f(ml.x - top), before = l == 0.f ? 0.f : ex2f(m - top);
    float sum = ml.y * w;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
    l = fmaf(l, before, sum);
    m = top;
#pragma unroll
    for (int e = 0; e < E; e++) v[e] *= before;
    for (int k = 0; k < cnt; k += NF) {
      if (k) request(k);
#pragma unroll
      for (int x = 0; x < NF; x++) {
        const float wk = __shfl_sync(FULL, w, (k + x) & 31);
        if (k + x >= cnt || wk == 0.f) continue;
#pragma unroll
        for (int e4 = 0; e4 < E / 4; e4++) {
          v[4 * e4] = fmaf(wk, f[x][e4].x, v[4 * e4]);
          v[4 * e4 + 1] = fmaf(wk, f[x][e4].y, v[4 * e4 + 1]);
          v[4 * e4 + 2] = fmaf(wk, f[x][e4].z, v[4 * e4 + 2]);
          v[4 * e4 + 3] = fmaf(wk, f[x][e4].w, v[4 * e4 + 3]);
        }
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; e++) v[e] *= inv;
  qp.template apply<true>(v);
  wht_warp<float, E>(v, lane);
  const size_t o = ((size_t)tok0 + t) * p.n_q_heads + h;
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

}  // namespace

// The smallest tile that takes all pairs, up to 64: every item reads and dequantises its blocks, so more pairs to an item are worth the
// columns that stay empty (16 sequences of 16 K rows, 8 KV heads: 16 columns 105 us, 32 132, not 210, 64 181, not 264; a sequence of 32 K
// rows with 240 pairs as four items of 64 96 us).
int tree_tile(int queries) { return queries <= 16 ? 16 : queries <= 32 ? 32 : 64; }

cudaError_t launch_tree_attention(const TreeParams& p, int head_dim, cudaStream_t stream) {
  const cudaError_t e = p.bits == 2 ? launch_tree_b2(p, head_dim, stream) : p.bits == 3 ? launch_tree_b3(p, head_dim, stream) : launch_tree_b4(p, head_dim, stream);
  if (e != cudaSuccess) return e;
  const long long heads = (long long)p.batch * p.n_tokens_max * p.n_q_heads;
  const dim3 grid((unsigned)((heads + MERGE_WARPS - 1) / MERGE_WARPS));
  return head_dim == 128 ? launch_after_predecessor(tree_merge_kernel<128>, grid, dim3(MERGE_WARPS * 32), 0, stream, p)
                         : launch_after_predecessor(tree_merge_kernel<256>, grid, dim3(MERGE_WARPS * 32), 0, stream, p);
}

}  // namespace iq
