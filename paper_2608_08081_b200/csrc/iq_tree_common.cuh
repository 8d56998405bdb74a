// Tree attention: which rows a sequence's drafted tokens see, and how the launch's blocks are dealt out.
#pragma once
#include "iq_common.cuh"

namespace iq {

// One sequence of the launch. Its blocks of 128 rows are numbered without those that no token sees: the first `sink_blocks`, then
// those from the window on.
struct TreeSeq {
  int ctx, tokens, rows;   // context rows, drafted tokens, rows of the two inside the cache
  int blocks, sink_blocks, skipped;
  int tiles;               // items per KV head
  long long weight;        // blocks of all its items, each item counting TREE_SEG_COST more
  __device__ __forceinline__ int block(int v) const { return v < sink_blocks ? v : v + skipped; }
};
__device__ __forceinline__ TreeSeq tree_seq(const TreeParams& p, int b) {
  TreeSeq s;
  s.ctx = max(0, min(p.ctx_lens[b], p.t_cap));
  s.tokens = p.n_tokens ? max(0, min(p.n_tokens[b], p.n_tokens_max)) : p.n_tokens_max;
  s.rows = min(s.ctx + s.tokens, p.t_cap);  // (t_cap + IQ_TREE_MAX_TOKENS fits 31 bits: the host's limit)
  const int total = (s.rows + 127) >> 7;
  s.sink_blocks = total;
  s.skipped = 0;
  if (p.window > 0) {
    s.sink_blocks = min(total, (p.sinks >> 7) + ((p.sinks & 127) != 0));
    // a token's position is ctx - 1 at least (it sees no drafted token): what lies before that one's window is seen by none
    s.skipped = max(0, (max(0, s.ctx - p.window) >> 7) - s.sink_blocks);
  }
  s.blocks = total - s.skipped;
  s.tiles = (s.tokens * p.group + p.tile - 1) / p.tile;
  s.weight = (long long)p.n_kv_heads * s.tiles * (s.blocks + TREE_SEG_COST);
  return s;
}

// The launch's items (sequence, KV head, tile of (token, head) pairs) laid end to end, each as TREE_SEG_COST + its blocks units long,
// and cut into one range of equal length per CTA (of as many CTAs as there are units: no range is empty, so the partials of an item are
// those of consecutive CTAs).
struct TreeRange {
  long long at, end, total;  // units
  int ctas;                  // CTAs that have a range
  int b;                     // the sequence in which the range starts
  long long seq_at;          // where that sequence starts
};
// (total < 2^47: the host's limits. The products of most launches fit 32 bits, whose division takes a fraction of the time.)
__device__ __forceinline__ long long tree_div(long long a, long long b) {
  return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}
__device__ __forceinline__ long long tree_cut(long long total, int cta, int ctas) { return tree_div(total * cta, ctas); }
__device__ __forceinline__ int tree_cta_of(long long unit, long long total, int ctas) { return (int)tree_div((unit + 1) * ctas - 1, total); }

// All threads; scratch: THREADS / 32 + 4 words of 8 bytes. Ends with a barrier.
template <int THREADS>
__device__ __forceinline__ TreeRange tree_range(const TreeParams& p, long long* scratch) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (p.batch + THREADS - 1) / THREADS;
  const int b0 = min(p.batch, tid * per), b1 = min(p.batch, b0 + per);
  long long sum = 0;
  for (int b = b0; b < b1; b++) sum += tree_seq(p, b).weight;
  long long x = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(FULL, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) scratch[warp] = x;
  __syncthreads();
  long long before = x - sum, total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; w++) {
    const long long t = scratch[w];
    if (w < warp) before += t;
    total += t;
  }
  TreeRange r;
  r.total = total;
  r.ctas = (int)min((long long)p.ctas, total);
  r.at = r.end = total;
  if (blockIdx.x < r.ctas) {
    r.at = tree_cut(total, blockIdx.x, r.ctas);
    r.end = tree_cut(total, blockIdx.x + 1, r.ctas);
  }
  if (r.at < r.end && before <= r.at && r.at < before + sum) {
    int b = b0;
    for (;; b++) {
      const long long w = tree_seq(p, b).weight;
      if (r.at < before + w) break;
      before += w;
    }
    scratch[THREADS / 32] = b;
    scratch[THREADS / 32 + 1] = before;
  }
  __syncthreads();
  r.b = (int)scratch[THREADS / 32];
  r.seq_at = scratch[THREADS / 32 + 1];
  return r;
}

// What the tokens of a tile see: per token its mask (without drafted tokens before its window) and the first context row of its window.
template <int TILE>
struct TreeMasks {
  uint32_t bits[TILE][IQ_TREE_MAX_TOKENS / 32];  // of token first + i
  int from[TILE];
  int from_max;  // of all tokens of the tile
};
__device__ __forceinline__ uint32_t tree_mask_word(const TreeParams& p, int b, int t, int w, int tokens) {
  const int left = tokens - 32 * w;  // bits of tokens that the sequence has
  const uint32_t have = left >= 32 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << left) - 1u;
  if (p.mask) return p.mask[((size_t)b * p.n_tokens_max + t) * p.mask_words + w] & have;
  const int k = t + 1 - 32 * w;  // the chain: tokens 0 .. t
  return have & (k >= 32 ? 0xFFFFFFFFu : k <= 0 ? 0u : (1u << k) - 1u);
}
__device__ __forceinline__ int tree_position(const TreeParams& p, int b, int t, const TreeSeq& s) {
  int n = 0;
  for (int w = 0; w < p.mask_words; w++) n += __popc(tree_mask_word(p, b, t, w, s.tokens));
  return s.ctx + n - 1;
}
// Threads tid, tid + threads, ... take a token each; the caller's barrier follows. from_max has to be 0 before (and behind a barrier).
template <int TILE>
__device__ __forceinline__ void tree_masks(const TreeParams& p, TreeMasks<TILE>& m, int b, const TreeSeq& s, int first, int n, int tid, int threads) {
  for (int i = tid; i < n; i += threads) {
    const int t = first + i;
    int from = 0;
    if (p.window > 0) from = max(0, tree_position(p, b, t, s) - p.window + 1);
    m.from[i] = from;
    if (from > 0) atomicMax(&m.from_max, from);
    for (int w = 0; w < p.mask_words; w++) {
      uint32_t bits = tree_mask_word(p, b, t, w, s.tokens);
      if (from > p.sinks && p.window <= s.tokens) {  // drafted tokens can lie before the window only if it is no longer than the tree
        for (uint32_t left = bits; left; left &= left - 1) {
          const int j = __ffs(left) - 1;
          const int pos = tree_position(p, b, 32 * w + j, s);
          if (pos < from && pos >= p.sinks) bits &= ~(1u << j);
        }
      }
      m.bits[i][w] = bits;
    }
  }
}
// Whether token first + i sees cache row r.
template <int TILE>
__device__ __forceinline__ bool tree_sees(const TreeMasks<TILE>& m, int i, int r, int ctx, int rows, int sinks) {
  if (r >= rows) return false;
  if (r < ctx) return r >= m.from[i] || r < sinks;
  const int j = r - ctx;
  return (m.bits[i][j >> 5] >> (j & 31)) & 1u;
}

}  // namespace iq
