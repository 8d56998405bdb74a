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
__device__ __forceinline__ uint32_t tree_mask_word(const TreeParams& p, int b, int t, int w, int tokens) {
  const int left = tokens - 32 * w;  // bits of tokens that the sequence has
  const uint32_t have = left >= 32 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << left) - 1u;
  if (p.mask) return p.mask[((size_t)b * p.n_tokens_max + t) * p.mask_words + w] & have;
  const int k = t + 1 - 32 * w;  // the chain: tokens 0 .. t
  return have & (k >= 32 ? 0xFFFFFFFFu : k <= 0 ? 0u : (1u << k) - 1u);
}
__device__ __forceinline__ int tree_seen(const TreeParams& p, int b, int t, int tokens) {  // drafted tokens that token t sees
  int n = 0;
  for (int w = 0; w < p.mask_words; w++) n += __popc(tree_mask_word(p, b, t, w, tokens));
  return n;
}
__device__ __forceinline__ int tree_position(const TreeParams& p, int b, int t, const TreeSeq& s) {
  return s.ctx + tree_seen(p, b, t, s.tokens) - 1;
}
template <int TILE>
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
    // The first token of a chain sees itself; by its mask a token may see no drafted token, and its window begin a row further back. (To
    // look at the masks here took a launch over one sequence 1 us. Where they say more, the pages that it concerns are not missed:
    // tree_block_row.)
    s.skipped = max(0, (max(0, s.ctx - p.window + (p.mask ? 0 : min(s.tokens, 1))) >> 7) - s.sink_blocks);
  }
  s.blocks = total - s.skipped;
  s.tiles = (s.tokens * p.group + TILE - 1) / TILE;
  s.weight = (long long)p.n_kv_heads * s.tiles * (s.blocks + TREE_SEG_COST);
  return s;
}

// The first context row of the tokens' windows, a token's being ctx - window + (drafted tokens that it sees).
__device__ __forceinline__ int tree_first_row(const TreeParams& p, int b, const TreeSeq& s) {
  int n = s.tokens;
  for (int t = 0; t < s.tokens; t++) n = min(n, tree_seen(p, b, t, s.tokens));
  return max(0, s.ctx - p.window + n);
}
// Row of the cache arrays where block v of the sequence starts. Its page may be missing if the block holds context rows only and lies before
// all windows: page 0, read in its place like in that of any entry outside the pool, is then not flagged, and no token sees it.
__device__ __forceinline__ size_t tree_block_row(const TreeParams& p, int b, int g, const TreeSeq& s, int v, uint32_t* status) {
  const int row = s.block(v) * 128;
  if (p.pm.table == nullptr) return cache_row(p.pm, b, g, row, nullptr);
  const int j = row / p.pm.page_rows;
  int page = p.pm.table[(size_t)b * (p.t_cap / p.pm.page_rows) + j];
  if (__builtin_expect((unsigned)page >= (unsigned)p.pm.num_pages, 0)) {
    page = 0;
    const bool unseen = p.window > 0 && v >= s.sink_blocks && row + 128 <= min(s.ctx, tree_first_row(p, b, s));
    if (status && !unseen) atomicOr(&status[0], IQ_STATUS_BAD_PAGE);
  }
  return ((size_t)page * p.n_kv_heads + g) * (size_t)p.pm.page_rows + (size_t)(row - j * p.pm.page_rows);
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
// (total * ctas < 2^63: an item takes 8 KB of the workspace, so a launch has some 2^25 of them at most, each of at most 2^24 blocks. The
// products of most launches fit 32 bits, whose division takes a fraction of the time.)
__device__ __forceinline__ long long tree_div(long long a, long long b) {
  return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}
__device__ __forceinline__ long long tree_cut(long long total, int cta, int ctas) { return tree_div(total * cta, ctas); }
__device__ __forceinline__ int tree_cta_of(long long unit, long long total, int ctas) { return (int)tree_div((unit + 1) * ctas - 1, total); }

// By one converged warp, 32 sequences at a time: first the launch's units, then the sequence that this CTA's range starts in. (The other
// warps need neither; with all of them at it, each fetching the code, a launch over one short sequence took 2 us longer.)
template <int TILE>
__device__ __forceinline__ TreeRange tree_range(const TreeParams& p, int lane) {
  TreeRange r;
  long long total = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 32)
    if (b0 + lane < p.batch) total += tree_seq<TILE>(p, b0 + lane).weight;
#pragma unroll 1
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(FULL, total, o);
  r.total = total;
  r.ctas = (int)min((long long)p.ctas, total);
  r.at = r.end = total;
  r.b = 0;
  r.seq_at = 0;
  if (blockIdx.x >= r.ctas) return r;
  r.at = tree_cut(total, blockIdx.x, r.ctas);
  r.end = tree_cut(total, blockIdx.x + 1, r.ctas);
  for (int b0 = 0;; b0 += 32) {
    const long long w = b0 + lane < p.batch ? tree_seq<TILE>(p, b0 + lane).weight : 0;
    long long x = w;
#pragma unroll 1
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(FULL, x, o);
      if (lane >= o) x += y;
    }
    const uint32_t behind = __ballot_sync(FULL, r.at < r.seq_at + x);  // lanes whose sequence ends behind the start
    if (behind) {
      const int at = __ffs(behind) - 1;
      r.b = b0 + at;
      r.seq_at += __shfl_sync(FULL, x - w, at);
      return r;
    }
    r.seq_at += __shfl_sync(FULL, x, 31);
  }
}

// What the tokens of a tile see: per token its mask (without drafted tokens before its window) and the first context row of its window.
template <int TILE>
struct TreeMasks {
  uint32_t bits[TILE][IQ_TREE_MAX_TOKENS / 32];  // of token first + i
  int from[TILE];
  int from_max;  // of all tokens of the tile
};
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
