// Chunk and cross attention: which rows a tile of queries sees, and how the launch's work is dealt out.
#pragma once
#include "iq_decode_common.cuh"

namespace iq {

constexpr int CHUNK_ROWS = 256;  // (token, query head) pairs of a tile: the rows of a product of two SMs

// One sequence of the launch.
struct ChunkSeq {
  int ctx, n, tiles;    // cached rows before its tokens (cross attention: all it has), tokens, tiles per KV head
  long long tok0;       // its first token among those of q and out, where they are packed; else batch row times n_tokens_max
};
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkParams& p, int b) {
  ChunkSeq s;
  s.ctx = max(0, min(p.ctx_lens[b], p.t_cap));
  if (p.token_start) {
    s.n = packed_tokens(p.token_start, b, p.n_tokens_max);
    s.tok0 = packed_start(p.token_start, b, p.n_tokens_max);
  } else {
    s.n = p.n_tokens ? max(0, min(p.n_tokens[b], p.n_tokens_max)) : p.n_tokens_max;
    s.tok0 = (long long)b * p.n_tokens_max;
  }
  if (s.n < p.least_tokens) s.n = 0;
  s.tiles = (int)(((long long)s.n * p.group + CHUNK_ROWS - 1) / CHUNK_ROWS);
  return s;
}

// Work is counted in units of 1 / group of a row: a tile counts the rows that its last token sees, a little rounded so that the sum over
// the first tiles of a sequence has a closed form, and p.seg_units more for its beginning and end.
__device__ __forceinline__ long long chunk_units(const ChunkParams& p, const ChunkSeq& s, int t) {
  const long long v = (long long)p.group * s.ctx;
  return p.seg_units + (p.causal ? min(v + (long long)CHUNK_ROWS * (t + 1), p.cap_units) : v);
}
// Units of tiles 0 .. t - 1 of a KV head.
__device__ __forceinline__ long long chunk_units_before(const ChunkParams& p, const ChunkSeq& s, int t) {
  const long long v = (long long)p.group * s.ctx;
  if (!p.causal) return t * (p.seg_units + v);
  const long long m = max(0ll, min((long long)t, (p.cap_units - v) / CHUNK_ROWS));  // tiles below the cap
  return t * p.seg_units + m * v + CHUNK_ROWS * (m * (m + 1) / 2) + (t - m) * p.cap_units;
}
__device__ __forceinline__ long long chunk_seq_units(const ChunkParams& p, const ChunkSeq& s) {
  return (long long)p.n_kv_heads * chunk_units_before(p, s, s.tiles);
}
__device__ __forceinline__ long long chunk_cut(long long total, int pair, int pairs) { return unit_div(total * pair, pairs); }

// The blocks of 128 rows that a tile's tokens see: the first `sink_blocks`, then those from the first window on.
struct ChunkTile {
  int t0, t1;                      // first and last token
  int end;                         // rows behind this are seen by none of them
  int blocks, sink_blocks, first;
  __device__ __forceinline__ int block(int v) const { return v < sink_blocks ? v : v - sink_blocks + first; }
};
__device__ __forceinline__ ChunkTile chunk_tile(const ChunkParams& p, const ChunkSeq& s, int t) {
  ChunkTile x;
  x.t0 = t * CHUNK_ROWS / p.group;  // (n_tokens_max * group fits 31 bits: the host's limit)
  x.t1 = min(s.n - 1, (t * CHUNK_ROWS + CHUNK_ROWS - 1) / p.group);
  x.end = p.causal ? min(s.ctx + x.t1 + 1, p.t_cap) : s.ctx;
  const int total = (x.end + 127) >> 7;
  x.first = p.window > 0 ? min(total, max(0, s.ctx + x.t0 - p.window + 1) >> 7) : 0;
  x.sink_blocks = min((p.sinks >> 7) + ((p.sinks & 127) != 0), x.first);
  x.blocks = total - x.first + x.sink_blocks;
  return x;
}
// Blocks of an item before its unit o. (units * blocks < 2^62: the host's limit.)
__device__ __forceinline__ int chunk_blocks_before(const ChunkParams& p, long long o, long long units, int blocks) {
  if (o >= units) return blocks;
  return o <= p.seg_units ? 0 : (int)unit_div((o - p.seg_units) * blocks, units - p.seg_units);
}

// The launch's items (sequence, KV head, tile), laid end to end and cut into one range of equal length per pair of CTAs.
struct ChunkRange {
  long long at, end, total;  // units
  long long seq_at;          // where sequence b, in which the range starts, starts
  int b, pairs;              // pairs of CTAs that have a range
  ChunkSeq sq;               // sequence b
};
// By one converged warp.
__device__ __forceinline__ ChunkRange chunk_range(const ChunkParams& p, int pair, int lane) {
  ChunkRange r;
  ChunkSeq s = {};
  long long total = 0, w = 0;
  for (int b = lane; b < p.batch; b += 32) {
    s = chunk_seq(p, b);
    w = chunk_seq_units(p, s);
    total += w;
  }
#pragma unroll 1
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(FULL, total, o);
  r.total = total;
  r.pairs = (int)max(1ll, min((long long)p.pairs, unit_div(total, p.least_units)));
  r.at = r.end = total;
  r.b = 0;
  r.seq_at = 0;
  if (total == 0 || pair >= r.pairs) return r;
  r.at = chunk_cut(total, pair, r.pairs);
  r.end = chunk_cut(total, pair + 1, r.pairs);
#pragma unroll 1
  for (int b0 = 0;; b0 += 32) {
    if (p.batch > 32) {  // (else they are the lanes' already)
      w = 0;
      if (b0 + lane < p.batch) {
        s = chunk_seq(p, b0 + lane);
        w = chunk_seq_units(p, s);
      }
    }
    long long x = w;
#pragma unroll 1
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(FULL, x, o);
      if (lane >= o) x += y;
    }
    const uint32_t behind = __ballot_sync(FULL, r.at < r.seq_at + x);
    if (behind) {
      const int at = __ffs(behind) - 1;
      r.b = b0 + at;
      r.seq_at += __shfl_sync(FULL, x - w, at);
      r.sq.ctx = __shfl_sync(FULL, s.ctx, at);
      r.sq.n = __shfl_sync(FULL, s.n, at);
      r.sq.tiles = __shfl_sync(FULL, s.tiles, at);
      r.sq.tok0 = __shfl_sync(FULL, s.tok0, at);
      return r;
    }
    r.seq_at += __shfl_sync(FULL, x, 31);
  }
}

// A piece: the blocks [lo, hi) of an item that lie in this pair's range.
struct ChunkPiece {
  ChunkSeq sq;
  ChunkTile x;
  int b, g, t;
  int lo, hi;
  int slot;  // of its partial; -1: it is the whole item
};
// The pieces of a range, one after the other; every warp walks for itself, converged.
struct ChunkWalk {
  ChunkSeq sq;
  int b, g, t;
  long long unit, end, item_at;  // next unit, end of the range, where item (b, g, t) starts
  bool begun;                    // that item begins in this range
  ChunkCut cut;                  // (last: 0 where there is such a tile, until it is known)
  long long cut_end;             // where that tile ends
  __device__ __forceinline__ void start(const ChunkParams& p, const ChunkRange& r) {
    unit = r.at;
    end = r.end;
    cut.last = -1;
    cut.partials = 0;
    b = g = t = 0;
    item_at = 0;
    begun = true;
    if (unit >= end) return;
    b = r.b;
    sq = r.sq;
    const long long head = chunk_units_before(p, sq, sq.tiles);
    long long rest = unit - r.seq_at;
    g = (int)unit_div(rest, head);
    rest -= g * head;
    int lo = 0, hi = sq.tiles;  // the last tile that starts at or before it
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (chunk_units_before(p, sq, m) <= rest) lo = m; else hi = m;
    }
    t = lo;
    item_at = unit - (rest - chunk_units_before(p, sq, t));
    begun = item_at == unit;
  }
  // False: the range is done. A piece without blocks is an item that no token of sees a row.
  __device__ __forceinline__ bool next(const ChunkParams& p, ChunkPiece& c) {
    while (unit < end) {
      const long long units = chunk_units(p, sq, t);
      c.sq = sq;
      c.b = b;
      c.g = g;
      c.t = t;
      c.x = chunk_tile(p, sq, t);
      c.lo = chunk_blocks_before(p, unit - item_at, units, c.x.blocks);
      c.hi = chunk_blocks_before(p, end - item_at, units, c.x.blocks);
      c.slot = c.lo == 0 && c.hi == c.x.blocks ? -1 : 2 * (int)(blockIdx.x >> 1) + (begun ? 1 : 0);
      const bool first = begun;
      if (begun && item_at + units > end) {
        cut.g = g;
        cut.t = t;
        cut.n = sq.n;
        cut.tok0 = sq.tok0;
        cut.last = 0;
        cut_end = item_at + units;
      }
      if (c.slot >= 0 && c.hi > c.lo) cut.partials |= begun ? 2 : 1;
      unit = min(end, item_at + units);
      item_at += units;
      begun = true;
      if (++t == sq.tiles && unit < end) {
        t = 0;
        if (++g == p.n_kv_heads) {
          g = 0;
          for (uint32_t some = 0; !some; b += some ? 0 : 32) {  // the next sequence with tiles (units are left, so there is one), 32 at a time
            const int x = b + 1 + (threadIdx.x & 31);
            some = __ballot_sync(FULL, x < p.batch && chunk_seq(p, x).tiles > 0);
            if (some) b += __ffs(some);
          }
          sq = chunk_seq(p, b);
        }
      }
      if (c.hi > c.lo || (c.x.blocks == 0 && first)) return true;
    }
    return false;
  }
};

}  // namespace iq
