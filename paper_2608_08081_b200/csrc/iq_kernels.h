// Internal interface between the C ABI (iq_api.cu) and the kernel translation units.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/isoquant.h"

namespace iq {

// Polls one mbarrier wait of a kernel may take before it gives up (IQ_STATUS_WAIT_TIMEOUT; the reconstruction: rows of NaN):
// with the 20 us suspend hint of a poll that is at most 65536 * 20 us = 1.3 s (and a few milliseconds at least). Waits that
// work last microseconds. A warp that has given up waits no more, and what it no longer signals runs out once for the warps that
// need it, so a CTA returns within about twice that time after its first failed wait.
constexpr uint32_t DEC_WAIT_LIMIT = 1u << 16;

// Addressing of the cache arrays: contiguous per sequence (table == nullptr) or a pool of pages with a block table
// (see cache_row in iq_common.cuh).
struct PageMap {
  const int32_t* table;
  int page_rows, num_pages, n_kv_heads, t_cap;
};

// ---- quantize-append
constexpr int QA_WARPS = 4;

struct QuantizeParams {
  const __half* k_new;
  const __half* v_new;
  long long stride_b, stride_t, stride_h;
  const int32_t* append_pos;
  const int32_t* n_new;
  int n_new_max;
  const int32_t* token_start;  // [batch + 1]: packed rows, n_rows of them in all (stride_b and n_new are then not read); or nullptr
  int n_rows;
  const float* rot;
  int bits;                 // 2, 3 or 4
  float thresholds_k[15];   // the first 2^bits - 1 are read
  float thresholds_v[15];
  uint8_t* k_codes;
  float* k_scales;
  uint8_t* v_codes;
  float* v_scales;
  uint32_t* status;
  int n_kv_heads, t_cap;
  PageMap pm;
  int scale_f16;
  float big;                // bulk: 0.5 over the band around a threshold (set by the launcher)
  uint32_t wait_polls;      // bulk: limit of the waits for tensor-core results: DEC_WAIT_LIMIT, or what the self-test asks for
};
#ifdef __CUDACC__
// Where packed sequence b starts among `places` places, and how many tokens it has. (Both starts are brought into range before their
// difference is taken, which then fits whatever they hold.)
__device__ __forceinline__ int packed_start(const int32_t* token_start, int b, int places) { return max(0, min(token_start[b], places)); }
__device__ __forceinline__ int packed_tokens(const int32_t* token_start, int b, int places) {
  return max(0, packed_start(token_start, b + 1, places) - packed_start(token_start, b, places));
}
// New rows of sequence b, and where its first one starts, in elements from k_new or v_new.
__device__ __forceinline__ int append_rows(const QuantizeParams& p, int b) {
  const int n = p.token_start ? packed_tokens(p.token_start, b, p.n_rows) : p.n_new ? p.n_new[b] : p.n_new_max;
  return min(n, p.n_new_max);
}
// Rows of packed sequence b that n_new_max leaves out: flagged, and counted `times` each. By one thread per sequence, or with times = 1 by one per
// (sequence, KV head, side).
__device__ __forceinline__ void append_left_out(const QuantizeParams& p, int b, int times) {
  if (p.token_start == nullptr || p.status == nullptr) return;
  const int left = packed_tokens(p.token_start, b, p.n_rows) - p.n_new_max;
  if (left <= 0) return;
  atomicOr(&p.status[0], IQ_STATUS_ROW_OUT_OF_RANGE);
  atomicAdd(&p.status[2], (uint32_t)left * (uint32_t)times);
}
__device__ __forceinline__ size_t append_source(const QuantizeParams& p, int b) {
  return p.token_start ? (size_t)packed_start(p.token_start, b, p.n_rows) * p.stride_t : (size_t)b * p.stride_b;
}
#endif
cudaError_t launch_quantize_append(const QuantizeParams& p, int head_dim, int batch, cudaStream_t stream);
bool append_bulk_takes(const QuantizeParams& p, int head_dim);
cudaError_t launch_append_bulk(const QuantizeParams& p, int head_dim, int batch, cudaStream_t stream);

// ---- calibration: histogram of the rotated, normalised coordinates of a set of rows
constexpr int HIST_MAX_BINS = 4096;
constexpr int HIST_ROWS_PER_WARP = 128;
struct HistogramParams {
  const __half* x;
  long long stride_b, stride_t, stride_h;
  const int32_t* n_rows;
  int n_rows_max;
  const float* rot;
  uint32_t* hist;
  int bins;
  float range;
  int n_kv_heads;
};
cudaError_t launch_rotated_histogram(const HistogramParams& p, int head_dim, int batch, cudaStream_t stream);

// ---- calibration of the rotation: z = sqrt(d) H x^ of a set of rows
struct WhtParams {
  const __half* x;
  long long stride_b, stride_t, stride_h;
  const int32_t* n_rows;
  int n_rows_max;
  float* z;  // [batch][n_rows_max][n_kv_heads][head_dim]
  int n_kv_heads;
};
cudaError_t launch_wht_coordinates(const WhtParams& p, int head_dim, int batch, cudaStream_t stream);

// ---- fused decode
constexpr int DEC_BLOCK_TOKENS = 128;  // cached rows per block of the decode kernel = rows of one transposed V block
// Constants of the lookups (iq_decode_common.cuh) that the kernels take as parameters: an addition of -0 or a product with -1 that the
// compiler sees as such becomes the logic that it is there to avoid.
struct LookupConst { uint32_t neg_zero, minus_one; };
constexpr LookupConst LOOKUP_CONST = {0x80008000u, 0xFFFFFFFFu};
constexpr int DEC_HEADS = 8;          // query heads of one KV head that a work item covers (they share the N columns of one MMA)

struct DecodeParams {
  const uint8_t* k_codes;
  const float* k_scales;
  const uint8_t* v_codes;
  const float* v_scales;
  const __half* q;
  const float* rot;
  const int32_t* seq_lens;
  float* part_acc;
  float* part_ml;
  int32_t* part_argmax;
  uint32_t* status;
  int batch, n_q_heads, n_kv_heads, group, head_groups, t_cap, splits;
  PageMap pm;
  int scale_f16;
  float sm_scale;
  int bits;  // 2, 3 or 4
  // fp16 path: low / high bytes of the fp16 levels of the K and V codebooks, 4 per register (2^bits / 4 registers used)
  uint32_t lut_lo[4], lut_hi[4], lut_v_lo[4], lut_v_hi[4];
  // integer path (levels on an 8-bit grid): level_j = lut8 byte j (int8) * delta, per side
  uint32_t lut8[4], lut8_v[4];
  float delta, delta_v;
  int use_i8;
  LookupConst lookup;
  // Decode with append (k_new != nullptr; otherwise none of the following is read): the step's new K and V rows
  // [batch][n_kv_heads][head_dim] are quantised and appended at row seq_lens[b] by one warp per (sequence, KV head),
  // which also writes the new row's own partial (new_acc [batch][n_q_heads][head_dim], new_ml [batch][n_q_heads][2]);
  // the blocks of the cache are read up to row seq_lens[b] - 1.
  const __half* k_new;
  const __half* v_new;
  float* new_acc;
  float* new_ml;
  int aux_ctas;  // CTAs at the start of the grid that only append (set by the launcher)
  int len_bias;  // added to every sequence length before it is clamped to [0, t_cap] (1: the lengths given are those before an append that has been enqueued)
  float thresholds_k[15], thresholds_v[15];
  float levels_k[16], levels_v[16];
};
cudaError_t launch_decode_attention(const DecodeParams& p, int head_dim, cudaStream_t stream);
int decode_ctas_per_sm(int head_dim);
int decode_groups_per_cta(int head_dim);
cudaError_t launch_bounded_wait_selftest(uint32_t* status, uint32_t polls, cudaStream_t stream);

// ---- combine + inverse rotation
struct CombineParams {
  const float* part_acc;
  const float* part_ml;
  const int32_t* part_argmax;
  const float* rot;
  void* out;
  float* lse;
  int32_t* argmax;
  int batch, n_q_heads, n_kv_heads, splits, out_is_fp16;
  // Context sharding: the partials of `shards` ranks laid out rank after rank (each [batch][n_q_heads][splits][..]);
  // a head then has shards * splits slots. row_offsets [shards][batch] (or nullptr) turns a shard's argmax rows into
  // rows of the whole sequence. shards = 1 is the plain layout.
  int shards;
  const int32_t* row_offsets;
  // Decode with append: the partial of the step's new row, one more slot per head (nullptr: none); its row is new_rows[b].
  const float* new_acc;
  const float* new_ml;
  const int32_t* new_rows;
};
cudaError_t launch_combine_splits(const CombineParams& p, int head_dim, cudaStream_t stream);

// ---- reconstruction of fp16 K/V rows from the packed cache (the reconstruct-then-compute model)
struct ReconstructParams {
  const uint8_t* k_codes;
  const float* k_scales;
  const uint8_t* v_codes;
  const float* v_scales;
  const float* rot;
  const int32_t* seq_lens;
  __half* k_out;
  __half* v_out;
  long long stride_b, stride_t, stride_h;  // in elements
  int n_kv_heads, t_cap, out_rows;
  PageMap pm;
  int scale_f16;
  int bits;
  float levels_k[16], levels_v[16];
  uint32_t wait_polls;  // limit of the waits for tensor-core results: DEC_WAIT_LIMIT, or what the self-test asks for
};
cudaError_t launch_reconstruct_rows(const ReconstructParams& p, int head_dim, int batch, cudaStream_t stream);
// The same on the tensor cores; false: the levels are not binary16 values times one factor per side.
bool launch_reconstruct_tiles(const ReconstructParams& p, int head_dim, int batch, cudaStream_t stream, cudaError_t& e);

// ---- tree attention: drafted tokens over the packed cache
// What an item of the launch costs beside its blocks (queries, first references, partial), in blocks. With 1, 5, 7, 9 in its place: 32
// sequences of 4000 and 100 rows in turn, 32 columns, 160, 90, 75, 73 us; 64 of 250 to 500 rows 68.9, 66.9, 62.4, 62.5; one of 32 K rows,
// 240 pairs, 101, 98, 95, 93; 64 windows of 1 K rows 58.2, 57.0, 56.6, 56.4; one of 1000 rows 17.5, 17.4, 17.9, 18.1.
constexpr int TREE_SEG_COST = 7;
struct TreeParams {
  const uint8_t* k_codes;
  const float* k_scales;
  const uint8_t* v_codes;
  const float* v_scales;
  const __half* q;
  long long qs_b, qs_t, qs_h;  // strides of q, in elements
  const float* rot;
  const int32_t* ctx_lens;
  const uint32_t* mask;      // [batch][n_tokens_max][mask_words], or nullptr: a chain
  const int32_t* n_tokens;   // [batch], or nullptr
  int n_tokens_max, mask_words, window, sinks;
  // For the short sequences of a step of any lengths: packed tokens (token_start [batch + 1] among `places`, or nullptr: `places` per sequence);
  // sequences of more than n_tokens_max tokens are left out; with `cross` no token has a row of its own. iq_tree_attention: nullptr,
  // n_tokens_max, 0, 0.
  const int32_t* token_start;
  int places, leave_longer, cross;
  int batch, n_q_heads, n_kv_heads, group, t_cap;
  PageMap pm;
  int scale_f16;
  int bits;
  // The levels, exact, times a unit per side (8-bit grid: the integers and delta; else the levels and 1). K: binary16 values, V: bfloat16
  // values, or where they have more than 8 bits sums of two (v_terms). Low and high bytes, 4 per register (2^bits / 4 registers used).
  uint32_t lut_lo[4], lut_hi[4], lut_v_lo[2][4], lut_v_hi[2][4];
  int v_terms;
  LookupConst lookup;
  float score_unit;          // sm_scale log2(e) unit_K / sqrt(d): a score in units of log2 is this times scale times the product
  float value_unit;          // unit_V / sqrt(d)
  int tile, tiles;           // (token, head) pairs of an item, items per (sequence, KV head)
  int ctas;                  // CTAs of the launch
  // Workspace. A partial belongs to (item, CTA): its number is the item's plus the CTA's, both of which only grow along the launch's
  // order of blocks.
  float* part_acc;           // [items + ctas][tile][head_dim], rotated space
  float* part_ml;            // [items + ctas][tile][2]: reference (log2 units), sum
  int2* item_info;           // [items]: first CTA, number of CTAs
  void* out;
  int out_is_fp16;
  float* lse;
  uint32_t* status;
  uint32_t wait_polls;       // limit of the waits: DEC_WAIT_LIMIT, or what the self-test asks for
};
cudaError_t launch_tree_attention(const TreeParams& p, int head_dim, cudaStream_t stream);
// CTAs per SM: two where they fit, so that one's items end and begin under the other's blocks: 64 sequences with a window of 1 K rows, 3
// tokens and 8 heads per KV head, 112 us instead of 130
constexpr int tree_ctas_per_sm(int head_dim, int tile) { return head_dim == 128 && tile <= 32 ? 2 : 1; }
int tree_tile(int queries);  // tile for that many (token, head) pairs of a KV head

// ---- chunk and cross attention: any number of new tokens over the packed cache
// What a pair of CTAs leaves for the merge.
struct alignas(16) ChunkCut {
  int g, t, n;       // the tile that begins in the pair's range and ends in a later one (last < 0: there is none): KV head, tile, tokens of its sequence,
  int last;          // the pair in which it ends,
  long long tok0;    // the sequence's first token among those of out
  int partials;      // bit 0: the pair has a partial of the tile that its range begins in the middle of; bit 1: of the one above
};
struct ChunkParams {
  const uint8_t* k_codes;
  const float* k_scales;
  const uint8_t* v_codes;
  const float* v_scales;
  const __half* q;
  long long qs_b, qs_t, qs_h;  // strides of q, in elements (packed tokens: qs_b is not read)
  const float* rot;
  const int32_t* ctx_lens;
  const int32_t* token_start;  // [batch + 1]: packed tokens, n_tokens_max of them in all; or nullptr: n_tokens_max places per sequence
  const int32_t* n_tokens;     // [batch], or nullptr
  int n_tokens_max, causal, window, sinks;
  int least_tokens;            // sequences of fewer tokens are left to the tree attention kernel
  int batch, n_q_heads, n_kv_heads, group, t_cap;
  PageMap pm;
  int scale_f16;
  int bits;
  // The levels as binary16 values, exact, times a unit per side (8-bit grid: the integers and delta; else the levels and 1). Low and high
  // bytes, 4 per register.
  uint32_t lut_lo[4], lut_hi[4], lut_v_lo[4], lut_v_hi[4];
  LookupConst lookup;
  float score_unit;            // sm_scale log2(e) unit_K / sqrt(d)
  float value_unit;            // unit_V / sqrt(d)
  int pairs;                   // pairs of CTAs of the launch
  long long seg_units, cap_units, least_units;  // see chunk_units; a launch has no more pairs at work than total / least_units
  // Workspace. Of a pair's items at most the first and the last are cut: two partials each.
  float* part_acc;             // [2 pairs][256][head_dim], rotated space
  float* part_ml;              // [2 pairs][256][2]: reference (log2 units), sum
  ChunkCut* cuts;              // [pairs]
  float4* kept;                // [2 pairs][chunk_kept]: of the segments of a CTA's piece so far
  __half* out;
  float* lse;
  uint32_t* status;
  uint32_t wait_polls;
};
// What an item costs beside its blocks (queries, outputs or a partial), and the least that a pair of CTAs is given, in blocks. With 3, 4, 6, 8 in
// place of 6: 2047 tokens of a prompt 111, 107, 101, 106 us; 1000 tokens of a window of 4096 rows, head_dim 256, 140, 139, 145, 145; 64
// tokens behind 1000 rows 28.3, 28.5, 28.6, 29.3; 4 for the least 30.6.
constexpr int CHUNK_SEG_COST = 6, CHUNK_LEAST = 2;
// (token, head) pairs of a KV head up to which a sequence of a step is the tree attention kernel's, whose tiles are that small: where the call
// says that no sequence has more (64 pairs of 16 sequences of 16 K rows 180 us, here 367; of one of 1000 rows 20 and 25); and where
// one may (a launch of its own for them, with the limit's tile; most such sequences have one token. 28 sequences of one token beside four of 500: 0.56
// ms, all of them here 0.99).
constexpr int CHUNK_SHORT = 64, CHUNK_SHORT_MIXED = 16;
// Places of a CTA's segments: references and sums, then O, a softmax thread's (256 of them) next to another's.
constexpr size_t chunk_kept(int head_dim) { return 256 * (size_t)(1 + head_dim / 8); }
cudaError_t launch_chunk_attention(const ChunkParams& p, int head_dim, cudaStream_t stream);

// ---- a step's tokens: places, positions, cache rows
struct PlanParams {
  const int32_t* ctx_lens;
  const int32_t* n_new;
  int batch, n_tokens_max;
  PageMap pm;
  int32_t* token_start;
  int32_t* positions;
  int32_t* sequences;
  int64_t* slots;
  uint32_t* status;
};
cudaError_t launch_plan_tokens(const PlanParams& p, cudaStream_t stream);

// ---- rotary positions
struct RotarySide {
  const __half* x;
  __half* y;
  long long xs_t, xs_h, ys_t, ys_h;  // strides in elements
  int heads;
};
struct RotaryParams {
  RotarySide side[2];
  const int32_t* positions;
  int n_tokens, head_dim;
  iq_rotary rotary;
};
cudaError_t launch_apply_rotary(const RotaryParams& p, cudaStream_t stream);

// ---- rows and pages of the cache
struct CacheArrays {
  uint8_t* k_codes;
  float* k_scales;
  uint8_t* v_codes;
  float* v_scales;
  int scale_f16;
};
struct KeepParams {
  CacheArrays c;
  PageMap pm;
  const int32_t* base;
  const int32_t* keep;
  const int32_t* n_keep;
  int n_keep_max;
  uint32_t* status;
};
cudaError_t launch_keep_rows(const KeepParams& p, int head_dim, int bits, int batch, cudaStream_t stream);

struct PoolParams {
  int32_t* table;
  int32_t* ref;
  int32_t* free_list;
  int32_t* state;  // [0] free pages, [1] arrivals (0 between launches), [4..] one bit per page (0 between launches)
  int n_seqs, pages_per_seq, num_pages, page_rows;
  const int32_t* first_row;
  const int32_t* end_row;
  uint32_t* status;
};
constexpr int POOL_MARKS = 4;  // where the bits start
cudaError_t launch_reserve_pages(const PoolParams& p, cudaStream_t stream);
cudaError_t launch_release_pages(const PoolParams& p, cudaStream_t stream);

struct CopyParams {
  CacheArrays c;
  int n_kv_heads, row_bytes;  // packed bytes of a row, a side
  PoolParams pool;            // (iq_copy_pages: only page_rows and num_pages)
  const int32_t* src;
  const int32_t* dst;
  const int32_t* rows;        // forks: rows of the branch
  int n;
  uint32_t* status;
};
cudaError_t launch_fork_sequences(const CopyParams& p, cudaStream_t stream);
cudaError_t launch_copy_pages(const CopyParams& p, cudaStream_t stream);

// ---- rotation parameters
cudaError_t launch_make_rotation(float* rot, int n_quats, uint64_t seed, cudaStream_t stream);
cudaError_t launch_normalize_rotation(float* rot, int n_quats, cudaStream_t stream);

}  // namespace iq
