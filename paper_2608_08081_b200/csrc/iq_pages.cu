// Rows and pages of the packed cache: rows of accepted drafted tokens moved together, pages copied, shared, taken from and given back to
// a pool. Integer work on a few kilobytes (the copies apart): what bounds these kernels is a launch and a few trips to memory one after
// the other, so each is one launch, and what has to be agreed on between CTAs (the top of the stack of free pages) is worked out by
// every CTA for itself and written by the one that arrives last. In a captured graph, one B200: three of five rows of one sequence kept
// 1.9 us, up to a quarter of 60 in each of 64 sequences (8 KV heads) 10.3; pages of 8 sequences given back and reserved 7.2, of 512 12.4;
// four branches given back and made anew 9.3, 64 with 13.7 MB of rows (16.9 MB with the rest of their blocks) copied 19.9; 512 pages of 53
// KB a side copied 24.5.
#include "iq_common.cuh"
#include "iq_format.cuh"

namespace iq {
namespace {

// ------------------------------------------------------------------------------------------------ rows
// Code v into entry e (0 .. 31) of a group of 32 entries, BITS words.
template <int BITS>
__device__ __forceinline__ void set_code(uint32_t (&w)[BITS], int e, uint32_t v) {
  if constexpr (BITS == 3) {
    if (e < 24) {
#pragma unroll
      for (int k = 0; k < 3; k++)
        if (k == e >> 3) w[k] = (w[k] & ~(7u << (4 * (e & 7)))) | (v << (4 * (e & 7)));
    } else {
      const int sh = 4 * (e - 24) + 3;
#pragma unroll
      for (int k = 0; k < 3; k++) w[k] = (w[k] & ~(1u << sh)) | (((v >> k) & 1u) << sh);
    }
  } else {
    int word, sh;
    packed_place<BITS>(e, word, sh);
#pragma unroll
    for (int k = 0; k < BITS; k++)
      if (k == word) w[k] = (w[k] & ~(((1u << BITS) - 1u) << sh)) | (v << sh);
  }
}

constexpr int KEEP_THREADS = 256;
static_assert(IQ_KEEP_MAX_ROWS <= KEEP_THREADS, "a thread finds the place of one row");

// CTA (KV head, sequence, side). Every source is read before any destination is written: the K rows wait in shared memory, the codes of
// a V coordinate belong to one thread, which holds all of them (in shared memory, 8 to a word) before it changes a word of the
// coordinate's records.
template <int D, int BITS>
__global__ void __launch_bounds__(KEEP_THREADS) keep_rows_kernel(const KeepParams p) {
  constexpr int P = PackedFormat<BITS>::row_bytes(D), UNITS = P / 16;
  __shared__ long long s_src[IQ_KEEP_MAX_ROWS], s_dst[IQ_KEEP_MAX_ROWS];  // rows of the arrays; src -1: nothing to do
  __shared__ __align__(16) uint8_t s_buf[IQ_KEEP_MAX_ROWS * (P > D / 2 ? P : D / 2)];
  grid_dependency_wait();
  allow_dependent_launch();
  const int g = blockIdx.x, b = blockIdx.y, side = blockIdx.z, tid = threadIdx.x;
  int n = p.n_keep ? p.n_keep[b] : p.n_keep_max;
  n = max(0, min(n, p.n_keep_max));
  if (n == 0) return;
  float scale = 0.f;
  float* const scales = side ? p.c.v_scales : p.c.k_scales;
  if (tid < n) {
    uint32_t* const status = side == 0 ? p.status : nullptr;  // (counted by one side)
    const long long base = p.base[b], from = base + p.keep[(size_t)b * p.n_keep_max + tid], to = base + tid;
    long long src = -1, dst = -1;
    if (from < 0 || from >= p.pm.t_cap || to < 0 || to >= p.pm.t_cap) {
      if (status) { atomicOr(&status[0], IQ_STATUS_ROW_OUT_OF_RANGE); atomicAdd(&status[2], 1u); }
    } else {
      size_t rs, rd;
      const bool ok_s = cache_row_for_write(p.pm, b, g, from, status, rs), ok_d = cache_row_for_write(p.pm, b, g, to, status, rd);
      if (!ok_s || !ok_d) {
        if (status) atomicAdd(&status[2], 1u);
      } else if (from != to) {
        src = (long long)rs;
        dst = (long long)rd;
        scale = load_scale(scales, rs, p.c.scale_f16);
      }
    }
    s_src[tid] = src;
    s_dst[tid] = dst;
  }
  __syncthreads();
  if (side == 0) {
    uint4* const buf = reinterpret_cast<uint4*>(s_buf);
    for (int i = tid; i < n * UNITS; i += KEEP_THREADS) {
      const long long r = s_src[i / UNITS];
      if (r >= 0) buf[i] = *reinterpret_cast<const uint4*>(p.c.k_codes + (size_t)r * P + 16 * (i % UNITS));
    }
    __syncthreads();
    for (int i = tid; i < n * UNITS; i += KEEP_THREADS)
      if (s_src[i / UNITS] >= 0) *reinterpret_cast<uint4*>(p.c.k_codes + (size_t)s_dst[i / UNITS] * P + 16 * (i % UNITS)) = buf[i];
  } else if (tid < D) {
    // the record of coordinate tid in the block of a row (a block starts at a row that is a multiple of 128 in its sequence or page, and
    // in the arrays)
    auto record = [&](long long row) { return reinterpret_cast<uint32_t*>(p.c.v_codes + (size_t)(row & ~127ll) * P + (size_t)tid * (16 * BITS)); };
    uint32_t* const codes = reinterpret_cast<uint32_t*>(s_buf) + tid;  // word j: codes of rows 8 j .. 8 j + 7
    for (int j = 0; 8 * j < n; j++) {
      uint32_t w = 0;
#pragma unroll
      for (int k = 0; k < 8; k++) {
        const int i = 8 * j + k;
        const long long r = i < n ? s_src[i] : -1;
        if (r >= 0) w |= packed_code<BITS>(record(r), (int)(r & 127)) << (4 * k);
      }
      codes[j * D] = w;
    }
    uint32_t w[BITS];
    uint32_t* at = nullptr;  // the group of 32 entries that w holds
    for (int i = 0; i < n; i++) {
      if (s_src[i] < 0) continue;
      const long long r = s_dst[i];
      uint32_t* const unit = record(r) + (((int)r & 127) >> 5) * BITS;
      if (unit != at) {
        if (at) {
#pragma unroll
          for (int k = 0; k < BITS; k++) at[k] = w[k];
        }
        at = unit;
#pragma unroll
        for (int k = 0; k < BITS; k++) w[k] = at[k];
      }
      set_code<BITS>(w, (int)r & 31, (codes[(i >> 3) * D] >> (4 * (i & 7))) & 15u);
    }
    if (at) {
#pragma unroll
      for (int k = 0; k < BITS; k++) at[k] = w[k];
    }
  }
  // (the scales were read before the first barrier)
  if (tid < n && s_src[tid] >= 0) store_scale(scales, (size_t)s_dst[tid], scale, p.c.scale_f16, nullptr);
}

// ------------------------------------------------------------------------------------------------ pool
// Sum of v over the threads of the CTA before this one, and over all of them. s_warp: 33 words. Ends with a barrier before s_warp is
// written again by the next call's first one.
template <int THREADS>
__device__ __forceinline__ int block_prefix(int v, int* s_warp, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(FULL, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  if (warp == 0) {
    const int t = lane < THREADS / 32 ? s_warp[lane] : 0;
    int y = t;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int z = __shfl_up_sync(FULL, y, o);
      if (lane >= o) y += z;
    }
    s_warp[lane] = y - t;
    if (lane == 31) s_warp[32] = y;
  }
  __syncthreads();
  total = s_warp[32];
  return s_warp[warp] + x - v;
}

// Whether this CTA is the last of the launch to get here; what the others wrote and counted before is then visible to all its threads.
// The count of arrivals is 0 again afterwards.
__device__ __forceinline__ bool last_to_arrive(int32_t* state, int ctas) {
  __shared__ int s_last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    s_last = atomicAdd(&state[1], 1) == ctas - 1;
    if (s_last) state[1] = 0;
  }
  __syncthreads();
  if (s_last) __threadfence();
  return s_last != 0;
}

constexpr int RESERVE_THREADS = 1024;
// One CTA: the order in which pages are taken runs over all sequences. 1024 sequences at a time: their ranges of entries laid end to
// end, a thread to an entry, the k-th entry without a page takes the k-th page from the top.
__global__ void __launch_bounds__(RESERVE_THREADS) reserve_kernel(const PoolParams p) {
  __shared__ int s_warp[33];
  __shared__ int s_start[RESERVE_THREADS + 1], s_entry[RESERVE_THREADS];  // where a sequence's entries start among those laid end to end; its first entry
  grid_dependency_wait();
  allow_dependent_launch();
  const int tid = threadIdx.x;
  const int n_free = max(0, min(p.state[0], p.num_pages));
  int taken = 0, missing = 0;
  for (int b0 = 0; b0 < p.n_seqs; b0 += RESERVE_THREADS) {
    const int b = b0 + tid;
    int lo = 0, count = 0;
    if (b < p.n_seqs) {
      const long long cap = (long long)p.pages_per_seq * p.page_rows;
      const long long first = max(0, p.first_row[b]), end = min((long long)p.end_row[b], cap);
      if (end > first) {
        lo = (int)(first / p.page_rows);
        count = (int)((end + p.page_rows - 1) / p.page_rows) - lo;
      }
    }
    int total;
    const int start = block_prefix<RESERVE_THREADS>(count, s_warp, total);  // (at most 1024 tables: the host bounds their entries)
    s_start[tid] = start;
    s_entry[tid] = lo;
    if (tid == 0) s_start[RESERVE_THREADS] = total;
    __syncthreads();
    for (int t0 = 0; t0 < total; t0 += RESERVE_THREADS) {
      const int t = t0 + tid;
      int32_t* e = nullptr;
      if (t < total) {
        int s = 0;  // the last sequence that starts at or before t (of those that start together, the one with entries)
#pragma unroll
        for (int step = RESERVE_THREADS / 2; step > 0; step >>= 1)
          if (s_start[s + step] <= t) s += step;
        e = p.table + (size_t)(b0 + s) * p.pages_per_seq + s_entry[s] + (t - s_start[s]);
        if (*e >= 0) e = nullptr;
      }
      int want;
      const int k = taken + block_prefix<RESERVE_THREADS>(e != nullptr, s_warp, want);
      if (e) {
        if (k < n_free) {
          const int page = p.free_list[n_free - 1 - k];
          if ((unsigned)page < (unsigned)p.num_pages) {
            *e = page;
            p.ref[page] = 1;
          } else if (p.status) {  // a damaged list
            atomicOr(&p.status[0], IQ_STATUS_BAD_PAGE);
            atomicAdd(&p.status[2], 1u);
          }
        }
      }
      missing += max(0, taken + want - max(n_free, taken));
      taken += want;
    }
    __syncthreads();
  }
  if (tid == 0) {
    p.state[0] = n_free - min(taken, n_free);
    if (missing > 0 && p.status) {
      atomicOr(&p.status[0], IQ_STATUS_NO_PAGE);
      atomicAdd(&p.status[2], (uint32_t)missing);
    }
  }
}

constexpr int RELEASE_THREADS = 512;
// A warp to a sequence: counts drop by atomics (whose order does not matter), and the entry that brings one to 0 marks the page. The CTA
// that arrives last puts the marked pages on the stack in ascending order and clears the marks.
__global__ void __launch_bounds__(RELEASE_THREADS) release_kernel(const PoolParams p) {
  __shared__ int s_warp[33];
  grid_dependency_wait();
  allow_dependent_launch();
  const int tid = threadIdx.x, lane = tid & 31;
  uint32_t* const marks = reinterpret_cast<uint32_t*>(p.state + POOL_MARKS);
  const int b = blockIdx.x * (RELEASE_THREADS / 32) + (tid >> 5);
  if (b < p.n_seqs) {
    const long long cap = (long long)p.pages_per_seq * p.page_rows;
    const long long first = max(0, p.first_row[b]), end = min((long long)p.end_row[b], cap);
    const int lo = (int)((first + p.page_rows - 1) / p.page_rows), hi = end > 0 ? (int)(end / p.page_rows) : 0;
    int32_t* const row = p.table + (size_t)b * p.pages_per_seq;
    constexpr int U = 8;  // entries of a lane in flight (512 tables of 252 entries and the reservation behind it 13.8 us, one by one 15.0)
    for (int j0 = lo + lane; j0 < hi; j0 += 32 * U) {
      int pages[U];
#pragma unroll
      for (int u = 0; u < U; u++) pages[u] = j0 + 32 * u < hi ? row[j0 + 32 * u] : -1;
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int page = pages[u];
        if (page < 0) continue;
        row[j0 + 32 * u] = -1;
        bool good = page < p.num_pages;
        if (good) {
          const int was = atomicSub(&p.ref[page], 1);
          if (was <= 0) {  // held by nobody, as the pool has it: the count stays
            atomicAdd(&p.ref[page], 1);
            good = false;
          } else if (was == 1) {
            atomicOr(&marks[page >> 5], 1u << (page & 31));
          }
        }
        if (!good && p.status) {
          atomicOr(&p.status[0], IQ_STATUS_BAD_PAGE);
          atomicAdd(&p.status[2], 1u);
        }
      }
    }
  }
  if (!last_to_arrive(p.state, gridDim.x)) return;
  constexpr int U = 8;  // words of a thread in flight (the same 12.1 us, one by one 13.9)
  const int words = (p.num_pages + 31) / 32;
  int top = max(0, min(__ldcg(&p.state[0]), p.num_pages));
  for (int c = 0; c < words; c += U * RELEASE_THREADS) {
    const int w0 = c + tid * U;
    uint32_t m[U];
    int count = 0, total;
#pragma unroll
    for (int u = 0; u < U; u++) m[u] = w0 + u < words ? __ldcg(&marks[w0 + u]) : 0u;
#pragma unroll
    for (int u = 0; u < U; u++) count += __popc(m[u]);
    int at = top + block_prefix<RELEASE_THREADS>(count, s_warp, total);
    if (count) {
#pragma unroll
      for (int u = 0; u < U; u++) {
        if (m[u]) marks[w0 + u] = 0;
        for (uint32_t x = m[u]; x; x &= x - 1, at++)
          if (at < p.num_pages) p.free_list[at] = 32 * (w0 + u) + __ffs(x) - 1;
      }
    }
    top = min(top + total, p.num_pages);
  }
  if (tid == 0) p.state[0] = top;
}

// ------------------------------------------------------------------------------------------------ copies
constexpr int COPY_THREADS = 256;
constexpr int COPY_ROWS = 512;  // of one KV head, per CTA: its rows lie one behind the other in each of the four arrays
__device__ __forceinline__ void copy_rows(const CacheArrays& c, int row_bytes, size_t src_row, size_t dst_row, int rows) {  // rows: a multiple of 128
  const int codes = rows * row_bytes / 16, scales = rows * (c.scale_f16 ? 2 : 4) / 16, all = 2 * (codes + scales);
  const size_t sb = c.scale_f16 ? 2 : 4;
  auto at = [&](int i, size_t row) -> uint4* {
    if (i < codes) return reinterpret_cast<uint4*>(c.k_codes + row * row_bytes) + i;
    i -= codes;
    if (i < codes) return reinterpret_cast<uint4*>(c.v_codes + row * row_bytes) + i;
    i -= codes;
    if (i < scales) return reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(c.k_scales) + row * sb) + i;
    return reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(c.v_scales) + row * sb) + (i - scales);
  };
  constexpr int U = 8;  // loads in flight per thread
  for (int i0 = threadIdx.x; i0 < all; i0 += U * COPY_THREADS) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; u++)
      if (i0 + u * COPY_THREADS < all) x[u] = *at(i0 + u * COPY_THREADS, src_row);
#pragma unroll
    for (int u = 0; u < U; u++)
      if (i0 + u * COPY_THREADS < all) *at(i0 + u * COPY_THREADS, dst_row) = x[u];
  }
}

// CTA (KV head and run of rows of a page, pair).
__global__ void __launch_bounds__(COPY_THREADS) copy_pages_kernel(const CopyParams p) {
  grid_dependency_wait();
  allow_dependent_launch();
  const int runs = (p.pool.page_rows + COPY_ROWS - 1) / COPY_ROWS;
  const int g = blockIdx.x / runs, at = (blockIdx.x - g * runs) * COPY_ROWS;
  for (int i = blockIdx.y; i < p.n; i += gridDim.y) {
    const int src = p.src[i], dst = p.dst[i];
    if ((unsigned)src >= (unsigned)p.pool.num_pages || (unsigned)dst >= (unsigned)p.pool.num_pages) {
      if (blockIdx.x == 0 && threadIdx.x == 0 && p.status) { atomicOr(&p.status[0], IQ_STATUS_BAD_PAGE); atomicAdd(&p.status[2], 1u); }
      continue;
    }
    if (src == dst) continue;
    const size_t in_page = (size_t)g * p.pool.page_rows + at, page = (size_t)p.n_kv_heads * p.pool.page_rows;
    copy_rows(p.c, p.row_bytes, src * page + in_page, dst * page + in_page, min(COPY_ROWS, p.pool.page_rows - at));
  }
}

// CTA (0: the table and the counts; 1 + KV head and run: a run of rows of the last page, fork). Which forks are good, and which free page a
// fork's copy takes, every CTA works out from the three lists alone, which nobody writes.
__global__ void __launch_bounds__(COPY_THREADS) fork_kernel(const CopyParams p) {
  extern __shared__ uint32_t s_bits[];  // two bits per sequence: is the src of a fork, is the dst of one
  __shared__ int s_twice;
  grid_dependency_wait();
  allow_dependent_launch();
  const PoolParams& pool = p.pool;
  const int tid = threadIdx.x, i = blockIdx.y, words = (pool.n_seqs + 31) / 32, P = pool.pages_per_seq;
  uint32_t* const is_src = s_bits;
  uint32_t* const is_dst = s_bits + words;
  for (int w = tid; w < 2 * words; w += COPY_THREADS) s_bits[w] = 0;
  if (tid == 0) s_twice = 0;
  __syncthreads();
  for (int j = tid; j < p.n; j += COPY_THREADS) {
    const int s = p.src[j], d = p.dst[j];
    if ((unsigned)s < (unsigned)pool.n_seqs) atomicOr(&is_src[s >> 5], 1u << (s & 31));
    if ((unsigned)d < (unsigned)pool.n_seqs && (atomicOr(&is_dst[d >> 5], 1u << (d & 31)) >> (d & 31) & 1u)) s_twice = 1;
  }
  __syncthreads();
  const bool twice = s_twice != 0;
  auto good = [&](int j) {
    const int s = p.src[j], d = p.dst[j], r = p.rows[j];
    if ((unsigned)s >= (unsigned)pool.n_seqs || (unsigned)d >= (unsigned)pool.n_seqs || r < 0 || (long long)r > (long long)P * pool.page_rows) return false;
    if (is_src[d >> 5] >> (d & 31) & 1u) return false;
    if (twice)  // some sequence is the dst of two forks: the first has it
      for (int k = 0; k < j; k++)
        if (p.dst[k] == d) return false;
    return true;
  };
  const int n_free = max(0, min(__ldcg(&pool.state[0]), pool.num_pages));
  int before = 0, copies = 0;  // forks with a page to copy: before fork i, in all
  for (int j0 = 0; j0 < p.n; j0 += COPY_THREADS) {
    const int j = j0 + tid;
    const bool c = j < p.n && p.rows[j] % pool.page_rows != 0 && good(j);
    before += __syncthreads_count(c && j < i);
    copies += __syncthreads_count(c);
  }
  const bool mine = good(i);
  const int rows = mine ? p.rows[i] : 0, part = rows % pool.page_rows, last = rows / pool.page_rows;
  const int s = p.src[i], d = p.dst[i];
  int fresh = -1;
  if (mine && part && before < n_free) {
    fresh = pool.free_list[n_free - 1 - before];
    if ((unsigned)fresh >= (unsigned)pool.num_pages) fresh = -1;
  }
  if (blockIdx.x == 0) {
    int bad = 0;
    if (mine) {
      for (int j = tid; j < P; j += COPY_THREADS) {
        int page = -1;
        if (j < last || (j == last && part)) {
          page = pool.table[(size_t)s * P + j];
          const bool in_pool = (unsigned)page < (unsigned)pool.num_pages;
          if (!in_pool) { page = -1; bad++; }
          if (j < last) {
            if (in_pool) atomicAdd(&pool.ref[page], 1);
          } else {
            page = fresh;
            if (fresh >= 0) pool.ref[fresh] = 1;
          }
        }
        pool.table[(size_t)d * P + j] = page;
      }
    }
    if (p.status) {
      if (bad) { atomicOr(&p.status[0], IQ_STATUS_BAD_PAGE); atomicAdd(&p.status[2], (uint32_t)bad); }
      if (tid == 0 && !mine) { atomicOr(&p.status[0], IQ_STATUS_BAD_SEQUENCE); atomicAdd(&p.status[2], 1u); }
      if (tid == 0 && part && fresh < 0) { atomicOr(&p.status[0], IQ_STATUS_NO_PAGE); atomicAdd(&p.status[2], 1u); }
    }
  } else {
    const int runs = (pool.page_rows + COPY_ROWS - 1) / COPY_ROWS, g = (blockIdx.x - 1) / runs, at = (blockIdx.x - 1 - g * runs) * COPY_ROWS;
    if (fresh >= 0 && at < part) {
      const int from = pool.table[(size_t)s * P + last];
      if ((unsigned)from < (unsigned)pool.num_pages) {
        const size_t in_page = (size_t)g * pool.page_rows + at, page = (size_t)p.n_kv_heads * pool.page_rows;
        copy_rows(p.c, p.row_bytes, from * page + in_page, fresh * page + in_page, min(COPY_ROWS, (part - at + 127) & ~127));
      }
    }
  }
  if (last_to_arrive(pool.state, gridDim.x * gridDim.y) && tid == 0) pool.state[0] = n_free - min(copies, n_free);
}

}  // namespace

cudaError_t launch_keep_rows(const KeepParams& p, int head_dim, int bits, int batch, cudaStream_t stream) {
  void (*k)(KeepParams) = nullptr;
  if (head_dim == 128) k = bits == 2 ? keep_rows_kernel<128, 2> : bits == 3 ? keep_rows_kernel<128, 3> : keep_rows_kernel<128, 4>;
  else k = bits == 2 ? keep_rows_kernel<256, 2> : bits == 3 ? keep_rows_kernel<256, 3> : keep_rows_kernel<256, 4>;
  return launch_after_predecessor(k, dim3(p.pm.n_kv_heads, batch, 2), dim3(KEEP_THREADS), 0, stream, p);
}
cudaError_t launch_reserve_pages(const PoolParams& p, cudaStream_t stream) {
  return launch_after_predecessor(reserve_kernel, dim3(1), dim3(RESERVE_THREADS), 0, stream, p);
}
cudaError_t launch_release_pages(const PoolParams& p, cudaStream_t stream) {
  constexpr int W = RELEASE_THREADS / 32;
  return launch_after_predecessor(release_kernel, dim3((p.n_seqs + W - 1) / W), dim3(RELEASE_THREADS), 0, stream, p);
}
cudaError_t launch_fork_sequences(const CopyParams& p, cudaStream_t stream) {
  const size_t smem = (size_t)((p.pool.n_seqs + 31) / 32) * 8;  // (n_seqs <= 65535: 16 KB)
  return launch_after_predecessor(fork_kernel, dim3(1 + p.n_kv_heads * ((p.pool.page_rows + COPY_ROWS - 1) / COPY_ROWS), p.n), dim3(COPY_THREADS), smem, stream, p);
}
cudaError_t launch_copy_pages(const CopyParams& p, cudaStream_t stream) {
  return launch_after_predecessor(copy_pages_kernel, dim3(p.n_kv_heads * ((p.pool.page_rows + COPY_ROWS - 1) / COPY_ROWS), p.n < 65535 ? p.n : 65535), dim3(COPY_THREADS), 0,
                                  stream, p);
}

}  // namespace iq
