// What a step over requests of any lengths needs besides the cache: the places, positions and cache rows of its tokens, and rotary positions.
#include "iq_common.cuh"

namespace iq {
namespace {

// ---- places of the step's tokens
constexpr int PLAN_THREADS = 256;
// A CTA: the tokens of PLAN_THREADS places. Every CTA adds up the requests' lengths for itself (a thread a run of sequences): the launch
// is bound by its trips to memory one after the other, and a second launch would be two more. 8 requests 2.9 us, 512 requests 3.1.
__global__ void __launch_bounds__(PLAN_THREADS) plan_kernel(const __grid_constant__ PlanParams p) {
  __shared__ long long run_at[PLAN_THREADS];  // tokens before a thread's run of sequences
  __shared__ long long warp_sum[PLAN_THREADS / 32];
  __shared__ uint32_t left_out;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) left_out = 0;
  grid_dependency_wait();
  allow_dependent_launch();
  const int per = (p.batch + PLAN_THREADS - 1) / PLAN_THREADS;
  const int b0 = min(p.batch, tid * per), b1 = min(p.batch, b0 + per);
  long long sum = 0;
  for (int b = b0; b < b1; b++) sum += max(0, p.n_new[b]);
  long long inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(FULL, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) warp_sum[warp] = inc;
  __syncthreads();
  long long before = 0;
  for (int w = 0; w < warp; w++) before += warp_sum[w];
  run_at[tid] = before + inc - sum;
  __syncthreads();
  long long total = 0;
  for (int w = 0; w < PLAN_THREADS / 32; w++) total += warp_sum[w];
  if (blockIdx.x == 0) {
    long long at = run_at[tid];
    for (int b = b0; b < b1; b++) {
      p.token_start[b] = (int32_t)min(at, (long long)p.n_tokens_max);
      at += max(0, p.n_new[b]);
    }
    if (tid == 0) {
      p.token_start[p.batch] = (int32_t)min(total, (long long)p.n_tokens_max);
      if (total > p.n_tokens_max && p.status) {
        atomicOr(&p.status[0], IQ_STATUS_ROW_OUT_OF_RANGE);
        atomicAdd(&p.status[2], (uint32_t)min(total - p.n_tokens_max, 0x7FFFFFFFll));
      }
    }
  }
  const long long i = (long long)blockIdx.x * PLAN_THREADS + tid;
  uint32_t flag = 0;
  if (i < p.n_tokens_max) {
    int position = IQ_NO_POSITION, b = -1;
    long long slot = -1;
    if (i < total) {
      int lo = 0, hi = PLAN_THREADS;  // the last run that starts at or before the token (empty runs start where the next one does)
      while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (run_at[m] <= i) lo = m; else hi = m;
      }
      long long at = run_at[lo];
      for (b = lo * per;; b++) {
        const int n = max(0, p.n_new[b]);
        if (i < at + n) break;
        at += n;
      }
      const long long pos = (long long)p.ctx_lens[b] + (i - at);
      position = (int)min(pos, (long long)INT32_MAX);
      if (p.slots) {
        if (pos < 0 || pos >= p.pm.t_cap) {
          flag = IQ_STATUS_ROW_OUT_OF_RANGE;
        } else if (p.pm.table == nullptr) {
          slot = (long long)b * p.pm.t_cap + pos;
        } else {
          const int j = (int)pos / p.pm.page_rows, page = p.pm.table[(size_t)b * (p.pm.t_cap / p.pm.page_rows) + j];
          if ((unsigned)page >= (unsigned)p.pm.num_pages) flag = IQ_STATUS_BAD_PAGE;
          else slot = (long long)page * p.pm.page_rows + (pos - (long long)j * p.pm.page_rows);
        }
      }
    }
    if (p.positions) p.positions[i] = position;
    if (p.sequences) p.sequences[i] = b;
    if (p.slots) p.slots[i] = slot;
  }
  if (flag) {
    atomicAdd(&left_out, 1u);
    if (p.status) atomicOr(&p.status[0], flag);
  }
  __syncthreads();
  if (tid == 0 && left_out && p.status) atomicAdd(&p.status[2], left_out);
}

// ---- rotary positions
constexpr int ROTARY_THREADS = 256;
constexpr int ROTARY_TOKENS = 16;  // most tokens of a CTA
// A CTA: `tokens` tokens, the angles of each once for all heads. An angle is position times frequency in turns, a 64-bit fraction: the
// product modulo 2^64 is the turn's fraction, exactly, however far the position. A thread takes 16 elements of a head, 8 pairs.
// Bound by memory: 8192 tokens, 64/8 heads of 128: 55.6 us = 5.4 TB/s read and written (one token 2.9). Two tasks of a thread in flight: slower;
// as many threads as fill all rounds: 57.4 us (1000 tokens, 32/8 heads: 6.05 for 6.75); the first elements asked for before the angles are worked out: 60.5 us (2107 tokens, 16/8 heads of 256, a quarter turned: 10.6 for 11.7).
__global__ void __launch_bounds__(ROTARY_THREADS) rotary_kernel(const __grid_constant__ RotaryParams p, int tokens) {
  __shared__ alignas(16) float2 turn[ROTARY_TOKENS * IQ_ROTARY_MAX_PAIRS];  // cosines and sines times the magnitude, [token][pair]; read two at a time
  __shared__ int position[ROTARY_TOKENS];
  const int tid = threadIdx.x, pairs = p.rotary.rotary_dim / 2;
  const int first = blockIdx.x * tokens, n = min(tokens, p.n_tokens - first);
  grid_dependency_wait();
  allow_dependent_launch();
  for (int i = tid; i < n * pairs; i += ROTARY_THREADS) {
    const int t = i / pairs, k = i - t * pairs, pos = p.positions[first + t];
    if (k == 0) position[t] = pos;
    const uint64_t x = (uint64_t)(int64_t)pos * p.rotary.turns[k];
    float sn, cs;
    sincospif((float)(int32_t)(x >> 32) * 4.656612873077393e-10f, &sn, &cs);  // 2^-31: half turns
    turn[t * pairs + k] = make_float2(cs * p.rotary.magnitude, sn * p.rotary.magnitude);
  }
  __syncthreads();
  const int per_head = p.head_dim / 16, turned = p.rotary.rotary_dim / 16;
  const int heads = p.side[0].heads + p.side[1].heads, per_token = heads * per_head;
  for (int i = tid; i < n * per_token; i += ROTARY_THREADS) {
    const int t = i / per_token, r = i - t * per_token, h0 = r / per_head, v = r - h0 * per_head;
    if (position[t] == IQ_NO_POSITION) continue;
    const int sd = h0 >= p.side[0].heads ? 1 : 0, h = h0 - (sd ? p.side[0].heads : 0);
    const RotarySide& s = p.side[sd];
    const __half* const x = s.x + (first + t) * s.xs_t + h * s.xs_h;
    __half* const y = s.y + (first + t) * s.ys_t + h * s.ys_h;
    if (v >= turned) {  // the rest of the head
      if (x != y) {
        const uint4 a = *reinterpret_cast<const uint4*>(x + 16 * v), b = *reinterpret_cast<const uint4*>(x + 16 * v + 8);
        *reinterpret_cast<uint4*>(y + 16 * v) = a;
        *reinterpret_cast<uint4*>(y + 16 * v + 8) = b;
      }
      continue;
    }
    // elements a and b of the two vectors; halves: pair k = (a_k, b_k), interleaved: pairs of neighbours
    const int at0 = p.rotary.interleaved ? 16 * v : 8 * v, at1 = p.rotary.interleaved ? 16 * v + 8 : pairs + 8 * v;
    uint4 a = *reinterpret_cast<const uint4*>(x + at0), b = *reinterpret_cast<const uint4*>(x + at1);
    const float4* const cs = reinterpret_cast<const float4*>(turn + t * pairs + 8 * v);
    uint32_t* const aw = reinterpret_cast<uint32_t*>(&a);
    uint32_t* const bw = reinterpret_cast<uint32_t*>(&b);
    auto rotate = [](float u, float w, float c, float sn, float& u1, float& w1) {
      u1 = fmaf(u, c, -(w * sn));
      w1 = fmaf(u, sn, w * c);
    };
    if (p.rotary.interleaved) {
#pragma unroll
      for (int k = 0; k < 4; k++) {
        const float4 f = cs[k];
        uint32_t& w0 = k < 2 ? aw[2 * k] : bw[2 * k - 4];
        uint32_t& w1 = k < 2 ? aw[2 * k + 1] : bw[2 * k - 3];
        const float2 p0 = __half22float2(*reinterpret_cast<const __half2*>(&w0)), p1 = __half22float2(*reinterpret_cast<const __half2*>(&w1));
        float u0, u1, v0, v1;
        rotate(p0.x, p0.y, f.x, f.y, u0, u1);
        rotate(p1.x, p1.y, f.z, f.w, v0, v1);
        w0 = pack_half2(u0, u1);
        w1 = pack_half2(v0, v1);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; k++) {
        const float4 f = cs[k];
        const float2 u = __half22float2(*reinterpret_cast<const __half2*>(&aw[k])), w = __half22float2(*reinterpret_cast<const __half2*>(&bw[k]));
        float u0, u1, w0, w1;
        rotate(u.x, w.x, f.x, f.y, u0, w0);
        rotate(u.y, w.y, f.z, f.w, u1, w1);
        aw[k] = pack_half2(u0, u1);
        bw[k] = pack_half2(w0, w1);
      }
    }
    *reinterpret_cast<uint4*>(y + at0) = a;
    *reinterpret_cast<uint4*>(y + at1) = b;
  }
}

}  // namespace

cudaError_t launch_plan_tokens(const PlanParams& p, cudaStream_t stream) {
  return launch_after_predecessor(plan_kernel, dim3((unsigned)max(1ll, ((long long)p.n_tokens_max + PLAN_THREADS - 1) / PLAN_THREADS)), dim3(PLAN_THREADS), 0, stream, p);
}

cudaError_t launch_apply_rotary(const RotaryParams& p, cudaStream_t stream) {
  // about two rounds of a CTA's threads
  const int tasks = (p.side[0].heads + p.side[1].heads) * (p.head_dim / 16);
  const int tokens = min(ROTARY_TOKENS, max(1, 2 * ROTARY_THREADS / tasks));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.n_tokens - 1) / tokens + 1));
  cfg.blockDim = dim3(ROTARY_THREADS);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, rotary_kernel, p, tokens);
}

}  // namespace iq
