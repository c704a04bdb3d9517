// k_cache.cu -- block tables, slots and positions of a step's new tokens, from lengths on the device
// (dopr_cache_extend).
//
// Row i holds len_i tokens and gets new_i: it needs ceil((len_i + new_i) / page) - ceil(len_i / page) new pages,
// which rows take from the top of a stack in row order, so that exclusive sums over the rows of new tokens and of
// needed pages say where each row's tokens lie in the packed order and which stack entries are its own.  Everything
// else follows for each token by itself: row (a search in the offsets), place, page, slot, position.
//
// Bound by latency: 2,000 rows are 24 KB of lengths and a chunk of 75,000 tokens 0.9 MB of results.  One CTA takes
// the sums; up to FILL_HERE tokens it writes the results too, beyond that a dependent launch over the whole device
// does (a store of 12 bytes a token by one SM takes about 1 us per 4,000 tokens, another launch about 1.5).
#include "device_common.cuh"
#include "internal.h"

namespace dopr {
namespace {

constexpr int FILL_THREADS = 256;
constexpr int FILL_HERE = 4096;
constexpr int FEW_THREADS = 128, MANY_THREADS = 1024;  // of the CTA that takes the sums

// Workspace header: the stack's height once released pages are back, new tokens (0 where the call does not go ahead).
enum { WS_TOP = 0, WS_TOKENS = 1 };

__device__ __forceinline__ void set_status(int32_t* status, int code) {
  if (status) atomicCAS(status, 0, code);
}
__device__ __forceinline__ int pages_of(int64_t n, int page) { return static_cast<int>((n + page - 1) / page); }

struct Sums {
  int64_t tokens;
  int64_t pages;
};
__device__ __forceinline__ Sums shfl_up(Sums v, int o) {
  v.tokens = __shfl_up_sync(0xffffffffu, v.tokens, o);
  v.pages = __shfl_up_sync(0xffffffffu, v.pages, o);
  return v;
}
// Exclusive sums over the block's threads in order; the block's totals through `total`.
template <int WARPS>
__device__ Sums block_exclusive(Sums v, Sums* warp_sum, Sums& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sums inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Sums u = shfl_up(inc, o);
    if (lane >= o) inc.tokens += u.tokens, inc.pages += u.pages;
  }
  __syncthreads();  // the last use of warp_sum is over
  if (lane == 31) warp_sum[warp] = inc;
  __syncthreads();
  Sums base{0, 0};
  if constexpr (WARPS <= 8) {
    total = Sums{0, 0};
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      if (w == warp) base = total;
      total.tokens += warp_sum[w].tokens, total.pages += warp_sum[w].pages;
    }
  } else {
    if (warp == 0) {
      Sums w = warp_sum[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const Sums u = shfl_up(w, o);
        if (lane >= o) w.tokens += u.tokens, w.pages += u.pages;
      }
      warp_sum[lane] = w;
    }
    __syncthreads();
    total = warp_sum[WARPS - 1];
    if (warp > 0) base = warp_sum[warp - 1];
  }
  return Sums{base.tokens + inc.tokens - v.tokens, base.pages + inc.pages - v.pages};
}

// Slot, position and, for the first token of a new page, table entry of token t.  off: the rows' offsets, of which
// rows [lo, hi] hold t.
__device__ void fill_token(const CacheExtendArgs& a, int t, const int32_t* off, int lo, int hi, int top) {
  while (lo < hi) {  // the last row whose offset is <= t: rows without tokens before it share the offset
    const int mid = (lo + hi + 1) >> 1;
    if (off[mid] <= t) lo = mid; else hi = mid - 1;
  }
  const int32_t* held = a.ws + CACHE_WS_HEAD;
  const int32_t* base = held + a.lay.n_seqs;
  const int32_t* first = base + a.lay.n_seqs;
  const int page = a.lay.page;
  const int at = held[lo] + t - off[lo], p = at / page, had = pages_of(held[lo], page);
  int32_t* entry = a.tables + static_cast<int64_t>(lo) * a.lay.max_blocks + p;
  // stack entries are read below `top` only: the sums checked that the needed pages are there
  const int block = p < had ? *entry : a.free_blocks[top - 1 - (first[lo] + p - had)];
  const bool good = block >= 0 && block < a.lay.n_blocks;
  if (!good) set_status(a.status, DOPR_ERR_INVALID_ARG);
  if (p >= had && at % page == 0) *entry = block;
  a.slots[t] = good ? static_cast<int64_t>(block) * page + at % page : -1;
  a.positions[t] = base[lo] + at;
}

template <int SUM_THREADS>
__global__ void __launch_bounds__(SUM_THREADS) k_cache_sums(CacheExtendArgs a, bool fill) {
  constexpr int WARPS = SUM_THREADS / 32;
  __shared__ Sums warp_sum[WARPS];
  __shared__ int2 gone_rows[SUM_THREADS];  // a released row, where its pages go on the stack
  __shared__ int bad;  // the error to be stored
  __shared__ int64_t released;
  const int n = a.lay.n_seqs, page = a.lay.page;
  const int64_t cap = static_cast<int64_t>(a.lay.max_blocks) * page;
  int32_t* held = a.ws + CACHE_WS_HEAD;
  int32_t* base = held + n;
  int32_t* first = base + n;
  if (threadIdx.x == 0) bad = 0, released = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();

  // the sums; a row's length, its prefix's and its place among the needed pages stay in the workspace, since the
  // outputs may be the inputs
  Sums carry{0, 0};
  int64_t my_released = 0;
  bool my_bad = false;
  for (int i0 = 0; i0 < n; i0 += SUM_THREADS) {
    const int i = i0 + threadIdx.x;
    Sums v{0, 0};
    int len = 0, b = 0;
    if (i < n) {
      len = a.seq_lens[i];
      const int add = a.new_lens[i], pre = a.prefix ? a.prefix[i] : -1;
      if (len < 0 || len > cap || add < -1 || (add > 0 && len + static_cast<int64_t>(add) > cap) || pre < -1 ||
          pre >= n || pre == i || (pre >= 0 && a.prefix[pre] != -1)) {
        my_bad = true;
      } else if (add < 0) {
        my_released += pages_of(len, page);
      } else {
        v.tokens = add;
        v.pages = pages_of(static_cast<int64_t>(len) + add, page) - pages_of(len, page);
        if (pre >= 0) {
          const int pl = a.seq_lens[pre], pa = a.new_lens[pre];
          const int64_t now = pa < 0 ? 0 : static_cast<int64_t>(pl) + pa;
          my_bad |= now < 0 || now + len + add > INT32_MAX;
          b = static_cast<int>(now);
        }
      }
    }
    Sums total;
    const Sums ex = block_exclusive<WARPS>(v, warp_sum, total);
    if (i < n) {
      held[i] = len;
      base[i] = b;
      a.tok_off[i] = static_cast<int32_t>(carry.tokens + ex.tokens);
      first[i] = static_cast<int32_t>(carry.pages + ex.pages);
    }
    carry.tokens += total.tokens;
    carry.pages += total.pages;
  }
  if (my_bad) atomicExch(&bad, DOPR_ERR_INVALID_ARG);
  if (my_released) atomicAdd(reinterpret_cast<unsigned long long*>(&released), static_cast<unsigned long long>(my_released));
  __syncthreads();
  const int64_t stack = *a.n_free, top = stack + released;
  int err = bad;
  if (!err && (carry.tokens > a.max_tokens || stack < 0 || top > a.lay.n_blocks)) err = DOPR_ERR_INVALID_ARG;
  if (!err && carry.pages > top) err = DOPR_ERR_OUT_OF_MEMORY;
  __syncthreads();  // everyone has read the stack's height, which n_free_out may be
  if (err) {
    for (int i = threadIdx.x; i < n; i += SUM_THREADS) a.tok_off[i] = 0;
    carry = Sums{0, 0};
    if (threadIdx.x == 0) bad = err;
  }
  if (threadIdx.x == 0) {
    a.tok_off[n] = static_cast<int32_t>(carry.tokens);
    a.ws[WS_TOP] = static_cast<int32_t>(top);
    a.ws[WS_TOKENS] = static_cast<int32_t>(carry.tokens);
    *a.n_free_out = static_cast<int32_t>(err ? stack : top - carry.pages);
  }
  if (!err && released > 0) {
    // pages of released rows onto the stack, in row and page order: their place is a sum over the rows again
    int64_t at = stack;
    for (int i0 = 0; i0 < n; i0 += SUM_THREADS) {
      const int i = i0 + threadIdx.x;
      const bool gone = i < n && a.new_lens[i] < 0;
      Sums total;
      const Sums ex = block_exclusive<WARPS>(Sums{gone ? 1 : 0, gone ? pages_of(held[i], page) : 0}, warp_sum, total);
      if (gone) gone_rows[ex.tokens] = make_int2(i, static_cast<int>(at + ex.pages));
      __syncthreads();
      for (int g = threadIdx.x >> 5; g < total.tokens; g += WARPS) {  // a warp a row
        const int2 it = gone_rows[g];
        const int np = pages_of(held[it.x], page);
        for (int p = threadIdx.x & 31; p < np; p += 32) {
          const int block = a.tables[static_cast<int64_t>(it.x) * a.lay.max_blocks + p];
          if (static_cast<uint32_t>(block) >= static_cast<uint32_t>(a.lay.n_blocks)) bad = DOPR_ERR_INVALID_ARG;
          a.free_blocks[it.y + p] = block;
        }
      }
      at += total.pages;
    }
  }
  for (int i = threadIdx.x; i < n; i += SUM_THREADS)
    a.seq_lens_out[i] = err ? held[i] : a.new_lens[i] < 0 ? 0 : held[i] + a.new_lens[i];
  __syncthreads();  // offsets, workspace and stack are written
  // (stored here for all errors: a second place cost 2,000 rows 0.3 us)
  if (threadIdx.x == 0 && bad) set_status(a.status, bad);
  if (!fill) return;
  for (int t = threadIdx.x; t < a.max_tokens; t += SUM_THREADS) {
    if (t < carry.tokens) {
      fill_token(a, t, a.tok_off, 0, n - 1, static_cast<int>(top));
    } else {
      a.slots[t] = -1;
      a.positions[t] = -1;
    }
  }
}

__global__ void __launch_bounds__(FILL_THREADS) k_cache_fill(CacheExtendArgs a) {
  static_assert((CACHE_MAX_SEQS + FILL_THREADS - 1) / FILL_THREADS <= FILL_THREADS, "two counts find a row");
  const int t0 = blockIdx.x * FILL_THREADS, t = t0 + threadIdx.x, n = a.lay.n_seqs;
  pdl_wait();
  pdl_trigger();
  const int tokens = a.ws[WS_TOKENS], top = a.ws[WS_TOP];
  // the rows of the block's first and last token bound every thread's search: all threads look at every step-th offset, then
  // at those between (one thread halving the range: 11 loads one after another for 2,000 rows)
  int rows[2] = {0, 0};
  if (t0 < tokens) {
    const int x0 = t0, x1 = t0 + min(FILL_THREADS, tokens - t0) - 1, step = (n + FILL_THREADS - 1) / FILL_THREADS;
    const int i = threadIdx.x * step, v = i < n ? a.tok_off[i] : INT32_MAX;
    rows[0] = (__syncthreads_count(v <= x0) - 1) * step;
    rows[1] = (__syncthreads_count(v <= x1) - 1) * step;
    const bool in = static_cast<int>(threadIdx.x) < step;
    const int i0 = rows[0] + threadIdx.x, i1 = rows[1] + threadIdx.x;
    const int v0 = in && i0 < n ? a.tok_off[i0] : INT32_MAX, v1 = in && i1 < n ? a.tok_off[i1] : INT32_MAX;
    rows[0] += __syncthreads_count(v0 <= x0) - 1;
    rows[1] += __syncthreads_count(v1 <= x1) - 1;
  }
  if (t >= a.max_tokens) return;
  if (t < tokens) {
    fill_token(a, t, a.tok_off, rows[0], rows[1], top);
  } else {
    a.slots[t] = -1;
    a.positions[t] = -1;
  }
}

}  // namespace

cudaError_t launch_cache_extend(const CacheExtendArgs& a, cudaStream_t st) {
  const bool here = a.max_tokens <= FILL_HERE;
  // a few rows need few threads, whose barriers are shorter
  const bool few = a.lay.n_seqs <= FEW_THREADS && a.max_tokens <= 4 * FEW_THREADS;
  const cudaError_t e = few ? launch_dependent(k_cache_sums<FEW_THREADS>, dim3(1), FEW_THREADS, 0, st, a, here)
                            : launch_dependent(k_cache_sums<MANY_THREADS>, dim3(1), MANY_THREADS, 0, st, a, here);
  if (e != cudaSuccess || here) return e;
  return launch_dependent(k_cache_fill, dim3((a.max_tokens - 1) / FILL_THREADS + 1), FILL_THREADS, 0, st, a);
}

}  // namespace dopr
