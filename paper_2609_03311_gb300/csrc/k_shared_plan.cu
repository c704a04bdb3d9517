// k_shared_plan.cu -- the split of a step's attention over the paged cache (dopr_shared_attention_plan), from offsets,
// lengths and prefixes on the device.
//
// One CTA: everything is sums over the step's rows, and the rows of a prefix brought together.  Rows usually come in
// prefix order; those that do not are sorted (a bitonic network over (prefix, row) in shared memory; rows of a
// prefix keep their order).  Bound by latency; made once a step and used by every layer.
#include <limits.h>

#include "shared_attn.cuh"

namespace dopr {
namespace {
using namespace shared_attn;

constexpr int THREADS = 1024;
constexpr int ROW_BITS = 14;
static_assert(CACHE_MAX_SEQS == 1 << ROW_BITS, "a sort key holds two row numbers");

// Exclusive sums over the block's threads in order; the block's total through `total`.
template <typename T>
__device__ T block_exclusive(T v, T* warp_sum, T& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  T inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T u = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += u;
  }
  __syncthreads();  // the last use of warp_sum is over
  if (lane == 31) warp_sum[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    T w = warp_sum[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T u = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += u;
    }
    warp_sum[lane] = w;
  }
  __syncthreads();
  total = warp_sum[31];
  return (warp > 0 ? warp_sum[warp - 1] : T(0)) + inc - v;
}

__global__ void __launch_bounds__(THREADS) k_shared_plan(SharedPlanArgs a, int n_ctas) {
  extern __shared__ uint32_t keys[];  // a power of two >= n_seqs
  __shared__ unsigned long long warp_sum[32];
  __shared__ int bad, unsorted;
  const int n = a.lay.n_seqs, Hkv = a.lay.n_kv_heads, G = a.Hq / Hkv, page = a.lay.page, page_blk = BLOCK / page;
  const int tile = tokens_a_tile(G), pair = 2 * tile;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t cap = static_cast<int64_t>(a.lay.max_blocks) * page;
  const Plan p = plan_view(a.plan, n, Hkv, G, a.max_tokens);
  int* sorted = p.scratch;          // rows with tokens, by group: their prefix, n where there are no prefix keys
  int* place = sorted + n;          // of a sorted entry: tokens of the entries before it
  int* group_of = place + n + 1;    // of a sorted entry
  int* group = group_of + n;        // of a group: tokens before its first
  int* group_item = group + n + 1;  // of a group: its first item
  if (threadIdx.x == 0) bad = 0, unsorted = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  Head head{};
  head.share = 1;
  head.n_seqs = n;
  head.n_kv_heads = Hkv;
  head.Hq = a.Hq;
  head.max_tokens = a.max_tokens;
  head.n_ctas = n_ctas;
  head.head_dim = a.lay.head_dim;
  head.page = page;
  auto tokens_of = [&](int i) { return a.tok_off[i + 1] - a.tok_off[i]; };

  // checks, and the rows with tokens
  unsigned long long total;
  int ns = 0;
  for (int i0 = 0; i0 < n; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    bool has = false;
    int g = n;
    if (i < n) {
      const int t0 = a.tok_off[i], t1 = a.tok_off[i + 1], pre = a.prefix ? a.prefix[i] : -1, len = a.seq_lens[i];
      if ((i == 0 && t0 != 0) || t1 < t0 || t1 > a.max_tokens || len < 0 || len > cap || pre < -1 || pre >= n || pre == i ||
          (pre >= 0 && a.prefix[pre] != -1))
        bad = 1;
      else
        has = t1 > t0;
      if (has && pre >= 0 && a.seq_lens[pre] > 0) g = pre;
    }
    const int at = ns + static_cast<int>(block_exclusive(static_cast<unsigned long long>(has), warp_sum, total));
    if (has) sorted[at] = i, group_of[at] = g;
    ns += static_cast<int>(total);
  }
  __syncthreads();
  if (bad) {
    if (threadIdx.x == 0) {
      *p.head = head;
      if (a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);
    }
    for (int c = threadIdx.x; c < MAX_CTAS; c += THREADS) p.first[c] = 0;
    return;
  }
  for (int i = threadIdx.x + 1; i < ns; i += THREADS)
    if (group_of[i] < group_of[i - 1]) unsorted = 1;
  __syncthreads();
  if (unsorted) {
    int m = 2;
    while (m < ns) m <<= 1;
    for (int i = threadIdx.x; i < m; i += THREADS)
      keys[i] = i < ns ? static_cast<uint32_t>(group_of[i]) << ROW_BITS | sorted[i] : 0xffffffffu;
    for (int k = 2; k <= m; k <<= 1)
      for (int j = k >> 1; j > 0; j >>= 1) {
        __syncthreads();
        for (int i = threadIdx.x; i < m; i += THREADS) {
          const int o = i ^ j;
          if (o > i) {
            const uint32_t x = keys[i], y = keys[o];
            if ((x > y) == ((i & k) == 0)) keys[i] = y, keys[o] = x;
          }
        }
      }
    __syncthreads();
    for (int i = threadIdx.x; i < ns; i += THREADS) sorted[i] = keys[i] & ((1 << ROW_BITS) - 1), group_of[i] = keys[i] >> ROW_BITS;
    __syncthreads();
  }
  int carry = 0;
  for (int i0 = 0; i0 < ns; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    const int tok = i < ns ? tokens_of(sorted[i]) : 0;
    const int at = carry + static_cast<int>(block_exclusive(static_cast<unsigned long long>(tok), warp_sum, total));
    if (i < ns) {
      place[i] = at;
      if (i == 0 || group_of[i - 1] != group_of[i]) group[group_of[i]] = at;
    }
    carry += static_cast<int>(total);
  }
  if (threadIdx.x == 0) place[ns] = carry;
  __syncthreads();

  // items, written by the last row of each group
  int n_items = 0;
  for (int i0 = 0; i0 < ns; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    const int g = i < ns ? group_of[i] : 0;
    int count = 0, tok = 0;
    if (i < ns && (i + 1 == ns || group_of[i + 1] != g)) {
      tok = place[i + 1] - group[g];
      count = (tok + pair - 1) / pair;
    }
    const int at = n_items + static_cast<int>(block_exclusive(static_cast<unsigned long long>(count), warp_sum, total));
    if (count > 0) group_item[g] = at;
    for (int c = 0; c < count; ++c) {
      Item it{};
      it.tok = group[g] + c * pair;
      it.n_tok = min(pair, tok - c * pair);
      it.prefix_keys = g < n ? a.seq_lens[g] : 0;
      p.items[at + c] = it;
    }
    n_items += static_cast<int>(total);
  }
  __syncthreads();

  // runs, by their rows: a row writes its own run in each item that has tokens of it, and the prefix's in each item
  // that begins with it
  int n_runs = 0;
  for (int i0 = 0; i0 < ns; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    int in = 0, tok = 0, k0 = 0, k1 = -1, begun = 0, g = 0;
    if (i < ns) {
      g = group_of[i];
      in = place[i] - group[g];
      tok = place[i + 1] - place[i];
      k0 = in / pair;
      k1 = (in + tok - 1) / pair;
      begun = k1 - (in + pair - 1) / pair + 1;  // items whose first token is one of the row's
    }
    const int count = k1 - k0 + 1 + (g < n ? begun : 0);
    int at = n_runs + static_cast<int>(block_exclusive(static_cast<unsigned long long>(count), warp_sum, total));
    for (int k = k0; k <= k1; ++k) {
      Item& it = p.items[group_item[g] + k];
      const int lo = max(in, k * pair), hi = min(in + tok, (k + 1) * pair);  // places in the group
      if (lo == k * pair) {
        it.run = at;
        if (g < n) {
          const int keys_ = a.seq_lens[g];
          p.runs[at++] = Run{g, 0, (keys_ + page - 1) / page, keys_, 0, it.n_tok, -1, 0};
        }
      }
      const int row = sorted[i], len = a.seq_lens[row];
      const int seen = max(0, len - (in + tok - hi));  // own keys of its last token here: each token behind it sees one more
      p.runs[at++] = Run{row, 0, (seen + page - 1) / page, seen, lo - k * pair, hi - k * pair, a.tok_off[row] + lo - in, 0};
    }
    n_runs += static_cast<int>(total);
  }
  __syncthreads();

  // a warp an item: where its runs' pages begin, and the tokens' records
  for (int k = warp; k < n_items; k += THREADS / 32) {
    Item it = p.items[k];
    it.n_runs = (k + 1 < n_items ? p.items[k + 1].run : n_runs) - it.run;
    int pages = 0, end0 = 0, begin1 = INT_MAX;
    for (int r0 = 0; r0 < it.n_runs; r0 += 32) {
      const int r = r0 + lane;
      Run run{};
      if (r < it.n_runs) run = p.runs[it.run + r];
      int inc = run.pages;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += u;
      }
      const int off = pages + inc - run.pages;
      if (r < it.n_runs) {
        p.runs[it.run + r].off = off;
        if (run.tok0 < tile) end0 = max(end0, off + run.pages);
        if (run.token >= 0 && run.tok1 > tile) begin1 = min(begin1, off);
        const int seen1 = run.keys - (run.tok1 - run.tok0);  // + 1 for the first token, and so on
        for (int x = run.tok0; run.token >= 0 && x < run.tok1; ++x) {
          const int t = run.token + x - run.tok0;
          p.order[it.tok + x] = t;
          // a row with more new tokens than keys: its first tokens see none, however many those of its last are
          const int own = max(0, run.keys > 0 ? seen1 + x - run.tok0 + 1 : 0);
          p.rec[t] = make_int4(k, x, off * page, own);
          p.own[it.tok + x] = make_int2(off * page, off * page + own);
        }
      }
      pages += __shfl_sync(0xffffffffu, inc, 31);
    }
    end0 = __reduce_max_sync(0xffffffffu, end0);
    begin1 = __reduce_min_sync(0xffffffffu, begin1);
    if (lane == 0) {
      it.pages = pages;
      it.blocks = (pages + page_blk - 1) / page_blk;
      it.end0 = (end0 + page_blk - 1) / page_blk;
      it.prefix_blocks = ((it.prefix_keys + page - 1) / page + page_blk - 1) / page_blk;
      it.begin1 = begin1 / page_blk;
      p.items[k] = it;
    }
  }
  __syncthreads();

  // the line
  unsigned long long line = 0;
  for (int i0 = 0; i0 < n_items; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    const uint32_t blocks = i < n_items ? p.items[i].blocks : 0;
    const unsigned long long cost = blocks > 0 ? static_cast<unsigned long long>(Hkv) * (blocks + OVERHEAD) : 0;
    const unsigned long long at = line + block_exclusive(cost, warp_sum, total);
    if (i < n_items) p.items[i].cost = static_cast<uint32_t>(at);
    line += total;
  }
  const bool fits = line < 0x80000000ull;
  const uint32_t share = fits ? max(1u, static_cast<uint32_t>((line + n_ctas - 1) / n_ctas)) : 1;
  const int n_flat = n_items * Hkv;
  for (int c = threadIdx.x; c < MAX_CTAS; c += THREADS) p.first[c] = n_flat;
  if (threadIdx.x == 0) {
    if (fits) {
      head.tokens = a.tok_off[n];
      head.n_items = n_items;
      head.n_flat = n_flat;
      head.share = share;
      head.total = static_cast<uint32_t>(line);
    }
    *p.head = head;
    if (!fits && a.status) atomicCAS(a.status, 0, DOPR_ERR_UNSUPPORTED);
  }
  __syncthreads();
  if (!fits) return;
  unsigned long long rows = 0;  // of partial results; in the upper half pieces of the join's list
  for (int f0 = 0; f0 < n_flat; f0 += THREADS) {
    const int f = f0 + threadIdx.x;
    unsigned long long count = 0;
    int entry_rows = 0;
    if (f < n_flat) {
      const Item it = p.items[f / Hkv];
      const bool two = two_tiles(it.n_tok, G);
      uint32_t segs = 0;
      if (it.blocks > 0) {
        const uint32_t b = blocks_begin(it, f % Hkv), e = b + it.blocks, start = b - OVERHEAD;
        segs = (e - 1) / share - b / share + 1;
        for (uint32_t c = (start + share - 1) / share; static_cast<unsigned long long>(c) * share < e; ++c)
          if (c < MAX_CTAS) p.first[c] = f;
      }
      if (!two || segs != 1) {  // also where there is no key at all
        entry_rows = it.n_tok * G;
        count = static_cast<unsigned long long>(segs) * entry_rows * (two ? 1 : 2) |
                static_cast<unsigned long long>((entry_rows + JOIN_ROWS - 1) / JOIN_ROWS) << 32;
      }
    }
    const unsigned long long at = rows + block_exclusive(count, warp_sum, total);
    if (f < n_flat) p.part[f] = static_cast<uint32_t>(at);
    for (int r = 0; r < entry_rows; r += JOIN_ROWS) p.join[(at >> 32) + r / JOIN_ROWS] = make_int2(f, r);
    rows += total;
  }
  if (threadIdx.x == 0) p.head->n_join = static_cast<int>(rows >> 32);
}

}  // namespace

int64_t shared_plan_bytes(const dopr_cache_layout& lay, int Hq, int max_tokens) {
  return plan_view(nullptr, lay.n_seqs, lay.n_kv_heads, Hq / lay.n_kv_heads, max_tokens).bytes;
}

cudaError_t launch_shared_plan(const SharedPlanArgs& a, int num_sms, cudaStream_t st) {
  int keys = 2;
  while (keys < a.lay.n_seqs) keys <<= 1;
  static_assert(CACHE_MAX_SEQS * 4 <= 65536, "shared memory of the sort");
  const cudaError_t e = cudaFuncSetAttribute(k_shared_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, 65536);
  if (e != cudaSuccess) return e;
  return launch_dependent(k_shared_plan, dim3(1), THREADS, keys * 4, st, a, num_sms < MAX_CTAS ? num_sms : MAX_CTAS);
}

}  // namespace dopr
