// k_shared_plan.cu -- the split of a step's attention over the paged cache (dopr_shared_attention_plan), from offsets,
// lengths and prefixes on the device.
//
// One CTA: everything is sums over the step's rows, and the rows of a prefix brought together.  Rows usually come in
// prefix order; those that do not are sorted (a bitonic network over (prefix, row) in shared memory; rows of a
// prefix keep their order).  Made once a step and used by every layer.  Bound by the latency of some twenty short phases:
// lists, items and runs stay in shared memory where they fit, a sum over the block takes one barrier and two counts where
// they fit, and what rows, items and entries hold several of (items, runs, tokens, segments) is spread over a warp's lanes.
// 512 threads: 12 us for one token, 18 for 64 queries of one document, 24 for 256 of 64 documents, 32 for 6,784 tokens of 200
// queries.  (As it was then, 1024 threads to 512 to 256: 12.1, 10.9, 10.7; 15.7, 14.1, 13.6; 20.8, 20.9, 25.9; 26.4, 28.7, 37.5:
// a barrier and a sum cost more the more warps there are.)
#include <limits.h>

#include "shared_attn.cuh"

namespace dopr {
namespace {
using namespace shared_attn;

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int ROW_BITS = 14;
constexpr int MAX_SHARED = 200 * 1024;
static_assert(CACHE_MAX_SEQS == 1 << ROW_BITS, "a sort key holds two row numbers");
static_assert(CACHE_MAX_SEQS * 4 <= MAX_SHARED, "the sort's keys");
enum { LISTS_SHARED = 1, ITEMS_SHARED = 2, RUNS_SHARED = 4 };

__device__ int warp_inclusive(int v) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) >= o) v += u;
  }
  return v;
}

// Exclusive sums over the block's threads in order, of which the first `count` have values; x: a thread's sum, y: all.  One
// barrier: the warps' sums lie in one of two places by turns, and who writes one has passed the barrier behind its last
// readers.  Warps without values only add up the others' sums.
__device__ __noinline__ int2 block_sum(int v, int count, int* sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool any = warp * 32 < count;
  int inc = any ? warp_inclusive(v) : 0;
  if (lane == 31) sums[warp] = inc;
  __syncthreads();
  const int w = sums[lane];
  if (any) inc += __reduce_add_sync(0xffffffffu, lane < warp ? w : 0) - v;
  return make_int2(inc, __reduce_add_sync(0xffffffffu, w));
}

// Division by a number that stays: m is 2^32 / d or up to one less, so the product's upper half is the quotient or one less.
struct Divisor {
  uint32_t d, m;
  __device__ explicit Divisor(uint32_t divisor) : d(divisor), m(divisor ? 0xffffffffu / divisor : 0) {}
  __device__ uint32_t of(uint32_t x) const {
    const uint32_t q = __umulhi(x, m);
    return x - q * d >= d ? q + 1 : q;
  }
};

// f(whether there is one, lane, i) for i below each lane's count, 32 at a time over the warp's lanes.
template <typename F>
__device__ void spread(int count, F f) {
  const int inc = warp_inclusive(count), total = __shfl_sync(0xffffffffu, inc, 31);
#pragma unroll 1
  for (int s = threadIdx.x & 31; s < (total + 31) / 32 * 32; s += 32) {
    int src = 0;  // lanes whose counts end at or before s
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (__shfl_sync(0xffffffffu, inc, src + o - 1) <= s) src += o;
    f(s < total, src, s - __shfl_sync(0xffffffffu, inc - count, src));
  }
}
__device__ __forceinline__ int of_lane(int v, int src) { return __shfl_sync(0xffffffffu, v, src); }

// Ascending; m, a power of two, 32 at least.  Steps within 32 keys by shuffles; the warps that have keys meet for the others.
__device__ void sort_keys(uint32_t* keys, int m) {
  const int threads = min(m, THREADS), tid = threadIdx.x;
  if (tid >= threads) return;
#pragma unroll 1
  for (int k = 2; k <= m; k <<= 1) {
    int j = k >> 1;
#pragma unroll 1
    for (; j >= 32; j >>= 1) {
#pragma unroll 1
      for (int i = tid; i < m; i += threads) {
        const int o = i ^ j;
        if (o > i) {
          const uint32_t x = keys[i], y = keys[o];
          if ((x > y) == ((i & k) == 0)) keys[i] = y, keys[o] = x;
        }
      }
      asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory");
    }
#pragma unroll 1
    for (int i = tid; i < m; i += threads) {
      uint32_t x = keys[i];
#pragma unroll 1
      for (int l = j; l > 0; l >>= 1) {
        const uint32_t y = __shfl_xor_sync(0xffffffffu, x, l);
        x = ((i & l) == 0) == ((i & k) == 0) ? min(x, y) : max(x, y);
      }
      keys[i] = x;
    }
    if (k >= 32) asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory");
  }
}

// Runs that a row has in the items before the c-th of those with tokens of it: one each if it has its own, and the prefix's in
// each that begins with it (all but the first, and that too where `first` says so).
__device__ __forceinline__ int run_before(int c, bool first, bool own, bool prefix) {
  return (own ? c : 0) + (prefix && c > 0 ? c - !first : 0);
}

__global__ void __launch_bounds__(THREADS) k_shared_plan(SharedPlanArgs a, Plan p, int n_ctas, int n_keys, int in_shared) {
  extern __shared__ __align__(16) uint32_t keys[];  // a power of two >= n_seqs, then what in_shared says
  __shared__ int sums_memory[2][32];
  __shared__ int first_of[SHARES];
  __shared__ int bad, unsorted, too_long;
  __shared__ unsigned long long lines[WARPS], tiles_line, both_lines;
  __shared__ int first_few;
  __shared__ uint32_t longest[2];  // entry of tiles, of few items
  const int n = a.lay.n_seqs, Hkv = a.lay.n_kv_heads, G = a.Hq / Hkv, page = a.lay.page, page_blk = BLOCK / page;
  const int tile = tokens_a_tile(G), few = tokens_a_few(G);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t cap = static_cast<int64_t>(a.lay.max_blocks) * page;
  uint8_t* at_shared = reinterpret_cast<uint8_t*>(keys + n_keys);
  auto shared = [&](int what, auto* global, int64_t count) {
    if (!(in_shared & what)) return global;
    auto* q = reinterpret_cast<decltype(global)>(at_shared);
    at_shared += (count * static_cast<int64_t>(sizeof(*global)) + 15) / 16 * 16;
    return q;
  };
  // rows with tokens, by group: their prefix, n where there are no prefix keys
  int* sorted = shared(LISTS_SHARED, p.scratch, plan_scratch_ints(n));
  Item* items = shared(ITEMS_SHARED, p.items, max_items(n, G, a.max_tokens));
  Run* runs = shared(RUNS_SHARED, p.runs, max_runs(n, G, a.max_tokens));
  int* group_of = sorted + n;        // of a sorted entry
  int* group_tok = group_of + n;     // of a group: its tokens
  // rows listed for tiles, then for few items, by key: the prefix, or n where the items hold no prefix keys; of few items
  // n + 1 more, and one key more (own keys beside tiles, then without a prefix)
  int* list = group_tok + n + 1;
  int* key = list + 2 * n;
  int* place = key + 2 * n;            // tokens of those before it
  int* row_run = place + 2 * n + 1;    // its first run
  int* first_tok = row_run + 2 * n;    // of a key: tokens before its first
  int* first_item = first_tok + 2 * n + 3;
  if (threadIdx.x == 0) bad = 0, unsorted = 0, too_long = 0, tiles_line = both_lines = 0, first_few = 0, longest[0] = longest[1] = 0;
  if (threadIdx.x < 64) sums_memory[threadIdx.x >> 5][lane] = 0;
#pragma unroll 1
  for (int c = threadIdx.x; c < SHARES; c += THREADS) first_of[c] = INT_MAX;
  int turn = 0;
  auto sum = [&](int v, int count, int& total) {
    const int2 r = block_sum(v, count, sums_memory[turn ^= 1]);
    total = r.y;
    return r.x;
  };
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  Head head{};
  head.few_share = 1;
  head.Hq = a.Hq;
  head.max_tokens = a.max_tokens;
  head.n_ctas = n_ctas;
  head.lay = a.lay;
  auto tokens_of = [&](int i) { return a.tok_off[i + 1] - a.tok_off[i]; };

  // checks, and the rows with tokens
  int ns = 0, n_sorted_tok = 0;
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    int tok = 0, g = n;
    if (i < n) {
      const int t0 = a.tok_off[i], t1 = a.tok_off[i + 1], pre = a.prefix ? a.prefix[i] : -1, len = a.seq_lens[i];
      if ((i == 0 && t0 != 0) || t0 < 0 || t1 < t0 || t1 > a.max_tokens || len < 0 || len > cap || pre < -1 || pre >= n || pre == i ||
          (pre >= 0 && a.prefix[pre] != -1))
        bad = 1;
      else
        tok = t1 - t0;
      if (tok > 0 && pre >= 0 && a.seq_lens[pre] > 0) g = pre;
    }
    int rows, toks;
    const int at = ns + sum(tok > 0, n - i0, rows), before = n_sorted_tok + sum(tok, n - i0, toks);
    if (tok > 0) sorted[at] = i, group_of[at] = g, place[at] = before;
    ns += rows;
    n_sorted_tok += toks;
  }
  __syncthreads();
  if (bad) {
    if (threadIdx.x == 0) {
      *p.head = head;
      if (a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);
    }
#pragma unroll 1
    for (int c = threadIdx.x; c < MAX_CTAS * WORKERS; c += THREADS) p.work[c] = make_int2(0, 0);
    return;
  }
#pragma unroll 1
  for (int t = threadIdx.x; t < n_sorted_tok; t += THREADS) p.rec[t] = make_int4(-1, 0, -1, 0);
#pragma unroll 1
  for (int i = threadIdx.x + 1; i < ns; i += THREADS)
    if (group_of[i] < group_of[i - 1]) unsorted = 1;
  __syncthreads();
  if (unsorted) {
    int m = 32;
#pragma unroll 1
    while (m < ns) m <<= 1;
#pragma unroll 1
    for (int i = threadIdx.x; i < m; i += THREADS)
      keys[i] = i < ns ? static_cast<uint32_t>(group_of[i]) << ROW_BITS | sorted[i] : 0xffffffffu;
    __syncthreads();
    sort_keys(keys, m);
    __syncthreads();
    int carry = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < ns; i0 += THREADS) {
      const int i = i0 + threadIdx.x;
      int tok = 0, total;
      if (i < ns) {
        sorted[i] = keys[i] & ((1 << ROW_BITS) - 1);
        group_of[i] = keys[i] >> ROW_BITS;
        tok = tokens_of(sorted[i]);
      }
      const int before = carry + sum(tok, ns - i0, total);
      if (i < ns) place[i] = before;
      carry += total;
    }
  }
  if (threadIdx.x == 0) place[ns] = n_sorted_tok;
  __syncthreads();
  // a group's tokens: its rows stand together
#pragma unroll 1
  for (int i = threadIdx.x; i < ns; i += THREADS)
    if (i == 0 || group_of[i - 1] != group_of[i]) first_tok[group_of[i]] = place[i];
  __syncthreads();
#pragma unroll 1
  for (int i = threadIdx.x; i < ns; i += THREADS)
    if (i + 1 == ns || group_of[i + 1] != group_of[i]) group_tok[group_of[i]] = place[i + 1] - first_tok[group_of[i]];
  __syncthreads();
  auto small = [&](int row) { return tokens_of(row) <= few; };
  auto few_group = [&](int g) { return g < n && group_tok[g] <= few; };

  // the lists: tiles: all but the prefixes that have few rows, and rows with few tokens that read no prefix.  few: those
  // prefixes' rows; rows with few tokens whose prefix tiles read; and those that read none
  int base[4] = {}, nl = 0;
#pragma unroll 1
  for (int pass = ns > THREADS ? 0 : 1; pass < 2; ++pass) {  // with more rows than threads: first the lists' lengths
    int seen[4] = {};
#pragma unroll 1
    for (int i0 = 0; i0 < ns; i0 += THREADS) {
      const int i = i0 + threadIdx.x;
      int row = 0, k = 0;
      bool in[4] = {};
      if (i < ns) {
        row = sorted[i];
        k = group_of[i];
        const bool fg = few_group(k), sm = small(row);
        in[0] = !fg && (k < n || !sm);
        in[1] = fg;
        in[2] = !fg && sm && k < n && a.seq_lens[row] > 0;
        in[3] = !fg && sm && k == n;
      }
      int v[4], total[4];
#pragma unroll
      for (int l = 0; l < 4; l += 2) {  // two counts a sum
        static_assert(THREADS < 1 << 15, "a count takes 16 bits");
        int both = 0;
        const int x = sum(in[l] | in[l + 1] << 16, ns - i0, both);
        v[l] = x & 0xffff, v[l + 1] = x >> 16;
        total[l] = both & 0xffff, total[l + 1] = both >> 16;
      }
      if (ns <= THREADS)
        for (int l = 1; l < 4; ++l) base[l] = base[l - 1] + total[l - 1];
#pragma unroll
      for (int l = 0; l < 4; ++l) {
        if (pass == 1 && in[l]) {
          const int at = base[l] + seen[l] + v[l];
          list[at] = row;
          key[at] = l == 0 ? k : l == 1 ? n + 1 + k : 2 * n - 1 + l;  // the last two keys: 2 n + 1, 2 n + 2
        }
        seen[l] += total[l];
      }
    }
    if (pass == 0) {
      for (int l = 1; l < 4; ++l) base[l] = base[l - 1] + seen[l - 1];
    } else {
      nl = base[3] + seen[3];
    }
  }
  __syncthreads();
  int n_listed_tok = 0;
#pragma unroll 1
  for (int i0 = 0; i0 < nl; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    int total;
    const int at = n_listed_tok + sum(i < nl ? tokens_of(list[i]) : 0, nl - i0, total);
    if (i < nl) {
      place[i] = at;
      if (i == 0 || key[i - 1] != key[i]) first_tok[key[i]] = at;
    }
    n_listed_tok += total;
  }
  if (threadIdx.x == 0) place[nl] = n_listed_tok;
  __syncthreads();
  auto is_few = [&](int k) { return k > n; };
  const Divisor by_pair(2 * tile), by_few(few), by_heads(Hkv);
  const int page_bits = __ffs(page) - 1, page_blk_bits = __ffs(page_blk) - 1;  // powers of two
  auto cut_of = [&](int k) { return is_few(k) ? few : 2 * tile; };
  auto in_cuts = [&](int k, int x) { return static_cast<int>(is_few(k) ? by_few.of(x) : by_pair.of(x)); };
  auto in_units = [&](bool of_few, int x) { return of_few ? (x + PIECE - 1) / PIECE : (x + page - 1) >> page_bits; };
  auto in_blocks = [&](int pages) { return (pages + page_blk - 1) >> page_blk_bits; };
  auto prefix_of = [&](int k) { return k < n ? k : k > n && k <= 2 * n ? k - n - 1 : -1; };

  // items, by the last row of each key
  int n_items = 0, n_runs = 0;
#pragma unroll 1
  for (int i0 = 0; i0 < nl; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    const int k = i < nl ? key[i] : 0;
    int count = 0, total, tok = 0;
    if (i < nl && (i + 1 == nl || key[i + 1] != k)) {
      tok = place[i + 1] - first_tok[k];
      count = in_cuts(k, tok + cut_of(k) - 1);
    }
    const int at = n_items + sum(count, nl - i0, total);
    if (count > 0) first_item[k] = at;
    spread(count, [&](bool on, int src, int c) {
      const int k_ = of_lane(k, src), at_ = of_lane(at, src), tok_ = of_lane(tok, src);
      if (!on) return;
      const int pre = prefix_of(k_), cut = cut_of(k_);
      Item it{};
      it.tok = first_tok[k_] + c * cut;
      it.n_tok = min(cut, tok_ - c * cut);
      it.prefix_keys = pre >= 0 ? a.seq_lens[pre] : 0;
      it.flags = is_few(k_) ? ITEM_FEW | (k_ == 2 * n + 1 ? 0u : ITEM_ALONE) : ITEM_ALONE;
      items[at_ + c] = it;
    });
    n_items += total;
  }
  __syncthreads();

  // runs, by their rows: a row has its own run in each item that has tokens of it (of tiles: unless a few item has its own
  // keys), and writes the prefix's in each item that begins with it.  A token with a few item beside its tiles spoils the
  // tiles' being alone.
#pragma unroll 1
  for (int i0 = 0; i0 < nl; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    int count = 0, total, in = 0, tok = 0, k0 = 0, n_in = 0, k = 0, row = 0;
    bool own = false, beside = false;
    if (i < nl) {
      k = key[i], row = list[i];
      in = place[i] - first_tok[k];
      tok = place[i + 1] - place[i];
      const int cut = cut_of(k);
      k0 = in_cuts(k, in);
      const int k1 = in_cuts(k, in + tok - 1);
      n_in = k1 - k0 + 1;
      own = is_few(k) || !small(row);
      beside = k < n && small(row) && a.seq_lens[row] > 0;
      // items whose first token is one of the row's: those up to k1 from the first that begins at or behind `in`
      count = (own ? n_in : 0) + (prefix_of(k) >= 0 ? k1 - in_cuts(k, in + cut - 1) + 1 : 0);
    }
    const int at = n_runs + sum(count, nl - i0, total);
    if (i < nl) row_run[i] = at;
    spread(n_in, [&](bool on, int src, int c) {
      const int k_ = of_lane(k, src), in_ = of_lane(in, src), tok_ = of_lane(tok, src), row_ = of_lane(row, src);
      const int own_ = of_lane(own, src), beside_ = of_lane(beside, src);
      int at_ = of_lane(at, src);
      const int k0_ = of_lane(k0, src), item = c + k0_;
      if (!on) return;
      const int cut = cut_of(k_), pre = prefix_of(k_);
      Item& it = items[first_item[k_] + item];
      const int lo = max(in_, item * cut), hi = min(in_ + tok_, (item + 1) * cut);  // places among the key's tokens
      at_ += run_before(c, in_ == k0_ * cut, own_, pre >= 0);
      if (lo == item * cut) {
        it.run = at_;
        if (pre >= 0) runs[at_++] = Run{pre, 0, in_units(is_few(k_), it.prefix_keys), it.prefix_keys, 0, it.n_tok, -1, 0};
      }
      if (beside_) it.flags = 0;
      if (!own_) return;
      const int seen = max(0, a.seq_lens[row_] - (in_ + tok_ - hi));  // own keys of its last token here
      runs[at_] = Run{row_, 0, in_units(is_few(k_), seen), seen, lo - item * cut, hi - item * cut, a.tok_off[row_] + lo - in_, 0};
    });
    n_runs += total;
  }
  __syncthreads();

  // eight lanes an item: where its runs' pages begin
#pragma unroll 1
  for (int c = threadIdx.x / 8; c < n_items; c += THREADS / 8) {
    const int part = threadIdx.x & 7;
    const uint32_t mask = 0xffu << (lane & 24);
    Item& it = items[c];
    const int run0 = it.run, it_runs = (c + 1 < n_items ? items[c + 1].run : n_runs) - run0;
    int pages = 0, end0 = 0, begin1 = INT_MAX;
    const int most = (INT_MAX - BLOCK) / (it.flags & ITEM_FEW ? PIECE : page);  // columns are counted in 31 bits
    bool fit = true;
#pragma unroll 1
    for (int r0 = 0; r0 < it_runs; r0 += 8) {
      Run* run = runs + run0 + r0 + part;
      const bool on = r0 + part < it_runs;
      const int mine = on ? run->pages : 0;
      int inc = mine;
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) {
        const int u = __shfl_up_sync(mask, inc, o, 8);
        if (part >= o) inc += u;
      }
      if (on) {
        const int off = pages + inc - mine;
        run->off = off;
        if (run->tok0 < tile) end0 = max(end0, off + mine);
        if (run->token >= 0 && run->tok1 > tile) begin1 = min(begin1, off);
      }
      inc = __shfl_sync(mask, inc, 7, 8);  // (a run has 2^27 pages at most, eight have 2^30)
      fit = fit && inc <= most - pages;
      pages = fit ? pages + inc : 0;
    }
    if (!fit) too_long = 1;
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
      end0 = max(end0, __shfl_xor_sync(mask, end0, o));
      begin1 = min(begin1, __shfl_xor_sync(mask, begin1, o));
    }
    if (part == 0) {
      it.n_runs = it_runs;
      it.pages = pages;
      it.blocks = it.flags & ITEM_FEW ? pages : in_blocks(pages);
      it.end0 = in_blocks(end0);
      it.prefix_blocks = in_blocks(in_units(false, it.prefix_keys));
      it.begin1 = begin1 >> page_blk_bits;
    }
  }
  __syncthreads();

  // a warp some rows: their tokens' items and own columns
  {
    const int rows_a_warp = (nl + WARPS - 1) / WARPS, end = min(nl, (warp + 1) * rows_a_warp);
#pragma unroll 1
    for (int i0 = warp * rows_a_warp; i0 < end; i0 += 32) {
      const int i = i0 + lane;
      int k = 0, in = 0, tok = 0, t0 = 0, own = 0, o0 = 0, run0 = 0, k0 = 0;
      if (i < end) {
        k = key[i], o0 = place[i], run0 = row_run[i];
        in = o0 - first_tok[k];
        tok = place[i + 1] - o0;
        k0 = in_cuts(k, in);
        t0 = a.tok_off[list[i]];
        own = is_few(k) || !small(list[i]);
      }
      spread(tok, [&](bool on, int src, int j) {
        const int k_ = of_lane(k, src), in_ = of_lane(in, src), t = of_lane(t0, src) + j, o = of_lane(o0, src) + j;
        const int own_ = of_lane(own, src), run0_ = of_lane(run0, src), k0_ = of_lane(k0, src);
        if (!on) return;
        const int cut = cut_of(k_), item = in_cuts(k_, in_ + j), at = in_ + j - item * cut;
        p.order[o] = t;
        reinterpret_cast<int2*>(p.rec + t)[is_few(k_)] = make_int2(first_item[k_] + item, at);
        int2 cols = make_int2(0, 0);
        if (own_) {
          const bool pre = prefix_of(k_) >= 0;
          const int c = item - k0_;
          const bool first = in_ == k0_ * cut;
          const Run& run = runs[run0_ + run_before(c, first, true, pre) + (pre && (c > 0 || first))];
          // the last token sees the run's keys, each before it one less
          const int from = run.off * (is_few(k_) ? PIECE : page);
          cols = make_int2(from, from + max(0, run.keys - (run.tok1 - 1 - at)));
        }
        p.own[o] = cols;
      });
    }
  }

  // the lines: the items of tiles come first
  unsigned long long line = 0;
#pragma unroll 1
  for (int i0 = 0; i0 < n_items; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    const unsigned long long v = i < n_items ? static_cast<unsigned long long>(Hkv) * length_of(items[i]) : 0;
    unsigned long long inc = v;
    if (warp * 32 < n_items - i0) {
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long u = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += u;
      }
    }
    if (lane == 31) lines[warp] = inc;
    __syncthreads();
    unsigned long long before = line;
#pragma unroll 1
    for (int w = 0; w < warp && w * 32 < n_items - i0; ++w) before += lines[w];
    before += inc - v;
    if (i < n_items) {
      items[i].start = static_cast<uint32_t>(before);  // of few items: the tiles' line before it too, for now
      atomicMax(&longest[items[i].flags & ITEM_FEW ? 1 : 0], length_of(items[i]));
      if ((items[i].flags & ITEM_FEW) && (i == 0 || !(items[i - 1].flags & ITEM_FEW))) tiles_line = before, first_few = i;
      if (i == n_items - 1) {
        both_lines = before + v;
        if (!(items[i].flags & ITEM_FEW)) tiles_line = before + v, first_few = n_items;
      }
    }
    if (i0 + THREADS < n_items) {
#pragma unroll 1
      for (int w = 0; w < WARPS; ++w) line += lines[w];
      __syncthreads();
    }
  }
  __syncthreads();
  const unsigned long long few_line = both_lines - tiles_line;
  // CTAs for each kind by what they take, one at least
  const bool both = tiles_line > 0 && few_line > 0, fits = !too_long && tiles_line < 0x20000000ull && few_line < 0x20000000ull && (!both || n_ctas > 1);
  int tile_ctas = few_line > 0 ? 0 : n_ctas;
  if (both) {
    const float tiles_cost = static_cast<float>(tiles_line), few_cost = static_cast<float>(few_line) * FEW_PER_TILES / WORKERS;
    tile_ctas = min(n_ctas - 1, max(1, __float2int_rn(n_ctas * tiles_cost / (tiles_cost + few_cost))));
  }
  const uint32_t few_ctas = n_ctas - tile_ctas;
  // a share of tiles holds a block at least, one of few items a few pieces: each share more is a part more to be added up; of
  // long entries more, where a share's time and that of joining the longest entry's parts meet
  uint32_t share = max(OTHER_BLOCK, (static_cast<uint32_t>(sqrtf(TILES_JOIN * longest[0])) / WHOLE_BLOCK + 1) * WHOLE_BLOCK);
  uint32_t few_share = max(MIN_FEW_SHARE, static_cast<uint32_t>(sqrtf(FEW_JOIN * longest[1])));
  if (fits && tile_ctas > 0) share = max(share, (static_cast<uint32_t>(tiles_line) + tile_ctas - 1) / tile_ctas);
  if (fits && few_ctas > 0) few_share = max(few_share, (static_cast<uint32_t>(few_line) + few_ctas * WORKERS - 1) / (few_ctas * WORKERS));
  const Divisor by_share(share), by_few_share(few_share);
#pragma unroll 1
  for (int i = first_few + threadIdx.x; i < n_items; i += THREADS) items[i].start -= static_cast<uint32_t>(tiles_line);
  __syncthreads();
  const int n_flat = fits ? n_items * Hkv : 0;
  // the shares' segments, rows of partial results, pieces of the join's list
  int n_segs = 0, n_rows = 0, n_join = 0;
#pragma unroll 1
  for (int f0 = 0; f0 < n_flat; f0 += THREADS) {
    const int f = f0 + threadIdx.x;
    int segs = 0, rows = 0, pieces = 0, cta0 = 0, right_away = 0;
    if (f < n_flat) {
      const int i = by_heads.of(f);
      const Item& it = items[i];
      const OnLine on = on_line(it, f - i * Hkv);
      const Divisor& by = it.flags & ITEM_FEW ? by_few_share : by_share;
      cta0 = by.of(on.begin);
      if (it.blocks > 0) segs = by.of(on.begin_of(it.blocks - 1)) - cta0 + 1;
      right_away = segs == 1 && (it.flags & ITEM_ALONE);
      if (!right_away) {
        rows = segs * it.n_tok * G;
        // rows of a few item beside tiles are joined by the tiles' pieces
        if ((it.flags & (ITEM_FEW | ITEM_ALONE)) != ITEM_FEW) pieces = (it.n_tok * G + rows_a_piece(segs) - 1) / rows_a_piece(segs);
      }
    }
    // two counts a sum: no more segments than entries and shares, 64 pieces an entry at most
    static_assert(4 * TILE / JOIN_ROWS * THREADS < 1 << 16 && THREADS + SHARES < 1 << 15, "a count takes 16 bits");
    int both, total;
    const uint32_t at = sum(segs << 16 | pieces, n_flat - f0, both);
    const int seg0 = n_segs + (at >> 16), piece0 = n_join + (at & 0xffff);
    const int part_row = n_rows + sum(rows, n_flat - f0, total);
    n_segs += static_cast<uint32_t>(both) >> 16, n_join += both & 0xffff, n_rows += total;
    if (f < n_flat && f == first_few * Hkv) first_of[tile_ctas] = seg0;  // the end of tiles
    if (f < n_flat) p.part[f] = part_row;
    spread(pieces, [&](bool on, int src, int i) {
      const int f_ = of_lane(f, src), piece = of_lane(piece0, src) + i, row0 = of_lane(part_row, src), parts = of_lane(segs, src);
      if (!on) return;
      const int item = by_heads.of(f_);
      const Item& it = items[item];
      p.join[piece] = Piece{it.tok, i * rows_a_piece(parts), it.n_tok * G, f_ - item * Hkv, static_cast<uint32_t>(row0), parts,
                            !(it.flags & (ITEM_FEW | ITEM_ALONE)), 0};
    });
    spread(segs, [&](bool on_, int src, int i) {
      const int f_ = of_lane(f, src), at = of_lane(seg0, src) + i, whole = of_lane(right_away, src), row0 = of_lane(part_row, src);
      const uint32_t c = of_lane(cta0, src) + i;
      if (!on_) return;
      const int item = by_heads.of(f_), h = f_ - item * Hkv;
      const Item& it = items[item];
      const OnLine on = on_line(it, h);
      const bool of_few = it.flags & ITEM_FEW;
      const uint32_t entry_share = of_few ? few_share : share;
      Segment sg{};
      sg.h = h;
      sg.b0 = on.block_from(c * entry_share, it.blocks);
      sg.b1 = on.block_from((c + 1) * entry_share, it.blocks);
      sg.tok = it.tok, sg.n_tok = it.n_tok, sg.run = it.run, sg.n_runs = it.n_runs;
      sg.prefix_keys = it.prefix_keys, sg.pages = it.pages;
      sg.end0 = it.end0, sg.begin1 = it.begin1, sg.prefix_blocks = it.prefix_blocks;
      sg.flags = (two_tiles(it, G) ? SEG_TWO : 0u) | (of_few ? SEG_FEW : 0u) | (whole ? SEG_WHOLE : 0u);
      sg.part_row = static_cast<uint32_t>(row0) + i * it.n_tok * G;
      const int page0 = sg.b0 * (of_few ? 1 : page_blk);
      int lo = 0, hi = it.n_runs - 1;
      while (lo < hi) {  // the last run that begins at or before the page (runs without pages share their successor's place)
        const int mid = (lo + hi + 1) >> 1;
        if (runs[it.run + mid].off <= page0) lo = mid; else hi = mid - 1;
      }
      const Run& run = runs[it.run + lo];
      sg.run_at = lo, sg.run_row = run.row, sg.run_off = run.off, sg.run_pages = run.pages, sg.run_keys = run.keys;
      p.segs[at] = sg;
      atomicMin(&first_of[of_few ? tile_ctas + 1 + c : c], at);
    });
  }
  // what the attention's kernels read of items and runs
  if (in_shared & ITEMS_SHARED)
#pragma unroll 1
    for (int i = threadIdx.x; i < n_items * static_cast<int>(sizeof(Item) / 16); i += THREADS)
      reinterpret_cast<int4*>(p.items)[i] = reinterpret_cast<const int4*>(items)[i];
  if (in_shared & RUNS_SHARED)
#pragma unroll 1
    for (int i = threadIdx.x; i < n_runs * static_cast<int>(sizeof(Run) / 16); i += THREADS)
      reinterpret_cast<int4*>(p.runs)[i] = reinterpret_cast<const int4*>(runs)[i];
  __syncthreads();
  // the shares' first segments; one without gets the next one's, the last the end
  {
    constexpr int EACH = (SHARES + THREADS - 1) / THREADS;
    int low[EACH], least = n_segs;
#pragma unroll
    for (int i = EACH - 1; i >= 0; --i) {
      const int c = threadIdx.x * EACH + i;
      if (c < SHARES) least = min(least, first_of[c]);
      low[i] = least;
    }
    int after = least;  // of this thread and those behind it in the warp
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_down_sync(0xffffffffu, after, o);
      if (lane + o < 32) after = min(after, u);
    }
    if (lane == 0) sums_memory[0][warp] = after;
    __syncthreads();
    const int behind = __reduce_min_sync(0xffffffffu, lane > warp && lane < WARPS ? sums_memory[0][lane] : INT_MAX);
    const int next = __shfl_down_sync(0xffffffffu, after, 1);
    const int rest = min(behind, lane < 31 ? next : INT_MAX);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int c = threadIdx.x * EACH + i;
      if (c < SHARES) first_of[c] = min(low[i], rest);
    }
  }
  __syncthreads();
  // the few items' shares are dealt to the CTAs' first warps, then to their second ones: few shares are spread over many SMs
#pragma unroll 1
  for (int i = threadIdx.x; i < n_ctas * WORKERS; i += THREADS) {
    const int cta = i / WORKERS, slot = cta < tile_ctas ? cta : tile_ctas + 1 + i % WORKERS * few_ctas + cta - tile_ctas;
    p.work[i] = make_int2(first_of[slot], first_of[slot + 1]);
  }
  if (threadIdx.x == 0) {
    if (fits) {
      head.n_join = n_join;
      head.few_share = few_share;
      head.tile_ctas = tile_ctas;
    }
    *p.head = head;
    if (!fits && a.status) atomicCAS(a.status, 0, DOPR_ERR_UNSUPPORTED);
  }
}

}  // namespace

int64_t shared_plan_bytes(const dopr_cache_layout& lay, int Hq, int max_tokens) {
  return plan_view(nullptr, lay.n_seqs, lay.n_kv_heads, Hq / lay.n_kv_heads, max_tokens).bytes;
}

cudaError_t launch_shared_plan(const SharedPlanArgs& a, int num_sms, cudaStream_t st) {
  const int n = a.lay.n_seqs, G = a.Hq / a.lay.n_kv_heads;
  int n_keys = 32, in_shared = 0;
#pragma unroll 1
  while (n_keys < n) n_keys <<= 1;
  int64_t bytes = 4 * static_cast<int64_t>(n_keys);
  auto take = [&](int what, int64_t more) {
    more = (more + 15) / 16 * 16;
    if (bytes + more > MAX_SHARED) return;
    bytes += more;
    in_shared |= what;
  };
  take(LISTS_SHARED, 4 * plan_scratch_ints(n));
  take(ITEMS_SHARED, max_items(n, G, a.max_tokens) * static_cast<int64_t>(sizeof(Item)));
  take(RUNS_SHARED, max_runs(n, G, a.max_tokens) * static_cast<int64_t>(sizeof(Run)));
  const cudaError_t e = cudaFuncSetAttribute(k_shared_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SHARED);
  if (e != cudaSuccess) return e;
  return launch_dependent(k_shared_plan, dim3(1), THREADS, static_cast<int>(bytes), st, a,
                          plan_view(a.plan, n, a.lay.n_kv_heads, G, a.max_tokens), num_sms < MAX_CTAS ? num_sms : MAX_CTAS, n_keys,
                          in_shared);
}

}  // namespace dopr
