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
  const int tile = tokens_a_tile(G), few = tokens_a_few(G);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t cap = static_cast<int64_t>(a.lay.max_blocks) * page;
  const Plan p = plan_view(a.plan, n, Hkv, G, a.max_tokens);
  int* sorted = p.scratch;          // rows with tokens, by group: their prefix, n where there are no prefix keys
  int* group_of = sorted + n;       // of a sorted entry
  int* group_tok = group_of + n;    // of a group: its tokens
  int* list = group_tok + n + 1;    // the rows of a kind of items, by key
  int* key = list + n;              // of a listed row: its prefix; n and n + 1 where the items hold no prefix keys
  int* place = key + n;             // of a listed row: tokens of those before it
  int* first_tok = place + n + 1;   // of a key: tokens before its first
  int* first_item = first_tok + n + 2;
  if (threadIdx.x == 0) bad = 0, unsorted = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  Head head{};
  head.share = head.few_share = 1;
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
    for (int c = threadIdx.x; c < SHARES; c += THREADS) p.first[c] = 0;
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
  // a group's tokens: its rows stand together
  {
    int carry = 0;
    for (int i0 = 0; i0 < ns; i0 += THREADS) {
      const int i = i0 + threadIdx.x;
      const int tok = i < ns ? tokens_of(sorted[i]) : 0;
      const int at = carry + static_cast<int>(block_exclusive(static_cast<unsigned long long>(tok), warp_sum, total));
      if (i < ns) {
        place[i] = at;
        if (i == 0 || group_of[i - 1] != group_of[i]) first_tok[group_of[i]] = at;
      }
      carry += static_cast<int>(total);
    }
    if (threadIdx.x == 0) place[ns] = carry;
    __syncthreads();
    for (int i = threadIdx.x; i < ns; i += THREADS)
      if (i + 1 == ns || group_of[i + 1] != group_of[i]) group_tok[group_of[i]] = place[i + 1] - first_tok[group_of[i]];
    __syncthreads();
  }
  auto small = [&](int row) { return tokens_of(row) <= few; };
  auto few_group = [&](int g) { return g < n && group_tok[g] <= few; };
  for (int t = threadIdx.x; t < a.tok_off[n]; t += THREADS) p.rec[t] = make_int4(-1, 0, -1, 0);

  // Both kinds are laid out alike: rows in the order of their keys, their tokens cut into items.
  int n_items = 0, n_runs = 0, n_tok = 0;
  for (int kind = 0; kind < 2; ++kind) {
    const int cut = kind ? few : 2 * tile, unit = kind ? PIECE : page, block_units = kind ? 1 : page_blk;
    int nl = 0;
    // tiles: all but the prefixes that have few rows, and rows with few tokens that read no prefix.  few: those prefixes'
    // rows; rows with few tokens whose prefix tiles read; and those that read none
    for (int part = 0; part < (kind ? (few > 0 ? 3 : 0) : 1); ++part) {
      for (int i0 = 0; i0 < ns; i0 += THREADS) {
        const int i = i0 + threadIdx.x;
        bool in = false;
        int row = 0, k = 0;
        if (i < ns) {
          row = sorted[i];
          k = group_of[i];
          const bool fg = few_group(k);
          if (kind == 0) {
            in = !fg && (k < n || !small(row));
          } else if (part == 0) {
            in = fg;
          } else {
            in = !fg && small(row) && (part == 1 ? k < n && a.seq_lens[row] > 0 : k == n);
            k = n + part - 1;
          }
        }
        const int at = nl + static_cast<int>(block_exclusive(static_cast<unsigned long long>(in), warp_sum, total));
        if (in) list[at] = row, key[at] = k;
        nl += static_cast<int>(total);
      }
    }
    __syncthreads();
    int carry = 0;
    for (int i0 = 0; i0 < nl; i0 += THREADS) {
      const int i = i0 + threadIdx.x;
      const int tok = i < nl ? tokens_of(list[i]) : 0;
      const int at = carry + static_cast<int>(block_exclusive(static_cast<unsigned long long>(tok), warp_sum, total));
      if (i < nl) {
        place[i] = at;
        if (i == 0 || key[i - 1] != key[i]) first_tok[key[i]] = at;
      }
      carry += static_cast<int>(total);
    }
    if (threadIdx.x == 0) place[nl] = carry;
    __syncthreads();

    // items, written by the last row of each key
    const int items0 = n_items;
    for (int i0 = 0; i0 < nl; i0 += THREADS) {
      const int i = i0 + threadIdx.x;
      const int k = i < nl ? key[i] : 0;
      int count = 0, tok = 0;
      if (i < nl && (i + 1 == nl || key[i + 1] != k)) {
        tok = place[i + 1] - first_tok[k];
        count = (tok + cut - 1) / cut;
      }
      const int at = n_items + static_cast<int>(block_exclusive(static_cast<unsigned long long>(count), warp_sum, total));
      if (count > 0) first_item[k] = at;
      for (int c = 0; c < count; ++c) {
        Item it{};
        it.tok = n_tok + first_tok[k] + c * cut;
        it.n_tok = min(cut, tok - c * cut);
        it.prefix_keys = k < n ? a.seq_lens[k] : 0;
        it.flags = kind == 0 ? ITEM_ALONE : ITEM_FEW | (k == n ? 0u : ITEM_ALONE);
        p.items[at + c] = it;
      }
      n_items += static_cast<int>(total);
    }
    __syncthreads();

    // runs, by their rows: a row writes its own run in each item that has tokens of it (of tiles: unless a few item has
    // its own keys), and the prefix's in each item that begins with it
    for (int i0 = 0; i0 < nl; i0 += THREADS) {
      const int i = i0 + threadIdx.x;
      int in = 0, tok = 0, k0 = 0, k1 = -1, begun = 0, k = 0;
      bool own = false;
      if (i < nl) {
        k = key[i];
        in = place[i] - first_tok[k];
        tok = place[i + 1] - place[i];
        k0 = in / cut;
        k1 = (in + tok - 1) / cut;
        begun = k1 - (in + cut - 1) / cut + 1;  // items whose first token is one of the row's
        own = kind == 1 || !small(list[i]);
      }
      const int count = (own ? k1 - k0 + 1 : 0) + (k < n ? begun : 0);
      int at = n_runs + static_cast<int>(block_exclusive(static_cast<unsigned long long>(count), warp_sum, total));
      for (int c = k0; c <= k1; ++c) {
        Item& it = p.items[first_item[k] + c];
        const int lo = max(in, c * cut), hi = min(in + tok, (c + 1) * cut);  // places among the key's tokens
        if (lo == c * cut) {
          it.run = at;
          if (k < n) {
            const int keys_ = a.seq_lens[k];
            p.runs[at++] = Run{k, 0, (keys_ + unit - 1) / unit, keys_, 0, it.n_tok, -1, 0};
          }
        }
        if (!own) continue;
        const int row = list[i];
        const int seen = max(0, a.seq_lens[row] - (in + tok - hi));  // own keys of its last token here
        p.runs[at++] = Run{row, 0, (seen + unit - 1) / unit, seen, lo - c * cut, hi - c * cut, a.tok_off[row] + lo - in, 0};
      }
      n_runs += static_cast<int>(total);
    }
    __syncthreads();

    // a warp a row: its tokens' items; a token with a few item beside its tiles spoils the tiles' being alone
    for (int i = warp; i < nl; i += THREADS / 32) {
      const int row = list[i], k = key[i], in = place[i] - first_tok[k], tok = place[i + 1] - place[i], t0 = a.tok_off[row];
      const bool beside = kind == 0 && k < n && small(row) && a.seq_lens[row] > 0;
      for (int j = lane; j < tok; j += 32) {
        const int item = first_item[k] + (in + j) / cut, at = (in + j) % cut;
        const int o = n_tok + place[i] + j;
        p.order[o] = t0 + j;
        p.own[o] = make_int2(0, 0);
        int2* rec = reinterpret_cast<int2*>(p.rec + t0 + j) + kind;
        *rec = make_int2(item, at);
        if (beside) p.items[item].flags = 0;
      }
    }
    __syncthreads();

    // a warp an item: where its runs' pages begin, and its tokens' own columns
    for (int c = items0 + warp; c < n_items; c += THREADS / 32) {
      Item it = p.items[c];
      it.n_runs = (c + 1 < n_items ? p.items[c + 1].run : n_runs) - it.run;
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
          // the last token sees the run's keys, each before it one less
          for (int x = run.tok0; run.token >= 0 && x < run.tok1; ++x)
            p.own[it.tok + x] = make_int2(off * unit, off * unit + max(0, run.keys - (run.tok1 - 1 - x)));
        }
        pages += __shfl_sync(0xffffffffu, inc, 31);
      }
      end0 = __reduce_max_sync(0xffffffffu, end0);
      begin1 = __reduce_min_sync(0xffffffffu, begin1);
      if (lane == 0) {
        it.pages = pages;
        it.blocks = (pages + block_units - 1) / block_units;
        it.end0 = (end0 + page_blk - 1) / page_blk;
        it.prefix_blocks = ((it.prefix_keys + page - 1) / page + page_blk - 1) / page_blk;
        it.begin1 = begin1 / page_blk;
        p.items[c] = it;
      }
    }
    n_tok += carry;
    __syncthreads();
  }

  // the line
  unsigned long long tiles_line = 0, few_line = 0;
  for (int i0 = 0; i0 < n_items; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    unsigned long long length = 0;
    bool is_few = false;
    if (i < n_items) {
      const Item it = p.items[i];
      length = static_cast<unsigned long long>(Hkv) * length_of(it, G);
      is_few = it.flags & ITEM_FEW;
    }
    const unsigned long long at_tiles = tiles_line + block_exclusive(is_few ? 0ull : length, warp_sum, total);
    tiles_line += total;
    const unsigned long long at_few = few_line + block_exclusive(is_few ? length : 0ull, warp_sum, total);
    few_line += total;
    if (i < n_items) p.items[i].start = static_cast<uint32_t>(is_few ? at_few : at_tiles);
  }
  // CTAs for each kind by what they take, one at least
  const bool both = tiles_line > 0 && few_line > 0, fits = tiles_line < 0x20000000ull && few_line < 0x20000000ull && (!both || n_ctas > 1);
  int tile_ctas = few_line > 0 ? 0 : n_ctas;
  if (both) {
    const unsigned long long few_cost = few_line * FEW_PER_TILES / WORKERS;
    tile_ctas = min(n_ctas - 1, max(1, static_cast<int>((n_ctas * tiles_line + (tiles_line + few_cost) / 2) / (tiles_line + few_cost))));
  }
  const uint32_t few_ctas = n_ctas - tile_ctas;
  // a share of tiles holds a block at least, one of few items a few pieces: each share more is a part more to be added up
  uint32_t share = block_length(false), few_share = MIN_FEW_SHARE;
  if (fits && tile_ctas > 0) share = max(share, static_cast<uint32_t>((tiles_line + tile_ctas - 1) / tile_ctas));
  if (fits && few_ctas > 0) few_share = max(few_share, static_cast<uint32_t>((few_line + few_ctas * WORKERS - 1) / (few_ctas * WORKERS)));
  __syncthreads();
  const int n_flat = fits ? n_items * Hkv : 0;
  // the CTAs' segments, rows of partial results, pieces of the join's list
  unsigned long long segments = 0, tile_segments = 0, rows = 0;  // in the upper half of rows: pieces
  for (int f0 = 0; f0 < n_flat; f0 += THREADS) {
    const int f = f0 + threadIdx.x;
    unsigned long long count = 0;
    uint32_t segs = 0, few_segs = 0, entry_share = 1;
    int entry_rows = 0;
    bool right_away = false;
    Item it{};
    OnLine on{0, 1};
    if (f < n_flat) {
      it = p.items[f / Hkv];
      on = on_line(it, f % Hkv, G);
      entry_share = it.flags & ITEM_FEW ? few_share : share;
      segs = on.segments(it.blocks, entry_share);
      if (it.flags & ITEM_FEW) few_segs = segs;
      right_away = segs == 1 && (it.flags & ITEM_ALONE) && copies_of(it, G) == 1;
      if (!right_away) {
        entry_rows = it.n_tok * G;
        count = static_cast<unsigned long long>(segs) * entry_rows * copies_of(it, G);
        // rows of a few item beside tiles are joined by the tiles' pieces
        if ((it.flags & (ITEM_FEW | ITEM_ALONE)) == ITEM_FEW) entry_rows = 0;
        count |= static_cast<unsigned long long>((entry_rows + JOIN_ROWS - 1) / JOIN_ROWS) << 32;
      }
    }
    const unsigned long long at = rows + block_exclusive(count, warp_sum, total);
    rows += total;
    if (f < n_flat) p.part[f] = static_cast<uint32_t>(at);
    for (int r = 0; r < entry_rows; r += JOIN_ROWS) p.join[(at >> 32) + r / JOIN_ROWS] = make_int2(f, r);
    const uint32_t seg0 = static_cast<uint32_t>(segments + block_exclusive(static_cast<unsigned long long>(segs), warp_sum, total));
    segments += total;
    block_exclusive(static_cast<unsigned long long>(segs - few_segs), warp_sum, total);
    tile_segments += total;
    for (uint32_t i = 0; i < segs; ++i) {
      const uint32_t c = on.cta_of(0, entry_share) + i;
      Segment sg{};
      sg.f = f;
      sg.h = f % Hkv;
      sg.b0 = on.block_from(c * entry_share, it.blocks);
      sg.b1 = on.block_from((c + 1) * entry_share, it.blocks);
      sg.tok = it.tok, sg.n_tok = it.n_tok, sg.run = it.run, sg.n_runs = it.n_runs;
      sg.prefix_keys = it.prefix_keys, sg.pages = it.pages;
      sg.end0 = it.end0, sg.begin1 = it.begin1, sg.prefix_blocks = it.prefix_blocks;
      sg.flags = (two_tiles(it, G) ? SEG_TWO : 0u) | (it.flags & ITEM_FEW ? SEG_FEW : 0u) | (right_away ? SEG_WHOLE : 0u);
      sg.part_row = static_cast<uint32_t>(at) + i * copies_of(it, G) * it.n_tok * G;
      p.segs[seg0 + i] = sg;
    }
  }
  // the shares' first segments
  __syncthreads();
  for (int c = threadIdx.x; c < SHARES; c += THREADS) {
    const bool of_few = c > tile_ctas;
    const uint32_t mine = of_few ? c - tile_ctas - 1 : c, kind_share = of_few ? few_share : share;
    int lo = of_few ? static_cast<int>(tile_segments) : 0, hi = static_cast<int>(of_few ? segments : tile_segments);
    while (lo < hi) {  // the first segment of this share or a later one
      const int mid = (lo + hi) >> 1;
      const Segment& sg = p.segs[mid];
      if (on_line(p.items[sg.f / Hkv], sg.h, G).cta_of(sg.b0, kind_share) < mine) lo = mid + 1; else hi = mid;
    }
    p.first[c] = lo;
  }
  if (threadIdx.x == 0) {
    if (fits) {
      head.tokens = a.tok_off[n];
      head.n_items = n_items;
      head.n_flat = n_flat;
      head.n_join = static_cast<int>(rows >> 32);
      head.share = share;
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
  int keys = 2;
  while (keys < a.lay.n_seqs) keys <<= 1;
  static_assert(CACHE_MAX_SEQS * 4 <= 65536, "shared memory of the sort");
  const cudaError_t e = cudaFuncSetAttribute(k_shared_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, 65536);
  if (e != cudaSuccess) return e;
  return launch_dependent(k_shared_plan, dim3(1), THREADS, keys * 4, st, a, num_sms < MAX_CTAS ? num_sms : MAX_CTAS);
}

}  // namespace dopr
