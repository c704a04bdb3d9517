// shared_attn.cuh -- how a step's attention over the paged cache is split: what k_shared_plan.cu lays down and
// k_shared_attn.cu walks through.
//
// Tokens of rows with one prefix (or of rows without) stand in one order, cut into items of up to two tiles of 128 rows
// (G = q heads a kv head rows a token).  An item's keys are a list of pages, as runs: the prefix's pages, which all its
// tokens see, then for each of its rows the row's own pages, as far as its last token in the item sees them; a token
// sees its own run's keys up to itself.  A page's place in the list is its place in the columns of S, so a token's keys
// are two intervals of columns.  128 columns are a block.
//
// An item and a kv head are a flat entry.  The flat entries' blocks lie one after another on a line on which each entry
// also takes OVERHEAD steps, and every CTA takes an equal share of the line.  What a CTA has of an entry is a segment; it
// leaves partial softmax results (maximum, sum, weighted values), which the joining kernel adds up by row; only an entry
// of two tiles that is whole in one CTA gives its rows' results right away.
#pragma once

#include "device_common.cuh"
#include "internal.h"

namespace dopr {
namespace shared_attn {

constexpr int TILE = 128;   // rows of a tile
constexpr int BLOCK = 128;  // columns of a block
constexpr uint32_t OVERHEAD = 2;
constexpr int MAX_CTAS = 256;
constexpr int JOIN_ROWS = 8;

struct alignas(16) Run {
  int row;    // table row
  int off;    // pages of the item before it
  int pages;
  int keys;   // of the row that the item sees
  int tok0, tok1;  // the item's tokens it belongs to; a prefix's: 0, the item's
  int token;  // the first of them; -1: a prefix
  int pad;
};
struct alignas(16) Item {
  int tok, n_tok;    // place of its first token in `order`
  int run, n_runs;
  int prefix_keys;
  int pages;
  uint32_t cost;     // where its first entry begins on the line
  uint32_t blocks;
  // blocks that concern the first tile's rows: [0, end0); the second's: [0, prefix_blocks) and from begin1 on
  uint32_t end0, begin1, prefix_blocks;
  int pad;
};
struct alignas(16) Head {
  int tokens, n_items, n_flat, n_join;
  uint32_t share, total;  // of the line: a CTA's part, all of it
  int n_seqs, n_kv_heads, Hq, max_tokens, n_ctas, head_dim, page;  // what the plan was made for
};
__host__ __device__ inline bool made_for(const Head& h, const dopr_cache_layout& lay, int Hq, int max_tokens, int n_ctas) {
  return h.n_seqs == lay.n_seqs && h.n_kv_heads == lay.n_kv_heads && h.Hq == Hq && h.max_tokens == max_tokens &&
         h.n_ctas == n_ctas && h.head_dim == lay.head_dim && h.page == lay.page;
}
struct Plan {
  Head* head;
  int* first;      // [MAX_CTAS] flat entry in which a CTA's share begins
  int4* rec;       // [tokens] item, place in it, first column of its own keys, own keys seen
  Item* items;
  Run* runs;
  uint32_t* part;  // [flat entry] first row of its partial results
  int2* join;      // flat entry, first of up to JOIN_ROWS rows that are to be added up from partial results
  int* order;      // [tokens]
  int2* own;       // [tokens, in that order] columns of its own keys, from and to
  int* scratch;    // 5 * n_seqs + 5, of the plan kernel
  int64_t bytes;
};
__host__ __device__ inline int tokens_a_tile(int G) { return TILE / G; }
__host__ __device__ inline int64_t max_items(int n_seqs, int G, int max_tokens) {
  const int pair = 2 * tokens_a_tile(G);
  return (static_cast<int64_t>(max_tokens) + pair - 1) / pair + (n_seqs < max_tokens ? n_seqs : max_tokens);
}
__host__ __device__ inline Plan plan_view(void* base, int n_seqs, int n_kv_heads, int G, int max_tokens) {
  uint8_t* b = static_cast<uint8_t*>(base);
  int64_t at = 0;
  auto take = [&](int64_t n) {
    uint8_t* p = b + at;
    at += (n + 15) / 16 * 16;
    return static_cast<void*>(p);
  };
  const int64_t items = max_items(n_seqs, G, max_tokens);
  Plan p;
  p.head = static_cast<Head*>(take(sizeof(Head)));
  p.first = static_cast<int*>(take(MAX_CTAS * 4));
  p.rec = static_cast<int4*>(take(16 * static_cast<int64_t>(max_tokens)));
  p.items = static_cast<Item*>(take(items * static_cast<int64_t>(sizeof(Item))));
  // a run for every row, one more wherever an item ends within a row, and the prefixes'
  p.runs = static_cast<Run*>(take((2 * items + (n_seqs < max_tokens ? n_seqs : max_tokens)) * static_cast<int64_t>(sizeof(Run))));
  p.part = static_cast<uint32_t*>(take(4 * items * n_kv_heads));
  p.join = static_cast<int2*>(take(8 * (items * n_kv_heads + static_cast<int64_t>(max_tokens) * G * n_kv_heads / JOIN_ROWS)));
  p.order = static_cast<int*>(take(4 * static_cast<int64_t>(max_tokens)));
  p.own = static_cast<int2*>(take(8 * static_cast<int64_t>(max_tokens)));
  p.scratch = static_cast<int*>(take(4 * (5 * static_cast<int64_t>(n_seqs) + 5)));
  p.bytes = at;
  return p;
}
// Rows of partial results at most.  An entry of two tiles leaves some only where it is split: a boundary between CTAs
// makes two segments of at most 256 rows.  An item of one tile (at most one for every prefix, hence for every row) leaves
// two for each segment, its two halves of the blocks.
__host__ __device__ inline int64_t max_part_rows(int n_seqs, int n_kv_heads, int G, int max_tokens, int n_ctas) {
  const int64_t all = static_cast<int64_t>(max_tokens) * G, single = static_cast<int64_t>(TILE) * n_seqs;
  return 2 * n_kv_heads * (all < single ? all : single) + 4 * TILE * static_cast<int64_t>(n_ctas);
}

__host__ __device__ inline bool two_tiles(int n_tok, int G) { return n_tok > tokens_a_tile(G); }
// Where the blocks of kv head h of an item begin on the line.
__device__ __forceinline__ uint32_t blocks_begin(const Item& it, int h) {
  return it.cost + h * (it.blocks + OVERHEAD) + OVERHEAD;
}

}  // namespace shared_attn
}  // namespace dopr
