// shared_attn.cuh -- how a step's attention over the paged cache is split: what k_shared_plan.cu lays down and
// k_shared_attn.cu walks through.
//
// Tokens that read the same keys form an item: up to two tiles of 128 rows (G = q heads a kv head rows a token) with
// one list of keys, either a prefix (tokens of every row that names it) or a row's own keys (its new tokens, each up
// to itself).  An item and a kv head are a flat entry; the flat entries' keys, in blocks of 128, lie one after another
// on a line on which each entry also takes OVERHEAD steps, and every CTA takes an equal share of the line.  What a CTA
// has of an entry is a segment; it leaves partial softmax results (maximum, sum, weighted values) which the joining
// kernel adds up by token.
#pragma once

#include "device_common.cuh"
#include "internal.h"

namespace dopr {
namespace shared_attn {

constexpr int TILE = 128;   // rows of a tile
constexpr int BLOCK = 128;  // keys of a block
constexpr uint32_t OVERHEAD = 2;
constexpr int MAX_CTAS = 256;

struct alignas(16) Item {
  int tok;        // first token: of a row's own keys the token itself, of a prefix its place in `order`
  int n_tok;
  int row;        // table row whose keys these are
  int n_keys;
  uint32_t cost;  // where its first entry begins on the line
  int seen;       // own keys: how many the first token sees, one more each further one; at most 0: none
  int own;        // 1: own keys, 0: a prefix
  int pad;
};
struct alignas(16) Head {
  int tokens, n_items, n_flat;
  uint32_t share, total;  // of the line: a CTA's part, all of it
  int n_seqs, n_kv_heads, Hq, max_tokens, n_ctas, head_dim;  // what the plan was made for
  int pad;
};
__host__ __device__ inline bool made_for(const Head& h, const dopr_cache_layout& lay, int Hq, int max_tokens, int n_ctas) {
  return h.n_seqs == lay.n_seqs && h.n_kv_heads == lay.n_kv_heads && h.Hq == Hq && h.max_tokens == max_tokens &&
         h.n_ctas == n_ctas && h.head_dim == lay.head_dim;
}
struct Plan {
  Head* head;
  int* first;      // [MAX_CTAS] flat entry in which a CTA's share begins
  int4* rec;       // [tokens] prefix item and place in it, own item and place in it (-1: none)
  Item* items;
  uint32_t* part;  // [flat entry] first row of its partial results
  int* order;      // [tokens] tokens by prefix
  int* scratch;    // 6 * n_seqs + 1, of the plan kernel
  int64_t bytes;
};
__host__ __device__ inline int tokens_a_tile(int G) { return TILE / G; }
__host__ __device__ inline int64_t max_items(int n_seqs, int G, int max_tokens) {
  const int pair = 2 * tokens_a_tile(G);
  return 2 * (static_cast<int64_t>(max_tokens + pair - 1) / pair + (n_seqs < max_tokens ? n_seqs : max_tokens));
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
  p.part = static_cast<uint32_t*>(take(4 * items * n_kv_heads));
  p.order = static_cast<int*>(take(4 * static_cast<int64_t>(max_tokens)));
  p.scratch = static_cast<int*>(take(4 * (6 * static_cast<int64_t>(n_seqs) + 1)));
  p.bytes = at;
  return p;
}
// Rows of partial results at most: an item of one tile leaves two for a segment (its two halves of the keys), one of
// two tiles one; every token has at most two items, and every boundary between CTAs adds a segment.
__host__ __device__ inline int64_t max_part_rows(int Hq, int max_tokens, int n_ctas) {
  return 4 * static_cast<int64_t>(max_tokens) * Hq + 2 * TILE * static_cast<int64_t>(n_ctas);
}

__host__ __device__ inline uint32_t blocks_of(int n_keys) { return static_cast<uint32_t>(n_keys + BLOCK - 1) / BLOCK; }
__host__ __device__ inline bool two_tiles(int n_tok, int G) { return n_tok > tokens_a_tile(G); }
// Where the keys of kv head h of an item begin on the line, and the CTAs that have some.
__device__ __forceinline__ uint32_t keys_begin(const Item& it, uint32_t blocks, int h) {
  return it.cost + h * (blocks + OVERHEAD) + OVERHEAD;
}

}  // namespace shared_attn
}  // namespace dopr
