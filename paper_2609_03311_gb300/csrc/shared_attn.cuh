// shared_attn.cuh -- how a step's attention over the paged cache is split: what k_shared_plan.cu lays down and
// k_shared_attn.cu walks through.
//
// Tokens that read the same keys stand together in an item.  There are two kinds, by the rows (G = q heads a kv head rows
// a token) that share the keys:
//   tiles  up to two tiles of 128 rows for the 5th-generation tensor cores: the tokens of rows with one prefix, or
//          without, cut into items;
//   few    up to 16 rows for warp-level products: all tokens of a prefix that has no more; and the own keys of rows with
//          few new tokens, beside the tiles that read their prefix (a step of one token a row: the prefix is read by
//          tiles of many rows, each row's own keys by its own few) or by themselves where there is no prefix.
// An item's keys are a list of pages, as runs: the prefix's pages, which all its tokens see, then the own pages of its rows,
// as far as their last token in the item sees them; a token sees its own run's keys up to itself.  A page's place in the
// list is its place in the columns of the scores, so a token's keys are two intervals of columns.  128 columns are a block.
//
// Of few items a block is a piece of 16 columns, and a run's last piece is its last one with keys.
//
// An item and a kv head are a flat entry.  The flat entries of each kind lie one after another on a line, on which an entry
// takes a length for its start and end and one for each block, longer where rows see a part of it.  Some CTAs take the tiles, the others the few items; a CTA
// of the former, a warp of the latter takes the blocks that begin in an equal share of its line.  What it has of an entry is
// a segment; it leaves partial softmax results (maximum, sum, weighted values), which
// the joining kernel adds up by row, unless they are all that its rows have: then it gives the rows' results right away.
#pragma once

#include "device_common.cuh"
#include "internal.h"

namespace dopr {
namespace shared_attn {

constexpr int TILE = 128;   // rows of a tile
constexpr int FEW = 16;     // rows of a few item
constexpr int BLOCK = 128;  // columns of a block of tiles
constexpr int PIECE = 16;   // of few items
constexpr int MAX_CTAS = 256;
constexpr int JOIN_ROWS = 8;
// Rows of more parts than this are joined by two warps each, JOIN_ROWS / 2 of them at a time.  Attention of n queries of one
// document, with one warp and with two: 11 to 13 parts a row: n = 1 9.3 and 9.0 us, 16 15.6 and 14.6, 64 20.4 and 19.8; 9 or 10:
// 1 8.8 and 9.0, 64 20.2 and 19.4, but 100 39.0 and 41.2, 128 41.8 and 43.5 (more rows than the SMs hold at once, two warps each);
// 19: 64 46.1 and 44.1.
constexpr int PARTS_A_WARP = 10;
__host__ __device__ inline int rows_a_piece(int parts) { return parts > PARTS_A_WARP ? JOIN_ROWS / 2 : JOIN_ROWS; }
constexpr int WORKERS = 8;  // warps of a CTA that take few items
// Lengths on the lines.  Tiles, about 480 clocks each: a block of keys that all rows see, another block (masked, and often of
// one tile), an entry's start and end.  Few items, about 1.5 us of a warp each (a CTA's eight share the SM's part of the
// memory's rate): a piece; an entry's start and end.  Fitted to the CTAs' times: 2,880 clocks a whole block, 5,200 to 6,900
// another, 10,200 to 12,200 an entry.  Queries of 16 documents: 163 us; other blocks at 10: 164.5, 14: 168; entries at 14:
// 165, 26: 167.  Ragged documents: a few entry at 4 53.0 us, at 2 53.4.
// An entry of no more than UNCUT behind its start goes whole to the CTA that it begins in: 290 tokens of six queries on 55 keys 19.0
// us cut, 17.0 whole; at 36 ten entries of four blocks keep too many CTAs idle (15.5 to 19).
constexpr uint32_t WHOLE_BLOCK = 6, OTHER_BLOCK = 12, FEW_PIECE = 1, UNCUT = 24;
__host__ __device__ constexpr uint32_t entry_length(bool few) { return few ? 4 : 20; }
constexpr uint32_t FEW_PER_TILES = 4;  // a length of few items in those of tiles
constexpr uint32_t MIN_FEW_SHARE = 3;  // one token on 536 keys: 8.2 us; 2: 8.5 (more parts to join), 4: 8.9, 6: 9.5

// Time of joining a part by that of a length, of tiles and of few items: 20 rows over 13,295 keys, cut into 104 parts or 52: 21.0
// and 16.5 us; 120 rows over 7,994 keys: 22.8 and 20.
constexpr float TILES_JOIN = 0.8f, FEW_JOIN = 0.14f;

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
  uint32_t start;    // where its first entry begins on the line
  uint32_t blocks;
  // tiles: blocks that concern the first tile's rows: [0, end0); the second's: [0, prefix_blocks) and from begin1 on
  uint32_t end0, begin1, prefix_blocks;
  uint32_t flags;
};
enum : uint32_t {
  ITEM_FEW = 1,    // a few item
  ITEM_ALONE = 2,  // its tokens are in no other item
};
// What a CTA has of a flat entry, with what its warps need to know of the item and of the run that its first page lies in: a
// load each from here to the block table and to the rows.
struct alignas(16) Segment {
  int h;              // kv head
  uint32_t b0, b1;    // its blocks here
  int tok, n_tok, run, n_runs;
  int prefix_keys, pages;
  uint32_t end0, begin1, prefix_blocks;
  uint32_t flags;
  uint32_t part_row;  // first row of its partial results
  int run_at;         // of the item's: the run of its first page (few items: piece), and what is needed of it
  int run_row, run_off, run_pages, run_keys;
};
enum : uint32_t {
  SEG_TWO = 1,    // two tiles
  SEG_FEW = 2,
  SEG_WHOLE = 4,  // gives its rows' results right away
};
// Up to rows_a_piece rows of an entry that are to be added up from partial results.
struct alignas(16) Piece {
  int tok;            // of the entry's item
  int row, rows;      // the first of them, and all of the item's
  int h;              // kv head
  uint32_t part_row;  // of the item's first row
  int parts;          // an item's rows after another
  int beside;         // the rows' own keys may be in a few item
  int pad;
};
struct alignas(16) Head {
  int n_join;
  uint32_t few_share;  // of the few items' line: a warp's part
  int tile_ctas;              // the CTAs that take tiles
  // what the plan was made for: its runs' pages lie in tables of max_blocks entries a row
  int Hq, max_tokens, n_ctas;
  dopr_cache_layout lay;
};
__host__ __device__ inline bool made_for(const Head& h, const dopr_cache_layout& lay, int Hq, int max_tokens, int n_ctas) {
  return h.lay.n_blocks == lay.n_blocks && h.lay.page == lay.page && h.lay.n_kv_heads == lay.n_kv_heads &&
         h.lay.head_dim == lay.head_dim && h.lay.dtype == lay.dtype && h.lay.n_seqs == lay.n_seqs &&
         h.lay.max_blocks == lay.max_blocks && h.Hq == Hq && h.max_tokens == max_tokens && h.n_ctas == n_ctas;
}
constexpr int SHARES = MAX_CTAS * WORKERS + 2;  // at most: a CTA has one or WORKERS
struct Plan {
  Head* head;
  int2* work;      // [CTA][WORKERS] segments of a CTA of tiles (WORKERS times), of a few items' CTA's warps: from and to
  Segment* segs;   // in the CTAs' order
  int4* rec;       // [tokens] item of tiles and place in it, few item and place in it (-1: none)
  Item* items;
  Run* runs;
  uint32_t* part;  // [flat entry] first row of its partial results
  Piece* join;
  int* order;      // [2 * tokens] the items' tokens
  int2* own;       // [2 * tokens, in that order] columns of its own keys, from and to
  int* scratch;    // plan_scratch_ints(n_seqs), of the plan kernel where its shared memory does not hold them
  int64_t bytes;
};
__host__ __device__ inline int tokens_a_tile(int G) { return TILE / G; }
__host__ __device__ inline int tokens_a_few(int G) { return FEW / G; }  // 0: no few items
__host__ __device__ inline int64_t max_items(int n_seqs, int G, int max_tokens) {
  const int pair = 2 * tokens_a_tile(G), few = tokens_a_few(G);
  const int64_t rows = n_seqs < max_tokens ? n_seqs : max_tokens;
  // whole items and a last one a prefix, of each kind
  return (static_cast<int64_t>(max_tokens) + pair - 1) / pair + rows +
         (few > 0 ? (static_cast<int64_t>(max_tokens) + few - 1) / few + rows + 2 : 0);
}
// a run for every row, one more wherever an item ends within a row, and the prefixes'
__host__ __device__ inline int64_t max_runs(int n_seqs, int G, int max_tokens) {
  return 2 * (max_items(n_seqs, G, max_tokens) + (n_seqs < max_tokens ? n_seqs : max_tokens));
}
__host__ __device__ inline int64_t plan_scratch_ints(int64_t n_seqs) { return 15 * n_seqs + 8; }
__host__ __device__ inline int64_t max_pieces(int n_seqs, int n_kv_heads, int G, int max_tokens) {
  return max_items(n_seqs, G, max_tokens) * n_kv_heads + static_cast<int64_t>(max_tokens) * G * n_kv_heads / (JOIN_ROWS / 2);
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
  p.work = static_cast<int2*>(take(MAX_CTAS * WORKERS * 8));
  p.rec = static_cast<int4*>(take(16 * static_cast<int64_t>(max_tokens)));
  p.segs = static_cast<Segment*>(take((items * n_kv_heads + SHARES) * static_cast<int64_t>(sizeof(Segment))));
  p.items = static_cast<Item*>(take(items * static_cast<int64_t>(sizeof(Item))));
  p.runs = static_cast<Run*>(take(max_runs(n_seqs, G, max_tokens) * static_cast<int64_t>(sizeof(Run))));
  p.part = static_cast<uint32_t*>(take(4 * items * n_kv_heads));
  p.join = static_cast<Piece*>(take(max_pieces(n_seqs, n_kv_heads, G, max_tokens) * static_cast<int64_t>(sizeof(Piece))));
  p.order = static_cast<int*>(take(8 * static_cast<int64_t>(max_tokens)));
  p.own = static_cast<int2*>(take(16 * static_cast<int64_t>(max_tokens)));
  p.scratch = static_cast<int*>(take(4 * plan_scratch_ints(n_seqs)));
  p.bytes = at;
  return p;
}
// Rows of partial results, at most and with room to spare.  Of tiles, a token's rows are left once where they have a few item
// too (counted twice here), of few items once; a tile item holds the tokens of some row with few tokens or ends a prefix, so
// there is at most one for every row.  A boundary between CTAs makes one segment more, of at most 256 rows, or two of what would
// have given its rows' results right away.
__host__ __device__ inline int64_t max_part_rows(int n_seqs, int n_kv_heads, int G, int max_tokens, int n_ctas) {
  const int64_t all = static_cast<int64_t>(max_tokens) * G, n = n_seqs;
  const int64_t tiles = 2 * all < 4 * TILE * n ? 2 * all : 4 * TILE * n, few = all < FEW * n ? all : FEW * n;
  // so that the values behind the maxima and sums begin on 32 bytes where the workspace does
  return (n_kv_heads * (tiles + few) + 3) / 4 * 4 + 4 * TILE * static_cast<int64_t>(n_ctas);
}

__host__ __device__ inline bool two_tiles(const Item& it, int G) { return !(it.flags & ITEM_FEW) && it.n_tok > tokens_a_tile(G); }
// The blocks of kv head h's entry on the line: where the first begins, how many are whole, and where those end.
struct OnLine {
  uint32_t begin, whole, whole_end;
  bool few, uncut;  // uncut: all blocks count as where the first begins
  __host__ __device__ uint32_t begin_of(uint32_t b) const {
    if (few) return begin + b * FEW_PIECE;
    if (uncut) return begin;
    return b <= whole ? begin + b * WHOLE_BLOCK : whole_end + (b - whole) * OTHER_BLOCK;
  }
  // first block that begins at or behind a place on the line
  __host__ __device__ uint32_t block_from(uint32_t at, uint32_t blocks) const {
    if (at <= begin) return 0;
    if (uncut) return blocks;
    const uint32_t b = few ? (at - begin + FEW_PIECE - 1) / FEW_PIECE
                       : at <= whole_end ? (at - begin + WHOLE_BLOCK - 1) / WHOLE_BLOCK
                                         : whole + (at - whole_end + OTHER_BLOCK - 1) / OTHER_BLOCK;
    return b < blocks ? b : blocks;
  }
  __host__ __device__ uint32_t cta_of(uint32_t block, uint32_t share) const { return begin_of(block) / share; }
  __host__ __device__ uint32_t segments(uint32_t blocks, uint32_t share) const {
    return blocks > 0 ? cta_of(blocks - 1, share) - cta_of(0, share) + 1 : 0;
  }
};
__host__ __device__ inline OnLine blocks_from(const Item& it, uint32_t begin) {
  const uint32_t all = it.prefix_keys / BLOCK, whole = all < it.blocks ? all : it.blocks;
  return OnLine{begin, whole, begin + whole * WHOLE_BLOCK, (it.flags & ITEM_FEW) != 0, false};
}
__host__ __device__ inline uint32_t length_of(const Item& it) {
  return it.blocks > 0 ? blocks_from(it, entry_length(it.flags & ITEM_FEW)).begin_of(it.blocks) : 0;
}
__host__ __device__ inline OnLine on_line(const Item& it, int h) {
  const uint32_t length = length_of(it), head = entry_length(it.flags & ITEM_FEW);
  OnLine on = blocks_from(it, it.start + h * length + head);
  on.uncut = !on.few && length <= head + UNCUT;
  return on;
}

}  // namespace shared_attn
}  // namespace dopr
