// k_shared_attn.cu -- attention of a step's tokens over a paged cache (dopr_shared_attention): the keys of the row's
// prefix, then the row's own up to the token, on the 5th-generation tensor cores.
//
// softmax(scale q k^T) v over any split of the keys: a part gives its maximum score m, the sum l of exp(score - m) and
// the sum o of exp(score - m) v; parts add up as exp(m_i - m) l_i and exp(m_i - m) o_i with m the largest m_i.  A
// part itself runs over its keys block by block the same way.
//
// k_shared_attn, a persistent CTA an SM, walks over its share of the plan's line (shared_attn.cuh), which holds either
// tiles or few items.
//   Tiles: an item of two tiles gives each block of 128 columns to the softmax groups of the tiles that it concerns, a tile
//   each; of one tile, blocks go to the groups in turn, so that one softmax runs beside the other's products either way, and
//   the group of the last block adds the other's O to its own (left to the joining kernel as two parts, 120 rows over 7,994
//   keys took 20.4 us for 17.4, 47 documents' queries 31.9 for 28.3).
//     warp 0, 2  copy K and V blocks into two rings, page by page (TMA; a page's rows of a kv head lie together)
//     warp 1     issues S = Q K^T (128 x 128, 32-bit, in TMEM) and O += P V (P in TMEM over the S it came from)
//     warp 3     brings the rows of Q by TMA: eight tokens that follow one another, others one by one (the rows of a token
//                and kv head are the heads of a box); of a view that a tensor map does not take, with 16-byte copies
//     warps 4-7, 8-11  softmax, a thread a row: the maximum, then P; O is scaled only when the maximum grew by more than
//                2^8 (f16: 2^4; P stays within the type's range until then)
//   P is rounded to the inputs' type for its product with V, as the tensor cores take it; maxima, sums, O and parts stay in 32
//   bits, and a row's sum adds up P before the rounding.
//   2,048 rows of 32 heads over 16,384 keys: 346 us, 1.59 PFLOP/s (1.46 in calls that follow one another for seconds, under the
//   power limit).  A block of two tiles takes 2,700 clocks of which the tensor
//   cores work 2,050: a tile's S, softmax, P V and next S wait for one another (TMEM, full with two of S and of O, has no
//   room for a second S), so a second tile fills the gaps and P goes over in halves (371 us when it went as one).  64 rows of
//   a token over 32,768 keys: 43 us, 26 of them in the blocks; the rest is start, partial results, joining.
//   Few items: warps 4-11 each walk over a share of their own, with 16-row warp-level products and 16-byte copies: a 16-row
//   box by TMA takes about 80 ns of an SM (256 tokens over 64 ragged documents in pages of 16: 73 us by TMA, 63 with 16-byte
//   copies then; 51 now, 5.0 TB/s).
// Columns that a row does not see are left out by selection, not by arithmetic: what a page holds there cannot matter.
// Values would (0 x NaN), so rows of V past a run's keys are zero in shared memory.  A value that one token sees and
// another of the item does not would too: rows that end with a NaN though their scores have none are looked at when the CTA has
// done everything else.
//
// k_shared_join, a warp a row, adds the parts up.
#include <limits.h>

#include <type_traits>

#include "shared_attn.cuh"

namespace dopr {
namespace {
using namespace shared_attn;

constexpr int THREADS = 128 + 2 * 128;
// group w: S at S_COL + 128 w, P over its upper half, O at O_COL + 128 w
constexpr uint32_t TMEM_COLS = 512, S_COL = 0, P_COL = 64, O_COL = 256;
// P = 2^(score - m), and O is scaled when m falls behind the maximum by more than RESCALE.  bf16 has the range of 32 bits: m is a
// maximum.  f16 reaches from 2^-24 to 2^16: m is BELOW a maximum by 11, so that P takes the whole range up to 2^15 and a row's
// smallest probabilities are rounded to steps of 2^-35 of its largest (with m the maximum, 2^-24: 131,071 keys of 2^-26 of one
// other, which make up 0.2 % of the sum, counted as nothing).
template <typename T>
constexpr float RESCALE = std::is_same_v<T, __half> ? 4.f : 8.f;
template <typename T>
constexpr float BELOW = std::is_same_v<T, __half> ? 11.f : 0.f;
// of the joining kernel on an SM (3 with twice the loads on their way: 64 rows a little faster, 16 documents 3 % slower)
constexpr int JOIN_CTAS = 4;
constexpr int HALF_BYTES = 128 * 128;  // 128 rows of 64 16-bit elements

template <int D>
struct Smem {
  static constexpr int HALVES = D / 64;
  static constexpr int TILE_BYTES = HALVES * HALF_BYTES;
  static constexpr int K_STAGES = D == 128 ? 2 : 5, V_STAGES = D == 128 ? 3 : 5;
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = OFF_Q + 2 * TILE_BYTES;
  static constexpr int OFF_V = OFF_K + K_STAGES * TILE_BYTES;
  static constexpr int OFF_ROW = OFF_V + V_STAGES * TILE_BYTES;  // the Q gatherer's rows' tokens
  static constexpr int OFF_ML = OFF_ROW + 128 * 4;      // maxima and sums that one softmax group leaves to the other
  static constexpr int OFF_KEYS = OFF_ML + 128 * 8;     // of each page of a V stage: rows that hold keys
  static constexpr int OFF_BAR = OFF_KEYS + 64;
  // few items: from 0 on, pieces of 16 columns of K and V, F_STAGES of them a warp
  static constexpr int F_STAGES = D == 128 ? 3 : 6;
  static_assert(WORKERS * F_STAGES * 2 * HALVES * PIECE * 128 <= OFF_ROW, "the few items' pieces");
  static constexpr int K_FULL = 0, K_EMPTY = K_FULL + K_STAGES, V_FULL = K_EMPTY + K_STAGES, V_EMPTY = V_FULL + V_STAGES,
                       Q_FULL = V_EMPTY + V_STAGES, Q_EMPTY = Q_FULL + 2, S_FULL = Q_EMPTY + 2, P_FULL = S_FULL + 2,
                       O_FULL = P_FULL + 4, ML_FULL = O_FULL + 2, ML_EMPTY = ML_FULL + 1, DRAIN = ML_EMPTY + 1, N_BARS = DRAIN + 1;
  static constexpr int BYTES = 1024 + OFF_BAR + N_BARS * 8 + 16;
  static_assert(V_STAGES * 8 <= 64, "a byte a page");
  static_assert(BYTES <= 227 * 1024, "shared memory budget");
};

struct Ring {
  int stage = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int n) {
    if (++stage == n) {
      stage = 0;
      phase ^= 1u;
    }
  }
};

template <typename T>
__host__ __device__ constexpr uint32_t type_bits() {  // operand formats of the instruction descriptor: 0 f16, 1 bf16
  return std::is_same_v<T, __half> ? 0u : (1u << 7 | 1u << 10);
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if constexpr (std::is_same_v<T, __half>) return pack_f16x2(x, y);
  else return pack_bf16x2(x, y);
}
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (std::is_same_v<T, __half>) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  else return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w));
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two at once: a * b + c, a + b.
__device__ __forceinline__ void fma2(float& x, float& y, float ax, float ay, float b, float c) {
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\tmov.b64 c, {%5, %5};\n\t"
      "fma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(x), "=f"(y)
      : "f"(ax), "f"(ay), "f"(b), "f"(c));
}
__device__ __forceinline__ void add2(float& x, float& y, float bx, float by) {
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\tadd.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "+f"(x), "+f"(y)
      : "f"(bx), "f"(by));
}
// Shares of the launch's registers (384 threads x 168): little for the warps that copy and issue, more where rows of S
// are held (152 and 176: 2,048 rows 353 us for 351.7).
constexpr int REGS_FEW = 136, REGS_MANY = 184;
static_assert(128 * REGS_FEW + 256 * REGS_MANY <= 384 * 168, "more registers than the launch has are waited for without end");
__device__ __forceinline__ void regs_few() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW)); }
__device__ __forceinline__ void regs_many() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_MANY)); }
__device__ __forceinline__ void st_global32(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
               "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void fence_proxy_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// D (16 x 8, 32-bit) += A (16 x 16) B (16 x 8) of T by a warp.
template <typename T>
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same_v<T, __half>) {
    mma_f16_16816(d, a, b0, b1);
  } else {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
}
// What the chains of loads at the start run through, brought into L2 while the CTA sets up.  A line a thread of the grid; of
// larger calls, whose work is long, a part.
__device__ __forceinline__ void prefetch_l2(const SharedAttnArgs& a, const Plan& plan) {
  const int64_t at = (static_cast<int64_t>(threadIdx.x) * gridDim.x + blockIdx.x) * 128;
  const char* from = static_cast<const char*>(a.plan);
  if (at < reinterpret_cast<const char*>(plan.scratch) - from) asm volatile("prefetch.global.L2 [%0];" ::"l"(from + at));
  if (at < static_cast<int64_t>(a.lay.n_seqs) * a.lay.max_blocks * 4)
    asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const char*>(a.tables) + at));
}
// One segment after another of a share: of tiles a CTA's, of few items a warp's.
struct Walk {
  const Segment* segs;
  int at, end;
  __device__ __forceinline__ Walk(const Plan& p, int2 work) : segs(p.segs), at(work.x), end(work.y) {}
  __device__ __forceinline__ bool next(Segment& s) {
    if (at >= end) return false;
    s = segs[at++];
    if (at < end) asm volatile("prefetch.global.L1 [%0];" ::"l"(segs + at));
    return true;
  }
};
// The softmax groups that take a block (a bit each): those whose tile it concerns, or in turn over all one-tile
// segments of the CTA.
struct Groups {
  uint32_t turn = 0;
  __device__ __forceinline__ uint32_t of(const Segment& s, uint32_t b) {
    if (s.flags & SEG_TWO) return (b < s.end0 ? 1u : 0u) | (b < s.prefix_blocks || b >= s.begin1 ? 2u : 0u);
    const uint32_t g = 1u << turn;
    turn ^= 1u;
    return g;
  }
  // The groups that take any block of the segment; goes past it.
  __device__ __forceinline__ uint32_t any(const Segment& s) {
    if (s.flags & SEG_TWO) return (s.b0 < s.end0 ? 1u : 0u) | (s.b0 < s.prefix_blocks || s.b1 > s.begin1 ? 2u : 0u);
    const uint32_t n = s.b1 - s.b0, g = n > 1 ? 3u : 1u << turn;
    turn ^= n & 1u;
    return g;
  }
};
// The last block of the segment that group w takes, if it takes any (of one tile: the last but one is another's last).
__device__ __forceinline__ bool last_block(const Segment& s, uint32_t b, int w) {
  if (!(s.flags & SEG_TWO)) return b + 2 >= s.b1;
  if (w == 0) return b + 1 == min(s.b1, s.end0);
  return b + 1 == (s.b1 > s.begin1 ? s.b1 : min(s.b1, s.prefix_blocks));
}
// The first block of the segment that is some group's last.
__device__ __forceinline__ uint32_t first_last(const Segment& s) {
  if (!(s.flags & SEG_TWO)) return s.b1 < 2 ? 0 : s.b1 - 2;
  const uint32_t last0 = min(s.b1, s.end0), last1 = s.b1 > s.begin1 ? s.b1 : min(s.b1, s.prefix_blocks);
  return min(last0, last1) - 1;  // (of a group that takes none: at most the other's)
}
// A lane's page of each block and the run it lies in.
struct PageCursor {
  Run run;
  int at, n_runs;
  const Run* runs;
  __device__ __forceinline__ PageCursor(const Plan& p, const Segment& s) : at(s.run_at), n_runs(s.n_runs), runs(p.runs + s.run) {
    run.row = s.run_row, run.off = s.run_off, run.pages = s.run_pages, run.keys = s.run_keys;
  }
  __device__ __forceinline__ void go(int page) {
    while (page >= run.off + run.pages && at + 1 < n_runs) run = runs[++at];
  }
};
// Waits for the loads from tensor memory before it; the values pass through, so that nothing that uses them moves ahead.
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                 "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]),
                 "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]),
                 "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])::"memory");
}
__device__ __forceinline__ void max32(const uint32_t (&v)[32], float& top) {
  float t[4] = {top, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < 32; ++i) t[i & 3] = fmaxf(t[i & 3], __uint_as_float(v[i]));
  top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
}
// 2^(s scale - base) of 32 columns as pairs of T, their sum in sum.
template <typename T>
__device__ __forceinline__ void exp_pack(const uint32_t (&v)[32], float scale_log2, float base, float (&sum)[4], uint32_t (&pk)[16]) {
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    float x, y;
    fma2(x, y, __uint_as_float(v[i]), __uint_as_float(v[i + 1]), scale_log2, -base);
    x = ex2(x), y = ex2(y);
    add2(sum[i & 2], sum[(i & 2) + 1], x, y);
    pk[i / 2] = pack2<T>(x, y);
  }
}

// Bits [lo, hi) of a word, the range clipped to it.
__device__ __forceinline__ uint32_t bits_in(int lo, int hi) {
  lo = max(lo, 0);
  hi = min(hi, 32);
  if (hi <= lo) return 0u;
  return (hi >= 32 ? 0xffffffffu : (1u << hi) - 1u) & ~((1u << lo) - 1u);
}

__device__ __forceinline__ float inverse(float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : l; }  // a NaN stays one
__device__ __forceinline__ float lse_of(float m, float l) { return (m + log2f(l)) * 0.6931471805599453f; }

// O of the softmax group at o_col += O of the other one; the groups' maxima and sums before, theirs together after.  Not inlined,
// as what is rare should not stand between the blocks' loop and its instructions: with this and the loops over V's tails
// unrolled, queries of 16 documents took 169 us, so 160.
template <int D>
__device__ __noinline__ float2 add_other(uint32_t o_col, float2 mine, float2 other) {
  const float top = fmaxf(mine.x, other.x), base = top == -INFINITY ? 0.f : top;
  const float by = ex2(mine.x - base), other_by = ex2(other.x - base);
#pragma unroll 1
  for (int c = 0; c < D; c += 16) {
    uint32_t v[32], x[16];
    tmem_ld16x2(o_col + c, (o_col ^ 128u) + c, v);
    tmem_ld_wait_for(v);
    // a group that summed nothing up leaves no values
#pragma unroll
    for (int i = 0; i < 16; ++i)
      x[i] = __float_as_uint((mine.y != 0.f ? __uint_as_float(v[i]) * by : 0.f) +
                             (other.y != 0.f ? __uint_as_float(v[16 + i]) * other_by : 0.f));
    tmem_st16(o_col + c, x);
  }
  tmem_st_wait();
  return make_float2(top, mine.y * by + other.y * other_by);
}

// A row of a segment whose values hold a NaN though its scores have none, by a warp; lane l holds elements [E l, E l + E) of the
// head.  The NaN stands where it came from a value that the row sees.  It may also be of one that only other rows of the item
// see: the products take in all columns of a block, at a weight of zero, and zero times a NaN or an infinity is not zero.
// Prefix columns are seen by all rows, so only the other rows' own keys are looked through; where a value there is not finite, in
// an element that holds a NaN, those elements are summed up again over the row's columns alone, 32 at a time: a lane a key's
// score, then the values row by row.  That ends early where they are all NaN again.  Rare and slow, so nobody waits for it.
// place: of the row's token in `order`; part: the row of its partial result, -1: the results themselves.
template <typename T, int D>
__device__ __noinline__ void mend_row(const SharedAttnArgs& a, const Plan& plan, const Segment& s, int place, int h, int64_t part, int lane) {
  constexpr int E = D / 32, W = E / 2, AHEAD = 8;
  const int page = a.lay.page, Hkv = a.lay.n_kv_heads, G = a.Hq / Hkv, t = plan.order[place];
  const float2* ml = reinterpret_cast<const float2*>(a.ws);
  float2* part_o = reinterpret_cast<float2*>(a.ws + max_part_rows(a.lay.n_seqs, Hkv, G, a.max_tokens, gridDim.x) * 8 + part * (4 * D)) + lane * W;
  uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head) + lane * W;
  // a part that summed nothing up left no values; a NaN among the scores makes all of them NaN
  if (part >= 0 && !(ml[part].y > 0.f)) return;
  float2 o[W];
  bool nan = false;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    o[i] = part < 0 ? unpack2<T>(out[i]) : part_o[i];
    nan |= o[i].x != o[i].x || o[i].y != o[i].y;
  }
  if (!__any_sync(0xffffffffu, nan)) return;
  const int unit = s.flags & SEG_FEW ? PIECE : page, block = s.flags & SEG_FEW ? PIECE : BLOCK;
  const int c0 = s.b0 * block, c1 = s.b1 * block;  // the segment's columns
  const int2 own = plan.own[place];
  // of the table row's key p: its row among the pool's [pages][kv heads][page]
  auto row_of = [&](int row, int p) {
    int block = a.tables[static_cast<int64_t>(row) * a.lay.max_blocks + p / page];
    if (block < 0 || block >= a.lay.n_blocks) block = 0;
    return (block * Hkv + s.h) * page + p % page;
  };
  auto value = [&](int at, int i) {
    return unpack2<T>((static_cast<const uint32_t*>(a.v_pool) + static_cast<int64_t>(at) * (D / 2) + lane * W)[i]);
  };
  bool unseen = false;
  for (int j = 0; j < s.n_runs && !unseen; ++j) {
    const Run run = plan.runs[s.run + j];
    if (run.token < 0) continue;
    const int from = run.off * unit, end = min(run.keys, c1 - from);
    for (int p = max(0, c0 - from); p < end && !unseen; p += AHEAD) {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (p + i >= end || (from + p + i >= own.x && from + p + i < own.y)) continue;
        const int at = row_of(run.row, p + i);
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float2 v = value(at, e);
          bad |= (o[e].x != o[e].x && !isfinite(v.x)) || (o[e].y != o[e].y && !isfinite(v.y));
        }
      }
      unseen = __any_sync(0xffffffffu, bad);
    }
  }
  if (!unseen) return;
  const uint4* qp = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + t * a.q_tok + h * a.q_head);
  const float scale_log2 = a.scale * 1.4426950408889634f;
  float2 x[W];
#pragma unroll
  for (int i = 0; i < W; ++i) x[i] = make_float2(0.f, 0.f);
  float m = -INFINITY, l = 0.f;
  // (the row's own keys first, the prefix last: where a step's new values are bad, all of its rows end at once)
  for (int j = s.n_runs - 1; j >= 0; --j) {
    const Run run = plan.runs[s.run + j];
    const int from = run.off * unit;
    if (run.token >= 0 && (own.x >= own.y || from != own.x || run.keys == 0)) continue;
    const int end = min(run.token < 0 ? s.prefix_keys : own.y - own.x, c1 - from);
    for (int p0 = max(0, c0 - from); p0 < end; p0 += 32) {
      const int here = min(32, end - p0);
      const int at = row_of(run.row, p0 + min(lane, here - 1));
      const uint4* kp = reinterpret_cast<const uint4*>(static_cast<const T*>(a.k_pool) + static_cast<int64_t>(at) * D);
      float sc = 0.f;
#pragma unroll 4
      for (int c = 0; c < D / 8; ++c) {
        const uint4 w = kp[c], u = qp[c];
        const uint32_t ks[4] = {w.x, w.y, w.z, w.w}, qs[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = unpack2<T>(ks[i]), g = unpack2<T>(qs[i]);
          sc += f.x * g.x + f.y * g.y;
        }
      }
      sc = lane < here ? sc * scale_log2 : -INFINITY;
      float top = sc;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      top = fmaxf(top, m);
      const float base = top == -INFINITY ? 0.f : top, old = exp2f(m - base), e = exp2f(sc - base);
      m = top;
      l = l * old + warp_sum(e);
#pragma unroll
      for (int i = 0; i < W; ++i) x[i].x *= old, x[i].y *= old;
#pragma unroll 8
      for (int i = 0; i < here; ++i) {
        const float by = __shfl_sync(0xffffffffu, e, i);
        const int row = __shfl_sync(0xffffffffu, at, i);
#pragma unroll
        for (int c = 0; c < W; ++c) {
          const float2 v = value(row, c);
          x[c].x += by * v.x;
          x[c].y += by * v.y;
        }
      }
      bool open = false;
#pragma unroll
      for (int i = 0; i < W; ++i) open |= (o[i].x != o[i].x && x[i].x == x[i].x) || (o[i].y != o[i].y && x[i].y == x[i].y);
      if (!__any_sync(0xffffffffu, open)) return;
    }
  }
  // parts are relative to the maximum that they were left with
  const float by = part < 0 ? inverse(l) : exp2f(m - ml[part].x);
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if (o[i].x == o[i].x && o[i].y == o[i].y) continue;
    const float2 y = make_float2(o[i].x != o[i].x ? x[i].x * by : o[i].x, o[i].y != o[i].y ? x[i].y * by : o[i].y);
    if (part < 0) out[i] = pack2<T>(y.x, y.y);
    else part_o[i] = y;
  }
}

// The marked segments of a softmax group's warp (quarter 32 rows of group w's tile) or of a few items' warp.
template <typename T, int D>
__device__ __noinline__ void mend_segments(const SharedAttnArgs& a, const Plan& plan, uint32_t marked, int worker, int lane) {
  const int G = a.Hq / a.lay.n_kv_heads, TT = tokens_a_tile(G);
  const int2 work = plan.work[blockIdx.x * WORKERS + worker];
  for (int at = work.x; at < work.y; ++at) {
    if (!(marked >> (at & 31) & 1u)) continue;
    const Segment& s = plan.segs[at];
    const int t0 = s.flags & SEG_TWO ? worker / 4 * TT : 0, rows = min(TT, s.n_tok - t0) * G;
    const int first = s.flags & SEG_FEW ? 0 : worker % 4 * 32;
    for (int r = first; r < min(rows, first + 32); ++r)
      mend_row<T, D>(a, plan, s, s.tok + t0 + r / G, s.h * G + r % G,
                     s.flags & SEG_WHOLE ? -1 : static_cast<int64_t>(s.part_row) + t0 * G + r, lane);
  }
}

// A share of few items by one warp, a piece of 16 columns at a time, three or six of them on their way in shared memory of
// its own: what a warp waits for, the others do not.  Fragments of the products: a thread has rows lane / 4 and lane / 4 + 8
// of the item, and of each 8 columns two from 2 (lane % 4).  Bound by the copies of K and V: 8 KB a piece of head size 128,
// 1.5 us of an eighth of an SM's part of the memory's rate, of which the products and the softmax take a third.
template <typename T, int D>
__device__ __forceinline__ void few_items(const SharedAttnArgs& a, const Plan& plan, uint32_t s0, int wi, int2 work, uint32_t* marked, int lane) {
  using L = Smem<D>;
  constexpr int HALF = PIECE * 128, KV = L::HALVES * HALF;  // 64 elements a row; K or V of a piece
  constexpr int CHUNKS = D / 8;                             // 16-byte chunks of a row
  const uint32_t base = s0 + wi * L::F_STAGES * 2 * KV;
  const int Hkv = a.lay.n_kv_heads, G = a.Hq / Hkv, page = a.lay.page;
  const float scale_log2 = a.scale * 1.4426950408889634f;
  const int quad = lane >> 2, in_quad = lane & 3;
  // copies run ahead of the products, over the ends of segments too
  Walk copies(plan, work);
  Segment c;
  bool more = copies.next(c);
  uint32_t next = more ? c.b0 : 0;
  int stage = 0, ahead = 0;        // of the piece at hand, of the next one to be copied
  int row_at = 0, valid_at = 0;    // where the next 32 pieces lie: a lane a piece
  auto find = [&](uint32_t b) {
    if (b >= c.b1) return;
    PageCursor cur(plan, c);
    cur.go(b);
    const Run& run = cur.run;
    const int key = (static_cast<int>(b) - run.off) * PIECE;
    int block = a.tables[static_cast<int64_t>(run.row) * a.lay.max_blocks + key / page];
    if (block < 0 || block >= a.lay.n_blocks) {
      if (a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);
      block = 0;
    }
    row_at = (block * Hkv + c.h) * page + key % page;
    valid_at = min(PIECE, run.keys - key);
  };
  // rows past the run's keys come as zeros; a group of copies also where there is no piece left
  auto copy = [&] {
    if (more && next == c.b1) {
      more = copies.next(c);
      next = c.b0;
    }
    if (more) {
      const int at = (next - c.b0) & 31;
      if (at == 0) find(next + lane);
      const int64_t row = __shfl_sync(0xffffffffu, row_at, at);
      const int valid = __shfl_sync(0xffffffffu, valid_at, at);
      const uint4* k = static_cast<const uint4*>(a.k_pool) + row * CHUNKS + lane;
      const uint4* v = static_cast<const uint4*>(a.v_pool) + row * CHUNKS + lane;
      const int x = lane % CHUNKS;
      const uint32_t dst = base + ahead * 2 * KV + (x >> 3) * HALF;
#pragma unroll
      for (int i = 0; i < PIECE * CHUNKS / 32; ++i) {
        const int r = lane / CHUNKS + i * (32 / CHUNKS);
        const uint32_t at_row = dst + r * 128 + (((x & 7) ^ (r & 7)) << 4);
        cp_async16(at_row, k + 32 * i, r < valid);
        cp_async16(at_row + KV, v + 32 * i, r < valid);
      }
      ++next;
    }
    cp_async_commit();
    ahead = ahead + 1 == L::F_STAGES ? 0 : ahead + 1;
  };
#pragma unroll 1
  for (int i = 0; i + 1 < L::F_STAGES; ++i) copy();

  Walk walk(plan, work);
  Segment s;
  while (walk.next(s)) {
    const int rows = s.n_tok * G;
    uint32_t q[D / 16][4];
    int own0[2], own1[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = quad + 8 * i;
      const bool valid = r < rows;
      const int o = s.tok + (valid ? r / G : 0);
      const int2 own = plan.own[o];
      own0[i] = valid ? own.x : 0, own1[i] = valid ? own.y : 0;
      const uint32_t* src = reinterpret_cast<const uint32_t*>(static_cast<const T*>(a.q) + plan.order[o] * a.q_tok +
                                                              static_cast<int64_t>(s.h * G + (valid ? r % G : 0)) * a.q_head) + in_quad;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        q[k][i] = valid ? src[8 * k] : 0u;
        q[k][2 + i] = valid ? src[8 * k + 4] : 0u;
      }
    }
    float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    for (uint32_t b = s.b0; b < s.b1; ++b) {
      copy();
      asm volatile("cp.async.wait_group %0;" ::"n"(L::F_STAGES - 1) : "memory");
      __syncwarp();
      const uint32_t k0 = base + stage * 2 * KV, v0 = k0 + KV;
      const int col0 = b * PIECE, row8 = lane & 7;
      float sc[2][4];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        sc[t][0] = sc[t][1] = sc[t][2] = sc[t][3] = 0.f;
#pragma unroll
        for (int k = 0; k < D / 16; k += 2) {
          const int c = 2 * k + (lane >> 3);  // 16-byte piece of the key's row
          uint32_t x[4];
          ldmatrix_x4(k0 + (c >> 3) * HALF + (row8 + 8 * t) * 128 + (((c & 7) ^ row8) << 4), x[0], x[1], x[2], x[3]);
          mma16<T>(sc[t], q[k], x[0], x[1]);
          mma16<T>(sc[t], q[k + 1], x[2], x[3]);
        }
      }
      if (s.prefix_keys < col0 + PIECE) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int c = col0 + 8 * t + 2 * in_quad + (e & 1), i = e >> 1;
            if (!(c < s.prefix_keys || (c >= own0[i] && c < own1[i]))) sc[t][e] = -INFINITY;
          }
      }
      uint32_t p[4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float top = fmaxf(fmaxf(sc[0][2 * i], sc[0][2 * i + 1]), fmaxf(sc[1][2 * i], sc[1][2 * i + 1]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)) * scale_log2 - BELOW<T>;
        if (m[i] == -INFINITY) m[i] = top;  // nothing but zeros has been summed
        const bool grow = top > m[i] + RESCALE<T>;
        if (__any_sync(0xffffffffu, grow)) {
          const float by = grow ? ex2(m[i] - top) : 1.f;
          if (grow) m[i] = top;
          l[i] *= by;
#pragma unroll
          for (int d = 0; d < D / 8; ++d) o[d][2 * i] *= by, o[d][2 * i + 1] *= by;
        }
        const float at_m = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float x = ex2(fmaf(sc[t][2 * i], scale_log2, -at_m)), y = ex2(fmaf(sc[t][2 * i + 1], scale_log2, -at_m));
          l[i] += x + y;  // this thread's columns: the quad's four sums are added up at the end
          p[2 * t + i] = pack2<T>(x, y);
        }
      }
#pragma unroll
      for (int d = 0; d < D / 8; d += 2) {
        const int c = d + (lane >> 4), row = lane & 15;
        uint32_t x[4];
        ldmatrix_x4_trans(v0 + (c >> 3) * HALF + row * 128 + (((c & 7) ^ (row & 7)) << 4), x[0], x[1], x[2], x[3]);
        mma16<T>(o[d], p, x[0], x[1]);
        mma16<T>(o[d + 1], p, x[2], x[3]);
      }
      __syncwarp();  // every lane has read the stage
      if (++stage == L::F_STAGES) stage = 0;
    }
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = quad + 8 * i;
      float sum = l[i] + __shfl_xor_sync(0xffffffffu, l[i], 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      float all = 0.f;  // a NaN where one of the values is (or they are infinite both ways: no harm)
      if (s.flags & SEG_WHOLE) {
        const int t = r < rows ? plan.order[s.tok + r / G] : 0, h = s.h * G + r % G;
        const float inv = inverse(sum);
        uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head) + in_quad;
#pragma unroll
        for (int d = 0; d < D / 8; ++d) {
          const float x = sum == 0.f ? 0.f : o[d][2 * i] * inv, y = sum == 0.f ? 0.f : o[d][2 * i + 1] * inv;
          all += x + y;
          if (r < rows) dst[4 * d] = pack2<T>(x, y);
        }
        if (r < rows && a.lse && in_quad == 0) a.lse[static_cast<int64_t>(t) * a.Hq + h] = lse_of(m[i], sum);
      } else if (r < rows) {
        float2* ml = reinterpret_cast<float2*>(a.ws);
        float* part_o = reinterpret_cast<float*>(ml + max_part_rows(a.lay.n_seqs, Hkv, G, a.max_tokens, gridDim.x));
        const int64_t row = static_cast<int64_t>(s.part_row) + r;
        if (in_quad == 0) ml[row] = make_float2(m[i], sum);
        if (sum != 0.f) {
#pragma unroll
          for (int d = 0; d < D / 8; ++d) {
            all += o[d][2 * i] + o[d][2 * i + 1];
            *reinterpret_cast<float2*>(part_o + row * D + 8 * d + 2 * in_quad) = make_float2(o[d][2 * i], o[d][2 * i + 1]);
          }
        }
      }
      odd |= r < rows && all != all && sum > 0.f;
    }
    // scores in order, values not: perhaps a value that the row does not see
    if (__any_sync(0xffffffffu, odd) && lane == 0) *marked |= 1u << (walk.at - 1 & 31);
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(THREADS, 1)
    k_shared_attn(const __grid_constant__ CUtensorMap tm_q8, const __grid_constant__ CUtensorMap tm_q1,
                  const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const __grid_constant__ SharedAttnArgs a, const __grid_constant__ Plan plan) {
  using L = Smem<D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint32_t marked[WORKERS];  // of each of the warps 4-11: segments (modulo 32) that hold rows to be mended
  __shared__ int gave_up;  // stands for the error word of the bounded waits: a CTA gives up alone
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t s0 = smem_u32(smem);
  auto bar = [&](int i) { return s0 + L::OFF_BAR + 8u * static_cast<uint32_t>(i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::OFF_BAR + L::N_BARS * 8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int Hkv = a.lay.n_kv_heads, G = a.Hq / Hkv, TT = tokens_a_tile(G);
  int* err = &gave_up;

  // An ordinary launch: everything before it is complete.  What begins the chain of loads comes while the CTA sets up.
  pdl_trigger();
  const int2 work = plan.work[blockIdx.x * WORKERS + (warp >= 4 ? warp - 4 : 0)];
  const Head head = *plan.head;
  prefetch_l2(a, plan);
  if (threadIdx.x < WORKERS) marked[threadIdx.x] = 0;
  if (threadIdx.x == 0) {
    gave_up = 0;
    for (int i = 0; i < L::N_BARS; ++i) mbar_init(bar(i), (i >= L::P_FULL && i < L::P_FULL + 4) || i == L::ML_FULL || i == L::ML_EMPTY ? 4 : 1);
    fence_mbar_init();
    tma_prefetch_desc(&tm_q8);
    tma_prefetch_desc(&tm_q1);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  Segment s;
  const bool good = made_for(head, a.lay, a.Hq, a.max_tokens, gridDim.x);
  const bool few = static_cast<int>(blockIdx.x) >= head.tile_ctas;
  if (!good && threadIdx.x == 0 && a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);

  if (!good) {
  } else if (few) {
    if (warp >= 4) {
      regs_many();
      few_items<T, D>(a, plan, s0, warp - 4, work, &marked[warp - 4], lane);
    } else {
      regs_few();
    }
  } else if (warp == 0 || warp == 2) {
    // ======================= K and V blocks, page by page: a lane a page and half of the head
    regs_few();
    const bool is_v = warp == 2;
    const CUtensorMap* map = is_v ? &tm_v : &tm_k;
    Walk walk(plan, work);
      const int stages = is_v ? L::V_STAGES : L::K_STAGES, full = is_v ? L::V_FULL : L::K_FULL, empty = full + stages;
    const uint32_t ring0 = s0 + (is_v ? L::OFF_V : L::OFF_K);
    const int page = a.lay.page, page_blk = BLOCK / page;
    const int pg = lane / L::HALVES, half = lane % L::HALVES;  // pages of a block: at most 8
    Ring r;
    uint32_t armed = 0, parity = 0;
    bool ok = true;
    while (ok && walk.next(s)) {
      PageCursor cur(plan, s);
      for (uint32_t b = s.b0; b < s.b1; ++b) {
        const int first = b * page_blk, pages = min(page_blk, s.pages - first);
        const bool mine = pg < pages;
        int block = 0;
        if (mine) {
          cur.go(first + pg);
          block = a.tables[static_cast<int64_t>(cur.run.row) * a.lay.max_blocks + first + pg - cur.run.off];
          if (block < 0 || block >= a.lay.n_blocks) {
            if (a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);
            block = 0;
          }
        }
        if (!mbar_wait_warp(bar(empty + r.stage), r.phase ^ 1u, err, WAIT_TIMEOUT_NS)) {
          ok = false;
          break;
        }
        const uint32_t fb = bar(full + r.stage);
        if (is_v && mine && half == 0)
          smem[L::OFF_KEYS + r.stage * 8 + pg] = static_cast<uint8_t>(min(page, cur.run.keys - (first + pg - cur.run.off) * page));
        __syncwarp();
        if (lane == 0) mbar_arrive_expect_tx(fb, pages * page * 128 * L::HALVES);
        __syncwarp();
        if (mine)
          tma_load_2d(ring0 + r.stage * L::TILE_BYTES + half * HALF_BYTES + pg * page * 128, map, fb, half * 64,
                      (block * Hkv + s.h) * page);
        __syncwarp();
        armed |= 1u << r.stage;
        parity = (parity & ~(1u << r.stage)) | r.phase << r.stage;
        r.next(stages);
      }
    }
    if (!ok)  // copies in flight land before the CTA ends
      for (int i = 0; i < stages; ++i)
        if (armed >> i & 1u) mbar_wait_warp(bar(full + i), parity >> i & 1u, err, 100000000ull);
  } else if (warp == 1) {
    // ======================= MMA issuer
    regs_few();
    const bool one = elect_one();
    const uint32_t sQ = s0 + L::OFF_Q, sK = s0 + L::OFF_K, sV = s0 + L::OFF_V;
    const int page = a.lay.page, page_blk = BLOCK / page;
    Walk walk(plan, work);
    Groups groups;
    bool ok = true;
    auto wait = [&](int b, uint32_t par) { return ok = ok && mbar_wait_warp(bar(b), par, err, WAIT_TIMEOUT_NS); };
    constexpr uint32_t idesc_o = umma_idesc_f16_bmn(TILE, D) | type_bits<T>();
    const uint64_t v_desc0 = umma_desc_sw128_mn(sV, HALF_BYTES, 1024), k_desc0 = umma_desc_sw128(sK), q_desc0 = umma_desc_sw128(sQ);
    uint32_t p_par = 0, q_par = 0;  // a bit a group

    // products P V that wait for their softmax, oldest first; at most one a group
    enum : uint32_t { FIRST = 1, LAST = 2, FREE_V = 4, FREE_K = 8 };
    struct Pending {
      int stage, cols;
      uint32_t phase, flags;  // FIRST, LAST of the group's segment, FREE_V: last use of the stage
      bool there;             // V has been seen to be
    } pend0{}, pend1{};
    uint32_t oldest = 0;
    int n_pend = 0;
    int freed[2] = {-1, -1};  // V stages that are free after the products issued: committed with the S behind them
    auto issue_pv = [&] {
      const uint32_t w = oldest;
      const Pending x = w ? pend1 : pend0;
      oldest ^= 1u;
      --n_pend;
      if (!x.there && !wait(L::V_FULL + x.stage, x.phase)) return;
      if (!wait(L::P_FULL + 2 + w, p_par >> w & 1u) || !wait(L::P_FULL + w, p_par >> w & 1u)) return;
      p_par ^= 1u << w;
      tc_fence_after();
      const uint64_t vd = v_desc0 + x.stage * (L::TILE_BYTES / 16);
      const uint32_t o = tmem + O_COL + 128 * w, pc = tmem + P_COL + 128 * w;
      if (one) {
        // (a loop of unknown length takes 115 clocks a product, one spelled out 26)
#pragma unroll
        for (int k = 0; k < BLOCK / 16; ++k)
          if (16 * k < x.cols) umma_f16_ts(o, pc + 8 * k, vd + k * (2048 / 16), idesc_o, k > 0 || !(x.flags & FIRST));
        if (x.flags & LAST) umma_commit(bar(L::O_FULL + w));
      }
      if (x.flags & FREE_V) freed[freed[0] >= 0] = x.stage;
    };
    auto commit_pv = [&] {
      if (one) {
        if (freed[0] >= 0) umma_commit(bar(L::V_EMPTY + freed[0]));
        if (freed[1] >= 0) umma_commit(bar(L::V_EMPTY + freed[1]));
      }
      freed[0] = freed[1] = -1;
    };
    // the next S: a block and a group that takes it
    Ring rk, rv;
    uint32_t b = 0, takes = 0, begun = 0;
    struct Next {
      uint32_t w, flags;
      int cols;
      bool valid, there;  // there: K, and Q where it is the first, have been seen to be
    } n{};
    bool in_segment = false, any_block = false;
    auto look = [&] {
      if (takes == 0) {
        if (!in_segment || ++b == s.b1) {
          n.valid = in_segment = walk.next(s);
          if (!n.valid) return;
          b = s.b0;
          begun = 0;
        }
        if (any_block) {
          rk.next(L::K_STAGES);
          rv.next(L::V_STAGES);
        }
        any_block = true;
        takes = groups.of(s, b);
        n.cols = min(page_blk, s.pages - static_cast<int>(b) * page_blk) * page;
      }
      n.w = takes & 1u ? 0 : 1;
      takes &= ~(1u << n.w);
      n.flags = (begun >> n.w & 1u ? 0 : FIRST) | (last_block(s, b, n.w) ? LAST : 0) | (takes == 0 ? FREE_V | FREE_K : 0);
      begun |= 1u << n.w;
      n.there = mbar_test_warp(bar(L::K_FULL + rk.stage), rk.phase);
      if (n.there && (n.flags & FIRST)) n.there = mbar_test_warp(bar(L::Q_FULL + n.w), q_par >> n.w & 1u);
      n.valid = true;
    };
    // One group's P V of an earlier block and S of a later one, all columns whole, the products back to back: the issuing
    // warp has few instruction slots beside the softmax, and a commit returns when the products before it are under way,
    // so what can be found out about the next step is, before the commits.
    bool v_there = false;
    auto step = [&](uint32_t w, int v_stage, bool acc, int k_stage, bool k_there, uint32_t k_phase, bool frees) {
      if (!wait(L::P_FULL + 2 + w, p_par >> w & 1u)) return;
      tc_fence_after();
      const uint32_t o = tmem + O_COL + 128 * w, sd = tmem + S_COL + 128 * w;
      const uint64_t vd = v_desc0 + v_stage * (L::TILE_BYTES / 16), kd = k_desc0 + k_stage * (L::TILE_BYTES / 16),
                     qd = q_desc0 + w * (L::TILE_BYTES / 16);
      if (one) {
#pragma unroll
        for (int k = 4; k < 8; ++k) umma_f16_ts(o, sd + (P_COL - S_COL) + 8 * k, vd + k * (2048 / 16), idesc_o, k > 4 || acc);
      }
      if (!wait(L::P_FULL + w, p_par >> w & 1u)) return;
      p_par ^= 1u << w;
      tc_fence_after();
      if (one) {
#pragma unroll
        for (int k = 0; k < 4; ++k) umma_f16_ts(o, sd + (P_COL - S_COL) + 8 * k, vd + k * (2048 / 16), idesc_o, true);
      }
      if (!k_there) {
        if (!wait(L::K_FULL + k_stage, k_phase)) return;
        tc_fence_after();
      }
      if (one) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const int off = ((k >> 2) * HALF_BYTES + (k & 3) * 32) / 16;
          umma_f16(sd, qd + off, kd + off, umma_idesc_f16(TILE, BLOCK) | type_bits<T>(), k > 0);
        }
      }
      v_there = mbar_test_warp(bar(L::V_FULL + rv.stage), rv.phase);
      if (one) {
        umma_commit(bar(L::S_FULL + w));
        if (frees) {
          umma_commit(bar(L::V_EMPTY + v_stage));
          umma_commit(bar(L::K_EMPTY + k_stage));
        }
      }
    };
    Next m{};
    int k_stage = -1;  // >= 0: S of m has been issued and not committed
    while (ok) {
      look();
      if (k_stage >= 0) {
        if (one) {
          umma_commit(bar(L::S_FULL + m.w));
          if (m.flags & FREE_K) umma_commit(bar(L::K_EMPTY + k_stage));
          if (m.flags & LAST) umma_commit(bar(L::Q_EMPTY + m.w));
        }
        k_stage = -1;
        commit_pv();
      }
      // whole blocks of the prefix, but for each group's first and last, which the general steps take
      const uint32_t margin = s.flags & SEG_TWO ? 1 : 2;
      const uint32_t hot = min(static_cast<uint32_t>(s.prefix_keys) / BLOCK, first_last(s));
      if (n.valid && b == s.b0 + margin && b < hot && (!(s.flags & SEG_TWO) || n.w == 0)) {
        Pending x = oldest ? pend1 : pend0, y = oldest ? pend0 : pend1;  // of two tiles: the same block
        bool k_there = n.there;
        if (!(s.flags & SEG_TWO)) groups.turn ^= 1u;  // back to before the block
        for (;;) {
          if (!x.there && !wait(L::V_FULL + x.stage, x.phase)) break;
          if (s.flags & SEG_TWO) {
            step(0, x.stage, !(x.flags & FIRST), rk.stage, k_there, rk.phase, false);
            if (ok) step(1, x.stage, !(x.flags & FIRST), rk.stage, true, 0, true);
          } else {
            step(oldest, x.stage, !(x.flags & FIRST), rk.stage, k_there, rk.phase, true);
          }
          if (!ok) break;
          const Pending z{rv.stage, BLOCK, rv.phase, FREE_V, v_there};
          x = s.flags & SEG_TWO ? z : y;
          y = z;
          if (!(s.flags & SEG_TWO)) {
            oldest ^= 1u;
            groups.turn ^= 1u;
          }
          if (b + 1 >= hot) break;
          ++b;
          rk.next(L::K_STAGES);
          rv.next(L::V_STAGES);
          k_there = mbar_test_warp(bar(L::K_FULL + rk.stage), rk.phase);
        }
        if (!ok) break;
        (oldest ? pend1 : pend0) = x;
        (oldest ? pend0 : pend1) = y;
        if (s.flags & SEG_TWO) pend0.flags &= ~FREE_V;
        takes = 0;
        continue;
      }
      // S of a group goes over its P: the product with it, and those before that, first
      while (ok && n_pend > 0 && (!n.valid || oldest == n.w || n_pend == 2)) issue_pv();
      if (!ok || !n.valid) break;
      m = n;
      if (!m.there) {
        commit_pv();
        if (m.flags & FIRST) wait(L::Q_FULL + m.w, q_par >> m.w & 1u);
        if (!wait(L::K_FULL + rk.stage, rk.phase)) break;
      }
      if (m.flags & FIRST) q_par ^= 1u << m.w;
      tc_fence_after();
      k_stage = rk.stage;
      if (one) {
        const uint64_t qd = q_desc0 + m.w * (L::TILE_BYTES / 16), kd = k_desc0 + k_stage * (L::TILE_BYTES / 16);
        const uint32_t idesc = umma_idesc_f16(TILE, m.cols) | type_bits<T>(), sd = tmem + S_COL + 128 * m.w;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const int off = ((k >> 2) * HALF_BYTES + (k & 3) * 32) / 16;
          umma_f16(sd, qd + off, kd + off, idesc, k > 0);
        }
      }
      const Pending x{rv.stage, m.cols, rv.phase, m.flags, mbar_test_warp(bar(L::V_FULL + rv.stage), rv.phase)};
      (m.w ? pend1 : pend0) = x;
      if (n_pend++ == 0) oldest = m.w;
    }
    commit_pv();
    if (one) umma_commit(bar(L::DRAIN));
    mbar_wait_warp(bar(L::DRAIN), 0, err, ok ? WAIT_TIMEOUT_NS : 100000000ull);
  } else if (warp == 3) {
    // ======================= rows of Q: row r of a group's tile is token r / G of the tile, head r % G of the kv head's
    regs_few();
    int* row = reinterpret_cast<int*>(smem + L::OFF_ROW);  // tokens of the rows
    Walk walk(plan, work);
    Groups groups;
    uint32_t used = 0, par = 0, filled = 0;  // a bit a group
    bool ok = true;
    const T* q = static_cast<const T*>(a.q);
    while (ok && walk.next(s)) {
      const uint32_t takes = groups.any(s);
      for (int w = 0; w < 2 && ok; ++w) {
        if (!(takes >> w & 1u)) continue;
        const int t0 = s.flags & SEG_TWO ? w * TT : 0, n = min(TT, s.n_tok - t0), rows = n * G;
        // tokens 8 i .. 8 i + 7 of the tile, a lane an i: whether they follow one another
        const int* tok = plan.order + s.tok + t0;
        int first = 0;
        bool run = a.q_boxes && 8 * lane + 8 <= n;
        if (run) {
          first = tok[8 * lane];
#pragma unroll
          for (int i = 1; i < 8; ++i) run = run & (tok[8 * lane + i] == first + i);
        }
        const uint32_t runs = __ballot_sync(0xffffffffu, run);
        for (int r = lane; !a.q_boxes && r < rows; r += 32) row[r] = tok[r / G];
        __syncwarp();
        if ((used >> w & 1u) && !mbar_wait_warp(bar(L::Q_EMPTY + w), par >> w & 1u, err, WAIT_TIMEOUT_NS)) {
          ok = false;
          break;
        }
        if (used >> w & 1u) par ^= 1u << w;
        used |= 1u << w;
        const uint32_t dst = s0 + L::OFF_Q + w * L::TILE_BYTES;
        if (a.q_boxes) {
          if (lane == 0) mbar_expect_tx(bar(L::Q_FULL + w), rows * 128 * L::HALVES);
          __syncwarp();
          if (run)
#pragma unroll
            for (int h = 0; h < L::HALVES; ++h)
              tma_load_3d(dst + h * HALF_BYTES + lane * 8 * G * 128, &tm_q8, bar(L::Q_FULL + w), 64 * h, s.h * G, first);
          // the others one by one (the swizzle goes by the address, so a box may begin at any row)
#pragma unroll 1
          for (int i = lane; i < n; i += 32) {
            if (runs >> (i / 8) & 1u) continue;
            const int t = tok[i];
#pragma unroll
            for (int h = 0; h < L::HALVES; ++h)
              tma_load_3d(dst + h * HALF_BYTES + i * G * 128, &tm_q1, bar(L::Q_FULL + w), 64 * h, s.h * G, t);
          }
          __syncwarp();
        } else {
          // a lane a 16-byte piece of the row, 32 / CHUNKS rows at once
          constexpr int CHUNKS = D / 8, STEP = 32 / CHUNKS;
          const int c = lane % CHUNKS;
          for (int r0 = lane / CHUNKS; r0 < rows; r0 += 8 * STEP) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int r = r0 + i * STEP;
              if (r < rows)
                cp_async16(dst + (c >> 3) * HALF_BYTES + r * 128 + (((c & 7) ^ (r & 7)) << 4),
                           q + row[r] * a.q_tok + static_cast<int64_t>(s.h * G + r % G) * a.q_head + 8 * c, true);
            }
          }
          cp_async_commit();
          cp_async_wait_all();
          fence_proxy_async_shared();
          __syncwarp();
        }
        if (lane == 0) mbar_arrive(bar(L::Q_FULL + w));
        filled ^= 1u << w;
      }
    }
    if (ld_volatile(err))  // copies in flight land before the CTA ends
      for (int w = 0; w < 2; ++w)
        if (used >> w & 1u) mbar_wait_warp(bar(L::Q_FULL + w), (filled >> w & 1u) ^ 1u, err, 100000000ull);
  } else {
    // ======================= softmax: thread r of group w has row r of its tile
    regs_many();
    const int w = (warp >> 2) - 1, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lane_base = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    const uint32_t s_col = lane_base + S_COL + 128 * w, o_col = lane_base + O_COL + 128 * w;
    const float scale_log2 = a.scale * 1.4426950408889634f;
    const int2* own_columns = plan.own;
    const int* order = plan.order;
    Walk walk(plan, work);
    Groups groups;
    Ring rv;
    uint32_t s_par = 0, o_par = 0;
    bool ok = true;
    // (the first group that takes a block) rows of V past a page's keys count as zero: before any of P is given
    auto ready_v = [&](int stage, uint32_t phase, int cols) {
      if (!mbar_wait_warp(bar(L::V_FULL + stage), phase, err, WAIT_TIMEOUT_NS)) return false;
      const int page = a.lay.page;
#pragma unroll 1
      for (int pg = 0; pg * page < cols; ++pg) {
        const int from = smem[L::OFF_KEYS + stage * 8 + pg];
#pragma unroll 1
        for (int i = r; i < (page - from) * 8 * L::HALVES; i += 128) {
          const int at = pg * page + from + i / (8 * L::HALVES), c = i % (8 * L::HALVES);
          *reinterpret_cast<uint4*>(smem + L::OFF_V + stage * L::TILE_BYTES + (c >> 3) * HALF_BYTES + at * 128 + (c & 7) * 16) =
              uint4{0, 0, 0, 0};
        }
      }
      fence_proxy_async_shared();
      return true;
    };
    // P is given in halves, the upper first: the products with it run while the other is made.  A barrier each: a warp may
    // give its second half before another gives its first.
    auto give = [&](int half) {
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(L::P_FULL + 2 * half + w));
    };
    // The group that took the last block of a segment of one tile adds the other's O to its own; the other begins a new one
    // when that is done.  In o_par beside O's parity, where the blocks' loop has no register to spare: that of such sums, and
    // whether this group left its O to the other.
    constexpr uint32_t SUMS = 2, LEFT = 4;
    while (ok && walk.next(s)) {
      if (o_par & LEFT) {
        if (!mbar_wait_warp(bar(L::ML_EMPTY), (o_par & SUMS) == 0, err, WAIT_TIMEOUT_NS)) break;
        o_par &= ~LEFT;
      }
      const int t0 = s.flags & SEG_TWO ? w * TT : 0, n = min(TT, s.n_tok - t0);
      const bool valid = r < n * G, any = __any_sync(0xffffffffu, valid);
      // the row sees columns [0, prefix) and [own0, own1)
      const int prefix = valid ? s.prefix_keys : 0;
      int own0 = 0, own1 = 0, token = 0;
      if (valid) {
        token = order[s.tok + t0 + r / G];
        const int2 own = own_columns[s.tok + t0 + r / G];
        own0 = own.x, own1 = own.y;
      }
      float m = -INFINITY, l = 0.f;
      int done = 0;
      for (uint32_t b = s.b0; b < s.b1 && ok; ++b) {
        const uint32_t takes = groups.of(s, b);
        const int v_stage = rv.stage;
        const uint32_t v_phase = rv.phase;
        rv.next(L::V_STAGES);
        if (!(takes >> w & 1u)) continue;
        if (!mbar_wait_warp(bar(L::S_FULL + w), s_par, err, WAIT_TIMEOUT_NS)) {
          ok = false;
          break;
        }
        s_par ^= 1u;
        ++done;
        tc_fence_after();
        const int key0 = b * BLOCK, cols = min(BLOCK, s.pages * a.lay.page - key0);
        const bool whole = s.prefix_keys - key0 >= BLOCK, ragged = !whole && !((s.flags & SEG_TWO) && w == 1 && (takes & 1u));
        const bool sees = valid && (prefix > key0 || (own1 > key0 && own0 < key0 + cols && own1 > own0));
        if (!__any_sync(0xffffffffu, sees)) {  // nothing here for this warp's rows; lanes that are no rows reach none
          const uint32_t zero[16] = {};
          if (any)
            for (int c = 0; c < 64; c += 16) tmem_st16(s_col + 64 + c, zero);
          if (ragged && !(ok = ready_v(v_stage, v_phase, cols))) break;
          give(1);
          give(0);
          continue;
        }
        uint32_t va[32], vb[32], pk[16];
        if (!whole) {
          // columns that a row does not see: -inf in their place (also past the block's last, where S holds anything)
#pragma unroll 1
          for (int c = 0; c < BLOCK; c += 32) {
            const int at = key0 + c;
            const uint32_t seen = bits_in(-at, prefix - at) | bits_in(own0 - at, own1 - at);
            if (__all_sync(0xffffffffu, seen == 0xffffffffu)) continue;
            tmem_ld32(s_col + c, va);
            tmem_ld_wait_for(va);
#pragma unroll
            for (int k = 0; k < 32; k += 16) {
#pragma unroll
              for (int i = 0; i < 16; ++i) pk[i] = seen >> (k + i) & 1u ? va[k + i] : 0xff800000u;
              tmem_st16(s_col + c + k, pk);
            }
          }
          tmem_st_wait();
        }
        // S is read twice, 32 columns at a time with the next ones on their way: first for the maximum, upwards, then
        // for P, downwards, where the last 64 are still held.  P of columns [32 c, 32 c + 32) goes to 64 + 16 c, over
        // columns that are read by then.
        float top = -INFINITY;
        tmem_ld32(s_col, va);
        tmem_ld_wait_for(va);
        tmem_ld32(s_col + 32, vb);
        max32(va, top);
        tmem_ld_wait_for(vb);
        tmem_ld32(s_col + 64, va);
        max32(vb, top);
        tmem_ld_wait_for(va);
        tmem_ld32(s_col + 96, vb);
        max32(va, top);
        tmem_ld_wait_for(vb);
        max32(vb, top);
        top = top * scale_log2 - BELOW<T>;
        if (m == -INFINITY) m = top;  // nothing but zeros has been summed
        const bool grow = top > m + RESCALE<T>;
        if (__any_sync(0xffffffffu, grow)) {
          // S is complete, so every product issued before it is: O stands still
          const float by = grow ? ex2(m - top) : 1.f;
          if (grow) m = top;
          l *= by;
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t v[32], x[16];
            tmem_ld32(o_col + c, v);
            tmem_ld_wait_for(v);
#pragma unroll
            for (int k = 0; k < 32; k += 16) {
#pragma unroll
              for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(__uint_as_float(v[k + i]) * by);
              tmem_st16(o_col + c + k, x);
            }
          }
        }
        const float base = m == -INFINITY ? 0.f : m;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        exp_pack<T>(vb, scale_log2, base, sum, pk);
        tmem_ld32(s_col + 32, vb);
        tmem_st16(s_col + 112, pk);
        exp_pack<T>(va, scale_log2, base, sum, pk);
        tmem_ld_wait_for(vb);
        tmem_ld32(s_col, va);
        tmem_st16(s_col + 96, pk);
        if (ragged && !(ok = ready_v(v_stage, v_phase, cols))) break;
        give(1);
        exp_pack<T>(vb, scale_log2, base, sum, pk);
        tmem_ld_wait_for(va);
        tmem_st16(s_col + 80, pk);
        exp_pack<T>(va, scale_log2, base, sum, pk);
        tmem_st16(s_col + 64, pk);
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        give(0);
      }
      if (!ok) break;
      if (done > 0) {
        if (!mbar_wait_warp(bar(L::O_FULL + w), o_par & 1u, err, WAIT_TIMEOUT_NS)) break;
        o_par ^= 1u;
        tc_fence_after();
      }
      // what only the end of a segment needs is read again here, not held in registers over its blocks
      const Segment& e = walk.segs[walk.at - 1];
      if (!(e.flags & SEG_TWO)) {
        float2* ml = reinterpret_cast<float2*>(smem + L::OFF_ML);
        const bool last = groups.turn != static_cast<uint32_t>(w), both = e.b1 - e.b0 > 1;
        if (both && !last) {
          ml[r] = make_float2(m, l);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(L::ML_FULL));
          o_par |= LEFT;
        } else if (both) {
          if (!mbar_wait_warp(bar(L::ML_FULL), (o_par & SUMS) != 0, err, WAIT_TIMEOUT_NS)) break;
          tc_fence_after();
          const float2 sum = add_other<D>(o_col, make_float2(m, l), ml[r]);
          m = sum.x, l = sum.y;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(L::ML_EMPTY));
        }
        if (both) o_par ^= SUMS;
        if (!last) continue;
      }
      float all = 0.f;  // the values' sum: a NaN where one of them is (or they are infinite both ways: no harm)
      if (e.flags & SEG_WHOLE) {
        // ---- the whole entry: the rows' results
        const int t = token, h = e.h * G + r % G;
        const float inv = inverse(l);
        T* dst = static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head;
        const bool wide = ((reinterpret_cast<uintptr_t>(a.out) | a.o_tok * 2 | a.o_head * 2) & 31) == 0;  // a store a sector
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t v[32] = {};
          if (done > 0) {
            tmem_ld32(o_col + c, v);
            tmem_ld_wait_for(v);
          }
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float x = l == 0.f ? 0.f : __uint_as_float(v[i]) * inv;
            all += x;
            v[i] = __float_as_uint(x);
          }
          if (valid) {
#pragma unroll
            for (int i = 0; i < 32; i += 16) {
              uint32_t x[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) x[k] = pack2<T>(__uint_as_float(v[i + 2 * k]), __uint_as_float(v[i + 2 * k + 1]));
              if (wide) {
                st_global32(dst + c + i, x);
              } else {
                *reinterpret_cast<uint4*>(dst + c + i) = uint4{x[0], x[1], x[2], x[3]};
                *reinterpret_cast<uint4*>(dst + c + i + 8) = uint4{x[4], x[5], x[6], x[7]};
              }
            }
          }
        }
        if (valid && a.lse) a.lse[static_cast<int64_t>(t) * a.Hq + h] = lse_of(m, l);
      } else {
        // ---- a partial result
        float2* ml = reinterpret_cast<float2*>(a.ws);
        float* part_o = reinterpret_cast<float*>(ml + max_part_rows(a.lay.n_seqs, Hkv, G, a.max_tokens, gridDim.x));
        const bool two = e.flags & SEG_TWO;
        const int64_t row = static_cast<int64_t>(e.part_row) + (two ? w * TT * G : 0) + r;
        if (valid) ml[row] = make_float2(m, l);
        float* dst = part_o + row * D;
#pragma unroll 1
        for (int c = 0; c < D && done > 0; c += 32) {
          uint32_t v[32];
          tmem_ld32(o_col + c, v);
          tmem_ld_wait_for(v);
          if (valid && l != 0.f) {  // (a NaN is not)
#pragma unroll
            for (int i = 0; i < 32; ++i) all += __uint_as_float(v[i]);
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
              const uint32_t x[8] = {v[i], v[i + 1], v[i + 2], v[i + 3], v[i + 4], v[i + 5], v[i + 6], v[i + 7]};
              st_global32(dst + c + i, x);
            }
          }
        }
      }
      // scores in order, values not: perhaps a value that the row does not see
      if (__any_sync(0xffffffffu, valid && all != all && l > 0.f) && lane == 0) marked[warp - 4] |= 1u << (walk.at - 1 & 31);
      tc_fence_before();
    }
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0 && gave_up && a.status) atomicCAS(a.status, 0, DOPR_ERR_TIMEOUT);
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc(tmem, TMEM_COLS);
  }
  // nobody waits for anybody any more
  if (warp >= 4 && marked[warp - 4] != 0) mend_segments<T, D>(a, plan, marked[warp - 4], warp - 4, lane);
}

// ------------------------------------------------------------------ joining the parts
// A warp a row, JOIN_ROWS rows of an entry at a time, or two warps a row of many parts.  Bound by latency where few rows have
// many parts, so what the plan says of a CTA's first piece is read while the attention ends, the first values are asked for
// beside the maxima and sums, and four parts are on their way at once (eight take registers that cost more rows at once).
// The plan may be read before this kernel's wait because the attention's launch is an ordinary one, which begins when the plan
// is complete, and this one begins behind it.  (The attention as a dependent launch and the plan read behind the wait: one
// token 9.2 us, 64 queries 46.1, ragged documents 54.7, 16 documents 161; so 8.9, 44.9, 53.9, 158.)
// With cold caches: 64 rows of a token, 19 parts each, 11.7 us; 6,784 tokens of 16 documents, a third of them in two parts, 15.3.
template <typename T, int D>
__global__ void __launch_bounds__(32 * JOIN_ROWS, JOIN_CTAS)
    k_shared_join(const __grid_constant__ SharedAttnArgs a, const __grid_constant__ Plan plan, int n_ctas) {
  constexpr int E = D / 32, AHEAD = 4;
  const int lane = threadIdx.x & 31, Hkv = a.lay.n_kv_heads, G = a.Hq / Hkv;
  const float2* ml = reinterpret_cast<const float2*>(a.ws);
  const float* part_o = reinterpret_cast<const float*>(ml + max_part_rows(a.lay.n_seqs, Hkv, G, a.max_tokens, n_ctas)) + lane * E;
  const Head head = *plan.head;
  const bool good = made_for(head, a.lay, a.Hq, a.max_tokens, n_ctas);
  __shared__ float halves[2][JOIN_ROWS / 2][D];
  __shared__ float2 halves_ml[2][JOIN_ROWS / 2];
  int turn = 0;
  bool waited = false;
  auto wait_once = [&] {
    if (!waited) pdl_wait(), pdl_trigger();
    waited = true;
  };
  Piece next{};
  if (good && static_cast<int>(blockIdx.x) < head.n_join) next = plan.join[blockIdx.x];
#pragma unroll 1
  for (int j = blockIdx.x; good && j < head.n_join; j += gridDim.x) {
    const Piece piece = next;
    if (j + static_cast<int>(gridDim.x) < head.n_join) next = plan.join[j + gridDim.x];
    // two warps a row, half of the parts each, where there are many
    const bool two = piece.parts > PARTS_A_WARP;
    const int warp = threadIdx.x >> 5, second = two ? warp & 1 : 0, row = piece.row + (two ? warp >> 1 : warp);
    if (row >= piece.rows) continue;
    const int t = plan.order[piece.tok + row / G], h = piece.h * G + row % G;
    float o[E], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = 0.f;
    // the piece's own entry, then the few entry that has a row's own keys beside tiles
    const uint32_t half = (piece.parts + 1) / 2;
    uint32_t parts = !two ? piece.parts : second ? piece.parts - half : half, rows = piece.rows, beside_parts = 0, beside_rows = 0;
    int64_t row0 = piece.part_row + row + static_cast<int64_t>(second ? half : 0) * rows, beside_row0 = 0;
    if (piece.beside && second == static_cast<int>(two)) {
      const int4 rec = plan.rec[t];
      if (rec.z >= 0) {
        const Item it = plan.items[rec.z];
        beside_parts = on_line(it, piece.h).segments(it.blocks, head.few_share);
        beside_rows = it.n_tok * G;
        beside_row0 = plan.part[rec.z * Hkv + piece.h] + static_cast<int64_t>(rec.w * G + h % G);
      }
    }
    wait_once();
#pragma unroll 1
    for (int k = 0; k < (beside_parts > 0 ? 2 : 1); ++k) {
      if (k) parts = beside_parts, rows = beside_rows, row0 = beside_row0;
#pragma unroll 1
      for (uint32_t p0 = 0; p0 < parts; p0 += 32) {
        const uint32_t n = min(32u, parts - p0);
        float v[AHEAD][E];
        auto load = [&](uint32_t from) {
#pragma unroll
          for (uint32_t i = 0; i < AHEAD; ++i) {
            if (from + i >= n) continue;
            const float* src = part_o + (row0 + static_cast<int64_t>(p0 + from + i) * rows) * D;
            if constexpr (E == 4) *reinterpret_cast<float4*>(v[i]) = *reinterpret_cast<const float4*>(src);
            else *reinterpret_cast<float2*>(v[i]) = *reinterpret_cast<const float2*>(src);
          }
        };
        const float2 x = lane < n ? ml[row0 + static_cast<int64_t>(p0 + lane) * rows] : make_float2(-INFINITY, 0.f);
        load(0);
        float top = x.x;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        top = fmaxf(top, m);
        const float base = top == -INFINITY ? 0.f : top;
        const float old = ex2(m - base), mine = ex2(x.x - base);
        l = l * old + warp_sum(x.y * mine);
        m = top;
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] *= old;
        // parts with no block, or nothing that the row sees, left no values
        const unsigned there = __ballot_sync(0xffffffffu, x.y != 0.f);
#pragma unroll 1
        for (uint32_t from = 0; from < n; from += AHEAD) {
          if (from > 0) load(from);
#pragma unroll
          for (uint32_t i = 0; i < AHEAD; ++i) {
            const float wgt = __shfl_sync(0xffffffffu, mine, (from + i) & 31);
            if (from + i < n && (there >> (from + i) & 1u)) {
#pragma unroll
              for (int e = 0; e < E; ++e) o[e] += wgt * v[i][e];
            }
          }
        }
      }
    }
    if (two) {
      // the second warp's half to the first; the places are used by turns, so that one barrier is enough
      turn ^= 1;
      float* at = halves[turn][warp >> 1] + lane * E;
      if (second) {
#pragma unroll
        for (int i = 0; i < E; ++i) at[i] = o[i];
        if (lane == 0) halves_ml[turn][warp >> 1] = make_float2(m, l);
      }
      asm volatile("bar.sync %0, 64;" ::"r"(1 + (warp >> 1)) : "memory");
      if (second) continue;
      const float2 x = halves_ml[turn][warp >> 1];
      const float top = fmaxf(m, x.x), base = top == -INFINITY ? 0.f : top;
      const float mine = ex2(m - base), other = ex2(x.x - base);
      l = l * mine + x.y * other;
      m = top;
#pragma unroll
      for (int i = 0; i < E; ++i) o[i] = o[i] * mine + at[i] * other;
    }
    const float inv = inverse(l);
    uint32_t* op = reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head) + lane * (E / 2);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) op[i] = pack2<T>(o[2 * i] * inv, o[2 * i + 1] * inv);
    if (a.lse && lane == 0) a.lse[static_cast<int64_t>(t) * a.Hq + h] = lse_of(m, l);
  }
  wait_once();
}

template <typename T, int D>
cudaError_t launch(const SharedAttnArgs& a, int num_sms, cudaStream_t st) {
  const int n_ctas = num_sms < MAX_CTAS ? num_sms : MAX_CTAS;
  CUtensorMap tm_q8, tm_q1, tm_k, tm_v;
  const int G = a.Hq / a.lay.n_kv_heads;
  const Plan plan = plan_view(const_cast<void*>(a.plan), a.lay.n_seqs, a.lay.n_kv_heads, G, a.max_tokens);
  const uint64_t rows = static_cast<uint64_t>(a.lay.n_blocks) * a.lay.n_kv_heads * a.lay.page;
  const bool half = std::is_same_v<T, __half>;
  if (!make_tmap_16b_2d(&tm_k, a.k_pool, D, rows, D * 2, 64, a.lay.page, true, half) ||
      !make_tmap_16b_2d(&tm_v, a.v_pool, D, rows, D * 2, 64, a.lay.page, true, half))
    return cudaErrorInvalidValue;
  // Q by boxes of eight tokens that follow one another and of one; views that a tensor map does not take (one row for all
  // tokens) are gathered
  SharedAttnArgs args = a;
  args.q_boxes = make_tmap_rows_of_heads(&tm_q1, a.q, D, a.Hq, a.max_tokens, a.q_head, a.q_tok, G, 1, half);
  if (!args.q_boxes) tm_q1 = tm_k;
  if (!args.q_boxes || tokens_a_tile(G) < 8) tm_q8 = tm_q1;
  else if (!make_tmap_rows_of_heads(&tm_q8, a.q, D, a.Hq, a.max_tokens, a.q_head, a.q_tok, G, 8, half)) return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(k_shared_attn<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<D>::BYTES);
  if (e != cudaSuccess) return e;
  // not a dependent launch: the joining kernel relies on that
  e = launch_ordinary(k_shared_attn<T, D>, dim3(n_ctas), THREADS, Smem<D>::BYTES, st, tm_q8, tm_q1, tm_k, tm_v, args, plan);
  if (e != cudaSuccess) return e;
  // as many blocks as could have work, up to what the SMs hold at once
  const int64_t pieces = max_items(a.lay.n_seqs, a.Hq / a.lay.n_kv_heads, a.max_tokens) * a.lay.n_kv_heads +
                         static_cast<int64_t>(a.max_tokens) * a.Hq / (JOIN_ROWS / 2);
  const int64_t held = JOIN_CTAS * static_cast<int64_t>(num_sms);
  return launch_dependent(k_shared_join<T, D>, dim3(static_cast<unsigned>(pieces < held ? pieces : held)), 32 * JOIN_ROWS, 0, st, a,
                          plan, n_ctas);
}

}  // namespace

int64_t shared_workspace_bytes(const dopr_cache_layout& lay, int Hq, int max_tokens, int num_sms) {
  const int n_ctas = num_sms < MAX_CTAS ? num_sms : MAX_CTAS;
  return max_part_rows(lay.n_seqs, lay.n_kv_heads, Hq / lay.n_kv_heads, max_tokens, n_ctas) * (8 + 4 * static_cast<int64_t>(lay.head_dim));
}

cudaError_t launch_shared_attention(const SharedAttnArgs& a, int num_sms, cudaStream_t st) {
  const bool half = a.lay.dtype == DOPR_F16;
  if (a.lay.head_dim == 128) return half ? launch<__half, 128>(a, num_sms, st) : launch<__nv_bfloat16, 128>(a, num_sms, st);
  return half ? launch<__half, 64>(a, num_sms, st) : launch<__nv_bfloat16, 64>(a, num_sms, st);
}

}  // namespace dopr
