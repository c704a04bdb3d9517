// shared_attn_device.cuh -- what the attention over the paged cache (k_shared_attn.cu) and that over its 4-bit form
// (k_shared_attn_4bit.cu) have in common: the CTA's roles, their barriers and shared memory, and the arithmetic of their parts.
// How they work together is described at the top of k_shared_attn.cu.
#pragma once

#include <limits.h>

#include <type_traits>

#include "pages4.cuh"
#include "shared_attn.cuh"

namespace dopr {
namespace {
using namespace shared_attn;

// (of the 4-bit cache: four warps more, which bring K and V to the products' type)
template <bool FOUR>
constexpr int THREADS = 128 + 2 * 128 + (FOUR ? 128 : 0);
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
constexpr int HALF_BYTES = 128 * 128;  // 128 rows of 64 16-bit elements

template <int D, bool FOUR = false>
struct Smem {
  static constexpr int HALVES = D / 64;
  static constexpr int TILE_BYTES = HALVES * HALF_BYTES;
  static constexpr int K_STAGES = FOUR ? (D == 128 ? 2 : 3) : D == 128 ? 2 : 5, V_STAGES = FOUR ? (D == 128 ? 2 : 3) : D == 128 ? 3 : 5;
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = OFF_Q + 2 * TILE_BYTES;
  static constexpr int OFF_V = OFF_K + K_STAGES * TILE_BYTES;
  // 4 bits: blocks as they come, in halves of 64 rows: codes and scales of a piece of at most 64 rows of a page, then of the next
  static constexpr int RAW_BYTES = 64 * (D / 2 + D / 32);
  static constexpr int RAW_K = FOUR ? 4 : 0, RAW_V = !FOUR ? 0 : D == 128 ? 3 : 4;
  static constexpr int OFF_RAW = OFF_V + V_STAGES * TILE_BYTES;
  static constexpr int OFF_ROW = OFF_RAW + (RAW_K + RAW_V) * RAW_BYTES;  // the Q gatherer's rows' tokens
  static constexpr int OFF_ML = OFF_ROW + 128 * 4;      // maxima and sums that one softmax group leaves to the other
  static constexpr int OFF_KEYS = OFF_ML + 128 * 8;     // of each page of a V stage (4 bits: of each piece of a half): rows that hold keys
  static constexpr int OFF_BAR = OFF_KEYS + 64;
  // few items: from 0 on, pieces of 16 columns of K and V, F_STAGES of them a warp
  static constexpr int F_STAGES = FOUR ? (D == 128 ? 8 : 12) : D == 128 ? 3 : 6;
  static constexpr int F_BYTES = FOUR ? 2 * PIECE * (D / 2 + D / 32) : 2 * HALVES * PIECE * 128;
  static constexpr int F_SCALES = WORKERS * F_STAGES * F_BYTES;  // 4 bits: what each warp takes of 32 keys' scales
  static constexpr int F_SCALE_BYTES = FOUR ? 32 * (D / 32) * 8 : 0;
  static_assert(F_SCALES + WORKERS * F_SCALE_BYTES <= OFF_ROW, "the few items' pieces");
  static constexpr int K_FULL = 0, K_EMPTY = K_FULL + K_STAGES, V_FULL = K_EMPTY + K_STAGES, V_EMPTY = V_FULL + V_STAGES,
                       Q_FULL = V_EMPTY + V_STAGES, Q_EMPTY = Q_FULL + 2, S_FULL = Q_EMPTY + 2, P_FULL = S_FULL + 2,
                       O_FULL = P_FULL + 4, ML_FULL = O_FULL + 2, ML_EMPTY = ML_FULL + 1, DRAIN = ML_EMPTY + 1, RAW_FULL = DRAIN + 1,
                       RAW_EMPTY = RAW_FULL + RAW_K + RAW_V, N_BARS = RAW_EMPTY + RAW_K + RAW_V;
  static constexpr int BYTES = 1024 + OFF_BAR + N_BARS * 8 + 16;
  static_assert(V_STAGES * 8 <= 64 && (RAW_K + RAW_V) * 4 <= 64, "a byte a page");
  static_assert(BYTES <= 227 * 1024, "shared memory budget");
};

// A wait of the CTA's roles.  4 bits: by counts, some two seconds whatever limit the caller gives (that is the clock's), each role by
// itself: where copies stop, the roles give up within two seconds of one another and their drains two seconds later, and the
// error is reported then; the clock's code and the atomic's, at twenty
// places, took more of the instruction caches than they can spare beside the warps that expand (200 queries on 16 documents: 182 us
// for 220 with the clock, 200 with the atomic; 2,048 rows on 16,384 keys: 420 for 427 and 433).
__device__ __forceinline__ bool wait_by_counts(uint32_t bar, uint32_t parity, int* err) {
#pragma unroll 1
  for (int i = 0; i < 1 << 26; ++i)
    if (mbar_try_wait(bar, parity)) return true;
  *reinterpret_cast<volatile int*>(err) = DEV_ERR_TIMEOUT;
  return false;
}
template <bool FOUR>
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, int* err, uint64_t timeout_ns) {
  if constexpr (FOUR) return __all_sync(0xffffffffu, wait_by_counts(bar, parity, err)) != 0;
  return mbar_wait_warp(bar, parity, err, timeout_ns);
}

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
// Shares of the launch's registers (384 threads x 168; 4 bits: 512 x 128): little for the warps that copy, expand and issue, more
// where rows of S are held (152 and 176: 2,048 rows 353 us for 351.7).
template <bool FOUR>
constexpr int REGS_FEW = FOUR ? 88 : 136;
template <bool FOUR>
constexpr int REGS_MANY = FOUR ? 168 : 184;
static_assert(128 * REGS_FEW<false> + 256 * REGS_MANY<false> <= 384 * 168 && 256 * REGS_FEW<true> + 256 * REGS_MANY<true> <= 512 * 128,
              "more registers than the launch has are waited for without end");
template <bool FOUR>
__device__ __forceinline__ void regs_few() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW<FOUR>)); }
template <bool FOUR>
__device__ __forceinline__ void regs_many() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_MANY<FOUR>)); }
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

// ------------------------------------------------------------------ the 4-bit cache
// What values, and with them scores and O, are to be multiplied by (pages4.cuh).
template <typename T, bool FOUR>
constexpr float HELD_UNIT = FOUR ? pages4::Widen<T>::UNIT : 1.f;

// Shared memory by its own addresses: what comes from a pointer made of a number is read and written as memory of any kind, with
// addresses of 64 bits (64 conversations so: 139 us).
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(at));
  return x;
}
__device__ __forceinline__ uint32_t lds16(uint32_t at) {
  uint16_t x;
  asm volatile("ld.shared.b16 %0, [%1];" : "=h"(x) : "r"(at));
  return x;
}
__device__ __forceinline__ uint32_t lds8(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x) : "r"(at));
  return x;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 x;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at));
  return x;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 x;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(at));
  return x;
}
__device__ __forceinline__ void sts64(uint32_t at, uint2 x) {
  asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(x.x), "r"(x.y) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t at, uint4 x) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}
// n bytes of 16, zeros for the others.
__device__ __forceinline__ void cp_async16_part(uint32_t dst, const void* src, int n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
               "r"(bar)
               : "memory");
}
// D (16 x 8, 32-bit) += A (16 x 16) B (16 x 8) of fp16 by a warp.
__device__ __forceinline__ void mma_f16_add(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// An 8 x 8 of 16-bit elements, row lane / 4 and columns 2 (lane % 4) and the next a lane, the other way round.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return reinterpret_cast<const __half2&>(x); }
// The four pairs of codes at 4 k and 16 + 4 k as fp16 numbers c 2^-9: n 2^-24 or 16 n 2^-24 as they stand, the type's lowest, to n 2^-9 less
// 8 2^-9, exactly.  (As they stand in the products, with 8 times the other operand taken off, is a fused step less for a pair, but the
// sums are off by up to 2^-15 of their largest terms: lighter keys beside a heavy one whose code is zero were lost, and scores of hundreds
// off by ten times what a product in 32 bits is.  It was no faster: 64 conversations 110 us for 106.)
__device__ __forceinline__ void as_codes(uint32_t w, uint32_t (&x)[4]) {
  const uint32_t n[4] = {w & 0x000f000fu, w & 0x00f000f0u, w >> 8 & 0x000f000fu, w >> 8 & 0x00f000f0u};
  const uint32_t up = 0x78007800u, up16 = 0x68006800u, from = 0xa400a400u;  // 2^15, 2^11, -8 2^-9
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const __half2 c = __hfma2(as_half2(n[k]), as_half2(k & 1 ? up16 : up), as_half2(from));
    x[k] = reinterpret_cast<const uint32_t&>(c);
  }
}
// The largest of a word's bytes.
__device__ __forceinline__ uint32_t max_byte(uint32_t w) {
  const uint32_t t = __vmaxu2(w & 0x00ff00ffu, w >> 8 & 0x00ff00ffu);
  return max(t & 0xffffu, t >> 16);
}

// A scale's byte; one that stands for NaN counts as zero and is noted.
__device__ __forceinline__ uint32_t scale_of(uint32_t byte, bool& bad) {
  bad |= byte > pages4::SCALE_LAST;
  return byte > pages4::SCALE_LAST ? 0u : byte;
}

// Where in a row of a piece its 16 bytes lie that are its c-th: at c ^ chunk_place, so that rows which lanes read at once lie in different banks.
template <int D>
__device__ __forceinline__ int chunk_place(int row) {
  return D == 128 ? (row & 2) | (row >> 2 & 1) : row >> 2 & 1;
}

// Up to 16 rows of a segment of few items by a warp, the rows on the products' long side: codes are widened in registers.  Of K a thread
// widens a key's elements from D / 4 t on, of Q it has the same ones; of V it widens the elements from D / 8 g on of four keys.
template <typename T, int D>
struct Few16 {
  static constexpr int ROW = D / 2, SROW = D / 32, CODES = PIECE * ROW, SCALES = PIECE * SROW, WORDS = D / 32, NT = D / 8;
  uint32_t q[D / 16][4];
  int own0[2], own1[2];
  float o[NT][4], m[2], l[2], scale_log2;

  __device__ __forceinline__ Few16(const SharedAttnArgs& a, const Plan& plan, const Segment& s, int rows, int G, int lane) {
    const int quad = lane >> 2, in_quad = lane & 3;
    scale_log2 = a.scale * 1.4426950408889634f * HELD_UNIT<T, true>;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = quad + 8 * i;
      const bool valid = r < rows;
      const int at = s.tok + (valid ? r / G : 0);
      const int2 own = plan.own[at];
      own0[i] = valid ? own.x : 0, own1[i] = valid ? own.y : 0;
      const uint2* src = reinterpret_cast<const uint2*>(static_cast<const T*>(a.q) + plan.order[at] * a.q_tok +
                                                        static_cast<int64_t>(s.h * G + (valid ? r % G : 0)) * a.q_head + in_quad * (D / 4));
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint2 x = valid ? src[k] : uint2{0, 0};
        q[k][i] = x.x;
        q[k][2 + i] = x.y;
      }
      m[i] = -INFINITY, l[i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  }

  // A piece of 16 keys, of which the first is column col0.
  __device__ __forceinline__ void step(uint32_t piece, int prefix_keys, int col0, bool& bad, int lane) {
    const int quad = lane >> 2, in_quad = lane & 3;
    const int key_col[2] = {in_quad, 4 + (in_quad ^ 1)};               // the keys, of eight, of this thread's columns of scores
    const int key_row = quad & 1 ? 4 + ((quad >> 1) ^ 1) : quad >> 1;  // the key that it widens
    float sc[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      sc[t][0] = sc[t][1] = sc[t][2] = sc[t][3] = 0.f;
      const int row = 8 * t + key_row;
      const uint32_t at = piece + row * ROW;
      uint32_t w[WORDS];
      if constexpr (D == 128) {
        const uint4 x = lds128(at + ((in_quad ^ chunk_place<D>(row)) << 4));
        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
      } else {
        const uint2 x = lds64(at + (((in_quad >> 1) ^ chunk_place<D>(row)) << 4) + 8 * (in_quad & 1));
        w[0] = x.x, w[1] = x.y;
      }
      const pages4::Widen<T> widen(scale_of(lds8(piece + 2 * CODES + row * SROW + in_quad * SROW / 4), bad) * 0x10001u);
#pragma unroll
      for (int j = 0; j < WORDS; ++j) {
        uint32_t x[4];
        widen(w[j], x);
        mma16<T>(sc[t], q[2 * j], x[0], x[1]);
        mma16<T>(sc[t], q[2 * j + 1], x[2], x[3]);
      }
    }
    if (prefix_keys < col0 + PIECE) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = col0 + 8 * t + key_col[e & 1], i = e >> 1;
          if (!(at < prefix_keys || (at >= own0[i] && at < own1[i]))) sc[t][e] = -INFINITY;
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
        for (int d = 0; d < NT; ++d) o[d][2 * i] *= by, o[d][2 * i + 1] *= by;
      }
      const float at_m = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float x = ex2(fmaf(sc[t][2 * i], scale_log2, -at_m)), y = ex2(fmaf(sc[t][2 * i + 1], scale_log2, -at_m));
        l[i] += x + y;  // this thread's columns: the quad's four sums are added up at the end
        p[2 * t + i] = pack2<T>(x, y);
      }
    }
    // V: tokens of the columns 2 t, 2 t + 1 (a, b) and 2 t + 8, 2 t + 9 (c, d)
    uint32_t w[4][(WORDS + 1) / 2], by[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * (i >> 1) + key_col[i & 1];
      const uint32_t at = piece + CODES + row * ROW;
      if constexpr (D == 128) {
        const uint2 x = lds64(at + (((quad >> 1) ^ chunk_place<D>(row)) << 4) + 8 * (quad & 1));
        w[i][0] = x.x, w[i][1] = x.y;
      } else {
        w[i][0] = lds32(at + (((quad >> 2) ^ chunk_place<D>(row)) << 4) + 4 * (quad & 3));
      }
      by[i] = scale_of(lds8(piece + 2 * CODES + SCALES + row * SROW + quad * SROW / 8), bad);
    }
    const pages4::Widen<T> ab(by[0] | by[1] << 16), cd(by[2] | by[3] << 16);
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
#pragma unroll
      for (int odd = 0; odd < 2; ++odd) {
        uint32_t x[4], y[4];
        ab(__byte_perm(w[0][j], w[1][j], odd ? 0x7632 : 0x5410), x);
        cd(__byte_perm(w[2][j], w[3][j], odd ? 0x7632 : 0x5410), y);
#pragma unroll
        for (int k = 0; k < 4; ++k) mma16<T>(o[8 * j + 2 * k + odd], p, x[k], y[k]);
      }
  }

  // Rows out: column n of the product d of O is element D / 8 * n + d, so a thread has D / 4 elements that follow one another of each row.
  __device__ __forceinline__ void finish(const SharedAttnArgs& a, const Plan& plan, const Segment& s, int rows, int G, int lane) {
    const int quad = lane >> 2, in_quad = lane & 3;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = quad + 8 * i;
      float sum = l[i] + __shfl_xor_sync(0xffffffffu, l[i], 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      if (r < rows && (s.flags & SEG_WHOLE)) {
        const int t = plan.order[s.tok + r / G], h = s.h * G + r % G;
        const float inv = sum == 0.f ? 0.f : inverse(sum) * HELD_UNIT<T, true>;
        uint4* dst = reinterpret_cast<uint4*>(static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head + 2 * NT * in_quad);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int d = 0; d < NT; d += 8) {
            uint32_t x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = pack2<T>(o[d + 2 * k][2 * i + e] * inv, o[d + 2 * k + 1][2 * i + e] * inv);
            dst[(e * NT + d) / 8] = uint4{x[0], x[1], x[2], x[3]};
          }
        if (a.lse && in_quad == 0) a.lse[static_cast<int64_t>(t) * a.Hq + h] = lse_of(m[i], sum);
      } else if (r < rows) {
        float2* ml = reinterpret_cast<float2*>(a.ws);
        float* part_o = reinterpret_cast<float*>(ml + max_part_rows(a.lay.n_seqs, a.lay.n_kv_heads, G, a.max_tokens, gridDim.x));
        const int64_t row = static_cast<int64_t>(s.part_row) + r;
        if (in_quad == 0) ml[row] = make_float2(m[i], sum);
        if (sum != 0.f) {
          float4* dst = reinterpret_cast<float4*>(part_o + row * D + 2 * NT * in_quad);
          constexpr float U = HELD_UNIT<T, true>;
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int d = 0; d < NT; d += 4)
              dst[(e * NT + d) / 4] = make_float4(o[d][2 * i + e] * U, o[d + 1][2 * i + e] * U, o[d + 2][2 * i + e] * U, o[d + 3][2 * i + e] * U);
        }
      }
    }
  }
};

// Up to 8 rows of a segment of few items, from row0 on, by a warp.  Thread (g, t) = (lane / 4, lane % 4) has scores of the keys g and g + 8 of a piece
// with rows 2 t and 2 t + 1, as the products leave them, and of O the elements that its words of V hold.
template <typename T, int D>
struct Few8 {
  static constexpr int GROUPS = D / 32, ROW = D / 2, SROW = D / 32, CODES = PIECE * ROW, SCALES = PIECE * SROW;
  uint32_t q[GROUPS][4];           // row g: 8 elements from 8 t on of each group
  float unit[2];                   // what their scores are multiplied by
  int own0[2], own1[2];
  int all0, all1;                  // own columns that all rows see
  float o[GROUPS][2][4];
  // P = 2^(score - m), m BELOW the largest sum of a score and its value's exponent e (scales below 2^e) among the keys that the row
  // sees: what is rounded is P times a scale, at most 2^15, and no key's value takes from another's unless it weighs more.  (Scales
  // taken relative to the largest of all keys so far: rows lost what they saw to large values at no weight, or that later tokens alone
  // see.)
  float m[2], l[2];

  __device__ __forceinline__ Few8(const SharedAttnArgs& a, const Plan& plan, const Segment& s, int row0, int rows, int G, int lane) {
    const int g = lane >> 2, t = lane & 3;
    const bool valid = g < rows;
    const int token = plan.order[s.tok + (row0 + (valid ? g : 0)) / G];
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + token * a.q_tok +
                                                      static_cast<int64_t>(s.h * G + (row0 + (valid ? g : 0)) % G) * a.q_head) + t;
    float x[GROUPS][8], most = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const uint4 w = valid ? src[4 * i] : uint4{0, 0, 0, 0};
      const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 f = unpack2<T>(v[k]);
        x[i][2 * k] = f.x, x[i][2 * k + 1] = f.y;
        most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
      }
    }
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
    // the row's largest to 2^13 and above: elements below 2^-27 of it are rounded, by at most 2^-38 of it
    const int e = most > 0.f ? min(100, 13 + 127 - static_cast<int>(__float_as_uint(most) >> 23)) : 0;
    const float up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23), down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) q[i][k] = pack_f16x2(x[i][2 * k] * up, x[i][2 * k + 1] * up);
    const float scale = a.scale * 1.4426950408889634f * 0x1p9f;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = 2 * t + j;
      unit[j] = scale * __shfl_sync(0xffffffffu, down, 4 * row);
      const int2 own = plan.own[s.tok + (row0 + (row < rows ? row : 0)) / G];
      own0[j] = row < rows ? own.x : 0, own1[j] = row < rows ? own.y : 0;
      m[j] = -INFINITY, l[j] = 0.f;
    }
    all0 = __reduce_max_sync(0xffffffffu, max(2 * t < rows ? own0[0] : 0, 2 * t + 1 < rows ? own0[1] : 0));
    all1 = __reduce_min_sync(0xffffffffu, min(2 * t < rows ? own1[0] : INT_MAX, 2 * t + 1 < rows ? own1[1] : INT_MAX));
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[i][0][k] = o[i][1][k] = 0.f;
  }

  static __device__ __forceinline__ void put_scales(uint32_t to, const float (&f)[GROUPS]) {
    if constexpr (GROUPS == 4) sts128(to, uint4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])});
    else sts64(to, uint2{__float_as_uint(f[0]), __float_as_uint(f[1])});
  }
  static __device__ __forceinline__ void get_scales(uint32_t from, float (&f)[GROUPS]) {
    if constexpr (GROUPS == 4) {
      const uint4 u = lds128(from);
      f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y), f[2] = __uint_as_float(u.z), f[3] = __uint_as_float(u.w);
    } else {
      const uint2 u = lds64(from);
      f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y);
    }
  }
  // Two pieces of 16 keys, of which the first is column col0; the second's address is the first's where there is one only.
  __device__ __forceinline__ void step(const uint32_t (&piece)[2], uint32_t scales, int prefix_keys, int col0, bool& bad, int lane) {
    constexpr int N = 2;
    const bool two = piece[1] != piece[0];
    const int g = lane >> 2, t = lane & 3;
    // each lane looks at a key's scales: bytes that stand for NaN become zeros; the exponent of the largest of V's; and what the products
    // take, a key's of K and of V in 32 bits
    float exponent;
    {
      const uint32_t ks = (lane < 16 ? piece[0] : piece[1]) + 2 * CODES + (lane & 15) * SROW;
      uint32_t kw, vw;
      if constexpr (D == 128) kw = lds32(ks), vw = lds32(ks + SCALES);
      else kw = lds16(ks), vw = lds16(ks + SCALES);
      if (lane >= 16 && !two) kw = vw = 0;
      uint32_t most = max_byte(vw);
      const bool odd = max(most, max_byte(kw)) > pages4::SCALE_LAST;
      if (__any_sync(0xffffffffu, odd)) {
        bad |= odd;
#pragma unroll
        for (int i = 0; i < SROW; ++i) {
          if ((kw >> 8 * i & 0xffu) > pages4::SCALE_LAST) kw &= ~(0xffu << 8 * i);
          if ((vw >> 8 * i & 0xffu) > pages4::SCALE_LAST) vw &= ~(0xffu << 8 * i);
        }
        most = max_byte(vw);
      }
      exponent = static_cast<float>(static_cast<int>(most >> 3) - 14);
      // a byte's exponent is 112 below as a 32-bit number's
      float f[GROUPS], v[GROUPS];
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        f[i] = __uint_as_float((i < 3 ? kw << (20 - 8 * i) : kw >> 4) & 0x0ff00000u) * 0x1p112f;
        v[i] = __uint_as_float((i < 3 ? vw << (20 - 8 * i) : vw >> 4) & 0x0ff00000u) * 0x1p112f;
      }
      const uint32_t to = scales + lane * (GROUPS * 4);
      put_scales(to, f);
      put_scales(to + 32 * GROUPS * 4, v);
      __syncwarp();
    }
    float sc[N][4];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int place = chunk_place<D>(g);
      const uint32_t kc = piece[n] + g * ROW + 4 * t, ks = scales + (16 * n + g) * (GROUPS * 4);
      float f0[GROUPS], f1[GROUPS];  // scales of the keys g and g + 8
      get_scales(ks, f0);
      get_scales(ks + 8 * GROUPS * 4, f1);
      sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.f;
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        uint32_t x[4], y[4];
        as_codes(lds32(kc + ((i ^ place) << 4)), x);
        as_codes(lds32(kc + ((i ^ place) << 4) + 8 * ROW), y);
        float d[4] = {0.f, 0.f, 0.f, 0.f};
        mma_f16_add(d, x[0], y[0], x[1], y[1], q[i][0], q[i][1]);
        mma_f16_add(d, x[2], y[2], x[3], y[3], q[i][2], q[i][3]);
        sc[n][0] = fmaf(d[0], f0[i], sc[n][0]), sc[n][1] = fmaf(d[1], f0[i], sc[n][1]);
        sc[n][2] = fmaf(d[2], f1[i], sc[n][2]), sc[n][3] = fmaf(d[3], f1[i], sc[n][3]);
      }
    }
    const int end = col0 + (two ? 2 : 1) * PIECE;
    if (!two || (prefix_keys < end && (col0 < all0 || end > all1))) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = col0 + PIECE * n + g + 8 * (e >> 1), j = e & 1;
          if (at >= end || !(at < prefix_keys || (at >= own0[j] && at < own1[j]))) sc[n][e] = -INFINITY;
        }
    }
    // a row's keys are those of this thread and of the lanes with the same t
    float top[2];
    {
      float e[N][2];
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) e[n][i] = __shfl_sync(0xffffffffu, exponent, 16 * n + 8 * i + g);
#pragma unroll
      for (int j = 0; j < 2; ++j)
        top[j] = fmaxf(fmaxf(fmaf(sc[0][j], unit[j], e[0][0]), fmaf(sc[0][2 + j], unit[j], e[0][1])),
                       fmaxf(fmaf(sc[1][j], unit[j], e[1][0]), fmaf(sc[1][2 + j], unit[j], e[1][1])));
    }
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
      top[0] = fmaxf(top[0], __shfl_xor_sync(0xffffffffu, top[0], d));
      top[1] = fmaxf(top[1], __shfl_xor_sync(0xffffffffu, top[1], d));
    }
    bool grow[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      top[j] -= BELOW<__half>;
      if (m[j] == -INFINITY) m[j] = top[j];  // nothing but zeros has been summed
      grow[j] = top[j] > m[j] + RESCALE<__half>;
    }
    if (__any_sync(0xffffffffu, grow[0] || grow[1])) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float by = grow[j] ? ex2(m[j] - top[j]) : 1.f;
        if (grow[j]) m[j] = top[j];
        l[j] *= by;
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) {
          o[i][0][j] *= by, o[i][0][2 + j] *= by, o[i][1][j] *= by, o[i][1][2 + j] *= by;
        }
      }
    }
    const float m0 = m[0] == -INFINITY ? 0.f : m[0], m1 = m[1] == -INFINITY ? 0.f : m[1];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float p0 = ex2(fmaf(sc[n][0], unit[0], -m0)), p1 = ex2(fmaf(sc[n][1], unit[1], -m1));
      const float p2 = ex2(fmaf(sc[n][2], unit[0], -m0)), p3 = ex2(fmaf(sc[n][3], unit[1], -m1));
      l[0] += p0 + p2, l[1] += p1 + p3;  // this thread's keys: the lanes' sums are added up at the end
      float f0[GROUPS], f1[GROUPS];
      const uint32_t vs = scales + (32 + 16 * n + g) * (GROUPS * 4);
      get_scales(vs, f0);
      get_scales(vs + 8 * GROUPS * 4, f1);
      const uint32_t vc = piece[n] + CODES + 2 * t * ROW + 4 * (g >> 1);
      const int place = chunk_place<D>(2 * t);
      const uint32_t half_word = g & 1 ? 0x7632u : 0x5410u;
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        // P times the scale, rounded once: row g, keys 2 t and 2 t + 1, and 8 more
        const uint32_t ba = transpose8(pack_f16x2(p0 * f0[i], p1 * f0[i])), bb = transpose8(pack_f16x2(p2 * f1[i], p3 * f1[i]));
        const uint32_t w = vc + ((i ^ place) << 4);
        uint32_t x[4], y[4];
        as_codes(__byte_perm(lds32(w), lds32(w + ROW), half_word), x);
        as_codes(__byte_perm(lds32(w + 8 * ROW), lds32(w + 9 * ROW), half_word), y);
        mma_f16_add(o[i][0], x[0], x[1], y[0], y[1], ba, bb);
        mma_f16_add(o[i][1], x[2], x[3], y[2], y[3], ba, bb);
      }
    }
  }

  // Rows out: of row 2 t + j thread (g, t) has elements 32 i + 8 (g / 2) + 2 k + g % 2; with its neighbour's it has 8 that follow one
  // another, of row 2 t where g is even, else of 2 t + 1.
  __device__ __forceinline__ void finish(const SharedAttnArgs& a, const Plan& plan, const Segment& s, int row0, int rows, int G, int lane) {
    const int g = lane >> 2, t = lane & 3, odd = g & 1, r = 2 * t + odd;
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
      l[0] += __shfl_xor_sync(0xffffffffu, l[0], d);
      l[1] += __shfl_xor_sync(0xffffffffu, l[1], d);
    }
    const float mm = odd ? m[1] : m[0], ll = odd ? l[1] : l[0];
    const bool whole = s.flags & SEG_WHOLE;
    float by = 0x1p9f;
    if (whole) by = ll == 0.f ? 0.f : by * inverse(ll);
    const int at = row0 + (r < rows ? r : 0), h = s.h * G + at % G, token = plan.order[s.tok + at / G];
    float2* ml = reinterpret_cast<float2*>(a.ws);
    const int64_t part = static_cast<int64_t>(s.part_row) + row0 + r;
    float* part_o = reinterpret_cast<float*>(ml + max_part_rows(a.lay.n_seqs, a.lay.n_kv_heads, G, a.max_tokens, gridDim.x)) + part * D;
    T* out = static_cast<T*>(a.out) + token * a.o_tok + h * a.o_head;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float(&x)[4] = o[i][k >> 1];  // O of code k
        const float e0 = x[2 * (k & 1)], e1 = x[2 * (k & 1) + 1];
        const float other = __shfl_xor_sync(0xffffffffu, odd ? e0 : e1, 4);
        v[2 * k] = odd ? other : e0, v[2 * k + 1] = odd ? e1 : other;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= by;
      const int d = 32 * i + 8 * (g >> 1);
      if (r < rows) {
        if (whole) {
          *reinterpret_cast<uint4*>(out + d) = uint4{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])};
        } else if (ll != 0.f) {
          *reinterpret_cast<float4*>(part_o + d) = make_float4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<float4*>(part_o + d + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
      }
    }
    if (r < rows && g < 2) {
      if (!whole) ml[part] = make_float2(mm, ll);
      else if (a.lse) a.lse[static_cast<int64_t>(token) * a.Hq + h] = lse_of(mm, ll);
    }
  }
};

// What a warp does at once of few items of the 4-bit cache: a segment, or where that has several long runs, whose tokens alone see
// them, a run of it.  A part for Few8 is of one run: the rows of others would see none of it.  Few8 takes
// 0.9 us a piece where Few16 takes 1.4 with eight warps at work, but its code beside Few16's does not stay in the instruction
// caches when parts are short (half of a warp's time then goes to waiting for instructions).  By the pieces from which Few8 takes a
// run (on average over a segment's), in us:
//           64 conversations of    256 of 50 to 400 keys,    32 of 1,000 to 3,000    8 of 16,000 keys,
//           2,000 to 6,000 keys    4 and 8 rows a token      keys, a row a token     8 rows a token
//      8          104                   64   71                     48                     61
//     12          104                   54   67                     48                     62
//     16          106                   45   52                     54                     63
//     24          108                   46   51                     54                     66
//   none          142                   46   51                     54                     78
// and a segment of one run: one token of 32 heads on 8 over 32,768 keys, 256 queries on 64 documents of 1 to 1,024 tokens: from 6
// pieces on 33.2 and 50.4, 12: 34.8 and 49.9, 24: 38.5 and 49.4, none: 38.5 and 48.6.
constexpr uint32_t LONG_RUN = 16, LONG_SEGMENT = 6;
struct Job {
  const Segment* s;
  int row0, rows;
  uint32_t from, to;  // pieces
  bool eight;         // by Few8
};
struct Jobs {
  const Plan& plan;
  const Segment* s = nullptr;
  int at, end, G, run = -1;
  __device__ __forceinline__ Jobs(const Plan& p, int2 work, int G_) : plan(p), at(work.x), end(work.y), G(G_) {}
  // The segment's runs; own: none is a prefix, and none has more than 8 rows.
  __device__ __forceinline__ uint32_t count(bool& own) const {
    const Run* runs = plan.runs + s->run;
    uint32_t of = 0;
    own = true;
    for (int i0 = s->run_at; i0 < s->n_runs; i0 += 32) {  // a lane a run
      const int i = i0 + static_cast<int>(threadIdx.x & 31u);
      const bool in = i < s->n_runs && static_cast<uint32_t>(runs[i].off) < s->b1;
      if (__any_sync(0xffffffffu, in && (runs[i].token < 0 || (runs[i].tok1 - runs[i].tok0) * G > 8))) own = false;
      of += __popc(__ballot_sync(0xffffffffu, in));
    }
    return of;
  }
  // starts: the segment is a new one, and its runs are jobs of their own
  __device__ __forceinline__ bool next(Job& j, bool& starts) {
    starts = false;
    for (;;) {
      if (run >= 0) {
        const Run* r = plan.runs + s->run + run;
        if (run < s->n_runs && static_cast<uint32_t>(r->off) < s->b1) {
          ++run;
          j.from = max(s->b0, static_cast<uint32_t>(r->off)), j.to = min(s->b1, static_cast<uint32_t>(r->off + r->pages));
          if (j.from >= j.to) continue;
          j.row0 = r->tok0 * G, j.rows = (r->tok1 - r->tok0) * G;
          return true;
        }
        run = -1;
      }
      if (at >= end) return false;
      s = j.s = plan.segs + at++;
      if (at < end) asm volatile("prefetch.global.L1 [%0];" ::"l"(plan.segs + at));
      j.from = s->b0, j.to = s->b1;
      j.row0 = 0, j.rows = s->n_tok * G;
      j.eight = false;
      const uint32_t n = j.to - j.from;
      if (n < LONG_SEGMENT) return true;
      bool own;
      const uint32_t of = count(own);
      if (of == 1 && j.rows <= 8) {
        j.eight = true;
        return true;
      }
      if (!own || n < LONG_RUN * of) return true;
      j.eight = true;
      run = s->run_at;
      starts = true;
    }
  }
};

// Results of rows of a segment whose runs are jobs of their own, but which have none in it.
template <typename T, int D>
__device__ __forceinline__ void rows_without_keys(const SharedAttnArgs& a, const Plan& plan, const Segment& s, int G, int lane) {
  const Run* runs = plan.runs + s.run;
  uint32_t seen = 0;  // a bit a row; a lane a run
  for (int i = s.run_at + lane; i < s.n_runs; i += 32) {
    const Run run = runs[i];
    const uint32_t off = run.off;
    if (max(off, s.b0) < min(off + run.pages, s.b1)) seen |= (1u << run.tok1 * G) - (1u << run.tok0 * G);
  }
  seen = __reduce_or_sync(0xffffffffu, seen);
  for (uint32_t none = ((1u << s.n_tok * G) - 1u) & ~seen; none != 0; none &= none - 1u) {
    const int r = __ffs(none) - 1;
    if (s.flags & SEG_WHOLE) {
      const int t = plan.order[s.tok + r / G], h = s.h * G + r % G;
      if (lane < D / 8) reinterpret_cast<uint4*>(static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head)[lane] = uint4{0, 0, 0, 0};
      if (lane == 0 && a.lse) a.lse[static_cast<int64_t>(t) * a.Hq + h] = -INFINITY;
    } else if (lane == 0) {
      reinterpret_cast<float2*>(a.ws)[static_cast<int64_t>(s.part_row) + r] = make_float2(-INFINITY, 0.f);
    }
  }
}

// Eight warps a CTA with a ring of pieces each, by 16-byte copies.  Scales of rows past a run's keys come as zeros, so such rows are zeros.
//
// Few16 has rows on the products' long side (16) and widens codes to 16 bits by masks, shifts and fused products.  Few8 has keys and
// values there, 16 of them for 8 rows, and codes go into the products without their scales, as c 2^-9 (as_codes): a mask, a fused step and a
// quarter of a shift a pair.  Scales come in where there is less of them: a group's products with Q are scaled when its 32 elements are
// summed up, and P is multiplied by V's scale for each group.  Q is brought to fp16 by a power of two for each row, P times a scale by the
// row's m: it is rounded to 11 bits, or lies on steps of 2^-34 of the row's largest, once (P rounded first, and the product of both in
// fp16: errors of 0.00035 of the outputs' norm for 0.00028).
// Bound by instructions, 476 a piece of 16 keys with starts and ends: two warps a quarter of the SM issue in 53 % of its cycles, each
// waiting for its own last result otherwise; the registers (168 a thread) hold no third.  64 tokens of 32 heads on 8 over 2,000 to 6,000
// keys each: 106 us (2.7 TB/s), 142 by Few16 alone.
template <typename T, int D>
__device__ __forceinline__ void few_items_4bit(const SharedAttnArgs& a, const Plan& plan, uint32_t s0, int warp, int2 work, int lane) {
  using L = Smem<D, true>;
  constexpr int ROW = D / 2, SROW = D / 32, CODES = PIECE * ROW, SCALES = PIECE * SROW, STAGE = L::F_BYTES, STAGES = L::F_STAGES;
  constexpr int CHUNKS = ROW / 16, SCALE_CHUNKS = SCALES / 16;
  const uint32_t base = s0 + warp * STAGES * STAGE, scales = s0 + L::F_SCALES + warp * L::F_SCALE_BYTES;
  const int Hkv = a.lay.n_kv_heads, G = a.Hq / Hkv, page = a.lay.page;
  const int64_t page_bytes = pages4::page_bytes(page, D);
  bool bad = false;
  // copies run ahead of the products, over the ends of jobs too; two stages are left to the products
  Jobs copies(plan, work, G);
  Job c{};
  bool unused, more = copies.next(c, unused);
  uint32_t first = more ? c.from : 0, k = 0, found = 0;  // of c, pieces from `first` on have been found, and k of them copied
  int stage = 0, ahead = 0;      // of the piece at hand, of the next one to be copied
  int64_t code_at = 0;           // where they lie: a lane a piece; its codes,
  int key_at = 0;                // its first row in the page, and 256 times its keys
  auto find = [&](uint32_t b) {
    if (b >= c.to) return;
    PageCursor cur(plan, *c.s);
    cur.go(b);
    const Run& run = cur.run;
    const int key = (static_cast<int>(b) - run.off) * PIECE;
    int block = a.tables[static_cast<int64_t>(run.row) * a.lay.max_blocks + key / page];
    if (block < 0 || block >= a.lay.n_blocks) {
      if (a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);
      block = 0;
    }
    code_at = (block * Hkv + c.s->h) * page_bytes + key % page * ROW;
    key_at = key % page + 256 * min(PIECE, run.keys - key);
  };
  const uint8_t *const k_lane = static_cast<const uint8_t*>(a.k_pool) + 16 * lane, *const v_lane = static_cast<const uint8_t*>(a.v_pool) + 16 * lane;
  const uint8_t* const s_lane = static_cast<const uint8_t*>(lane < SCALE_CHUNKS ? a.k_pool : a.v_pool) + page * ROW + 16 * (lane % SCALE_CHUNKS);
  uint32_t to_lane[CODES / 512];
#pragma unroll
  for (int i = 0; i < CODES / 512; ++i) {
    const int x = lane + 32 * i, r = x / CHUNKS;
    to_lane[i] = r * ROW + (((x % CHUNKS) ^ chunk_place<D>(r)) << 4);
  }
  auto copy = [&] {
    if (k == found && more) {
      first += k;
      k = 0;
      if (first == c.to) {  // (no segment is empty)
        more = copies.next(c, unused);
        first = c.from;
      }
      found = more ? min(32u, c.to - first) : 0;
      if (more) find(first + lane);
    }
    if (k < found) {
      const int64_t at = __shfl_sync(0xffffffffu, code_at, k);
      const int key = __shfl_sync(0xffffffffu, key_at, k);
      const uint32_t dst = base + ahead * STAGE;
#pragma unroll
      for (int i = 0; i < CODES / 512; ++i) {
        cp_async16(dst + to_lane[i], k_lane + at + 512 * i, true);
        cp_async16(dst + CODES + to_lane[i], v_lane + at + 512 * i, true);
      }
      if (lane < 2 * SCALE_CHUNKS)
        cp_async16_part(dst + 2 * CODES + 16 * lane, s_lane + at - (key & 255) * (ROW - SROW),
                        min(16, max(0, (key >> 8) * SROW - 16 * (lane % SCALE_CHUNKS))));
      ++k;
    }
    cp_async_commit();
    ahead = ahead + 1 == STAGES ? 0 : ahead + 1;
  };
#pragma unroll 1
  for (int i = 0; i + 2 < STAGES; ++i) copy();

  Jobs jobs(plan, work, G);
  Job j{};
  bool starts;
#pragma unroll 1
  while (jobs.next(j, starts)) {
    if (starts) rows_without_keys<T, D>(a, plan, *j.s, G, lane);
    const int prefix_keys = j.s->prefix_keys;
    auto wait = [&] {
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
      __syncwarp();
    };
    auto stage_at = [&] {
      const uint32_t at = base + stage * STAGE;
      if (++stage == STAGES) stage = 0;
      return at;
    };
    if (!j.eight) {
      Few16<T, D> f(a, plan, *j.s, j.rows, G, lane);
#pragma unroll 1
      for (uint32_t b = j.from; b < j.to; ++b) {
        copy();
        wait();
        f.step(stage_at(), prefix_keys, b * PIECE, bad, lane);
        __syncwarp();  // every lane has read the stage
      }
      f.finish(a, plan, *j.s, j.rows, G, lane);
      continue;
    }
    Few8<T, D> f(a, plan, *j.s, j.row0, j.rows, G, lane);
#pragma unroll 1
    for (uint32_t b = j.from; b < j.to; b += 2) {
      const bool two = b + 1 < j.to;
      copy();
      if (two) copy();
      wait();
      const uint32_t first = stage_at(), at[2] = {first, two ? stage_at() : first};
      f.step(at, scales, prefix_keys, b * PIECE, bad, lane);
      __syncwarp();
    }
    f.finish(a, plan, *j.s, j.row0, j.rows, G, lane);
  }
  if (bad && a.status) atomicCAS(a.status, 0, DOPR_ERR_RANGE);
}

// Tiles: K's or V's blocks into the raw ring, in halves of 64 rows.  A lane a piece: a page, or 64 rows of one of 128.
template <typename T, int D>
__device__ __forceinline__ void copy_4bit(const SharedAttnArgs& a, const Plan& plan, uint8_t* smem, uint32_t s0, int2 work, bool is_v, int* err,
                                          int lane) {
  using L = Smem<D, true>;
  constexpr int ROW = D / 2, SROW = D / 32;
  const int page = a.lay.page, page_blk = BLOCK / page, piece = min(page, 64), pieces_half = 64 / piece, Hkv = a.lay.n_kv_heads;
  const int stages = is_v ? L::RAW_V : L::RAW_K, stage0 = is_v ? L::RAW_K : 0;
  const uint8_t* pool = static_cast<const uint8_t*>(is_v ? a.v_pool : a.k_pool);
  const int64_t page_bytes = pages4::page_bytes(page, D);
  auto bar = [&](int i) { return s0 + L::OFF_BAR + 8u * static_cast<uint32_t>(i); };
  Walk walk(plan, work);
  Segment s;
  Ring r;
  uint32_t armed = 0, parity = 0;
  bool ok = true;
  const int pg = lane * piece / page, inside = lane * piece % page, my_half = lane / pieces_half;
  while (ok && walk.next(s)) {
    PageCursor cur(plan, s);
    for (uint32_t b = s.b0; b < s.b1 && ok; ++b) {
      const int first = b * page_blk, pages = min(page_blk, s.pages - first), cols = pages * page;
      const bool mine = pg < pages && lane * piece < cols;
      int keys = 0;
      const uint8_t* src = pool;
      if (mine) {
        cur.go(first + pg);
        int block = a.tables[static_cast<int64_t>(cur.run.row) * a.lay.max_blocks + first + pg - cur.run.off];
        if (block < 0 || block >= a.lay.n_blocks) {
          if (a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);
          block = 0;
        }
        keys = max(0, min(piece, cur.run.keys - (first + pg - cur.run.off) * page - inside));
        src += (block * Hkv + s.h) * page_bytes;
      }
      for (int half = 0; half * 64 < cols; ++half) {
        if (!wait_warp<true>(bar(L::RAW_EMPTY + stage0 + r.stage), r.phase ^ 1u, err, WAIT_TIMEOUT_NS)) {
          ok = false;
          break;
        }
        const uint32_t fb = bar(L::RAW_FULL + stage0 + r.stage);
        const bool now = mine && my_half == half;
        const int at = lane % pieces_half;
        if (now) smem[L::OFF_KEYS + (stage0 + r.stage) * 4 + at] = static_cast<uint8_t>(keys);
        __syncwarp();
        if (lane == 0) mbar_arrive_expect_tx(fb, min(64, cols - 64 * half) * (ROW + SROW));
        __syncwarp();
        if (now) {
          const uint32_t dst = s0 + L::OFF_RAW + (stage0 + r.stage) * L::RAW_BYTES + at * piece * (ROW + SROW);
          if (page == piece) {
            bulk_load(dst, src, piece * (ROW + SROW), fb);
          } else {
            bulk_load(dst, src + inside * ROW, 64 * ROW, fb);
            bulk_load(dst + 64 * ROW, src + page * ROW + inside * SROW, 64 * SROW, fb);
          }
        }
        __syncwarp();
        armed |= 1u << r.stage;
        parity = (parity & ~(1u << r.stage)) | r.phase << r.stage;
        r.next(stages);
      }
    }
  }
  if (!ok)  // copies in flight land before the CTA ends
    for (int i = 0; i < stages; ++i)
      if (armed >> i & 1u) wait_warp<true>(bar(L::RAW_FULL + stage0 + i), parity >> i & 1u, err, 100000000ull);
}

// Tiles: each block of K or V, by two warps, from the raw ring into the products' ring, in the layout that copies of 16-bit rows have
// there.  Bound by what fetching and waiting for instructions cost a warp alone on its part of a scheduler: loads of 16 rows before
// their stores took 2,048 rows on 16,384 keys from 482 us to 440, addresses once for 16 rows to 427; four such loads at once 450.
// Warp `part` takes 32 rows of each half, so that both pass every stage of the ring: a warp that skipped some could take the
// parity of a stage's phase before last for the one it waits for.  A lane a group: 16 bytes of codes to 64 of values.  Rows past a
// run's keys are zeros.
template <typename T, int D>
__device__ __forceinline__ void expand_4bit(const SharedAttnArgs& a, const Plan& plan, uint32_t s0, int2 work, bool is_v, int part,
                                            int* err, int lane) {
  using L = Smem<D, true>;
  constexpr int ROW = D / 2, SROW = D / 32, AT_ONCE = 32 / SROW, TIMES = 16 / AT_ONCE;
  const int page = a.lay.page, page_blk = BLOCK / page, piece = min(page, 64), bits = __ffs(piece) - 1;
  const int stages = is_v ? L::V_STAGES : L::K_STAGES, full = is_v ? L::V_FULL : L::K_FULL, empty = full + stages;
  const int raw_stages = is_v ? L::RAW_V : L::RAW_K, stage0 = is_v ? L::RAW_K : 0;
  auto bar = [&](int i) { return s0 + L::OFF_BAR + 8u * static_cast<uint32_t>(i); };
  const int group = lane % SROW, first = 32 * part + lane / SROW;
  // the half of the head, the row, and the first of four 16-byte places in it; lanes of the upper half of the head begin with their
  // third word, so that those that store at once meet all banks
  const bool swap = D == 128 && group >= 2;
  const uint32_t tile0 = s0 + (is_v ? L::OFF_V : L::OFF_K) + (D == 128 ? group >> 1 : 0) * HALF_BYTES + first * 128 +
                         ((((D == 128 ? group & 1 : group) * 4 + (swap ? 2 : 0)) ^ (first & 7)) << 4);
  Walk walk(plan, work);
  Segment s;
  Ring r, raw;
  bool ok = true, bad = false;
  while (ok && walk.next(s)) {
    for (uint32_t b = s.b0; b < s.b1 && ok; ++b) {
      const int cols = min(page_blk, s.pages - static_cast<int>(b) * page_blk) * page;
      if (!wait_warp<true>(bar(empty + r.stage), r.phase ^ 1u, err, WAIT_TIMEOUT_NS)) {
        ok = false;
        break;
      }
      for (int half = 0; 64 * half < cols; ++half) {
        const int rs = stage0 + raw.stage, rows = cols - 64 * half - 32 * part;  // of this warp's 32; a multiple of 16
        if (!wait_warp<true>(bar(L::RAW_FULL + rs), raw.phase, err, WAIT_TIMEOUT_NS)) {
          ok = false;
          break;
        }
        const uint32_t from = s0 + L::OFF_RAW + rs * L::RAW_BYTES, keys = lds32(s0 + L::OFF_KEYS + rs * 4);
        const uint32_t to = tile0 + r.stage * L::TILE_BYTES + 64 * half * 128;
        // 16 rows at a time, of one piece: codes and scales first, for the stores may not pass the loads, nor the other way round
#pragma unroll 1
        for (int r0 = 0; r0 < rows && r0 < 32; r0 += 16) {
          const int row = 32 * part + r0, at = row >> bits, in = row & (piece - 1);
          const int left = static_cast<int>(keys >> 8 * at & 0xffu) - in - lane / SROW;  // keys of the run from this lane's row on
          const uint32_t p = from + at * piece * (ROW + SROW), codes = p + in * ROW + 16 * lane, scales = p + piece * ROW + in * SROW + lane;
          uint4 w[TIMES];
          uint32_t byte[TIMES];
#pragma unroll
          for (int i = 0; i < TIMES; ++i) {
            w[i] = lds128(codes + i * 512);
            byte[i] = lds8(scales + i * 32);
          }
#pragma unroll
          for (int i = 0; i < TIMES; ++i) {
            const pages4::Widen<T> widen((i * AT_ONCE < left ? scale_of(byte[i], bad) : 0u) * 0x10001u);
            if (swap) w[i] = uint4{w[i].z, w[i].w, w[i].x, w[i].y};
            const uint32_t words[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              uint32_t x[4];
              widen(words[j], x);
              sts128((to ^ (j << 4)) + (r0 + i * AT_ONCE) * 128, uint4{x[0], x[1], x[2], x[3]});
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(L::RAW_EMPTY + rs));
        raw.next(raw_stages);
      }
      if (!ok) break;
      fence_proxy_async_shared();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(full + r.stage));
      r.next(stages);
    }
  }
  if (bad && a.status) atomicCAS(a.status, 0, DOPR_ERR_RANGE);
}

// The CTA: its threads take their roles here.  FOUR: the pools are those of the 4-bit cache (tm_k and tm_v are not used).
template <typename T, int D, bool FOUR>
__device__ __forceinline__ void attend(const CUtensorMap& tm_q8, const CUtensorMap& tm_q1, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                                       const SharedAttnArgs& a, const Plan& plan) {
  using L = Smem<D, FOUR>;
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
  const int2 work = plan.work[blockIdx.x * WORKERS + (warp >= 4 && warp < 12 ? warp - 4 : 0)];
  const Head head = *plan.head;
  prefetch_l2(a, plan);
  if (threadIdx.x < WORKERS) marked[threadIdx.x] = 0;
  if (threadIdx.x == 0) {
    gave_up = 0;
    for (int i = 0; i < L::N_BARS; ++i)
      mbar_init(bar(i), (i >= L::P_FULL && i < L::P_FULL + 4) || i == L::ML_FULL || i == L::ML_EMPTY ? 4
                        : FOUR && (i < L::K_EMPTY || (i >= L::V_FULL && i < L::V_EMPTY) || i >= L::RAW_EMPTY) ? 2  // two warps expand
                                                                                                              : 1);
    fence_mbar_init();
    tma_prefetch_desc(&tm_q8);
    tma_prefetch_desc(&tm_q1);
    if constexpr (!FOUR) {
      tma_prefetch_desc(&tm_k);
      tma_prefetch_desc(&tm_v);
    }
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  Segment s{};
  const bool good = made_for(head, a.lay, a.Hq, a.max_tokens, gridDim.x);
  const bool few = static_cast<int>(blockIdx.x) >= head.tile_ctas;
  if (!good && threadIdx.x == 0 && a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);

  if (!good) {
  } else if (few) {
    if (warp >= 4 && warp < 12) {
      regs_many<FOUR>();
      if constexpr (FOUR) few_items_4bit<T, D>(a, plan, s0, warp - 4, work, lane);
      else few_items<T, D>(a, plan, s0, warp - 4, work, &marked[warp - 4], lane);
    } else {
      regs_few<FOUR>();
    }
  } else if (warp == 0 || warp == 2) {
    // ======================= K and V blocks, page by page: a lane a page and half of the head (4 bits: a piece of a page)
    regs_few<FOUR>();
    if constexpr (FOUR) {
      copy_4bit<T, D>(a, plan, smem, s0, work, warp == 2, err, lane);
    } else {
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
          if (!wait_warp<FOUR>(bar(empty + r.stage), r.phase ^ 1u, err, WAIT_TIMEOUT_NS)) {
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
          if (armed >> i & 1u) wait_warp<FOUR>(bar(full + i), parity >> i & 1u, err, 100000000ull);
    }
  } else if (FOUR && warp >= 12) {
    // ======================= 4 bits: K (warps 12, 13) and V (14, 15) to the products' type
    regs_few<FOUR>();
    if constexpr (FOUR) expand_4bit<T, D>(a, plan, s0, work, warp >= 14, warp & 1, err, lane);
  } else if (warp == 1) {
    // ======================= MMA issuer
    regs_few<FOUR>();
    const bool one = elect_one();
    const uint32_t sQ = s0 + L::OFF_Q, sK = s0 + L::OFF_K, sV = s0 + L::OFF_V;
    const int page = a.lay.page, page_blk = BLOCK / page;
    Walk walk(plan, work);
    Groups groups;
    bool ok = true;
    auto wait = [&](int b, uint32_t par) { return ok = ok && wait_warp<FOUR>(bar(b), par, err, WAIT_TIMEOUT_NS); };
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
    wait_warp<FOUR>(bar(L::DRAIN), 0, err, ok ? WAIT_TIMEOUT_NS : 100000000ull);
  } else if (warp == 3) {
    // ======================= rows of Q: row r of a group's tile is token r / G of the tile, head r % G of the kv head's
    regs_few<FOUR>();
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
        if ((used >> w & 1u) && !wait_warp<FOUR>(bar(L::Q_EMPTY + w), par >> w & 1u, err, WAIT_TIMEOUT_NS)) {
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
        if (used >> w & 1u) wait_warp<FOUR>(bar(L::Q_FULL + w), (filled >> w & 1u) ^ 1u, err, 100000000ull);
  } else {
    // ======================= softmax: thread r of group w has row r of its tile
    regs_many<FOUR>();
    const int w = (warp >> 2) - 1, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lane_base = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    const uint32_t s_col = lane_base + S_COL + 128 * w, o_col = lane_base + O_COL + 128 * w;
    const float scale_log2 = a.scale * 1.4426950408889634f * HELD_UNIT<T, FOUR>;
    const int2* own_columns = plan.own;
    const int* order = plan.order;
    Walk walk(plan, work);
    Groups groups;
    Ring rv;
    uint32_t s_par = 0, o_par = 0;
    bool ok = true;
    // (the first group that takes a block) rows of V past a page's keys count as zero: before any of P is given
    auto ready_v = [&](int stage, uint32_t phase, int cols) {
      if (!wait_warp<FOUR>(bar(L::V_FULL + stage), phase, err, WAIT_TIMEOUT_NS)) return false;
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
        if (!wait_warp<FOUR>(bar(L::ML_EMPTY), (o_par & SUMS) == 0, err, WAIT_TIMEOUT_NS)) break;
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
        if (!wait_warp<FOUR>(bar(L::S_FULL + w), s_par, err, WAIT_TIMEOUT_NS)) {
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
          if (!FOUR && ragged && !(ok = ready_v(v_stage, v_phase, cols))) break;
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
        if (!FOUR && ragged && !(ok = ready_v(v_stage, v_phase, cols))) break;
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
        if (!wait_warp<FOUR>(bar(L::O_FULL + w), o_par & 1u, err, WAIT_TIMEOUT_NS)) break;
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
          if (!wait_warp<FOUR>(bar(L::ML_FULL), (o_par & SUMS) != 0, err, WAIT_TIMEOUT_NS)) break;
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
        const float inv = inverse(l) * HELD_UNIT<T, FOUR>;
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
              uint32_t x[8] = {v[i], v[i + 1], v[i + 2], v[i + 3], v[i + 4], v[i + 5], v[i + 6], v[i + 7]};
              if constexpr (HELD_UNIT<T, FOUR> != 1.f) {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * HELD_UNIT<T, FOUR>);
              }
              st_global32(dst + c + i, x);
            }
          }
        }
      }
      // scores in order, values not: perhaps a value that the row does not see
      if (!FOUR && __any_sync(0xffffffffu, valid && all != all && l > 0.f) && lane == 0) marked[warp - 4] |= 1u << (walk.at - 1 & 31);
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
  if constexpr (!FOUR) {
    if (warp >= 4 && marked[warp - 4] != 0) mend_segments<T, D>(a, plan, marked[warp - 4], warp - 4, lane);
  }
}
// Q by boxes of eight tokens that follow one another and of one; views that a tensor map does not take (one row for all
// tokens) are gathered, and `other` stands for the maps.
inline bool make_q_maps(SharedAttnArgs& a, bool half, CUtensorMap* tm_q8, CUtensorMap* tm_q1, const CUtensorMap& other) {
  const int G = a.Hq / a.lay.n_kv_heads, D = a.lay.head_dim;
  a.q_boxes = make_tmap_rows_of_heads(tm_q1, a.q, D, a.Hq, a.max_tokens, a.q_head, a.q_tok, G, 1, half);
  if (!a.q_boxes) *tm_q1 = other;
  if (a.q_boxes && tokens_a_tile(G) >= 8) return make_tmap_rows_of_heads(tm_q8, a.q, D, a.Hq, a.max_tokens, a.q_head, a.q_tok, G, 8, half);
  *tm_q8 = *tm_q1;
  return true;
}

}  // namespace
}  // namespace dopr
