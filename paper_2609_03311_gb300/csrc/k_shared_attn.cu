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
#include "shared_attn_device.cuh"

namespace dopr {
namespace {

// of the joining kernel on an SM (3 with twice the loads on their way: 64 rows a little faster, 16 documents 3 % slower)
constexpr int JOIN_CTAS = 4;

template <typename T, int D>
__global__ void __launch_bounds__(THREADS<false>, 1)
    k_shared_attn(const __grid_constant__ CUtensorMap tm_q8, const __grid_constant__ CUtensorMap tm_q1,
                  const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const __grid_constant__ SharedAttnArgs a, const __grid_constant__ Plan plan) {
  pdl_trigger();
  attend<T, D, false>(tm_q8, tm_q1, tm_k, tm_v, a, plan);
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
cudaError_t launch_join(const SharedAttnArgs& a, int num_sms, cudaStream_t st);

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
  SharedAttnArgs args = a;
  if (!make_q_maps(args, half, &tm_q8, &tm_q1, tm_k)) return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(k_shared_attn<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<D>::BYTES);
  if (e != cudaSuccess) return e;
  // not a dependent launch: the joining kernel relies on that
  e = launch_ordinary(k_shared_attn<T, D>, dim3(n_ctas), THREADS<false>, Smem<D>::BYTES, st, tm_q8, tm_q1, tm_k, tm_v, args, plan);
  if (e != cudaSuccess) return e;
  return launch_join<T, D>(a, num_sms, st);
}

template <typename T, int D>
cudaError_t launch_join(const SharedAttnArgs& a, int num_sms, cudaStream_t st) {
  const int n_ctas = num_sms < MAX_CTAS ? num_sms : MAX_CTAS;
  const Plan plan = plan_view(const_cast<void*>(a.plan), a.lay.n_seqs, a.lay.n_kv_heads, a.Hq / a.lay.n_kv_heads, a.max_tokens);
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

cudaError_t launch_shared_join(const SharedAttnArgs& a, int num_sms, cudaStream_t st) {
  const bool half = a.lay.dtype == DOPR_F16;
  if (a.lay.head_dim == 128) return half ? launch_join<__half, 128>(a, num_sms, st) : launch_join<__nv_bfloat16, 128>(a, num_sms, st);
  return half ? launch_join<__half, 64>(a, num_sms, st) : launch_join<__nv_bfloat16, 64>(a, num_sms, st);
}

cudaError_t launch_shared_attention(const SharedAttnArgs& a, int num_sms, cudaStream_t st) {
  const bool half = a.lay.dtype == DOPR_F16;
  if (a.lay.head_dim == 128) return half ? launch<__half, 128>(a, num_sms, st) : launch<__nv_bfloat16, 128>(a, num_sms, st);
  return half ? launch<__half, 64>(a, num_sms, st) : launch<__nv_bfloat16, 64>(a, num_sms, st);
}

}  // namespace dopr