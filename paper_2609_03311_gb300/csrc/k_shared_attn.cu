// k_shared_attn.cu -- attention of a step's tokens over a paged cache (dopr_shared_attention): the keys of the row's
// prefix, then the row's own up to the token.
//
// softmax(scale q k^T) v in one pass over the keys: with m the running maximum of the scores and l the running sum of
// exp(score - m), a new score s > m scales what was summed by exp(m - s).
#include "device_common.cuh"
#include "internal.h"

namespace dopr {
namespace {

constexpr int PLAN_THREADS = 1024, ROW_WARPS = 4;
constexpr int PLAN_HEAD = 16;  // ints; [0]: tokens (0 where the plan is empty)
// Then an int4 a token: own row, own keys it sees, prefix row (-1: none), prefix keys.

__global__ void __launch_bounds__(PLAN_THREADS) k_shared_plan(SharedPlanArgs a) {
  __shared__ int bad;
  const int n = a.lay.n_seqs;
  const int64_t cap = static_cast<int64_t>(a.lay.max_blocks) * a.lay.page;
  if (threadIdx.x == 0) bad = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += PLAN_THREADS) {
    const int t0 = a.tok_off[i], t1 = a.tok_off[i + 1], pre = a.prefix ? a.prefix[i] : -1;
    if ((i == 0 && t0 != 0) || t1 < t0 || t1 > a.max_tokens || a.seq_lens[i] < 0 || a.seq_lens[i] > cap || pre < -1 || pre >= n ||
        pre == i || (pre >= 0 && a.prefix[pre] != -1))
      bad = 1;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    a.plan[0] = bad ? 0 : a.tok_off[n];
    if (bad && a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);
  }
  if (bad) return;
  int4* rec = reinterpret_cast<int4*>(a.plan + PLAN_HEAD);
  for (int t = threadIdx.x; t < a.tok_off[n]; t += PLAN_THREADS) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.tok_off[mid] <= t) lo = mid; else hi = mid - 1;
    }
    const int pre = a.prefix ? a.prefix[lo] : -1;
    const int own = a.seq_lens[lo] - (a.tok_off[lo + 1] - a.tok_off[lo]) + (t - a.tok_off[lo]) + 1;
    rec[t] = make_int4(lo, min(max(own, 0), a.seq_lens[lo]), pre, pre >= 0 ? a.seq_lens[pre] : 0);
  }
}

template <typename T>
__device__ __forceinline__ float2 pair_f32(uint32_t w) {
  if constexpr (sizeof(T) && std::is_same_v<T, __half>) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  else return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w));
}
template <typename T>
__device__ __forceinline__ uint32_t pack_f32(float x, float y) {
  if constexpr (std::is_same_v<T, __half>) return pack_f16x2(x, y);
  else return pack_bf16x2(x, y);
}

// A warp per token and q head, a key at a time; lane l holds elements [E l, E l + E) of the head.
template <typename T, int D>
__global__ void __launch_bounds__(32 * ROW_WARPS) k_attn_rows(SharedAttnArgs a) {
  constexpr int E = D / 32, W = E / 2;  // elements and 32-bit words a lane
  const int lane = threadIdx.x & 31;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * ROW_WARPS + (threadIdx.x >> 5);
  pdl_wait();
  pdl_trigger();
  const int32_t* plan = static_cast<const int32_t*>(a.plan);
  if (unit >= static_cast<int64_t>(plan[0]) * a.Hq) return;
  const int t = static_cast<int>(unit / a.Hq), h = static_cast<int>(unit % a.Hq);
  const int4 rec = reinterpret_cast<const int4*>(plan + PLAN_HEAD)[t];
  const int page = a.lay.page, Hkv = a.lay.n_kv_heads, kvh = h / (a.Hq / Hkv);
  const uint32_t* qp = reinterpret_cast<const uint32_t*>(static_cast<const T*>(a.q) + t * a.q_tok + h * a.q_head) + lane * W;
  float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const float2 f = pair_f32<T>(qp[i]);
    q[2 * i] = f.x * a.scale, q[2 * i + 1] = f.y * a.scale;
    o[2 * i] = o[2 * i + 1] = 0.f;
  }
  for (int part = 0; part < 2; ++part) {
    const int row = part ? rec.x : rec.z, n = part ? rec.y : rec.w;
    for (int p = 0; p < n; ++p) {
      int block = a.tables[static_cast<int64_t>(row) * a.lay.max_blocks + p / page];
      if (block < 0 || block >= a.lay.n_blocks) {
        if (a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);
        block = 0;
      }
      const int64_t at = ((static_cast<int64_t>(block) * Hkv + kvh) * page + p % page) * (D / 2) + lane * W;
      const uint32_t* kp = static_cast<const uint32_t*>(a.k_pool) + at;
      const uint32_t* vp = static_cast<const uint32_t*>(a.v_pool) + at;
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float2 f = pair_f32<T>(kp[i]);
        s += q[2 * i] * f.x + q[2 * i + 1] * f.y;
      }
      s = warp_sum(s);
      const float top = fmaxf(m, s), shift = top == -INFINITY ? 0.f : top;
      const float old = expf(m - shift), e = expf(s - shift);
      m = top;
      l = l * old + e;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float2 f = pair_f32<T>(vp[i]);
        o[2 * i] = o[2 * i] * old + e * f.x;
        o[2 * i + 1] = o[2 * i + 1] * old + e * f.y;
      }
    }
  }
  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;  // a NaN stays one
  uint32_t* op = reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + t * a.o_tok + h * a.o_head) + lane * W;
#pragma unroll
  for (int i = 0; i < W; ++i) op[i] = pack_f32<T>(o[2 * i] * inv, o[2 * i + 1] * inv);
  if (a.lse && lane == 0) a.lse[static_cast<int64_t>(t) * a.Hq + h] = m + logf(l);
}

template <typename T, int D>
cudaError_t launch_rows(const SharedAttnArgs& a, cudaStream_t st) {
  const int64_t units = static_cast<int64_t>(a.max_tokens) * a.Hq;
  return launch_dependent(k_attn_rows<T, D>, dim3(static_cast<unsigned>((units + ROW_WARPS - 1) / ROW_WARPS)), 32 * ROW_WARPS,
                          0, st, a);
}

}  // namespace

int64_t shared_plan_bytes(const dopr_cache_layout&, int, int max_tokens) {
  return PLAN_HEAD * 4 + static_cast<int64_t>(max_tokens) * 16;
}
int64_t shared_workspace_bytes(const dopr_cache_layout&, int, int, int) { return 16; }

cudaError_t launch_shared_plan(const SharedPlanArgs& a, cudaStream_t st) {
  return launch_dependent(k_shared_plan, dim3(1), PLAN_THREADS, 0, st, a);
}
cudaError_t launch_shared_attention(const SharedAttnArgs& a, cudaStream_t st) {
  const bool half = a.lay.dtype == DOPR_F16;
  if (a.lay.head_dim == 128) return half ? launch_rows<__half, 128>(a, st) : launch_rows<__nv_bfloat16, 128>(a, st);
  return half ? launch_rows<__half, 64>(a, st) : launch_rows<__nv_bfloat16, 64>(a, st);
}

}  // namespace dopr
