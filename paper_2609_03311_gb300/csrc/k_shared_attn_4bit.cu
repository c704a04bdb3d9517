// k_shared_attn_4bit.cu -- attention of a step's tokens over a paged cache in 4 bits (dopr_shared_attention_4bit): the work of
// k_shared_attn.cu by the same plan, with keys and values that are held as pages4.cuh says.
//
// softmax(scale q k^T) v, k and v the values c s that the codes and scales stand for.  They are exact in the products' type, so
// the arithmetic is that of the 16-bit cache on those values.
//   Tiles: 512 threads a CTA.  Blocks come as they are held, by bulk copies of a page each (codes and scales lie together), into a
//   ring of halves of 64 rows; four warps widen them into the rings that the products read.
//   Few items: a warp a part of one; codes go into the products without their scales, or are widened in registers where
//   parts are short.
// Every finite scale gives finite values, and one that stands for NaN counts as zero and is an error, so a column that a row does
// not see can add nothing to it, and no row is looked at again.
#include "shared_attn_device.cuh"

namespace dopr {
namespace {

template <typename T, int D>
__global__ void __launch_bounds__(THREADS<true>, 1)
    k_shared_attn_4bit(const __grid_constant__ CUtensorMap tm_q8, const __grid_constant__ CUtensorMap tm_q1,
                       const __grid_constant__ SharedAttnArgs a, const __grid_constant__ Plan plan) {
  pdl_trigger();
  attend<T, D, true>(tm_q8, tm_q1, tm_q1, tm_q1, a, plan);
}

template <typename T, int D>
cudaError_t launch(const SharedAttnArgs& a, int num_sms, cudaStream_t st) {
  using L = Smem<D, true>;
  const int n_ctas = num_sms < MAX_CTAS ? num_sms : MAX_CTAS;
  const Plan plan = plan_view(const_cast<void*>(a.plan), a.lay.n_seqs, a.lay.n_kv_heads, a.Hq / a.lay.n_kv_heads, a.max_tokens);
  SharedAttnArgs args = a;
  CUtensorMap tm_q8, tm_q1;
  // (stands for the maps where Q is gathered: nothing is copied by it)
  CUtensorMap other;
  const bool half = std::is_same_v<T, __half>;
  if (!make_tmap_16b_2d(&other, a.k_pool, 64, 1, 128, 64, 1, true, half) || !make_q_maps(args, half, &tm_q8, &tm_q1, other))
    return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(k_shared_attn_4bit<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
  if (e != cudaSuccess) return e;
  // not a dependent launch: the joining kernel relies on that
  e = launch_ordinary(k_shared_attn_4bit<T, D>, dim3(n_ctas), THREADS<true>, L::BYTES, st, tm_q8, tm_q1, args, plan);
  if (e != cudaSuccess) return e;
  return launch_shared_join(a, num_sms, st);
}

}  // namespace

cudaError_t launch_shared_attention_4bit(const SharedAttnArgs& a, int num_sms, cudaStream_t st) {
  const bool half = a.lay.dtype == DOPR_F16;
  if (a.lay.head_dim == 128) return half ? launch<__half, 128>(a, num_sms, st) : launch<__nv_bfloat16, 128>(a, num_sms, st);
  return half ? launch<__half, 64>(a, num_sms, st) : launch<__nv_bfloat16, 64>(a, num_sms, st);
}

}  // namespace dopr
