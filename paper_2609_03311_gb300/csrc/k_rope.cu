// k_rope.cu -- rotary positions on packed rows of heads (dopr_rope_apply), and the same with keys and values on
// their way into the cache's pages (dopr_cache_append).
//
// A pair of elements is a point in the plane that turns by position * f_i.  Far positions times a frequency lose
// their angle in 32 bits (at 250,000 radians a step is 0.016), so angles and their cos and sin are taken in 64 bits,
// once, into a table; what is left for a row is four products of 32 bits a pair.
//
// Bound by HBM: a row is read once and written once, 24 KB of 16-bit q, k and v for 32 + 2 x 8 heads of 128.  26,800 of them
// take 110 us, 6.0 TB/s; 4,097 rows of 24 heads in 32 bits, 17.3 us, 5.8 TB/s.  A thread takes one unit of 2 x VEC
// elements (16 bytes of each half of the pairs; 32 contiguous bytes where pairs are interleaved) and walks over the
// heads with it, so that it reads its cos and sin once a row.  Two or three heads on their way a thread were slower (115 us
// a chunk): what counts is how many threads an SM holds.  Views that 16-byte accesses do not fit go element by element.
#include <type_traits>

#include "device_common.cuh"
#include "internal.h"

namespace dopr {
namespace {

constexpr int MAX_THREADS = 256;

template <typename T>
__device__ __forceinline__ float to_f32(T x) {
  if constexpr (std::is_same_v<T, float>) return x;
  else if constexpr (std::is_same_v<T, __half>) return __half2float(x);
  else return __bfloat162float(x);
}
template <typename T>
__device__ __forceinline__ T from_f32(float x) {
  if constexpr (std::is_same_v<T, float>) return x;
  else if constexpr (std::is_same_v<T, __half>) return __float2half_rn(x);
  else return __float2bfloat16_rn(x);
}

// VEC elements, 16 bytes of them at once where VEC > 1.
template <typename T, int VEC>
struct alignas(VEC > 1 ? 16 : sizeof(T)) Pack {
  T v[VEC];
};

__global__ void __launch_bounds__(256) k_rope_table(const double* freq, double gain, int max_position, int half,
                                                    float2* table) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= static_cast<int64_t>(max_position) * half) return;
  double s, c;
  sincos(static_cast<double>(i / half) * freq[i % half], &s, &c);
  table[i] = make_float2(static_cast<float>(c * gain), static_cast<float>(s * gain));
}

// (x, y) turned.  The fused steps are spelled out so that every variant gives the same bits.
template <typename T>
__device__ __forceinline__ void turn_pair(T& a, T& b, float c, float s) {
  const float x = to_f32(a), y = to_f32(b);
  a = from_f32<T>(__fmaf_rn(x, c, -__fmul_rn(y, s)));
  b = from_f32<T>(__fmaf_rn(y, c, __fmul_rn(x, s)));
}

// One unit of one head: elements a[] and b[], VEC each, at offsets ia and ib of the head.
template <typename T, int VEC, bool INTER>
__device__ __forceinline__ void turn(Pack<T, VEC>& a, Pack<T, VEC>& b, const float (&c)[VEC], const float (&s)[VEC]) {
  if constexpr (INTER && VEC > 1) {
    // pairs (2i, 2i + 1) lie in order over a, then b
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) {
      turn_pair(a.v[2 * i], a.v[2 * i + 1], c[i], s[i]);
      turn_pair(b.v[2 * i], b.v[2 * i + 1], c[VEC / 2 + i], s[VEC / 2 + i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) turn_pair(a.v[i], b.v[i], c[i], s[i]);
  }
}

template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(MAX_THREADS) k_rope(RopeArgs a) {
  const int units = a.head_dim / (2 * VEC), turning = a.rotary / (2 * VEC);
  const int lanes = blockDim.x / units;  // heads at once
  const int u = threadIdx.x % units, h0 = threadIdx.x / units;
  // unit u's two runs of VEC elements
  const int ia = u < turning && !INTER ? u * VEC : u * 2 * VEC;
  const int ib = u < turning && !INTER ? ia + a.rotary / 2 : ia + VEC;
  const int heads = a.q.n_heads + a.k.n_heads + a.v.n_heads;
  const int page_bits = __ffs(a.page) - 1;  // a power of two
  pdl_wait();
  pdl_trigger();
  if (h0 >= lanes) return;
  // (compared as unsigned: the step behind the last of 2^31 - 1 tokens; an unsigned t takes 8 registers more, and 4,097 rows 18.0 us)
  for (int t = blockIdx.x; static_cast<uint32_t>(t) < static_cast<uint32_t>(a.n_tokens); t = static_cast<int>(t + gridDim.x)) {
    const int pos = a.rotary > 0 ? a.positions[t] : 0;
    const int64_t slot = a.slots ? a.slots[t] : -1;
    // the first head's elements are asked for beside the position and the table
    Pack<T, VEC> p0, p1;
    auto load = [&](int h) {
      const bool is_q = h < a.q.n_heads, is_v = h >= a.q.n_heads + a.k.n_heads;
      const RopeView& view = is_q ? a.q : is_v ? a.v : a.k;
      const int hh = is_q ? h : is_v ? h - a.q.n_heads - a.k.n_heads : h - a.q.n_heads;
      const T* x = static_cast<const T*>(view.in) + t * view.in_tok + hh * view.in_head;
      p0 = *reinterpret_cast<const Pack<T, VEC>*>(x + ia);
      p1 = *reinterpret_cast<const Pack<T, VEC>*>(x + ib);
    };
    if (h0 < heads) load(h0);
    float c[VEC], s[VEC];
    if (a.rotary > 0) {
      if (pos < 0) continue;
      if (pos >= a.max_position) {
        if (a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);
        continue;
      }
      if (u < turning) {
        const float2* cs = a.table + static_cast<int64_t>(pos) * (a.rotary / 2) + u * VEC;
        if constexpr (VEC > 1) {
#pragma unroll
          for (int i = 0; i < VEC; i += 2) {
            const float4 e = __ldg(reinterpret_cast<const float4*>(cs + i));
            c[i] = e.x, s[i] = e.y, c[i + 1] = e.z, s[i + 1] = e.w;
          }
        } else {
          const float2 e = __ldg(cs);
          c[0] = e.x, s[0] = e.y;
        }
        if (a.inverse) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) s[i] = -s[i];
        }
      }
    }
    if (slot >= a.n_slots && a.slots) {
      if (a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);
      continue;
    }
    for (int h = h0; h < heads;) {
      const bool is_q = h < a.q.n_heads, is_v = h >= a.q.n_heads + a.k.n_heads;
      if (!is_q && a.slots && slot < 0) break;  // the row is not stored; heads go up
      const RopeView& view = is_q ? a.q : is_v ? a.v : a.k;
      const int hh = is_q ? h : is_v ? h - a.q.n_heads - a.k.n_heads : h - a.q.n_heads;
      T* y;
      if (is_q || !a.slots) {
        y = static_cast<T*>(view.out) + t * view.out_tok + hh * view.out_head;
      } else {
        const int64_t row = (((slot >> page_bits) * a.k.n_heads + hh) << page_bits) + (slot & (a.page - 1));
        y = static_cast<T*>(is_v ? a.v_pool : a.k_pool) + row * a.head_dim;
      }
      if (u < turning && !is_v) turn<T, VEC, INTER>(p0, p1, c, s);
      *reinterpret_cast<Pack<T, VEC>*>(y + ia) = p0;
      *reinterpret_cast<Pack<T, VEC>*>(y + ib) = p1;
      h += lanes;
      if (h < heads) load(h);
    }
  }
}

bool aligned16(const void* p, int64_t s0, int64_t s1, int size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s0 * size % 16 == 0 && s1 * size % 16 == 0;
}

template <typename T, int VEC, bool INTER>
cudaError_t launch(const RopeArgs& a, cudaStream_t st) {
  // few tokens leave most SMs idle: more threads a token make fewer turns over the heads; of many tokens the heads fill 128 more
  // evenly.  40 heads of 128 in bf16, with 256 threads and with 128: one token 2.5 and 2.8 us, 128 2.6 and 2.9, 256 3.0 and 3.2,
  // 384 3.7 and 3.4, 640 5.6 and 4.0; a chunk of 26,800 into the cache 138 and 110.  (24 heads in 32 bits: 384 2.8 and 3.0, 512
  // 3.6 and 3.2; 10 heads of 64: the same to 256, 384 2.4 and 2.0.)
  const int threads = a.n_tokens <= 256 ? MAX_THREADS : MAX_THREADS / 2;
  return launch_dependent(k_rope<T, VEC, INTER>, dim3(a.n_tokens < 65536 ? a.n_tokens : 65536), threads, 0, st, a);
}
template <typename T>
cudaError_t launch_type(const RopeArgs& a, cudaStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  bool wide = a.rotary / 2 % VEC == 0 && (a.head_dim - a.rotary) % (2 * VEC) == 0;
  for (const RopeView* v : {&a.q, &a.k, &a.v}) {
    if (v->n_heads == 0) continue;
    wide = wide && aligned16(v->in, v->in_tok, v->in_head, sizeof(T));
    if (v->out) wide = wide && aligned16(v->out, v->out_tok, v->out_head, sizeof(T));
  }
  if (wide) return a.interleaved ? launch<T, VEC, true>(a, st) : launch<T, VEC, false>(a, st);
  return a.interleaved ? launch<T, 1, true>(a, st) : launch<T, 1, false>(a, st);
}

}  // namespace

cudaError_t launch_rope_table(const double* freq, double gain, int max_position, int half, float2* table,
                              cudaStream_t st) {
  const int64_t n = static_cast<int64_t>(max_position) * half;
  return launch_ordinary(k_rope_table, dim3(static_cast<unsigned>((n + 255) / 256)), 256, 0, st, freq, gain, max_position, half, table);
}

cudaError_t launch_rope(int dtype, const RopeArgs& a, cudaStream_t st) {
  if (a.n_tokens == 0) return cudaSuccess;
  switch (dtype) {
    case DOPR_F16: return launch_type<__half>(a, st);
    case DOPR_BF16: return launch_type<__nv_bfloat16>(a, st);
    default: return launch_type<float>(a, st);
  }
}

}  // namespace dopr
