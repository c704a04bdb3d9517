// k_head_norm.cu -- RMSNorm of each query and key head with a gain, and rotary positions, in one pass (dopr_head_norm_rope),
// its gradients (dopr_head_norm_rope_backward), and the same on the way into 4-bit pages (dopr_cache_append_4bit).
//
// x a head of D elements, r = (sum x^2 / D + eps)^-1/2, y = x r g, z = R y with R the turn of k_rope.cu.  The gradient: with
// dz that of z, dy = R^T dz (the turn back, times the same factor), w = dy g:
//   dx = r (w - x r^2 (sum w x) / D),   dg = the sum of dy x r over all rows and heads.
// r is made again from x, which has to be read anyway.  Sums are of 32 bits.
//
// Bound by HBM: rows are read once and written once (backward: two read, one written).  A head's elements lie in a power of two
// of lanes of one warp, a unit of 2 x VEC elements each (16 bytes of each half of the pairs, 32 contiguous bytes where pairs are
// interleaved), so that its sums take shuffles alone; views that 16-byte accesses do not fit go element by element, a
// warp a head.
#include <type_traits>

#include "internal.h"
#include "pages4.cuh"

namespace dopr {
namespace {

constexpr int THREADS = 128, MAX_DIM = 256;

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

__device__ __forceinline__ float gain_at(const void* gain, int dtype, int i) {
  if (!gain) return 1.f;
  if (dtype == DOPR_F32) return static_cast<const float*>(gain)[i];
  if (dtype == DOPR_F16) return __half2float(static_cast<const __half*>(gain)[i]);
  return __bfloat162float(static_cast<const __nv_bfloat16*>(gain)[i]);
}

__device__ __forceinline__ void set_status(int32_t* status, int what) {
  if (status) atomicCAS(status, 0, what);
}

// NU units of a head, a lane's: where their runs of VEC elements begin, and the cos and sin of their pairs.
template <int VEC, int NU, bool INTER>
struct Units {
  int ia[NU], ib[NU];
  bool there[NU], turns[NU];
  __device__ __forceinline__ Units(int sub, int head_dim, int rotary) {
    const int units = head_dim / (2 * VEC), turning = rotary / (2 * VEC);
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int u = sub + 32 * i;
      there[i] = u < units;
      turns[i] = u < turning;
      ia[i] = turns[i] && !INTER ? u * VEC : u * 2 * VEC;
      ib[i] = turns[i] && !INTER ? ia[i] + rotary / 2 : ia[i] + VEC;
    }
  }
  // back: the turn the other way
  __device__ __forceinline__ void angles(const float2* table, int64_t pos, int rotary, int sub, bool back, float (&c)[NU][VEC],
                                         float (&s)[NU][VEC]) const {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      if (!turns[i]) continue;
      const float2* cs = table + pos * (rotary / 2) + (sub + 32 * i) * VEC;
      if constexpr (VEC > 1) {
#pragma unroll
        for (int j = 0; j < VEC; j += 2) {
          const float4 e = __ldg(reinterpret_cast<const float4*>(cs + j));
          c[i][j] = e.x, s[i][j] = e.y, c[i][j + 1] = e.z, s[i][j + 1] = e.w;
        }
      } else {
        const float2 e = __ldg(cs);
        c[i][0] = e.x, s[i][0] = e.y;
      }
      if (back) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) s[i][j] = -s[i][j];
      }
    }
  }
  // Elements [0, VEC) of x are a unit's first run, the others its second.
  __device__ __forceinline__ void turn(float (&x)[NU][2 * VEC], const float (&c)[NU][VEC], const float (&s)[NU][VEC]) const {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      if (!turns[i]) continue;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        // interleaved: pairs lie in order over both runs
        constexpr bool APART = !INTER || VEC == 1;
        float &a = APART ? x[i][j] : x[i][2 * j], &b = APART ? x[i][VEC + j] : x[i][2 * j + 1];
        const float u = a, v = b;
        a = __fmaf_rn(u, c[i][j], -__fmul_rn(v, s[i][j]));
        b = __fmaf_rn(v, c[i][j], __fmul_rn(u, s[i][j]));
      }
    }
  }
  template <typename T>
  __device__ __forceinline__ void load(const T* row, bool valid, Pack<T, VEC> (&a)[NU], Pack<T, VEC> (&b)[NU]) const {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      if (!there[i] || !valid) continue;
      a[i] = *reinterpret_cast<const Pack<T, VEC>*>(row + ia[i]);
      b[i] = *reinterpret_cast<const Pack<T, VEC>*>(row + ib[i]);
    }
  }
  template <typename T>
  __device__ __forceinline__ void widen(const Pack<T, VEC> (&a)[NU], const Pack<T, VEC> (&b)[NU], bool valid, float (&x)[NU][2 * VEC]) const {
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        x[i][j] = there[i] && valid ? to_f32(a[i].v[j]) : 0.f;
        x[i][VEC + j] = there[i] && valid ? to_f32(b[i].v[j]) : 0.f;
      }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, const float (&x)[NU][2 * VEC]) const {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      if (!there[i]) continue;
      Pack<T, VEC> a, b;
#pragma unroll
      for (int j = 0; j < VEC; ++j) a.v[j] = from_f32<T>(x[i][j]), b.v[j] = from_f32<T>(x[i][VEC + j]);
      *reinterpret_cast<Pack<T, VEC>*>(row + ia[i]) = a;
      *reinterpret_cast<Pack<T, VEC>*>(row + ib[i]) = b;
    }
  }
  __device__ __forceinline__ void gains(const float* from, float (&g)[NU][2 * VEC]) const {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      if (!there[i]) continue;
#pragma unroll
      for (int j = 0; j < VEC; ++j) g[i][j] = from[ia[i] + j], g[i][VEC + j] = from[ib[i] + j];
    }
  }
};

// Adds up over the `lanes` (a power of two) lanes that hold a head.
__device__ __forceinline__ float head_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// PAGES: keys and values go to 4-bit pages.
template <typename T, int VEC, int NU, bool INTER, bool PAGES>
__global__ void __launch_bounds__(THREADS) k_head_norm(const __grid_constant__ HeadNormArgs a, int lanes) {
  __shared__ float gain[2][MAX_DIM];
  __shared__ __align__(16) float most[PAGES ? THREADS / 4 : 1][16];  // of each head at work, the largest magnitudes of its runs of eight
  const int D = a.head_dim, lane = threadIdx.x & 31, sub = lane & (lanes - 1), per_warp = 32 / lanes;
  const int at_once = THREADS / lanes, h_first = blockIdx.y * at_once + (threadIdx.x >> 5) * per_warp;
  const int heads = a.q.n_heads + a.k.n_heads + a.v.n_heads, step = at_once * gridDim.y;
  const Units<VEC, NU, INTER> units(sub, D, a.rotary);
  const int page_bits = PAGES ? __ffs(a.page) - 1 : 0;
  pdl_wait();
  pdl_trigger();
  if (a.eps > 0.f) {
    for (int i = threadIdx.x; i < D; i += THREADS) {
      gain[0][i] = gain_at(a.q_gain, a.gain_dtype, i);
      gain[1][i] = gain_at(a.k_gain, a.gain_dtype, i);
    }
    __syncthreads();
  }
  const float inv_d = 1.f / D;
  for (int t = blockIdx.x; static_cast<uint32_t>(t) < static_cast<uint32_t>(a.n_tokens); t = static_cast<int>(t + gridDim.x)) {
    const int pos = a.rotary > 0 ? a.positions[t] : 0;
    const int64_t slot = PAGES ? a.slots[t] : 0;
    Pack<T, VEC> p0[NU], p1[NU];
    auto load = [&](int h) {
      const bool is_q = h < a.q.n_heads, is_v = h >= a.q.n_heads + a.k.n_heads;
      const RopeView& view = is_q ? a.q : is_v ? a.v : a.k;
      const int hh = is_q ? h : is_v ? h - a.q.n_heads - a.k.n_heads : h - a.q.n_heads;
      units.load(static_cast<const T*>(view.in) + t * view.in_tok + hh * view.in_head, h < heads, p0, p1);
    };
    load(h_first + lane / lanes);
    if (pos < 0) continue;
    float c[NU][VEC], s[NU][VEC];
    if (a.rotary > 0) {
      if (pos >= a.max_position) {
        set_status(a.status, DOPR_ERR_INVALID_ARG);
        continue;
      }
      units.angles(a.table, pos, a.rotary, sub, false, c, s);
    }
    if (PAGES && slot >= a.n_slots) {
      set_status(a.status, DOPR_ERR_INVALID_ARG);
      continue;
    }
    float g[NU][2 * VEC];
    int held = -1;  // whose gain g is
#pragma unroll 1
    for (int h0 = h_first; h0 < heads; h0 += step) {
      const int h = h0 + lane / lanes;
      const bool is_q = h < a.q.n_heads, is_v = h >= a.q.n_heads + a.k.n_heads, valid = h < heads;
      const int hh = is_q ? h : is_v ? h - a.q.n_heads - a.k.n_heads : h - a.q.n_heads;
      float x[NU][2 * VEC];
      units.widen(p0, p1, valid, x);
      if (h0 + step < heads) load(h + step);
      if (a.eps > 0.f) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
          for (int j = 0; j < 2 * VEC; ++j) sum = __fmaf_rn(x[i][j], x[i][j], sum);
        sum = head_sum(sum, lanes);
        if (!is_v) {
          if (held != (is_q ? 0 : 1)) units.gains(gain[held = is_q ? 0 : 1], g);
          const float r = rsqrtf(__fmaf_rn(sum, inv_d, a.eps));
#pragma unroll
          for (int i = 0; i < NU; ++i)
#pragma unroll
            for (int j = 0; j < 2 * VEC; ++j) x[i][j] = __fmul_rn(__fmul_rn(x[i][j], r), g[i][j]);
        }
      }
      if (a.rotary > 0 && !is_v) units.turn(x, c, s);
      if (!PAGES || is_q) {
        const RopeView& view = is_q ? a.q : a.k;
        if (valid) units.store(static_cast<T*>(view.out) + t * view.out_tok + hh * view.out_head, x);
      }
      if constexpr (PAGES) {
        static_assert(VEC == 8 && NU == 1, "runs of eight");
        // what the row's type holds goes into the page: the same as a row stored and appended
        float top[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 2 * VEC; ++j) {
          x[0][j] = to_f32(from_f32<T>(x[0][j]));
          track_range(top[j / VEC], x[0][j]);
        }
        float* of_head = most[threadIdx.x / lanes];
        __syncwarp();  // the head before has been read
        if (units.there[0]) of_head[units.ia[0] / 8] = top[0], of_head[units.ib[0] / 8] = top[1];
        __syncwarp();
        if (valid && !is_q && slot >= 0 && units.there[0]) {
          uint8_t* base = (is_v ? a.v_pool : a.k_pool) + ((slot >> page_bits) * a.k.n_heads + hh) * pages4::page_bytes(a.page, D);
          const int row = static_cast<int>(slot) & (a.page - 1);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int run = (k ? units.ib[0] : units.ia[0]) / 8;
            const float4 m = *reinterpret_cast<const float4*>(of_head + (run & ~3));
            float all = m.x, inverse;
            track_range(all, m.y), track_range(all, m.z), track_range(all, m.w);
            const uint32_t byte = pages4::scale_byte(all, inverse);
            uint32_t word = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) word |= pages4::code_of(x[0][8 * k + j], inverse) << (4 * (j / 2) + 16 * (j & 1));
            if (byte == pages4::SCALE_NAN) word = 0x88888888u;
            *reinterpret_cast<uint32_t*>(base + row * (D / 2) + 4 * run) = word;
            if ((run & 3) == 0) {
              base[a.page * (D / 2) + row * (D / 32) + run / 4] = static_cast<uint8_t>(byte);
              if (byte == pages4::SCALE_NAN) set_status(a.status, DOPR_ERR_RANGE);
            }
          }
        }
      }
    }
  }
}

// Gradients of the inputs, and each block's part of the gains'.
template <typename T, int VEC, int NU, bool INTER>
__global__ void __launch_bounds__(THREADS) k_head_norm_back(const __grid_constant__ HeadNormArgs a, int lanes) {
  __shared__ float gain[2][MAX_DIM];
  __shared__ float part[THREADS / 32][2][MAX_DIM];
  const int D = a.head_dim, lane = threadIdx.x & 31, sub = lane & (lanes - 1), per_warp = 32 / lanes, warp = threadIdx.x >> 5;
  const int at_once = THREADS / lanes, h_first = warp * per_warp, heads = a.q.n_heads + a.k.n_heads;
  const Units<VEC, NU, INTER> units(sub, D, a.rotary);
  pdl_wait();
  pdl_trigger();
  for (int i = threadIdx.x; i < D; i += THREADS) {
    gain[0][i] = gain_at(a.q_gain, a.gain_dtype, i);
    gain[1][i] = gain_at(a.k_gain, a.gain_dtype, i);
  }
  __syncthreads();
  const float inv_d = 1.f / D;
  float dg[2][NU][2 * VEC] = {};
  for (int t = blockIdx.x; static_cast<uint32_t>(t) < static_cast<uint32_t>(a.n_tokens); t = static_cast<int>(t + gridDim.x)) {
    const int pos = a.rotary > 0 ? a.positions[t] : 0;
    if (pos < 0) continue;
    float c[NU][VEC], s[NU][VEC];
    if (a.rotary > 0) {
      if (pos >= a.max_position) {
        set_status(a.status, DOPR_ERR_INVALID_ARG);
        continue;
      }
      units.angles(a.table, pos, a.rotary, sub, true, c, s);
    }
#pragma unroll 1
    for (int h0 = h_first; h0 < heads; h0 += at_once) {
      const int h = h0 + lane / lanes;
      const bool is_q = h < a.q.n_heads, valid = h < heads;
      const int hh = is_q ? h : h - a.q.n_heads;
      const RopeView &view = is_q ? a.q : a.k, &from = is_q ? a.qx : a.kx;
      Pack<T, VEC> p0[NU], p1[NU], p2[NU], p3[NU];
      units.load(static_cast<const T*>(from.in) + t * from.in_tok + hh * from.in_head, valid, p0, p1);
      units.load(static_cast<const T*>(view.in) + t * view.in_tok + hh * view.in_head, valid, p2, p3);
      float x[NU][2 * VEC], dy[NU][2 * VEC];
      units.widen(p0, p1, valid, x);
      units.widen(p2, p3, valid, dy);
      if (a.rotary > 0) units.turn(dy, c, s);
      const float* g = gain[is_q ? 0 : 1];
      float sum = 0.f, dot = 0.f;
#pragma unroll
      for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < 2 * VEC; ++j) {
          const float w = units.there[i] ? dy[i][j] * g[(j < VEC ? units.ia[i] : units.ib[i] - VEC) + j] : 0.f;
          sum = __fmaf_rn(x[i][j], x[i][j], sum);
          dot = __fmaf_rn(x[i][j], w, dot);
        }
      sum = head_sum(sum, lanes);
      dot = head_sum(dot, lanes);
      const float r = rsqrtf(__fmaf_rn(sum, inv_d, a.eps)), by = dot * inv_d * r * r;
#pragma unroll
      for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < 2 * VEC; ++j) {
          const float n = dy[i][j] * x[i][j] * r;
          dg[0][i][j] += is_q ? n : 0.f;
          dg[1][i][j] += is_q ? 0.f : n;
          const float w = units.there[i] ? dy[i][j] * g[(j < VEC ? units.ia[i] : units.ib[i] - VEC) + j] : 0.f;
          x[i][j] = r * (w - x[i][j] * by);
        }
      if (valid) units.store(static_cast<T*>(view.out) + t * view.out_tok + hh * view.out_head, x);
    }
  }
  if (!a.dq_gain && !a.dk_gain) return;
  // the lanes of a warp that hold the same elements, then the warps, in a fixed order
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int j = 0; j < 2 * VEC; ++j) {
        float v = dg[k][i][j];
        for (int o = lanes; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane < lanes && units.there[i]) part[warp][k][(j < VEC ? units.ia[i] : units.ib[i] - VEC) + j] = v;
      }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += THREADS) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) v += part[w][i / D][i % D];
    a.ws[static_cast<int64_t>(blockIdx.x) * 2 * D + i] = v;
  }
}

// The blocks' parts of the gains' gradients, in a fixed order: 32 columns a block, a warp every eighth part.
__global__ void __launch_bounds__(256) k_head_norm_gains(const float* ws, int parts, int D, float* dq_gain, float* dk_gain) {
  __shared__ float sums[8][32];
  const int i = blockIdx.x * 32 + (threadIdx.x & 31), warp = threadIdx.x >> 5;
  pdl_wait();
  pdl_trigger();
  float v = 0.f;
  if (i < 2 * D)
    for (int p = warp; p < parts; p += 8) v += ws[static_cast<int64_t>(p) * 2 * D + i];
  sums[warp][threadIdx.x & 31] = v;
  __syncthreads();
  if (warp > 0 || i >= 2 * D) return;
#pragma unroll
  for (int w = 1; w < 8; ++w) v += sums[w][threadIdx.x];
  float* out = i < D ? dq_gain : dk_gain;
  if (out) out[i % D] = v;
}

bool aligned16(const void* p, int64_t s0, int64_t s1, int size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s0 * size % 16 == 0 && s1 * size % 16 == 0;
}
// Whether 16-byte accesses fit all views and the units.
bool wide(const HeadNormArgs& a, int size) {
  const int vec = 16 / size;
  bool ok = a.rotary / 2 % vec == 0 && a.head_dim % (2 * vec) == 0 && (a.head_dim - a.rotary) % (2 * vec) == 0;
  for (const RopeView* v : {&a.q, &a.k, &a.v, &a.qx, &a.kx}) {
    if (v->n_heads == 0) continue;
    ok = ok && aligned16(v->in, v->in_tok, v->in_head, size);
    if (v->out) ok = ok && aligned16(v->out, v->out_tok, v->out_head, size);
  }
  return ok;
}
int lanes_of(int head_dim, int vec) {
  int lanes = 1;
  while (lanes < 32 && lanes * 2 * vec < head_dim) lanes *= 2;
  return lanes;
}

template <typename T, int VEC, int NU, bool INTER, bool PAGES>
cudaError_t launch(const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  const int lanes = lanes_of(a.head_dim, VEC), at_once = THREADS / lanes;
  const int heads = a.q.n_heads + a.k.n_heads + a.v.n_heads;
  // few tokens leave most SMs idle: a token's heads over several blocks
  const int turns = (heads + at_once - 1) / at_once, spare = a.n_tokens < 4 * num_sms ? 4 * num_sms / a.n_tokens : 1;
  const dim3 grid(a.n_tokens < 65536 ? a.n_tokens : 65536, turns < spare ? turns : spare);
  return launch_dependent(k_head_norm<T, VEC, NU, INTER, PAGES>, grid, THREADS, 0, st, a, lanes);
}
template <typename T>
cudaError_t launch_type(const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  if (wide(a, sizeof(T)))
    return a.interleaved ? launch<T, VEC, 1, true, false>(a, num_sms, st) : launch<T, VEC, 1, false, false>(a, num_sms, st);
  return a.interleaved ? launch<T, 1, 4, true, false>(a, num_sms, st) : launch<T, 1, 4, false, false>(a, num_sms, st);
}
template <typename T, int VEC, int NU, bool INTER>
cudaError_t launch_back(const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  int blocks = 4 * num_sms < HEAD_NORM_MAX_BLOCKS ? 4 * num_sms : HEAD_NORM_MAX_BLOCKS;
  if (a.n_tokens < blocks) blocks = a.n_tokens;
  if (blocks > 0) {
    const cudaError_t e = launch_dependent(k_head_norm_back<T, VEC, NU, INTER>, dim3(blocks), THREADS, 0, st, a, lanes_of(a.head_dim, VEC));
    if (e != cudaSuccess) return e;
  }
  if (!a.dq_gain && !a.dk_gain) return cudaSuccess;
  return launch_dependent(k_head_norm_gains, dim3((2 * a.head_dim + 31) / 32), 256, 0, st, a.ws, blocks, a.head_dim, a.dq_gain, a.dk_gain);
}
template <typename T>
cudaError_t launch_back_type(const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  if (wide(a, sizeof(T)))
    return a.interleaved ? launch_back<T, VEC, 1, true>(a, num_sms, st) : launch_back<T, VEC, 1, false>(a, num_sms, st);
  return a.interleaved ? launch_back<T, 1, 4, true>(a, num_sms, st) : launch_back<T, 1, 4, false>(a, num_sms, st);
}

// ------------------------------------------------------------------ rows out of 4-bit pages
// A thread a run of eight elements: a word and its group's scale in, 16 bytes out.  c s is exact.
template <typename T>
__global__ void __launch_bounds__(THREADS) k_read_4bit(const __grid_constant__ Read4Args a) {
  const int D = a.head_dim, runs = D / 8, at_once = THREADS / runs, run = threadIdx.x % runs;
  const int page_bits = __ffs(a.page) - 1;
  pdl_wait();
  pdl_trigger();
  for (int t = blockIdx.x; static_cast<uint32_t>(t) < static_cast<uint32_t>(a.n_rows); t = static_cast<int>(t + gridDim.x)) {
    const int64_t slot = a.slots[t];
    if (slot < 0) continue;
    if (slot >= a.n_slots) {
      set_status(a.status, DOPR_ERR_INVALID_ARG);
      continue;
    }
    const int row = static_cast<int>(slot) & (a.page - 1);
    for (int h = threadIdx.x / runs; h < 2 * a.n_kv_heads; h += at_once) {
      const bool is_v = h >= a.n_kv_heads;
      const int hh = is_v ? h - a.n_kv_heads : h;
      const uint8_t* base = (is_v ? a.v_pool : a.k_pool) + ((slot >> page_bits) * a.n_kv_heads + hh) * pages4::page_bytes(a.page, D);
      const uint32_t word = *reinterpret_cast<const uint32_t*>(base + row * (D / 2) + 4 * run);
      const uint32_t byte = base[a.page * (D / 2) + row * (D / 32) + run / 4];
      const float s = byte > pages4::SCALE_LAST ? __uint_as_float(0x7fc00000u) : __half2float(__ushort_as_half(static_cast<unsigned short>(byte << 7)));
      Pack<T, 8> out;
#pragma unroll
      for (int j = 0; j < 8; ++j) out.v[j] = from_f32<T>((static_cast<int>(word >> (4 * (j / 2) + 16 * (j & 1)) & 15u) - 8) * s);
      const RopeView& view = is_v ? a.v : a.k;
      *reinterpret_cast<Pack<T, 8>*>(static_cast<T*>(view.out) + t * view.out_tok + hh * view.out_head + 8 * run) = out;
    }
  }
}

}  // namespace

cudaError_t launch_head_norm(int dtype, const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  if (a.n_tokens == 0) return cudaSuccess;
  switch (dtype) {
    case DOPR_F16: return launch_type<__half>(a, num_sms, st);
    case DOPR_BF16: return launch_type<__nv_bfloat16>(a, num_sms, st);
    default: return launch_type<float>(a, num_sms, st);
  }
}

cudaError_t launch_head_norm_backward(int dtype, const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  switch (dtype) {
    case DOPR_F16: return launch_back_type<__half>(a, num_sms, st);
    case DOPR_BF16: return launch_back_type<__nv_bfloat16>(a, num_sms, st);
    default: return launch_back_type<float>(a, num_sms, st);
  }
}

cudaError_t launch_append_4bit(int dtype, const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  if (a.n_tokens == 0) return cudaSuccess;
  if (dtype == DOPR_F16)
    return a.interleaved ? launch<__half, 8, 1, true, true>(a, num_sms, st) : launch<__half, 8, 1, false, true>(a, num_sms, st);
  return a.interleaved ? launch<__nv_bfloat16, 8, 1, true, true>(a, num_sms, st) : launch<__nv_bfloat16, 8, 1, false, true>(a, num_sms, st);
}

cudaError_t launch_read_4bit(int dtype, const Read4Args& a, int num_sms, cudaStream_t st) {
  if (a.n_rows == 0) return cudaSuccess;
  const dim3 grid(a.n_rows < 65536 ? a.n_rows : 65536);
  return dtype == DOPR_F16 ? launch_dependent(k_read_4bit<__half>, grid, THREADS, 0, st, a)
                           : launch_dependent(k_read_4bit<__nv_bfloat16>, grid, THREADS, 0, st, a);
}

}  // namespace dopr
