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

// A run of VEC elements from and to memory.
template <typename T, int VEC>
__device__ __forceinline__ void widen_run(const Pack<T, VEC>& p, float* x) {
  if constexpr (VEC > 1 && sizeof(T) == 2) {
    const uint4 w = reinterpret_cast<const uint4&>(p);
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float2 f;
      if constexpr (std::is_same_v<T, __half>) f = __half22float2(reinterpret_cast<const __half2&>(v[i]));
      else f = __bfloat1622float2(reinterpret_cast<const __nv_bfloat162&>(v[i]));
      x[2 * i] = f.x, x[2 * i + 1] = f.y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = to_f32(p.v[j]);
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_run(T* to, const float* x) {
  if constexpr (VEC > 1 && sizeof(T) == 2) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = std::is_same_v<T, __half> ? pack_f16x2(x[2 * i], x[2 * i + 1]) : pack_bf16x2(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<uint4*>(to) = uint4{v[0], v[1], v[2], v[3]};
  } else {
    Pack<T, VEC> p;
#pragma unroll
    for (int j = 0; j < VEC; ++j) p.v[j] = from_f32<T>(x[j]);
    *reinterpret_cast<Pack<T, VEC>*>(to) = p;
  }
}
// Two at once: a * b + c, a * b.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

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
  // (zeros where there is nothing)
  template <typename T>
  __device__ __forceinline__ void load(const T* row, bool valid, Pack<T, VEC> (&a)[NU], Pack<T, VEC> (&b)[NU]) const {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      a[i] = Pack<T, VEC>{}, b[i] = Pack<T, VEC>{};
      if (!there[i] || !valid) continue;
      a[i] = *reinterpret_cast<const Pack<T, VEC>*>(row + ia[i]);
      b[i] = *reinterpret_cast<const Pack<T, VEC>*>(row + ib[i]);
    }
  }
  template <typename T>
  __device__ __forceinline__ void widen(const Pack<T, VEC> (&a)[NU], const Pack<T, VEC> (&b)[NU], float (&x)[NU][2 * VEC]) const {
#pragma unroll
    for (int i = 0; i < NU; ++i) widen_run(a[i], x[i]), widen_run(b[i], x[i] + VEC);
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, const float (&x)[NU][2 * VEC]) const {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      if (!there[i]) continue;
      store_run<T, VEC>(row + ia[i], x[i]);
      store_run<T, VEC>(row + ib[i], x[i] + VEC);
    }
  }
  // The sum of x y over this lane's units.
  static __device__ __forceinline__ float dot(const float (&x)[NU][2 * VEC], const float (&y)[NU][2 * VEC]) {
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int j = 0; j < 2 * VEC; j += 2) sum = fma2(make_float2(x[i][j], x[i][j + 1]), make_float2(y[i][j], y[i][j + 1]), sum);
    return sum.x + sum.y;
  }
};

// Adds up over the `lanes` (a power of two) lanes that hold a head.
__device__ __forceinline__ float head_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// How the work is cut: a block takes one of the views (a role: q, k or, on the way into pages, v), so that a thread's gain stays with
// it and sums of gradients have one place; a warp takes units, a slice of one token's heads each, and walks over the slice with
// the token's cos and sin.
struct Roles {
  int end[3];     // blocks before the end of each
  int slices[3];  // of a token's heads
};
struct Role {
  int what, block, blocks, slices, per_slice;
  __device__ __forceinline__ Role(const Roles& r, const HeadNormArgs& a, int per_warp) {
    const int b = blockIdx.x;
    what = b < r.end[0] ? 0 : b < r.end[1] ? 1 : 2;
    const int from = what > 0 ? r.end[what - 1] : 0;
    block = b - from;
    blocks = r.end[what] - from;
    slices = r.slices[what];
    const int heads = view(a).n_heads, turns = (heads + per_warp - 1) / per_warp;
    per_slice = (turns + slices - 1) / slices * per_warp;
  }
  __device__ __forceinline__ const RopeView& view(const HeadNormArgs& a) const { return what == 0 ? a.q : what == 1 ? a.k : a.v; }
};

// PAGES: keys and values go to 4-bit pages.
template <typename T, int VEC, int NU, bool INTER, bool PAGES>
__global__ void __launch_bounds__(THREADS, PAGES ? 5 : 6) k_head_norm(const __grid_constant__ HeadNormArgs a, const __grid_constant__ Roles roles, int lanes) {
  __shared__ __align__(16) float most[PAGES ? THREADS / 4 : 1][16];  // of each head at work, the largest magnitudes of its runs of eight
  const int D = a.head_dim, lane = threadIdx.x & 31, sub = lane & (lanes - 1), per_warp = 32 / lanes;
  const Units<VEC, NU, INTER> units(sub, D, a.rotary);
  const Role role(roles, a, per_warp);
  const bool is_v = role.what == 2, normed = a.eps > 0.f && !is_v, turned = a.rotary > 0 && !is_v;
  const RopeView view = role.view(a);
  const int page_bits = PAGES ? __ffs(a.page) - 1 : 0;
  const float inv_d = 1.f / D;
  pdl_wait();
  pdl_trigger();
  const int64_t n = static_cast<int64_t>(a.n_tokens) * role.slices, step = static_cast<int64_t>(role.blocks) * (THREADS / 32);
#pragma unroll 1
  for (int64_t unit = static_cast<int64_t>(role.block) * (THREADS / 32) + (threadIdx.x >> 5); unit < n; unit += step) {
    const int t = static_cast<int>(role.slices > 1 ? unit / role.slices : unit);
    const int first = (role.slices > 1 ? static_cast<int>(unit - static_cast<int64_t>(t) * role.slices) : 0) * role.per_slice;
    const int end = min(view.n_heads, first + role.per_slice);
    const int pos = a.rotary > 0 ? a.positions[t] : 0;
    const int64_t slot = PAGES ? a.slots[t] : 0;
    // the first heads' elements are asked for beside the position and the table
    const T* x0 = static_cast<const T*>(view.in) + t * view.in_tok;
    Pack<T, VEC> p0[NU], p1[NU];
    int h = first + lane / lanes;
    units.load(x0 + h * view.in_head, h < end, p0, p1);
    if (pos < 0) continue;
    if (a.rotary > 0 && pos >= a.max_position) {
      set_status(a.status, DOPR_ERR_INVALID_ARG);
      continue;
    }
    if constexpr (PAGES) {
      if (slot >= a.n_slots) {
        set_status(a.status, DOPR_ERR_INVALID_ARG);
        continue;
      }
      if (role.what > 0 && slot < 0) continue;
    }
    // z_a = r (x_a ga c - x_b gb s), z_b = r (x_b gb c + x_a ga s): the gains go with cos and sin, once a token
    float ac[NU][VEC], bs[NU][VEC], bc[NU][VEC], as[NU][VEC];
    {
      float g[NU][2 * VEC], c[NU][VEC], s[NU][VEC];
      const void* gain = role.what == 0 ? a.q_gain : a.k_gain;
#pragma unroll
      for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          g[i][j] = normed && units.there[i] ? gain_at(gain, a.gain_dtype, units.ia[i] + j) : 1.f;
          g[i][VEC + j] = normed && units.there[i] ? gain_at(gain, a.gain_dtype, units.ib[i] + j) : 1.f;
          c[i][j] = 1.f, s[i][j] = 0.f;
        }
      if (turned) units.angles(a.table, pos, a.rotary, sub, false, c, s);
#pragma unroll
      for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          constexpr bool APART = !INTER || VEC == 1;
          const bool pair = turned && units.turns[i];
          const float ga = APART || !pair ? g[i][j] : g[i][2 * j], gb = APART || !pair ? g[i][VEC + j] : g[i][2 * j + 1];
          ac[i][j] = __fmul_rn(ga, c[i][j]), as[i][j] = __fmul_rn(ga, s[i][j]);
          bc[i][j] = __fmul_rn(gb, c[i][j]), bs[i][j] = __fmul_rn(gb, s[i][j]);
        }
    }
#pragma unroll 1
    for (int h0 = first; h0 < end; h0 += per_warp) {
      const bool valid = h < end;
      const int hh = h;
      float x[NU][2 * VEC];
      units.widen(p0, p1, x);
      h += per_warp;
      units.load(x0 + h * view.in_head, h < end, p0, p1);
      float r = 1.f;
      if (normed) {
        r = rsqrtf(__fmaf_rn(head_sum(units.dot(x, x), lanes), inv_d, a.eps));
      }
      if (normed || turned) {
        constexpr bool APART = !INTER || VEC == 1;
        const float2 rr = make_float2(r, r);
#pragma unroll
        for (int i = 0; i < NU; ++i) {
          if (!(turned && units.turns[i])) {  // (c 1: ac and bc are the gains)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
              x[i][j] = __fmul_rn(__fmul_rn(x[i][j], ac[i][j]), r);
              x[i][VEC + j] = __fmul_rn(__fmul_rn(x[i][VEC + j], bc[i][j]), r);
            }
          } else if constexpr (APART && VEC > 1) {
#pragma unroll
            for (int j = 0; j < VEC; j += 2) {
              const float2 u = make_float2(x[i][j], x[i][j + 1]), v = make_float2(x[i][VEC + j], x[i][VEC + j + 1]);
              const float2 y = mul2(v, make_float2(-bs[i][j], -bs[i][j + 1])), z = mul2(u, make_float2(as[i][j], as[i][j + 1]));
              const float2 za = mul2(fma2(u, make_float2(ac[i][j], ac[i][j + 1]), y), rr);
              const float2 zb = mul2(fma2(v, make_float2(bc[i][j], bc[i][j + 1]), z), rr);
              x[i][j] = za.x, x[i][j + 1] = za.y, x[i][VEC + j] = zb.x, x[i][VEC + j + 1] = zb.y;
            }
          } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
              float &xa = APART ? x[i][j] : x[i][2 * j], &xb = APART ? x[i][VEC + j] : x[i][2 * j + 1];
              const float u = xa, v = xb;
              xa = __fmul_rn(__fmaf_rn(u, ac[i][j], -__fmul_rn(v, bs[i][j])), r);
              xb = __fmul_rn(__fmaf_rn(v, bc[i][j], __fmul_rn(u, as[i][j])), r);
            }
          }
        }
      }
      if (!PAGES || role.what == 0) {
        if (valid) units.store(static_cast<T*>(view.out) + t * view.out_tok + hh * view.out_head, x);
      } else {
        if constexpr (PAGES) {
          static_assert(VEC == 8 && NU == 1, "runs of eight");
          // what the row's type holds goes into the page: the same as a row stored and appended
          float top[2] = {0.f, 0.f};
          if (normed || turned) {
#pragma unroll
            for (int j = 0; j < 2 * VEC; ++j) x[0][j] = to_f32(from_f32<T>(x[0][j]));
          }
#pragma unroll
          for (int j = 0; j < 2 * VEC; ++j) track_range(top[j / VEC], x[0][j]);
          float* of_head = most[threadIdx.x / lanes];
          __syncwarp();  // the head before has been read
          if (units.there[0]) of_head[units.ia[0] / 8] = top[0], of_head[units.ib[0] / 8] = top[1];
          __syncwarp();
          if (valid && units.there[0]) {
            uint8_t* base = (is_v ? a.v_pool : a.k_pool) + ((slot >> page_bits) * a.k.n_heads + hh) * pages4::page_bytes(a.page, D);
            const int row = static_cast<int>(slot) & (a.page - 1);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int run = (k ? units.ib[0] : units.ia[0]) / 8;
              const float4 m = *reinterpret_cast<const float4*>(of_head + (run & ~3));
              float all = m.x, inverse;
              track_range(all, m.y), track_range(all, m.z), track_range(all, m.w);
              const uint32_t byte = pages4::scale_byte(all, inverse);
              uint32_t word = pages4::codes_of(x[0] + 8 * k, inverse);
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
}

// Gradients of the inputs, and each block's part of its gain's.
template <typename T, int VEC, int NU, bool INTER>
__global__ void __launch_bounds__(THREADS, 4) k_head_norm_back(const __grid_constant__ HeadNormArgs a, const __grid_constant__ Roles roles, int lanes) {
  __shared__ float part[THREADS / 32][MAX_DIM];
  const int D = a.head_dim, lane = threadIdx.x & 31, sub = lane & (lanes - 1), per_warp = 32 / lanes, warp = threadIdx.x >> 5;
  const Units<VEC, NU, INTER> units(sub, D, a.rotary);
  const Role role(roles, a, per_warp);
  const RopeView view = role.view(a), from = role.what == 0 ? a.qx : a.kx;
  pdl_wait();
  pdl_trigger();
  const float inv_d = 1.f / D;
  float dg[NU][2 * VEC] = {}, g[NU][2 * VEC];
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int j = 0; j < 2 * VEC; ++j)
      g[i][j] = units.there[i] ? gain_at(role.what == 0 ? a.q_gain : a.k_gain, a.gain_dtype, (j < VEC ? units.ia[i] : units.ib[i] - VEC) + j) : 0.f;
  const int64_t n = static_cast<int64_t>(a.n_tokens) * role.slices, step = static_cast<int64_t>(role.blocks) * (THREADS / 32);
#pragma unroll 1
  for (int64_t unit = static_cast<int64_t>(role.block) * (THREADS / 32) + warp; unit < n; unit += step) {
    const int t = static_cast<int>(role.slices > 1 ? unit / role.slices : unit);
    const int first = (role.slices > 1 ? static_cast<int>(unit - static_cast<int64_t>(t) * role.slices) : 0) * role.per_slice;
    const int end = min(view.n_heads, first + role.per_slice);
    const int pos = a.rotary > 0 ? a.positions[t] : 0;
    const T *x0 = static_cast<const T*>(from.in) + t * from.in_tok, *z0 = static_cast<const T*>(view.in) + t * view.in_tok;
    Pack<T, VEC> p0[NU], p1[NU], p2[NU], p3[NU];
    int h = first + lane / lanes;
    units.load(x0 + h * from.in_head, h < end, p0, p1);
    units.load(z0 + h * view.in_head, h < end, p2, p3);
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
    for (int h0 = first; h0 < end; h0 += per_warp) {
      const bool valid = h < end;
      const int hh = h;
      float x[NU][2 * VEC], w[NU][2 * VEC];
      units.widen(p0, p1, x);
      units.widen(p2, p3, w);
      h += per_warp;
      units.load(x0 + h * from.in_head, h < end, p0, p1);
      units.load(z0 + h * view.in_head, h < end, p2, p3);
      if (a.rotary > 0) units.turn(w, c, s);
      // sum x^2 is there first; sum w x = sum dy x g too, so that dg's terms dy x serve both
      const float r = rsqrtf(__fmaf_rn(head_sum(units.dot(x, x), lanes), inv_d, a.eps));
      float2 dot = make_float2(0.f, 0.f);
      const float2 rr = make_float2(r, r);
#pragma unroll
      for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < 2 * VEC; j += 2) {
          const float2 gg = make_float2(g[i][j], g[i][j + 1]), dy = make_float2(w[i][j], w[i][j + 1]);
          const float2 yx = mul2(dy, make_float2(x[i][j], x[i][j + 1]));
          const float2 sum = fma2(yx, rr, make_float2(dg[i][j], dg[i][j + 1]));
          dg[i][j] = sum.x, dg[i][j + 1] = sum.y;
          dot = fma2(yx, gg, dot);
        }
      // dx = (dy g - x by) r
      const float by = head_sum(dot.x + dot.y, lanes) * inv_d * r * r;
#pragma unroll
      for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < 2 * VEC; j += 2) {
          const float2 xb = mul2(make_float2(x[i][j], x[i][j + 1]), make_float2(-by, -by));
          const float2 d = mul2(fma2(make_float2(w[i][j], w[i][j + 1]), make_float2(g[i][j], g[i][j + 1]), xb), rr);
          x[i][j] = d.x, x[i][j + 1] = d.y;
        }
      if (valid) units.store(static_cast<T*>(view.out) + t * view.out_tok + hh * view.out_head, x);
    }
  }
  if (!(role.what == 0 ? a.dq_gain : a.dk_gain)) return;
  // the lanes of a warp that hold the same elements, then the warps, in a fixed order
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int j = 0; j < 2 * VEC; ++j) {
      float v = dg[i][j];
      for (int o = lanes; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane < lanes && units.there[i]) part[warp][(j < VEC ? units.ia[i] : units.ib[i] - VEC) + j] = v;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < D; i += THREADS) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) v += part[w][i];
    a.ws[static_cast<int64_t>(blockIdx.x) * D + i] = v;
  }
}

// The blocks' parts of the gains' gradients, in a fixed order: 32 columns of one gain a block, a warp every 32nd part.
__global__ void __launch_bounds__(1024) k_head_norm_gains(const float* ws, int q_parts, int k_parts, int D, float* dq_gain, float* dk_gain) {
  __shared__ float sums[32][33];
  const int i = blockIdx.x * 32 + (threadIdx.x & 31), warp = threadIdx.x >> 5;
  const bool is_k = blockIdx.y > 0;
  float* out = is_k ? dk_gain : dq_gain;
  pdl_wait();
  pdl_trigger();
  if (!out) return;
  float v = 0.f;
  if (i < D)
    for (int p = warp; p < (is_k ? k_parts : q_parts); p += 32) v += ws[static_cast<int64_t>(p + (is_k ? q_parts : 0)) * D + i];
  sums[warp][threadIdx.x & 31] = v;
  __syncthreads();
  // warp w adds up column w
  v = sums[threadIdx.x & 31][warp];
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0 && blockIdx.x * 32 + warp < D) out[blockIdx.x * 32 + warp] = v;
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

// Blocks for each role, by the heads: few tokens leave most SMs idle, so their heads go to several warps.
Roles roles_of(const HeadNormArgs& a, int lanes, int most_blocks) {
  const int heads[3] = {a.q.n_heads, a.k.n_heads, a.v.n_heads}, per_warp = 32 / lanes, warps = THREADS / 32;
  const int all = heads[0] + heads[1] + heads[2];
  Roles r{};
  int at = 0;
  for (int i = 0; i < 3; ++i) {
    const int turns = (heads[i] + per_warp - 1) / per_warp;
    const int64_t room = static_cast<int64_t>(most_blocks) * warps * heads[i] / (all > 0 ? all : 1);  // warps
    int64_t slices = a.n_tokens > 0 ? room / a.n_tokens : 1;
    slices = slices < 1 ? 1 : slices > turns ? (turns > 0 ? turns : 1) : slices;
    // as many as are not empty
    const int per = turns > 0 ? static_cast<int>((turns + slices - 1) / slices) : 1;
    slices = turns > 0 ? (turns + per - 1) / per : 1;
    const int64_t units = static_cast<int64_t>(a.n_tokens) * slices, need = (units + warps - 1) / warps, part = (room + warps - 1) / warps;
    r.slices[i] = static_cast<int>(slices);
    at += heads[i] > 0 ? static_cast<int>(need < part ? need : part > 0 ? part : 1) : 0;
    r.end[i] = at;
  }
  return r;
}

template <typename T, int VEC, int NU, bool INTER, bool PAGES>
cudaError_t launch(const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  const int lanes = lanes_of(a.head_dim, VEC);
  const Roles r = roles_of(a, lanes, 12 * num_sms);
  return launch_dependent(k_head_norm<T, VEC, NU, INTER, PAGES>, dim3(r.end[2]), THREADS, 0, st, a, r, lanes);
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
  const int lanes = lanes_of(a.head_dim, VEC);
  const int blocks = 4 * num_sms < HEAD_NORM_MAX_BLOCKS - 2 ? 4 * num_sms : HEAD_NORM_MAX_BLOCKS - 2;  // (a part may be rounded up)
  Roles r{};
  if (a.n_tokens > 0) {
    r = roles_of(a, lanes, blocks);
    const cudaError_t e = launch_dependent(k_head_norm_back<T, VEC, NU, INTER>, dim3(r.end[1]), THREADS, 0, st, a, r, lanes);
    if (e != cudaSuccess) return e;
  }
  if (!a.dq_gain && !a.dk_gain) return cudaSuccess;
  return launch_dependent(k_head_norm_gains, dim3((a.head_dim + 31) / 32, 2), 1024, 0, st, a.ws, r.end[0], r.end[1] - r.end[0], a.head_dim,
                          a.dq_gain, a.dk_gain);
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
  const int D = a.head_dim, runs = D / 8, at_once = THREADS / runs, run = threadIdx.x % runs, h0 = threadIdx.x / runs;
  const int page_bits = __ffs(a.page) - 1;
  const int64_t page_bytes = pages4::page_bytes(a.page, D);
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
    const int64_t base = (slot >> page_bits) * a.n_kv_heads * page_bytes;
    const uint8_t *k = a.k_pool + base, *v = a.v_pool + base;
    const int code = row * (D / 2) + 4 * run, scale = a.page * (D / 2) + row * (D / 32) + run / 4;
    T *ko = static_cast<T*>(a.k.out) + t * a.k.out_tok + 8 * run, *vo = static_cast<T*>(a.v.out) + t * a.v.out_tok + 8 * run;
    for (int h = h0; h < a.n_kv_heads; h += at_once) {
      const int64_t at = h * page_bytes;
      // a key's and a value's at once
      const uint32_t word[2] = {*reinterpret_cast<const uint32_t*>(k + at + code), *reinterpret_cast<const uint32_t*>(v + at + code)};
      const uint32_t byte[2] = {k[at + scale], v[at + scale]};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t x[4];
        const pages4::Widen<T> widen(byte[i] * 0x10001u);
        widen(word[i], x);
        if constexpr (std::is_same_v<T, __half>) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const __half2 y = __hmul2(reinterpret_cast<const __half2&>(x[j]), __float2half2_rn(pages4::Widen<T>::UNIT));
            x[j] = reinterpret_cast<const uint32_t&>(y);
          }
        }
        if (byte[i] > pages4::SCALE_LAST) x[0] = x[1] = x[2] = x[3] = 0x7fff7fffu;  // NaN
        *reinterpret_cast<uint4*>((i ? vo + h * a.v.out_head : ko + h * a.k.out_head)) = uint4{x[0], x[1], x[2], x[3]};
      }
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
