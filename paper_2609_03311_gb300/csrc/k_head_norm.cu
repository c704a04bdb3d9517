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
// Blocks an SM holds, by the registers that they get; and in the whole grid, for each SM, of many tokens: a view's blocks are not equally
// long, so several rounds of them even out.  26,800 rows of 40 heads: 5 held, 40 in all 89 us; 5 and 20 89, 5 and 12 95; 4 and 40
// 95; 6 and 12 102; 6 and 36 90; 7 and 42 98 (registers run out).  With the keys and values on the way into pages: 5 and 40 133, 4 and
// 40 132, 5 and 20 136, 6 and 36 144, 7 and 42 187 (five hold 96 registers a thread, of which these kernels spill up to eleven words
// where pairs are halves apart; four hold 128).  Gradients of 8,192 rows: 4 held 43, 3 45, 5 63; their partial sums want few blocks.
constexpr int HELD = 5, GRID = 40, BACK_HELD = 4;

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

// Lanes that hold a head: a power of two.
__host__ __device__ constexpr int lanes_of(int head_dim, int vec) {
  int lanes = 1;
  while (lanes < 32 && lanes * 2 * vec < head_dim) lanes *= 2;
  return lanes;
}
// Adds up over the `lanes` (a power of two) lanes that hold a head.
__device__ __forceinline__ float head_sum(float v, int lanes) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < lanes) v += __shfl_xor_sync(0xffffffffu, v, o);
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

// A warp's units, one ahead: the next one's position and slot, and its first heads' elements, are asked for before this one's work.
struct Unit {
  int t, first, end, pos;
  int64_t slot;
  bool there;
};
template <bool PAGES, bool POSITIONS = true>
struct Walk {
  const HeadNormArgs& a;
  const Role& role;
  const int n_heads;
  int64_t unit, n, step;
  __device__ __forceinline__ Walk(const HeadNormArgs& args, const Role& r, int heads)
      : a(args), role(r), n_heads(heads), unit(static_cast<int64_t>(r.block) * (THREADS / 32) + (threadIdx.x >> 5)),
        n(static_cast<int64_t>(args.n_tokens) * r.slices), step(static_cast<int64_t>(r.blocks) * (THREADS / 32)) {}
  __device__ __forceinline__ Unit next() {
    Unit u{};
    u.there = unit < n;
    if (!u.there) return u;
    u.t = static_cast<int>(unit);
    if (role.slices > 1) {
      u.t = static_cast<int>(static_cast<uint32_t>(unit) / static_cast<uint32_t>(role.slices));  // (slices of few tokens: below 2^31)
      u.first = (static_cast<int>(unit) - u.t * role.slices) * role.per_slice;
    }
    u.end = min(n_heads, u.first + role.per_slice);
    if (POSITIONS && a.rotary > 0) u.pos = a.positions[u.t];
    if (POSITIONS && PAGES) u.slot = a.slots[u.t];
    unit += step;
    return u;
  }
};

// The next unit's cos and sin into L1.
__device__ __forceinline__ void prefetch_angles(const HeadNormArgs& a, const Unit& u, int lane) {
  if (u.pos < 0 || u.pos >= a.max_position) return;
  const char* cs = reinterpret_cast<const char*>(a.table + static_cast<int64_t>(u.pos) * (a.rotary / 2));
  for (int i = lane * 128; i < a.rotary * 4; i += 32 * 128) asm volatile("prefetch.global.L1 [%0];" ::"l"(cs + i));
}

// The elements of a warp's heads, turn after turn over its units, of one or two views (backward: the inputs and the outputs'
// gradients).  What bounds these kernels is how much is on its way: 16-byte copies into shared memory run AHEAD turns before they
// are taken (one turn ahead, in registers, as these kernels were then: a chunk of 26,800 rows 112 us).  A lane takes what it has copied itself.
template <typename T, int VEC, int NU, bool INTER, int VIEWS, int AHEAD>
struct Stream {
  static constexpr bool RING = VEC > 1;
  static constexpr int STAGES = AHEAD + 1, BYTES = RING ? (THREADS / 32) * STAGES * VIEWS * 1024 : 16;
  using P = Pack<T, VEC>;
  const Units<VEC, NU, INTER>& units;
  const RopeView (&views)[VIEWS];
  Walk<false, false> walk;
  Unit u;
  int h, stage = 0, lanes;
  uint8_t* ring;
  P p[RING ? 1 : VIEWS][2][NU];
  __device__ __forceinline__ Stream(const Units<VEC, NU, INTER>& un, const HeadNormArgs& a, const Role& role, const RopeView (&v)[VIEWS],
                                    uint8_t* smem, int lanes_)
      : units(un), views(v), walk(a, role, v[0].n_heads), lanes(lanes_), ring(smem + (threadIdx.x >> 5) * STAGES * VIEWS * 1024) {
    u = walk.next();
    h = u.first;
    if constexpr (RING) {
#pragma unroll 1
      for (int i = 0; i < AHEAD; ++i) put(i);
    } else {
      put(0);
    }
  }
  __device__ __forceinline__ void put(int at) {
    if (RING && !u.there) {
      cp_async_commit();
      return;
    }
    const int lane = threadIdx.x & 31, mine = h + lane / lanes;
    const bool valid = u.there && mine < u.end;
#pragma unroll
    for (int i = 0; i < VIEWS; ++i) {
      const T* row = static_cast<const T*>(views[i].in) + u.t * views[i].in_tok + mine * views[i].in_head;
      if constexpr (RING) {
        const uint32_t to = smem_u32(ring) + (at * VIEWS + i) * 1024 + lane * 16;
        if (units.there[0]) {
          cp_async16(to, row + units.ia[0], valid);
          cp_async16(to + 512, row + units.ib[0], valid);
        }
      } else {
        units.load(row, valid, p[i][0], p[i][1]);
      }
    }
    if constexpr (RING) cp_async_commit();
    if (u.there) {
      h += 32 / lanes;
      if (h >= u.end) {
        u = walk.next();
        h = u.first;
      }
    }
  }
  // The next turn's elements, in 32 bits; the one AHEAD turns behind it is asked for.
  __device__ __forceinline__ void take(float (&x)[VIEWS][NU][2 * VEC]) {
    if constexpr (RING) {
      put(stage == 0 ? AHEAD : stage - 1);  // the stage taken last
      asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD) : "memory");
      const int lane = threadIdx.x & 31;
#pragma unroll
      for (int i = 0; i < VIEWS; ++i) {
        const P* from = reinterpret_cast<const P*>(ring + (stage * VIEWS + i) * 1024) + lane;
        if (units.there[0]) {
          widen_run(from[0], x[i][0]);
          widen_run(from[32], x[i][0] + VEC);
        } else {
#pragma unroll
          for (int j = 0; j < 2 * VEC; ++j) x[i][0][j] = 0.f;
        }
      }
      stage = stage == AHEAD ? 0 : stage + 1;
    } else {
#pragma unroll
      for (int i = 0; i < VIEWS; ++i) units.widen(p[i][0], p[i][1], x[i]);
      put(0);
    }
  }
  // Goes past a unit.
  __device__ __forceinline__ void skip(const Unit& past) {
    for (int i = past.first; i < past.end; i += 32 / lanes) {
      float x[VIEWS][NU][2 * VEC];
      take(x);
    }
  }
};

// PAGES: keys and values go to 4-bit pages.  DIM: the head size, or 0: head_dim.
template <typename T, int VEC, int NU, bool INTER, bool PAGES, int DIM>
__global__ void __launch_bounds__(THREADS, HELD) k_head_norm(const __grid_constant__ HeadNormArgs a, const __grid_constant__ Roles roles) {
  using S = Stream<T, VEC, NU, INTER, 1, 4>;
  __shared__ __align__(16) uint8_t ring[S::BYTES];
  __shared__ __align__(16) float gains[MAX_DIM];
  __shared__ __align__(16) float most[PAGES ? THREADS / 4 : 1][16];  // of each head at work, the largest magnitudes of its runs of eight
  const int D = DIM > 0 ? DIM : a.head_dim, lanes = lanes_of(D, VEC), lane = threadIdx.x & 31, sub = lane & (lanes - 1), per_warp = 32 / lanes;
  const Units<VEC, NU, INTER> units(sub, D, a.rotary);
  const Role role(roles, a, per_warp);
  const bool is_v = role.what == 2, normed = a.eps > 0.f && !is_v, turned = a.rotary > 0 && !is_v;
  const RopeView view = role.view(a);
  const int page_bits = PAGES ? __ffs(a.page) - 1 : 0;
  const float inv_d = 1.f / D;
  pdl_wait();
  pdl_trigger();
  if (normed) {
    for (int i = threadIdx.x; i < D; i += THREADS) gains[i] = gain_at(role.what == 0 ? a.q_gain : a.k_gain, a.gain_dtype, i);
    __syncthreads();
  }
  Walk<PAGES> walk(a, role, view.n_heads);
  const RopeView views[1] = {view};
  S stream(units, a, role, views, ring, lanes);
  Unit next = walk.next();
#pragma unroll 1
  while (next.there) {
    const Unit u = next;
    next = walk.next();
    int h = u.first + lane / lanes;
    bool skip = u.pos < 0 || (PAGES && role.what > 0 && u.slot < 0);
    if ((a.rotary > 0 && u.pos >= a.max_position) || (PAGES && u.pos >= 0 && u.slot >= a.n_slots)) {
      set_status(a.status, DOPR_ERR_INVALID_ARG);
      skip = true;
    }
    if (skip) {
      stream.skip(u);
      continue;
    }
    // z_a = r (x_a ga c - x_b gb s), z_b = r (x_b gb c + x_a ga s): the gains go with cos and sin, once a token
    float ac[NU][VEC], bs[NU][VEC], bc[NU][VEC], as[NU][VEC];
    {
      float c[NU][VEC], s[NU][VEC];
#pragma unroll
      for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) c[i][j] = 1.f, s[i][j] = 0.f;
      if (turned) units.angles(a.table, u.pos, a.rotary, sub, false, c, s);
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        float g[2 * VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          g[j] = normed && units.there[i] ? gains[units.ia[i] + j] : 1.f;
          g[VEC + j] = normed && units.there[i] ? gains[units.ib[i] + j] : 1.f;
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          constexpr bool APART = !INTER || VEC == 1;
          const bool pair = turned && units.turns[i];
          const float ga = APART || !pair ? g[j] : g[2 * j], gb = APART || !pair ? g[VEC + j] : g[2 * j + 1];
          ac[i][j] = __fmul_rn(ga, c[i][j]), as[i][j] = __fmul_rn(ga, s[i][j]);
          bc[i][j] = __fmul_rn(gb, c[i][j]), bs[i][j] = __fmul_rn(gb, -s[i][j]);
        }
      }
    }
#pragma unroll 1
    for (int h0 = u.first; h0 < u.end; h0 += per_warp) {
      const bool valid = h < u.end;
      const int hh = h;
      float taken[1][NU][2 * VEC];
      stream.take(taken);
      auto& x = taken[0];
      h += per_warp;
      if (h0 == u.first && turned && next.there) prefetch_angles(a, next, lane);
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
              const float2 u2 = make_float2(x[i][j], x[i][j + 1]), v = make_float2(x[i][VEC + j], x[i][VEC + j + 1]);
              const float2 y = mul2(v, make_float2(bs[i][j], bs[i][j + 1])), z = mul2(u2, make_float2(as[i][j], as[i][j + 1]));
              const float2 za = mul2(fma2(u2, make_float2(ac[i][j], ac[i][j + 1]), y), rr);
              const float2 zb = mul2(fma2(v, make_float2(bc[i][j], bc[i][j + 1]), z), rr);
              x[i][j] = za.x, x[i][j + 1] = za.y, x[i][VEC + j] = zb.x, x[i][VEC + j + 1] = zb.y;
            }
          } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
              float &xa = APART ? x[i][j] : x[i][2 * j], &xb = APART ? x[i][VEC + j] : x[i][2 * j + 1];
              const float ua = xa, ub = xb;
              xa = __fmul_rn(__fmaf_rn(ua, ac[i][j], __fmul_rn(ub, bs[i][j])), r);
              xb = __fmul_rn(__fmaf_rn(ub, bc[i][j], __fmul_rn(ua, as[i][j])), r);
            }
          }
        }
      }
      if (!PAGES || role.what == 0) {
        if (valid) units.store(static_cast<T*>(view.out) + u.t * view.out_tok + hh * view.out_head, x);
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
            uint8_t* base = (is_v ? a.v_pool : a.k_pool) + ((u.slot >> page_bits) * a.k.n_heads + hh) * pages4::page_bytes(a.page, D);
            const int row = static_cast<int>(u.slot) & (a.page - 1);
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

// Rows into 4-bit pages as they are: a lane 16 elements that follow one another, two lanes a group.
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) k_append_4bit(const __grid_constant__ HeadNormArgs a, const __grid_constant__ Roles roles) {
  constexpr int LANES = D / 16, PER_WARP = 32 / LANES;
  const int lane = threadIdx.x & 31, sub = lane % LANES, page_bits = __ffs(a.page) - 1;
  const Role role(roles, a, PER_WARP);
  const RopeView view = role.view(a);
  uint8_t* const pool = role.what == 1 ? a.k_pool : a.v_pool;
  const int64_t page_bytes = pages4::page_bytes(a.page, D);
  pdl_wait();
  pdl_trigger();
  Walk<true> walk(a, role, view.n_heads);
  uint4 p[2];
  auto load = [&](const Unit& u, int h) {
    const uint4* from = reinterpret_cast<const uint4*>(static_cast<const T*>(view.in) + u.t * view.in_tok + h * view.in_head) + 2 * sub;
    p[0] = p[1] = uint4{0, 0, 0, 0};
    if (u.there && h < u.end) p[0] = from[0], p[1] = from[1];
  };
  Unit next = walk.next();
  load(next, next.first + lane / LANES);
#pragma unroll 1
  while (next.there) {
    const Unit u = next;
    next = walk.next();
    int h = u.first + lane / LANES;
    if (u.slot < 0 || u.slot >= a.n_slots) {
      if (u.slot >= 0) set_status(a.status, DOPR_ERR_INVALID_ARG);
      load(next, next.first + lane / LANES);
      continue;
    }
    const int row = static_cast<int>(u.slot) & (a.page - 1);
    uint8_t* const base = pool + (u.slot >> page_bits) * a.k.n_heads * page_bytes;
#pragma unroll 1
    for (int h0 = u.first; h0 < u.end; h0 += PER_WARP) {
      const bool valid = h < u.end;
      uint8_t* to = base + h * page_bytes;
      float x[16];
      widen_run(reinterpret_cast<const Pack<T, 8>&>(p[0]), x);
      widen_run(reinterpret_cast<const Pack<T, 8>&>(p[1]), x + 8);
      h += PER_WARP;
      const bool last = h0 + PER_WARP >= u.end;
      load(last ? next : u, last ? next.first + lane / LANES : h);
      float top[4] = {0.f, 0.f, 0.f, 0.f}, inverse;
#pragma unroll
      for (int j = 0; j < 16; ++j) track_range(top[j & 3], x[j]);
      track_range(top[0], top[1]), track_range(top[2], top[3]), track_range(top[0], top[2]);
      track_range(top[0], __shfl_xor_sync(0xffffffffu, top[0], 1));
      const uint32_t byte = pages4::scale_byte(top[0], inverse);
      uint2 words = make_uint2(pages4::codes_of(x, inverse), pages4::codes_of(x + 8, inverse));
      if (byte == pages4::SCALE_NAN) words = make_uint2(0x88888888u, 0x88888888u);
      // the head's scales to its first lane
      uint32_t scales = byte << (8 * (sub >> 1));
#pragma unroll
      for (int o = 2; o < LANES; o <<= 1) scales |= __shfl_xor_sync(0xffffffffu, scales, o);
      if (valid) {
        *reinterpret_cast<uint2*>(to + row * (D / 2) + 8 * sub) = words;
        if (sub == 0) {
          uint8_t* s = to + a.page * (D / 2) + row * (D / 32);
          if constexpr (D == 128) *reinterpret_cast<uint32_t*>(s) = scales;
          else *reinterpret_cast<uint16_t*>(s) = static_cast<uint16_t>(scales);
        }
        if (byte == pages4::SCALE_NAN) set_status(a.status, DOPR_ERR_RANGE);
      }
    }
  }
}

// Gradients of the inputs, and each block's part of its gain's.
template <typename T, int VEC, int NU, bool INTER, int DIM>
__global__ void __launch_bounds__(THREADS, BACK_HELD) k_head_norm_back(const __grid_constant__ HeadNormArgs a, const __grid_constant__ Roles roles) {
  using S = Stream<T, VEC, NU, INTER, 2, 3>;
  __shared__ __align__(16) uint8_t ring[S::BYTES];
  __shared__ float part[THREADS / 32][MAX_DIM];
  const int D = DIM > 0 ? DIM : a.head_dim, lanes = lanes_of(D, VEC), lane = threadIdx.x & 31, sub = lane & (lanes - 1), per_warp = 32 / lanes,
            warp = threadIdx.x >> 5;
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
  Walk<false> walk(a, role, view.n_heads);
  const RopeView views[2] = {from, view};
  S stream(units, a, role, views, ring, lanes);
  Unit next = walk.next();
#pragma unroll 1
  while (next.there) {
    const Unit u = next;
    next = walk.next();
    int h = u.first + lane / lanes;
    if (u.pos < 0 || (a.rotary > 0 && u.pos >= a.max_position)) {
      if (u.pos >= 0) set_status(a.status, DOPR_ERR_INVALID_ARG);
      stream.skip(u);
      continue;
    }
    float c[NU][VEC], s[NU][VEC];
    if (a.rotary > 0) units.angles(a.table, u.pos, a.rotary, sub, true, c, s);
#pragma unroll 1
    for (int h0 = u.first; h0 < u.end; h0 += per_warp) {
      const bool valid = h < u.end;
      const int hh = h;
      float taken[2][NU][2 * VEC];
      stream.take(taken);
      auto &x = taken[0], &w = taken[1];
      h += per_warp;
      if (h0 == u.first && a.rotary > 0 && next.there) prefetch_angles(a, next, lane);
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
      if (valid) units.store(static_cast<T*>(view.out) + u.t * view.out_tok + hh * view.out_head, x);
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

// The blocks' parts of the gains' gradients, in a fixed order: 8 columns of one gain a block (a sector of a part's), eight threads
// every 128th part.  Latency: gradients of 8,192 rows 42.9 us, with 32 columns and every 32nd part 43.4.
constexpr int GAIN_COLS = 8;
__global__ void __launch_bounds__(1024) k_head_norm_gains(const float* ws, int q_parts, int k_parts, int D, float* dq_gain, float* dk_gain) {
  __shared__ float sums[32][GAIN_COLS + 1];
  const int col = threadIdx.x % GAIN_COLS, i = blockIdx.x * GAIN_COLS + col, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool is_k = blockIdx.y > 0;
  float* out = is_k ? dk_gain : dq_gain;
  pdl_wait();
  pdl_trigger();
  if (!out) return;
  float v = 0.f;
  if (i < D)
    for (int p = threadIdx.x / GAIN_COLS; p < (is_k ? k_parts : q_parts); p += 1024 / GAIN_COLS)
      v += ws[static_cast<int64_t>(p + (is_k ? q_parts : 0)) * D + i];
#pragma unroll
  for (int o = GAIN_COLS; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane < GAIN_COLS) sums[warp][lane] = v;
  __syncthreads();
  // warp w adds up column w
  if (warp >= GAIN_COLS) return;
  v = warp_sum(sums[lane][warp]);
  if (lane == 0 && blockIdx.x * GAIN_COLS + warp < D) out[blockIdx.x * GAIN_COLS + warp] = v;
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
// Blocks for each role, by its work: turns of heads a warp, and about one for a token's cos and sin (by the heads alone the keys'
// blocks end last).  Few tokens leave most SMs idle, so their heads go to several warps.
// one_round: all blocks run at once, so what counts is the warp with most turns (1,021 rows of fp32, one slice a token: 14.2 us, by
// this 13.7).
Roles roles_of(const HeadNormArgs& a, int lanes, int most_blocks, bool one_round) {
  const int heads[3] = {a.q.n_heads, a.k.n_heads, a.v.n_heads}, per_warp = 32 / lanes, warps = THREADS / 32;
  int turns[3], all = 0;
  for (int i = 0; i < 3; ++i) {
    turns[i] = (heads[i] + per_warp - 1) / per_warp;
    all += turns[i] > 0 ? turns[i] + 1 : 0;
  }
  Roles r{};
  int at = 0;
  for (int i = 0; i < 3; ++i) {
    r.slices[i] = 1;
    if (turns[i] > 0) {
      const int64_t blocks = static_cast<int64_t>(most_blocks) * (turns[i] + 1) / all, part = blocks > 0 ? blocks : 1;
      int64_t slices = a.n_tokens > 0 ? part * warps / a.n_tokens : 1;
      slices = slices < 1 ? 1 : slices > turns[i] ? turns[i] : slices;
      if (one_round && slices < turns[i]) {
        int64_t least = INT64_MAX;
        for (int n = 1; n <= turns[i] && n <= 16 && static_cast<int64_t>(a.n_tokens) * n <= INT32_MAX; ++n) {
          const int64_t units = (static_cast<int64_t>(a.n_tokens) * n + part * warps - 1) / (part * warps), took = units * ((turns[i] + n - 1) / n + 1);
          if (took < least) least = took, slices = n;
        }
      }
      const int per = static_cast<int>((turns[i] + slices - 1) / slices);  // as many slices as are not empty
      r.slices[i] = (turns[i] + per - 1) / per;
      const int64_t need = (static_cast<int64_t>(a.n_tokens) * r.slices[i] + warps - 1) / warps;
      at += static_cast<int>(need < part ? need : part);
    }
    r.end[i] = at;
  }
  return r;
}

template <typename T, int VEC, int NU, bool INTER, bool PAGES, int DIM>
cudaError_t launch(const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  const Roles r = roles_of(a, lanes_of(a.head_dim, VEC), GRID * num_sms, false);
  return launch_dependent(k_head_norm<T, VEC, NU, INTER, PAGES, DIM>, dim3(r.end[2]), THREADS, 0, st, a, r);
}
template <typename T, bool INTER>
cudaError_t launch_type(const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  if (!wide(a, sizeof(T))) return launch<T, 1, 4, INTER, false, 0>(a, num_sms, st);
  return a.head_dim == 128 ? launch<T, VEC, 1, INTER, false, 128>(a, num_sms, st) : launch<T, VEC, 1, INTER, false, 0>(a, num_sms, st);
}
template <typename T, bool INTER>
cudaError_t launch_pages(const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  return a.head_dim == 128 ? launch<T, 8, 1, INTER, true, 128>(a, num_sms, st) : launch<T, 8, 1, INTER, true, 64>(a, num_sms, st);
}
template <typename T, int D>
cudaError_t launch_append(const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  const Roles r = roles_of(a, D / 16, 16 * num_sms, false);
  return launch_dependent(k_append_4bit<T, D>, dim3(r.end[2]), THREADS, 0, st, a, r);
}
template <typename T, int VEC, int NU, bool INTER, int DIM>
cudaError_t launch_back(const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  const int blocks = BACK_HELD * num_sms < HEAD_NORM_MAX_BLOCKS - 2 ? BACK_HELD * num_sms : HEAD_NORM_MAX_BLOCKS - 2;  // (a part may be rounded up)
  Roles r{};
  if (a.n_tokens > 0) {
    r = roles_of(a, lanes_of(a.head_dim, VEC), blocks, true);
    const cudaError_t e = launch_dependent(k_head_norm_back<T, VEC, NU, INTER, DIM>, dim3(r.end[1]), THREADS, 0, st, a, r);
    if (e != cudaSuccess) return e;
  }
  if (!a.dq_gain && !a.dk_gain) return cudaSuccess;
  return launch_dependent(k_head_norm_gains, dim3((a.head_dim + GAIN_COLS - 1) / GAIN_COLS, 2), 1024, 0, st, a.ws, r.end[0], r.end[1] - r.end[0], a.head_dim,
                          a.dq_gain, a.dk_gain);
}
template <typename T, bool INTER>
cudaError_t launch_back_type(const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  if (!wide(a, sizeof(T))) return launch_back<T, 1, 4, INTER, 0>(a, num_sms, st);
  return a.head_dim == 128 ? launch_back<T, VEC, 1, INTER, 128>(a, num_sms, st) : launch_back<T, VEC, 1, INTER, 0>(a, num_sms, st);
}

// ------------------------------------------------------------------ rows out of 4-bit pages
// A thread 16 elements of a head: two words and their group's scale in, 32 bytes out.  c s is exact.  Bound by how much is on its way: a
// thread asks for ITEMS heads' words before it works on them.  26,800 rows of 8 heads: 23.1 us; a
// thread a run of 8, 25.8.  Few rows: a block as few as make one for each SM (64 rows: 2.4 us).
constexpr int READ_ITEMS = 4;
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) k_read_4bit(const __grid_constant__ Read4Args a) {
  constexpr int LANES = D / 16, GROUPS = THREADS / LANES;
  const int sub = threadIdx.x % LANES, group = threadIdx.x / LANES, page_bits = __ffs(a.page) - 1, Hkv = a.n_kv_heads, rows = a.rows;
  const int64_t page_bytes = pages4::page_bytes(a.page, D);
  bool wide = true;  // a store a sector
  for (const RopeView* v : {&a.k, &a.v}) wide = wide && ((reinterpret_cast<uintptr_t>(v->out) | v->out_tok * 2 | v->out_head * 2) & 31) == 0;
  const int row_of = group / Hkv, head_of = group - row_of * Hkv, row_step = GROUPS / Hkv, head_step = GROUPS - row_step * Hkv;
  pdl_wait();
  pdl_trigger();
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * rows; t0 < a.n_rows; t0 += static_cast<int64_t>(gridDim.x) * rows) {
    const int n = static_cast<int>(min(static_cast<int64_t>(rows), a.n_rows - t0));
    int r = row_of, h = head_of;
    while (r < n) {
      int64_t slot[READ_ITEMS];
      int row[READ_ITEMS], head[READ_ITEMS];
#pragma unroll
      for (int i = 0; i < READ_ITEMS; ++i) {
        row[i] = r, head[i] = h;
        slot[i] = r < n ? a.slots[t0 + r] : -1;
        r += row_step, h += head_step;
        if (h >= Hkv) h -= Hkv, ++r;
        if (slot[i] >= a.n_slots) {
          set_status(a.status, DOPR_ERR_INVALID_ARG);
          slot[i] = -1;
        }
      }
      uint2 word[READ_ITEMS][2];
      uint32_t byte[READ_ITEMS][2];
#pragma unroll
      for (int i = 0; i < READ_ITEMS; ++i) {
        if (slot[i] < 0) continue;
        const int in = static_cast<int>(slot[i]) & (a.page - 1);
        const int64_t at = ((slot[i] >> page_bits) * Hkv + head[i]) * page_bytes;
        const int code = in * (D / 2) + 8 * sub, scale = a.page * (D / 2) + in * (D / 32) + sub / 2;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint8_t* p = (k ? a.v_pool : a.k_pool) + at;
          word[i][k] = *reinterpret_cast<const uint2*>(p + code);
          byte[i][k] = p[scale];
        }
      }
#pragma unroll
      for (int i = 0; i < READ_ITEMS; ++i) {
        if (slot[i] < 0) continue;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t x[8];
          const pages4::Widen<T> widen(byte[i][k] * 0x10001u);
          widen(word[i][k].x, reinterpret_cast<uint32_t(&)[4]>(x[0]));
          widen(word[i][k].y, reinterpret_cast<uint32_t(&)[4]>(x[4]));
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if constexpr (std::is_same_v<T, __half>) {
              const __half2 y = __hmul2(reinterpret_cast<const __half2&>(x[j]), __float2half2_rn(pages4::Widen<T>::UNIT));
              x[j] = reinterpret_cast<const uint32_t&>(y);
            } else {
              const __nv_bfloat162 y = __hmul2(reinterpret_cast<const __nv_bfloat162&>(x[j]), __float2bfloat162_rn(pages4::Widen<T>::UNIT));
              x[j] = reinterpret_cast<const uint32_t&>(y);
            }
            if (byte[i][k] > pages4::SCALE_LAST) x[j] = 0x7fff7fffu;  // NaN
          }
          const RopeView& out = k ? a.v : a.k;
          T* to = static_cast<T*>(out.out) + (t0 + row[i]) * out.out_tok + head[i] * out.out_head + 16 * sub;
          if (wide) {
            st_global32(to, x);
          } else {
            *reinterpret_cast<uint4*>(to) = uint4{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<uint4*>(to + 8) = uint4{x[4], x[5], x[6], x[7]};
          }
        }
      }
    }
  }
}

}  // namespace

cudaError_t launch_head_norm(int dtype, const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  if (a.n_tokens == 0) return cudaSuccess;
  switch (dtype) {
    case DOPR_F16: return a.interleaved ? launch_type<__half, true>(a, num_sms, st) : launch_type<__half, false>(a, num_sms, st);
    case DOPR_BF16: return a.interleaved ? launch_type<__nv_bfloat16, true>(a, num_sms, st) : launch_type<__nv_bfloat16, false>(a, num_sms, st);
    default: return a.interleaved ? launch_type<float, true>(a, num_sms, st) : launch_type<float, false>(a, num_sms, st);
  }
}

cudaError_t launch_head_norm_backward(int dtype, const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  switch (dtype) {
    case DOPR_F16: return a.interleaved ? launch_back_type<__half, true>(a, num_sms, st) : launch_back_type<__half, false>(a, num_sms, st);
    case DOPR_BF16: return a.interleaved ? launch_back_type<__nv_bfloat16, true>(a, num_sms, st) : launch_back_type<__nv_bfloat16, false>(a, num_sms, st);
    default: return a.interleaved ? launch_back_type<float, true>(a, num_sms, st) : launch_back_type<float, false>(a, num_sms, st);
  }
}

cudaError_t launch_append_4bit(int dtype, const HeadNormArgs& a, int num_sms, cudaStream_t st) {
  if (a.n_tokens == 0) return cudaSuccess;
  const bool half = dtype == DOPR_F16;
  if (a.eps == 0.f && a.rotary == 0) {  // rows as they are, and no q
    if (a.head_dim == 128) return half ? launch_append<__half, 128>(a, num_sms, st) : launch_append<__nv_bfloat16, 128>(a, num_sms, st);
    return half ? launch_append<__half, 64>(a, num_sms, st) : launch_append<__nv_bfloat16, 64>(a, num_sms, st);
  }
  if (a.interleaved) return half ? launch_pages<__half, true>(a, num_sms, st) : launch_pages<__nv_bfloat16, true>(a, num_sms, st);
  return half ? launch_pages<__half, false>(a, num_sms, st) : launch_pages<__nv_bfloat16, false>(a, num_sms, st);
}

cudaError_t launch_read_4bit(int dtype, const Read4Args& a, int num_sms, cudaStream_t st) {
  if (a.n_rows == 0) return cudaSuccess;
  Read4Args args = a;
  const int most = READ_ITEMS * THREADS / (a.head_dim / 16) / a.n_kv_heads, even = (a.n_rows - 1) / num_sms + 1;
  args.rows = most < 1 ? 1 : most < even ? most : even;
  const int blocks = (a.n_rows - 1) / args.rows + 1;
  const dim3 grid(blocks < 64 * num_sms ? blocks : 64 * num_sms);
  if (a.head_dim == 128)
    return dtype == DOPR_F16 ? launch_dependent(k_read_4bit<__half, 128>, grid, THREADS, 0, st, args)
                             : launch_dependent(k_read_4bit<__nv_bfloat16, 128>, grid, THREADS, 0, st, args);
  return dtype == DOPR_F16 ? launch_dependent(k_read_4bit<__half, 64>, grid, THREADS, 0, st, args)
                           : launch_dependent(k_read_4bit<__nv_bfloat16, 64>, grid, THREADS, 0, st, args);
}

}  // namespace dopr
