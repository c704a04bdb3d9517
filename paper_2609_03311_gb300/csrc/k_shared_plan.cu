// k_shared_plan.cu -- the split of a step's attention over the paged cache (dopr_shared_attention_plan), from offsets,
// lengths and prefixes on the device.
//
// One CTA: everything is sums over the step's rows, and the rows of a prefix brought together.  Rows usually come in
// prefix order; those that do not are sorted (a bitonic network over (prefix, row) in shared memory; rows of a
// prefix keep their order).  Bound by latency; made once a step and used by every layer.
#include "shared_attn.cuh"

namespace dopr {
namespace {
using namespace shared_attn;

constexpr int THREADS = 1024;
constexpr int ROW_BITS = 14;
static_assert(CACHE_MAX_SEQS == 1 << ROW_BITS, "a sort key holds two row numbers");

// Exclusive sums over the block's threads in order; the block's total through `total`.
template <typename T>
__device__ T block_exclusive(T v, T* warp_sum, T& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  T inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T u = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += u;
  }
  __syncthreads();  // the last use of warp_sum is over
  if (lane == 31) warp_sum[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    T w = warp_sum[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T u = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += u;
    }
    warp_sum[lane] = w;
  }
  __syncthreads();
  total = warp_sum[31];
  return (warp > 0 ? warp_sum[warp - 1] : T(0)) + inc - v;
}

__global__ void __launch_bounds__(THREADS) k_shared_plan(SharedPlanArgs a, int n_ctas) {
  extern __shared__ uint32_t keys[];  // a power of two >= n_seqs
  __shared__ unsigned long long warp_sum[32];
  __shared__ int bad, unsorted;
  const int n = a.lay.n_seqs, Hkv = a.lay.n_kv_heads, G = a.Hq / Hkv;
  const int tile = tokens_a_tile(G), pair = 2 * tile;
  const int64_t cap = static_cast<int64_t>(a.lay.max_blocks) * a.lay.page;
  const Plan p = plan_view(a.plan, n, Hkv, G, a.max_tokens);
  int* sorted = p.scratch;        // rows that read a prefix, by prefix
  int* place = sorted + n;        // of a sorted entry: tokens of the entries before it
  int* group = place + n + 1;     // of a prefix: tokens before its first
  int* group_item = group + n;    // of a prefix: its first item
  int* own_item = group_item + n; // of a row: its first item
  int* in_group = own_item + n;   // of a row: its first token's place among its prefix's tokens; -1 if it reads none
  if (threadIdx.x == 0) bad = 0, unsorted = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  Head head{};
  head.share = 1;
  head.n_seqs = n;
  head.n_kv_heads = Hkv;
  head.Hq = a.Hq;
  head.max_tokens = a.max_tokens;
  head.n_ctas = n_ctas;
  head.head_dim = a.lay.head_dim;
  auto tokens_of = [&](int i) { return a.tok_off[i + 1] - a.tok_off[i]; };
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const int t0 = a.tok_off[i], t1 = a.tok_off[i + 1], pre = a.prefix ? a.prefix[i] : -1;
    if ((i == 0 && t0 != 0) || t1 < t0 || t1 > a.max_tokens || a.seq_lens[i] < 0 || a.seq_lens[i] > cap || pre < -1 ||
        pre >= n || pre == i || (pre >= 0 && a.prefix[pre] != -1))
      bad = 1;
  }
  __syncthreads();
  if (bad) {
    if (threadIdx.x == 0) {
      *p.head = head;
      if (a.status) atomicCAS(a.status, 0, DOPR_ERR_INVALID_ARG);
    }
    for (int c = threadIdx.x; c < MAX_CTAS; c += THREADS) p.first[c] = 0;
    return;
  }

  // rows that read a prefix
  unsigned long long total;
  int ns = 0;
  for (int i0 = 0; i0 < n; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    const int pre = i < n && a.prefix ? a.prefix[i] : -1;
    const bool reads = pre >= 0 && tokens_of(i) > 0 && a.seq_lens[pre] > 0;
    const int at = ns + static_cast<int>(block_exclusive(static_cast<unsigned long long>(reads), warp_sum, total));
    if (reads) sorted[at] = i;
    if (i < n) in_group[i] = -1;
    ns += static_cast<int>(total);
  }
  __syncthreads();
  for (int i = threadIdx.x + 1; i < ns; i += THREADS)
    if (a.prefix[sorted[i]] < a.prefix[sorted[i - 1]]) unsorted = 1;
  __syncthreads();
  if (unsorted) {
    int m = 2;
    while (m < ns) m <<= 1;
    for (int i = threadIdx.x; i < m; i += THREADS)
      keys[i] = i < ns ? static_cast<uint32_t>(a.prefix[sorted[i]]) << ROW_BITS | sorted[i] : 0xffffffffu;
    for (int k = 2; k <= m; k <<= 1)
      for (int j = k >> 1; j > 0; j >>= 1) {
        __syncthreads();
        for (int i = threadIdx.x; i < m; i += THREADS) {
          const int o = i ^ j;
          if (o > i) {
            const uint32_t x = keys[i], y = keys[o];
            if ((x > y) == ((i & k) == 0)) keys[i] = y, keys[o] = x;
          }
        }
      }
    __syncthreads();
    for (int i = threadIdx.x; i < ns; i += THREADS) sorted[i] = keys[i] & ((1 << ROW_BITS) - 1);
    __syncthreads();
  }
  int carry = 0;
  for (int i0 = 0; i0 < ns; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    const int tok = i < ns ? tokens_of(sorted[i]) : 0;
    const int at = carry + static_cast<int>(block_exclusive(static_cast<unsigned long long>(tok), warp_sum, total));
    if (i < ns) {
      place[i] = at;
      const int pre = a.prefix[sorted[i]];
      if (i == 0 || a.prefix[sorted[i - 1]] != pre) group[pre] = at;
    }
    carry += static_cast<int>(total);
  }
  if (threadIdx.x == 0) place[ns] = carry;
  __syncthreads();

  // items of prefixes, written by the last row of each; then of own keys, by their rows
  int n_items = 0;
  for (int i0 = 0; i0 < ns; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    const int pre = i < ns ? a.prefix[sorted[i]] : -1;
    int count = 0, tok = 0;
    if (i < ns) {
      in_group[sorted[i]] = place[i] - group[pre];
      if (i + 1 == ns || a.prefix[sorted[i + 1]] != pre) {
        tok = place[i + 1] - group[pre];
        count = (tok + pair - 1) / pair;
      }
    }
    const int at = n_items + static_cast<int>(block_exclusive(static_cast<unsigned long long>(count), warp_sum, total));
    if (count > 0) group_item[pre] = at;
    for (int c = 0; c < count; ++c) {
      Item it{};
      it.tok = group[pre] + c * pair;
      it.n_tok = min(pair, tok - c * pair);
      it.row = pre;
      it.n_keys = a.seq_lens[pre];
      p.items[at + c] = it;
    }
    n_items += static_cast<int>(total);
  }
  for (int i0 = 0; i0 < n; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    const int tok = i < n ? tokens_of(i) : 0, len = tok > 0 ? a.seq_lens[i] : 0;
    const int count = len > 0 ? (tok + pair - 1) / pair : 0;
    const int at = n_items + static_cast<int>(block_exclusive(static_cast<unsigned long long>(count), warp_sum, total));
    if (i < n) own_item[i] = count > 0 ? at : -1;
    for (int c = 0; c < count; ++c) {
      Item it{};
      it.tok = a.tok_off[i] + c * pair;
      it.n_tok = min(pair, tok - c * pair);
      it.row = i;
      it.seen = len - tok + c * pair + 1;
      it.n_keys = max(0, it.seen + it.n_tok - 1);
      it.own = 1;
      p.items[at + c] = it;
    }
    n_items += static_cast<int>(total);
  }
  __syncthreads();

  // every token's items and places, a warp a row
  for (int i = threadIdx.x >> 5; i < n; i += THREADS / 32) {
    const int t0 = a.tok_off[i], tok = tokens_of(i), in = in_group[i], own = own_item[i];
    const int pre = in >= 0 ? a.prefix[i] : 0;
    for (int j = threadIdx.x & 31; j < tok; j += 32) {
      int4 r = make_int4(-1, 0, -1, 0);
      if (in >= 0) {
        r.x = group_item[pre] + (in + j) / pair;
        r.y = (in + j) % pair;
        p.order[group[pre] + in + j] = t0 + j;
      }
      if (own >= 0) {
        r.z = own + j / pair;
        r.w = j % pair;
      }
      p.rec[t0 + j] = r;
    }
  }

  // the line
  unsigned long long line = 0;
  for (int i0 = 0; i0 < n_items; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    const uint32_t blocks = i < n_items ? blocks_of(p.items[i].n_keys) : 0;
    const unsigned long long cost = blocks > 0 ? static_cast<unsigned long long>(Hkv) * (blocks + OVERHEAD) : 0;
    const unsigned long long at = line + block_exclusive(cost, warp_sum, total);
    if (i < n_items) p.items[i].cost = static_cast<uint32_t>(at);
    line += total;
  }
  const bool fits = line < 0x80000000ull;
  const uint32_t share = fits ? max(1u, static_cast<uint32_t>((line + n_ctas - 1) / n_ctas)) : 1;
  const int n_flat = n_items * Hkv;
  for (int c = threadIdx.x; c < MAX_CTAS; c += THREADS) p.first[c] = n_flat;
  if (threadIdx.x == 0) {
    if (fits) {
      head.tokens = a.tok_off[n];
      head.n_items = n_items;
      head.n_flat = n_flat;
      head.share = share;
      head.total = static_cast<uint32_t>(line);
    }
    *p.head = head;
    if (!fits && a.status) atomicCAS(a.status, 0, DOPR_ERR_UNSUPPORTED);
  }
  __syncthreads();
  if (!fits) return;
  unsigned long long rows = 0;
  for (int f0 = 0; f0 < n_flat; f0 += THREADS) {
    const int f = f0 + threadIdx.x;
    unsigned long long count = 0;
    if (f < n_flat) {
      const Item it = p.items[f / Hkv];
      const uint32_t blocks = blocks_of(it.n_keys);
      if (blocks > 0) {
        const uint32_t b = keys_begin(it, blocks, f % Hkv), e = b + blocks, start = b - OVERHEAD;
        const uint32_t segs = (e - 1) / share - b / share + 1;
        count = static_cast<unsigned long long>(segs) * it.n_tok * G * (two_tiles(it.n_tok, G) ? 1 : 2);
        for (uint32_t c = (start + share - 1) / share; static_cast<unsigned long long>(c) * share < e; ++c)
          if (c < MAX_CTAS) p.first[c] = f;
      }
    }
    const unsigned long long at = rows + block_exclusive(count, warp_sum, total);
    if (f < n_flat) p.part[f] = static_cast<uint32_t>(at);
    rows += total;
  }
}

}  // namespace

int64_t shared_plan_bytes(const dopr_cache_layout& lay, int Hq, int max_tokens) {
  return plan_view(nullptr, lay.n_seqs, lay.n_kv_heads, Hq / lay.n_kv_heads, max_tokens).bytes;
}

cudaError_t launch_shared_plan(const SharedPlanArgs& a, int num_sms, cudaStream_t st) {
  int keys = 2;
  while (keys < a.lay.n_seqs) keys <<= 1;
  static_assert(CACHE_MAX_SEQS * 4 <= 65536, "shared memory of the sort");
  const cudaError_t e = cudaFuncSetAttribute(k_shared_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, 65536);
  if (e != cudaSuccess) return e;
  return launch_dependent(k_shared_plan, dim3(1), THREADS, keys * 4, st, a, num_sms < MAX_CTAS ? num_sms : MAX_CTAS);
}

}  // namespace dopr
