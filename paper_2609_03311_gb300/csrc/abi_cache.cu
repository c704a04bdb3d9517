// abi_cache.cu -- C entry points of the paged prefix cache's operators (include/dopr.h): arguments are checked here,
// what lies on the device is checked by the kernels.  Nothing here allocates (dopr_rope_create aside), synchronises
// or throws.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <initializer_list>
#include <new>

#include "device_common.cuh"
#include "internal.h"
#include "pages4.cuh"

struct dopr_rope : dopr::Rope {};

namespace dopr {
namespace {

dopr_status fail(dopr_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  set_last_error_message(buf);
  return st;
}
#define STATUS_TRY(call)          \
  do {                            \
    dopr_status s_ = (call);      \
    if (s_ != DOPR_OK) return s_; \
  } while (0)

dopr_status cuda_status(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return DOPR_OK;
  return fail(e == cudaErrorMemoryAllocation ? DOPR_ERR_OUT_OF_MEMORY : DOPR_ERR_CUDA, "%s failed: %s", what,
              cudaGetErrorString(e));
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// Pointers to 32-bit numbers (NULL is aligned), which the kernels read and write whole.
dopr_status check_words(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!aligned(p, 4)) return fail(DOPR_ERR_INVALID_ARG, "a pointer to 32-bit numbers is not aligned to 4 bytes");
  return DOPR_OK;
}

dopr_status check_layout(const dopr_cache_layout* l) {
  if (!l) return fail(DOPR_ERR_INVALID_ARG, "layout is NULL");
  if (l->n_blocks <= 0 || l->n_kv_heads <= 0 || l->n_seqs <= 0 || l->max_blocks <= 0)
    return fail(DOPR_ERR_INVALID_ARG, "layout sizes must be positive");
  if (l->page != 16 && l->page != 32 && l->page != 64 && l->page != 128)
    return fail(DOPR_ERR_UNSUPPORTED, "page must be 16, 32, 64 or 128 (got %d)", l->page);
  if (l->head_dim != 64 && l->head_dim != 128)
    return fail(DOPR_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", l->head_dim);
  if (l->dtype != DOPR_F16 && l->dtype != DOPR_BF16) return fail(DOPR_ERR_UNSUPPORTED, "the cache holds F16 or BF16");
  if (l->n_seqs > CACHE_MAX_SEQS) return fail(DOPR_ERR_UNSUPPORTED, "n_seqs above %d", CACHE_MAX_SEQS);
  if ((int64_t)l->max_blocks * l->page > INT32_MAX) return fail(DOPR_ERR_UNSUPPORTED, "max_blocks * page above 2^31 - 1");
  if ((int64_t)l->n_blocks * l->page > INT32_MAX / l->n_kv_heads)
    return fail(DOPR_ERR_UNSUPPORTED, "n_blocks * n_kv_heads * page above 2^31 - 1");
  return DOPR_OK;
}

// A view that is read or written; `vectors`: 16-byte alignment is required.
dopr_status check_view(const dopr_heads* v, const char* name, int head_dim, int size, bool vectors, int heads) {
  if (!v || !v->data) return fail(DOPR_ERR_INVALID_ARG, "%s is NULL", name);
  if (v->n_heads <= 0 || v->n_heads > 65535) return fail(DOPR_ERR_INVALID_ARG, "%s: n_heads outside 1 .. 65535", name);
  if (heads > 0 && v->n_heads != heads)
    return fail(DOPR_ERR_INVALID_ARG, "%s: %d heads where %d belong", name, v->n_heads, heads);
  if (v->token_stride < 0 || v->head_stride < 0 || (v->n_heads > 1 && v->head_stride < head_dim))
    return fail(DOPR_ERR_INVALID_ARG, "%s: a stride is negative, or heads overlap", name);
  if (!aligned(v->data, size)) return fail(DOPR_ERR_INVALID_ARG, "%s is not aligned to its type", name);
  if (vectors && (!aligned(v->data, 16) || v->token_stride * size % 16 || (v->n_heads > 1 && v->head_stride * size % 16)))
    return fail(DOPR_ERR_INVALID_ARG, "%s: data and strides must be multiples of 16 bytes", name);
  return DOPR_OK;
}

// A view that is written: no two of its rows share elements.
dopr_status check_output(const dopr_heads* v, const char* name, int head_dim, int size, bool vectors, int heads, int tokens) {
  STATUS_TRY(check_view(v, name, head_dim, size, vectors, heads));
  if (tokens <= 1) return DOPR_OK;
  const bool heads_inside = v->n_heads == 1 || v->head_stride <= v->token_stride;
  const int64_t inner = v->n_heads == 1 ? head_dim : heads_inside ? v->head_stride : v->token_stride;
  const int64_t outer = heads_inside ? v->token_stride : v->head_stride, n = heads_inside ? v->n_heads : tokens;
  if (inner < head_dim || (outer - head_dim) / (n > 1 ? n - 1 : 1) < (n > 1 ? inner : 0) || outer < head_dim)
    return fail(DOPR_ERR_INVALID_ARG, "%s: rows of an output overlap or interleave", name);
  return DOPR_OK;
}

int type_size(int dtype) { return dtype == DOPR_F32 ? 4 : 2; }

dopr_status check_rope_use(const dopr_rope* r, int head_dim, const int32_t* positions) {
  if (r->cfg.rotary_dim > head_dim)
    return fail(DOPR_ERR_INVALID_ARG, "rotary_dim %d above head_dim %d", r->cfg.rotary_dim, head_dim);
  int dev = -1;
  STATUS_TRY(cuda_status(cudaGetDevice(&dev), "cudaGetDevice"));
  if (dev != r->device)
    return fail(DOPR_ERR_INVALID_ARG, "the rotary table is on device %d, device %d is current", r->device, dev);
  if (!positions) return fail(DOPR_ERR_INVALID_ARG, "positions is NULL");
  return DOPR_OK;
}

RopeArgs rope_args(const dopr_rope* r, int n_tokens, int head_dim, const int32_t* positions, int32_t* status) {
  RopeArgs a{};
  a.n_tokens = n_tokens;
  a.head_dim = head_dim;
  a.page = 1;
  a.status = status;
  a.positions = positions;
  if (r) {
    a.rotary = r->cfg.rotary_dim;
    a.interleaved = r->cfg.layout == DOPR_ROPE_INTERLEAVED;
    a.table = r->table;
    a.max_position = r->cfg.max_position;
  }
  return a;
}
RopeView rope_view(const dopr_heads* in, const dopr_heads* out) {
  RopeView v{};
  v.in = in->data;
  v.in_tok = in->token_stride;
  v.in_head = in->head_stride;
  v.n_heads = in->n_heads;
  if (out) {
    v.out = out->data;
    v.out_tok = out->token_stride;
    v.out_head = out->head_stride;
  }
  return v;
}

dopr_status check_rope_config(const dopr_rope_config* c) {
  if (!c) return fail(DOPR_ERR_INVALID_ARG, "config is NULL");
  if (c->max_position <= 0 || c->rotary_dim <= 0) return fail(DOPR_ERR_INVALID_ARG, "config sizes must be positive");
  if (c->max_position > (1 << 22)) return fail(DOPR_ERR_UNSUPPORTED, "max_position above 2^22");
  if (c->rotary_dim % 2 || c->rotary_dim > 256) return fail(DOPR_ERR_UNSUPPORTED, "rotary_dim must be even, at most 256");
  if (c->layout != DOPR_ROPE_HALF && c->layout != DOPR_ROPE_INTERLEAVED)
    return fail(DOPR_ERR_INVALID_ARG, "unknown layout %d", c->layout);
  if (c->scaling < DOPR_ROPE_PLAIN || c->scaling > DOPR_ROPE_RAMP)
    return fail(DOPR_ERR_INVALID_ARG, "unknown scaling %d", c->scaling);
  if (!(c->theta > 1.0) || !isfinite(c->theta)) return fail(DOPR_ERR_INVALID_ARG, "theta must be above 1");
  if (c->scaling == DOPR_ROPE_PLAIN) return DOPR_OK;
  if (!(c->factor >= 1.0) || !isfinite(c->factor)) return fail(DOPR_ERR_INVALID_ARG, "factor must be at least 1");
  if (c->scaling == DOPR_ROPE_NTK && c->rotary_dim < 4) return fail(DOPR_ERR_INVALID_ARG, "NTK needs rotary_dim >= 4");
  if (c->scaling >= DOPR_ROPE_BANDS) {
    if (c->original_max_position <= 0 || !(c->low > 0.0) || !(c->high > c->low) || !isfinite(c->high))
      return fail(DOPR_ERR_INVALID_ARG, "original_max_position > 0 and 0 < low < high are needed");
    if (c->scaling == DOPR_ROPE_RAMP && (!(c->attention_factor >= 0.0) || !isfinite(c->attention_factor)))
      return fail(DOPR_ERR_INVALID_ARG, "attention_factor must be at least 0");
  }
  return DOPR_OK;
}

// Radians a position of each pair; returns the factor on cos and sin.
double rope_frequencies(const dopr_rope_config& c, double* f) {
  const double pi2 = 6.283185307179586476925286766559;
  const int d = c.rotary_dim;
  const double base = c.scaling == DOPR_ROPE_NTK ? c.theta * pow(c.factor, d / (d - 2.0)) : c.theta;
  double lo = 0, hi = 0;
  if (c.scaling == DOPR_ROPE_RAMP) {
    auto index = [&](double turns) { return d * log(c.original_max_position / (turns * pi2)) / (2 * log(c.theta)); };
    lo = fmax(floor(index(c.high)), 0.0);
    hi = fmin(ceil(index(c.low)), d - 1.0);
  }
  for (int i = 0; i < d / 2; ++i) {
    const double g = pow(base, -2.0 * i / d);
    f[i] = g;
    if (c.scaling == DOPR_ROPE_LINEAR) f[i] = g / c.factor;
    if (c.scaling == DOPR_ROPE_BANDS || c.scaling == DOPR_ROPE_RAMP) {
      // t: the share of the unscaled frequency
      const double t = c.scaling == DOPR_ROPE_BANDS ? (c.original_max_position * g / pi2 - c.low) / (c.high - c.low)
                                                    : 1.0 - (i - lo) / fmax(hi - lo, 1e-3);
      const double u = fmin(fmax(t, 0.0), 1.0);
      f[i] = (1.0 - u) * g / c.factor + u * g;
    }
  }
  if (c.scaling != DOPR_ROPE_RAMP) return 1.0;
  return c.attention_factor > 0 ? c.attention_factor : 0.1 * log(c.factor) + 1.0;
}

dopr_status check_attention(const dopr_cache_layout* l, int n_q_heads, int max_tokens) {
  STATUS_TRY(check_layout(l));
  if (n_q_heads <= 0 || max_tokens < 0) return fail(DOPR_ERR_INVALID_ARG, "n_q_heads must be positive, max_tokens not negative");
  if (n_q_heads % l->n_kv_heads || n_q_heads / l->n_kv_heads > 64)
    return fail(DOPR_ERR_UNSUPPORTED, "%d q heads on %d kv heads: the quotient must be whole, 1 .. 64", n_q_heads, l->n_kv_heads);
  if ((int64_t)max_tokens * n_q_heads > INT32_MAX / 8)
    return fail(DOPR_ERR_UNSUPPORTED, "max_tokens * n_q_heads above 2^28");
  return DOPR_OK;
}

// Arguments that a norm of heads has in common with its gradients and with the append.
dopr_status check_norm(float eps, int gain_dtype, const void* q_gain, const void* k_gain) {
  if (!(eps > 0.f) || !isfinite(eps)) return fail(DOPR_ERR_INVALID_ARG, "eps must be positive");
  if (!q_gain && !k_gain) return DOPR_OK;
  if (gain_dtype < DOPR_F16 || gain_dtype > DOPR_F32) return fail(DOPR_ERR_INVALID_ARG, "unknown gain_dtype %d", gain_dtype);
  if (!aligned(q_gain, type_size(gain_dtype)) || !aligned(k_gain, type_size(gain_dtype)))
    return fail(DOPR_ERR_INVALID_ARG, "a gain is not aligned to its type");
  return DOPR_OK;
}
dopr_status check_head_dim(int head_dim) {
  if (head_dim <= 0 || head_dim % 2 || head_dim > 256)
    return fail(DOPR_ERR_UNSUPPORTED, "head_dim must be even, at most 256 (got %d)", head_dim);
  return DOPR_OK;
}
HeadNormArgs norm_args(const dopr_rope* r, int n_tokens, int head_dim, const int32_t* positions, float eps, int gain_dtype,
                       const void* q_gain, const void* k_gain, int32_t* status) {
  HeadNormArgs a{};
  a.n_tokens = n_tokens;
  a.head_dim = head_dim;
  a.eps = eps;
  a.positions = positions;
  a.gain_dtype = gain_dtype;
  a.q_gain = q_gain;
  a.k_gain = k_gain;
  a.page = 1;
  a.status = status;
  if (r) {
    a.rotary = r->cfg.rotary_dim;
    a.interleaved = r->cfg.layout == DOPR_ROPE_INTERLEAVED;
    a.table = r->table;
    a.max_position = r->cfg.max_position;
  }
  return a;
}

// SMs of the current device.
dopr_status sm_count(int* n) {
  int dev = -1;
  STATUS_TRY(cuda_status(cudaGetDevice(&dev), "cudaGetDevice"));
  return cuda_status(cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev), "cudaDeviceGetAttribute");
}

// dopr_shared_attention over 16-bit pools and over those of the 4-bit cache.
dopr_status attention(bool four, const dopr_cache_layout* layout, const void* plan, int32_t max_tokens, const dopr_heads* q, const void* k_pool,
                      const void* v_pool, const int32_t* block_tables, float scale, const dopr_heads* out, float* lse, void* workspace,
                      int32_t* status, void* cuda_stream) {
  if (!q) return fail(DOPR_ERR_INVALID_ARG, "q is NULL");
  STATUS_TRY(check_attention(layout, q->n_heads, max_tokens));
  if (max_tokens == 0) return DOPR_OK;  // views of no rows have no data
  if (!plan || !k_pool || !v_pool || !block_tables || !workspace)
    return fail(DOPR_ERR_INVALID_ARG, "plan, k_pool, v_pool, block_tables or workspace is NULL");
  if (!aligned(plan, 16) || !aligned(k_pool, 16) || !aligned(v_pool, 16))
    return fail(DOPR_ERR_INVALID_ARG, "plan and pools must be 16-byte aligned");
  STATUS_TRY(check_words({block_tables, lse, status}));
  if (!(scale > 0.f) || !isfinite(scale)) return fail(DOPR_ERR_INVALID_ARG, "scale must be positive");
  STATUS_TRY(check_view(q, "q", layout->head_dim, 2, true, 0));
  STATUS_TRY(check_output(out, "out", layout->head_dim, 2, true, q->n_heads, max_tokens));
  if (!aligned(workspace, 32)) return fail(DOPR_ERR_INVALID_ARG, "the workspace must be 32-byte aligned");
  SharedAttnArgs a{};
  a.lay = *layout;
  a.Hq = q->n_heads;
  a.max_tokens = max_tokens;
  a.plan = plan;
  a.q = q->data;
  a.q_tok = q->token_stride;
  a.q_head = q->head_stride;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.tables = block_tables;
  a.scale = scale;
  a.out = out->data;
  a.o_tok = out->token_stride;
  a.o_head = out->head_stride;
  a.lse = lse;
  a.ws = static_cast<uint8_t*>(workspace);
  a.status = status;
  int sms = 0;
  STATUS_TRY(sm_count(&sms));
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return four ? cuda_status(launch_shared_attention_4bit(a, sms, st), "dopr_shared_attention_4bit")
              : cuda_status(launch_shared_attention(a, sms, st), "dopr_shared_attention");
}

}  // namespace
}  // namespace dopr

using namespace dopr;

extern "C" {

dopr_status dopr_cache_extend(const dopr_cache_layout* layout, const int32_t* seq_lens, int32_t* block_tables,
                              int32_t* free_blocks, const int32_t* n_free, const int32_t* prefix, const int32_t* new_lens,
                              int32_t max_tokens, int32_t* seq_lens_out, int32_t* n_free_out, int32_t* tok_off,
                              int64_t* slots, int32_t* positions, void* workspace, int32_t* status, void* cuda_stream) {
  STATUS_TRY(check_layout(layout));
  if (max_tokens < 0) return fail(DOPR_ERR_INVALID_ARG, "max_tokens is negative");
  if (!seq_lens || !block_tables || !free_blocks || !n_free || !new_lens || !seq_lens_out || !n_free_out || !tok_off ||
      (max_tokens > 0 && (!slots || !positions)) || !workspace)
    return fail(DOPR_ERR_INVALID_ARG, "a pointer is NULL");
  if (!aligned(workspace, 16)) return fail(DOPR_ERR_INVALID_ARG, "the workspace must be 16-byte aligned");
  if (!aligned(slots, 8)) return fail(DOPR_ERR_INVALID_ARG, "slots must be 8-byte aligned");
  STATUS_TRY(check_words({seq_lens, block_tables, free_blocks, n_free, prefix, new_lens, seq_lens_out, n_free_out, tok_off, positions,
                          status}));
  CacheExtendArgs a{};
  a.lay = *layout;
  a.seq_lens = seq_lens;
  a.tables = block_tables;
  a.free_blocks = free_blocks;
  a.n_free = n_free;
  a.prefix = prefix;
  a.new_lens = new_lens;
  a.max_tokens = max_tokens;
  a.seq_lens_out = seq_lens_out;
  a.n_free_out = n_free_out;
  a.tok_off = tok_off;
  a.slots = slots;
  a.positions = positions;
  a.ws = static_cast<int32_t*>(workspace);
  a.status = status;
  return cuda_status(launch_cache_extend(a, static_cast<cudaStream_t>(cuda_stream)), "dopr_cache_extend");
}

int64_t dopr_cache_extend_workspace(const dopr_cache_layout* layout) {
  if (check_layout(layout) != DOPR_OK) return -1;
  return (CACHE_WS_HEAD + 3 * (int64_t)layout->n_seqs) * (int64_t)sizeof(int32_t);
}

dopr_status dopr_rope_create(const dopr_rope_config* cfg, dopr_rope** out) {
  if (!out) return fail(DOPR_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  STATUS_TRY(check_rope_config(cfg));
  double f[128];
  const double gain = rope_frequencies(*cfg, f);
  const int half = cfg->rotary_dim / 2;
  dopr_rope* r = new (std::nothrow) dopr_rope();
  if (!r) return fail(DOPR_ERR_OUT_OF_MEMORY, "no host memory for the rotary table's handle");
  r->cfg = *cfg;
  double* d_f = nullptr;
  cudaError_t e = cudaGetDevice(&r->device);
  if (e == cudaSuccess) e = cudaMalloc(&r->table, sizeof(float2) * half * (size_t)cfg->max_position);
  if (e == cudaSuccess) e = cudaMalloc(&d_f, sizeof(double) * half);
  if (e == cudaSuccess) e = cudaMemcpy(d_f, f, sizeof(double) * half, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = launch_rope_table(d_f, gain, cfg->max_position, half, r->table, nullptr);
  if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
  if (d_f) cudaFree(d_f);
  if (e != cudaSuccess) {
    cudaGetLastError();  // a refused allocation is not left behind for the next launch to find
    if (r->table) cudaFree(r->table);
    delete r;
    return cuda_status(e, "dopr_rope_create");
  }
  *out = r;
  return DOPR_OK;
}

dopr_status dopr_rope_destroy(dopr_rope* rope) {
  if (!rope) return DOPR_OK;
  int dev = -1;
  cudaGetDevice(&dev);
  if (dev != rope->device) cudaSetDevice(rope->device);
  cudaFree(rope->table);
  if (dev >= 0 && dev != rope->device) cudaSetDevice(dev);
  delete rope;
  return DOPR_OK;
}

dopr_status dopr_rope_apply(const dopr_rope* rope, int32_t dtype, int32_t head_dim, int32_t n_tokens,
                            const int32_t* positions, const dopr_heads* q, const dopr_heads* q_out, const dopr_heads* k,
                            const dopr_heads* k_out, int32_t inverse, int32_t* status, void* cuda_stream) {
  if (!rope) return fail(DOPR_ERR_INVALID_ARG, "rope is NULL");
  if (dtype < DOPR_F16 || dtype > DOPR_F32) return fail(DOPR_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (n_tokens < 0) return fail(DOPR_ERR_INVALID_ARG, "n_tokens is negative");
  if (head_dim <= 0 || head_dim % 2 || head_dim > 256)
    return fail(DOPR_ERR_UNSUPPORTED, "head_dim must be even, at most 256 (got %d)", head_dim);
  if (!k != !k_out) return fail(DOPR_ERR_INVALID_ARG, "k and k_out belong together");
  if (n_tokens == 0) return DOPR_OK;  // views of no rows have no data
  STATUS_TRY(check_rope_use(rope, head_dim, positions));
  STATUS_TRY(check_words({positions, status}));
  const int size = type_size(dtype);
  STATUS_TRY(check_view(q, "q", head_dim, size, false, 0));
  STATUS_TRY(check_output(q_out, "q_out", head_dim, size, false, q->n_heads, n_tokens));
  RopeArgs a = rope_args(rope, n_tokens, head_dim, positions, status);
  a.inverse = inverse != 0;
  a.q = rope_view(q, q_out);
  if (k) {
    STATUS_TRY(check_view(k, "k", head_dim, size, false, 0));
    STATUS_TRY(check_output(k_out, "k_out", head_dim, size, false, k->n_heads, n_tokens));
    a.k = rope_view(k, k_out);
  }
  return cuda_status(launch_rope(dtype, a, static_cast<cudaStream_t>(cuda_stream)), "dopr_rope_apply");
}

dopr_status dopr_cache_append(const dopr_cache_layout* layout, const dopr_rope* rope, int32_t n_tokens,
                              const int32_t* positions, const int64_t* slots, const dopr_heads* q, const dopr_heads* q_out,
                              const dopr_heads* k, const dopr_heads* v, void* k_pool, void* v_pool, int32_t* status,
                              void* cuda_stream) {
  STATUS_TRY(check_layout(layout));
  if (n_tokens < 0) return fail(DOPR_ERR_INVALID_ARG, "n_tokens is negative");
  if (n_tokens == 0) return DOPR_OK;  // views of no rows have no data
  if (!slots || !k_pool || !v_pool) return fail(DOPR_ERR_INVALID_ARG, "slots, k_pool or v_pool is NULL");
  if (!aligned(k_pool, 16) || !aligned(v_pool, 16)) return fail(DOPR_ERR_INVALID_ARG, "the pools must be 16-byte aligned");
  if (!aligned(slots, 8)) return fail(DOPR_ERR_INVALID_ARG, "slots must be 8-byte aligned");
  STATUS_TRY(check_words({rope ? positions : nullptr, status}));
  if (!q != !q_out) return fail(DOPR_ERR_INVALID_ARG, "q and q_out belong together");
  if (q && !rope) return fail(DOPR_ERR_INVALID_ARG, "q without a rotary table");
  if (rope) STATUS_TRY(check_rope_use(rope, layout->head_dim, positions));
  const int D = layout->head_dim, size = type_size(layout->dtype);
  STATUS_TRY(check_view(k, "k", D, size, false, layout->n_kv_heads));
  STATUS_TRY(check_view(v, "v", D, size, false, layout->n_kv_heads));
  RopeArgs a = rope_args(rope, n_tokens, D, positions, status);
  if (q) {
    STATUS_TRY(check_view(q, "q", D, size, false, 0));
    STATUS_TRY(check_output(q_out, "q_out", D, size, false, q->n_heads, n_tokens));
    a.q = rope_view(q, q_out);
  }
  a.k = rope_view(k, nullptr);
  a.v = rope_view(v, nullptr);
  a.slots = slots;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.page = layout->page;
  a.n_slots = (int64_t)layout->n_blocks * layout->page;
  return cuda_status(launch_rope(layout->dtype, a, static_cast<cudaStream_t>(cuda_stream)), "dopr_cache_append");
}

dopr_status dopr_head_norm_rope(const dopr_rope* rope, int32_t dtype, int32_t head_dim, int32_t n_tokens, const int32_t* positions,
                                float eps, int32_t gain_dtype, const dopr_heads* q, const void* q_gain, const dopr_heads* q_out,
                                const dopr_heads* k, const void* k_gain, const dopr_heads* k_out, int32_t* status,
                                void* cuda_stream) {
  if (dtype < DOPR_F16 || dtype > DOPR_F32) return fail(DOPR_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (n_tokens < 0) return fail(DOPR_ERR_INVALID_ARG, "n_tokens is negative");
  STATUS_TRY(check_head_dim(head_dim));
  STATUS_TRY(check_norm(eps, gain_dtype, q_gain, k_gain));
  if (!k != !k_out) return fail(DOPR_ERR_INVALID_ARG, "k and k_out belong together");
  if (n_tokens == 0) return DOPR_OK;  // views of no rows have no data
  if (rope) STATUS_TRY(check_rope_use(rope, head_dim, positions));
  STATUS_TRY(check_words({rope ? positions : nullptr, status}));
  const int size = type_size(dtype);
  STATUS_TRY(check_view(q, "q", head_dim, size, false, 0));
  STATUS_TRY(check_output(q_out, "q_out", head_dim, size, false, q->n_heads, n_tokens));
  HeadNormArgs a = norm_args(rope, n_tokens, head_dim, positions, eps, gain_dtype, q_gain, k_gain, status);
  a.q = rope_view(q, q_out);
  if (k) {
    STATUS_TRY(check_view(k, "k", head_dim, size, false, 0));
    STATUS_TRY(check_output(k_out, "k_out", head_dim, size, false, k->n_heads, n_tokens));
    a.k = rope_view(k, k_out);
  }
  int sms = 0;
  STATUS_TRY(sm_count(&sms));
  return cuda_status(launch_head_norm(dtype, a, sms, static_cast<cudaStream_t>(cuda_stream)), "dopr_head_norm_rope");
}

dopr_status dopr_head_norm_rope_backward(const dopr_rope* rope, int32_t dtype, int32_t head_dim, int32_t n_tokens,
                                         const int32_t* positions, float eps, int32_t gain_dtype, const dopr_heads* dq_out,
                                         const dopr_heads* q, const void* q_gain, const dopr_heads* dq, float* dq_gain,
                                         const dopr_heads* dk_out, const dopr_heads* k, const void* k_gain, const dopr_heads* dk,
                                         float* dk_gain, void* workspace, int32_t* status, void* cuda_stream) {
  if (dtype < DOPR_F16 || dtype > DOPR_F32) return fail(DOPR_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (n_tokens < 0) return fail(DOPR_ERR_INVALID_ARG, "n_tokens is negative");
  STATUS_TRY(check_head_dim(head_dim));
  STATUS_TRY(check_norm(eps, gain_dtype, q_gain, k_gain));
  if (!k != !dk_out || !k != !dk) return fail(DOPR_ERR_INVALID_ARG, "dk_out, k and dk belong together");
  if (!k && dk_gain) return fail(DOPR_ERR_INVALID_ARG, "dk_gain without k");
  if ((dq_gain || dk_gain) && (!workspace || !aligned(workspace, 16)))
    return fail(DOPR_ERR_INVALID_ARG, "the gains' gradients need a workspace, 16-byte aligned");
  STATUS_TRY(check_words({rope ? positions : nullptr, status, dq_gain, dk_gain}));
  HeadNormArgs a = norm_args(rope, n_tokens, head_dim, positions, eps, gain_dtype, q_gain, k_gain, status);
  a.dq_gain = dq_gain;
  a.dk_gain = dk_gain;
  a.ws = static_cast<float*>(workspace);
  if (n_tokens > 0) {  // views of no rows have no data; the gains' gradients are zero then
    if (rope) STATUS_TRY(check_rope_use(rope, head_dim, positions));
    const int size = type_size(dtype);
    STATUS_TRY(check_view(q, "q", head_dim, size, false, 0));
    STATUS_TRY(check_view(dq_out, "dq_out", head_dim, size, false, q->n_heads));
    STATUS_TRY(check_output(dq, "dq", head_dim, size, false, q->n_heads, n_tokens));
    a.q = rope_view(dq_out, dq);
    a.qx = rope_view(q, nullptr);
    if (k) {
      STATUS_TRY(check_view(k, "k", head_dim, size, false, 0));
      STATUS_TRY(check_view(dk_out, "dk_out", head_dim, size, false, k->n_heads));
      STATUS_TRY(check_output(dk, "dk", head_dim, size, false, k->n_heads, n_tokens));
      a.k = rope_view(dk_out, dk);
      a.kx = rope_view(k, nullptr);
    }
  }
  int sms = 0;
  STATUS_TRY(sm_count(&sms));
  return cuda_status(launch_head_norm_backward(dtype, a, sms, static_cast<cudaStream_t>(cuda_stream)), "dopr_head_norm_rope_backward");
}

int64_t dopr_head_norm_rope_workspace(int32_t head_dim) {
  if (check_head_dim(head_dim) != DOPR_OK) return -1;
  return static_cast<int64_t>(HEAD_NORM_MAX_BLOCKS) * head_dim * static_cast<int64_t>(sizeof(float));
}

int64_t dopr_cache_4bit_pool_bytes(const dopr_cache_layout* layout) {
  if (check_layout(layout) != DOPR_OK) return -1;
  return layout->n_blocks * static_cast<int64_t>(layout->n_kv_heads) * pages4::page_bytes(layout->page, layout->head_dim);
}

dopr_status dopr_cache_append_4bit(const dopr_cache_layout* layout, const dopr_rope* rope, int32_t n_tokens,
                                   const int32_t* positions, const int64_t* slots, float eps, int32_t gain_dtype,
                                   const dopr_heads* q, const void* q_gain, const dopr_heads* q_out, const dopr_heads* k,
                                   const void* k_gain, const dopr_heads* v, void* k_pool, void* v_pool, int32_t* status,
                                   void* cuda_stream) {
  STATUS_TRY(check_layout(layout));
  if (n_tokens < 0) return fail(DOPR_ERR_INVALID_ARG, "n_tokens is negative");
  if (eps != 0.f) STATUS_TRY(check_norm(eps, gain_dtype, q_gain, k_gain));
  else if (q_gain || k_gain) return fail(DOPR_ERR_INVALID_ARG, "a gain without a norm (eps 0)");
  if (!q != !q_out) return fail(DOPR_ERR_INVALID_ARG, "q and q_out belong together");
  if (q && !rope && eps == 0.f) return fail(DOPR_ERR_INVALID_ARG, "q without a norm or a rotary table");
  if (n_tokens == 0) return DOPR_OK;  // views of no rows have no data
  if (!slots || !k_pool || !v_pool) return fail(DOPR_ERR_INVALID_ARG, "slots, k_pool or v_pool is NULL");
  if (!aligned(k_pool, 16) || !aligned(v_pool, 16)) return fail(DOPR_ERR_INVALID_ARG, "the pools must be 16-byte aligned");
  if (!aligned(slots, 8)) return fail(DOPR_ERR_INVALID_ARG, "slots must be 8-byte aligned");
  STATUS_TRY(check_words({rope ? positions : nullptr, status}));
  const int D = layout->head_dim;
  if (rope) {
    STATUS_TRY(check_rope_use(rope, D, positions));
    if (rope->cfg.rotary_dim % 16) return fail(DOPR_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16 (got %d)", rope->cfg.rotary_dim);
  }
  STATUS_TRY(check_view(k, "k", D, 2, true, layout->n_kv_heads));
  STATUS_TRY(check_view(v, "v", D, 2, true, layout->n_kv_heads));
  HeadNormArgs a = norm_args(rope, n_tokens, D, positions, eps, gain_dtype, q_gain, k_gain, status);
  if (q) {
    STATUS_TRY(check_view(q, "q", D, 2, true, 0));
    STATUS_TRY(check_output(q_out, "q_out", D, 2, true, q->n_heads, n_tokens));
    a.q = rope_view(q, q_out);
  }
  a.k = rope_view(k, nullptr);
  a.v = rope_view(v, nullptr);
  a.slots = slots;
  a.k_pool = static_cast<uint8_t*>(k_pool);
  a.v_pool = static_cast<uint8_t*>(v_pool);
  a.page = layout->page;
  a.n_slots = (int64_t)layout->n_blocks * layout->page;
  int sms = 0;
  STATUS_TRY(sm_count(&sms));
  return cuda_status(launch_append_4bit(layout->dtype, a, sms, static_cast<cudaStream_t>(cuda_stream)), "dopr_cache_append_4bit");
}

dopr_status dopr_cache_read_4bit(const dopr_cache_layout* layout, int32_t n_rows, const int64_t* slots, const void* k_pool,
                                 const void* v_pool, const dopr_heads* k_out, const dopr_heads* v_out, int32_t* status,
                                 void* cuda_stream) {
  STATUS_TRY(check_layout(layout));
  if (n_rows < 0) return fail(DOPR_ERR_INVALID_ARG, "n_rows is negative");
  if (n_rows == 0) return DOPR_OK;  // views of no rows have no data
  if (!slots || !k_pool || !v_pool) return fail(DOPR_ERR_INVALID_ARG, "slots, k_pool or v_pool is NULL");
  if (!aligned(k_pool, 16) || !aligned(v_pool, 16)) return fail(DOPR_ERR_INVALID_ARG, "the pools must be 16-byte aligned");
  if (!aligned(slots, 8)) return fail(DOPR_ERR_INVALID_ARG, "slots must be 8-byte aligned");
  STATUS_TRY(check_words({status}));
  const int D = layout->head_dim;
  STATUS_TRY(check_output(k_out, "k_out", D, 2, true, layout->n_kv_heads, n_rows));
  STATUS_TRY(check_output(v_out, "v_out", D, 2, true, layout->n_kv_heads, n_rows));
  Read4Args a{};
  a.n_rows = n_rows;
  a.head_dim = D;
  a.n_kv_heads = layout->n_kv_heads;
  a.page = layout->page;
  a.n_slots = (int64_t)layout->n_blocks * layout->page;
  a.slots = slots;
  a.k_pool = static_cast<const uint8_t*>(k_pool);
  a.v_pool = static_cast<const uint8_t*>(v_pool);
  a.k = rope_view(k_out, k_out);
  a.v = rope_view(v_out, v_out);
  a.status = status;
  int sms = 0;
  STATUS_TRY(sm_count(&sms));
  return cuda_status(launch_read_4bit(layout->dtype, a, sms, static_cast<cudaStream_t>(cuda_stream)), "dopr_cache_read_4bit");
}

dopr_status dopr_shared_attention_plan(const dopr_cache_layout* layout, int32_t n_q_heads, int32_t max_tokens,
                                       const int32_t* tok_off, const int32_t* seq_lens, const int32_t* prefix, void* plan,
                                       int32_t* status, void* cuda_stream) {
  STATUS_TRY(check_attention(layout, n_q_heads, max_tokens));
  if (!tok_off || !seq_lens || !plan) return fail(DOPR_ERR_INVALID_ARG, "tok_off, seq_lens or plan is NULL");
  if (!aligned(plan, 16)) return fail(DOPR_ERR_INVALID_ARG, "the plan must be 16-byte aligned");
  STATUS_TRY(check_words({tok_off, seq_lens, prefix, status}));
  SharedPlanArgs a{};
  a.lay = *layout;
  a.Hq = n_q_heads;
  a.max_tokens = max_tokens;
  a.tok_off = tok_off;
  a.seq_lens = seq_lens;
  a.prefix = prefix;
  a.plan = static_cast<int32_t*>(plan);
  a.status = status;
  int sms = 0;
  STATUS_TRY(sm_count(&sms));
  return cuda_status(launch_shared_plan(a, sms, static_cast<cudaStream_t>(cuda_stream)), "dopr_shared_attention_plan");
}

int64_t dopr_shared_attention_plan_bytes(const dopr_cache_layout* layout, int32_t n_q_heads, int32_t max_tokens) {
  if (check_attention(layout, n_q_heads, max_tokens) != DOPR_OK) return -1;
  return shared_plan_bytes(*layout, n_q_heads, max_tokens);
}

dopr_status dopr_shared_attention(const dopr_cache_layout* layout, const void* plan, int32_t max_tokens, const dopr_heads* q,
                                  const void* k_pool, const void* v_pool, const int32_t* block_tables, float scale,
                                  const dopr_heads* out, float* lse, void* workspace, int32_t* status, void* cuda_stream) {
  return attention(false, layout, plan, max_tokens, q, k_pool, v_pool, block_tables, scale, out, lse, workspace, status, cuda_stream);
}

dopr_status dopr_shared_attention_4bit(const dopr_cache_layout* layout, const void* plan, int32_t max_tokens, const dopr_heads* q,
                                       const void* k_pool, const void* v_pool, const int32_t* block_tables, float scale,
                                       const dopr_heads* out, float* lse, void* workspace, int32_t* status, void* cuda_stream) {
  return attention(true, layout, plan, max_tokens, q, k_pool, v_pool, block_tables, scale, out, lse, workspace, status, cuda_stream);
}

int64_t dopr_shared_attention_workspace(const dopr_cache_layout* layout, int32_t n_q_heads, int32_t max_tokens) {
  if (check_attention(layout, n_q_heads, max_tokens) != DOPR_OK) return -1;
  int sms = 0;
  if (sm_count(&sms) != DOPR_OK) return -1;
  return shared_workspace_bytes(*layout, n_q_heads, max_tokens, sms);
}

}  // extern "C"
