// C-ABI entry points of the token cache (include/grand.h, second half): argument checks, the workspace that is allocated at
// creation, and the choice of kernel.  Nothing here throws or synchronises (grand_cache_status excepted).
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>

#include "../../include/grand.h"
#include "grand_cache.h"

using namespace grand;

struct grand_cache {
  grand_cache_options o;
  int device;
  FastDiv page, group;
  uint32_t* status = nullptr;   // device word
  uint32_t* arrived = nullptr;  // join counters of the attend kernels, zero between calls
  float* partial = nullptr;     // their partial results
  unsigned long long launches = 0;
  char last_error[256] = "";
};

namespace {

int fail(const grand_cache* c, int code, const char* format, ...) {
  if (c) {
    va_list v;
    va_start(v, format);
    vsnprintf(const_cast<grand_cache*>(c)->last_error, sizeof c->last_error, format, v);
    va_end(v);
  }
  return code;
}
int done(const grand_cache* c, cudaError_t e, const char* what) {
  if (e == cudaSuccess) return GRAND_OK;
  cudaGetLastError();  // reported here, not by the caller's next call
  return fail(c, GRAND_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

void* cache_alloc(size_t bytes, void*) {
  void* p = nullptr;
  return cudaMalloc(&p, bytes) == cudaSuccess ? p : nullptr;
}
void cache_free(void* p, void*) { cudaFree(p); }

// The pool and the sequences of a call, checked as far as the host can see (`news`: the call reads new tokens).
int views(const grand_cache* c, const grand_pool* p, const grand_seqs* q, bool weights, bool news, PoolView* pool, SeqView* seq) {
  if (!p || !q) return fail(c, GRAND_ERR_INVALID_ARG, "pool or seqs is null");
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev != c->device) return fail(c, GRAND_ERR_INVALID_ARG, "the handle belongs to device %d, not to the current one", c->device);
  if (!p->k || !p->v || !aligned(p->k, 16) || !aligned(p->v, 16)) return fail(c, GRAND_ERR_INVALID_ARG, "k and v of the pool must be 16-byte aligned device arrays");
  if (p->page_stride % 8 || p->slot_stride % 8 || p->head_stride % 8 || p->page_stride < 0 || p->slot_stride < 0 || p->head_stride < 0)
    return fail(c, GRAND_ERR_INVALID_ARG, "the pool's strides must be multiples of 8 elements");
  if (weights && (!p->weights || c->o.weight_groups == 0)) return fail(c, GRAND_ERR_INVALID_ARG, "the cache keeps no weights");
  if (q->batch && (!q->page_table || !q->kv_lens)) return fail(c, GRAND_ERR_INVALID_ARG, "page_table or kv_lens is null");
  if (q->batch > c->o.max_batch) return fail(c, GRAND_ERR_CAPACITY, "%u sequences, max_batch is %u", q->batch, c->o.max_batch);
  if (news && q->tokens > c->o.max_tokens) return fail(c, GRAND_ERR_CAPACITY, "%u new tokens, max_tokens is %u", q->tokens, c->o.max_tokens);
  if (news && !q->cu_new && q->tokens != q->batch) return fail(c, GRAND_ERR_INVALID_ARG, "without cu_new every sequence has one new token");
  *pool = PoolView{static_cast<uint8_t*>(p->k), static_cast<uint8_t*>(p->v), c->o.weight_groups ? p->weights : nullptr,
                   p->page_stride, p->slot_stride, p->head_stride, (uint32_t)c->o.num_pages, c->page, c->o.kv_heads,
                   c->o.head_dim, c->o.weight_groups};
  const uint64_t most = (uint64_t)q->pages_per_seq * c->o.page_size;
  *seq = SeqView{q->page_table, q->kv_lens, news ? q->cu_new : nullptr, q->table_stride, (uint32_t)(most < (1ull << 30) ? most : 1ull << 30), q->batch, q->tokens};
  return GRAND_OK;
}

int check_rope(const grand_cache* c, uint32_t dim, uint32_t rot, const float* table, uint64_t rows, const int32_t* positions) {
  if (rot % 2 || rot > dim) return fail(c, GRAND_ERR_INVALID_ARG, "rot must be even and at most the head's size");
  if (rot && (!table || !positions || rows == 0)) return fail(c, GRAND_ERR_INVALID_ARG, "a rotation needs a table and positions");
  return GRAND_OK;
}

}  // namespace

namespace grand {
cudaError_t allow_dynamic_smem(const void* kernel, int bytes, SmemOptIn* done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  if (__atomic_load_n(&done->done[dev], __ATOMIC_ACQUIRE)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) __atomic_store_n(&done->done[dev], 1, __ATOMIC_RELEASE);
  return e;
}
}  // namespace grand

extern "C" {

int grand_cache_create(const grand_cache_options* opts, grand_cache** out) {
  if (!out) return GRAND_ERR_INVALID_ARG;
  *out = nullptr;
  if (!opts) return GRAND_ERR_INVALID_ARG;
  grand_cache_options o = *opts;
  if (!o.max_batch) o.max_batch = 256;
  if (!o.max_tokens) o.max_tokens = 8192;
  if (!o.dev_alloc) o.dev_alloc = cache_alloc, o.dev_free = cache_free;
  if (!o.q_heads || !o.kv_heads || o.q_heads % o.kv_heads || o.q_heads > 4096 || !o.page_size || o.page_size > (1u << 20) || !o.num_pages ||
      o.num_pages >= (1ull << 31) || (o.weight_groups > 1 && o.weight_groups != o.kv_heads) || o.max_batch > 4096 ||
      (uint64_t)o.max_tokens * o.q_heads >= (1ull << 31) || !o.dev_free)
    return GRAND_ERR_INVALID_ARG;
  if (o.dtype != GRAND_F16 && o.dtype != GRAND_BF16) return GRAND_ERR_UNSUPPORTED;
  if (!o.head_dim || o.head_dim % 8 || o.head_dim > 128) return GRAND_ERR_UNSUPPORTED;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return GRAND_ERR_CUDA;
  grand_cache* c = new (std::nothrow) grand_cache;
  if (!c) return GRAND_ERR_NOMEM;
  c->o = o;
  c->device = dev;
  c->page = make_div(o.page_size);
  c->group = make_div(o.q_heads / o.kv_heads);
  const uint64_t sms = (uint64_t)sm_count();
  // one block of memory: status word and 2 counters per SM (cleared), then the partial results (2 x 2 stream slots or 2
  // tensor-core slots per SM)
  const size_t head = ((1 + 2 * sms) * 4 + 255) / 256 * 256, slots = sms * 4 * std::max(2 * 2 * kStreamSlot, 2 * kTcSlot), bytes = head + slots;
  uint8_t* p = static_cast<uint8_t*>(o.dev_alloc(bytes, o.user));
  if (!p) {
    delete c;
    return GRAND_ERR_NOMEM;
  }
  c->status = reinterpret_cast<uint32_t*>(p);
  c->arrived = c->status + 1;
  c->partial = reinterpret_cast<float*>(p + head);
  if (cudaMemset(p, 0, head) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
    o.dev_free(p, o.user);
    delete c;
    return GRAND_ERR_CUDA;
  }
  *out = c;
  return GRAND_OK;
}

int grand_cache_destroy(grand_cache* c) {
  if (!c) return GRAND_OK;
  cudaDeviceSynchronize();
  c->o.dev_free(c->status, c->o.user);
  delete c;
  return GRAND_OK;
}

const char* grand_cache_last_error(const grand_cache* c) { return c ? c->last_error : ""; }

int grand_cache_status(grand_cache* c, uint32_t* bits, grand_stream stream) {
  if (!c || !bits) return GRAND_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  uint32_t v = 0;
  cudaError_t e = cudaMemcpyAsync(&v, c->status, 4, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaMemsetAsync(c->status, 0, 4, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  *bits = v;
  return done(c, e, "grand_cache_status");
}

int grand_cache_launches(const grand_cache* c, uint64_t* n) {
  if (!c || !n) return GRAND_ERR_INVALID_ARG;
  *n = c->launches;
  return GRAND_OK;
}

int grand_rope(const void* x, void* out, uint32_t dtype, uint64_t tokens, uint32_t heads, uint32_t dim, int64_t x_tok, int64_t x_head,
               int64_t o_tok, int64_t o_head, const float* table, uint64_t rows, uint32_t rot, const int32_t* positions,
               uint32_t interleaved, uint32_t inverse, grand_stream stream) {
  return grand_rope_checked(x, out, dtype, tokens, heads, dim, x_tok, x_head, o_tok, o_head, table, rows, rot, positions, interleaved,
                            inverse, nullptr, stream);
}

int grand_rope_checked(const void* x, void* out, uint32_t dtype, uint64_t tokens, uint32_t heads, uint32_t dim, int64_t x_tok, int64_t x_head,
                       int64_t o_tok, int64_t o_head, const float* table, uint64_t rows, uint32_t rot, const int32_t* positions,
                       uint32_t interleaved, uint32_t inverse, uint32_t* status, grand_stream stream) {
  if (dtype != GRAND_F32 && dtype != GRAND_F16 && dtype != GRAND_BF16) return GRAND_ERR_UNSUPPORTED;
  if (dim == 0 || dim > 256) return GRAND_ERR_UNSUPPORTED;
  if (rot % 2 || rot > dim) return GRAND_ERR_INVALID_ARG;
  if (tokens >= (1ull << 31) || heads > (1u << 20)) return GRAND_ERR_CAPACITY;
  if (tokens == 0 || heads == 0) return GRAND_OK;
  if (int rc = check_rope(nullptr, dim, rot, table, rows, positions)) return rc;
  if (!x || !out) return GRAND_ERR_INVALID_ARG;
  const uintptr_t size = dtype == GRAND_F32 ? 4 : 2;
  if (!aligned(x, size) || !aligned(out, size) || !aligned(table, 4) || !aligned(positions, 4) || !aligned(status, 4)) return GRAND_ERR_INVALID_ARG;
  RopeArgs a{x, out, x_tok, x_head, o_tok, o_head, heads, dim, tokens, table, rows, rot, positions, interleaved != 0, inverse ? -1.0f : 1.0f, status};
  return done(nullptr, launch_rope(a, dtype, static_cast<cudaStream_t>(stream)), "rope");
}

int grand_cache_append(grand_cache* c, const grand_pool* p, const grand_seqs* q, const void* x, void* x_out, const void* k, const void* v,
                       const int64_t* strides, const float* table, uint64_t rows, uint32_t rot, const int32_t* positions,
                       uint32_t interleaved, grand_stream stream) {
  if (!c) return GRAND_ERR_INVALID_ARG;
  AppendArgs a{};
  if (int rc = views(c, p, q, false, true, &a.pool, &a.seq)) return rc;
  if (rot % 2 || rot > c->o.head_dim) return fail(c, GRAND_ERR_INVALID_ARG, "rot must be even and at most the head's size");
  if (q->tokens == 0 || q->batch == 0) return GRAND_OK;
  if (int rc = check_rope(c, c->o.head_dim, rot, table, rows, positions)) return rc;
  if (!k || !v || !strides || (x && !x_out)) return fail(c, GRAND_ERR_INVALID_ARG, "k, v, q_out or strides is null");
  if (!aligned(x, 2) || !aligned(x_out, 2) || !aligned(k, 2) || !aligned(v, 2)) return fail(c, GRAND_ERR_INVALID_ARG, "misaligned elements");
  a.q = RopeArgs{x, x_out, strides[0], strides[1], (int64_t)c->o.q_heads * c->o.head_dim, c->o.head_dim, x ? c->o.q_heads : 0, c->o.head_dim,
                 q->tokens, table, rows, rot, positions, interleaved != 0, 1.0f, c->status};
  a.k = k; a.v = v;
  a.k_tok = strides[2]; a.k_head = strides[3]; a.v_tok = strides[4]; a.v_head = strides[5];
  LaunchScope scope(&c->launches);
  return done(c, launch_append(a, c->o.dtype, static_cast<cudaStream_t>(stream)), "append");
}

int grand_cache_attend(grand_cache* c, const grand_pool* p, const grand_seqs* s, const void* q, int64_t q_tok, int64_t q_head, float scale,
                       uint32_t causal, uint32_t window, void* out, float* lse, grand_stream stream) {
  if (!c) return GRAND_ERR_INVALID_ARG;
  AttendArgs a{};
  if (int rc = views(c, p, s, false, true, &a.pool, &a.seq)) return rc;
  if (window && !causal) return fail(c, GRAND_ERR_INVALID_ARG, "a window needs causal attention");
  // (times log2(e) it has to be a finite float)
  if (!(std::fabs(scale) <= 2.0e38f)) return fail(c, GRAND_ERR_INVALID_ARG, "scale must be at most 2e38");
  if (s->tokens == 0 || s->batch == 0) return GRAND_OK;
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || q_tok % 8 || q_head % 8)
    return fail(c, GRAND_ERR_INVALID_ARG, "q and out must be 16-byte aligned, q's strides multiples of 8");
  a.q = q; a.q_tok = q_tok; a.q_head = q_head;
  a.group = c->group;
  a.scale_log2 = (float)((double)scale * 1.4426950408889634);
  a.causal = causal != 0;
  a.window = window < (1u << 30) ? window : 0;  // (as wide as any sequence: no window)
  a.out = out; a.lse = lse;
  a.partial = c->partial; a.arrived = c->arrived;
  a.status = c->status;
  LaunchScope scope(&c->launches);
  // The streaming kernel reads the keys once per 32 rows of a kv head; with more rows than that the tensor-core kernel,
  // which takes 256, is the faster one.
  const bool many = (uint64_t)s->tokens * c->group.d > (uint64_t)s->batch * 32;
  return done(c, (many ? launch_attend_tc : launch_attend_stream)(a, c->o.dtype, static_cast<cudaStream_t>(stream)), "attend");
}

int grand_cache_weigh(grand_cache* c, const grand_pool* p, const grand_seqs* s, const void* q, int64_t q_tok, int64_t q_head, const float* lse,
                      float scale, uint32_t causal, uint32_t window, float decay, grand_stream stream) {
  if (!c) return GRAND_ERR_INVALID_ARG;
  WeighArgs a{};
  if (int rc = views(c, p, s, true, true, &a.pool, &a.seq)) return rc;
  if (window && !causal) return fail(c, GRAND_ERR_INVALID_ARG, "a window needs causal attention");
  if (!(std::fabs(scale) <= 2.0e38f) || !(std::fabs(decay) <= 3.0e38f)) return fail(c, GRAND_ERR_INVALID_ARG, "scale must be at most 2e38, decay finite");
  if (s->batch == 0) return GRAND_OK;
  if (s->tokens && (!q || !lse || !aligned(q, 16) || q_tok % 8 || q_head % 8))
    return fail(c, GRAND_ERR_INVALID_ARG, "q must be 16-byte aligned with strides that are multiples of 8, lse given");
  a.q = q; a.q_tok = q_tok; a.q_head = q_head;
  a.group = c->group;
  a.lse = lse;
  a.scale_log2 = (float)((double)scale * 1.4426950408889634);
  a.decay = decay;
  a.causal = causal != 0;
  a.window = window < (1u << 30) ? window : 0;
  a.status = c->status;
  LaunchScope scope(&c->launches);
  a.partial = c->partial; a.arrived = c->arrived;
  // The streaming kernel reads the keys once per 32 rows of a kv head, the tensor-core kernel once.
  const bool many = (uint64_t)s->tokens * c->group.d > (uint64_t)s->batch * 32 && c->group.d <= 128;
  return done(c, (many ? launch_weigh_tc : launch_weigh_stream)(a, c->o.dtype, static_cast<cudaStream_t>(stream)), "weigh");
}

int grand_cache_evict(grand_cache* c, const grand_pool* p, const grand_seqs* s, uint32_t keep, uint32_t sinks, uint32_t recent,
                      const int32_t* into, int64_t into_stride, uint32_t into_pages, int32_t* kept, int32_t* lens_out, grand_stream stream) {
  if (!c) return GRAND_ERR_INVALID_ARG;
  if (!s) return fail(c, GRAND_ERR_INVALID_ARG, "seqs is null");
  EvictArgs a{};
  if (int rc = views(c, p, s, true, false, &a.pool, &a.seq)) return rc;
  if (keep == 0 || keep > 0x3FFFFFFFu || (uint64_t)sinks + recent > keep) return fail(c, GRAND_ERR_INVALID_ARG, "keep must be at least 1 and at least sinks + recent");
  if (into && (uint64_t)into_pages * c->o.page_size < keep) return fail(c, GRAND_ERR_INVALID_ARG, "the pages of `into` hold less than `keep` tokens");
  if (s->batch == 0) return GRAND_OK;
  if (!kept || !lens_out) return fail(c, GRAND_ERR_INVALID_ARG, "kept_out or lens_out is null");
  // (lengths are read while others are written)
  if (lens_out < s->kv_lens + s->batch && s->kv_lens < lens_out + s->batch) return fail(c, GRAND_ERR_INVALID_ARG, "lens_out must not be kv_lens");
  a.keep = keep; a.sinks = sinks; a.recent = recent;
  a.into = into; a.into_stride = into_stride;
  a.kept = kept; a.lens_out = lens_out;
  a.status = c->status;
  LaunchScope scope(&c->launches);
  return done(c, launch_evict(a, static_cast<cudaStream_t>(stream)), "evict");
}

}  // extern "C"
