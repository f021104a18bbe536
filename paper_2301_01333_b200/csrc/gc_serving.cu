// Host side of the operators of a served attention block (include/gc.h): checks of arguments, tensor maps, launches.
// Nothing is kept between calls.
#include <cmath>
#include <cstdio>

#include "ptx.cuh"
#include "serving.cuh"

using namespace gc;

gc_status_t gc_set_error(gc_status_t st, const char* msg);                                       // gc_api.cu
gc_status_t gc_make_tmap_heads(CUtensorMap* m, const void* ptr, uint64_t inner, uint64_t heads, uint64_t tokens,
                               uint64_t head_stride_bytes, uint64_t token_stride_bytes, uint32_t box_inner, uint32_t box_tokens);

#define REFUSE(status, ...)                        \
  do {                                             \
    char msg__[256];                               \
    snprintf(msg__, sizeof(msg__), __VA_ARGS__);   \
    return gc_set_error(status, msg__);            \
  } while (0)
#define RUN(expr)                                                                          \
  do {                                                                                     \
    cudaError_t e__ = (expr);                                                              \
    if (e__ != cudaSuccess) return gc_set_error(GC_ERR_CUDA, cudaGetErrorString(e__));     \
  } while (0)

namespace {
bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

// The device of the descriptor for the length of a call; the thread's own afterwards.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    err_ = cudaGetDevice(&before_);
    if (err_ == cudaSuccess && before_ != device) {
      err_ = cudaSetDevice(device);
      moved_ = err_ == cudaSuccess;
    }
  }
  ~OnDevice() {
    if (moved_) cudaSetDevice(before_);
  }
  cudaError_t err() const { return err_; }

 private:
  int before_ = 0;
  bool moved_ = false;
  cudaError_t err_;
};

cudaError_t sm_count(int device, int* n) { return cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, device); }

gc_status_t check_heads(const char* who, const char* name, const gc_heads_t& h, int esz, bool strict) {
  if (!h.data) REFUSE(GC_ERR_INVALID_ARG, "%s: %s is null", who, name);
  if (misaligned(h.data, esz)) REFUSE(GC_ERR_ALIGNMENT, "%s: %s is not aligned to its element size", who, name);
  if (h.token_stride < 0 || h.head_stride < 0) REFUSE(GC_ERR_SHAPE, "%s: %s has a negative stride", who, name);
  if (strict && (misaligned(h.data, 16) || h.token_stride % 8 || h.head_stride % 8))
    REFUSE(GC_ERR_ALIGNMENT, "%s: %s needs 16-byte aligned rows", who, name);
  return GC_OK;
}

gc_status_t check_cache(const char* who, const gc_kv4_cache_t* c) {
  if (!c) REFUSE(GC_ERR_INVALID_ARG, "%s: null cache", who);
  if (!c->k_codes || !c->k_params || !c->v_codes || !c->v_params) REFUSE(GC_ERR_INVALID_ARG, "%s: the cache has a null array", who);
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128)
    REFUSE(GC_ERR_UNSUPPORTED, "%s: head_dim %d (64, 96 or 128)", who, c->head_dim);
  if ((c->group != 32 && c->group != 64 && c->group != 128) || c->head_dim % c->group)
    REFUSE(GC_ERR_UNSUPPORTED, "%s: group %d (32, 64 or 128, a divisor of head_dim)", who, c->group);
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
    REFUSE(GC_ERR_UNSUPPORTED, "%s: page_size %d (a power of two, 16 to 256)", who, c->page_size);
  if (c->num_pages < 1 || c->kv_heads < 1) REFUSE(GC_ERR_SHAPE, "%s: the cache has no pages or no heads", who);
  if (c->num_pages > 0x7FFFFFFFLL || c->kv_heads > 65535) REFUSE(GC_ERR_UNSUPPORTED, "%s: too many pages or heads", who);
  if (misaligned(c->k_codes, 16) || misaligned(c->k_params, 16) || misaligned(c->v_codes, 16) || misaligned(c->v_params, 16))
    REFUSE(GC_ERR_ALIGNMENT, "%s: the arrays of the cache must be 16-byte aligned", who);
  if (misaligned(c->status, 4)) REFUSE(GC_ERR_ALIGNMENT, "%s: the status word must be 4-byte aligned", who);
  return GC_OK;
}

gc_status_t check_rows(const char* who, const gc_kv4_cache_t* c, int dtype, int64_t tokens, const gc_heads_t* k, const gc_heads_t* v,
                       const int64_t* slots) {
  gc_status_t st = check_cache(who, c);
  if (st != GC_OK) return st;
  if (dtype != GC_F32 && dtype != GC_BF16) REFUSE(GC_ERR_UNSUPPORTED, "%s: rows are fp32 or bf16", who);
  if (tokens < 0) REFUSE(GC_ERR_SHAPE, "%s: negative number of tokens", who);
  if (tokens == 0) return GC_OK;
  if (!k || !v || !slots) REFUSE(GC_ERR_INVALID_ARG, "%s: null argument", who);
  if (misaligned(slots, 8)) REFUSE(GC_ERR_ALIGNMENT, "%s: slots must be 8-byte aligned", who);
  const int esz = dtype == GC_F32 ? 4 : 2;
  if ((st = check_heads(who, "k", *k, esz, false)) != GC_OK) return st;
  if ((st = check_heads(who, "v", *v, esz, false)) != GC_OK) return st;
  if (tokens > 0x7FFFFFFFLL / c->kv_heads) REFUSE(GC_ERR_UNSUPPORTED, "%s: too many rows for one launch", who);
  return GC_OK;
}

// How one call of gc_attention_kv4 is laid out over the GPU.
struct Layout {
  int cols, col_chunks, block, ctas, solo;
  size_t bytes;
};

gc_status_t check_attend(const char* who, const gc_kv4_cache_t* c, const gc_attention_kv4_t* d) {
  gc_status_t st = check_cache(who, c);
  if (st != GC_OK) return st;
  if (!d) REFUSE(GC_ERR_INVALID_ARG, "%s: null argument", who);
  if (d->batch < 0 || d->q_heads < 1 || d->q_heads % c->kv_heads)
    REFUSE(GC_ERR_SHAPE, "%s: %d query heads over %d key/value heads", who, d->q_heads, c->kv_heads);
  if (d->queries < 1 || d->queries > 16) REFUSE(GC_ERR_UNSUPPORTED, "%s: %d queries per sequence (1 to 16)", who, d->queries);
  if (d->q_heads / c->kv_heads > 256) REFUSE(GC_ERR_UNSUPPORTED, "%s: more than 256 query heads share a key/value head", who);
  if (!(d->scale > 0.f) || !std::isfinite(d->scale)) REFUSE(GC_ERR_INVALID_ARG, "%s: scale must be finite and positive", who);
  if (d->max_length < 0 || d->table_width < 0 || d->table_stride < 0) REFUSE(GC_ERR_SHAPE, "%s: negative length or table size", who);
  if (d->max_length > static_cast<int64_t>(d->table_width) * c->page_size)
    REFUSE(GC_ERR_SHAPE, "%s: max_length %d exceeds table_width %d pages of %d", who, d->max_length, d->table_width, c->page_size);
  if (d->max_length > 0x7FFFFFFF - 65536) REFUSE(GC_ERR_UNSUPPORTED, "%s: max_length too large", who);
  if (static_cast<int64_t>(d->batch) * c->kv_heads > (1 << 22)) REFUSE(GC_ERR_UNSUPPORTED, "%s: batch times heads too large", who);
  if (static_cast<int64_t>(d->batch) * d->queries * d->q_heads > 0x7FFFFFFF)
    REFUSE(GC_ERR_UNSUPPORTED, "%s: batch times queries times heads too large", who);
  return GC_OK;
}

// One wave of CTAs, as many as fit, or one per 128 tokens where there are fewer.  Sequences of up to 512 tokens are not split:
// joining their pieces would take another launch, longer than the three blocks it would save.  Where there are more units of
// work (sequence, head, chunk of columns) than CTAs fit, or a unit is a single tile, a warp takes a unit alone: what such a unit
// costs is its chain of latencies, of which four times as many then overlap, and no warps have to be joined.  64 tokens, 120
// sequences of 8 heads: 7.6 us against 14.0; 225 tokens, 8 queries of 64 heads on 4, 120 sequences: 65 against 135; 512
// tokens, 200 sequences: 28 against 37; but 40 sequences of 512, fewer than fit: 16 against 11.  Up to 1024 tokens from three
// times that many on (1000 tokens, 200 sequences: 50 against 61; 120 of them: 44 against 40): a long sequence among many
// short ones is one warp's work.
Layout lay_out(const gc_kv4_cache_t& c, const gc_attention_kv4_t& d, int num_sms) {
  Layout s = {};
  const int columns = d.queries * (d.q_heads / c.kv_heads);
  s.cols = attn_kv4_cols(columns);
  s.col_chunks = (columns + s.cols - 1) / s.cols;
  const int64_t units = static_cast<int64_t>(d.batch) * c.kv_heads * s.col_chunks;
  const int64_t fit = static_cast<int64_t>(num_sms) * attn_kv4_resident(c.head_dim, c.group, s.cols);
  s.solo = d.max_length <= 32 || units > (d.max_length <= 512 ? fit : d.max_length <= 1024 ? 3 * fit : INT64_MAX);
  s.block = s.solo || d.max_length <= 512 ? 1024 : 128;
  const int64_t most = units * ((static_cast<int64_t>(d.max_length) + s.block - 1) / s.block);
  // (without splitting, a CTA per unit, and the hardware deals them out)
  s.ctas = static_cast<int>(s.solo ? (units + 3) / 4 : s.block >= d.max_length ? units : most < fit ? most : fit);
  // two pieces a CTA (outputs, maximum and sum of every column), and which they are
  s.bytes = s.block >= d.max_length || s.ctas == 1 ? 0 : s.ctas * (2 * static_cast<size_t>(s.cols) * (c.head_dim + 2) * sizeof(float) + 8);
  return s;
}
}  // namespace

extern "C" gc_status_t gc_qk_norm_rope(void* cuda_stream, const gc_qk_norm_rope_t* d) {
  const char* who = "gc_qk_norm_rope";
  if (!d) REFUSE(GC_ERR_INVALID_ARG, "%s: null argument", who);
  if (d->dtype != GC_F32 && d->dtype != GC_BF16) REFUSE(GC_ERR_UNSUPPORTED, "%s: fp32 or bf16", who);
  if (d->tokens < 0 || d->q_heads < 0 || d->k_heads < 0) REFUSE(GC_ERR_SHAPE, "%s: negative size", who);
  if (d->head_dim < 2 || d->head_dim > 256 || d->head_dim % 2) REFUSE(GC_ERR_UNSUPPORTED, "%s: head_dim %d (even, 2 to 256)", who, d->head_dim);
  if (d->rot_dim < 0 || d->rot_dim > d->head_dim || d->rot_dim % 2)
    REFUSE(GC_ERR_SHAPE, "%s: rot_dim %d (even, 0 to head_dim)", who, d->rot_dim);
  if (!(d->eps >= 0.f) || !std::isfinite(d->eps) || !std::isfinite(d->attention_factor))
    REFUSE(GC_ERR_INVALID_ARG, "%s: eps must be finite and not negative, attention_factor finite", who);
  if (d->q_heads > 4096 || d->k_heads > 4096) REFUSE(GC_ERR_UNSUPPORTED, "%s: more than 4096 heads", who);
  if (d->tokens == 0 || d->q_heads + d->k_heads == 0) return GC_OK;
  if (d->tokens > 0x7FFFFFFFLL) REFUSE(GC_ERR_UNSUPPORTED, "%s: too many tokens for one launch", who);
  const int esz = d->dtype == GC_F32 ? 4 : 2;
  gc_status_t st;
  if (d->q_heads && ((st = check_heads(who, "q", d->q, esz, false)) != GC_OK || (st = check_heads(who, "q_out", d->q_out, esz, false)) != GC_OK))
    return st;
  if (d->k_heads && ((st = check_heads(who, "k", d->k, esz, false)) != GC_OK || (st = check_heads(who, "k_out", d->k_out, esz, false)) != GC_OK))
    return st;
  if (d->rot_dim && (!d->positions || !d->inv_freq)) REFUSE(GC_ERR_INVALID_ARG, "%s: positions and inv_freq are needed to rotate", who);
  if (misaligned(d->positions, 8) || misaligned(d->inv_freq, 4) || misaligned(d->q_weight, esz) || misaligned(d->k_weight, esz))
    REFUSE(GC_ERR_ALIGNMENT, "%s: an array is not aligned to its element size", who);
  OnDevice on(d->cuda_device);
  RUN(on.err());
  int sms = 0;
  RUN(sm_count(d->cuda_device, &sms));
  RUN(launch_qk_norm_rope(*d, sms, static_cast<cudaStream_t>(cuda_stream)));
  return GC_OK;
}

extern "C" gc_status_t gc_kv4_append(void* cuda_stream, const gc_kv4_cache_t* cache, int32_t dtype, int64_t tokens, const gc_heads_t* k,
                                     const gc_heads_t* v, const int64_t* slots) {
  gc_status_t st = check_rows("gc_kv4_append", cache, dtype, tokens, k, v, slots);
  if (st != GC_OK || tokens == 0) return st;
  OnDevice on(cache->cuda_device);
  RUN(on.err());
  RUN(launch_kv4_append(*cache, dtype, tokens, *k, *v, slots, static_cast<cudaStream_t>(cuda_stream)));
  return GC_OK;
}

extern "C" gc_status_t gc_kv4_read(void* cuda_stream, const gc_kv4_cache_t* cache, int32_t dtype, int64_t tokens, const gc_heads_t* k,
                                   const gc_heads_t* v, const int64_t* slots) {
  gc_status_t st = check_rows("gc_kv4_read", cache, dtype, tokens, k, v, slots);
  if (st != GC_OK || tokens == 0) return st;
  OnDevice on(cache->cuda_device);
  RUN(on.err());
  RUN(launch_kv4_read(*cache, dtype, tokens, *k, *v, slots, static_cast<cudaStream_t>(cuda_stream)));
  return GC_OK;
}

extern "C" gc_status_t gc_attention_kv4_workspace_bytes(const gc_kv4_cache_t* cache, const gc_attention_kv4_t* d, size_t* bytes) {
  const char* who = "gc_attention_kv4_workspace_bytes";
  if (!bytes) REFUSE(GC_ERR_INVALID_ARG, "%s: null argument", who);
  gc_status_t st = check_attend(who, cache, d);
  if (st != GC_OK) return st;
  int sms = 0;
  RUN(sm_count(cache->cuda_device, &sms));
  *bytes = lay_out(*cache, *d, sms).bytes;
  return GC_OK;
}

extern "C" gc_status_t gc_attention_kv4(void* cuda_stream, const gc_kv4_cache_t* cache, const gc_attention_kv4_t* d, void* workspace_dev,
                                        size_t workspace_bytes) {
  const char* who = "gc_attention_kv4";
  gc_status_t st = check_attend(who, cache, d);
  if (st != GC_OK) return st;
  if (d->batch == 0) return GC_OK;
  if (!d->q || !d->out || !d->lengths || (d->max_length && !d->block_table)) REFUSE(GC_ERR_INVALID_ARG, "%s: null argument", who);
  if (misaligned(d->block_table, 4) || misaligned(d->lengths, 4)) REFUSE(GC_ERR_ALIGNMENT, "%s: block_table and lengths must be 4-byte aligned", who);
  const int64_t strides[6] = {d->q_batch_stride, d->q_query_stride, d->q_head_stride, d->o_batch_stride, d->o_query_stride, d->o_head_stride};
  for (int64_t s : strides) {
    if (s < 0) REFUSE(GC_ERR_SHAPE, "%s: negative stride", who);
    if (s % 8) REFUSE(GC_ERR_ALIGNMENT, "%s: q and out need 16-byte aligned rows", who);
  }
  if (misaligned(d->q, 16) || misaligned(d->out, 16)) REFUSE(GC_ERR_ALIGNMENT, "%s: q and out need 16-byte aligned rows", who);
  OnDevice on(cache->cuda_device);
  RUN(on.err());
  int sms = 0;
  RUN(sm_count(cache->cuda_device, &sms));
  const Layout sp = lay_out(*cache, *d, sms);
  if (sp.bytes) {
    if (!workspace_dev || workspace_bytes < sp.bytes) REFUSE(GC_ERR_INVALID_ARG, "%s: the workspace must have %zu bytes", who, sp.bytes);
    if (misaligned(workspace_dev, 16)) REFUSE(GC_ERR_ALIGNMENT, "%s: the workspace must be 16-byte aligned", who);
  }
  Kv4AttnParams p = {};
  p.B = d->batch; p.n = d->queries; p.Hq = d->q_heads; p.Hk = cache->kv_heads; p.g = d->q_heads / cache->kv_heads;
  while ((1 << p.page_shift) < cache->page_size) ++p.page_shift;
  p.max_len = d->max_length;
  p.num_pages = cache->num_pages; p.table_stride = d->table_stride;
  p.c = d->scale * 1.4426950408889634f;
  p.block = sp.block; p.ctas = sp.ctas; p.col_chunks = sp.col_chunks; p.solo = sp.solo;
  p.q = static_cast<const __nv_bfloat16*>(d->q);
  p.qb = d->q_batch_stride; p.qn = d->q_query_stride; p.qh = d->q_head_stride;
  p.o = static_cast<__nv_bfloat16*>(d->out);
  p.ob = d->o_batch_stride; p.on = d->o_query_stride; p.oh = d->o_head_stride;
  p.table = d->block_table; p.lengths = d->lengths;
  p.k_codes = static_cast<const uint8_t*>(cache->k_codes); p.k_params = static_cast<const uint32_t*>(cache->k_params);
  p.v_codes = static_cast<const uint8_t*>(cache->v_codes); p.v_params = static_cast<const uint32_t*>(cache->v_params);
  p.ws = static_cast<float*>(workspace_dev);
  p.status = cache->status;
  RUN(launch_attn_kv4(p, cache->head_dim, cache->group, static_cast<cudaStream_t>(cuda_stream)));
  return GC_OK;
}

extern "C" gc_status_t gc_attention_prompt(void* cuda_stream, const gc_attention_prompt_t* d) {
  const char* who = "gc_attention_prompt";
  if (!d) REFUSE(GC_ERR_INVALID_ARG, "%s: null argument", who);
  if (d->head_dim != 64 && d->head_dim != 96 && d->head_dim != 128) REFUSE(GC_ERR_UNSUPPORTED, "%s: head_dim %d (64, 96 or 128)", who, d->head_dim);
  if (d->batch < 0 || d->q_tokens < 0 || d->k_tokens < 0) REFUSE(GC_ERR_SHAPE, "%s: negative size", who);
  if (d->q_heads < 1 || d->kv_heads < 1 || d->q_heads % d->kv_heads)
    REFUSE(GC_ERR_SHAPE, "%s: %d query heads over %d key/value heads", who, d->q_heads, d->kv_heads);
  if (d->q_heads > 4096) REFUSE(GC_ERR_UNSUPPORTED, "%s: more than 4096 heads", who);
  if (!(d->scale > 0.f) || !std::isfinite(d->scale)) REFUSE(GC_ERR_INVALID_ARG, "%s: scale must be finite and positive", who);
  if (d->q_tokens > (1LL << 28) || d->k_tokens > (1LL << 28) || d->batch > (1 << 20))
    REFUSE(GC_ERR_UNSUPPORTED, "%s: too many tokens or sequences", who);
  if (d->batch == 0 || d->q_tokens == 0) return GC_OK;
  gc_status_t st;
  if ((st = check_heads(who, "q", d->q, 2, true)) != GC_OK || (st = check_heads(who, "out", d->out, 2, true)) != GC_OK) return st;
  if (d->k_tokens && ((st = check_heads(who, "k", d->k, 2, true)) != GC_OK || (st = check_heads(who, "v", d->v, 2, true)) != GC_OK)) return st;
  if (!d->cu_q || !d->cu_k) REFUSE(GC_ERR_INVALID_ARG, "%s: null sequence offsets", who);
  if (misaligned(d->cu_q, 4) || misaligned(d->cu_k, 4) || misaligned(d->status, 4))
    REFUSE(GC_ERR_ALIGNMENT, "%s: sequence offsets and the status word must be 4-byte aligned", who);
  OnDevice on(d->cuda_device);
  RUN(on.err());
  int sms = 0;
  RUN(sm_count(d->cuda_device, &sms));
  CUtensorMap tm[3];
  const gc_heads_t* src[3] = {&d->q, d->k_tokens ? &d->k : &d->q, d->k_tokens ? &d->v : &d->q};
  for (int i = 0; i < 3; ++i) {
    const uint64_t heads = src[i] == &d->q ? d->q_heads : d->kv_heads, tokens = src[i] == &d->q ? d->q_tokens : d->k_tokens;
    // the stride of an axis of one element is never used: any valid one
    const uint64_t hs = heads == 1 ? d->head_dim : src[i]->head_stride, ts = tokens == 1 ? heads * d->head_dim : src[i]->token_stride;
    if (hs == 0 || ts == 0) REFUSE(GC_ERR_UNSUPPORTED, "%s: q, k and v need strides other than 0", who);
    st = gc_make_tmap_heads(&tm[i], src[i]->data, d->head_dim, heads, tokens, hs * 2, ts * 2, 64, 128);
    if (st != GC_OK) return st;
  }
  PromptParams p = {};
  p.B = d->batch; p.Hq = d->q_heads; p.Hk = d->kv_heads; p.D = d->head_dim; p.causal = d->causal;
  p.q_tokens = d->q_tokens; p.k_tokens = d->k_tokens;
  p.c = d->scale * 1.4426950408889634f;
  p.o = static_cast<__nv_bfloat16*>(d->out.data);
  p.o_tok = d->out.token_stride; p.o_head = d->out.head_stride;
  p.cu_q = d->cu_q; p.cu_k = d->cu_k; p.status = d->status;
  RUN(launch_attn_prompt(tm[0], tm[1], tm[2], p, sms, static_cast<cudaStream_t>(cuda_stream)));
  return GC_OK;
}

extern "C" gc_status_t gc_serving_status(void* cuda_stream, uint32_t* status_dev) {
  if (!status_dev) return gc_set_error(GC_ERR_INVALID_ARG, "gc_serving_status: null argument");
  if (misaligned(status_dev, 4)) return gc_set_error(GC_ERR_ALIGNMENT, "gc_serving_status: the status word must be 4-byte aligned");
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  uint32_t word = 0;
  RUN(cudaMemcpyAsync(&word, status_dev, sizeof(word), cudaMemcpyDeviceToHost, s));
  RUN(cudaStreamSynchronize(s));
  if (word == 0) return GC_OK;
  RUN(cudaMemsetAsync(status_dev, 0, sizeof(word), s));
  RUN(cudaStreamSynchronize(s));
  switch (word) {
    case DEV_BAD_SLOT: return gc_set_error(GC_ERR_INVALID_ARG, "a slot lies outside the cache");
    case DEV_BAD_PAGE: return gc_set_error(GC_ERR_INVALID_ARG, "a page number in the block table lies outside the cache");
    case DEV_BAD_LENGTH: return gc_set_error(GC_ERR_INVALID_ARG, "a sequence is longer than max_length, or its length is negative");
    case DEV_BAD_OFFSETS: return gc_set_error(GC_ERR_INVALID_ARG, "sequence offsets decrease or leave the packed tokens");
    case DEV_LARGE_VALUE: return gc_set_error(GC_ERR_INVALID_ARG, "a value in the cache exceeds 2^32 in size, more than attention over it can sum");
    case DEV_LARGE_SCORE: return gc_set_error(GC_ERR_INVALID_ARG, "an attention score exceeds 2^26 in size, more than its weights can be taken from");
    default: break;
  }
  REFUSE(GC_ERR_TIMEOUT, "a device-side wait expired (code 0x%x)", word);
}
