// Host side of the paged cache and of the rotary positions: argument checks, the handle, the C ABI.
#include <math.h>
#include <string.h>

#include <mutex>
#include <new>

#include "xkv_paged_internal.cuh"

using namespace xkv;

namespace {

constexpr int kMaxDevices = 64;
constexpr int kMaxHeads = 64;
constexpr int64_t kMaxStride = (int64_t)1 << 38;       // elements; a tensor map's strides stay below 2^40 bytes

// Per device, on first use with that device current: the number of multiprocessors and the kernels' attributes.
std::mutex g_setup_mutex;
int g_sm_count[kMaxDevices] = {0};

int device_setup(int* device, int* sm_count) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return XKV_E_CUDA;
  if (dev < 0 || dev >= kMaxDevices) return XKV_E_UNSUPPORTED;
  std::lock_guard<std::mutex> lock(g_setup_mutex);
  if (g_sm_count[dev] == 0) {
    int sms = 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return XKV_E_CUDA;
    if (evict_device_setup() != cudaSuccess || attn_few_setup() != cudaSuccess || attn_chunk_setup() != cudaSuccess ||
        weights_setup() != cudaSuccess) return XKV_E_CUDA;
    g_sm_count[dev] = sms;
  }
  *device = dev;
  *sm_count = g_sm_count[dev];
  return XKV_OK;
}

bool aligned(const void* p, size_t a) { return p && (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool stride_ok(int64_t s) { return s > 0 && s % 8 == 0 && s < kMaxStride; }
bool rows_ok(const xkv_rows& r) { return aligned(r.data, 16) && stride_ok(r.tok_stride) && stride_ok(r.head_stride); }
// An output may be its input.
bool in_place_ok(const xkv_rows& in, const xkv_rows& out) {
  return in.data != out.data || (in.tok_stride == out.tok_stride && in.head_stride == out.head_stride);
}

int log2_of(int x) {
  int l = 0;
  while ((1 << l) < x) ++l;
  return l;
}

bool params_ok(const xkv_paged_params* p) {
  if (!p || p->reserved != 0) return false;
  if (p->n_kv_heads < 1 || p->n_kv_heads > kMaxHeads || p->n_heads < 1 || p->n_heads > kMaxHeads || p->n_heads % p->n_kv_heads) return false;
  if (p->head_dim != 64 && p->head_dim != 128) return false;
  if (p->dtype != XKV_BF16 && p->dtype != XKV_FP16) return false;
  if (p->page_tokens < 16 || p->page_tokens > 256 || (p->page_tokens & (p->page_tokens - 1))) return false;
  if (p->n_pages < 1 || p->max_seqs < 1 || p->max_seqs > kMaxSeqs) return false;
  if (!stride_ok(p->page_stride) || !stride_ok(p->head_stride) || !stride_ok(p->slot_stride)) return false;
  return p->slot_stride >= p->head_dim;
}

// Workspace: the status word, then the scratch of attention for one block per multiprocessor (arrival counts, marks of sequences, running
// maxima and sums, accumulators: two partial results per block).
struct Layout { size_t off_count, off_again, off_cuts, off_ml, off_o, total; };
Layout make_layout(const xkv_paged_params* p, int sms) {
  Layout l;
  size_t off = 256;
  auto take = [&](size_t bytes) { const size_t o = off; off += (bytes + 255) / 256 * 256; return o; };
  l.off_count = take((size_t)sms * sizeof(unsigned int));
  l.off_again = take((size_t)(2 + p->max_seqs) * sizeof(unsigned int));
  l.off_cuts = take((size_t)sms * attn_chunk_cut_bytes());
  l.off_ml = take((size_t)2 * sms * kChunkRows * sizeof(float2));
  l.off_o = take((size_t)2 * sms * kChunkRows * p->head_dim * sizeof(float));
  l.total = off;
  return l;
}

// Most units of work that the device's numbers could amount to, for counters of 32 bits.
bool work_ok(const xkv_paged* c, const xkv_paged_batch* b) {
  const int64_t units = (int64_t)b->table_width * c->p.page_tokens / 128 + 2;
  const int64_t tiles = (int64_t)b->max_new * c->view.group / (kChunkRows / 2) + 2;
  return (double)b->n_seqs * c->p.n_kv_heads * (double)(units + 2) * (double)tiles < 4294967296.0;
}

bool batch_ok(const xkv_paged* c, const xkv_paged_batch* b, bool tokens) {
  if (!b || b->n_seqs < 1 || b->n_seqs > c->p.max_seqs || b->table_width < 0) return false;
  if ((int64_t)b->table_width * c->p.page_tokens >= ((int64_t)1 << 31) - (1 << 16)) return false;
  if (!aligned(b->lens, 4) || (b->table_width > 0 && !aligned(b->table, 4))) return false;
  if (!tokens) return true;
  return b->n_tokens >= 0 && b->n_tokens <= (1 << 28) && b->max_new >= 0 && aligned(b->q_start, 4);
}

SeqView seq_view(const xkv_paged_batch* b) {
  SeqView s;
  s.n_seqs = b->n_seqs; s.n_tokens = b->n_tokens; s.max_new = b->max_new; s.table_width = b->table_width;
  s.q_start = b->q_start; s.lens = b->lens; s.table = b->table;
  return s;
}

// Turns per position of every pair of an axis.
bool plan_rotary(const xkv_rotary_params* p, int head_dim, bool inverse, const int32_t* positions, int64_t pos_stride, int n, RotaryPlan* r) {
  if (!p || p->n_axes < 1 || p->n_axes > 4 || p->rotary_dim < 2 || p->rotary_dim % 2 || p->rotary_dim > head_dim ||
      p->rotary_dim * p->n_axes > head_dim) return false;
  if (!(p->base > 1.0) || !(p->factor >= 1.0) || !(p->magnitude > 0.0) || !isfinite(p->base) || !isfinite(p->factor) || !isfinite(p->magnitude)) return false;
  if (p->original_tokens < 0) return false;
  if (p->original_tokens > 0 && (!(p->beta_slow >= 0.0) || !(p->beta_fast > p->beta_slow) || !isfinite(p->beta_fast))) return false;
  if (n > 0 && !aligned(positions, 4)) return false;
  if (p->n_axes > 1 && pos_stride < n) return false;
  r->axes = p->n_axes; r->rot = p->rotary_dim; r->pairs = p->rotary_dim / 2; r->interleaved = p->interleaved != 0;
  r->magnitude = (float)p->magnitude;
  r->positions = positions; r->pos_stride = pos_stride;
  const double two_pi = 6.283185307179586476925286766559;
  // (powers one from another in 80 bits: a call of pow for each would take longer than the launch)
  const long double ratio = powl((long double)p->base, -2.0L / p->rotary_dim);
  long double power = 1.0L;
  for (int i = 0; i < r->pairs; ++i, power *= ratio) {
    double w = (double)power;
    if (p->original_tokens > 0) {
      double keep = (p->original_tokens * w / two_pi - p->beta_slow) / (p->beta_fast - p->beta_slow);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      w = w * keep + w / p->factor * (1.0 - keep);
    } else {
      w /= p->factor;
    }
    r->turns[i] = (inverse ? -w : w) / two_pi;
  }
  return true;
}

TokenTensor token_tensor(const xkv_rows& in, const xkv_rows& out, int heads) {
  TokenTensor t;
  t.in = reinterpret_cast<const uint8_t*>(in.data); t.out = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(out.data));
  t.in_ts = in.tok_stride; t.in_hs = in.head_stride; t.out_ts = out.tok_stride; t.out_hs = out.head_stride; t.heads = heads;
  return t;
}

// The handle's device has to be the current one.
int on_device(const xkv_paged* c) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return XKV_E_CUDA;
  return dev == c->device ? XKV_OK : XKV_E_INVALID;
}

int from_cuda(cudaError_t e) {
  return e == cudaSuccess ? XKV_OK : e == cudaErrorNotSupported ? XKV_E_UNSUPPORTED : XKV_E_CUDA;
}

}  // namespace

extern "C" {

int xkv_rotary(const xkv_rotary_params* params, int32_t dtype, int32_t head_dim, const int32_t* positions, int64_t pos_stride, int32_t n,
               const xkv_rows* x, int32_t n_q_heads, int32_t n_k_heads, int32_t inverse, xkv_stream stream) {
  if (dtype != XKV_BF16 && dtype != XKV_FP16) return XKV_E_INVALID;
  if (head_dim < 8 || head_dim > 2 * kMaxPairs || head_dim % 8) return XKV_E_INVALID;
  if (n < 0 || n > (1 << 28) || n_q_heads < 1 || n_q_heads > 1024 || n_k_heads < 0 || n_k_heads > 1024) return XKV_E_INVALID;
  TokenArgs a;
  memset(&a, 0, sizeof(a));
  if (!plan_rotary(params, head_dim, inverse != 0, positions, pos_stride, n, &a.rot)) return XKV_E_INVALID;
  if (n == 0) return XKV_OK;
  if (!x || !rows_ok(x[0]) || !rows_ok(x[1]) || !in_place_ok(x[0], x[1])) return XKV_E_INVALID;
  if (n_k_heads > 0 && (!rows_ok(x[2]) || !rows_ok(x[3]) || !in_place_ok(x[2], x[3]))) return XKV_E_INVALID;
  int dev, sms;
  const int rc = device_setup(&dev, &sms);
  if (rc != XKV_OK) return rc;
  a.n = n; a.head_dim = head_dim;
  a.q = token_tensor(x[0], x[1], n_q_heads);
  if (n_k_heads > 0) a.k = token_tensor(x[2], x[3], n_k_heads);
  return from_cuda(launch_tokens(a, dtype, sms, reinterpret_cast<cudaStream_t>(stream)));
}

size_t xkv_paged_workspace_bytes(const xkv_paged_params* params, int32_t multiprocessors) {
  if (!params_ok(params) || multiprocessors < 1 || multiprocessors > 1024) return 0;
  return make_layout(params, multiprocessors).total;
}

int xkv_paged_create(const xkv_paged_params* params, void* k_pages, void* v_pages, float* weights, void* dev_workspace, size_t bytes,
                     xkv_stream stream, xkv_paged** out) {
  if (!out) return XKV_E_INVALID;
  *out = nullptr;
  if (!params) return XKV_E_INVALID;
  if (!params_ok(params)) {
    if (params->head_dim > 0 && params->head_dim != 64 && params->head_dim != 128) return XKV_E_UNSUPPORTED;
    if (params->page_tokens > 0 && (params->page_tokens < 16 || params->page_tokens > 256 || (params->page_tokens & (params->page_tokens - 1))))
      return XKV_E_UNSUPPORTED;
    return XKV_E_INVALID;
  }
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16) || (weights && !aligned(weights, 4)) || !aligned(dev_workspace, 256)) return XKV_E_INVALID;
  int dev, sms;
  const int rc = device_setup(&dev, &sms);
  if (rc != XKV_OK) return rc;
  const Layout layout = make_layout(params, sms);
  const size_t need = layout.total;
  if (bytes < need) return XKV_E_NOMEM;
  xkv_paged* c = new (std::nothrow) xkv_paged;
  if (!c) return XKV_E_NOMEM;
  memset(c, 0, sizeof(*c));
  c->p = *params;
  c->device = dev;
  c->sm_count = sms;
  c->ws = reinterpret_cast<uint8_t*>(dev_workspace);
  c->ws_bytes = need;
  PagedView& v = c->view;
  v.k = reinterpret_cast<uint8_t*>(k_pages); v.v = reinterpret_cast<uint8_t*>(v_pages); v.weights = weights;
  v.page_stride = params->page_stride; v.head_stride = params->head_stride; v.slot_stride = params->slot_stride;
  v.n_heads = params->n_heads; v.n_kv_heads = params->n_kv_heads; v.group = params->n_heads / params->n_kv_heads;
  v.page_shift = log2_of(params->page_tokens); v.n_pages = params->n_pages;
  v.status = reinterpret_cast<int*>(c->ws);
  c->scratch.count = reinterpret_cast<unsigned int*>(c->ws + layout.off_count);
  c->scratch.again = reinterpret_cast<unsigned int*>(c->ws + layout.off_again);
  c->scratch.ml = reinterpret_cast<float2*>(c->ws + layout.off_ml);
  c->scratch.o = reinterpret_cast<float*>(c->ws + layout.off_o);
  c->cuts = c->ws + layout.off_cuts;
  if (make_pool_maps(v, params->head_dim, params->dtype, 16, &c->maps16) != cudaSuccess ||
      make_pool_maps(v, params->head_dim, params->dtype, params->page_tokens < 128 ? params->page_tokens : 128, &c->maps_page) != cudaSuccess) { delete c; return XKV_E_CUDA; }
  if (cudaMemsetAsync(c->ws, 0, need, reinterpret_cast<cudaStream_t>(stream)) != cudaSuccess) { delete c; return XKV_E_CUDA; }
  *out = c;
  return XKV_OK;
}

int xkv_paged_destroy(xkv_paged* c) {
  if (!c) return XKV_E_INVALID;
  delete c;
  return XKV_OK;
}

int xkv_paged_poll_status(xkv_paged* c, xkv_stream stream) {
  if (!c) return XKV_E_INVALID;
  const int rc = on_device(c);
  if (rc != XKV_OK) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  int v = 0;
  if (cudaMemcpyAsync(&v, c->view.status, sizeof(v), cudaMemcpyDeviceToHost, st) != cudaSuccess) return XKV_E_CUDA;
  if (cudaStreamSynchronize(st) != cudaSuccess) return XKV_E_CUDA;
  if (v != 0 && cudaMemsetAsync(c->view.status, 0, sizeof(v), st) != cudaSuccess) return XKV_E_CUDA;
  return v;
}

int kv_paged_append(xkv_paged* c, const xkv_paged_batch* b, const xkv_rows* x, const xkv_rotary_params* rotary, const int32_t* positions,
                    int64_t pos_stride, xkv_stream stream) {
  if (!c || !batch_ok(c, b, true)) return XKV_E_INVALID;
  TokenArgs a;
  memset(&a, 0, sizeof(a));
  if (rotary && !plan_rotary(rotary, c->p.head_dim, false, positions, pos_stride, b->n_tokens, &a.rot)) return XKV_E_INVALID;
  const int rc = on_device(c);
  if (rc != XKV_OK) return rc;
  if (b->n_tokens == 0) return XKV_OK;
  if (!x || !rows_ok(x[0]) || !rows_ok(x[1])) return XKV_E_INVALID;
  if (x[2].data && (!rows_ok(x[2]) || !rows_ok(x[3]) || !in_place_ok(x[2], x[3]))) return XKV_E_INVALID;
  a.n = b->n_tokens; a.head_dim = c->p.head_dim; a.append = 1;
  const xkv_rows none = {nullptr, 0, 0};
  if (x[2].data) a.q = token_tensor(x[2], x[3], c->p.n_heads);
  a.k = token_tensor(x[0], none, c->p.n_kv_heads);
  a.v = token_tensor(x[1], none, c->p.n_kv_heads);
  a.cache = c->view; a.seqs = seq_view(b);
  return from_cuda(launch_tokens(a, c->p.dtype, c->sm_count, reinterpret_cast<cudaStream_t>(stream)));
}

int attn_paged_causal(xkv_paged* c, const xkv_paged_batch* b, const xkv_rows* x, float* lse, float scale, int32_t mask, int32_t impl,
                      xkv_stream stream) {
  if (!c || !batch_ok(c, b, true) || !(scale > 0.f) || !isfinite(scale) || (mask != XKV_MASK_CAUSAL && mask != XKV_MASK_FULL) || (impl != 0 && impl != 1))
    return XKV_E_INVALID;
  const int rc = on_device(c);
  if (rc != XKV_OK) return rc;
  if (b->n_tokens == 0 || b->max_new == 0) return XKV_OK;
  if (!x || !rows_ok(x[0]) || !rows_ok(x[1]) || (lse && !aligned(lse, 4))) return XKV_E_INVALID;
  PagedAttnArgs a;
  memset(&a, 0, sizeof(a));
  a.cache = c->view; a.seqs = seq_view(b);
  a.q = reinterpret_cast<const uint8_t*>(x[0].data); a.q_ts = x[0].tok_stride; a.q_hs = x[0].head_stride;
  a.out = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(x[1].data)); a.o_ts = x[1].tok_stride; a.o_hs = x[1].head_stride;
  a.lse = lse; a.scale_log2 = scale * 1.4426950408889634f; a.full = mask == XKV_MASK_FULL;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (impl == 1) return from_cuda(launch_paged_attn_simple(a, c->p.head_dim, c->p.dtype, st));
  if (!work_ok(c, b)) return XKV_E_LIMIT;
  if ((int64_t)b->max_new * c->view.group <= kFewRows)
    return from_cuda(launch_attn_few(a, c->maps16, c->scratch, c->p.head_dim, c->p.dtype, c->sm_count, st));
  return from_cuda(launch_attn_chunk(a, c->maps_page, c->scratch, c->cuts, c->p.head_dim, c->p.dtype, c->sm_count, st));
}

int kv_paged_weights(xkv_paged* c, const xkv_paged_batch* b, const xkv_rows* q, const float* lse, float scale, float decay, int32_t mask,
                     xkv_stream stream) {
  if (!c || !batch_ok(c, b, true) || !(scale > 0.f) || !isfinite(scale) || !(decay >= 0.f) || !isfinite(decay) ||
      (mask != XKV_MASK_CAUSAL && mask != XKV_MASK_FULL)) return XKV_E_INVALID;
  const int rc = on_device(c);
  if (rc != XKV_OK) return rc;
  if (!c->view.weights) return XKV_E_STATE;
  if (b->n_tokens == 0 || b->max_new == 0 || b->table_width == 0) return XKV_OK;
  if (!q || !rows_ok(*q) || !aligned(lse, 4)) return XKV_E_INVALID;
  PagedWeightArgs a;
  memset(&a, 0, sizeof(a));
  a.cache = c->view; a.seqs = seq_view(b);
  a.q = reinterpret_cast<const uint8_t*>(q->data); a.q_ts = q->tok_stride; a.q_hs = q->head_stride;
  a.lse = lse; a.scale_log2 = scale * 1.4426950408889634f; a.decay = decay; a.full = mask == XKV_MASK_FULL;
  if (!work_ok(c, b)) return XKV_E_LIMIT;
  return from_cuda(launch_paged_weights(a, c->maps_page, c->p.head_dim, c->p.dtype, c->sm_count, reinterpret_cast<cudaStream_t>(stream)));
}

int kv_paged_evict(xkv_paged* c, const xkv_paged_batch* b, const int32_t* dst_table, int32_t dst_width, int32_t keep, int32_t n_first,
                   int32_t n_recent, int32_t* kept, int32_t* lens_out, xkv_stream stream) {
  if (!c || !batch_ok(c, b, false)) return XKV_E_INVALID;
  if (keep < 1 || n_first < 0 || n_recent < 0 || (int64_t)n_first + n_recent > keep) return XKV_E_INVALID;
  if (dst_width < 1 || (int64_t)dst_width * c->p.page_tokens < keep || (int64_t)dst_width * c->p.page_tokens >= ((int64_t)1 << 31) - (1 << 16))
    return XKV_E_INVALID;
  if (!aligned(dst_table, 4) || !aligned(kept, 4) || !aligned(lens_out, 4)) return XKV_E_INVALID;
  // (blocks of the call read the lengths while others write the new ones)
  if (lens_out < b->lens + b->n_seqs && b->lens < lens_out + b->n_seqs) return XKV_E_INVALID;
  if (dst_table == b->table) return XKV_E_INVALID;
  const int rc = on_device(c);
  if (rc != XKV_OK) return rc;
  if (!c->view.weights) return XKV_E_STATE;
  EvictArgs a;
  memset(&a, 0, sizeof(a));
  a.cache = c->view; a.seqs = seq_view(b);
  a.dst_table = dst_table; a.dst_width = dst_width; a.keep = keep; a.n_first = n_first; a.n_recent = n_recent;
  a.head_dim = c->p.head_dim; a.kept = kept; a.lens_out = lens_out;
  return from_cuda(launch_evict(a, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
