// Host side of the window forward's operators declared in include/sjd.h:
// argument checks, the handle, launches.

#include <cmath>
#include <cstdio>
#include <new>

#include "sjd_kv.h"

using namespace sjd_kv_ops;

struct sjd_kv {
  sjd_kv_config cfg;
  unsigned char* ws;  // the status word, then the attention's scratch from kAlign on
  cudaStream_t stream;
  int sms;
  char last_error[256];
};

namespace {

constexpr size_t kAlign = 256;

bool valid(const sjd_kv_config* c) {
  return c && c->batch >= 1 && c->kv_heads >= 1 && c->heads >= c->kv_heads && c->heads % c->kv_heads == 0 &&
         c->heads / c->kv_heads <= 128 && c->head_dim >= 8 && c->head_dim <= kMaxDim && c->head_dim % 8 == 0 &&
         c->page_size >= 1 && c->n_pages >= 1 && c->max_pages >= 1 && c->max_new >= 1 &&
         static_cast<long long>(c->max_pages) * c->page_size <= (1LL << 30) && c->kv_heads <= 65536 &&
         // (vectors are counted in 32 bits)
         static_cast<double>(c->n_pages) * c->kv_heads * c->page_size < 4294967295.0 &&
         static_cast<long long>(c->batch) * c->max_new <= 0x7fffffffLL / 256 &&
         (c->kv_dtype == SJD_BF16 || c->kv_dtype == SJD_E4M3 || c->kv_dtype == SJD_S8);
}

int fail(sjd_kv* kv, int code, const char* why) {
  std::snprintf(kv->last_error, sizeof kv->last_error, "%s", why);
  return code;
}

int launched(sjd_kv* kv, cudaError_t e, const char* what) {
  if (e == cudaSuccess) return SJD_OK;
  std::snprintf(kv->last_error, sizeof kv->last_error, "%s: %s", what, cudaGetErrorString(e));
  return SJD_ERR_CUDA;
}

bool count_sms(int* sms) {  // of the current device
  int device = 0;
  return cudaGetDevice(&device) == cudaSuccess && cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device) == cudaSuccess;
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

const char* bad_rope(const sjd_rope* r, int dim) {
  if (!r->turns_dev || !r->axis_dev) return "rope: NULL table";
  if (r->pairs < 4 || r->pairs % 4 || 2 * r->pairs > dim) return "rope: pairs must be a multiple of 4, at most dim / 2";
  if (r->axes < 1 || r->axes > kMaxAxes) return "rope: axes must be in [1, 8]";
  if (r->interleaved != 0 && r->interleaved != 1) return "rope: interleaved must be 0 or 1";
  return nullptr;
}

Rope rope_of(const sjd_rope* r, const int32_t* positions, int inverse, uint32_t* status) {
  return {r->turns_dev, r->axis_dev, positions, r->pairs, r->axes, r->interleaved, inverse, status};
}

View view_of(const sjd_view* v) { return {v->data_dev, v->batch_stride, v->token_stride, v->head_stride}; }

size_t size_of(int dtype) { return dtype == SJD_BF16 ? 2 : 4; }

// The cache and spans of a call; a text if an argument is wrong.
const char* cache_of(sjd_kv* kv, const sjd_kv_layer* l, const sjd_kv_span* s, long long most, Cache* c) {
  const sjd_kv_config& g = kv->cfg;
  if (!l || !s) return "layer or span is NULL";
  if (!l->k_dev || !l->v_dev || !aligned(l->k_dev, 16) || !aligned(l->v_dev, 16)) return "layer: keys and values must be 16-byte aligned device memory";
  const bool scaled = g.kv_dtype != SJD_BF16;
  if (scaled && (!l->k_scale_dev || !l->v_scale_dev || !aligned(l->k_scale_dev, 4) || !aligned(l->v_scale_dev, 4)))
    return "layer: an 8-bit cache needs scales";
  if (!s->table_dev || !s->start_dev) return "span: table or start is NULL";
  if (s->n < 1 || s->n > most) return "span: n out of range";
  const int group = g.heads / g.kv_heads;
  const Divisor page = divisor(g.page_size), heads = divisor(group);
  *c = {g.batch, g.heads, g.kv_heads, g.head_dim, g.page_size, g.n_pages, g.max_pages, l->k_dev, l->v_dev,
        scaled ? l->k_scale_dev : nullptr, scaled ? l->v_scale_dev : nullptr, s->table_dev, s->start_dev, s->count_dev,
        s->n, reinterpret_cast<uint32_t*>(kv->ws), group, page.mul, heads.mul, page.shift, heads.shift};
  return nullptr;
}

}  // namespace

extern "C" {

int sjd_rope_turns(const double* freq, int32_t n, uint64_t* turns) {
  if (!freq || !turns || n < 0) return SJD_ERR_ARG;
  for (int i = 0; i < n; ++i) {
    const double t = freq[i] / (2.0 * 3.14159265358979323846);
    if (!(std::fabs(t) < 9007199254740992.0)) return SJD_ERR_ARG;
    // (the fraction, below 1 and exact, times 2^64; the product rounds to an integer below 2^64 + 1)
    double f = std::rint(std::ldexp(t - std::floor(t), 64));
    if (f >= 18446744073709551616.0) f = 0.0;
    turns[i] = static_cast<uint64_t>(f);
  }
  return SJD_OK;
}

int sjd_rotate(const sjd_rope* rope, const sjd_view* x, const sjd_view* y, const int32_t* positions, int32_t batch, int32_t n,
               int32_t heads, int32_t dim, int32_t dtype, int32_t inverse, void* stream) {
  if (!rope || !x || !y || !x->data_dev || !y->data_dev || !positions) return SJD_ERR_ARG;
  if (batch < 1 || n < 1 || heads < 1 || heads > (1 << 20) || static_cast<long long>(batch) * n > 0x7fffffffLL) return SJD_ERR_ARG;
  if (dim < 8 || dim > kMaxRotateDim || dim % 8 || (dtype != SJD_F32 && dtype != SJD_BF16)) return SJD_ERR_ARG;
  if ((inverse != 0 && inverse != 1) || bad_rope(rope, dim)) return SJD_ERR_ARG;
  if (!aligned(x->data_dev, size_of(dtype)) || !aligned(y->data_dev, size_of(dtype))) return SJD_ERR_ARG;
  const RotateParams p{rope_of(rope, positions, inverse, nullptr), view_of(x), view_of(y), batch, n, heads, dim};
  int sms = 0;
  if (!count_sms(&sms)) return SJD_ERR_CUDA;
  return launch_rotate(p, dtype, sms, static_cast<cudaStream_t>(stream)) == cudaSuccess ? SJD_OK : SJD_ERR_CUDA;
}

size_t sjd_kv_workspace_size(const sjd_kv_config* cfg) {
  if (!valid(cfg)) return 0;
  return kAlign + attend_scratch_bytes(cfg->head_dim, static_cast<long long>(cfg->max_new) * (cfg->heads / cfg->kv_heads));
}

int sjd_kv_init(const sjd_kv_config* cfg, void* workspace, size_t ws_bytes, void* stream, sjd_kv** out) {
  if (!out) return SJD_ERR_ARG;
  *out = nullptr;
  if (!valid(cfg) || !workspace || !aligned(workspace, kAlign)) return SJD_ERR_ARG;
  if (ws_bytes < sjd_kv_workspace_size(cfg)) return SJD_ERR_CAPACITY;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int sms = 0;
  if (!count_sms(&sms)) return SJD_ERR_CUDA;
  if (prepare_attend(cfg->kv_dtype, cfg->head_dim) != cudaSuccess) return SJD_ERR_CUDA;
  if (cudaMemsetAsync(workspace, 0, kAlign + attend_counter_bytes(), s) != cudaSuccess) return SJD_ERR_CUDA;
  sjd_kv* kv = new (std::nothrow) sjd_kv{*cfg, static_cast<unsigned char*>(workspace), s, sms, ""};
  if (!kv) return SJD_ERR_CAPACITY;
  *out = kv;
  return SJD_OK;
}

int sjd_kv_write(sjd_kv* kv, const sjd_kv_layer* layer, const sjd_kv_span* span, int32_t dtype, const sjd_view* k,
                 const sjd_view* v, const sjd_rope* rope, const int32_t* positions, const sjd_view* q, const sjd_view* q_out) {
  if (!kv) return SJD_ERR_ARG;
  WriteParams p{};
  if (const char* why = cache_of(kv, layer, span, kv->cfg.max_new, &p.c)) return fail(kv, SJD_ERR_ARG, why);
  if (dtype != SJD_F32 && dtype != SJD_BF16) return fail(kv, SJD_ERR_ARG, "dtype must be SJD_F32 or SJD_BF16");
  if (!k || !v || !k->data_dev || !v->data_dev) return fail(kv, SJD_ERR_ARG, "keys or values are NULL");
  if (!aligned(k->data_dev, size_of(dtype)) || !aligned(v->data_dev, size_of(dtype)))
    return fail(kv, SJD_ERR_ARG, "keys or values are not aligned to their type");
  p.k = view_of(k);
  p.v = view_of(v);
  if (rope) {
    if (const char* why = bad_rope(rope, kv->cfg.head_dim)) return fail(kv, SJD_ERR_ARG, why);
    if (!positions) return fail(kv, SJD_ERR_ARG, "positions are NULL");
    p.rope = rope_of(rope, positions, 0, reinterpret_cast<uint32_t*>(kv->ws));
  }
  if ((q != nullptr) != (q_out != nullptr) || (q && !rope)) return fail(kv, SJD_ERR_ARG, "queries come with rope and q_out");
  if (q) {
    if (!q->data_dev || !q_out->data_dev || !aligned(q->data_dev, size_of(dtype)) || !aligned(q_out->data_dev, size_of(dtype)))
      return fail(kv, SJD_ERR_ARG, "queries are NULL or not aligned to their type");
    p.q = view_of(q);
    p.q_out = view_of(q_out);
  }
  return launched(kv, launch_write(p, dtype, kv->cfg.kv_dtype, kv->sms, kv->stream), "write");
}

int sjd_kv_read(sjd_kv* kv, const sjd_kv_layer* layer, const sjd_kv_span* span, int32_t dtype, void* k_out, void* v_out) {
  if (!kv) return SJD_ERR_ARG;
  ReadParams p{};
  const long long room = static_cast<long long>(kv->cfg.max_pages) * kv->cfg.page_size;
  if (const char* why = cache_of(kv, layer, span, room, &p.c)) return fail(kv, SJD_ERR_ARG, why);
  if (dtype != SJD_F32 && dtype != SJD_BF16) return fail(kv, SJD_ERR_ARG, "dtype must be SJD_F32 or SJD_BF16");
  if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16)) return fail(kv, SJD_ERR_ARG, "outputs must be 16-byte aligned");
  if (static_cast<long long>(p.c.B) * p.c.n > 0x7fffffffLL) return fail(kv, SJD_ERR_ARG, "span: too many tokens");
  p.k_out = k_out;
  p.v_out = v_out;
  return launched(kv, launch_read(p, dtype, kv->cfg.kv_dtype, kv->sms, kv->stream), "read");
}

int sjd_kv_attend(sjd_kv* kv, const sjd_kv_layer* layer, const sjd_kv_span* span, const sjd_view* q, int32_t mask_kind,
                  const uint8_t* mask, int64_t mask_batch_stride, int64_t mask_row_stride, float scale, void* o, float* lse) {
  if (!kv) return SJD_ERR_ARG;
  AttendParams p{};
  if (const char* why = cache_of(kv, layer, span, kv->cfg.max_new, &p.c)) return fail(kv, SJD_ERR_ARG, why);
  // (the stride of a dimension of one element means nothing)
  if (!q || !q->data_dev || !aligned(q->data_dev, 16) || (kv->cfg.batch > 1 && q->batch_stride % 8) ||
      (span->n > 1 && q->token_stride % 8) || (kv->cfg.heads > 1 && q->head_stride % 8))
    return fail(kv, SJD_ERR_ARG, "queries must have 16-byte aligned rows");
  if (mask_kind != SJD_MASK_CAUSAL && mask_kind != SJD_MASK_ALL && mask_kind != SJD_MASK_GIVEN)
    return fail(kv, SJD_ERR_ARG, "unknown mask kind");
  if ((mask_kind == SJD_MASK_GIVEN) != (mask != nullptr)) return fail(kv, SJD_ERR_ARG, "mask_dev goes with SJD_MASK_GIVEN");
  // (the kernel's factor, |scale| log2 e, is to be a number)
  if (!(std::fabs(scale) <= 0x1p127f)) return fail(kv, SJD_ERR_ARG, "scale must be finite and at most 2^127");
  if (!o || !aligned(o, 16) || !aligned(lse, 4)) return fail(kv, SJD_ERR_ARG, "output is NULL or not aligned");
  p.q = view_of(q);
  p.mask_kind = mask_kind;
  p.mask = mask;
  p.mask_b = mask_batch_stride;
  p.mask_r = mask_row_stride;
  p.scale = scale;
  p.o = o;
  p.lse = lse;
  return launched(kv, launch_attend(p, kv->cfg.kv_dtype, kv->sms, kv->ws + kAlign, kv->stream), "attend");
}

int sjd_kv_sync(sjd_kv* kv) {
  if (!kv) return SJD_ERR_ARG;
  uint32_t bits = 0;
  cudaError_t e = cudaMemcpyAsync(&bits, kv->ws, sizeof bits, cudaMemcpyDeviceToHost, kv->stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(kv->stream);
  if (e == cudaSuccess && bits) {
    // (a kernel that gave up may have left its counters)
    e = cudaMemsetAsync(kv->ws, 0, bits & status_bit(SJD_ERR_TIMEOUT) ? kAlign + attend_counter_bytes() : sizeof bits, kv->stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(kv->stream);
  }
  if (e != cudaSuccess) return launched(kv, e, "sync");
  if (bits & status_bit(SJD_ERR_TIMEOUT)) return fail(kv, SJD_ERR_TIMEOUT, "a wait inside the attention kernel ran out");
  if (bits & status_bit(SJD_ERR_BOUNDS)) return fail(kv, SJD_ERR_BOUNDS, "an index outside its array (bounds-checked build); the access was clamped");
  if (bits & status_bit(SJD_ERR_PAGE)) return fail(kv, SJD_ERR_PAGE, "a span outside its page table, or a page outside the cache");
  return SJD_OK;
}

const char* sjd_kv_last_error(const sjd_kv* kv) { return kv ? kv->last_error : "no handle"; }

void sjd_kv_destroy(sjd_kv* kv) { delete kv; }

}  // extern "C"
