// Host side of the iteration operators: argument checks, nothing else.
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "gnr_iter_internal.h"

namespace gnr {
namespace {

constexpr int64_t kMaxTokens = int64_t(1) << 30;
constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr int64_t kMaxPlaceStride = int64_t(1) << 24;   // (sixteen of them are an offset of 32 bits)
constexpr int kMaxHeads = 4096;

bool aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// strides of rows that start at 16-byte boundaries, small enough for offsets of 64 bits
bool strides_ok(int bytes_of_element, int64_t a, int64_t b, int64_t c)
{
  const int64_t unit = 16 / bytes_of_element;
  for (const int64_t s : {a, b, c})
    if (s < 0 || s > kMaxStride || s % unit != 0) return false;
  return true;
}

bool span_ok(int64_t n, int64_t stride) { return n <= 0 || stride <= (int64_t(1) << 60) / n; }

bool plane_ok(const iter_cache &c, const iter_plane &p)
{
  const int size = c.type == ITER_FP8 ? 1 : 2;
  if (!strides_ok(size, p.page_stride, p.head_stride, p.place_stride) || !span_ok(c.pages, p.page_stride) || p.place_stride > kMaxPlaceStride) return false;
  if (c.pages > 0 && (!p.data || !aligned(p.data))) return false;
  if (c.type != ITER_FP8) return p.exp == nullptr;
  for (const int64_t s : {p.exp_page_stride, p.exp_head_stride, p.exp_place_stride})
    if (s < 0 || s > kMaxStride) return false;
  return p.exp_place_stride <= kMaxPlaceStride && span_ok(c.pages, p.exp_page_stride) && (c.pages == 0 || p.exp != nullptr);
}

bool cache_ok(const iter_cache *c)
{
  if (!c || c->type < ITER_BF16 || c->type > ITER_FP8) return false;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return false;
  if (c->kv_heads < 1 || c->kv_heads > kMaxHeads || c->page < 1 || c->page > 65536 || (c->page & (c->page - 1)) != 0) return false;
  if (c->pages < 0 || c->pages > INT32_MAX) return false;
  return plane_ok(*c, c->k) && plane_ok(*c, c->v);
}

bool type_fits(const iter_cache &c, int type)
{
  return (type == ITER_BF16 || type == ITER_FP16) && (c.type == ITER_FP8 || c.type == type);
}

bool rows_ok(const iter_rows *r, int64_t tokens)
{
  if (!r || !strides_ok(2, r->token_stride, r->head_stride, 0) || !span_ok(tokens, r->token_stride)) return false;
  return tokens == 0 || (r->data && aligned(r->data));
}

int check_kv(const iter_cache *c, int type, const iter_rows *k, const iter_rows *v, const int64_t *slots, int64_t tokens)
{
  if (!cache_ok(c) || !type_fits(*c, type) || tokens < 0 || tokens > kMaxTokens) return SIM_EINVAL;
  if (!rows_ok(k, tokens) || !rows_ok(v, tokens) || (tokens > 0 && !slots)) return SIM_EINVAL;
  return SIM_OK;
}

int check_batch(const iter_cache *c, const iter_batch *b, int heads)
{
  if (!cache_ok(c) || !b || heads < 1 || heads > kMaxHeads || heads % c->kv_heads != 0) return SIM_EINVAL;
  // (numbers of tiles fit 32 bits whatever the device finds in q_start, where every second request may claim all tokens)
  if (b->requests < 0 || b->requests > ITER_MAX_REQUESTS || b->tokens < 0 || b->tokens > ITER_MAX_TOKENS) return SIM_EINVAL;
  if (b->tokens * (heads / c->kv_heads) > 16 * int64_t(ITER_MAX_TOKENS) || b->max_q < 0 || (b->tokens > 0 && b->requests == 0)) return SIM_EINVAL;
  if (b->table_stride < 0 || b->table_stride > kMaxStride || b->table_width < 0 || b->table_width > INT32_MAX) return SIM_EINVAL;
  return SIM_OK;
}

}  // namespace
}  // namespace gnr

using namespace gnr;

extern "C" {

int iter_kv_write(const iter_cache *c, int type, const iter_rows *k, const iter_rows *v, const int64_t *slots, int64_t tokens, void *hip_stream)
{
  const int rc = check_kv(c, type, k, v, slots, tokens);
  if (rc != SIM_OK || tokens == 0) return rc;
  return launch_kv_write(*c, type, *k, *v, slots, tokens, hip_stream);
}

int iter_kv_read(const iter_cache *c, int type, const iter_rows *k, const iter_rows *v, const int64_t *slots, int64_t tokens, void *hip_stream)
{
  const int rc = check_kv(c, type, k, v, slots, tokens);
  if (rc != SIM_OK || tokens == 0) return rc;
  return launch_kv_read(*c, type, *k, *v, slots, tokens, hip_stream);
}

int iter_attention_bytes(const iter_cache *c, const iter_batch *b, int heads, size_t *out_bytes)
{
  const int rc = check_batch(c, b, heads);
  if (rc != SIM_OK || !out_bytes) return SIM_EINVAL;
  *out_bytes = attention_bytes(*c, *b, heads);
  return SIM_OK;
}

int iter_attention(const iter_cache *c, const iter_batch *b, int type, int heads, const iter_rows *q, const iter_rows *out,
                   double scale, int64_t window, void *workspace, size_t bytes, uint32_t *status, void *hip_stream)
{
  const int rc = check_batch(c, b, heads);
  if (rc != SIM_OK) return rc;
  if (!type_fits(*c, type) || !rows_ok(q, b->tokens) || !rows_ok(out, b->tokens)) return SIM_EINVAL;
  if (!std::isfinite(scale) || window < 0) return SIM_EINVAL;
  if (b->tokens == 0) return SIM_OK;
  if (q->data == out->data) return SIM_EINVAL;
  if (!b->q_start || !b->kv_len || (!b->page_table && b->table_width > 0)) return SIM_EINVAL;
  const size_t need = attention_bytes(*c, *b, heads);
  if (need > 0 && (!workspace || !aligned(workspace))) return SIM_EINVAL;
  if (bytes < need) return SIM_ENOMEM;
  AttentionParams p{};
  p.cache = *c; p.batch = *b; p.q = *q; p.out = *out;
  p.type = type; p.heads = heads; p.group = heads / c->kv_heads;
  p.page_shift = __builtin_ctz(static_cast<unsigned>(c->page));
  // (its sign goes into the queries; a scale of zero is a tiny one, so that a hidden key's score of -infinity stays what it is)
  p.scale_log2 = static_cast<float>(std::fmax(std::fabs(scale * 1.4426950408889634), 1e-30));
  p.flip = scale < 0.0 ? 0x80008000u : 0u;
  p.window = static_cast<int>(window < (int64_t(1) << 30) ? window : 0);   // no request is longer
  p.workspace = static_cast<float *>(workspace);
  p.status = status;
  return launch_attention(p, hip_stream);
}

int iter_adapters_bytes(const iter_adapter_set *s, int64_t tokens, size_t *out_bytes)
{
  if (!s || !out_bytes || tokens < 0 || tokens > ITER_MAX_TOKENS || s->rank < 8 || s->rank > ITER_MAX_RANK || s->rank % 8 != 0) return SIM_EINVAL;
  if (s->width_in < 8 || s->width_in > (1 << 24) || s->adapters < 0 || s->adapters > ITER_MAX_ADAPTERS) return SIM_EINVAL;
  *out_bytes = adapters_bytes(*s, tokens);
  return SIM_OK;
}

int iter_adapters(const iter_adapter_set *s, int type, int requests, int64_t tokens, const int32_t *q_start, const int32_t *adapter,
                  const void *x, int64_t x_stride, const void *base, int64_t base_stride, void *out, int64_t out_stride,
                  void *workspace, size_t bytes, uint32_t *status, void *hip_stream)
{
  size_t need = 0;
  const int rc = iter_adapters_bytes(s, tokens, &need);
  if (rc != SIM_OK) return rc;
  if (type != ITER_BF16 && type != ITER_FP16) return SIM_EINVAL;
  if (s->width_in % 8 != 0 || s->width_out < 8 || s->width_out > (1 << 24) || s->width_out % 8 != 0) return SIM_EINVAL;
  if (requests < 0 || requests > ITER_MAX_REQUESTS || (tokens > 0 && requests == 0)) return SIM_EINVAL;
  if (!strides_ok(2, x_stride, base_stride, out_stride) || !span_ok(tokens, x_stride) || !span_ok(tokens, base_stride) || !span_ok(tokens, out_stride))
    return SIM_EINVAL;
  if (tokens == 0) return SIM_OK;
  if (!q_start || !adapter || !x || !base || !out || !aligned(x) || !aligned(base) || !aligned(out)) return SIM_EINVAL;
  if (s->adapters > 0 && (!s->down || !s->up || !s->scale || !aligned(s->down) || !aligned(s->up))) return SIM_EINVAL;
  if (need > 0 && (!workspace || !aligned(workspace))) return SIM_EINVAL;
  if (bytes < need) return SIM_ENOMEM;
  AdapterParams p{};
  p.set = *s; p.type = type; p.requests = requests; p.tokens = tokens; p.q_start = q_start; p.adapter = adapter;
  p.x = x; p.base = base; p.out = out; p.x_stride = x_stride; p.base_stride = base_stride; p.out_stride = out_stride;
  p.workspace = static_cast<float *>(workspace);
  p.status = status;
  return launch_adapters(p, hip_stream);
}

int iter_abi_sizes(size_t *out5)
{
  if (!out5) return SIM_EINVAL;
  out5[0] = sizeof(iter_plane); out5[1] = sizeof(iter_cache); out5[2] = sizeof(iter_rows); out5[3] = sizeof(iter_batch);
  out5[4] = sizeof(iter_adapter_set);
  return SIM_OK;
}

}  // extern "C"
