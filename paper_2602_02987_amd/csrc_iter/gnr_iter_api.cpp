// Host side of the iteration operators: argument checks, nothing else.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <memory>
#include <new>
#include <numeric>

#include "gnr_iter_internal.h"

namespace gnr {
namespace {

constexpr int64_t kMaxTokens = int64_t(1) << 30;
constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr int64_t kMaxPlaceStride = int64_t(1) << 24;   // (sixteen of them are an offset of 32 bits)
constexpr int kMaxHeads = 4096;

bool aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// strides of rows that start at 16-byte boundaries, small enough for offsets of 64 bits
bool strides_ok(int bits_of_element, int64_t a, int64_t b, int64_t c)
{
  const int64_t unit = 128 / bits_of_element;
  for (const int64_t s : {a, b, c})
    if (s < 0 || s > kMaxStride || s % unit != 0) return false;
  return true;
}

bool span_ok(int64_t n, int64_t stride) { return n <= 0 || stride <= (int64_t(1) << 60) / n; }

bool plane_ok(const iter_cache &c, const iter_plane &p)
{
  const bool scaled = c.type == ITER_FP8 || c.type == ITER_FP4;
  if (!strides_ok(c.type == ITER_FP4 ? 4 : scaled ? 8 : 16, p.page_stride, p.head_stride, p.place_stride) || !span_ok(c.pages, p.page_stride) || p.place_stride > kMaxPlaceStride) return false;
  if (c.pages > 0 && (!p.data || !aligned(p.data))) return false;
  if (!scaled) return p.exp == nullptr;
  for (const int64_t s : {p.exp_page_stride, p.exp_head_stride, p.exp_place_stride})
    if (s < 0 || s > kMaxStride) return false;
  return p.exp_place_stride <= kMaxPlaceStride && span_ok(c.pages, p.exp_page_stride) && (c.pages == 0 || p.exp != nullptr);
}

bool cache_ok(const iter_cache *c)
{
  if (!c || c->type < ITER_BF16 || c->type > ITER_FP4) return false;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return false;
  if (c->kv_heads < 1 || c->kv_heads > kMaxHeads || c->page < 1 || c->page > 65536 || (c->page & (c->page - 1)) != 0) return false;
  if (c->pages < 0 || c->pages > INT32_MAX) return false;
  return plane_ok(*c, c->k) && plane_ok(*c, c->v);
}

bool type_fits(const iter_cache &c, int type)
{
  return (type == ITER_BF16 || type == ITER_FP16) && (c.type == ITER_FP8 || c.type == ITER_FP4 || c.type == type);
}

bool rows_ok(const iter_rows *r, int64_t tokens)
{
  if (!r || !strides_ok(16, r->token_stride, r->head_stride, 0) || !span_ok(tokens, r->token_stride)) return false;
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

// The remainder of a division that is rounded down.
int64_t remainder_of(int64_t n, int64_t d) { return (n % d + d) % d; }

// Whether pieces of `dim` elements at `off` and any multiples of `step` from there leave those at 0 and any multiples of it alone.
bool alternate(int64_t off, int64_t step, int dim)
{
  if (step < 2 * static_cast<int64_t>(dim)) return false;
  const int64_t at = remainder_of(off, step);
  return at >= dim && at + dim <= step;
}

// The stride of two counts of pieces, of which single ones have none; 0 if there is none in common.
int64_t common(int64_t a, int64_t count_a, int64_t b, int64_t count_b) { return count_a > 1 && count_b > 1 ? (a == b ? a : 0) : count_a > 1 ? a : count_b > 1 ? b : 0; }

// Whether pieces lie apart in the rows, `step` elements each, of one matrix, where those of a and b take `row_a` and `row_b`: beside each other, or, if neither's go on into the next row
// of the other, in turn (`inner`: the greatest common divisor of the strides within a row).
bool apart_in_matrix(int64_t between, int64_t step, int64_t row_a, int64_t row_b, int64_t inner, int dim)
{
  if (row_a > step || row_b > step) return false;
  const int64_t beside = remainder_of(between, step);
  if (beside >= row_a && beside + row_b <= step) return true;
  return (beside + row_b <= step && alternate(beside, inner, dim)) || (step - beside + row_a <= step && alternate(beside - step, inner, dim));
}

// Whether rows of `heads` heads of `dim` elements share no element with others: their bytes lie apart, they alternate (two pieces are as far apart as the rows' beginnings and multiples of the
// strides, which are multiples of the strides' greatest common divisor), or they lie apart in the rows of one matrix, as a projection leaves queries, keys and values, or in those of the heads.
bool apart(const iter_rows &a, int heads_a, const iter_rows &b, int heads_b, int64_t tokens, int dim)
{
  const uintptr_t at_a = reinterpret_cast<uintptr_t>(a.data), at_b = reinterpret_cast<uintptr_t>(b.data);
  const int64_t token_a = (heads_a - 1) * a.head_stride + dim, token_b = (heads_b - 1) * b.head_stride + dim, head_a = (tokens - 1) * a.token_stride + dim, head_b = (tokens - 1) * b.token_stride + dim;
  const uintptr_t end_a = at_a + 2 * static_cast<uintptr_t>(head_a - dim + token_a), end_b = at_b + 2 * static_cast<uintptr_t>(head_b - dim + token_b);
  if (end_a <= at_b || end_b <= at_a) return true;
  const int64_t between = static_cast<int64_t>(at_b - at_a) / 2;
  const int64_t heads = std::gcd(heads_a > 1 ? a.head_stride : 0, heads_b > 1 ? b.head_stride : 0), all = tokens > 1 ? std::gcd(a.token_stride, b.token_stride) : 0;
  return alternate(between, std::gcd(heads, all), dim) || apart_in_matrix(between, common(a.token_stride, tokens, b.token_stride, tokens), token_a, token_b, heads, dim) ||
         apart_in_matrix(between, common(a.head_stride, heads_a, b.head_stride, heads_b), head_a, head_b, all, dim);
}

bool same_rows(const iter_rows &a, const iter_rows &b, int64_t tokens, int heads)
{
  return a.data == b.data && (tokens == 1 || a.token_stride == b.token_stride) && (heads == 1 || a.head_stride == b.head_stride);
}

bool turns_ok(const iter_turns *t, int head_dim)
{
  return t && t->dims >= 16 && t->dims <= head_dim && t->dims % 16 == 0 && std::isfinite(t->magnitude);
}

bool alike(const iter_plane &a, const iter_plane &b)
{
  return a.page_stride == b.page_stride && a.head_stride == b.head_stride && a.place_stride == b.place_stride && a.exp_page_stride == b.exp_page_stride &&
         a.exp_head_stride == b.exp_head_stride && a.exp_place_stride == b.exp_place_stride;
}

bool alike(const iter_cache &a, const iter_cache &b)
{
  return a.type == b.type && a.kv_heads == b.kv_heads && a.head_dim == b.head_dim && a.page == b.page && a.pages == b.pages && alike(a.k, b.k) && alike(a.v, b.v);
}

// Whether no target is there twice or is a source as well.
int check_moves(const int64_t *source, const int64_t *target, int64_t count)
{
  if (count <= 64) {
    for (int64_t i = 0; i < count; ++i)
      for (int64_t j = 0; j < count; ++j)
        if (target[i] == source[j] || (i != j && target[i] == target[j])) return SIM_EINVAL;
    return SIM_OK;
  }
  const std::unique_ptr<int64_t[]> s(new (std::nothrow) int64_t[count]), t(new (std::nothrow) int64_t[count]);
  if (!s || !t) return SIM_ENOMEM;
  std::copy(source, source + count, s.get());
  std::copy(target, target + count, t.get());
  std::sort(s.get(), s.get() + count);
  std::sort(t.get(), t.get() + count);
  for (int64_t i = 0, j = 0; i < count; ++i) {
    if (i > 0 && t[i] == t[i - 1]) return SIM_EINVAL;
    while (j < count && s[j] < t[i]) ++j;
    if (j < count && s[j] == t[i]) return SIM_EINVAL;
  }
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
  if (!strides_ok(16, x_stride, base_stride, out_stride) || !span_ok(tokens, x_stride) || !span_ok(tokens, base_stride) || !span_ok(tokens, out_stride))
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

int iter_rotary(int type, int heads, int head_dim, const iter_turns *turns, const int64_t *positions, int64_t tokens, const iter_rows *x,
                const iter_rows *out, void *hip_stream)
{
  if (type != ITER_BF16 && type != ITER_FP16) return SIM_EINVAL;
  if (heads < 1 || heads > kMaxHeads || (head_dim != 64 && head_dim != 128 && head_dim != 256) || tokens < 0 || tokens > kMaxTokens) return SIM_EINVAL;
  if (!turns_ok(turns, head_dim) || !rows_ok(x, tokens) || !rows_ok(out, tokens)) return SIM_EINVAL;
  if (tokens == 0) return SIM_OK;
  if (!positions || !turns->turns) return SIM_EINVAL;
  if (!same_rows(*x, *out, tokens, heads) && !apart(*x, heads, *out, heads, tokens, head_dim)) return SIM_EINVAL;
  RotaryParams p{};
  p.type = type; p.heads = heads; p.head_dim = head_dim; p.turns = *turns; p.positions = positions; p.tokens = tokens; p.q = *x; p.out = *out;
  return launch_rotary(p, hip_stream);
}

int iter_rotary_write(const iter_cache *c, int type, int heads, const iter_turns *turns, const int64_t *positions, const iter_rows *q, const iter_rows *q_out,
                      const iter_rows *k, const iter_rows *v, const int64_t *slots, int64_t tokens, void *hip_stream)
{
  const int rc = check_kv(c, type, k, v, slots, tokens);
  if (rc != SIM_OK) return rc;
  if (heads < 0 || heads > kMaxHeads || !turns_ok(turns, c->head_dim)) return SIM_EINVAL;
  if (heads > 0 && (!rows_ok(q, tokens) || !rows_ok(q_out, tokens))) return SIM_EINVAL;
  if (tokens == 0) return SIM_OK;
  if (!positions || !turns->turns) return SIM_EINVAL;
  RotaryParams p{};
  if (heads > 0) {
    const int dim = c->head_dim;
    if (!same_rows(*q, *q_out, tokens, heads) && !apart(*q, heads, *q_out, heads, tokens, dim)) return SIM_EINVAL;
    if (!apart(*q_out, heads, *k, c->kv_heads, tokens, dim) || !apart(*q_out, heads, *v, c->kv_heads, tokens, dim)) return SIM_EINVAL;
    p.q = *q; p.out = *q_out;
  }
  p.type = type; p.heads = heads; p.head_dim = c->head_dim; p.turns = *turns; p.positions = positions; p.tokens = tokens;
  p.cache = *c; p.k = *k; p.v = *v; p.slots = slots;
  return launch_rotary(p, hip_stream);
}

int iter_copy_pages(const iter_cache *layers, int n_layers, const int64_t *source, const int64_t *target, const int64_t *places, int64_t count, void *hip_stream)
{
  if (n_layers < 0 || n_layers > ITER_MAX_LAYERS || (n_layers > 0 && !layers) || count < 0 || (count > 0 && (!source || !target))) return SIM_EINVAL;
  for (int i = 0; i < n_layers; ++i)
    if (!cache_ok(layers + i) || !alike(layers[0], layers[i])) return SIM_EINVAL;
  if (n_layers == 0 || count == 0) return SIM_OK;
  if (count > layers[0].pages) return SIM_EINVAL;      // (more targets than pages)
  if (int64_t(layers[0].page) * layers[0].kv_heads * layers[0].head_dim > (int64_t(1) << 33)) return SIM_EINVAL;   // (a page's pieces are numbers of 32 bits)
  for (int64_t i = 0; i < count; ++i) {
    if (source[i] < 0 || source[i] >= layers[0].pages || target[i] < 0 || target[i] >= layers[0].pages) return SIM_EINVAL;
    if (places && (places[i] < 0 || places[i] > layers[0].page)) return SIM_EINVAL;
  }
  const int rc = check_moves(source, target, count);
  return rc == SIM_OK ? launch_copy_pages(layers, n_layers, source, target, places, count, hip_stream) : rc;
}

int iter_turns_size(size_t *out_bytes)
{
  if (!out_bytes) return SIM_EINVAL;
  *out_bytes = sizeof(iter_turns);
  return SIM_OK;
}

int iter_abi_sizes(size_t *out5)
{
  if (!out5) return SIM_EINVAL;
  out5[0] = sizeof(iter_plane); out5[1] = sizeof(iter_cache); out5[2] = sizeof(iter_rows); out5[3] = sizeof(iter_batch);
  out5[4] = sizeof(iter_adapter_set);
  return SIM_OK;
}

}  // extern "C"
