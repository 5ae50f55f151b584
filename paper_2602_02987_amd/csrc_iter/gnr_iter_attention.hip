// Attention of a mixed batch over the paged cache (gfx950): every token of every request over its own request's keys.
#include "gnr_iter_device.h"

namespace gnr {

constexpr int kWaves = 4;

// Reads 8 elements of a cache row, widened.
template <class T, bool kFp8>
__device__ __forceinline__ void load8(const iter_plane &p, int64_t at, float scale, float *x)
{
  u32x4 w;
  if constexpr (kFp8) {
    const u32x2 codes = *reinterpret_cast<const u32x2 *>(static_cast<const uint8_t *>(p.data) + at);
    w[0] = T::template from_e4m3<false>(codes[0], scale);
    w[1] = T::template from_e4m3<true>(codes[0], scale);
    w[2] = T::template from_e4m3<false>(codes[1], scale);
    w[3] = T::template from_e4m3<true>(codes[1], scale);
  } else {
    w = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p.data) + at);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = T::widen(w[i] & 0xFFFFu);
    x[2 * i + 1] = T::widen(w[i] >> 16);
  }
}

// One wave for each (token, query head): a lane scores one key of 64, then the wave adds up the 64 values, a lane for every
// head_dim / 64 elements. Simple and right; every key is read once for every query.
template <class T, int kDim, bool kFp8>
__global__ void __launch_bounds__(64 * kWaves) gnr_attention_kernel(const AttentionParams p)
{
  __shared__ float qs[kWaves][kDim];
  __shared__ int64_t row_v[kWaves][64];
  __shared__ float scale_v[kWaves][64];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int64_t token = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
  if (token >= p.batch.tokens) return;
  const int head = blockIdx.y, kv_head = head / p.group;
  // the request that owns the token, the first if the bounds contradict each other
  int own = -1;
  bool bad = false;
  for (int r0 = 0; r0 < p.batch.requests; r0 += 64) {
    const int r = r0 + lane;
    bool hit = false;
    if (r < p.batch.requests) {
      const int b = p.batch.q_start[r], e = p.batch.q_start[r + 1];
      hit = b <= token && token < e;
      bad |= b < 0 || e < b || e > p.batch.tokens;
    }
    const uint64_t m = __ballot(hit);
    if (m && own < 0) own = r0 + __ffsll(static_cast<unsigned long long>(m)) - 1;
  }
  bad = __any(bad);
  if (own < 0) {
    if (p.status && lane == 0) atomicOr(p.status, ITER_BAD_BATCH);
    return;
  }
  int64_t length = p.batch.kv_len[own];
  const int64_t room = p.batch.table_width << p.page_shift;
  if (length < 0 || length > room) bad = true;
  if (bad && p.status && lane == 0) atomicOr(p.status, ITER_BAD_BATCH);
  const int64_t pos = length - p.batch.q_start[own + 1] + token;
  int64_t end = pos + 1 < room ? pos + 1 : room;
  int64_t begin = p.window ? pos - p.window + 1 : 0;
  begin = begin < 0 ? 0 : begin;
  const uint16_t *q = static_cast<const uint16_t *>(p.q.data) + token * p.q.token_stride + head * p.q.head_stride;
  for (int d = lane; d < kDim; d += 64) qs[wave][d] = T::widen(q[d]) * p.scale_log2;
  __builtin_amdgcn_wave_barrier();
  constexpr int kMine = kDim / 64;
  float acc[kMine] = {};
  float top = -INFINITY, sum = 0.0f;
  for (int64_t j0 = begin; j0 < end; j0 += 64) {
    const int64_t j = j0 + lane;
    float s = -INFINITY;
    int64_t at_v = -1;
    float sv = 1.0f;
    if (j < end) {
      const int64_t page = p.batch.page_table[own * p.batch.table_stride + (j >> p.page_shift)];
      const int64_t place = j & (p.cache.page - 1);
      if (page >= 0 && page < p.cache.pages) {
        const iter_plane &k = p.cache.k, &v = p.cache.v;
        float sk = 1.0f;
        if constexpr (kFp8) {
          sk = exponent_scale(k.exp[page * k.exp_page_stride + kv_head * k.exp_head_stride + place * k.exp_place_stride]);
          sv = exponent_scale(v.exp[page * v.exp_page_stride + kv_head * v.exp_head_stride + place * v.exp_place_stride]);
        }
        const int64_t at = page * k.page_stride + kv_head * k.head_stride + place * k.place_stride;
        at_v = page * v.page_stride + kv_head * v.head_stride + place * v.place_stride;
        float dot = 0.0f;
        for (int d = 0; d < kDim; d += 8) {
          float x[8];
          load8<T, kFp8>(k, at + d, sk, x);
#pragma unroll
          for (int i = 0; i < 8; ++i) dot = __builtin_fmaf(x[i], qs[wave][d + i], dot);
        }
        s = dot;
      } else if (p.status) {
        atomicOr(p.status, ITER_BAD_PAGE);
      }
    }
    row_v[wave][lane] = at_v;
    scale_v[wave][lane] = sv;
    float m = s;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    const float next = fmaxf(top, m);
    const float ref = next == -INFINITY ? 0.0f : next;
    const float w = __builtin_amdgcn_exp2f(s - ref), keep = __builtin_amdgcn_exp2f(top - ref);
    float all = w;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) all += __shfl_xor(all, d);
    sum = __builtin_fmaf(sum, keep, all);
    top = next;
#pragma unroll
    for (int i = 0; i < kMine; ++i) acc[i] *= keep;
    __builtin_amdgcn_wave_barrier();
    for (int l = 0; l < 64; ++l) {
      const int64_t at = row_v[wave][l];
      if (at < 0) continue;
      const float wl = __shfl(w, l);
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        float x;
        if constexpr (kFp8) {
          const uint32_t code = static_cast<const uint8_t *>(p.cache.v.data)[at + lane * kMine + i];
          x = T::widen(T::template from_e4m3<false>(code, scale_v[wave][l]) & 0xFFFFu);
        } else {
          x = T::widen(static_cast<const uint16_t *>(p.cache.v.data)[at + lane * kMine + i]);
        }
        acc[i] = __builtin_fmaf(wl, x, acc[i]);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  uint16_t *out = static_cast<uint16_t *>(p.out.data) + token * p.out.token_stride + head * p.out.head_stride;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const float o = top == -INFINITY ? 0.0f : acc[i] / sum;
    out[lane * kMine + i] = static_cast<uint16_t>(T::narrow2(o, 0.0f));
  }
}

size_t attention_bytes(const iter_cache &, const iter_batch &, int) { return 0; }

template <class T, bool kFp8>
static void launch(const AttentionParams &p, hipStream_t stream)
{
  const dim3 grid(static_cast<unsigned>((p.batch.tokens + kWaves - 1) / kWaves), static_cast<unsigned>(p.heads));
  switch (p.cache.head_dim) {
    case 64: gnr_attention_kernel<T, 64, kFp8><<<grid, 64 * kWaves, 0, stream>>>(p); break;
    case 128: gnr_attention_kernel<T, 128, kFp8><<<grid, 64 * kWaves, 0, stream>>>(p); break;
    default: gnr_attention_kernel<T, 256, kFp8><<<grid, 64 * kWaves, 0, stream>>>(p); break;
  }
}

int launch_attention(const AttentionParams &p, void *stream)
{
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool fp8 = p.cache.type == ITER_FP8;
  if (p.type == ITER_BF16) fp8 ? launch<Bf16, true>(p, s) : launch<Bf16, false>(p, s);
  else fp8 ? launch<Fp16, true>(p, s) : launch<Fp16, false>(p, s);
  return iter_hip_ok(hipGetLastError());
}

}  // namespace gnr
