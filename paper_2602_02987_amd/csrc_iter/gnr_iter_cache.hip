// Writing rows into the paged cache, in 8 bits or as they are, and reading them back (gfx950).
#include "gnr_iter_device.h"

namespace gnr {

constexpr int kThreads = 256;

// Both kernels: a row is held by head_dim / 8 neighbouring lanes, 16 bytes of 16-bit values each; a workgroup takes the rows
// of one head (of the keys or of the values) for a few neighbouring tokens, whose exponents and, in a cache laid out by heads, whose
// rows are neighbours in memory too. They stream: every byte is touched once, and what bounds them is the memory.
struct CacheJob {
  iter_cache cache;
  iter_rows k, v;
  const int64_t *slots;
  int64_t tokens;
  int page_shift;
};

template <int kDim>
struct RowOf {
  static constexpr int kLanes = kDim / 8, kRows = kThreads / kLanes;
  const bool values;
  const int head, lane;
  const int64_t token, slot;
  bool there;
  int64_t at, exp_at;
  __device__ __forceinline__ RowOf(const CacheJob &j)
      : values(blockIdx.y >= static_cast<unsigned>(j.cache.kv_heads)),
        head(blockIdx.y - (values ? j.cache.kv_heads : 0)), lane(threadIdx.x % kLanes),
        token(static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kLanes), slot(token < j.tokens ? j.slots[token] : -1)
  {
    const iter_plane &p = values ? j.cache.v : j.cache.k;
    const int64_t page = slot >> j.page_shift, place = slot & (j.cache.page - 1);
    there = slot >= 0 && page < j.cache.pages;
    at = page * p.page_stride + head * p.head_stride + place * p.place_stride + lane * 8;
    exp_at = page * p.exp_page_stride + head * p.exp_head_stride + place * p.exp_place_stride;
  }
};

template <class T, int kDim, bool kFp8>
__global__ void __launch_bounds__(kThreads) gnr_kv_write_kernel(const CacheJob j)
{
  typedef RowOf<kDim> Row;
  const Row r(j);
  const iter_rows &src = r.values ? j.v : j.k;
  const iter_plane &dst = r.values ? j.cache.v : j.cache.k;
  u32x4 x = {0, 0, 0, 0};
  if (r.there)
    x = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(src.data) + r.token * src.token_stride + r.head * src.head_stride + r.lane * 8);
  if constexpr (!kFp8) {
    if (r.there) *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(dst.data) + r.at) = x;
  } else {
    // the largest magnitude: without the sign, the bits of both types are in the order of their values, NaN above infinity
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = x[i] & 0x7FFFu, hi = (x[i] >> 16) & 0x7FFFu;
      most = most > lo ? most : lo;
      most = most > hi ? most : hi;
    }
#pragma unroll
    for (int d = 1; d < Row::kLanes; d *= 2) {
      const uint32_t o = __shfl_xor(most, d);
      most = most > o ? most : o;
    }
    if (!r.there) return;
    // most = m * 2^x with m in [1, 2), 448 = 1.75 * 2^8: the row fits with e = x - 8, or x - 7 if m > 1.75
    const uint32_t w = bits<uint32_t>(T::widen(most));
    int e = static_cast<int>(w >> 23) - 127 - 8 + ((w & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    e = e < -126 ? -126 : e;
    const bool finite = most < T::kInf;
    if (most == 0 || !finite) e = 0;
    const float scale = exponent_scale(static_cast<uint32_t>(e + 127));
    u32x2 codes;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s16x2 c = {0, 0};
      c = T::template to_e4m3<false>(c, x[2 * i], scale);
      c = T::template to_e4m3<true>(c, x[2 * i + 1], scale);
      codes[i] = finite ? bits<uint32_t>(c) : 0x7F7F7F7Fu;
    }
    *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(dst.data) + r.at) = codes;
    if (r.lane == 0) dst.exp[r.exp_at] = static_cast<uint8_t>(e + 127);
  }
}

template <class T, int kDim, bool kFp8>
__global__ void __launch_bounds__(kThreads) gnr_kv_read_kernel(const CacheJob j)
{
  typedef RowOf<kDim> Row;
  const Row r(j);
  if (r.token >= j.tokens) return;
  const iter_rows &dst = r.values ? j.v : j.k;
  const iter_plane &src = r.values ? j.cache.v : j.cache.k;
  u32x4 x = {0, 0, 0, 0};
  if (r.there) {
    if constexpr (kFp8) {
      const u32x2 codes = *reinterpret_cast<const u32x2 *>(static_cast<const uint8_t *>(src.data) + r.at);
      const float scale = exponent_scale(src.exp[r.exp_at]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[2 * i] = T::template from_e4m3<false>(codes[i], scale);
        x[2 * i + 1] = T::template from_e4m3<true>(codes[i], scale);
      }
    } else {
      x = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(src.data) + r.at);
    }
  }
  *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(dst.data) + r.token * dst.token_stride + r.head * dst.head_stride + r.lane * 8) = x;
}

template <class T, int kDim, bool kFp8>
static int launch_cache(bool write, const CacheJob &j, hipStream_t stream)
{
  constexpr int rows = RowOf<kDim>::kRows;
  const dim3 grid(static_cast<unsigned>((j.tokens + rows - 1) / rows), 2u * static_cast<unsigned>(j.cache.kv_heads));
  if (write) gnr_kv_write_kernel<T, kDim, kFp8><<<grid, kThreads, 0, stream>>>(j);
  else gnr_kv_read_kernel<T, kDim, kFp8><<<grid, kThreads, 0, stream>>>(j);
  return iter_hip_ok(hipGetLastError());
}

template <class T, bool kFp8>
static int launch_cache_dim(bool write, const CacheJob &j, hipStream_t stream)
{
  switch (j.cache.head_dim) {
    case 64: return launch_cache<T, 64, kFp8>(write, j, stream);
    case 128: return launch_cache<T, 128, kFp8>(write, j, stream);
    default: return launch_cache<T, 256, kFp8>(write, j, stream);
  }
}

static int launch_cache_job(bool write, const iter_cache &c, int type, const iter_rows &k, const iter_rows &v, const int64_t *slots,
                            int64_t tokens, void *stream)
{
  const CacheJob j{c, k, v, slots, tokens, __builtin_ctz(static_cast<unsigned>(c.page))};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (c.type != ITER_FP8) return launch_cache_dim<Bf16, false>(write, j, s);   // 16 bits as they are, whatever they mean
  return type == ITER_BF16 ? launch_cache_dim<Bf16, true>(write, j, s) : launch_cache_dim<Fp16, true>(write, j, s);
}

int launch_kv_write(const iter_cache &c, int type, const iter_rows &k, const iter_rows &v, const int64_t *slots, int64_t tokens, void *stream)
{
  return launch_cache_job(true, c, type, k, v, slots, tokens, stream);
}

int launch_kv_read(const iter_cache &c, int type, const iter_rows &k, const iter_rows &v, const int64_t *slots, int64_t tokens, void *stream)
{
  return launch_cache_job(false, c, type, k, v, slots, tokens, stream);
}

}  // namespace gnr
