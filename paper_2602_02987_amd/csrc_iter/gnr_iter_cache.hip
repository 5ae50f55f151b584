// Writing rows into the paged cache, in 8 bits or as they are, and reading them back (gfx950).
#include "gnr_iter_device.h"

namespace gnr {

constexpr int kThreads = 256;
// From here on a workgroup takes four heads (two and eight measure the same) and a read's results, more than the caches hold, are stored past them: 98309 tokens
// of 8 heads are read back in 103 us (5.9 TB/s) instead of 142, 115 without the stores; 8191 tokens are written in 9.5 us instead of 10.7. With fewer rows
// four heads leave compute units idle.
constexpr int kManyHeads = 4;
constexpr int64_t kManyRows = 1 << 15;

// Both kernels: a row is held by head_dim / 8 neighbouring lanes, 16 bytes of 16-bit values each; a workgroup takes the rows
// of kHeads neighbouring heads (of the keys or of the values) for a few neighbouring tokens, and the workgroups of other heads of the same tokens
// run beside it: what is written to or read from the tokens' side is then whole rows of all heads. They stream: every byte is touched
// once, and what bounds them is the memory.
struct CacheJob {
  iter_cache cache;
  iter_rows k, v;
  const int64_t *slots;
  int64_t tokens;
  int page_shift;
};

template <int kDim, int kHeads>
struct RowsOf {
  static constexpr int kLanes = kDim / 8, kRows = kThreads / kLanes;
  const bool values;
  const int head, lane;                                         // the first head
  const int64_t token, slot;
  bool there;
  int64_t at, exp_at;
  __device__ __forceinline__ RowsOf(const CacheJob &j)
      : values(blockIdx.x * kHeads >= static_cast<unsigned>(j.cache.kv_heads)),
        head(blockIdx.x * kHeads - (values ? j.cache.kv_heads : 0)), lane(threadIdx.x % kLanes),
        token((static_cast<int64_t>(blockIdx.z) * gridDim.y + blockIdx.y) * kRows + threadIdx.x / kLanes), slot(token < j.tokens ? j.slots[token] : -1)
  {
    const iter_plane &p = values ? j.cache.v : j.cache.k;
    const int64_t page = slot >> j.page_shift, place = slot & (j.cache.page - 1);
    there = slot >= 0 && page < j.cache.pages;
    at = page * p.page_stride + head * p.head_stride + place * p.place_stride + lane * 8;
    exp_at = page * p.exp_page_stride + head * p.exp_head_stride + place * p.exp_place_stride;
  }
};

// A row's 16-bit values in units of 2^e: codes and the byte of e (all lanes of the row take part).
template <class T, int kLanes>
__device__ __forceinline__ u32x2 quantise(u32x4 x, uint8_t &exp)
{
  // the largest magnitude: without the sign, the bits of both types are in the order of their values, NaN above infinity
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = x[i] & 0x7FFFu, hi = (x[i] >> 16) & 0x7FFFu;
    most = most > lo ? most : lo;
    most = most > hi ? most : hi;
  }
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) {
    const uint32_t o = __shfl_xor(most, d);
    most = most > o ? most : o;
  }
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
  exp = static_cast<uint8_t>(e + 127);
  return codes;
}

template <class T, int kDim, bool kFp8, int kHeads>
__global__ void __launch_bounds__(kThreads) gnr_kv_write_kernel(const CacheJob j)
{
  typedef RowsOf<kDim, kHeads> Rows;
  const Rows r(j);
  const iter_rows &src = r.values ? j.v : j.k;
  const iter_plane &dst = r.values ? j.cache.v : j.cache.k;
  u32x4 x[kHeads];
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    x[h] = u32x4{0, 0, 0, 0};
    if (r.there)
      x[h] = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(src.data) + r.token * src.token_stride + (r.head + h) * src.head_stride + r.lane * 8);
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    if constexpr (!kFp8) {
      if (r.there) *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(dst.data) + r.at + h * dst.head_stride) = x[h];
    } else {
      uint8_t exp;
      const u32x2 codes = quantise<T, Rows::kLanes>(x[h], exp);
      if (r.there) {
        *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(dst.data) + r.at + h * dst.head_stride) = codes;
        if (r.lane == 0) dst.exp[r.exp_at + h * dst.exp_head_stride] = exp;
      }
    }
  }
}

template <class T, int kDim, bool kFp8, int kHeads>
__global__ void __launch_bounds__(kThreads) gnr_kv_read_kernel(const CacheJob j)
{
  typedef RowsOf<kDim, kHeads> Rows;
  const Rows r(j);
  if (r.token >= j.tokens) return;
  const iter_rows &dst = r.values ? j.v : j.k;
  const iter_plane &src = r.values ? j.cache.v : j.cache.k;
  u32x4 x[kHeads];
  u32x2 codes[kHeads];
  uint8_t exp[kHeads];
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    x[h] = u32x4{0, 0, 0, 0};
    if constexpr (kFp8) {
      codes[h] = u32x2{0, 0};
      exp[h] = 127;
      if (r.there) {
        codes[h] = *reinterpret_cast<const u32x2 *>(static_cast<const uint8_t *>(src.data) + r.at + h * src.head_stride);
        exp[h] = src.exp[r.exp_at + h * src.exp_head_stride];
      }
    } else {
      if (r.there) x[h] = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(src.data) + r.at + h * src.head_stride);
    }
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    if constexpr (kFp8) {
      const float scale = exponent_scale(exp[h]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[h][2 * i] = T::template from_e4m3<false>(codes[h][i], scale);
        x[h][2 * i + 1] = T::template from_e4m3<true>(codes[h][i], scale);
      }
    }
    u32x4 *to = reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(dst.data) + r.token * dst.token_stride + (r.head + h) * dst.head_stride + r.lane * 8);
    if constexpr (kHeads > 1) __builtin_nontemporal_store(x[h], to);
    else *to = x[h];
  }
}

template <class T, int kDim, bool kFp8, int kHeads>
static int launch_cache_heads(bool write, const CacheJob &j, hipStream_t stream)
{
  constexpr int rows = RowsOf<kDim, kHeads>::kRows;
  const int64_t blocks = (j.tokens + rows - 1) / rows, y = blocks < 32768 ? blocks : 32768;
  const dim3 grid(2u * static_cast<unsigned>(j.cache.kv_heads) / kHeads, static_cast<unsigned>(y), static_cast<unsigned>((blocks + y - 1) / y));
  if (write) gnr_kv_write_kernel<T, kDim, kFp8, kHeads><<<grid, kThreads, 0, stream>>>(j);
  else gnr_kv_read_kernel<T, kDim, kFp8, kHeads><<<grid, kThreads, 0, stream>>>(j);
  return iter_hip_ok(hipGetLastError());
}

template <class T, int kDim, bool kFp8>
static int launch_cache(bool write, const CacheJob &j, hipStream_t stream)
{
  if (j.cache.kv_heads % kManyHeads == 0 && j.tokens * j.cache.kv_heads >= kManyRows) return launch_cache_heads<T, kDim, kFp8, kManyHeads>(write, j, stream);
  return launch_cache_heads<T, kDim, kFp8, 1>(write, j, stream);
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
