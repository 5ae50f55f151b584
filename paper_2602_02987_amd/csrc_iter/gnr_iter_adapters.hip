// Low-rank adapters of a batch's requests, added to a projection that they share (gfx950).
#include "gnr_iter_device.h"

namespace gnr {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kTile = 16;              // tokens of a tile: they share an adapter
constexpr int kDepth = 64;             // elements of a row of x that a wave multiplies at a time
constexpr int kColumns = 128;          // columns of the output to a wave

// Sum of a value over the threads before this one, and over all.
__device__ __forceinline__ int scan(int v, int *scratch, int &total)
{
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  int x = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(x, d);
    if (lane >= d) x += o;
  }
  __syncthreads();
  if (lane == 63) scratch[wave] = x;
  __syncthreads();
  int before = x - v;
  total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += scratch[w];
    total += scratch[w];
  }
  return before;
}

// A request's tokens and adapter (`adapters` for none). Numbers out of range are cut down to what is inside.
__device__ __forceinline__ int tokens_of(const AdapterParams &p, int r, int &first, int &which, uint32_t &flags)
{
  const int total = static_cast<int>(p.tokens);
  int b = p.q_start[r], e = p.q_start[r + 1];
  if (b < 0 || e < b || e > total || (r == 0 && b != 0) || (r == p.requests - 1 && e != total)) flags |= ITER_BAD_BATCH;
  b = min(max(b, 0), total);
  e = min(max(e, b), total);
  first = b;
  which = p.adapter[r];
  if (which < -1 || which >= p.set.adapters) flags |= ITER_BAD_ADAPTER;
  if (which < 0 || which >= p.set.adapters) which = p.set.adapters;
  return e - b;
}

// Tokens are taken in tiles of sixteen with the same adapter, in the order of the batch; those without one come last. Every workgroup
// finds its tile from the batch itself. Returns the adapter, or -1 when there are fewer tiles; tokens[i] is -1 beyond the tile's last.
__device__ __forceinline__ int find_tile(const AdapterParams &p, int tile, bool with_none, int *counts, int *tokens, int *scratch)
{
  const int n = p.set.adapters + (with_none ? 1 : 0);
  for (int a = threadIdx.x; a <= p.set.adapters; a += kThreads) counts[a] = 0;
  if (threadIdx.x < kTile) tokens[threadIdx.x] = -1;
  __syncthreads();
  uint32_t flags = 0;
  for (int r = threadIdx.x; r < p.requests; r += kThreads) {
    int first, which;
    const int len = tokens_of(p, r, first, which, flags);
    if (len) atomicAdd(&counts[which], len);   // (whole numbers: the order does not matter)
  }
  if (flags && p.status && blockIdx.x == 0 && blockIdx.y == 0) atomicOr(p.status, flags);
  __syncthreads();
  int mine = -1, at = 0, before = 0;
  for (int a0 = 0; a0 < n; a0 += kThreads) {
    const int a = a0 + threadIdx.x, tiles = a < n ? (counts[a] + kTile - 1) / kTile : 0;
    int total;
    const int start = before + scan(tiles, scratch, total);
    if (tile >= start && tile < start + tiles) {
      mine = a;
      at = (tile - start) * kTile;
    }
    before += total;
  }
  __shared__ int found[2];
  if (threadIdx.x == 0) found[0] = -1;
  __syncthreads();
  if (mine >= 0) {
    found[0] = mine;
    found[1] = at;
  }
  __syncthreads();
  const int which = __builtin_amdgcn_readfirstlane(found[0]), from = __builtin_amdgcn_readfirstlane(found[1]);
  if (which < 0) return -1;
  int done = 0;
  for (int r0 = 0; r0 < p.requests && done < from + kTile; r0 += kThreads) {
    const int r = r0 + threadIdx.x;
    int first = 0, a = -1, len = 0;
    if (r < p.requests) len = tokens_of(p, r, first, a, flags);
    if (a != which) len = 0;
    int total;
    const int rank = done + scan(len, scratch, total);
    for (int i = max(from, rank); i < min(from + kTile, rank + len); ++i) tokens[i - from] = first + i - rank;
    done += total;
  }
  __syncthreads();
  return which;
}

// down x of a tile, over a share of the elements of x: a wave multiplies every fourth 64 of them, H^T = down X^T with the rows of down as the left
// operand, so that no operand passes through shared memory; the waves' sums are added there. Bound by reading x once, and for few tokens by the
// latency of a load or two, which is why the elements are shared out over workgroups until the chip is full.
template <class T, int kRankTiles>
__global__ void __launch_bounds__(kThreads) gnr_adapters_down_kernel(const AdapterParams p)
{
  typedef typename T::oct oct;
  extern __shared__ int counts[];
  __shared__ int tokens[kTile], scratch[kWaves];
  __shared__ float sums[kWaves][kRankTiles * 16][kTile + 1];
  const int which = find_tile(p, blockIdx.x, false, counts, tokens, scratch);
  if (which < 0) return;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, n = lane % 16, g = lane / 16;
  const int rank = p.set.rank, width = static_cast<int>(p.set.width_in), token = tokens[n];
  const uint16_t *x = static_cast<const uint16_t *>(p.x) + static_cast<int64_t>(max(token, 0)) * p.x_stride;
  const uint16_t *down = static_cast<const uint16_t *>(p.set.down) + static_cast<int64_t>(which) * rank * width;
  const int blocks = (width + kDepth - 1) / kDepth, each = (blocks + gridDim.y - 1) / gridDim.y;
  const int end = min(blocks, static_cast<int>(blockIdx.y + 1) * each);
  f32x4 acc[kRankTiles];
#pragma unroll
  for (int i = 0; i < kRankTiles; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int block = blockIdx.y * each + wave; block < end; block += kWaves) {
#pragma unroll
    for (int half = 0; half < kDepth / 32; ++half) {
      const int d = block * kDepth + half * 32 + 8 * g;
      const bool in = d < width;
      u32x4 b = {0, 0, 0, 0};
      if (in && token >= 0) b = *reinterpret_cast<const u32x4 *>(x + d);
#pragma unroll
      for (int i = 0; i < kRankTiles; ++i) {
        u32x4 a = {0, 0, 0, 0};
        if (in && 16 * i + n < rank) a = *reinterpret_cast<const u32x4 *>(down + static_cast<int64_t>(16 * i + n) * width + d);
        acc[i] = T::mfma16(bits<oct>(a), bits<oct>(b), acc[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kRankTiles; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) sums[wave][16 * i + 4 * g + k][n] = acc[i][k];
  __syncthreads();
  for (int i = threadIdx.x; i < kTile * rank; i += kThreads) {
    const int t = i / rank, r = i % rank;
    if (tokens[t] < 0) break;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += sums[w][r][t];
    p.workspace[(static_cast<int64_t>(blockIdx.y) * p.tokens + tokens[t]) * rank + r] = s;
  }
}

// out = base + scale up h of a tile, 128 columns to a wave: Y^T = up H^T with 16 rows of up at a time as the left operand. h is in 32 bits; it goes
// into the product as the sum of two 16-bit numbers, relative to a power of two near the token's largest, so that neither type's range nor
// its precision shows. The rows of up that a product takes are chosen so that a lane ends up with 32 neighbouring columns of its token: base
// and out are read and written 16 bytes at a time. Bound by these two.
template <class T, int kRankSteps>
__global__ void __launch_bounds__(kThreads) gnr_adapters_up_kernel(const AdapterParams p, int splits)
{
  typedef typename T::oct oct;
  constexpr int kProducts = kColumns / 16, kRun = kColumns / 4;
  extern __shared__ int counts[];
  __shared__ int tokens[kTile], scratch[kWaves];
  __shared__ float h[kTile][kRankSteps * 32 + 4];
  const int which = find_tile(p, blockIdx.x, true, counts, tokens, scratch);
  if (which < 0) return;
  const bool none = which == p.set.adapters;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, n = lane % 16, g = lane / 16;
  const int rank = p.set.rank, width = static_cast<int>(p.set.width_out), token = tokens[n];
  if (!none) {
    for (int i = threadIdx.x; i < kTile * kRankSteps * 32; i += kThreads) {
      const int t = i / (kRankSteps * 32), r = i % (kRankSteps * 32);
      float s = 0.0f;
      if (r < rank && tokens[t] >= 0)
        for (int k = 0; k < splits; ++k) s += p.workspace[(static_cast<int64_t>(k) * p.tokens + tokens[t]) * rank + r];
      h[t][r] = s;
    }
    __syncthreads();
  }
  const int column0 = (blockIdx.y * kWaves + wave) * kColumns, column = column0 + g * kRun;
  f32x4 acc[kProducts];
#pragma unroll
  for (int j = 0; j < kProducts; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float factor = 0.0f;
  if (!none) {
    float most = 0.0f;
    for (int i = 0; i < kRankSteps; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) most = fmaxf(most, __builtin_fabsf(h[n][32 * i + 8 * g + k]));
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    // 2^-e with most = m 2^e, m in [1, 2); none for what has no such e
    const uint32_t e = bits<uint32_t>(most) >> 23;
    const bool plain = e < 1 || e > 253;
    const float shrink = plain ? 1.0f : bits<float>((254 - e) << 23), grow = plain ? 1.0f : bits<float>(e << 23);
    factor = p.set.scale[which] * grow;
    const uint16_t *up = static_cast<const uint16_t *>(p.set.up) + static_cast<int64_t>(which) * width * rank;
#pragma unroll
    for (int i = 0; i < kRankSteps; ++i) {
      u32x4 hi, lo;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float a = h[n][32 * i + 8 * g + 2 * k] * shrink, b = h[n][32 * i + 8 * g + 2 * k + 1] * shrink;
        hi[k] = T::narrow2(a, b);
        const float c = a - T::widen(hi[k] & 0xFFFFu), d = b - T::widen(hi[k] >> 16);
        lo[k] = T::narrow2(c == c ? c : 0.0f, d == d ? d : 0.0f);   // (an infinity is its own upper part)
      }
#pragma unroll
      for (int j = 0; j < kProducts; ++j) {
        const int row = column0 + n / 4 * kRun + 4 * j + n % 4, r = 32 * i + 8 * g;
        u32x4 a = {0, 0, 0, 0};
        if (row < width && r < rank) a = *reinterpret_cast<const u32x4 *>(up + static_cast<int64_t>(row) * rank + r);
        acc[j] = T::mfma16(bits<oct>(a), bits<oct>(hi), acc[j]);
        acc[j] = T::mfma16(bits<oct>(a), bits<oct>(lo), acc[j]);
      }
    }
  }
  if (token < 0) return;
  const uint16_t *base = static_cast<const uint16_t *>(p.base) + static_cast<int64_t>(token) * p.base_stride;
  uint16_t *out = static_cast<uint16_t *>(p.out) + static_cast<int64_t>(token) * p.out_stride;
#pragma unroll
  for (int j = 0; j < kProducts; j += 2) {
    const int c = column + 4 * j;
    if (c >= width) break;
    u32x4 y = *reinterpret_cast<const u32x4 *>(base + c);
    if (!none) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float a = acc[j + k / 2][2 * (k % 2)], b = acc[j + k / 2][2 * (k % 2) + 1];
        y[k] = T::narrow2(__builtin_fmaf(a, factor, T::widen(y[k] & 0xFFFFu)), __builtin_fmaf(b, factor, T::widen(y[k] >> 16)));
      }
    }
    *reinterpret_cast<u32x4 *>(out + c) = y;
  }
}

static int tiles_bound(const iter_adapter_set &s, int requests, int64_t tokens, bool with_none)
{
  // tiles that are full, and for every adapter in use one that is not
  const int64_t used = (requests < s.adapters ? requests : s.adapters) + (with_none ? 1 : 0);
  return static_cast<int>(tokens / kTile + (used < tokens ? used : tokens));
}

// Shares of the elements of x: enough that few tiles fill the chip, at least two blocks to a wave.
static int splits_for(const iter_adapter_set &s, int64_t tokens)
{
  const int64_t tiles = (tokens + kTile - 1) / kTile, depth = s.width_in / (2 * kDepth * kWaves);
  int64_t n = 512 / (tiles < 1 ? 1 : tiles);
  n = n < depth ? n : depth;
  return static_cast<int>(n < 1 ? 1 : n < 16 ? n : 16);
}

size_t adapters_bytes(const iter_adapter_set &s, int64_t tokens)
{
  return static_cast<size_t>(splits_for(s, tokens)) * static_cast<size_t>(tokens) * static_cast<size_t>(s.rank) * sizeof(float);
}

template <class T>
static int launch(const AdapterParams &p, hipStream_t s)
{
  const size_t lds = static_cast<size_t>(p.set.adapters + 1) * sizeof(int);
  const int splits = splits_for(p.set, p.tokens);
  const dim3 down(static_cast<unsigned>(tiles_bound(p.set, p.requests, p.tokens, false)), static_cast<unsigned>(splits));
  const dim3 up(static_cast<unsigned>(tiles_bound(p.set, p.requests, p.tokens, true)), static_cast<unsigned>((p.set.width_out + kColumns * kWaves - 1) / (kColumns * kWaves)));
  if (p.set.adapters > 0) {
    if (p.set.rank <= 16) gnr_adapters_down_kernel<T, 1><<<down, kThreads, lds, s>>>(p);
    else if (p.set.rank <= 32) gnr_adapters_down_kernel<T, 2><<<down, kThreads, lds, s>>>(p);
    else if (p.set.rank <= 64) gnr_adapters_down_kernel<T, 4><<<down, kThreads, lds, s>>>(p);
    else gnr_adapters_down_kernel<T, 8><<<down, kThreads, lds, s>>>(p);
    const int rc = iter_hip_ok(hipGetLastError());
    if (rc != SIM_OK) return rc;
  }
  if (p.set.rank <= 32) gnr_adapters_up_kernel<T, 1><<<up, kThreads, lds, s>>>(p, splits);
  else if (p.set.rank <= 64) gnr_adapters_up_kernel<T, 2><<<up, kThreads, lds, s>>>(p, splits);
  else gnr_adapters_up_kernel<T, 4><<<up, kThreads, lds, s>>>(p, splits);
  return iter_hip_ok(hipGetLastError());
}

int launch_adapters(const AdapterParams &p, void *stream)
{
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return p.type == ITER_BF16 ? launch<Bf16>(p, s) : launch<Fp16>(p, s);
}

}  // namespace gnr
