// Low-rank adapters of a batch's requests, added to a projection that they share (gfx950).
#include "gnr_iter_device.h"

namespace gnr {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kDepth = 64;             // elements of a row of x that a wave multiplies at a time
constexpr int kColumns = 128;          // columns of the output to a wave
constexpr int kManyTokens = 2048;      // from here on a tile has 64 tokens instead of 16 (see the kernels; 8191 tokens: 128 -> 97 us)

// A request's tokens and adapter (`adapters` for none). Numbers out of range are cut down to what is inside.
__device__ __forceinline__ int tokens_of(const AdapterParams &p, int r, int &which, uint32_t &flags)
{
  const int total = static_cast<int>(p.tokens);
  int b = p.q_start[r], e = p.q_start[r + 1];
  which = p.adapter[r];
  if (b < 0 || e < b || e > total || (r == 0 && b != 0) || (r == p.requests - 1 && e != total)) flags |= ITER_BAD_BATCH;
  if (which < -1 || which >= p.set.adapters) flags |= ITER_BAD_ADAPTER;
  if (which < 0 || which >= p.set.adapters) which = p.set.adapters;
  b = min(max(b, 0), total);
  return min(max(e, b), total) - b;
}

__device__ __forceinline__ int wave_scan(int v)   // of the lanes up to this one
{
  const int lane = threadIdx.x % 64;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// Tokens are taken in tiles with the same adapter, in the order of the batch; those without one come last. Every workgroup finds its tile
// from the batch itself, every wave for itself once the numbers are in shared memory (a barrier costs more). Returns the adapter, or
// -1 when there are fewer tiles; tokens[i] is -1 beyond the tile's last. numbers: shared, adapters + 1 and two for each request.
template <int kTile, int kCount = kThreads>
__device__ __forceinline__ int find_tile(const AdapterParams &p, int tile, bool with_none, int *numbers, int *tokens)
{
  const int all = p.set.adapters + 1, n = p.requests, lane = threadIdx.x % 64;
  int *counts = numbers, *lens = numbers + all, *whose = lens + n;
  uint32_t flags = 0;
  for (int a = threadIdx.x; a < all; a += kCount) counts[a] = 0;
  for (int r = threadIdx.x; r < n; r += kCount) {
    int which;
    lens[r] = tokens_of(p, r, which, flags);
    whose[r] = which;
  }
  if (threadIdx.x < kTile) tokens[threadIdx.x] = -1;
  __syncthreads();
  for (int r = threadIdx.x; r < n; r += kCount)
    if (lens[r]) atomicAdd(&counts[whose[r]], lens[r]);   // (whole numbers: the order does not matter)
  if (flags && p.status && blockIdx.x == 0 && blockIdx.y == 0) atomicOr(p.status, flags);
  __syncthreads();
  int which = -1, from = 0, before = 0;
  for (int a0 = 0; a0 < all - (with_none ? 0 : 1) && which < 0; a0 += 64) {
    const int a = a0 + lane, tiles = a < all - (with_none ? 0 : 1) ? (counts[a] + kTile - 1) / kTile : 0, end = before + wave_scan(tiles);
    const uint64_t mine = __ballot(tile < end && tile >= end - tiles);
    if (mine) {
      const int l = __ffsll(static_cast<unsigned long long>(mine)) - 1;
      which = a0 + l;
      from = (tile - __shfl(end - tiles, l)) * kTile;
    }
    before = __shfl(end, 63);
  }
  if (which < 0) return -1;
  if (threadIdx.x < 64) {
    int done = 0;
    for (int r0 = 0; r0 < n && done < from + kTile; r0 += 64) {
      const int r = r0 + lane, len = r < n && whose[r] == which ? lens[r] : 0, end = done + wave_scan(len);
      if (len && end > from && end - len < from + kTile) {
        const int first = min(max(p.q_start[r], 0), static_cast<int>(p.tokens));
        for (int i = max(from, end - len); i < min(from + kTile, end); ++i) tokens[i - from] = first + i - (end - len);
      }
      done = __shfl(end, 63);
    }
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(which);
}

// down x of a tile of 16 kSub tokens, over a share of the elements of x: a wave multiplies every fourth 64 of them, H^T = down X^T with the rows
// of down as the left operand, so that no operand passes through shared memory; the waves' sums are added there. Bound by reading x once, and
// for few tokens by the latency of a load or two, which is why the elements are shared out over workgroups until the chip is full. Of many tokens
// a tile takes 64, so that a row of down is read once for them. 8191 tokens, width 4096,
// rank 32: 22 us (3.1 TB/s); 128 tokens: 6 us. Asking for the next elements before these are multiplied changes nothing.
template <class T, int kRankTiles, int kSub>
__global__ void __launch_bounds__(kThreads) gnr_adapters_down_kernel(const AdapterParams p)
{
  typedef typename T::oct oct;
  constexpr int kTile = 16 * kSub;
  extern __shared__ int numbers[];
  __shared__ int tokens[kTile];
  __shared__ float sums[kWaves][kRankTiles * 16][17];
  const int which = find_tile<kTile>(p, blockIdx.y, false, numbers, tokens);
  if (which < 0) return;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, n = lane % 16, g = lane / 16;
  const int rank = p.set.rank, width = static_cast<int>(p.set.width_in);
  const uint16_t *x[kSub];
#pragma unroll
  for (int s = 0; s < kSub; ++s) x[s] = static_cast<const uint16_t *>(p.x) + static_cast<int64_t>(max(tokens[16 * s + n], 0)) * p.x_stride;   // (what is beyond the tile's last is not kept)
  const uint16_t *down = static_cast<const uint16_t *>(p.set.down) + static_cast<int64_t>(which) * rank * width;
  const int blocks = (width + kDepth - 1) / kDepth, each = (blocks + gridDim.x - 1) / gridDim.x;
  const int end = min(blocks, static_cast<int>(blockIdx.x + 1) * each);
  f32x4 acc[kSub][kRankTiles];
#pragma unroll
  for (int s = 0; s < kSub; ++s)
#pragma unroll
    for (int i = 0; i < kRankTiles; ++i) acc[s][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int block = blockIdx.x * each + wave; block < end; block += kWaves) {
    u32x4 a[2][kRankTiles], b[2][kSub];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int d = block * kDepth + half * 32 + 8 * g;
      const bool in = d < width;
#pragma unroll
      for (int s = 0; s < kSub; ++s) {
        b[half][s] = u32x4{0, 0, 0, 0};
        if (in) b[half][s] = *reinterpret_cast<const u32x4 *>(x[s] + d);
      }
#pragma unroll
      for (int i = 0; i < kRankTiles; ++i) {
        a[half][i] = u32x4{0, 0, 0, 0};
        if (in && 16 * i + n < rank) a[half][i] = *reinterpret_cast<const u32x4 *>(down + static_cast<int64_t>(16 * i + n) * width + d);
      }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int i = 0; i < kRankTiles; ++i) acc[s][i] = T::mfma16(bits<oct>(a[half][i]), bits<oct>(b[half][s]), acc[s][i]);
  }
#pragma unroll
  for (int s = 0; s < kSub; ++s) {
    if (s) __syncthreads();
#pragma unroll
    for (int i = 0; i < kRankTiles; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) sums[wave][16 * i + 4 * g + k][n] = acc[s][i][k];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * rank; i += kThreads) {
      const int t = i / rank, r = i % rank, token = tokens[16 * s + t];
      if (token < 0) break;
      float h = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) h += sums[w][r][t];
      p.workspace[(static_cast<int64_t>(blockIdx.x) * p.tokens + token) * rank + r] = h;
    }
  }
}

// up h of 16 tokens for kCols columns of a wave: Y^T = up H^T with 16 rows of up at a time as the left operand. h is in 32 bits; it goes
// into the product as the sum of two 16-bit numbers, relative to a power of two near the token's largest, so that neither type's range nor
// its precision shows. The rows of up that two products take are chosen so that a lane ends up with eight neighbouring columns of its token, and the four
// lanes of a token with 32: base and out are read and written 16 bytes a lane, 64 a token.
template <class T, int kRankSteps, int kCols>
struct Columns {
  typedef typename T::oct oct;
  static constexpr int kProducts = kCols / 16, kLoads = kCols / 32;
  const int n, g, column0, column, width;                       // column: this lane's first, 32 on for the next load
  u32x4 rows[kRankSteps][kProducts];

  __device__ __forceinline__ Columns(int lane, int first, int all) : n(lane % 16), g(lane / 16), column0(first), column(first + 8 * g), width(all) {}

  __device__ __forceinline__ void load_rows(const AdapterParams &p, int which)
  {
    const int rank = p.set.rank;
    const uint16_t *up = static_cast<const uint16_t *>(p.set.up) + static_cast<int64_t>(which) * width * rank;
#pragma unroll
    for (int i = 0; i < kRankSteps; ++i)
#pragma unroll
      for (int j = 0; j < kProducts; ++j) {
        const int row = column0 + 32 * (j / 2) + 8 * (n / 4) + 4 * (j % 2) + n % 4, r = 32 * i + 8 * g;
        rows[i][j] = u32x4{0, 0, 0, 0};
        if (row < width && r < rank) rows[i][j] = *reinterpret_cast<const u32x4 *>(up + static_cast<int64_t>(row) * rank + r);
      }
  }

  __device__ __forceinline__ void load_base(const AdapterParams &p, int token, u32x4 (&y)[kLoads]) const
  {
    const uint16_t *base = static_cast<const uint16_t *>(p.base) + static_cast<int64_t>(max(token, 0)) * p.base_stride;
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      if (column + 32 * j < width) y[j] = *reinterpret_cast<const u32x4 *>(base + column + 32 * j);
  }

  // z += by * up h for this lane's token, h (32 kRankSteps numbers) in shared memory
  __device__ __forceinline__ void add(const float *h, float by, u32x4 (&z)[kLoads]) const
  {
    float v[kRankSteps][8], most = 0.0f;
#pragma unroll
    for (int i = 0; i < kRankSteps; ++i) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(h + 32 * i + 8 * g + 4 * k);
#pragma unroll
        for (int l = 0; l < 4; ++l) {
          v[i][4 * k + l] = x[l];
          most = fmaxf(most, __builtin_fabsf(x[l]));
        }
      }
    }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    // 2^-e with most = m 2^e, m in [1, 2); none for what has no such e
    const uint32_t e = bits<uint32_t>(most) >> 23;
    const bool plain = e < 1 || e > 253;
    const float shrink = plain ? 1.0f : bits<float>((254 - e) << 23);
    const float factor = by * (plain ? 1.0f : bits<float>(e << 23));
    f32x4 acc[kProducts];
#pragma unroll
    for (int j = 0; j < kProducts; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kRankSteps; ++i) {
      u32x4 hi, lo;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float a = v[i][2 * k] * shrink, b = v[i][2 * k + 1] * shrink;
        hi[k] = T::narrow2(a, b);
        const float c = a - T::widen(hi[k] & 0xFFFFu), d = b - T::widen(hi[k] >> 16);
        lo[k] = T::narrow2(c == c ? c : 0.0f, d == d ? d : 0.0f);   // (an infinity is its own upper part)
      }
#pragma unroll
      for (int j = 0; j < kProducts; ++j) {
        acc[j] = T::mfma16(bits<oct>(rows[i][j]), bits<oct>(hi), acc[j]);
        acc[j] = T::mfma16(bits<oct>(rows[i][j]), bits<oct>(lo), acc[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float a = acc[2 * j + k / 2][2 * (k % 2)], b = acc[2 * j + k / 2][2 * (k % 2) + 1];
        z[j][k] = T::narrow2(__builtin_fmaf(a, factor, T::widen(z[j][k] & 0xFFFFu)), __builtin_fmaf(b, factor, T::widen(z[j][k] >> 16)));
      }
  }

  __device__ __forceinline__ void store(const AdapterParams &p, int token, const u32x4 (&z)[kLoads]) const
  {
    uint16_t *out = static_cast<uint16_t *>(p.out) + static_cast<int64_t>(max(token, 0)) * p.out_stride;
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      if (token >= 0 && column + 32 * j < width) *reinterpret_cast<u32x4 *>(out + column + 32 * j) = z[j];
  }
};

// out = base + scale up h of a tile, 128 columns to a wave. Bound by reading base and writing out; base and the rows of up are asked for
// before h is added up. 8191 tokens, width 6144, rank 32: 48 us (4.2 TB/s).
template <class T, int kRankSteps, int kSub>
__global__ void __launch_bounds__(kThreads, kRankSteps == 4 ? 2 : 3) gnr_adapters_up_kernel(const AdapterParams p, int splits)
{
  typedef Columns<T, kRankSteps, kColumns> Mine;
  constexpr int kTile = 16 * kSub, kPitch = kRankSteps * 32 + 4;
  extern __shared__ int numbers[];
  __shared__ int tokens[kTile];
  __shared__ __attribute__((aligned(16))) float h[kTile][kPitch];
  const int which = find_tile<kTile>(p, blockIdx.y, true, numbers, tokens);
  if (which < 0) return;
  const bool none = which == p.set.adapters;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, rank = p.set.rank;
  Mine mine(lane, (blockIdx.x * kWaves + wave) * kColumns, static_cast<int>(p.set.width_out));
  // base of all of the tile's tokens where there is room in registers (whole prompt 81 -> 77 us), else of sixteen at a time
  constexpr int kBuffers = kRankSteps == 1 ? kSub : 1;
  u32x4 y[kBuffers][Mine::kLoads];
#pragma unroll
  for (int s = 0; s < kBuffers; ++s) mine.load_base(p, tokens[16 * s + mine.n], y[s]);
  float by = 0.0f;
  if (!none) {
    mine.load_rows(p, which);
    by = p.set.scale[which];
    for (int i = threadIdx.x; i < kTile * kRankSteps * 8; i += kThreads) {
      const int t = i / (kRankSteps * 8), r = i % (kRankSteps * 8) * 4, token = tokens[t];
      f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
      if (r < rank && token >= 0) {
        const float *from = p.workspace + static_cast<int64_t>(token) * rank + r;
#pragma unroll 4
        for (int k = 0; k < splits; ++k) sum += *reinterpret_cast<const f32x4 *>(from + static_cast<int64_t>(k) * p.tokens * rank);
      }
      *reinterpret_cast<f32x4 *>(&h[t][r]) = sum;
    }
    __syncthreads();
  }
#pragma unroll
  for (int s = 0; s < kSub; ++s) {
    const int token = tokens[16 * s + mine.n];
    u32x4 z[Mine::kLoads];
#pragma unroll
    for (int j = 0; j < Mine::kLoads; ++j) z[j] = y[s % kBuffers][j];
    if (!none) mine.add(h[16 * s + mine.n], by, z);
    if (s + kBuffers < kSub) mine.load_base(p, tokens[16 * (s + kBuffers) + mine.n], y[s % kBuffers]);
    mine.store(p, token, z);
  }
}

// Both products of a tile of 16 tokens in one launch, for 512 columns: every workgroup multiplies down x by itself, sixteen waves over the elements of x, so that
// no wave has to wait for memory more than a time or two. For few tokens, which latency bounds: a launch less pays for x and down being read
// again for every 512 columns (see launch_tiles for where).
constexpr int kBothWaves = 16, kBothThreads = 64 * kBothWaves, kBothColumns = 32;
template <class T, int kRankTiles>
__global__ void __launch_bounds__(kBothThreads) gnr_adapters_both_kernel(const AdapterParams p)
{
  typedef typename T::oct oct;
  constexpr int kRankSteps = (kRankTiles + 1) / 2, kPitch = kRankSteps * 32 + 4;
  typedef Columns<T, kRankSteps, kBothColumns> Mine;
  extern __shared__ int numbers[];
  __shared__ int tokens[16];
  __shared__ float sums[kBothWaves][kRankTiles * 16][17];
  __shared__ __attribute__((aligned(16))) float h[16][kPitch];
  const int which = find_tile<16, kBothThreads>(p, blockIdx.y, true, numbers, tokens);
  if (which < 0) return;
  const bool none = which == p.set.adapters;
  const int lane = threadIdx.x % 64, wave = uniform(static_cast<int>(threadIdx.x / 64)), rank = p.set.rank, width = static_cast<int>(p.set.width_in);
  Mine mine(lane, (blockIdx.x * kBothWaves + wave) * kBothColumns, static_cast<int>(p.set.width_out));
  const int n = mine.n, g = mine.g, token = tokens[n];
  u32x4 y[Mine::kLoads];
  mine.load_base(p, token, y);
  if (!none) {
    mine.load_rows(p, which);
    const float by = p.set.scale[which];
    const uint16_t *x = static_cast<const uint16_t *>(p.x) + static_cast<int64_t>(max(token, 0)) * p.x_stride;   // (what is beyond the tile's last is not kept)
    const uint16_t *down = static_cast<const uint16_t *>(p.set.down) + static_cast<int64_t>(which) * rank * width;
    f32x4 acc[kRankTiles];
#pragma unroll
    for (int i = 0; i < kRankTiles; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int kAtOnce = kRankTiles == 4 ? 2 : 4, kElements = 32 * kBothWaves * kAtOnce;   // (by the registers that 1024 threads leave a lane)
    for (int d0 = 32 * wave; d0 < width; d0 += kElements) {
      u32x4 a[kAtOnce][kRankTiles], b[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int d = d0 + 32 * kBothWaves * u + 8 * g;
        const bool in = d < width;
        b[u] = u32x4{0, 0, 0, 0};
        if (in) b[u] = *reinterpret_cast<const u32x4 *>(x + d);
#pragma unroll
        for (int i = 0; i < kRankTiles; ++i) {
          a[u][i] = u32x4{0, 0, 0, 0};
          if (in && 16 * i + n < rank) a[u][i] = *reinterpret_cast<const u32x4 *>(down + static_cast<int64_t>(16 * i + n) * width + d);
        }
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
        for (int i = 0; i < kRankTiles; ++i) acc[i] = T::mfma16(bits<oct>(a[u][i]), bits<oct>(b[u]), acc[i]);
    }
#pragma unroll
    for (int i = 0; i < kRankTiles; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) sums[wave][16 * i + 4 * g + k][n] = acc[i][k];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * 32 * kRankSteps; i += kBothThreads) {
      const int t = i % 16, r = i / 16;
      float sum = 0.0f;
      if (r < rank) {
#pragma unroll
        for (int w = 0; w < kBothWaves; ++w) sum += sums[w][r][t];
      }
      h[t][r] = sum;
    }
    __syncthreads();
    mine.add(h[n], by, y);
  }
  mine.store(p, token, y);
}

static int tile_tokens(int64_t tokens) { return tokens >= kManyTokens ? 64 : 16; }

static int tiles_bound(const iter_adapter_set &s, int requests, int64_t tokens, bool with_none)
{
  // tiles that are full, and for every adapter in use one that is not
  const int64_t used = (requests < s.adapters ? requests : s.adapters) + (with_none ? 1 : 0);
  return static_cast<int>(tokens / tile_tokens(tokens) + (used < tokens ? used : tokens));
}

// Shares of the elements of x: enough that few tiles fill the chip, at least two blocks to a wave.
static int splits_for(const iter_adapter_set &s, int64_t tokens)
{
  const int64_t tile = tile_tokens(tokens), tiles = (tokens + tile - 1) / tile, depth = s.width_in / (2 * kDepth * kWaves);
  int64_t n = 512 / (tiles < 1 ? 1 : tiles);
  n = n < depth ? n : depth;
  return static_cast<int>(n < 1 ? 1 : n < 16 ? n : 16);
}

size_t adapters_bytes(const iter_adapter_set &s, int64_t tokens)
{
  return static_cast<size_t>(splits_for(s, tokens)) * static_cast<size_t>(tokens) * static_cast<size_t>(s.rank) * sizeof(float);
}

template <class T, int kSub>
static int launch(const AdapterParams &p, hipStream_t s)
{
  const size_t lds = static_cast<size_t>(p.set.adapters + 1 + 2 * p.requests) * sizeof(int);
  const int splits = splits_for(p.set, p.tokens);
  // the workgroups of a tile run beside each other, so that whole rows of x, base and out are read and written at a time (whole prompt 87 -> 81 us,
  // mixed iteration 20.2 -> 17.8)
  const dim3 down(static_cast<unsigned>(splits), static_cast<unsigned>(tiles_bound(p.set, p.requests, p.tokens, false)));
  const dim3 up(static_cast<unsigned>((p.set.width_out + kColumns * kWaves - 1) / (kColumns * kWaves)), static_cast<unsigned>(tiles_bound(p.set, p.requests, p.tokens, true)));
  if (p.set.adapters > 0) {
    if (p.set.rank <= 16) gnr_adapters_down_kernel<T, 1, kSub><<<down, kThreads, lds, s>>>(p);
    else if (p.set.rank <= 32) gnr_adapters_down_kernel<T, 2, kSub><<<down, kThreads, lds, s>>>(p);
    else if (p.set.rank <= 64) gnr_adapters_down_kernel<T, 4, kSub><<<down, kThreads, lds, s>>>(p);
    else gnr_adapters_down_kernel<T, 8, kSub><<<down, kThreads, lds, s>>>(p);
    const int rc = iter_hip_ok(hipGetLastError());
    if (rc != SIM_OK) return rc;
  }
  if (p.set.rank <= 32) gnr_adapters_up_kernel<T, 1, kSub><<<up, kThreads, lds, s>>>(p, splits);
  else if (p.set.rank <= 64) gnr_adapters_up_kernel<T, 2, kSub><<<up, kThreads, lds, s>>>(p, splits);
  else gnr_adapters_up_kernel<T, 4, kSub><<<up, kThreads, lds, s>>>(p, splits);
  return iter_hip_ok(hipGetLastError());
}

// One launch for both products as long as what a workgroup reads of x and down is little, and what all of them do. us by two launches and by one, (tokens, rank, width in,
// width out): (128, 32, 1024, 1024) 11.7 and 8.4, (700, 32, 512, 512) 18.7 and 10.4, (40, 24, 2000, 8000) 11.2 and 8.4, (1500, 16, 2048, 2048) 25.5 and 20.1; where a workgroup reads more,
// (128, 16, 4096, 6144) 11.6 and 12.8, (128, 64, 4096, 4096) 15.0 and 25.8; where they all read 91 MB, (1000, 64, 1024, 4096), 29.8 and 34.0.
// Not where out may overlap x: a workgroup would read rows of x that another of the tile's has written over. (Of two launches the first has read all of x.)
constexpr int64_t kBothBytes = 160 << 10, kBothAll = 64 << 20;
static bool may_overlap_x(const AdapterParams &p)
{
  const auto first = [](const void *at) { return static_cast<int64_t>(reinterpret_cast<uintptr_t>(at)); };
  const int64_t x = first(p.x), out = first(p.out), x_row = 2 * p.set.width_in, out_row = 2 * p.set.width_out, step = 2 * p.x_stride;
  if (out >= x + (p.tokens - 1) * step + x_row || x >= out + (p.tokens - 1) * 2 * p.out_stride + out_row) return false;
  // rows of one buffer side by side, each with its own columns
  if (p.x_stride != p.out_stride || step == 0) return true;
  const int64_t ahead = ((out - x) % step + step) % step;
  return ahead < x_row || ahead + out_row > step;
}

template <class T>
static int launch_tiles(const AdapterParams &p, hipStream_t s)
{
  if (tile_tokens(p.tokens) == 64) return launch<T, 4>(p, s);
  const dim3 both(static_cast<unsigned>((p.set.width_out + kBothColumns * kBothWaves - 1) / (kBothColumns * kBothWaves)), static_cast<unsigned>(tiles_bound(p.set, p.requests, p.tokens, true)));
  const int64_t bytes = (16 + static_cast<int64_t>(p.set.rank)) * p.set.width_in * 2;
  if (p.set.rank <= 64 && bytes <= kBothBytes && bytes * both.x * both.y <= kBothAll && !may_overlap_x(p)) {
    const size_t lds = static_cast<size_t>(p.set.adapters + 1 + 2 * p.requests) * sizeof(int);
    if (p.set.rank <= 16) gnr_adapters_both_kernel<T, 1><<<both, kBothThreads, lds, s>>>(p);
    else if (p.set.rank <= 32) gnr_adapters_both_kernel<T, 2><<<both, kBothThreads, lds, s>>>(p);
    else gnr_adapters_both_kernel<T, 4><<<both, kBothThreads, lds, s>>>(p);
    return iter_hip_ok(hipGetLastError());
  }
  return launch<T, 1>(p, s);
}

int launch_adapters(const AdapterParams &p, void *stream)
{
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return p.type == ITER_BF16 ? launch_tiles<Bf16>(p, s) : launch_tiles<Fp16>(p, s);
}

}  // namespace gnr
