// What the attention kernels share (gfx950): the requests of a batch, how their work is shared out over the chip, and the parts
// that are joined where a row's keys were.
#ifndef GNR_ITER_ATTENTION_H
#define GNR_ITER_ATTENTION_H

#include <cfloat>

#include "gnr_iter_device.h"

namespace gnr {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kPartTail = 4;                   // words of a part after its sums: maximum, sum of weights, two of padding

// A kernel takes the requests with `least` to `most` rows (tokens times query heads of a kv head), in tiles of kRows rows and blocks
// of kKeys keys, about kPieces pieces to a workgroup.
struct RowsShape { static constexpr int kRows = 16, kKeys = 32 * kWaves, kPieces = 4, kPlan = 0; };
struct ChunkShape { static constexpr int kRows = 128, kKeys = 64, kPieces = 1, kPlan = 1; };
// Workgroups that a compute unit holds at once, by their registers.
constexpr int kComputeUnits = 256;
constexpr int rows_blocks(int dim, bool fp8) { return dim == 256 ? 1 : dim == 128 && !fp8 ? 2 : 3; }
constexpr int chunk_blocks(int dim) { return dim == 256 ? 1 : 2; }
constexpr int kFewRows = 16;

// What a request asks for. Bounds that contradict each other or the arrays are cut down to what is inside them. Positions are below 2^30.
struct Request {
  int first, tokens;        // of the batch
  int base;                 // position of the first token (negative for one whose key the cache does not hold)
  int begin, end;           // keys that any of its tokens sees, [begin, end); begin is a multiple of 64
};

__device__ __forceinline__ Request request_of(const AttentionParams &p, int r, uint32_t *flags)
{
  const int total = static_cast<int>(p.batch.tokens);
  int b = p.batch.q_start[r], e = p.batch.q_start[r + 1], length = p.batch.kv_len[r];
  if (b < 0 || e < b || e > total || length < 0 || length > p.room || (r == 0 && b != 0) || (r == p.batch.requests - 1 && e != total))
    *flags |= ITER_BAD_BATCH;
  b = min(max(b, 0), total);
  e = min(max(e, b), total);
  length = min(max(length, 0), p.room);
  Request q;
  q.first = b;
  q.tokens = e - b;
  q.base = length - q.tokens;
  q.end = p.cache.pages == 0 ? 0 : length;
  q.begin = p.window ? max(0, q.base - p.window + 1) & ~63 : 0;
  q.end = max(q.end, q.begin);
  return q;
}

// The plan of a launch, found by every workgroup for itself: before request r lie start[r] units (a piece of the keys of a tile of
// rows), part[r] rows of parts and join[r] rows that are joined from them.
struct Plan {
  int *start, *part, *join;
};

// Sum of a value over the workgroup and of those of the threads before this one.
__device__ __forceinline__ void block_scan(int v, int *scratch, int &before, int &total)
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
  before = x - v;
  total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += scratch[w];
    total += scratch[w];
  }
}

__device__ __forceinline__ int64_t block_sum(int64_t v, unsigned long long *scratch)
{
#pragma unroll
  for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
  __syncthreads();
  if (threadIdx.x % 64 == 0) scratch[threadIdx.x / 64] = static_cast<unsigned long long>(v);
  __syncthreads();
  int64_t all = 0;
  for (int w = 0; w < kWaves; ++w) all += static_cast<int64_t>(scratch[w]);
  return all;
}

// The keys of a request are shared out in pieces, so that few long rows fill the chip and a long request does not outlast the others: whole
// blocks of keys, the pieces of a request as long as each other, no more of them in all than fill the workgroups evenly. It is a
// function of the batch alone, so the same rows are summed in the same order every time, and costs a launch two microseconds, which
// spares the host from knowing the lengths.
template <class Shape>
__device__ __forceinline__ void share_out(const AttentionParams &p, const Plan &plan, int blocks)
{
  __shared__ int scratch[kWaves];
  __shared__ unsigned long long sums[kWaves];
  const int n = p.batch.requests;
  uint32_t flags = 0;
  const auto work = [&](int r, int &tiles, int &keys, int &rows) {
    const Request q = request_of(p, r, &flags);
    rows = q.tokens * p.group;
    const bool mine = q.tokens > 0 && rows >= p.least[Shape::kPlan] && rows <= p.most[Shape::kPlan];
    tiles = mine ? (rows + Shape::kRows - 1) / Shape::kRows : 0;
    keys = (q.end - q.begin + Shape::kKeys - 1) / Shape::kKeys;
  };
  int64_t all = 0;
  int tiles, keys, rows;
  for (int r = threadIdx.x; r < n; r += kThreads) {
    work(r, tiles, keys, rows);
    all += static_cast<int64_t>(tiles) * keys;
  }
  all = block_sum(all, sums) * p.cache.kv_heads;
  if (flags && p.status && blockIdx.x == 0) atomicOr(p.status, flags);
  const int64_t pieces = static_cast<int64_t>(blocks) * Shape::kPieces;
  int size = static_cast<int>(max(int64_t(1), (all + pieces - 1) / pieces));
  for (int round = 0; round < 6; ++round) {      // last pieces that are short make it more than there is room for: take longer ones
    int64_t units = 0;
    for (int r = threadIdx.x; r < n; r += kThreads) {
      work(r, tiles, keys, rows);
      units += static_cast<int64_t>(tiles) * max(1, (keys + size - 1) / size);
    }
    if (block_sum(units, sums) * p.cache.kv_heads <= pieces) break;
    size += size / 8 + 1;
  }
  int done[3] = {0, 0, 0};
  for (int r0 = 0; r0 < n; r0 += kThreads) {
    const int r = r0 + threadIdx.x;
    int v[3] = {0, 0, 0};
    if (r < n) {
      work(r, tiles, keys, rows);
      const int splits = max(1, (keys + size - 1) / size);
      v[0] = tiles * splits;
      v[1] = tiles && splits > 1 ? rows * splits : 0;
      v[2] = v[1] ? rows : 0;
    }
    int *const to[3] = {plan.start, plan.part, plan.join};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      int before, total;
      block_scan(v[i], scratch, before, total);
      if (r < n) to[i][r] = done[i] + before;
      done[i] += total;
    }
  }
  if (threadIdx.x == 0) {
    plan.start[n] = done[0];
    plan.part[n] = done[1];
    plan.join[n] = done[2];
  }
  __syncthreads();
}

// The last of n + 1 ascending numbers' first n that is not above `at`.
__device__ __forceinline__ int last_not_above(const int *numbers, int n, int at)
{
  int r = 0;
  for (int step = ITER_MAX_REQUESTS / 2; step; step /= 2)
    if (r + step < n && numbers[r + step] <= at) r += step;
  return r;
}

// Plans as they are kept in the workspace for the kernel that joins: start, part and join of each kernel.
__device__ __forceinline__ int *kept_plan(const AttentionParams &p, int which) { return reinterpret_cast<int *>(p.workspace) + which * 3 * (p.batch.requests + 1); }

__device__ __forceinline__ void keep_plan(const AttentionParams &p, const Plan &plan, int which)
{
  int *to = kept_plan(p, which);
  const int n = p.batch.requests + 1;
  for (int r = threadIdx.x; r < n; r += kThreads) {
    to[r] = plan.start[r];
    to[n + r] = plan.part[r];
    to[2 * n + r] = plan.join[r];
  }
}

// Units of a request: the pieces of a tile one after the other; a chunk's last tokens, which see the most keys, go first.
template <class Shape>
__device__ __forceinline__ int tile_of_unit(int unit, int tiles, int splits)
{
  return Shape::kPlan == ChunkShape::kPlan ? tiles - 1 - unit / splits : unit / splits;
}

// Whether a unit (times kv head) met something that it leaves to the kernel that joins, which computes the rows of its tile again: a
// page that is not there, or values that its products cannot hide from the rows that do not see them.
__device__ __forceinline__ void mark_unit(const AttentionParams &p, int which, int64_t unit, int again)
{
  if (unit < p.units[which]) reinterpret_cast<int *>(p.workspace)[p.marks[which] + unit] = again;
}

// Whether any of the pages that hold keys [from, to) is not there; they are looked at by the whole workgroup. The kernels read another page in its place.
__device__ __forceinline__ int missing_page(const AttentionParams &p, const int32_t *table, int from, int to)
{
  bool missing = false;
  for (int i = (from >> p.page_shift) + threadIdx.x; i <= (to - 1) >> p.page_shift; i += kThreads) missing |= static_cast<uint32_t>(table[i]) >= static_cast<uint32_t>(p.cache.pages);
  if (missing && p.status) atomicOr(p.status, ITER_BAD_PAGE);
  return missing;
}

__device__ __forceinline__ int usable_page(const AttentionParams &p, int page) { return static_cast<uint32_t>(page) < static_cast<uint32_t>(p.cache.pages) ? page : 0; }

// Where a row's results go when its keys were shared out: the sum of weighted values, relative to the maximum, then maximum and sum.
__device__ __forceinline__ float *part_of(const AttentionParams &p, int which, int64_t row, int head)
{
  return p.workspace + p.parts[which] + (row * p.cache.kv_heads + head) * (p.cache.head_dim + kPartTail);
}

// Four elements of an output row from d on: weighted values over the sum of the weights, zeros where no key was seen.
template <class T>
__device__ __forceinline__ void write_row(const AttentionParams &p, int64_t token, int64_t head, int d, f32x4 o, float sum)
{
  const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
  u32x2 w;
  w[0] = T::narrow2(o[0] * f, o[1] * f);
  w[1] = T::narrow2(o[2] * f, o[3] * f);
  *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(p.out.data) + token * p.out.token_stride + head * p.out.head_stride + d) = w;
}

int launch_attention_rows(const AttentionParams &p, hipStream_t stream);
int launch_attention_chunk(const AttentionParams &p, hipStream_t stream);

}  // namespace gnr
#endif
