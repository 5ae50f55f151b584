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
// of kKeys keys.
struct RowsShape { static constexpr int kRows = 16, kKeys = 32 * kWaves, kPlan = 0; };
struct ChunkShape { static constexpr int kRows = 128, kKeys = 64, kPlan = 1; };
// Workgroups that a compute unit holds at once, by their registers.
constexpr int kComputeUnits = 256;
constexpr int rows_blocks(int dim) { return dim == 256 ? 1 : dim == 128 ? 2 : 3; }
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

// Sum of a value over the workgroup's threads before this one, and over all.
template <class V>
__device__ __forceinline__ void block_scan(V v, V *scratch, V &before, V &total)
{
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  V x = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const V o = __shfl_up(x, d);
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

// A request's tiles of rows (none, if the kernel does not take it) and the blocks of keys that they see, at least one.
template <class Shape>
__device__ __forceinline__ int tiles_of(const AttentionParams &p, const Request &q, int &rows, int &keys)
{
  rows = q.tokens * p.group;
  keys = max(1, (q.end - q.begin + Shape::kKeys - 1) / Shape::kKeys);
  const bool mine = q.tokens > 0 && rows >= p.least[Shape::kPlan] && rows <= p.most[Shape::kPlan];
  return mine ? (rows + Shape::kRows - 1) / Shape::kRows : 0;
}

// How a launch shares out its work, found by every workgroup for itself: it is a function of the batch alone, so the same rows are summed in the
// same order every time, and costs a launch two microseconds, which spares the host from knowing the lengths.
//
// Few rows: all blocks of keys of all (tile, kv head) in a row, cut into as many pieces of the same length as there are workgroups: every one reads as
// much of the cache, however long the requests are. A (tile, kv head) that is cut leaves parts, two at most to a workgroup: one that began
// before it (slot 0) and one that ends after it or is cut at its very beginning (slot 1).
struct RowsPlan {
  int64_t *start;           // blocks of keys before request r, for one kv head
  int *tiles;               // tiles before request r
  int64_t total;            // blocks of keys, all heads
  int blocks;               // workgroups that have any
  __device__ __forceinline__ int64_t cut(int64_t b) const { return b * total / blocks; }
  __device__ __forceinline__ int block_of(int64_t x) const { return static_cast<int>(((x + 1) * blocks + total - 1) / total - 1); }
};

// What the workgroup in which a (tile, kv head) begins that is cut leaves for the join beside slot 1: where its rows are and the last workgroup with a
// part of it. Every workgroup writes one, with `rows` = 0 if there is none.
struct alignas(16) CutTile {
  int rows, tile, head, request, token, last, mark[2];   // mark: of the slots 0 and 1
};

__device__ __forceinline__ RowsPlan share_out_rows(const AttentionParams &p, void *memory, int blocks)
{
  __shared__ int64_t scratch64[kWaves];
  __shared__ int scratch[kWaves];
  const int n = p.batch.requests;
  RowsPlan plan{static_cast<int64_t *>(memory), reinterpret_cast<int *>(static_cast<int64_t *>(memory) + n + 1), 0, 0};
  uint32_t flags = 0;
  int64_t done64 = 0;
  int done = 0;
  for (int r0 = 0; r0 < n; r0 += kThreads) {
    const int r = r0 + threadIdx.x;
    int rows = 0, keys = 0, tiles = 0;
    if (r < n) tiles = tiles_of<RowsShape>(p, request_of(p, r, &flags), rows, keys);
    int64_t before64, total64;
    int before, total;
    block_scan<int64_t>(static_cast<int64_t>(tiles) * keys, scratch64, before64, total64);
    block_scan<int>(tiles, scratch, before, total);
    if (r < n) {
      plan.start[r] = done64 + before64;
      plan.tiles[r] = done + before;
    }
    done64 += total64;
    done += total;
  }
  if (threadIdx.x == 0) {
    plan.start[n] = done64;
    plan.tiles[n] = done;
  }
  if (flags && p.status && blockIdx.x == 0) atomicOr(p.status, flags);
  plan.total = uniform(done64) * p.cache.kv_heads;
  plan.blocks = static_cast<int>(min(plan.total, static_cast<int64_t>(blocks)));
  __syncthreads();
  return plan;
}

// Chunks: a tile of rows is whole where there are many. Where there are few, their keys are cut into pieces, as long as each other within a
// request, no more of them in all than there are workgroups. Before request r lie start[r] units (a piece of a tile's keys), part[r] rows of parts
// and join[r] rows that are joined from them.
struct ChunkPlan {
  int *start, *part, *join;
};

__device__ __forceinline__ void share_out_chunks(const AttentionParams &p, const ChunkPlan &plan, int blocks)
{
  __shared__ int scratch[kWaves];
  __shared__ int64_t sums[kWaves];
  const int n = p.batch.requests;
  uint32_t flags = 0;
  int64_t all = 0, before64;
  int rows, keys;
  for (int r = threadIdx.x; r < n; r += kThreads) all += static_cast<int64_t>(tiles_of<ChunkShape>(p, request_of(p, r, &flags), rows, keys)) * keys;
  block_scan<int64_t>(all, sums, before64, all);
  if (flags && p.status && blockIdx.x == 0) atomicOr(p.status, flags);
  int size = blocks_of_a_piece(all * p.cache.kv_heads, blocks);
  for (int round = 0; round < 6; ++round) {      // last pieces that are short make it more than there is room for: take longer ones
    int64_t units = 0;
    for (int r = threadIdx.x; r < n; r += kThreads) {
      const int tiles = tiles_of<ChunkShape>(p, request_of(p, r, &flags), rows, keys);
      units += static_cast<int64_t>(tiles) * ((keys + size - 1) / size);
    }
    block_scan<int64_t>(units, sums, before64, units);
    if (units * p.cache.kv_heads <= blocks) break;
    size += size / 8 + 1;
  }
  int done[3] = {0, 0, 0};
  for (int r0 = 0; r0 < n; r0 += kThreads) {
    const int r = r0 + threadIdx.x;
    int v[3] = {0, 0, 0};
    if (r < n) {
      const int tiles = tiles_of<ChunkShape>(p, request_of(p, r, &flags), rows, keys), splits = (keys + size - 1) / size;
      v[0] = tiles * splits;
      v[1] = tiles && splits > 1 ? rows * splits : 0;
      v[2] = v[1] ? rows : 0;
    }
    int *const to[3] = {plan.start, plan.part, plan.join};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      int before, total;
      block_scan<int>(v[i], scratch, before, total);
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
template <class V>
__device__ __forceinline__ int last_not_above(const V *numbers, int n, V at)
{
  int r = 0;
  for (int step = ITER_MAX_REQUESTS / 2; step; step /= 2)
    if (r + step < n && numbers[r + step] <= at) r += step;
  return r;
}

// Plans as they are kept in the workspace for the kernel that joins (and what it copies to shared memory).
__device__ __forceinline__ int *kept_plan(const AttentionParams &p, int which) { return reinterpret_cast<int *>(p.workspace) + which * 3 * (p.batch.requests + 1); }

__device__ __forceinline__ void copy_plan(const AttentionParams &p, int *to, const int *from)
{
  for (int i = threadIdx.x; i < 3 * (p.batch.requests + 1); i += kThreads) to[i] = from[i];
}

// Units of a chunk: the pieces of a tile one after the other; the last tokens, which see the most keys, go first.
__device__ __forceinline__ int tile_of_unit(int unit, int tiles, int splits) { return tiles - 1 - unit / splits; }

__device__ __forceinline__ CutTile *cut_tiles(const AttentionParams &p) { return reinterpret_cast<CutTile *>(p.workspace + p.cuts); }

// Marks: whether a unit met something that it leaves to the kernel that joins, which computes the rows of its tile again: a
// page that is not there, or values that its products cannot hide from the rows that do not see them.
__device__ __forceinline__ int *marks_of(const AttentionParams &p, int which) { return reinterpret_cast<int *>(p.workspace) + p.marks[which]; }

__device__ __forceinline__ void mark(const AttentionParams &p, int which, int64_t unit, int again)
{
  if (unit < p.units[which]) marks_of(p, which)[unit] = again;
}

// Whether any of the pages that hold keys [from, to) is not there; they are looked at by the whole workgroup. The kernels read another page in its place. (Blocks of keys
// begin at multiples of 64, which may be before the first key that a window leaves to see: `from` is that key, what pages before it are does not matter.)
__device__ __forceinline__ int missing_page(const AttentionParams &p, const int32_t *table, int from, int to)
{
  bool missing = false;
  for (int i = (from >> p.page_shift) + threadIdx.x; from < to && i <= (to - 1) >> p.page_shift; i += kThreads) missing |= static_cast<uint32_t>(table[i]) >= static_cast<uint32_t>(p.cache.pages);
  if (missing && p.status) atomicOr(p.status, ITER_BAD_PAGE);
  return missing;
}

__device__ __forceinline__ int usable_page(const AttentionParams &p, int page) { return static_cast<uint32_t>(page) < static_cast<uint32_t>(p.cache.pages) ? page : 0; }

// Where a row's results go when its keys were shared out: the sum of weighted values, relative to the maximum, then maximum and sum.
__device__ __forceinline__ float *part_of(const AttentionParams &p, int which, int64_t row)
{
  return p.workspace + p.parts[which] + row * (p.cache.head_dim + kPartTail);
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

constexpr size_t plan_bytes(int requests) { return (static_cast<size_t>(requests) + 1) * 3 * sizeof(int); }

int launch_attention_rows(const AttentionParams &p, hipStream_t stream);
int launch_attention_chunk(const AttentionParams &p, hipStream_t stream);

}  // namespace gnr
#endif
