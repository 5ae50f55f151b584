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
// Workgroups that a compute unit holds at once, by their registers. Shared memory (34.6 KB of a workgroup with 128 elements, 67.4 with 256, and 20 bytes a request) holds as many too, but over 4 bits
// only up to 999 requests with 128 elements and 726 with 256: of more, the last third or half of the workgroups begin when others end, with the same results. Few rows of 256 elements over 4 bits fit twice, over 8 and 16 bits
// once: 60 ragged decodes around 2000 keys (16 heads over 4) 74 -> 57 us with the second, 127 of them 137 -> 122, 3 around 30000
// 43 -> 39, one of 1093 keys 16.6 -> 16.4. A fourth at 64 elements would spill (127 ragged decodes 160 -> 144 us, but 3 around 60000
// keys 20 -> 26).
constexpr int kComputeUnits = 256;
constexpr int rows_blocks(int dim, int bits) { return dim == 256 ? (bits > 4 ? 1 : 2) : dim == 128 && bits > 4 ? 2 : 3; }
constexpr int chunk_blocks(int dim) { return dim == 256 ? 1 : 2; }
constexpr int kFewRows = 16;

// What a request asks for. Bounds that contradict each other or the arrays are cut down to what is inside them. Positions are below 2^30.
struct Request {
  int first, tokens;        // of the batch
  int base;                 // position of the first token (negative for one whose key the cache does not hold)
  int begin, end;           // keys that any of its tokens sees, [begin, end); begin is a multiple of 64
};

__device__ __forceinline__ Request request_of(const AttentionParams &p, int r, int b, int e, int length, uint32_t *flags)
{
  const int total = static_cast<int>(p.batch.tokens);
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

__device__ __forceinline__ Request request_of(const AttentionParams &p, int r, uint32_t *flags) { return request_of(p, r, p.batch.q_start[r], p.batch.q_start[r + 1], p.batch.kv_len[r], flags); }

// The same in scalar registers: what is computed from it stays there too (multiplications of addresses take a vector unit four times as long as other instructions).
__device__ __forceinline__ Request uniform(const Request &q) { return Request{uniform(q.first), uniform(q.tokens), uniform(q.base), uniform(q.begin), uniform(q.end)}; }

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

// The same for a plan; with a single request every thread has its numbers, and nothing is exchanged or waited for: one decode over 4 bits 13.1 -> 12.0 us, a chunk of a
// single request 154.6 -> 151.9. (A scan by every wave for itself, with up to 64 requests, gains 0.4 us of 59 and is not worth a third plan in each kernel.)
template <bool kOne, class V>
__device__ __forceinline__ void plan_scan(V v, V *scratch, V &before, V &total)
{
  if constexpr (kOne) {
    before = 0;
    total = v;
  } else {
    block_scan<V>(v, scratch, before, total);
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
// much of the cache, however long the requests are. Over 4 bits, where a block takes 3 us and the change from one tile to the next three times as long, a tile counts for three blocks more than it has: a workgroup with many short ones
// was the last by far (127 decodes of 453000 keys in all, ragged: 127 -> 112 us; of 100 with 500 on the average 46 -> 34; counted for two blocks 114 and 34, for six 116 and 36). A (tile, kv head) that is cut leaves parts, two at most to a workgroup: one that began
// before it (slot 0) and one that ends after it or is cut at its very beginning (slot 1).
struct RowsPlan {
  int64_t *start;           // blocks of keys before request r, for one kv head
  int *tiles;               // tiles before request r
  int *first, *lengths;     // q_start and kv_len, at hand where a request begins
  int64_t total;            // blocks of keys, all heads
  int extra;                // blocks that a (tile, kv head) counts for beside its own, at its beginning
  int blocks;               // workgroups that have any
  __device__ __forceinline__ int64_t cut(int64_t b) const { return b * total / blocks; }
  __device__ __forceinline__ Request request(const AttentionParams &p, int r) const
  {
    uint32_t flags = 0;
    return uniform(request_of(p, r, first[r], first[r + 1], lengths[r], &flags));
  }
  __device__ __forceinline__ int block_of(int64_t x) const { return static_cast<int>(((x + 1) * blocks + total - 1) / total - 1); }
};

// What a workgroup leaves for the join beside its parts: of a (tile, kv head) that begins in it and is cut (`rows` = 0 if there is none) where its rows are and the last workgroup
// with a part of it, and the workgroup in which the one began that it goes on with, if that one has more than kFewParts parts (-1: else). Every workgroup writes one.
constexpr int kFewParts = 24;
struct alignas(16) CutTile {
  int rows = 0, tile = 0, head = 0, request = 0, token = 0, last = 0, from = -1, mark[2] = {0, 0};   // mark: of the slots 0 and 1
};

template <bool kOne>
__device__ __forceinline__ RowsPlan plan_rows(const AttentionParams &p, void *memory, int blocks)
{
  __shared__ int64_t scratch64[kWaves];
  __shared__ int scratch[kWaves];
  const int n = p.batch.requests;
  RowsPlan plan{static_cast<int64_t *>(memory), reinterpret_cast<int *>(static_cast<int64_t *>(memory) + n + 1), nullptr, nullptr, 0, 0, 0};
  plan.first = plan.tiles + n + 1;
  plan.lengths = plan.first + n + 1;
  uint32_t flags = 0;
  int64_t done64 = 0;
  int done = 0;
  for (int r0 = 0; r0 < n; r0 += kThreads) {
    const int r = kOne ? 0 : r0 + threadIdx.x;
    int rows = 0, keys = 0, tiles = 0;
    if (r < n) {
      const int begin = p.batch.q_start[r], end = p.batch.q_start[r + 1], length = p.batch.kv_len[r];
      tiles = tiles_of<RowsShape>(p, request_of(p, r, begin, end, length, &flags), rows, keys);
      plan.first[r] = begin;
      plan.lengths[r] = length;
      if (r == n - 1) plan.first[n] = end;
    }
    int64_t before64, total64;
    int before, total;
    plan_scan<kOne, int64_t>(static_cast<int64_t>(tiles) * keys, scratch64, before64, total64);
    plan_scan<kOne, int>(tiles, scratch, before, total);
    if (r < n) {
      plan.start[r] = done64 + before64;
      plan.tiles[r] = done + before;
    }
    done64 += total64;
    done += total;
  }
  done64 = uniform(done64);
  done = uniform(done);
  // (fewer tiles than workgroups: what a tile takes beside its keys is everybody's; of little more than a block each: they are dealt out well as they are, 127 requests of 100 keys 25.6 us and 27.4 with it)
  plan.extra = !kOne && static_cast<int64_t>(done) * p.cache.kv_heads >= blocks && done64 >= 2 * static_cast<int64_t>(done) ? p.tile_cost : 0;
  if (plan.extra)
    for (int r = threadIdx.x; r < n; r += kThreads) plan.start[r] += static_cast<int64_t>(plan.extra) * plan.tiles[r];
  done64 += static_cast<int64_t>(plan.extra) * done;
  if (threadIdx.x == 0) {
    plan.start[n] = done64;
    plan.tiles[n] = done;
  }
  if (flags && p.status && blockIdx.x == 0) atomicOr(p.status, flags);
  plan.total = done64 * p.cache.kv_heads;
  plan.blocks = static_cast<int>(min(plan.total, static_cast<int64_t>(blocks)));
  __syncthreads();
  return plan;
}

__device__ __forceinline__ RowsPlan share_out_rows(const AttentionParams &p, void *memory, int blocks)
{
  return p.batch.requests == 1 ? plan_rows<true>(p, memory, blocks) : plan_rows<false>(p, memory, blocks);
}

// Chunks: a tile of rows is whole where there are many. Where there are few, their keys are cut into pieces, as long as each other within a
// request, no more of them in all than there are workgroups. Before request r lie start[r] units (a piece of a tile's keys), part[r] rows of parts
// and join[r] rows that are joined from them.
struct ChunkPlan {
  int *start, *part, *join;
};

template <bool kOne>
__device__ __forceinline__ void plan_chunks(const AttentionParams &p, const ChunkPlan &plan, int blocks)
{
  __shared__ int scratch[kWaves];
  __shared__ int64_t sums[kWaves];
  const int n = p.batch.requests;
  uint32_t flags = 0;
  int64_t all = 0, before64;
  int rows, keys;
  for (int r = kOne ? 0 : threadIdx.x; r < n; r += kThreads) all += static_cast<int64_t>(tiles_of<ChunkShape>(p, request_of(p, r, &flags), rows, keys)) * keys;
  plan_scan<kOne, int64_t>(all, sums, before64, all);
  if (flags && p.status && blockIdx.x == 0) atomicOr(p.status, flags);
  int size = blocks_of_a_piece(all * p.cache.kv_heads, blocks);
  for (int round = 0; round < 6; ++round) {      // last pieces that are short make it more than there is room for: take longer ones
    int64_t units = 0;
    for (int r = kOne ? 0 : threadIdx.x; r < n; r += kThreads) {
      const int tiles = tiles_of<ChunkShape>(p, request_of(p, r, &flags), rows, keys);
      units += static_cast<int64_t>(tiles) * ((keys + size - 1) / size);
    }
    plan_scan<kOne, int64_t>(units, sums, before64, units);
    if (units * p.cache.kv_heads <= blocks) break;
    size += size / 8 + 1;
  }
  int done[3] = {0, 0, 0};
  for (int r0 = 0; r0 < n; r0 += kThreads) {
    const int r = kOne ? 0 : r0 + threadIdx.x;
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
      plan_scan<kOne, int>(v[i], scratch, before, total);
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

__device__ __forceinline__ void share_out_chunks(const AttentionParams &p, const ChunkPlan &plan, int blocks)
{
  if (p.batch.requests == 1) plan_chunks<true>(p, plan, blocks);
  else plan_chunks<false>(p, plan, blocks);
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
constexpr size_t rows_plan_bytes(int requests) { return plan_bytes(requests) + (static_cast<size_t>(requests) * 2 + 1) * sizeof(int); }

int launch_attention_rows(const AttentionParams &p, hipStream_t stream);
int launch_attention_chunk(const AttentionParams &p, hipStream_t stream);

}  // namespace gnr
#endif
