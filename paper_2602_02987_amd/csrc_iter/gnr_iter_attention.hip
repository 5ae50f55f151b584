// Attention of a mixed batch over the paged cache (gfx950): which kernels run, and the join of rows whose keys were shared out.
#include "gnr_iter_attention.h"

namespace gnr {

constexpr int kJoinBlocks = 1024;

// One row from the beginning, key by key: a wave, a lane for a key of 64 and then for head_dim / 64 elements. For rows that share a
// block of keys with a NaN or an infinity they do not see.
template <class T, int kDim>
__device__ __forceinline__ void one_row(const AttentionParams &p, int r, const Request &rq, int row, int head)
{
  constexpr int kMine = kDim / 64;
  const int lane = threadIdx.x % 64;
  const bool fp8 = p.cache.type == ITER_FP8;
  const int64_t token = rq.first + row / p.group, query_head = head * p.group + row % p.group;
  const uint16_t *q = static_cast<const uint16_t *>(p.q.data) + token * p.q.token_stride + query_head * p.q.head_stride;
  const int pos = rq.base + row / p.group, end = min(pos + 1, rq.end), begin = p.window ? max(0, pos - p.window + 1) : 0;
  const int32_t *table = p.batch.page_table + r * p.batch.table_stride;
  const iter_plane &k = p.cache.k, &v = p.cache.v;
  const auto element = [&](const iter_plane &c, int64_t at, float scale) {
    return fp8 ? T::widen(T::template from_e4m3<false>(static_cast<const uint8_t *>(c.data)[at], scale) & 0xFFFFu)
               : T::widen(static_cast<const uint16_t *>(c.data)[at]);
  };
  float top = -FLT_MAX, sum = 0.0f, acc[kMine] = {};
  for (int k0 = begin; k0 < end; k0 += 64) {
    const int key = k0 + lane, place = key & (p.cache.page - 1);
    int page = -1;
    if (key < end) page = table[key >> p.page_shift];
    if (page >= p.cache.pages) page = -1;
    float s = -INFINITY;
    if (page >= 0) {
      const int64_t at = static_cast<int64_t>(page) * k.page_stride + head * k.head_stride + place * k.place_stride;
      const float scale = fp8 ? exponent_scale(k.exp[page * k.exp_page_stride + head * k.exp_head_stride + place * k.exp_place_stride]) : 1.0f;
      float dot = 0.0f;
      for (int d = 0; d < kDim; ++d) dot = __builtin_fmaf(element(k, at + d, scale), T::widen(q[d]), dot);
      s = (p.flip ? -dot : dot) * p.scale_log2;
    }
    float high = s;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) high = fmaxf(high, __shfl_xor(high, d));
    const float next = fmaxf(top, high), keep = __builtin_amdgcn_exp2f(top - next);
    top = next;
    const float weight = __builtin_amdgcn_exp2f(s - top);
    float all = weight;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) all += __shfl_xor(all, d);
    sum = __builtin_fmaf(sum, keep, all);
#pragma unroll
    for (int i = 0; i < kMine; ++i) acc[i] *= keep;
    for (int l = 0; l < 64; ++l) {
      const int64_t of = __shfl(page, l);
      if (of < 0) continue;
      const float w = __shfl(weight, l);
      const int in = (k0 + l) & (p.cache.page - 1);
      const float scale = fp8 ? exponent_scale(v.exp[of * v.exp_page_stride + head * v.exp_head_stride + in * v.exp_place_stride]) : 1.0f;
      const int64_t at = of * v.page_stride + head * v.head_stride + in * v.place_stride + lane * kMine;
#pragma unroll
      for (int i = 0; i < kMine; ++i) acc[i] = __builtin_fmaf(w, element(v, at + i, scale), acc[i]);
    }
  }
  const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint16_t *out = static_cast<uint16_t *>(p.out.data) + token * p.out.token_stride + query_head * p.out.head_stride + lane * kMine;
#pragma unroll
  for (int i = 0; i < kMine; ++i) out[i] = static_cast<uint16_t>(T::narrow2(acc[i] * f, 0.0f));
}

// Adds a part of a row to those before, four elements to a lane.
template <int kDim>
__device__ __forceinline__ void add_part(const float *from, int lane, float &top, float &sum, f32x4 &o)
{
  const f32x4 x = *reinterpret_cast<const f32x4 *>(from + 4 * lane);
  const float m = from[kDim], l = from[kDim + 1], next = fmaxf(top, m);
  const float a = __builtin_amdgcn_exp2f(top - next), b = __builtin_amdgcn_exp2f(m - next);
  top = next;
  sum = sum * a + l * b;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = o[k] * a + x[k] * b;
}

// What the kernel for few rows left: a tile (of a kv head) that was cut is joined from its parts by the workgroup with the number of the one in
// which it begins, a group of lanes a row; one that is marked is computed again.
template <class T, int kDim>
__device__ __forceinline__ void finish_rows(const AttentionParams &p)
{
  constexpr int kLanes = kDim / 4, kGroups = kThreads / kLanes, which = RowsShape::kPlan;
  const int n = p.batch.requests, kv_heads = p.cache.kv_heads, lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  uint32_t flags = 0;
  if (static_cast<int>(blockIdx.x) < p.blocks[which]) {
    const int first = blockIdx.x;
    const CutTile cut = cut_tiles(p)[first];
    if (cut.rows) {
      int marked = threadIdx.x == 0 ? cut.mark[1] : 0;
      for (int b = first + 1 + static_cast<int>(threadIdx.x); b <= cut.last; b += kThreads) marked |= cut_tiles(p)[b].mark[0];
      for (int y = group; y < cut.rows; y += kGroups) {
        float top = -FLT_MAX, sum = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        add_part<kDim>(part_of(p, which, (2 * static_cast<int64_t>(first) + 1) * RowsShape::kRows + y), lane, top, sum, o);
#pragma unroll 4
        for (int b = first + 1; b <= cut.last; ++b) add_part<kDim>(part_of(p, which, 2 * static_cast<int64_t>(b) * RowsShape::kRows + y), lane, top, sum, o);
        const int row = cut.tile * 16 + y;
        write_row<T>(p, cut.token + row / p.group, cut.head * p.group + row % p.group, 4 * lane, o, sum);
      }
      if (__syncthreads_or(marked)) {                           // (and what was written above is written over)
        const Request rq = request_of(p, cut.request, &flags);
        for (int y = threadIdx.x / 64; y < cut.rows; y += kWaves) one_row<T, kDim>(p, cut.request, rq, cut.tile * 16 + y, cut.head);
      }
    }
  }
  // tiles that were not cut
  const int *marks = marks_of(p, which);
  const int64_t *start = reinterpret_cast<const int64_t *>(kept_plan(p, which));
  const int *tiles = reinterpret_cast<const int *>(start + n + 1);
  const int64_t items = min(p.units[which], static_cast<int64_t>(tiles[n]) * kv_heads);
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    if (!marks[item]) continue;
    const int r = last_not_above<int>(tiles, n, static_cast<int>(item / kv_heads));
    const Request rq = request_of(p, r, &flags);
    int all_rows, blocks;
    tiles_of<RowsShape>(p, rq, all_rows, blocks);
    const int64_t nth = item - static_cast<int64_t>(tiles[r]) * kv_heads;
    const int tile = static_cast<int>(nth / kv_heads), head = static_cast<int>(nth % kv_heads);
    for (int y = threadIdx.x / 64; y < min(16, all_rows - tile * 16); y += kWaves) one_row<T, kDim>(p, r, rq, tile * 16 + y, head);
  }
}

// What the kernel for chunks left: the rows of marked units, a wave for a row ...
template <class T, int kDim>
__device__ __forceinline__ void marked_chunks(const AttentionParams &p, int *starts)
{
  constexpr int which = ChunkShape::kPlan;
  const int n = p.batch.requests;
  const int *start = kept_plan(p, which), *marks = marks_of(p, which);
  const int64_t units = min(p.units[which], static_cast<int64_t>(start[n]) * p.cache.kv_heads);
  bool any = false;
  for (int64_t u = blockIdx.x + static_cast<int64_t>(threadIdx.x) * gridDim.x; u < units; u += static_cast<int64_t>(kThreads) * gridDim.x) any |= marks[u] != 0;
  if (!__syncthreads_or(any)) return;                           // (and nobody looks at joins any more)
  for (int r = threadIdx.x; r <= n; r += kThreads) starts[r] = start[r];
  __syncthreads();
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    if (!marks[u]) continue;
    const int unit = static_cast<int>(u / p.cache.kv_heads), head = static_cast<int>(u % p.cache.kv_heads);
    const int r = last_not_above<int>(starts, n, unit);
    uint32_t flags = 0;
    const Request rq = request_of(p, r, &flags);
    const int rows = rq.tokens * p.group, tiles = (rows + ChunkShape::kRows - 1) / ChunkShape::kRows, splits = (starts[r + 1] - starts[r]) / tiles;
    const int tile = tile_of_unit(unit - starts[r], tiles, splits), first = (unit - starts[r]) / splits * splits;
    // of the marked pieces of a tile the first one's workgroup computes its rows
    bool before = false;
    for (int s = first; s < unit - starts[r]; ++s) before |= marks[static_cast<int64_t>(starts[r] + s) * p.cache.kv_heads + head] != 0;
    if (before) continue;
    for (int row = tile * ChunkShape::kRows + threadIdx.x / 64; row < min(rows, (tile + 1) * ChunkShape::kRows); row += kWaves) one_row<T, kDim>(p, r, rq, row, head);
  }
}

// ... and rows whose keys were cut: a group of lanes for a row.
template <class T, int kDim>
__device__ __forceinline__ void join_chunks(const AttentionParams &p, int *joins)
{
  constexpr int kLanes = kDim / 4, kGroups = kThreads / kLanes, which = ChunkShape::kPlan;
  const int n = p.batch.requests, lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int *start = kept_plan(p, which), *part = start + n + 1, *join = part + n + 1, *marks = marks_of(p, which);
  const int64_t items = static_cast<int64_t>(join[n]) * p.cache.kv_heads;
  if (items == 0) return;
  for (int r = threadIdx.x; r <= n; r += kThreads) joins[r] = join[r];
  __syncthreads();
  for (int64_t item = static_cast<int64_t>(blockIdx.x) * kGroups + group; item < items; item += static_cast<int64_t>(gridDim.x) * kGroups) {
    const int head = static_cast<int>(item % p.cache.kv_heads), at = static_cast<int>(item / p.cache.kv_heads);
    const int r = last_not_above<int>(joins, n, at), row = at - joins[r], rows = joins[r + 1] - joins[r];
    const int64_t first = part[r];
    const int splits = (part[r + 1] - part[r]) / rows, tiles = (rows + ChunkShape::kRows - 1) / ChunkShape::kRows;
    const int64_t unit = start[r] + static_cast<int64_t>(tiles - 1 - row / ChunkShape::kRows) * splits;
    uint32_t flags = 0;
    const Request rq = request_of(p, r, &flags);
    float top = -FLT_MAX, sum = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    int marked = 0;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
      add_part<kDim>(part_of(p, which, (first + static_cast<int64_t>(s) * rows + row) * p.cache.kv_heads + head), lane, top, sum, o);
      const int64_t mark = (unit + s) * p.cache.kv_heads + head;
      if (mark < p.units[which]) marked |= marks[mark];
    }
    if (!marked) write_row<T>(p, rq.first + row / p.group, head * p.group + row % p.group, 4 * lane, o, sum);
  }
}

template <class T, int kDim, bool kChunks>
__global__ void __launch_bounds__(kThreads, 4) gnr_attention_join_kernel(const AttentionParams p)
{
  extern __shared__ int64_t memory[];
  if constexpr (kChunks) {
    join_chunks<T, kDim>(p, reinterpret_cast<int *>(memory));
    marked_chunks<T, kDim>(p, reinterpret_cast<int *>(memory));
  } else {
    finish_rows<T, kDim>(p);
  }
}

// Fills in what the host decides: which kernel takes which requests, how many workgroups each has, and where its parts lie. Returns
// the words of the workspace.
static int64_t decide(AttentionParams &p)
{
  const int64_t rows = p.batch.tokens * p.group, longest = p.batch.max_q * p.group;
  const int64_t keys = p.batch.table_width << p.page_shift;
  p.room = static_cast<int>(keys < (int64_t(1) << 30) ? keys : int64_t(1) << 30);
  // one request alone has every row; else what the caller expects of the longest says whether there are chunks
  const bool chunks = p.batch.requests == 1 ? rows > kFewRows : longest > kFewRows;
  const bool few = p.batch.requests > 1 || !chunks;
  p.least[0] = 0; p.most[0] = chunks ? kFewRows : INT32_MAX;
  p.least[1] = few ? kFewRows + 1 : 0; p.most[1] = INT32_MAX;
  const auto blocks = [&](bool used, int64_t most, int64_t tile, int64_t block) -> int64_t {
    // no more workgroups than there can be tiles and blocks of keys
    const int64_t units = (p.batch.requests + rows / tile) * ((keys + block - 1) / block + 1) * p.cache.kv_heads;
    return !used ? 0 : units < most ? units : most;
  };
  p.blocks[0] = static_cast<int>(blocks(few, kComputeUnits * rows_blocks(p.cache.head_dim), RowsShape::kRows, RowsShape::kKeys));
  p.blocks[1] = static_cast<int>(blocks(chunks, kComputeUnits * chunk_blocks(p.cache.head_dim), ChunkShape::kRows, ChunkShape::kKeys));
  // Marks of the kernel for few rows: every (tile, head); of the one for chunks: units, as many as there are
  // workgroups and one more for each tile. Parts: of the former the slots' rows; of the latter, a request that is cut has fewer than
  // twice as many pieces as its keys fill.
  const int64_t words = p.cache.head_dim + kPartTail, heads = p.cache.kv_heads;
  int64_t at = (6 * static_cast<int64_t>(p.batch.requests + 1) + 15) / 16 * 16;
  const int64_t units[2] = {(p.batch.requests + rows / RowsShape::kRows) * heads, p.blocks[1] + (p.batch.requests + rows / ChunkShape::kRows) * heads};
  const int64_t parts[2] = {2 * static_cast<int64_t>(p.blocks[0]) * RowsShape::kRows, 2 * static_cast<int64_t>(p.blocks[1]) * ChunkShape::kRows};
  for (int i = 0; i < 2; ++i) {
    p.marks[i] = at;
    p.units[i] = p.blocks[i] ? units[i] : 0;
    at += (p.units[i] + 15) / 16 * 16;
    p.parts[i] = at;
    at += parts[i] * words;
  }
  p.cuts = at;
  return at + p.blocks[0] * static_cast<int64_t>(sizeof(CutTile) / sizeof(float));
}

size_t attention_bytes(const iter_cache &c, const iter_batch &b, int heads)
{
  AttentionParams p{};
  p.cache = c;
  p.batch = b;
  p.group = heads / c.kv_heads;
  p.page_shift = __builtin_ctz(static_cast<unsigned>(c.page));
  return static_cast<size_t>(decide(p)) * sizeof(float);
}

template <class T, bool kChunks>
static int launch_join(const AttentionParams &p, hipStream_t stream)
{
  const size_t lds = plan_bytes(p.batch.requests);
  const int64_t items = p.batch.tokens * p.group * p.cache.kv_heads;
  const unsigned blocks = static_cast<unsigned>(!kChunks ? p.blocks[RowsShape::kPlan] : items < kJoinBlocks ? items : kJoinBlocks);
  switch (p.cache.head_dim) {
    case 64: gnr_attention_join_kernel<T, 64, kChunks><<<blocks, kThreads, lds, stream>>>(p); break;
    case 128: gnr_attention_join_kernel<T, 128, kChunks><<<blocks, kThreads, lds, stream>>>(p); break;
    default: gnr_attention_join_kernel<T, 256, kChunks><<<blocks, kThreads, lds, stream>>>(p); break;
  }
  return iter_hip_ok(hipGetLastError());
}

int launch_attention(const AttentionParams &params, void *stream)
{
  const hipStream_t s = static_cast<hipStream_t>(stream);
  AttentionParams p = params;
  decide(p);
  int rc = SIM_OK;
  if (p.blocks[0]) rc = launch_attention_rows(p, s);
  if (rc == SIM_OK && p.blocks[1]) rc = launch_attention_chunk(p, s);
  if (rc == SIM_OK && p.blocks[0]) rc = p.type == ITER_BF16 ? launch_join<Bf16, false>(p, s) : launch_join<Fp16, false>(p, s);
  if (rc == SIM_OK && p.blocks[1]) rc = p.type == ITER_BF16 ? launch_join<Bf16, true>(p, s) : launch_join<Fp16, true>(p, s);
  return rc;
}

}  // namespace gnr
