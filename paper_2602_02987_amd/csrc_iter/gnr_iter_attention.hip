// Attention of a mixed batch over the paged cache (gfx950): every token of every request over its own request's keys.
#include "gnr_iter_attention.h"

namespace gnr {

// ---- sharing the work out

// What a request asks for. Bounds that contradict each other or the arrays are cut down to what is inside them.
struct Request {
  int first, tokens;        // of the batch
  int64_t last;             // position of the last token
  int64_t begin, end;       // keys that any of its tokens sees, [begin, end); begin is a multiple of 32
};

__device__ __forceinline__ Request request_of(const AttentionParams &p, int r, uint32_t *flags)
{
  const int64_t total = p.batch.tokens;
  int64_t b = p.batch.q_start[r], e = p.batch.q_start[r + 1];
  const int64_t length = p.batch.kv_len[r], room = p.batch.table_width << p.page_shift;
  if (b < 0 || e < b || e > total || length < 0 || length > room || (r == 0 && b != 0) || (r == p.batch.requests - 1 && e != total))
    *flags |= ITER_BAD_BATCH;
  b = b < 0 ? 0 : b > total ? total : b;
  e = e < b ? b : e > total ? total : e;
  Request q;
  q.first = static_cast<int>(b);
  q.tokens = static_cast<int>(e - b);
  q.last = length - 1;
  q.end = length < 0 ? 0 : length > room ? room : length;
  int64_t begin = p.window ? length - q.tokens - p.window + 1 : 0;
  begin = begin < 0 ? 0 : begin;
  q.begin = begin & ~int64_t(31);
  if (q.end < q.begin) q.end = q.begin;
  return q;
}

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

// The keys of a request are shared out in pieces, so that few long rows fill the chip and a long request does not outlast the others:
// about kPiecesPerBlock pieces to a workgroup, whole blocks of kBlockKeys keys, the pieces of a request as long as each other. Every workgroup finds the
// same partition from the batch itself, which costs two microseconds of a launch and spares the host from knowing the lengths.
// start[r]: units (pieces of a tile of 16 rows) before request r; part[r]: of those that leave a part to be joined.
__device__ __forceinline__ void share_out(const AttentionParams &p, int blocks, int *start, int *part, int *scratch)
{
  const int n = p.batch.requests;
  uint32_t flags = 0;
  int64_t all = 0;
  __shared__ unsigned long long sum;
  if (threadIdx.x == 0) sum = 0;
  __syncthreads();
  for (int r = threadIdx.x; r < n; r += kThreads) {
    const Request q = request_of(p, r, &flags);
    if (q.tokens) all += (static_cast<int64_t>(q.tokens) * p.group + 15) / 16 * ((q.end - q.begin + kBlockKeys - 1) / kBlockKeys);
  }
#pragma unroll
  for (int d = 32; d; d /= 2) all += __shfl_xor(all, d);
  if (threadIdx.x % 64 == 0) atomicAdd(&sum, static_cast<unsigned long long>(all));
  if (flags && p.status && blockIdx.x == 0) atomicOr(p.status, flags);
  __syncthreads();
  const int64_t pieces = static_cast<int64_t>(blocks) * kPiecesPerBlock;
  const int64_t size = max(int64_t(1), (static_cast<int64_t>(sum) * p.cache.kv_heads + pieces - 1) / pieces);
  int units = 0, parts = 0;
  for (int r0 = 0; r0 < n; r0 += kThreads) {
    const int r = r0 + threadIdx.x;
    int u = 0, l = 0;
    if (r < n) {
      const Request q = request_of(p, r, &flags);
      if (q.tokens) {
        const int64_t keys = (q.end - q.begin + kBlockKeys - 1) / kBlockKeys, tiles = (static_cast<int64_t>(q.tokens) * p.group + 15) / 16;
        const int64_t splits = max(int64_t(1), (keys + size - 1) / size);
        u = static_cast<int>(tiles * splits);
        l = splits > 1 ? u : 0;
      }
    }
    int before, total;
    block_scan(u, scratch, before, total);
    if (r < n) start[r] = units + before;
    units += total;
    block_scan(l, scratch, before, total);
    if (r < n) part[r] = parts + before;
    parts += total;
  }
  if (threadIdx.x == 0) {
    start[n] = units;
    part[n] = parts;
  }
  __syncthreads();
}

// ---- a tile of 16 rows

// Sixteen rows (the query heads of a kv head, for one token or a few) against a piece of their keys. Transposed products keep everything in
// registers: S^T = K Q^T leaves a lane with four keys of one row, which is what the second product, O^T = V^T P^T, wants of its right
// operand, if keys are numbered alike on both sides: lane group g and element j stand for key 16 (j / 4) + 4 g + j % 4 of 32. A lane reads head_dim / 16
// neighbouring elements of eight keys' values and swaps halves of registers to have eight keys of one element; no shared memory is used,
// every byte of the cache goes from memory to the registers of the wave that multiplies it. Each wave takes every fourth block of 32 keys with a
// running maximum and sum of its own; the waves are joined at the end.
//   Bound by the memory: 2 head_dim bytes a key and element size against 16 rows of products is far below the matrix rate.
template <class T, int kDim, bool kFp8, bool kSmallPages>
struct Tile {
  static constexpr int kVec = kDim / 16;                        // elements of a value row a lane reads
  static constexpr int kFrags = kDim / 32;                      // matrix products over the elements of a key
  static constexpr int kKeyWords = kFp8 ? kDim / 16 : kDim / 8; // words of a key a lane reads
  static constexpr int kValWords = kFp8 ? kVec / 4 : kVec / 2;
  typedef typename T::oct oct;

  const AttentionParams &p;
  const int lane, n, g;                                         // n: row, and key or element index of the operands; g: group of 16 lanes
  oct q[kFrags];
  f32x4 acc[kVec];
  float top, sum;                                               // of row n; `sum` of this lane's keys only
  uint32_t kw[2][kKeyWords], vw[8][kValWords];
  float ks[2], vs[8];

  __device__ __forceinline__ Tile(const AttentionParams &params, int l) : p(params), lane(l), n(l % 16), g(l / 16) {}

  // elements of a row that fragment f of a lane holds; the 8-bit cache is read 16 elements at a time
  __device__ __forceinline__ int element(int f) const { return kFp8 ? 64 * (f / 2) + 16 * g + 8 * (f % 2) : 32 * f + 8 * g; }

  __device__ __forceinline__ void begin(const uint16_t *row)
  {
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {
      u32x4 w = {0, 0, 0, 0};
      if (row) w = *reinterpret_cast<const u32x4 *>(row + element(f));
      q[f] = bits<oct>(w);
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) acc[e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    top = -FLT_MAX;
    sum = 0.0f;
  }

  template <int kWords>
  static __device__ __forceinline__ void load_words(const void *at, uint32_t *w)
  {
    if constexpr (kWords == 1) w[0] = *static_cast<const uint32_t *>(at);
    else if constexpr (kWords == 2) {
      const u32x2 x = *static_cast<const u32x2 *>(at);
      w[0] = x[0]; w[1] = x[1];
    } else {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const u32x4 x = static_cast<const u32x4 *>(at)[i];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[4 * i + k] = x[k];
      }
    }
  }

  static constexpr int kSize = kFp8 ? 1 : 2;

  // The key `key` (0..15) of the sixteen at `page` from `place` on.
  __device__ __forceinline__ void load_key(int t, int64_t page, int64_t place, int head)
  {
    const iter_plane &c = p.cache.k;
    const char *row = static_cast<const char *>(c.data) + (page * c.page_stride + head * c.head_stride + place * c.place_stride) * kSize;
    if constexpr (kFp8) {
      ks[t] = exponent_scale(c.exp[page * c.exp_page_stride + head * c.exp_head_stride + place * c.exp_place_stride]);
#pragma unroll
      for (int i = 0; i < kKeyWords / 4; ++i) load_words<4>(row + 64 * i + 16 * g, &kw[t][4 * i]);
    } else {
#pragma unroll
      for (int i = 0; i < kKeyWords / 4; ++i) load_words<4>(row + 64 * i + 16 * g, &kw[t][4 * i]);
    }
  }

  __device__ __forceinline__ void load_value(int j, int64_t page, int64_t place, int head)
  {
    const iter_plane &c = p.cache.v;
    const char *row = static_cast<const char *>(c.data) + (page * c.page_stride + head * c.head_stride + place * c.place_stride) * kSize;
    if constexpr (kFp8) vs[j] = exponent_scale(c.exp[page * c.exp_page_stride + head * c.exp_head_stride + place * c.exp_place_stride]);
    load_words<kValWords>(row + kVec * kSize * n, vw[j]);
  }

  // Pages of the two sixteens of a block of keys: uniform, or (pages of fewer than 16 tokens) looked up key by key.
  __device__ __forceinline__ void load_keys(int64_t k0, const int *pages, const int32_t *table, int64_t end, int head)
  {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int64_t key = k0 + 16 * t + n;
      if constexpr (kSmallPages) load_key(t, page_of(key, table, end), key & (p.cache.page - 1), head);
      else load_key(t, max(pages[t], 0), ((k0 + 16 * t) & (p.cache.page - 1)) + n, head);
    }
  }

  __device__ __forceinline__ void load_values(int64_t k0, const int *pages, const int32_t *table, int64_t end, int head)
  {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = j / 4, in = 4 * g + j % 4;
      const int64_t key = k0 + 16 * t + in;
      if constexpr (kSmallPages) load_value(j, page_of(key, table, end), key & (p.cache.page - 1), head);
      else load_value(j, max(pages[t], 0), ((k0 + 16 * t) & (p.cache.page - 1)) + in, head);
    }
  }

  // a page that holds the key, or page 0 for one that is not there (whose scores and values are not used)
  __device__ __forceinline__ int64_t page_of(int64_t key, const int32_t *table, int64_t end) const
  {
    if (key >= end) return 0;
    const int page = table[key >> p.page_shift];
    return page >= 0 && page < p.cache.pages ? page : 0;
  }
  __device__ __forceinline__ bool page_there(int64_t key, const int32_t *table, int64_t end) const
  {
    if (key >= end) return false;
    const int page = table[key >> p.page_shift];
    const bool there = page >= 0 && page < p.cache.pages;
    if (!there && p.status) atomicOr(p.status, ITER_BAD_PAGE);
    return there;
  }

  // scores of the 32 keys: s[t][i] belongs to key 16 t + 4 g + i
  __device__ __forceinline__ void scores(f32x4 *s) const
  {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        u32x4 w;
        if constexpr (kFp8) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t c = kw[t][4 * (f / 2) + 2 * (f % 2) + i];
            w[2 * i] = T::template from_e4m3<false>(c, ks[t]);
            w[2 * i + 1] = T::template from_e4m3<true>(c, ks[t]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = kw[t][4 * f + i];
        }
        s[t] = T::mfma16(bits<oct>(w), q[f], s[t]);
      }
    }
  }

  // Weights of the 32 keys; the running maximum moves when a score exceeds it by 2^8, so that most blocks need no exchange between
  // lanes and no rescaling (weights stay below 2^8, sums and products lose nothing).
  __device__ __forceinline__ void weigh(f32x4 *s, uint32_t *w)
  {
    float high = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) high = fmaxf(high, s[t][i]);
    if (__any(high - top > 8.0f)) {
      high = fmaxf(high, __shfl_xor(high, 16));
      high = fmaxf(high, __shfl_xor(high, 32));
      const float next = fmaxf(top, high);
      const float keep = __builtin_amdgcn_exp2f(top - next);
      top = next;
      sum *= keep;
#pragma unroll
      for (int e = 0; e < kVec; ++e) acc[e] *= keep;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[t][i] = __builtin_amdgcn_exp2f(s[t][i] - top);
        sum += s[t][i];
      }
      w[2 * t] = T::narrow2(s[t][0], s[t][1]);
      w[2 * t + 1] = T::narrow2(s[t][2], s[t][3]);
    }
  }

  // the values as 16-bit words, still eight keys of kVec elements
  __device__ __forceinline__ void widen_values(uint32_t (*v)[kVec / 2]) const
  {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < kVec / 2; ++i) {
        if constexpr (kFp8) v[j][i] = i % 2 ? T::template from_e4m3<true>(vw[j][i / 2], vs[j]) : T::template from_e4m3<false>(vw[j][i / 2], vs[j]);
        else v[j][i] = vw[j][i];
      }
  }

  __device__ __forceinline__ void add_values(uint32_t (*v)[kVec / 2], const uint32_t *w)
  {
    const oct weights = bits<oct>(u32x4{w[0], w[1], w[2], w[3]});
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      u32x4 a;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        a[i] = __builtin_amdgcn_perm(v[2 * i + 1][e / 2], v[2 * i][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
      acc[e] = T::mfma16(bits<oct>(a), weights, acc[e]);
    }
  }
};

// Where a row's results go when its keys were shared out: the sum of weighted values, relative to the maximum, then maximum and sum.
__device__ __forceinline__ float *part_row(const AttentionParams &p, int dim, int64_t part, int row)
{
  return p.workspace + p.header + (part * 16 + row) * (dim + kPartTail);
}

template <class T, int kDim, bool kFp8, bool kSmallPages>
__global__ void __launch_bounds__(kThreads, kDim == 256 ? 1 : 3) gnr_attention_rows_kernel(const AttentionParams p)
{
  typedef Tile<T, kDim, kFp8, kSmallPages> Rows;
  extern __shared__ int shared[];
  __shared__ int scratch[kWaves];
  __shared__ float tops[kWaves][16], sums[kWaves][16];
  __shared__ float outs[kWaves][16][kDim + 4];
  const int requests = p.batch.requests, kv_heads = p.cache.kv_heads;
  int *start = shared, *part = shared + requests + 1;
  share_out(p, gridDim.x, start, part, scratch);
  if (blockIdx.x == 0) {
    int *plan = reinterpret_cast<int *>(p.workspace);
    for (int r = threadIdx.x; r <= requests; r += kThreads) {
      plan[2 * r] = start[r];
      plan[2 * r + 1] = part[r];
    }
  }
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Rows rows(p, lane);
  const int64_t units = static_cast<int64_t>(start[requests]) * kv_heads;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int unit = static_cast<int>(u / kv_heads), head = static_cast<int>(u % kv_heads);
    int r = 0;                                                   // the last request that starts at or before `unit`
    for (int step = 2048; step; step /= 2)
      if (r + step < requests && start[r + step] <= unit) r += step;
    uint32_t flags = 0;
    const Request rq = request_of(p, r, &flags);
    const int tiles = (rq.tokens * p.group + 15) / 16, splits = (start[r + 1] - start[r]) / tiles;
    const int tile = (unit - start[r]) / splits, split = (unit - start[r]) % splits;
    const int64_t blocks = (rq.end - rq.begin + kBlockKeys - 1) / kBlockKeys, each = (blocks + splits - 1) / splits;
    const int64_t from = rq.begin + min(blocks, split * each) * kBlockKeys;
    const int64_t to = min(rq.end, rq.begin + min(blocks, (split + 1) * each) * kBlockKeys);
    const int32_t *table = p.batch.page_table + r * p.batch.table_stride;
    const int row = tile * 16 + rows.n, token = row / p.group;
    const bool real = row < rq.tokens * p.group;
    const uint16_t *q = static_cast<const uint16_t *>(p.q.data) + static_cast<int64_t>(rq.first + token) * p.q.token_stride +
                        (head * p.group + row % p.group) * p.q.head_stride;
    rows.begin(real ? q : nullptr);
    // the keys this lane's row sees, and those that every row sees
    const int last_token = min(rq.tokens - 1, (tile * 16 + 15) / p.group);
    const int64_t pos = rq.last - (rq.tokens - 1) + min(token, rq.tokens - 1);
    const int64_t see_end = min(pos + 1, rq.end), see_begin = p.window ? pos - p.window + 1 : 0;
    const int64_t pos_first = rq.last - (rq.tokens - 1) + tile * 16 / p.group, pos_last = rq.last - (rq.tokens - 1) + last_token;
    const int64_t all_end = min(pos_first + 1, rq.end), all_begin = p.window ? pos_last - p.window + 1 : 0;
    const int64_t stop = min(to, pos_last + 1);                  // nobody sees what is beyond
    // the pages of 32 blocks of this wave at a time: lane 2 i + t holds the t-th sixteen's of the i-th
    int pages_ahead = 0;
    const auto look_up = [&](int64_t k0) {
      const int64_t key = k0 + (lane / 2) * kBlockKeys + 16 * (lane % 2);
      int page = 0;
      if (key < stop) {
        page = table[key >> p.page_shift];
        if (page < 0 || page >= p.cache.pages) {
          page = -1;
          if (p.status) atomicOr(p.status, ITER_BAD_PAGE);
        }
      }
      pages_ahead = page;
    };
    int64_t k0 = from + 32 * wave;
    int step = 0;
    int pages[2] = {0, 0}, next[2] = {0, 0};
    if (k0 < stop && p.cache.pages > 0) {
      if constexpr (!kSmallPages) {
        look_up(k0);
        pages[0] = __builtin_amdgcn_readlane(pages_ahead, 0);
        pages[1] = __builtin_amdgcn_readlane(pages_ahead, 1);
      }
      rows.load_keys(k0, pages, table, stop, head);
      rows.load_values(k0, pages, table, stop, head);
      while (true) {
        const int64_t k1 = k0 + kBlockKeys;
        const bool more = k1 < stop;
        ++step;
        if constexpr (!kSmallPages) {
          if (step == 32) {
            look_up(k1);
            step = 0;
          }
          next[0] = __builtin_amdgcn_readlane(pages_ahead, 2 * step);
          next[1] = __builtin_amdgcn_readlane(pages_ahead, 2 * step + 1);
        }
        f32x4 s[2];
        rows.scores(s);
        if (more) rows.load_keys(k1, next, table, stop, head);
        bool ragged = k0 < all_begin || k0 + 32 > all_end;
        if constexpr (kSmallPages) ragged = true;
        else ragged |= (pages[0] | pages[1]) < 0;
        uint32_t seen = 0xFFu;                                   // bit 4 t + i: whether row n sees key 16 t + 4 g + i
        if (ragged) {
          seen = 0;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int64_t key = k0 + 16 * t + 4 * rows.g + i;
              bool see = key >= see_begin && key < see_end;
              if constexpr (kSmallPages) see = rows.page_there(key, table, stop) && see;
              else see = see && pages[t] >= 0;
              seen |= see ? 1u << (4 * t + i) : 0u;
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][i] = seen >> (4 * t + i) & 1u ? s[t][i] * p.scale_log2 : -INFINITY;
        uint32_t w[4];
        rows.weigh(s, w);
        uint32_t v[8][Rows::kVec / 2];
        rows.widen_values(v);
        if (ragged) {
          // A weight of zero does not silence a NaN or an infinity. Where any stands among the values of these keys, the
          // products are made one by one for the rows that see the key.
          bool odd = false;
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < Rows::kVec / 2; ++i)
              odd |= (v[j][i] & T::kInf) == T::kInf || (v[j][i] >> 16 & T::kInf) == T::kInf;
          if (__any(odd)) {
            for (int key = 0; key < 32; ++key) {
              const int t = key / 16, owner = key % 16 / 4 * 16, i = key % 4;
              const float mine = i == 0 ? s[t][0] : i == 1 ? s[t][1] : i == 2 ? s[t][2] : s[t][3];
              const float weight = T::widen(T::narrow2(__shfl(mine, owner + rows.n), 0.0f));
              const bool see = __shfl(seen, owner + rows.n) >> (4 * t + i) & 1u;
#pragma unroll
              for (int e = 0; e < Rows::kVec; ++e)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  // element kVec (4 g + k) + e of the key is held by lane 16 (key % 16 / 4) + 4 g + k
                  const uint32_t word = t ? (i == 0 ? v[4][e / 2] : i == 1 ? v[5][e / 2] : i == 2 ? v[6][e / 2] : v[7][e / 2])
                                          : (i == 0 ? v[0][e / 2] : i == 1 ? v[1][e / 2] : i == 2 ? v[2][e / 2] : v[3][e / 2]);
                  const uint32_t got = __shfl(word, owner + 4 * rows.g + k);
                  const float value = T::widen(e % 2 ? got >> 16 : got & 0xFFFFu);
                  if (see) rows.acc[e][k] = __builtin_fmaf(weight, value, rows.acc[e][k]);
                }
            }
          } else {
            rows.add_values(v, w);
          }
        } else {
          rows.add_values(v, w);
        }
        if (!more) break;
        rows.load_values(k1, next, table, stop, head);
        k0 = k1;
        pages[0] = next[0];
        pages[1] = next[1];
      }
    }
    // join the waves
    float sum = rows.sum;
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    __syncthreads();                                             // the unit before has been read
    if (rows.g == 0) {
      tops[wave][rows.n] = rows.top;
      sums[wave][rows.n] = sum;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < Rows::kVec; ++e) outs[wave][rows.n][Rows::kVec * (4 * rows.g + i) + e] = rows.acc[e][i];
    __syncthreads();
    const int real_rows = min(16, rq.tokens * p.group - tile * 16);
    for (int i = threadIdx.x; i < real_rows * (kDim / 4); i += kThreads) {
      const int y = i / (kDim / 4), d = i % (kDim / 4) * 4;
      float most = tops[0][y];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) most = fmaxf(most, tops[w][y]);
      float all = 0.0f;
      f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(tops[w][y] - most);
        all = __builtin_fmaf(sums[w][y], f, all);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = __builtin_fmaf(outs[w][y][d + k], f, o[k]);
      }
      if (splits == 1) {
        const int at = tile * 16 + y;
        write_row<T>(p, rq.first + at / p.group, head * p.group + at % p.group, d, o, all);
      } else {
        float *to_part = part_row(p, kDim, (static_cast<int64_t>(part[r]) + unit - start[r]) * kv_heads + head, y);
        *reinterpret_cast<f32x4 *>(to_part + d) = o;
        if (d == 0) {
          to_part[kDim] = most;
          to_part[kDim + 1] = all;
        }
      }
    }
  }
}

// Joins the parts of the rows whose keys were shared out: a workgroup for a row at a time, eight groups of lanes with every eighth part each.
template <class T, int kDim>
__global__ void __launch_bounds__(kThreads) gnr_attention_join_kernel(const AttentionParams p)
{
  constexpr int kLanes = kDim / 4, kGroups = kThreads / kLanes;
  __shared__ float tops[kGroups], sums[kGroups];
  __shared__ f32x4 outs[kGroups][kLanes];
  const int *plan = reinterpret_cast<const int *>(p.workspace);
  const int r = blockIdx.x / p.cache.kv_heads, head = blockIdx.x % p.cache.kv_heads;
  const int parts = plan[2 * (r + 1) + 1] - plan[2 * r + 1];
  if (parts == 0) return;
  uint32_t flags = 0;
  const Request rq = request_of(p, r, &flags);
  const int rows = rq.tokens * p.group, tiles = (rows + 15) / 16, splits = parts / tiles;
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  for (int row = blockIdx.y; row < rows; row += gridDim.y) {
    const int64_t first = static_cast<int64_t>(plan[2 * r + 1]) + row / 16 * splits;
    float top = -FLT_MAX, sum = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = group; s < splits; s += kGroups) {
      const float *from = part_row(p, kDim, (first + s) * p.cache.kv_heads + head, row % 16);
      const f32x4 x = *reinterpret_cast<const f32x4 *>(from + 4 * lane);
      const float m = from[kDim], l = from[kDim + 1], next = fmaxf(top, m);
      const float a = __builtin_amdgcn_exp2f(top - next), b = __builtin_amdgcn_exp2f(m - next);
      top = next;
      sum = sum * a + l * b;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = o[k] * a + x[k] * b;
    }
    __syncthreads();
    if (lane == 0) {
      tops[group] = top;
      sums[group] = sum;
    }
    outs[group][lane] = o;
    __syncthreads();
    if (group == 0) {
      float most = top;
#pragma unroll
      for (int s = 1; s < kGroups; ++s) most = fmaxf(most, tops[s]);
      float all = 0.0f;
      o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < kGroups; ++s) {
        const float f = __builtin_amdgcn_exp2f(tops[s] - most);
        all = __builtin_fmaf(sums[s], f, all);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = __builtin_fmaf(outs[s][lane][k], f, o[k]);
      }
      write_row<T>(p, rq.first + row / p.group, head * p.group + row % p.group, 4 * lane, o, all);
    }
  }
}

// ---- host

static int64_t blocks_for(const iter_cache &c, const iter_batch &b, int heads)
{
  // no more workgroups than there are blocks of keys
  const int64_t tiles = b.requests + b.tokens * (heads / c.kv_heads) / 16;
  const int64_t keys = (b.table_width * c.page + kBlockKeys - 1) / kBlockKeys;
  const int64_t most = tiles * (keys < 1 ? 1 : keys);
  return most * c.kv_heads < kBlocks ? most * c.kv_heads : kBlocks;
}

static size_t header_floats(const iter_batch &b) { return (static_cast<size_t>(b.requests + 1) * 2 + 15) / 16 * 16; }

size_t attention_bytes(const iter_cache &c, const iter_batch &b, int heads)
{
  // a request that is shared out has fewer than twice as many pieces as its keys fill
  const int64_t blocks = blocks_for(c, b, heads);
  const size_t parts = static_cast<size_t>(2 * blocks * kPiecesPerBlock + 2 * c.kv_heads);
  return (header_floats(b) + parts * 16 * (c.head_dim + kPartTail)) * sizeof(float);
}

template <class T, int kDim, bool kFp8>
static int launch_rows(const AttentionParams &p, hipStream_t stream)
{
  const unsigned blocks = static_cast<unsigned>(blocks_for(p.cache, p.batch, p.heads));
  const size_t lds = static_cast<size_t>(p.batch.requests + 1) * 2 * sizeof(int);
  if (p.cache.page < 16) gnr_attention_rows_kernel<T, kDim, kFp8, true><<<blocks, kThreads, lds, stream>>>(p);
  else gnr_attention_rows_kernel<T, kDim, kFp8, false><<<blocks, kThreads, lds, stream>>>(p);
  const int rc = iter_hip_ok(hipGetLastError());
  if (rc != SIM_OK) return rc;
  const dim3 join(static_cast<unsigned>(p.batch.requests) * static_cast<unsigned>(p.cache.kv_heads), p.group < 16 ? p.group : 16);
  gnr_attention_join_kernel<T, kDim><<<join, kThreads, 0, stream>>>(p);
  return iter_hip_ok(hipGetLastError());
}

template <class T, bool kFp8>
static int launch_dim(const AttentionParams &p, hipStream_t stream)
{
  switch (p.cache.head_dim) {
    case 64: return launch_rows<T, 64, kFp8>(p, stream);
    case 128: return launch_rows<T, 128, kFp8>(p, stream);
    default: return launch_rows<T, 256, kFp8>(p, stream);
  }
}

int launch_attention(const AttentionParams &params, void *stream)
{
  const hipStream_t s = static_cast<hipStream_t>(stream);
  AttentionParams p = params;
  p.header = static_cast<int64_t>(header_floats(p.batch));
  const bool fp8 = p.cache.type == ITER_FP8;
  if (p.type == ITER_BF16) return fp8 ? launch_dim<Bf16, true>(p, s) : launch_dim<Bf16, false>(p, s);
  return fp8 ? launch_dim<Fp16, true>(p, s) : launch_dim<Fp16, false>(p, s);
}

}  // namespace gnr
