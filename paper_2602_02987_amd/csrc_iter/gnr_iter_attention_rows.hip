// Attention of requests with few rows (decodes) over the paged cache (gfx950).
#include "gnr_iter_attention.h"

namespace gnr {

// Sixteen rows (the query heads of a kv head, for one token or a few) against a piece of their keys. Transposed products keep
// everything in registers: S^T = K Q^T leaves a lane with four keys of one row, which is what the second product, O^T = V^T P^T, wants
// of its right operand if keys are numbered alike on both sides: lane group g and element j stand for key 16 (j / 4) + 4 g + j % 4 of 32 (in 4 bits 16 (j / 4) + 4 (j % 4) + g). A lane reads
// head_dim / 16 neighbouring elements of eight keys' values and swaps halves of registers to have eight keys of one element; no
// shared memory is used, every byte of the cache goes from memory to the registers of the wave that multiplies it. Each wave takes every
// fourth block of 32 keys with a running maximum and sum of its own; the waves are joined at the end.
//   Bound by the memory: sixteen rows of products for a key are far below the matrix rate. 127 decodes of 435000 keys beside a chunk (1.8 GB, 16 bits): 374 us in all,
// 4.8 TB/s; 32 decodes of 100000 keys in 8 bits: 46 us, 4.5 TB/s. A single decode of 1093 keys takes 8 us: the chain from bounds to page table to keys to values.
//   In 4 bits codes go through the conversion instructions as well: the scaled matrix instructions would take them as they are, but the queries and weights would have to be codes of 8 bits or fewer
// there too. 127 decodes of 453000 keys (0.49 GB): 106 to 109 us, 4.5 to 4.7 TB/s, vector instructions 53 % of the cycles. A workgroup has 2.3 tiles of
// these on the average, and between two of them nothing on its way. Three workgroups a compute unit instead of two: 132 -> 125 us with the join (before tiles counted for more than their keys, see RowsPlan); two blocks of keys on
// their way at once change nothing.
// Three decodes of 131000 keys (0.21 GB): 49 us, 4.4 TB/s.
template <class T, int kDim, int kBits, bool kSmallPages>
struct Tile {
  static constexpr int kVec = kDim / 16;                        // elements of a value row a lane reads
  static constexpr int kFrags = kDim / 32;                      // matrix products over the elements of a key
  static constexpr int kKeyWords = kDim * kBits / 128;          // words of a key a lane reads
  static constexpr int kValWords = kVec * kBits < 32 ? 1 : kVec * kBits / 32;
  static constexpr int kPart = kKeyWords < 4 ? 4 * kKeyWords : 16;   // bytes of a key a lane reads at once
  static constexpr int kKeyExps = kBits == 4 && kDim == 256 ? 2 : 1, kExps = exps_of_row(kBits, kDim);
  static constexpr bool kScaled = kBits < 16;
  // Of 4 bits a load of values takes the rows of neighbouring keys, half a cache line each: element i of lane group g is key 4 i + g of sixteen then instead of 4 g + i.
  static constexpr bool kSpread = kBits == 4;
  typedef typename T::oct oct;

  const int n, g;                                               // n: row, and key or element of the operands; g: group of 16 lanes
  oct q[kFrags];
  f32x4 acc[kVec];
  float top, sum;                                               // of row n; `sum` of this lane's keys only
  uint32_t kw[2][kKeyWords], vw[8][kValWords];
  uint8_t ks[2][kKeyExps], vs[8];
  // rows of this kv head
  const char *keys, *values;
  const uint8_t *key_exps, *value_exps;

  __device__ __forceinline__ Tile(int lane) : n(lane % 16), g(lane / 16) {}

  // elements of a row that fragment f of a lane holds, and the first one that it multiplies with values; caches of fewer bits are read more elements at a time
  __device__ __forceinline__ int element(int f) const
  {
    constexpr int kAtOnce = 8 * kPart / kBits, kFs = kAtOnce / 8;
    return 4 * kAtOnce * (f / kFs) + kAtOnce * g + 8 * (f % kFs);
  }
  __device__ __forceinline__ int key_at(int i) const { return kSpread ? 4 * i : i; }       // and
  __device__ __forceinline__ int first_key() const { return kSpread ? g : 4 * g; }          // their sum: the key, of sixteen, of the lane's score i
  __device__ __forceinline__ int operand_key() const { return kSpread ? 4 * (n % 4) + n / 4 : n; }
  __device__ __forceinline__ int key_exp() const { return kBits == 4 ? kDim == 64 ? g / 2 : g : 0; }
  __device__ __forceinline__ int value_exp() const { return kBits == 4 ? kVec * n / 32 : 0; }

  __device__ __forceinline__ void begin(const AttentionParams &p, int head, const uint16_t *row)
  {
    keys = static_cast<const char *>(p.cache.k.data) + bytes_of<kBits>(head * p.cache.k.head_stride);
    values = static_cast<const char *>(p.cache.v.data) + bytes_of<kBits>(head * p.cache.v.head_stride);
    key_exps = value_exps = nullptr;
    if constexpr (kScaled) {
      key_exps = p.cache.k.exp + head * p.cache.k.exp_head_stride;
      value_exps = p.cache.v.exp + head * p.cache.v.exp_head_stride;
    }
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {
      u32x4 w = {0, 0, 0, 0};
      if (row) w = *reinterpret_cast<const u32x4 *>(row + element(f)) ^ p.flip;
      q[f] = bits<oct>(w);
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) acc[e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    top = -FLT_MAX;
    sum = 0.0f;
  }

  // An offset that stays one of 32 bits, beside an address in scalar registers: the compiler would keep each as a 64-bit number of its own (160 -> 142 registers in 4 bits).
  static __device__ __forceinline__ uint32_t here(uint32_t offset)
  {
    asm volatile("" : "+v"(offset));
    return offset;
  }

  template <int kWords, bool kHalf = false>
  static __device__ __forceinline__ void load_words(const void *at, uint32_t *w)
  {
    if constexpr (kHalf) w[0] = *static_cast<const uint16_t *>(at);
    else if constexpr (kWords == 1) w[0] = *static_cast<const uint32_t *>(at);
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

  // The 32 keys from k0 on. pages: of the first and the second sixteen (pages of fewer than 16 tokens are looked up key by key). Keys
  // from `stop` on may be any rows of the cache.
  __device__ __forceinline__ void load_keys(const AttentionParams &p, int k0, const int *pages, const int32_t *table, int stop)
  {
    const iter_plane &c = p.cache.k;
    if constexpr (kSmallPages) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int key = min(k0 + 16 * t + operand_key(), stop - 1), place = key & (p.cache.page - 1);
        const int64_t page = usable_page(p, table[key >> p.page_shift]);
        load_key(t, keys + bytes_of<kBits>(page * c.page_stride + place * c.place_stride) + kPart * g, key_exps + (kScaled ? page * c.exp_page_stride + place * c.exp_place_stride + key_exp() : 0));
      }
    } else {
      // (a wave's address in scalar registers and a lane's offset of 32 bits, which is always the same)
      const uint32_t lane_row = operand_key() * static_cast<uint32_t>(bytes_of<kBits>(c.place_stride)) + kPart * g, lane_exp = operand_key() * static_cast<uint32_t>(c.exp_place_stride) + key_exp();
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int64_t page = pages[t], place = (k0 + 16 * t) & (p.cache.page - 1);
        load_key(t, keys + bytes_of<kBits>(page * c.page_stride + place * c.place_stride) + here(lane_row), key_exps + (kScaled ? page * c.exp_page_stride + place * c.exp_place_stride + here(lane_exp) : 0));
      }
    }
  }

  __device__ __forceinline__ void load_key(int t, const char *row, const uint8_t *exp)
  {
#pragma unroll
    for (int i = 0; i < 4 * kKeyWords / kPart; ++i) load_words<kPart / 4>(row + 64 * i, &kw[t][4 * i]);
    if constexpr (kScaled)
#pragma unroll
      for (int i = 0; i < kKeyExps; ++i) ks[t][i] = exp[4 * i];
  }

  __device__ __forceinline__ void load_values(const AttentionParams &p, int k0, const int *pages, const int32_t *table, int stop)
  {
    const iter_plane &c = p.cache.v;
    if constexpr (kSmallPages) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int key = min(k0 + 16 * (j / 4) + key_at(j % 4) + first_key(), stop - 1), place = key & (p.cache.page - 1);
        const int64_t page = usable_page(p, table[key >> p.page_shift]);
        load_words<kValWords, kVec * kBits < 32>(values + bytes_of<kBits>(page * c.page_stride + place * c.place_stride) + bytes_of<kBits>(kVec) * n, vw[j]);
        if constexpr (kScaled) vs[j] = value_exps[page * c.exp_page_stride + place * c.exp_place_stride + value_exp()];
      }
    } else {
      // (the sixteen's address in scalar registers; a lane's rows of it are four offsets of 32 bits)
      const uint32_t step = static_cast<uint32_t>(bytes_of<kBits>(c.place_stride)), exp_step = static_cast<uint32_t>(c.exp_place_stride);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int64_t page = pages[t], place = (k0 + 16 * t) & (p.cache.page - 1);
        const char *const row = values + bytes_of<kBits>(page * c.page_stride + place * c.place_stride);
        const uint8_t *const exp = value_exps + (kScaled ? page * c.exp_page_stride + place * c.exp_place_stride : 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          load_words<kValWords, kVec * kBits < 32>(row + here((key_at(j) + first_key()) * step + bytes_of<kBits>(kVec) * n), vw[4 * t + j]);
          if constexpr (kScaled) vs[4 * t + j] = exp[here((key_at(j) + first_key()) * exp_step + value_exp())];
        }
      }
    }
  }

  // scores of the 32 keys: s[t][i] belongs to key 16 t + key_at(i) + first_key()
  __device__ __forceinline__ void scores(f32x4 *s) const
  {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        u32x4 w;
        if constexpr (kBits == 4) {
          const float scale = exponent_scale(ks[t][f / 4 % kKeyExps]);
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = pair_of_e2m1<T>(kw[t][f], i, scale);
        } else if constexpr (kBits == 8) {
          const float scale = exponent_scale(ks[t][0]);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t c = kw[t][4 * (f / 2) + 2 * (f % 2) + i];
            w[2 * i] = T::template from_e4m3<false>(c, scale);
            w[2 * i + 1] = T::template from_e4m3<true>(c, scale);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = kw[t][4 * f + i];
        }
        s[t] = T::mfma16(bits<oct>(w), q[f], s[t]);
      }
    }
  }

  // Weights of the 32 keys, each as two 16-bit numbers (words 4 on hold the lower ones, see split2), which are multiplied one after the other: the matrix cores have little
  // to do here, so that the result's own rounding is all that shows (relative error against 64 bits in bfloat16 2.2e-3 -> 1.6e-3) costs 0.1 us of a decode, 0.4 of 32 decodes
  // over 8 bits (60.2) and 1.3 of a mixed iteration (374). The running maximum moves when a score exceeds it by 2^8, so that most blocks need no exchange between
  // lanes and no rescaling (weights stay below 2^8, sums and products lose nothing).
  __device__ __forceinline__ void weigh(f32x4 *s, uint32_t *w, float scale)
  {
    float high = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) high = fmaxf(high, s[t][i]);
    high *= scale;
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
        s[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], scale, T::kSplitShift - top));
        sum += s[t][i];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) T::split2(s[t][2 * i], s[t][2 * i + 1], w[2 * t + i], w[4 + 2 * t + i]);
    }
  }

  // Values of keys outside [start, stop) are nobody's: zeros in their place. Returns whether any of the others is no number.
  __device__ __forceinline__ bool clear_values(int k0, int start, int stop)
  {
    bool strange = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int key = k0 + 16 * (j / 4) + key_at(j % 4) + first_key();
      const bool in = key >= start && key < stop;
#pragma unroll
      for (int i = 0; i < kValWords; ++i) vw[j][i] = in ? vw[j][i] : 0;
      if constexpr (kScaled) vs[j] = in ? vs[j] : 127;          // (zeros times a factor that is no number are none)
#pragma unroll
      for (int i = 0; i < kVec / 2; ++i) strange |= no_number<T>(value_word(j, i));
    }
    return strange;
  }

  // word i (two elements) of key j's values
  __device__ __forceinline__ uint32_t value_word(int j, int i) const
  {
    if constexpr (kBits == 4) return pair_of_e2m1<T>(vw[j][i / 4], i % 4, exponent_scale(vs[j]));
    else if constexpr (kBits == 8) return i % 2 ? T::template from_e4m3<true>(vw[j][i / 2], exponent_scale(vs[j])) : T::template from_e4m3<false>(vw[j][i / 2], exponent_scale(vs[j]));
    else return vw[j][i];
  }

  __device__ __forceinline__ void add_values(const uint32_t *w)
  {
    const oct upper = bits<oct>(u32x4{w[0], w[1], w[2], w[3]}), lower = bits<oct>(u32x4{w[4], w[5], w[6], w[7]});
#pragma unroll
    for (int e = 0; e < kVec; e += 2) {
      uint32_t v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = value_word(j, e / 2);
      u32x4 a, b;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x05040100u);
        b[i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x07060302u);
      }
      acc[e] = T::mfma16(bits<oct>(a), upper, acc[e]);
      acc[e + 1] = T::mfma16(bits<oct>(b), upper, acc[e + 1]);
      acc[e] = T::mfma16(bits<oct>(a), lower, acc[e]);
      acc[e + 1] = T::mfma16(bits<oct>(b), lower, acc[e + 1]);
    }
  }
};

template <class T, int kDim, int kBits, bool kSmallPages>
__global__ void __launch_bounds__(kThreads, rows_blocks(kDim, kBits)) gnr_attention_rows_kernel(const AttentionParams p)
{
  typedef Tile<T, kDim, kBits, kSmallPages> Rows;
  extern __shared__ int64_t shared[];
  __shared__ float tops[kWaves][16], sums[kWaves][16];
  __shared__ float outs[kWaves][16][kDim + 4];
  const int requests = p.batch.requests, kv_heads = p.cache.kv_heads;
  const RowsPlan plan = share_out_rows(p, shared, gridDim.x);
  if (blockIdx.x == 0) copy_plan(p, kept_plan(p, RowsShape::kPlan), reinterpret_cast<const int *>(shared));
  CutTile cut_tile{};
  if (static_cast<int>(blockIdx.x) >= plan.blocks) {
    if (threadIdx.x == 0) cut_tiles(p)[blockIdx.x] = cut_tile;
    return;
  }
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Rows rows(lane);
  const int64_t cut = uniform(plan.cut(blockIdx.x + 1));
  for (int64_t x = uniform(plan.cut(blockIdx.x)); x < cut;) {
    const int r = uniform(last_not_above<int64_t>(plan.start, requests, x / kv_heads));
    const Request rq = plan.request(p, r);
    int all_rows, blocks;
    tiles_of<RowsShape>(p, rq, all_rows, blocks);
    blocks += plan.extra;
    // the (tile, head) that x is in, its blocks of keys from `first` to `last`, and whether these are all
    const int64_t local = x - uniform(plan.start[r]) * kv_heads;
    const int nth = uniform(static_cast<int>(local / blocks)), tile = uniform(nth / kv_heads), head = nth - tile * kv_heads;
    const int first = uniform(static_cast<int>(local - static_cast<int64_t>(nth) * blocks));
    const int last = uniform(static_cast<int>(min(static_cast<int64_t>(blocks), first + (cut - x))));
    const bool whole = first == 0 && last == blocks;
    x += last - first;
    // what the tile's tokens see: the last one's end, and what all of them see
    const int first_pos = uniform(rq.base + tile * 16 / p.group), last_pos = uniform(rq.base + min(rq.tokens - 1, (tile * 16 + 15) / p.group));
    const int all_end = min(first_pos + 1, rq.end), all_begin = p.window ? last_pos - p.window + 1 : 0, any_begin = p.window ? first_pos - p.window + 1 : 0;
    const int from = rq.begin + max(0, first - plan.extra) * RowsShape::kKeys, stop = min(min(rq.end, last_pos + 1), rq.begin + max(0, last - plan.extra) * RowsShape::kKeys);
    const int32_t *table = p.batch.page_table + r * p.batch.table_stride;
    const int row = min(tile * 16 + rows.n, all_rows - 1), pos = rq.base + row / p.group;   // (rows beyond the last repeat it; nobody reads them)
    rows.begin(p, head, static_cast<const uint16_t *>(p.q.data) + static_cast<int64_t>(rq.first + row / p.group) * p.q.token_stride + (head * p.group + row % p.group) * p.q.head_stride);
    int again = 0;
    if (from < stop) {
      again = missing_page(p, table, max(from, any_begin), stop);
      // the pages of 32 blocks of this wave at a time: lane 2 i + t holds the t-th sixteen's of the i-th
      int pages_ahead = 0, step = 0, pages[2] = {0, 0};
      const auto look_up = [&](int k0) {
        const int key = min(k0 + (lane / 2) * RowsShape::kKeys + 16 * (lane % 2), stop - 1);
        pages_ahead = usable_page(p, table[key >> p.page_shift]);
      };
      const auto next_pages = [&](int k0) {
        if constexpr (!kSmallPages) {
          if (step == 32) {
            look_up(k0);
            step = 0;
          }
          pages[0] = __builtin_amdgcn_readlane(pages_ahead, 2 * step);
          pages[1] = __builtin_amdgcn_readlane(pages_ahead, 2 * step + 1);
          ++step;
        }
      };
      int k0 = from + 32 * wave;
      if (k0 < stop) {
        step = 32;
        next_pages(k0);
        rows.load_keys(p, k0, pages, table, stop);
        rows.load_values(p, k0, pages, table, stop);
        while (true) {
          const int k1 = k0 + RowsShape::kKeys;
          const bool more = k1 < stop, ragged = k0 < all_begin || k0 + 32 > min(all_end, stop);
          f32x4 s[2];
          rows.scores(s);
          if (more) {
            next_pages(k1);
            rows.load_keys(p, k1, pages, table, stop);
          }
          if (ragged) {
            const int see_end = min(pos + 1, stop) - k0 - rows.first_key(), see_begin = (p.window ? pos - p.window + 1 : 0) - k0 - rows.first_key();
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i) s[t][i] = 16 * t + rows.key_at(i) >= see_begin && 16 * t + rows.key_at(i) < see_end ? s[t][i] : -INFINITY;
            // A weight of zero does not silence a NaN or an infinity: where any stands among values that not every row sees, the
            // rows are computed again by the kernel that joins.
            again |= rows.clear_values(k0, any_begin, stop) && first_pos != last_pos;
          }
          uint32_t w[8];
          rows.weigh(s, w, p.scale_log2);
          rows.add_values(w);
          if (!more) break;
          rows.load_values(p, k1, pages, table, stop);
          k0 = k1;
        }
      }
    }
    // join the waves
    float sum = rows.sum;
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    again = __syncthreads_or(again);                             // (the unit before has been read)
    if (first == 0 && threadIdx.x == 0) mark(p, RowsShape::kPlan, (static_cast<int64_t>(plan.tiles[r]) + tile) * kv_heads + head, whole ? again : 0);
    if (first == 0 && !whole) {
      cut_tile.rows = min(16, all_rows - tile * 16);
      cut_tile.tile = tile;
      cut_tile.head = head;
      cut_tile.request = r;
      cut_tile.token = rq.first;
      cut_tile.last = plan.block_of(x - last + blocks - 1);
      cut_tile.mark[1] = again;
    } else if (first != 0) {
      // (64-bit divisions, which a single decode would wait 0.3 us for: not where the tile cannot have so many parts)
      if (static_cast<int64_t>(blocks) * plan.blocks > (kFewParts - 2) * plan.total) {
        const int from_block = plan.block_of(x - last);
        if (plan.block_of(x - last + blocks - 1) - from_block >= kFewParts) cut_tile.from = from_block;
      }
      cut_tile.mark[0] = again;
    }
    if (rows.g == 0) {
      tops[wave][rows.n] = rows.top;
      sums[wave][rows.n] = sum;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < Rows::kVec; ++e) outs[wave][rows.n][Rows::kVec * (4 * rows.g + i) + e] = rows.acc[e][i];
    __syncthreads();
    const int real_rows = min(16, all_rows - tile * 16);
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
      const int at = tile * 16 + y;
      if (whole) {
        write_row<T>(p, rq.first + at / p.group, head * p.group + at % p.group, d, o, all);
      } else {
        float *to_part = part_of(p, RowsShape::kPlan, (2 * static_cast<int64_t>(blockIdx.x) + (first == 0)) * RowsShape::kRows + y);
        *reinterpret_cast<f32x4 *>(to_part + d) = o;
        if (d == 0) {
          to_part[kDim] = most;
          to_part[kDim + 1] = all;
        }
      }
    }
  }
  if (threadIdx.x == 0) cut_tiles(p)[blockIdx.x] = cut_tile;
}

template <class T, int kDim, int kBits>
static int launch(const AttentionParams &p, hipStream_t stream)
{
  const unsigned blocks = static_cast<unsigned>(p.blocks[RowsShape::kPlan]);
  const size_t lds = rows_plan_bytes(p.batch.requests);
  if (p.cache.page < 16) gnr_attention_rows_kernel<T, kDim, kBits, true><<<blocks, kThreads, lds, stream>>>(p);
  else gnr_attention_rows_kernel<T, kDim, kBits, false><<<blocks, kThreads, lds, stream>>>(p);
  return iter_hip_ok(hipGetLastError());
}

template <class T, int kBits>
static int launch_dim(const AttentionParams &p, hipStream_t stream)
{
  switch (p.cache.head_dim) {
    case 64: return launch<T, 64, kBits>(p, stream);
    case 128: return launch<T, 128, kBits>(p, stream);
    default: return launch<T, 256, kBits>(p, stream);
  }
}

template <class T>
static int launch_bits(const AttentionParams &p, hipStream_t stream)
{
  switch (p.cache.type) {
    case ITER_FP4: return launch_dim<T, 4>(p, stream);
    case ITER_FP8: return launch_dim<T, 8>(p, stream);
    default: return launch_dim<T, 16>(p, stream);
  }
}

int launch_attention_rows(const AttentionParams &p, hipStream_t stream) { return p.type == ITER_BF16 ? launch_bits<Bf16>(p, stream) : launch_bits<Fp16>(p, stream); }

}  // namespace gnr
