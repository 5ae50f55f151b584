// Attention of requests with many rows (prefill chunks) over the paged cache (gfx950).
#include "gnr_iter_attention.h"

namespace gnr {

// A workgroup takes 128 rows (tokens of a chunk times query heads of a kv head), 32 to a wave, against 64 keys at a time, which lie in
// shared memory twice: one block of keys and values is multiplied while the next comes in. The products are transposed as in the kernel for few
// rows: S^T = K Q^T leaves a lane with the scores of one row for keys 8 (i / 4) + 4 h + i % 4 (h: half of the wave), and O^T = V^T P^T numbers its
// keys the same way, so the weights go from one product to the next within registers, and maximum, sum and rescaling of a row stay in its two lanes.
// V^T is read with the transposing LDS load. Bound by the matrix cores and the vector instructions beside them (exponentials, sums, in 8 bits the widening):
// 49 and 47 % of the cycles of a whole prompt, 36 and 41 in 8 bits; then by the LDS reads (a byte of keys or values for every 32 rows). A prompt of 8191 tokens, 32 heads over 8: 548 to 570 us (machines differ), 1.0 PFLOP/s of
// what the mask leaves; 251 tokens after 32517, 28 heads over 4, 8 bits: 161 us with the join, 0.73.
//   Rows of the LDS blocks are 16-byte pieces in an order that depends on the key, so that the 32 keys of a K operand and the four
// keys of a transposing load lie in different banks.
template <int kDim>
__device__ __forceinline__ int piece_of(int key, int piece)
{
  if constexpr (kDim == 64) return piece ^ ((key >> 1 & 1) << 2 | (key >> 2 & 3));
  else return piece ^ ((key & 3) << 2 | (key >> 2 & 3));
}

// Brings blocks of keys, or of values, from the cache into shared memory. A wave's load covers kRows neighbouring keys, within a page unless
// pages are small; 16-bit rows go there directly, 8-bit codes by way of registers, where they are widened.
template <class T, int kDim, bool kFp8, bool kSmallPages>
struct Loader {
  static constexpr int kRowBytes = kDim * 2, kCacheBytes = kFp8 ? kDim : kDim * 2, kSize = kFp8 ? 1 : 2;
  static constexpr int kLanes = kCacheBytes / 16;                        // lanes of a row of the cache, 16 bytes each
  static constexpr int kRows = 64 / kLanes, kStep = kWaves * kRows;      // keys of a wave's load, and those between a thread's
  static constexpr int kMine = ChunkShape::kKeys / kStep;                // loads of a thread for a block
  // Rows of 256 elements in 8 bits are loaded when they are due: there are no registers to hold them meanwhile.
  static constexpr bool kLate = kFp8 && kDim == 256;
  const iter_plane &plane;
  const int wave, in, part;                                              // this thread's key of a wave's load, and its part of the row
  const int widened_at;                                                  // where the first half of a part goes once it is widened (pieces are in the same order every 16 keys)
  const char *rows;                                                      // of the kv head
  const uint8_t *exps;
  u32x4 codes[kFp8 ? kMine : 1];
  uint8_t exp[kFp8 ? kMine : 1];
  int pages_ahead, next_block;                                           // pages of the sixteens of 16 blocks, a lane for each

  __device__ __forceinline__ Loader(const iter_plane &c, int w, int lane) : plane(c), wave(w), in(lane / kLanes), part(lane % kLanes),
                                                                                      widened_at((w * kRows + in) * kRowBytes + piece_of<kDim>(w * kRows + in, 2 * part) * 16)
  {
    static_assert(!kFp8 || kStep % 16 == 0, "pieces in the same order");
  }

  __device__ __forceinline__ void begin(int head)
  {
    rows = static_cast<const char *>(plane.data) + head * plane.head_stride * kSize;
    exps = kFp8 ? plane.exp + head * plane.exp_head_stride : nullptr;
    next_block = 16;
  }

  // bytes of a row that a lane reads: a 16-bit row goes to shared memory as it comes, so its pieces are put in order here
  __device__ __forceinline__ uint32_t offset_in_row(int i) const { return kFp8 ? part * 16 : piece_of<kDim>(i * kStep + wave * kRows + in, part) * 16; }

  __device__ __forceinline__ void fetch(int i, const char *row, const uint8_t *e, char *lds)
  {
    if constexpr (kFp8) {
      codes[i] = *reinterpret_cast<const u32x4 *>(row);
      exp[i] = *e;
    } else {
      load_to_lds(row, lds + (i * kStep + wave * kRows) * kRowBytes);
    }
  }

  // Loads the block of keys from k0 on; what lies beyond `to` is any row of the cache.
  __device__ __forceinline__ void load(const AttentionParams &p, const int32_t *table, int k0, int to, char *lds)
  {
    if constexpr (kSmallPages) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int key = min(k0 + i * kStep + wave * kRows + in, to - 1), place = key & (p.cache.page - 1);
        const int64_t page = usable_page(p, table[key >> p.page_shift]);
        fetch(i, rows + (page * plane.page_stride + place * plane.place_stride) * kSize + offset_in_row(i), kFp8 ? exps + page * plane.exp_page_stride + place * plane.exp_place_stride : nullptr, lds);
      }
    } else {
      if (next_block == 16) {
        const int at = min(k0 + 16 * static_cast<int>(threadIdx.x % 64), to - 1);
        pages_ahead = usable_page(p, table[at >> p.page_shift]);
        next_block = 0;
      }
      // Addresses in scalar registers but for what does not change: the row within a load's and the part of it. A wave issues one instruction
      // at a time, and this runs beside the products.
      constexpr int kPeriod = kFp8 || kStep >= 16 ? 1 : 16 / kStep;       // loads until the order of pieces repeats
      uint32_t offset[kPeriod];
#pragma unroll
      for (int i = 0; i < kPeriod; ++i) offset[i] = in * static_cast<uint32_t>(plane.place_stride * kSize) + offset_in_row(i);
      const uint32_t exp_offset = kFp8 ? in * static_cast<uint32_t>(plane.exp_place_stride) : 0;
      const char *from = nullptr;
      const uint8_t *e = nullptr;
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int row0 = i * kStep + wave * kRows;
        if (i == 0 || p.page_shift < 6) {
          const int64_t page = __builtin_amdgcn_readlane(pages_ahead, 4 * next_block + row0 / 16), place = (k0 + row0) & (p.cache.page - 1);
          from = rows + (page * plane.page_stride + place * plane.place_stride) * kSize;
          if constexpr (kFp8) e = exps + (page * plane.exp_page_stride + place * plane.exp_place_stride);
        } else {
          from += kStep * kSize * plane.place_stride;
          if constexpr (kFp8) e += kStep * plane.exp_place_stride;
        }
        fetch(i, from + offset[i % kPeriod], e + exp_offset, lds);
      }
      ++next_block;
    }
  }

  // Starts on a block of keys.
  __device__ __forceinline__ void bring(const AttentionParams &p, const int32_t *table, int k0, int to, char *lds)
  {
    if constexpr (!kLate) load(p, table, k0, to, lds);
  }

  // The block that was started on is there for the workgroup after the next barrier.
  __device__ __forceinline__ void arrive(const AttentionParams &p, const int32_t *table, int k0, int to, char *lds)
  {
    if constexpr (kFp8) {
      if constexpr (kLate) load(p, table, k0, to, lds);
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const float scale = exponent_scale(exp[i]);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t a = codes[i][2 * half], b = codes[i][2 * half + 1];
          *reinterpret_cast<u32x4 *>(lds + (widened_at ^ 16 * half) + i * kStep * kRowBytes) =
              u32x4{T::template from_e4m3<false>(a, scale), T::template from_e4m3<true>(a, scale), T::template from_e4m3<false>(b, scale), T::template from_e4m3<true>(b, scale)};
        }
      }
    } else {
      wait_for_lds_loads();
    }
  }

  // Rows of the block at k0 that nobody sees (keys outside [from, to)) become zeros. Returns whether any of the others that this thread looks at
  // holds no number.
  static __device__ __forceinline__ int clear(char *lds, int k0, int from, int to)
  {
    bool strange = false;
#pragma unroll
    for (int i = threadIdx.x; i < ChunkShape::kKeys * kRowBytes / 16; i += kThreads) {
      const int key = k0 + i / (kRowBytes / 16);
      u32x4 *at = reinterpret_cast<u32x4 *>(lds) + i;
      if (key < from || key >= to) {
        *at = u32x4{0, 0, 0, 0};
      } else {
        const u32x4 v = *at;
#pragma unroll
        for (int k = 0; k < 4; ++k) strange |= no_number<T>(v[k]);
      }
    }
    return strange;
  }
};

template <class T, int kDim, bool kFp8, bool kSmallPages>
__global__ void __launch_bounds__(kThreads, chunk_blocks(kDim)) gnr_attention_chunk_kernel(const AttentionParams p)
{
  typedef typename T::oct oct;
  constexpr int kKeys = ChunkShape::kKeys, kRowBytes = kDim * 2, kFrags = kDim / 16, kTiles = kDim / 32;
  extern __shared__ int shared[];
  __shared__ __attribute__((aligned(16))) char keys[2 * kKeys * kRowBytes], values[2 * kKeys * kRowBytes];
  const int requests = p.batch.requests, kv_heads = p.cache.kv_heads;
  const ChunkPlan plan{shared, shared + requests + 1, shared + 2 * (requests + 1)};
  share_out_chunks(p, plan, gridDim.x);
  if (blockIdx.x == 0) copy_plan(p, kept_plan(p, ChunkShape::kPlan), shared);
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int n = lane % 32, h = lane / 32;
  Loader<T, kDim, kFp8, kSmallPages> key_loader(p.cache.k, wave, lane), value_loader(p.cache.v, wave, lane);
  const int64_t units = static_cast<int64_t>(plan.start[requests]) * kv_heads;
  // Units are dealt out heaviest first and back and forth, so that every workgroup has as much to do; a head stays with the workgroups of
  // one place among eight, which share a cache.
  const int dealt = gridDim.x % kv_heads == 0 ? kv_heads : 1, back = gridDim.x / dealt - 1 - blockIdx.x / dealt;
  for (int64_t round = 0; round * gridDim.x < units; ++round) {
    const int64_t u = round * gridDim.x + (round % 2 ? back * dealt + blockIdx.x % dealt : blockIdx.x);
    if (u >= units) continue;
    const int unit = static_cast<int>(u / kv_heads), head = static_cast<int>(u % kv_heads);
    const int r = uniform(last_not_above<int>(plan.start, requests, unit));
    uint32_t flags = 0;
    const Request rq = request_of(p, r, &flags);
    const int all_rows = rq.tokens * p.group, tiles = (all_rows + ChunkShape::kRows - 1) / ChunkShape::kRows;
    const int splits = uniform(plan.start[r + 1] - plan.start[r]) / tiles, local = unit - uniform(plan.start[r]);
    const int tile = tile_of_unit(local, tiles, splits), split = local % splits;
    const int32_t *table = p.batch.page_table + r * p.batch.table_stride;
    // the keys that a row sees end before end_of and begin at begin_of
    const auto pos_of = [&](int row) { return rq.base + min(row, all_rows - 1) / p.group; };
    const auto end_of = [&](int row) { return max(0, min(pos_of(row) + 1, rq.end)); };
    const auto begin_of = [&](int row) { return p.window ? max(0, pos_of(row) - p.window + 1) : 0; };
    const int row0 = tile * ChunkShape::kRows, wave_row = row0 + 32 * wave, row = wave_row + n;
    const int tile_from = begin_of(row0), tile_to = end_of(row0 + ChunkShape::kRows - 1);
    const int tile_begin = tile_from & ~63, blocks = max(0, tile_to - tile_begin + kKeys - 1) / kKeys, each = (blocks + splits - 1) / splits;
    const int from = tile_begin + min(blocks, split * each) * kKeys, to = min(tile_to, tile_begin + min(blocks, (split + 1) * each) * kKeys);
    // what all rows of the tile see, and all of this wave's
    const int tile_all_begin = begin_of(row0 + ChunkShape::kRows - 1), tile_all_end = end_of(row0);
    const int wave_all_begin = begin_of(wave_row + 31), wave_all_end = end_of(wave_row);
    const int see_begin = begin_of(row) - 4 * h, see_end = end_of(row) - 4 * h;
    oct q[kFrags];
    {
      const int real = min(row, all_rows - 1);                  // (rows beyond the last repeat it; nobody reads them)
      const uint16_t *at = static_cast<const uint16_t *>(p.q.data) + static_cast<int64_t>(rq.first + real / p.group) * p.q.token_stride +
                           (head * p.group + real % p.group) * p.q.head_stride + 8 * h;
#pragma unroll
      for (int f = 0; f < kFrags; ++f) q[f] = bits<oct>(*reinterpret_cast<const u32x4 *>(at + 16 * f) ^ p.flip);
    }
    f32x16 acc[kTiles];
#pragma unroll
    for (int e = 0; e < kTiles; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[e][i] = 0.0f;
    float top = -FLT_MAX, sum = 0.0f;

    // Operands from shared memory, asked for kAhead products before they are due. What a product and the work beside it need stays together
    // (sched_barrier): left to itself the compiler reads far ahead and runs out of registers.
    constexpr int kAhead = kFp8 ? 3 : 4, kScoreProducts = 2 * kFrags, kValueProducts = 4 * kTiles, kBuffer = kKeys * kRowBytes;
    // The order of pieces is an exclusive or, so the places of a lane's pieces are one number and constants; another bit says which of two
    // buffers. The numbers are made anew for every block (by an empty asm): kept, the places of all pieces would fill thirty registers.
    int key_at = n * kRowBytes + piece_of<kDim>(n, h) * 16, value_at;
    {
      const int group = lane / 16, key = 4 * (group / 2) + lane % 16 / 4;
      value_at = key * kRowBytes + piece_of<kDim>(key, 2 * (group % 2) + lane % 4 / 2) * 16 + lane % 2 * 8;
    }
    const auto key_operand = [&](auto i) GNR_INLINE {           // of the i-th product: keys 32 (i % 2) on, elements 16 (i / 2) on
      return *reinterpret_cast<const u32x4 *>(keys + (key_at ^ 32 * (i / 2)) + 32 * (i % 2) * kRowBytes);
    };
    const auto value_operand = [&](auto i) GNR_INLINE {         // of the i-th product: keys 16 (i / kTiles) on, elements 32 (i % kTiles) on
      const s16x4 a = read_transposed(values + (value_at ^ 64 * (i % kTiles)) + 16 * (i / kTiles) * kRowBytes);
      const s16x4 b = read_transposed(values + (value_at ^ (64 * (i % kTiles) + 32)) + (16 * (i / kTiles) + 8) * kRowBytes);
      return bits<u32x4>(__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    f32x16 low, high;                                           // scores of this lane's row: keys 8 (i / 4) + 4 h + i % 4 of a block's halves
    u32x4 w[4];                                                 // weights of a block
    const auto score = [&]() GNR_INLINE {
      u32x4 operand[kAhead];
      repeat<kAhead>([&](auto i) GNR_INLINE { operand[i] = key_operand(i); });
      low = high = f32x16{0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
      repeat<kScoreProducts>([&](auto i) GNR_INLINE {
        f32x16 &x = i % 2 ? high : low;
        x = T::mfma32(bits<oct>(operand[i % kAhead]), q[i / 2], x);
        if constexpr (i + kAhead < kScoreProducts) operand[i % kAhead] = key_operand(std::integral_constant<int, i + kAhead>{});
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    // Hides what the row does not see. The running maximum moves when a score exceeds it by 2^8: most blocks need no exchange and no
    // rescaling. Returns what to scale the sums before by (1: nothing moved, in the whole wave).
    const auto settle = [&](int k0) GNR_INLINE {
      if (k0 < wave_all_begin || k0 + kKeys > wave_all_end) {
        const int see_from = see_begin - k0, see_to = see_end - k0;
        repeat<16>([&](auto i) GNR_INLINE {
          constexpr int at = i, key = 8 * (i / 4) + i % 4;      // (4 h is in the bounds)
          low[at] = key >= see_from && key < see_to ? low[at] : -INFINITY;
          high[at] = key + 32 >= see_from && key + 32 < see_to ? high[at] : -INFINITY;
        });
      }
      float most = -INFINITY;
      repeat<16>([&](auto i) GNR_INLINE {
        constexpr int at = i;
        most = fmaxf(fmaxf(most, low[at]), high[at]);
      });
      most *= p.scale_log2;
      float keep = 1.0f;
      if (__any(most - top > 8.0f)) {
        most = fmaxf(most, __shfl_xor(most, 32));
        const float next = fmaxf(top, most);
        keep = __builtin_amdgcn_exp2f(top - next);
        top = next;
        sum *= keep;
      }
      return keep;
    };
    // Weights are rounded to 16 bits for their product, relative to the row's largest (their sum is of 32-bit ones). Held as two numbers each, as in the kernel for few
    // rows, they would double these products: whole prompt 558 -> 737 us for an error against 64 bits of 1.6e-3 instead of 2.2e-3, where the result's own rounding is 1.6e-3.
    const auto weigh = [&](auto i) GNR_INLINE {                 // scores 2 i and 2 i + 1
      constexpr int j = 2 * (i % 8), word = i % 4;
      const f32x16 &x = i < 8 ? low : high;
      const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], p.scale_log2, -top)), b = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j + 1], p.scale_log2, -top));
      sum += a;
      sum += b;
      uint32_t both = T::narrow2(a, b);
      asm volatile("" : "+v"(both));                            // (stays where it is: the compiler would move it all behind the products)
      w[i / 4][word] = both;
    };
    // The weights' products with their values and, beside them, the weights of the block after, whose scores are there already. They take the places of
    // weights that have been multiplied, so the sixteen words are spread from the last product of the first four words on: as many by the end of product n as
    // due(n). (A second set of words and its copies: whole prompt 571 -> 568 us, long prompt's chunk 163.5 -> 161.5 without.)
    constexpr auto due = [](int products) {
      const int free = products / kTiles * 4, of = kValueProducts - kTiles + 1, n = products - kTiles + 1, share = n <= 0 ? 0 : (n * 16 + of - 1) / of;
      return share < free ? share : free;
    };
    const auto add = [&](auto also) GNR_INLINE {
      u32x4 operand[kAhead];
      repeat<kAhead>([&](auto i) GNR_INLINE { operand[i] = value_operand(i); });
      repeat<kValueProducts>([&](auto i) GNR_INLINE {
        acc[i % kTiles] = T::mfma32(bits<oct>(operand[i % kAhead]), bits<oct>(w[i / kTiles]), acc[i % kTiles]);
        if constexpr (i + kAhead < kValueProducts) operand[i % kAhead] = value_operand(std::integral_constant<int, i + kAhead>{});
        if constexpr (also) repeat<due(i + 1) - due(i)>([&](auto k) GNR_INLINE { weigh(std::integral_constant<int, due(i) + k>{}); });
        __builtin_amdgcn_sched_barrier(0);
      });
    };

    int again = 0;
    if (from < to) {
      again = missing_page(p, table, max(from, tile_from), to);
      key_loader.begin(head);
      value_loader.begin(head);
      int buffer = 0;                                           // kBuffer for the second one; of the block whose values are due
      key_loader.bring(p, table, from, to, keys);
      key_loader.arrive(p, table, from, to, keys);
      __syncthreads();
      value_loader.bring(p, table, from, to, values);
      if (from + kKeys < to) key_loader.bring(p, table, from + kKeys, to, keys + kBuffer);
      score();
      settle(from);
      repeat<16>([&](auto i) GNR_INLINE { weigh(i); });
      // A weight of zero does not silence a NaN or an infinity: where any stands among values that not every row sees, the rows are
      // computed again by the kernel that joins.
      const auto check_values = [&](int k0) GNR_INLINE {
        if (k0 + kKeys > min(to, tile_all_end) || k0 < tile_all_begin) {
          again |= value_loader.clear(values + buffer, k0, tile_from, to);
          __syncthreads();
        }
      };
      // Keys come in a block ahead of values: the scores of the block after are there when a block's weights meet their values, so that the
      // exponentials run beside these products.
      int k0 = from;
      for (; k0 + kKeys < to; k0 += kKeys) {
        asm volatile("" : "+v"(key_at), "+v"(value_at));
        key_at ^= kBuffer;
        value_loader.arrive(p, table, k0, to, values + buffer);
        key_loader.arrive(p, table, k0 + kKeys, to, keys + (buffer ^ kBuffer));
        __syncthreads();                                        // they are there, and nobody reads the ones before any more
        check_values(k0);
        value_loader.bring(p, table, k0 + kKeys, to, values + (buffer ^ kBuffer));
        if (k0 + 2 * kKeys < to) key_loader.bring(p, table, k0 + 2 * kKeys, to, keys + buffer);
        // (of a SIMD's two waves the one whose products are due goes first: long prompt's chunk 173 -> 164 us, whole prompt 596 -> 590)
        __builtin_amdgcn_s_setprio(1);
        score();
        __builtin_amdgcn_s_setprio(0);
        const float keep = settle(k0 + kKeys);
        __builtin_amdgcn_s_setprio(2);
        add(std::true_type{});
        __builtin_amdgcn_s_setprio(0);
        if (__any(keep != 1.0f)) repeat<kTiles>([&](auto e) GNR_INLINE { acc[e] *= keep; });
        value_at ^= kBuffer;
        buffer ^= kBuffer;
      }
      value_loader.arrive(p, table, k0, to, values + buffer);
      __syncthreads();
      check_values(k0);
      add(std::false_type{});
    }
    again = __syncthreads_or(again);                            // (and nobody reads the last block any more)
    if (threadIdx.x == 0) mark(p, ChunkShape::kPlan, u, again);
    sum += __shfl_xor(sum, 32);
    if (row < all_rows) {
      const int64_t token = rq.first + row / p.group;
      const int64_t part_row = static_cast<int64_t>(plan.part[r]) + static_cast<int64_t>(split) * all_rows + row;
      float *part = part_of(p, ChunkShape::kPlan, part_row * kv_heads + head);
#pragma unroll
      for (int e = 0; e < kTiles; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 o = {acc[e][4 * i], acc[e][4 * i + 1], acc[e][4 * i + 2], acc[e][4 * i + 3]};
          const int d = 32 * e + 8 * i + 4 * h;
          if (splits == 1) write_row<T>(p, token, head * p.group + row % p.group, d, o, sum);
          else *reinterpret_cast<f32x4 *>(part + d) = o;
        }
      if (splits > 1 && h == 0) {
        part[kDim] = top;
        part[kDim + 1] = sum;
      }
    }
  }
}

template <class T, int kDim, bool kFp8>
static int launch(const AttentionParams &p, hipStream_t stream)
{
  const unsigned blocks = static_cast<unsigned>(p.blocks[ChunkShape::kPlan]);
  const size_t lds = plan_bytes(p.batch.requests);
  if (p.cache.page < 16) gnr_attention_chunk_kernel<T, kDim, kFp8, true><<<blocks, kThreads, lds, stream>>>(p);
  else gnr_attention_chunk_kernel<T, kDim, kFp8, false><<<blocks, kThreads, lds, stream>>>(p);
  return iter_hip_ok(hipGetLastError());
}

template <class T, bool kFp8>
static int launch_dim(const AttentionParams &p, hipStream_t stream)
{
  switch (p.cache.head_dim) {
    case 64: return launch<T, 64, kFp8>(p, stream);
    case 128: return launch<T, 128, kFp8>(p, stream);
    default: return launch<T, 256, kFp8>(p, stream);
  }
}

int launch_attention_chunk(const AttentionParams &p, hipStream_t stream)
{
  const bool fp8 = p.cache.type == ITER_FP8;
  if (p.type == ITER_BF16) return fp8 ? launch_dim<Bf16, true>(p, stream) : launch_dim<Bf16, false>(p, stream);
  return fp8 ? launch_dim<Fp16, true>(p, stream) : launch_dim<Fp16, false>(p, stream);
}

}  // namespace gnr
