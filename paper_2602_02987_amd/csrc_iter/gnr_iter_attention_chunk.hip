// Attention of requests with many rows (prefill chunks) over the paged cache (gfx950).
#include "gnr_iter_attention.h"

namespace gnr {

// A workgroup takes 128 rows (tokens of a chunk times query heads of a kv head), 32 to a wave, against 64 keys at a time, which lie in
// shared memory twice: one block of keys and values is multiplied while the next comes in. The products are transposed as in the kernel for few
// rows: S^T = K Q^T leaves a lane with the scores of one row for keys 8 (i / 4) + 4 h + i % 4 (h: half of the wave), and O^T = V^T P^T numbers its
// keys the same way, so the weights go from one product to the next within registers, and maximum, sum and rescaling of a row stay in its two lanes.
// V^T is read with the transposing LDS load. Bound by the matrix cores, the exponentials beside them and the LDS reads (a byte of keys
// or values for every 32 rows).
//   Rows of the LDS blocks are 16-byte pieces in an order that depends on the key, so that the 32 keys of a K operand and the four
// keys of a transposing load lie in different banks.
template <int kDim>
__device__ __forceinline__ int piece_of(int key, int piece)
{
  if constexpr (kDim == 64) return piece ^ ((key >> 1 & 1) << 2 | (key >> 2 & 3));
  else return piece ^ ((key & 3) << 2 | (key >> 2 & 3));
}

// Brings blocks of keys and values from the cache into shared memory. A wave's load covers kRows neighbouring keys, within a page unless pages are
// small; 16-bit rows go there directly, 8-bit codes by way of registers, where they are widened.
template <class T, int kDim, bool kFp8, bool kSmallPages>
struct Loader {
  static constexpr int kPieces = kDim / 8, kRowBytes = kDim * 2;
  static constexpr int kMine = ChunkShape::kKeys * kPieces / kThreads;   // pieces of a block that a thread brings in
  static constexpr int kRows = 64 / kPieces;                             // keys of a wave's load; kWaves * kRows lie between a thread's
  static constexpr int kSize = kFp8 ? 1 : 2;
  const int wave, key, piece;                                            // this thread's first key of a block, and its place in LDS rows
  const char *keys, *values;                                             // rows of the kv head
  const uint8_t *key_exps, *value_exps;
  u32x2 kr[kFp8 ? kMine : 1], vr[kFp8 ? kMine : 1];
  uint8_t ks[kFp8 ? kMine : 1], vs[kFp8 ? kMine : 1];
  int pages_ahead, next_block;                                           // pages of the sixteens of 16 blocks, a lane for each

  __device__ __forceinline__ Loader(int wave_, int lane) : wave(wave_), key(wave_ * kRows + lane / kPieces), piece(lane % kPieces) {}

  __device__ __forceinline__ void begin(const AttentionParams &p, int head)
  {
    keys = static_cast<const char *>(p.cache.k.data) + head * p.cache.k.head_stride * kSize;
    values = static_cast<const char *>(p.cache.v.data) + head * p.cache.v.head_stride * kSize;
    if constexpr (kFp8) {
      key_exps = p.cache.k.exp + head * p.cache.k.exp_head_stride;
      value_exps = p.cache.v.exp + head * p.cache.v.exp_head_stride;
    }
    next_block = 16;
  }

  // Rows of 256 elements in 8 bits are loaded when they are due: there are no registers to hold them meanwhile.
  static constexpr bool kLate = kFp8 && kDim == 256;

  // A thread's i-th piece of the block at k0: where it lies in the cache. What lies beyond `to` is any row.
  __device__ __forceinline__ void locate(const AttentionParams &p, const int32_t *table, int k0, int to, int i, int &page, int &place) const
  {
    const int row0 = (i * kWaves + wave) * kRows, in = key - wave * kRows;   // of the block
    if constexpr (kSmallPages) {
      const int at = min(k0 + row0 + in, to - 1);
      page = usable_page(p, table[at >> p.page_shift]);
      place = at & (p.cache.page - 1);
    } else {
      page = __builtin_amdgcn_readlane(pages_ahead, 4 * next_block + row0 / 16);
      place = ((k0 + row0) & (p.cache.page - 1)) + in;
    }
  }

  __device__ __forceinline__ void look_up(const AttentionParams &p, const int32_t *table, int k0, int to)
  {
    if constexpr (!kSmallPages) {
      if (next_block == 16) {
        const int at = min(k0 + 16 * static_cast<int>(threadIdx.x % 64), to - 1);
        pages_ahead = usable_page(p, table[at >> p.page_shift]);
        next_block = 0;
      }
    }
  }

  __device__ __forceinline__ void load_codes(const AttentionParams &p, int page, int place, u32x2 &k, u32x2 &v, uint8_t &k_exp, uint8_t &v_exp) const
  {
    k = *reinterpret_cast<const u32x2 *>(keys + page * p.cache.k.page_stride + place * p.cache.k.place_stride + piece * 8);
    v = *reinterpret_cast<const u32x2 *>(values + page * p.cache.v.page_stride + place * p.cache.v.place_stride + piece * 8);
    k_exp = key_exps[page * p.cache.k.exp_page_stride + place * p.cache.k.exp_place_stride];
    v_exp = value_exps[page * p.cache.v.exp_page_stride + place * p.cache.v.exp_place_stride];
  }

  // Starts on the block of keys from k0 on.
  __device__ __forceinline__ void bring(const AttentionParams &p, const int32_t *table, int k0, int to, char *key_rows, char *value_rows)
  {
    if constexpr (kLate) return;
    look_up(p, table, k0, to);
    if constexpr (!kFp8 && !kSmallPages) {
      // Addresses in scalar registers but for what does not change: the row within a load's and the piece. A wave issues one instruction
      // at a time, and this runs beside the products.
      constexpr int kPeriod = 16 / (kWaves * kRows) > 1 ? 16 / (kWaves * kRows) : 1;   // loads until the order of pieces repeats
      const int in = key - wave * kRows;
      uint32_t k_off[kPeriod], v_off[kPeriod];
#pragma unroll
      for (int i = 0; i < kPeriod; ++i) {
        const int piece16 = piece_of<kDim>(i * kWaves * kRows + key, piece) * 16;
        k_off[i] = in * static_cast<uint32_t>(p.cache.k.place_stride * 2) + piece16;
        v_off[i] = in * static_cast<uint32_t>(p.cache.v.place_stride * 2) + piece16;
      }
      const char *k = nullptr, *v = nullptr;
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int row0 = (i * kWaves + wave) * kRows;
        if (i == 0 || p.page_shift < 6) {
          const int64_t page = __builtin_amdgcn_readlane(pages_ahead, 4 * next_block + row0 / 16), place = (k0 + row0) & (p.cache.page - 1);
          k = keys + (page * p.cache.k.page_stride + place * p.cache.k.place_stride) * 2;
          v = values + (page * p.cache.v.page_stride + place * p.cache.v.place_stride) * 2;
        } else {
          k += kWaves * kRows * 2 * p.cache.k.place_stride;
          v += kWaves * kRows * 2 * p.cache.v.place_stride;
        }
        load_to_lds(k + k_off[i % kPeriod], key_rows + row0 * kRowBytes);
        load_to_lds(v + v_off[i % kPeriod], value_rows + row0 * kRowBytes);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        int page, place;
        locate(p, table, k0, to, i, page, place);
        if constexpr (kFp8) {
          load_codes(p, page, place, kr[i], vr[i], ks[i], vs[i]);
        } else {
          const int row0 = (i * kWaves + wave) * kRows, from = piece_of<kDim>(row0 + key - wave * kRows, piece) * 16;
          load_to_lds(keys + page * p.cache.k.page_stride * 2 + place * p.cache.k.place_stride * 2 + from, key_rows + row0 * kRowBytes);
          load_to_lds(values + page * p.cache.v.page_stride * 2 + place * p.cache.v.place_stride * 2 + from, value_rows + row0 * kRowBytes);
        }
      }
    }
    ++next_block;
  }

  // The block that was started on is there for the workgroup after the next barrier.
  __device__ __forceinline__ void arrive(const AttentionParams &p, const int32_t *table, int k0, int to, char *key_rows, char *value_rows)
  {
    if constexpr (kFp8) {
      if constexpr (kLate) look_up(p, table, k0, to);
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int row = i * kWaves * kRows + key, at = row * kRowBytes + piece_of<kDim>(row, piece) * 16;
        if constexpr (kLate) {
          int page, place;
          locate(p, table, k0, to, i, page, place);
          load_codes(p, page, place, kr[i], vr[i], ks[i], vs[i]);
        }
        *reinterpret_cast<u32x4 *>(key_rows + at) = widen(kr[i], exponent_scale(ks[i]));
        *reinterpret_cast<u32x4 *>(value_rows + at) = widen(vr[i], exponent_scale(vs[i]));
      }
      if constexpr (kLate) ++next_block;
    } else {
      wait_for_lds_loads();
    }
  }

  static __device__ __forceinline__ u32x4 widen(u32x2 x, float scale)
  {
    return u32x4{T::template from_e4m3<false>(x[0], scale), T::template from_e4m3<true>(x[0], scale),
                 T::template from_e4m3<false>(x[1], scale), T::template from_e4m3<true>(x[1], scale)};
  }

  // Values of the block at k0 that nobody sees (keys outside [from, to)) become zeros. Returns whether any of the others that this thread looks at is no number.
  __device__ __forceinline__ int clear_values(char *value_rows, int k0, int from, int to) const
  {
    bool strange = false;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int row = i * kWaves * kRows + key;
      u32x4 *at = reinterpret_cast<u32x4 *>(value_rows + row * kRowBytes + piece * 16);
      if (k0 + row < from || k0 + row >= to) {
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
__global__ void __launch_bounds__(kThreads, kDim == 256 ? 1 : 2) gnr_attention_chunk_kernel(const AttentionParams p)
{
  typedef typename T::oct oct;
  constexpr int kKeys = ChunkShape::kKeys, kRowBytes = kDim * 2, kFrags = kDim / 16, kTiles = kDim / 32;
  extern __shared__ int shared[];
  __shared__ __attribute__((aligned(16))) char keys[2][kKeys * kRowBytes], values[2][kKeys * kRowBytes];
  const int requests = p.batch.requests, kv_heads = p.cache.kv_heads;
  const Plan plan{shared, shared + requests + 1, shared + 2 * (requests + 1)};
  share_out<ChunkShape>(p, plan, gridDim.x);
  if (blockIdx.x == 0) keep_plan(p, plan, ChunkShape::kPlan);
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int n = lane % 32, h = lane / 32;
  Loader<T, kDim, kFp8, kSmallPages> loader(wave, lane);
  const int64_t units = static_cast<int64_t>(plan.start[requests]) * kv_heads;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int unit = static_cast<int>(u / kv_heads), head = static_cast<int>(u % kv_heads);
    const int r = __builtin_amdgcn_readfirstlane(last_not_above(plan.start, requests, unit));
    uint32_t flags = 0;
    const Request rq = request_of(p, r, &flags);
    const int all_rows = rq.tokens * p.group, tiles = (all_rows + ChunkShape::kRows - 1) / ChunkShape::kRows;
    const int splits = __builtin_amdgcn_readfirstlane(plan.start[r + 1] - plan.start[r]) / tiles, local = unit - __builtin_amdgcn_readfirstlane(plan.start[r]);
    const int tile = tile_of_unit<ChunkShape>(local, tiles, splits), split = local % splits;
    const int32_t *table = p.batch.page_table + r * p.batch.table_stride;
    // the keys that a row sees end before end_of and begin at begin_of
    const auto pos_of = [&](int row) { return rq.base + min(row, all_rows - 1) / p.group; };
    const auto end_of = [&](int row) { return max(0, min(pos_of(row) + 1, rq.end)); };
    const auto begin_of = [&](int row) { return p.window ? max(0, pos_of(row) - p.window + 1) : 0; };
    const int row0 = tile * ChunkShape::kRows, wave_row = row0 + 32 * wave, row = wave_row + n;
    const int tile_from = begin_of(row0), tile_to = end_of(row0 + ChunkShape::kRows - 1);
    const int tile_begin = tile_from & ~63, blocks = max(0, tile_to - tile_begin + kKeys - 1) / kKeys, each = (blocks + splits - 1) / splits;
    const int from = tile_begin + min(blocks, split * each) * kKeys, to = min(tile_to, tile_begin + min(blocks, (split + 1) * each) * kKeys);
    // what all rows of the tile see, of this wave's, and what any of this wave's sees
    const int tile_all_begin = begin_of(row0 + ChunkShape::kRows - 1), tile_all_end = end_of(row0);
    const int wave_all_begin = begin_of(wave_row + 31), wave_all_end = end_of(wave_row), wave_begin = begin_of(wave_row), wave_end = end_of(wave_row + 31);
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

    const auto multiply = [&](int k0, const char *key_rows, const char *value_rows) {
      if (k0 >= wave_end || k0 + kKeys <= wave_begin) return;
      f32x16 s[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kt][i] = 0.0f;
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
          const int key = 32 * kt + n;
          const u32x4 a = *reinterpret_cast<const u32x4 *>(key_rows + key * kRowBytes + piece_of<kDim>(key, 2 * f + h) * 16);
          s[kt] = T::mfma32(bits<oct>(a), q[f], s[kt]);
        }
      }
      if (k0 < wave_all_begin || k0 + kKeys > wave_all_end) {
        const int see_from = see_begin - k0, see_to = see_end - k0;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = 32 * kt + 8 * (i / 4) + i % 4;      // (4 h is in the bounds)
            s[kt][i] = key >= see_from && key < see_to ? s[kt][i] : -INFINITY;
          }
      }
      float high = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) high = fmaxf(high, s[kt][i]);
      // the running maximum moves when a score exceeds it by 2^8: most blocks need no exchange and no rescaling
      high *= p.scale_log2;
      if (__any(high - top > 8.0f)) {
        high = fmaxf(high, __shfl_xor(high, 32));
        const float next = fmaxf(top, high), keep = __builtin_amdgcn_exp2f(top - next);
        top = next;
        sum *= keep;
#pragma unroll
        for (int e = 0; e < kTiles; ++e)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[e][i] *= keep;
      }
      oct w[4];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[kt][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][i], p.scale_log2, -top));
          sum += s[kt][i];
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          u32x4 x;
#pragma unroll
          for (int k = 0; k < 4; ++k) x[k] = T::narrow2(s[kt][8 * half + 2 * k], s[kt][8 * half + 2 * k + 1]);
          w[2 * kt + half] = bits<oct>(x);
        }
      }
      const int group = lane / 16, from_key = 4 * (group / 2) + lane % 16 / 4, from_piece = 2 * (group % 2) + lane % 4 / 2;
#pragma unroll
      for (int e = 0; e < kTiles; ++e)
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          s16x4 part[2];
#pragma unroll
          for (int jj = 0; jj < 2; ++jj) {
            const int key = 16 * kb + 8 * jj + from_key;
            part[jj] = read_transposed(value_rows + key * kRowBytes + piece_of<kDim>(key, 4 * e + from_piece) * 16 + lane % 2 * 8);
          }
          const s16x8 a = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
          acc[e] = T::mfma32(bits<oct>(a), w[kb], acc[e]);
        }
    };

    int again = 0;
    if (from < to) {
      again = missing_page(p, table, from, to);
      loader.begin(p, head);
      loader.bring(p, table, from, to, keys[0], values[0]);
      const auto block = [&](int k0, char *key_rows, char *value_rows, char *next_keys, char *next_values) {
        loader.arrive(p, table, k0, to, key_rows, value_rows);
        __syncthreads();                                        // it is there, and nobody reads the other one any more
        if (k0 + kKeys > min(to, tile_all_end) || k0 < tile_all_begin) {
          // A weight of zero does not silence a NaN or an infinity: where any stands among values that not every row sees, the rows
          // are computed again by the kernel that joins.
          again |= loader.clear_values(value_rows, k0, tile_from, to);
          __syncthreads();
        }
        if (k0 + kKeys < to) loader.bring(p, table, k0 + kKeys, to, next_keys, next_values);
        multiply(k0, key_rows, value_rows);
      };
      for (int k0 = from; k0 < to; k0 += 2 * kKeys) {           // (two at a time: addresses in shared memory are constants)
        block(k0, keys[0], values[0], keys[1], values[1]);
        if (k0 + kKeys < to) block(k0 + kKeys, keys[1], values[1], keys[0], values[0]);
      }
    }
    again = __syncthreads_or(again);                            // (and nobody reads the last block any more)
    if (threadIdx.x == 0) mark_unit(p, ChunkShape::kPlan, u, again);
    sum += __shfl_xor(sum, 32);
    if (row < all_rows) {
      const int64_t token = rq.first + row / p.group;
      const int64_t part_row = static_cast<int64_t>(plan.part[r]) + static_cast<int64_t>(split) * all_rows + row;
      float *part = part_of(p, ChunkShape::kPlan, part_row, head);
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
  const size_t lds = static_cast<size_t>(p.batch.requests + 1) * 3 * sizeof(int);
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
