// Shared by the host side and the kernels of the operators of one batch iteration.
#ifndef GNR_ITER_INTERNAL_H
#define GNR_ITER_INTERNAL_H

#include <cstddef>
#include <cstdint>

#include "gnr_iter.h"

namespace gnr {

struct AttentionParams {
  iter_cache cache;
  iter_batch batch;
  iter_rows q, out;
  int type, heads, group;      // group: query heads to a kv head
  int page_shift;
  float scale_log2;            // |scale| / ln 2: weights are powers of two
  uint32_t flip;               // sign bits of two 16-bit elements if the scale is negative
  int window, room;            // room: the most keys a request can have
  float *workspace;
  // of the kernel for few rows (0) and the one for chunks (1): rows of the requests it takes, workgroups, first word of its parts
  int least[2], most[2], blocks[2];
  int64_t parts[2];
  int64_t marks[2], units[2];  // first word of the units' marks and how many there can be
  int64_t cuts;                // first word of the records of cut tiles
  uint32_t *status;
};

struct AdapterParams {
  iter_adapter_set set;
  int type, requests;
  int64_t tokens;
  const int32_t *q_start, *adapter;
  const void *x, *base;
  void *out;
  int64_t x_stride, base_stride, out_stride;
  float *workspace;
  uint32_t *status;
};

// Blocks of keys of a piece if `all` are shared out over `workgroups`. No request has as many as the most it returns (positions are below 2^30, a block is 64 of them): a
// batch with more work than pieces of that length then has none of its tiles cut.
constexpr int blocks_of_a_piece(int64_t all, int workgroups)
{
  constexpr int64_t most = int64_t(1) << 25;
  const int64_t share = (all + workgroups - 1) / workgroups;
  return static_cast<int>(share < 1 ? 1 : share > most ? most : share);
}

// All return a sim_err; arguments have been checked.
int launch_kv_write(const iter_cache &c, int type, const iter_rows &k, const iter_rows &v, const int64_t *slots, int64_t tokens, void *stream);
int launch_kv_read(const iter_cache &c, int type, const iter_rows &k, const iter_rows &v, const int64_t *slots, int64_t tokens, void *stream);
size_t attention_bytes(const iter_cache &c, const iter_batch &b, int heads);
int launch_attention(const AttentionParams &p, void *stream);
size_t adapters_bytes(const iter_adapter_set &s, int64_t tokens);
int launch_adapters(const AdapterParams &p, void *stream);

}  // namespace gnr
#endif
