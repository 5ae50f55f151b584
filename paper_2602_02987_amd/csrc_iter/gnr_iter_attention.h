// Constants and device functions of the attention kernels (gfx950).
#ifndef GNR_ITER_ATTENTION_H
#define GNR_ITER_ATTENTION_H

#include <cfloat>

#include "gnr_iter_device.h"

namespace gnr {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kBlockKeys = 32 * kWaves;        // keys a workgroup takes at a time, 32 to a wave
constexpr int kBlocks = 768;                   // workgroups of a launch: three to a compute unit
constexpr int kPiecesPerBlock = 4;
constexpr int kPartTail = 4;                   // maximum, sum, two of padding

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

}  // namespace gnr
#endif
