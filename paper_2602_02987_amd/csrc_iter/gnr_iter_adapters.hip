// Low-rank adapters of a batch's requests, added to a projection that they share (gfx950).
#include "gnr_iter_device.h"

namespace gnr {

constexpr int kThreads = 256;

// The adapter of a token (-1: none), found by one wave from the bounds of the requests; `token` and the result are uniform.
__device__ __forceinline__ int adapter_of(const AdapterParams &p, int64_t token, int lane)
{
  int own = -1;
  bool bad = false;
  for (int r0 = 0; r0 < p.requests; r0 += 64) {
    const int r = r0 + lane;
    bool hit = false;
    if (r < p.requests) {
      const int b = p.q_start[r], e = p.q_start[r + 1];
      hit = b <= token && token < e;
      bad |= b < 0 || e < b || e > p.tokens;
    }
    const uint64_t m = __ballot(hit);
    if (m && own < 0) own = r0 + __ffsll(static_cast<unsigned long long>(m)) - 1;
  }
  uint32_t flags = own < 0 || __any(bad) ? ITER_BAD_BATCH : 0;
  int a = -1;
  if (own >= 0) {
    a = p.adapter[own];
    if (a < -1 || a >= p.set.adapters) {
      flags |= ITER_BAD_ADAPTER;
      a = -1;
    }
  } else {
    a = -2;
  }
  if (flags && p.status && lane == 0) atomicOr(p.status, flags);
  return a;
}

// A workgroup for each token: h = down x, then out = base + scale * up h.
template <class T>
__global__ void __launch_bounds__(kThreads) gnr_adapters_kernel(const AdapterParams p)
{
  __shared__ float h[ITER_MAX_RANK];
  __shared__ int which;
  const int64_t token = blockIdx.x;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, rank = p.set.rank;
  if (wave == 0) {
    const int found = adapter_of(p, token, lane);
    if (lane == 0) which = found;
  }
  __syncthreads();
  const int a = which;
  if (a == -2) return;
  const uint16_t *x = static_cast<const uint16_t *>(p.x) + token * p.x_stride;
  if (a >= 0) {
    const uint16_t *down = static_cast<const uint16_t *>(p.set.down) + static_cast<int64_t>(a) * rank * p.set.width_in;
    for (int r = wave; r < rank; r += kThreads / 64) {
      float s = 0.0f;
      for (int64_t d = lane; d < p.set.width_in; d += 64) s = __builtin_fmaf(T::widen(x[d]), T::widen(down[r * p.set.width_in + d]), s);
      for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
      if (lane == 0) h[r] = s;
    }
  }
  __syncthreads();
  const uint16_t *base = static_cast<const uint16_t *>(p.base) + token * p.base_stride;
  uint16_t *out = static_cast<uint16_t *>(p.out) + token * p.out_stride;
  for (int64_t o = threadIdx.x; o < p.set.width_out; o += kThreads) {
    float y = T::widen(base[o]);
    if (a >= 0) {
      const uint16_t *up = static_cast<const uint16_t *>(p.set.up) + (static_cast<int64_t>(a) * p.set.width_out + o) * rank;
      float s = 0.0f;
      for (int r = 0; r < rank; ++r) s = __builtin_fmaf(h[r], T::widen(up[r]), s);
      y = __builtin_fmaf(p.set.scale[a], s, y);
    }
    out[o] = static_cast<uint16_t>(T::narrow2(y, 0.0f));
  }
}

size_t adapters_bytes(const iter_adapter_set &, int64_t) { return 0; }

int launch_adapters(const AdapterParams &p, void *stream)
{
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned grid = static_cast<unsigned>(p.tokens);
  if (p.type == ITER_BF16) gnr_adapters_kernel<Bf16><<<grid, kThreads, 0, s>>>(p);
  else gnr_adapters_kernel<Fp16><<<grid, kThreads, 0, s>>>(p);
  return iter_hip_ok(hipGetLastError());
}

}  // namespace gnr
