// Element types and small device functions of the iteration operators (gfx950).
#ifndef GNR_ITER_DEVICE_H
#define GNR_ITER_DEVICE_H

#include <hip/hip_runtime.h>

#include <type_traits>

#include "gnr_iter_internal.h"

namespace gnr {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) short s16x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

template <class To, class From>
__device__ __forceinline__ To bits(From f)
{
  static_assert(sizeof(To) == sizeof(From), "same size");
  return __builtin_bit_cast(To, f);
}

// The 16-bit types: T::split2 makes two numbers of each of two weights from 0 to 2^15, an upper one (cut off) and what it leaves (rounded), together within 2^-14 of it
// (bfloat16) or 2^-20 (float16). Neither is zero or negative where the weight counts, so that an infinite value times both is the same infinity: a little less than the weight is cut
// off, and a lower number that would vanish is float16's smallest. There weights are multiplied by 2^kSplitShift, as their sum is, to have room for lower numbers.
// T::from_e4m3 reads two codes (the lower or upper half of a word) times a power of two, exactly but for
// what leaves the type's range, in one instruction (the attention kernels take cached rows that way too: powers of two that went through scores and weights instead would cost one
// for each of these, and change nothing where the rows fit the queries' type); T::to_e4m3 is its inverse, rounded to nearest even, for values within 448 * 2^e.
struct Bf16 {
  typedef __bf16 elem;
  typedef bf16x2 pair;
  typedef bf16x8 oct;
  static constexpr uint32_t kInf = 0x7F80u;
  static __device__ __forceinline__ float widen(uint32_t w) { return bits<float>(w << 16); }
  static __device__ __forceinline__ uint32_t narrow2(float a, float b) { pair p = {static_cast<__bf16>(a), static_cast<__bf16>(b)}; return bits<uint32_t>(p); }
  static constexpr float kSplitShift = 0.0f;
  static __device__ __forceinline__ void split2(float a, float b, uint32_t &upper, uint32_t &lower)
  {
    const uint32_t x = bits<uint32_t>(a * 0x1.FFp-1f), y = bits<uint32_t>(b * 0x1.FFp-1f);
    upper = __builtin_amdgcn_perm(y, x, 0x07060302u);
    lower = narrow2(a - bits<float>(x & 0xFFFF0000u), b - bits<float>(y & 0xFFFF0000u));
  }
  static __device__ __forceinline__ f32x4 mfma16(oct a, oct b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x16 mfma32(oct a, oct b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  template <bool kUpper>
  static __device__ __forceinline__ uint32_t from_e4m3(uint32_t codes, float scale) { return bits<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, kUpper)); }
  template <bool kUpper>
  static __device__ __forceinline__ s16x2 to_e4m3(s16x2 codes, uint32_t w, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(codes, bits<pair>(w), scale, kUpper); }
};
struct Fp16 {
  typedef _Float16 elem;
  typedef f16x2 pair;
  typedef f16x8 oct;
  static constexpr uint32_t kInf = 0x7C00u;
  static __device__ __forceinline__ float widen(uint32_t w) { return static_cast<float>(bits<_Float16>(static_cast<uint16_t>(w))); }
  static __device__ __forceinline__ uint32_t narrow2(float a, float b) { pair p = {static_cast<_Float16>(a), static_cast<_Float16>(b)}; return bits<uint32_t>(p); }
  static constexpr float kSplitShift = 7.0f;
  static __device__ __forceinline__ void split2(float a, float b, uint32_t &upper, uint32_t &lower)
  {
    upper = bits<uint32_t>(__builtin_amdgcn_cvt_pkrtz(a * 0x1.FFEp-1f, b * 0x1.FFEp-1f));
    lower = narrow2(fmaxf(a - widen(upper & 0xFFFFu), fminf(a, 0x1p-24f)), fmaxf(b - widen(upper >> 16), fminf(b, 0x1p-24f)));
  }
  static __device__ __forceinline__ f32x4 mfma16(oct a, oct b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x16 mfma32(oct a, oct b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  template <bool kUpper>
  static __device__ __forceinline__ uint32_t from_e4m3(uint32_t codes, float scale) { return bits<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, kUpper)); }
  template <bool kUpper>
  static __device__ __forceinline__ s16x2 to_e4m3(s16x2 codes, uint32_t w, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(codes, bits<pair>(w), scale, kUpper); }
};

__device__ __forceinline__ float exponent_scale(uint32_t byte) { return bits<float>(byte << 23); }

// f(0) .. f(kN - 1) with numbers that are constants: arrays that are indexed by them stay in registers.
template <int kN, int kAt = 0, class F>
__device__ __forceinline__ void repeat(const F &f)
{
  if constexpr (kAt < kN) {
    f(std::integral_constant<int, kAt>{});
    repeat<kN, kAt + 1>(f);
  }
}
#define GNR_INLINE __attribute__((always_inline))

// Whether either of two 16-bit values is a NaN or an infinity.
template <class T>
__device__ __forceinline__ bool no_number(uint32_t w) { return (w & T::kInf) == T::kInf || (w >> 16 & T::kInf) == T::kInf; }

// A number that is the same in all lanes, in scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v)
{
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(v)), hi = __builtin_amdgcn_readfirstlane(static_cast<int>(v >> 32));
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// A wave's load of 64 x 16 bytes from memory to 1 KB of shared memory, lane after lane; wait_for_lds_loads waits for all of the wave's.
__device__ __forceinline__ void load_to_lds(const void *from, char *to)
{
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}
__device__ __forceinline__ void wait_for_lds_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Transposing LDS load: of 16 lanes, lanes 4 r to 4 r + 3 point at row r of a matrix of 4 x 16 16-bit elements; lane i gets column i.
__device__ __forceinline__ s16x4 read_transposed(const char *at)
{
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at);
}

inline int iter_hip_ok(hipError_t e) { return e == hipSuccess ? SIM_OK : SIM_EHIP; }

}  // namespace gnr
#endif
