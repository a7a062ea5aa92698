// What the entry points over an 8-bit cache share (include/pctree.h, "The cache
// in 8 bits"): blocks of slots with a scale, codes and their conversions.
#pragma once

#include <cuda_fp8.h>

#include "kv_rows.cuh"

namespace pct {

constexpr int kMinExp = -15, kMaxExp = 7;    // of the scales: code * 2^e is exact in fp16
constexpr int kExpBias = 127;                // a scale's byte is e + 127 (e8m0)

// Division of 0 .. 2^31 - 1 by a number known on the host.
struct FastDiv {
  uint32_t mul;
  int shift, by;
};
inline FastDiv fast_div(int by) {
  // floor(n / by) = (n * mul) >> (32 + shift) with mul = ceil(2^(32 + shift) / by), 2^shift the
  // largest power of two <= by: the error n * (mul * by - 2^(32 + shift)) / by < n * 2^-31 stays
  // below 2^(32 + shift) / by, since n < 2^31
  int shift = 0;
  while ((2ll << shift) <= by) ++shift;
  const unsigned long long top = 1ull << (32 + shift);
  const unsigned long long mul = (top + by - 1) / by;
  return {mul >> 32 ? 0u : static_cast<uint32_t>(mul), shift, by};
}
__device__ __forceinline__ int div_by(int n, const FastDiv& d) {
  // (mul 0 stands for 2^32: by a power of two)
  return d.mul == 0 ? n >> d.shift
                    : static_cast<int>(__umulhi(static_cast<uint32_t>(n), d.mul) >> d.shift);
}

// Pages in blocks of 2^shift slots (the last of a page may be shorter).
struct Kv8Blocks {
  FastDiv page;
  int shift, per_page;
};
inline Kv8Blocks kv8_blocks(int page_size, int scale_block) {
  int shift = 0;
  while ((1 << shift) < scale_block) ++shift;
  return {fast_div(page_size), shift,
          static_cast<int>((static_cast<long long>(page_size) + scale_block - 1) >> shift)};
}
inline bool kv8_block_ok(int scale_block) {
  return scale_block >= 1 && scale_block <= 128 && (scale_block & (scale_block - 1)) == 0;
}

// The smallest e in the scales' range with 448 * 2^e >= top (finite, >= 0).
__device__ __forceinline__ int least_exp(float top) {
  const uint32_t u = __float_as_uint(top);
  // top = f * 2^x, f in [1, 2); 448 = 1.75 * 2^8
  const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(kMinExp, min(kMaxExp, e));
}
__device__ __forceinline__ float exp2_of(int e) {        // 2^e, |e| < 127
  return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}
// The exponent of a scale's byte, brought into the range that scales have.
__device__ __forceinline__ int scale_exp(uint32_t byte) {
  return max(kMinExp, min(kMaxExp, static_cast<int>(byte) - kExpBias));
}
__device__ __forceinline__ bool scale_ok(uint32_t byte) {
  return byte >= kExpBias + kMinExp && byte <= kExpBias + kMaxExp;
}

// Two floats as codes, rounded to nearest even, past 448 to 448 (the lower byte
// holds the first); two codes as halves.
__device__ __forceinline__ uint32_t codes2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ uint32_t halves2(uint32_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(codes)));
  return r;
}
// Four codes of a scale as codes of another, `by` the scales' quotient.
__device__ __forceinline__ uint32_t rescaled4(uint32_t w, float by) {
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t h = halves2(w >> (16 * i));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    out |= codes2(f.x * by, f.y * by) << (16 * i);
  }
  return out;
}
__device__ __forceinline__ uint4 rescaled16(const uint4& x, float by) {
  return make_uint4(rescaled4(x.x, by), rescaled4(x.y, by), rescaled4(x.z, by),
                    rescaled4(x.w, by));
}

}  // namespace pct
