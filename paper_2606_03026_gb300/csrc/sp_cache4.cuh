// sp_cache4.cuh -- the form of a KV cache held in 4 bits: codes e2m1 (sign, 2
// exponent and 1 mantissa bits: 0 0.5 1 1.5 2 3 4 6), and per 16 elements a scale of
// 8 bits, which are those of a half-precision number from its exponent down to
// three mantissa bits.  A value, code times scale, has at most six significant bits
// and lies within half precision (the largest scale is 10240), so that products of
// the two in half precision are exact.
#pragma once

#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "sp_cache.h"

namespace sp {

struct Cache4Shape {
  int32_t max_T, Hq, Hkv, D, capacity, dtype;
};

constexpr int kGroup4 = 16;                // elements of a scale
constexpr uint32_t kNaNScale4 = 0xff;      // scale of a group with a NaN or an infinity
constexpr float kMaxScale4 = 10240.f;

struct Cache4Workspace {
  size_t slots, bytes;                     // parts of units; notes on the units lie before them
};
Cache4Workspace cache4_workspace(const Cache4Shape& s, int sms);

// Tiles of entries that an attend call has at most (its kernels count them in 32 bits).
int64_t attend4_tiles(const Cache4Shape& s, const sp_attend4& c);
cudaError_t launch_write4(const Cache4Shape& s, const sp_write4& c, cudaStream_t stream);
cudaError_t launch_read4(const Cache4Shape& s, const sp_read4& c, cudaStream_t stream);
cudaError_t launch_attend4(const Cache4Shape& s, const sp_attend4& c, uint8_t* ws, size_t slots, int* err, int fault,
                           cudaStream_t stream);

// n / d and n % d for n < 2^31, d < 2^31.
struct Divide {
  uint32_t mul = 0, shift = 0, d = 0;
  Divide() = default;
  explicit Divide(uint32_t by) : d(by) {
    while ((1ull << shift) < by) ++shift;
    mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - by)) / by + 1);
  }
#ifdef __CUDACC__
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const {
    return (uint32_t)(((uint64_t)__umulhi(n, mul) + n) >> shift);
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t n, uint32_t* rest) const {
    const uint32_t q = (*this)(n);
    *rest = n - q * d;
    return q;
  }
#endif
};

#ifdef __CUDACC__
// Four code pairs of a word, in half precision (without their scale).
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// The bits of a where the mask is 1, those of b where it is 0.
template <uint32_t MASK>
__device__ __forceinline__ uint32_t select_bits(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xe4;" : "=r"(r) : "r"(a), "r"(b), "n"(MASK));
  return r;
}
// Two scale bytes (the lower ones of x) in half precision; a product of both halves of x
// with one of them (an operand of the instruction that takes it twice).
__device__ __forceinline__ uint32_t scales_half2(uint32_t x) { return __byte_perm(x, 0, 0x4140) << 7; }
template <int WHICH>
__device__ __forceinline__ uint32_t mul_half2_by(uint32_t x, uint32_t scales) {
  const __half2 s = *reinterpret_cast<const __half2*>(&scales), a = *reinterpret_cast<const __half2*>(&x);
  const __half2 r = __hmul2_rn(a, WHICH ? __high2half2(s) : __low2half2(s));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// A scale byte as two equal half-precision numbers.
__device__ __forceinline__ uint32_t scale_half2(uint32_t byte) { return byte * 0x00800080u; }

// Two floats in one 64-bit register, for the packed FP32 instructions.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 halves(f32x2 x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
#endif

}  // namespace sp
