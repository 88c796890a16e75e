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

// How the R query rows of a K/V head are taken: by warps or by CTAs, in units of as many
// rows, workers.  A warp's registers hold O of 8 rows of 128-wide heads, of 16 of 64-wide
// ones, and it decodes an entry for these alone; the CTAs of attend4_rows_kernel decode it
// for up to 96, in a pipeline that takes as long for one row as for 64.  us by warps and by CTAs:
// 64-wide heads, 32 sequences up to 8000, 6 rows 25, 49; 15 rows 36, 50; 16 rows of 64
// sequences up to 16384 131, 218; 32 rows (two units of 16 side by side) 248, 225.  128-wide
// heads, 64 sequences up to 16384, 8 rows 131, 262; 12 rows (two units) 245, 264; 24 (three)
// 364, 271; 16 sequences up to 6000, 16 rows 34, 37; 24 rows 45, 38.
constexpr int kWarps4 = 4;                 // of a block of attend4_kernel
constexpr int kRowsMost4 = 96;             // of a unit of attend4_rows_kernel
// Blocks of an SM, by the registers that NT x 8 rows take (and scales that come in pieces).
constexpr int attend4_blocks(int NT, bool plain) { return NT == 1 && plain ? 4 : 3; }
constexpr int rows4_workers(int sms) { return 2 * sms; }
struct Plan4 {
  bool wide, plain, by_ctas;
  int blocks, rows, NT, workers;
};
inline Plan4 plan4_of(int R, int D, int sms) {
  Plan4 x;
  x.wide = D > 64;
  x.plain = D == (x.wide ? 128 : 64);
  x.by_ctas = R > 16;
  x.blocks = ceil_div(R, x.by_ctas ? kRowsMost4 : x.wide ? 8 : 16);
  x.rows = ceil_div(R, x.blocks);
  x.NT = ceil_div(x.rows, 8);
  x.workers = x.by_ctas ? rows4_workers(sms) : sms * attend4_blocks(x.NT, x.plain) * kWarps4;
  return x;
}

// A handle's workspace: notes on the units, then the slots of parts, two a worker: a row's
// reference and sums (16 bytes), and its DK elements.
struct Slots4 {
  size_t ml, o, end;                       // bytes from the first slot's on
};
inline Slots4 slots4_of(const Plan4& x) {
  const size_t rows = 2 * (size_t)x.workers * 8 * x.NT;
  return Slots4{0, rows * 16, rows * (16 + (x.wide ? 128 : 64) * 4)};
}
struct Cache4Workspace {
  size_t slots, bytes;                     // parts of units; notes on the units lie before them
};
inline Cache4Workspace cache4_workspace(const Cache4Shape& s, int sms) {
  size_t units = 0, most = 0;
  for (int T = 1; T <= s.max_T; ++T) {
    const Plan4 x = plan4_of(T * (s.Hq / s.Hkv), s.D, sms);
    const size_t u = (size_t)SPIKE_PROJ_CACHE_MAX_B * s.Hkv * x.blocks * 8, p = slots4_of(x).end;
    units = u > units ? u : units;
    most = p > most ? p : most;
  }
  const size_t slots = (units + 255) / 256 * 256;
  return Cache4Workspace{slots, slots + most};
}

// A unit's parts, as merge4_kernel finds them noted: in slot `slot` >= 0, and in the first
// slots, 2 w, of the workers w behind that one (slot / 2) that walk beside it, up to `last` (none:
// last <= slot / 2).  Where attend4_rows_kernel gave up on a wait the note may be an earlier call's,
// of more workers with fewer rows each: whether it is of slots that this call has, of
// `workers` workers.
inline __host__ __device__ bool parts_within(int32_t slot, int32_t last, int32_t workers) {
  return slot < 2 * workers && last < workers;
}

// Tiles of entries that an attend call has at most (its kernels count them in 32 bits).
int64_t attend4_tiles(const Cache4Shape& s, const sp_attend4& c);
cudaError_t launch_write4(const Cache4Shape& s, const sp_write4& c, cudaStream_t stream);
cudaError_t launch_read4(const Cache4Shape& s, const sp_read4& c, cudaStream_t stream);
cudaError_t launch_attend4(const Cache4Shape& s, const sp_attend4& c, uint8_t* ws, size_t slots, int* err, int fault,
                           cudaStream_t stream);

// n / d and n % d for n < 2^31, d < 2^31: a product with the reciprocal, rounded up to 33 bits
// (Granlund and Montgomery, "Division by invariant integers using multiplication", 1994).
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
