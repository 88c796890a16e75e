// sp_cache4.cu -- entries of a KV cache into 4 bits and back (see
// spike_proj_cache4_write and spike_proj_cache4_read).  Per group of 16 elements
//
//   a = max |x|,  s = a / 6 rounded to 3 mantissa bits,  code = nearest of
//   0 0.5 1 1.5 2 3 4 6 to |x| / s, ties to the even code
//
// Every rounding is exact, whatever its precision: x has at most 11 significant
// bits and s 4, so that a quotient that is not a tie (of few bits) is at least
// 2^-12 of itself away from one, and FP32 is off by 2^-22.
//
// write4_kernel, read4_kernel: a thread has 8 elements, two threads a group.
// Bound by memory.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "sp_cache4.cuh"
#include "sp_ptx.cuh"

namespace sp {
namespace {

constexpr int kThreads = 256;
constexpr int kItems = 4;                  // of 8 elements, of a thread

struct Strides {
  int64_t batch, token, head;
};
__device__ __forceinline__ int64_t offset(const Strides& s, int b, int t, int h) {
  return b * s.batch + t * s.token + h * s.head;
}

// Rows of one of K and V: 16 bits (elements) and 4 bits (bytes).
struct Side {
  const uint16_t* in;
  uint16_t* out;
  Strides in_s, out_s;
  sp_kv4 held;
};
struct Params {
  Side side[2];
  const int32_t *at, *n;
  int32_t T, Hkv, capacity;
  uint32_t items;                          // of a sequence
  Divide row, head;                        // items of a row, heads of a token
};

// Where an item of a sequence is.
struct Place {
  int t, h, part;
  int64_t slot;
  bool there, held;                        // a token of the sequence; with a slot in the cache
};
__device__ __forceinline__ Place place_of(const Params& p, uint32_t item, int n, int64_t at) {
  Place x;
  uint32_t part, h;
  const uint32_t row = p.row(item, &part);
  x.t = p.head(row, &h);
  x.h = h;
  x.part = part;
  x.slot = at + x.t;
  x.there = item < p.items && x.t < n;
  x.held = x.there && x.slot >= 0 && x.slot < p.capacity;
  return x;
}
__device__ __forceinline__ int tokens_of(const Params& p, int b) {
  return p.n ? min(max(__ldg(p.n + b), 0), p.T) : p.T;
}

template <bool BF16>
__device__ __forceinline__ float2 to_float(uint32_t x) {
  if constexpr (BF16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&x));
}
// The values of 8 codes, in the type (both conversions are exact).
template <bool BF16>
__device__ __forceinline__ uint4 values_of(uint32_t codes, uint32_t scale) {
  uint32_t v[4];
  codes_to_half(codes, v);
  const uint32_t s = scale_half2(scale);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = mul_half2(v[i], s);
    if constexpr (BF16) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v[i]));
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v[i]) : "f"(f.y), "f"(f.x));
    }
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// The scale of a group whose largest magnitude is a (finite): a / 6 to the nearest
// of 3 mantissa bits, below 2^-14 to the nearest multiple of 2^-17, ties to even.
__device__ __forceinline__ float scale_of(float a) {
  const float v = __fdiv_rn(a, 6.f);
  const uint32_t u = __float_as_uint(v);
  const float normal = __uint_as_float((u + 0x7ffffu + (u >> 20 & 1)) & 0xfff00000u);
  const float small = __fsub_rn(__fadd_rn(v, 96.f), 96.f);     // (96 = 1.5 * 2^23 * 2^-17)
  return fminf(v < 0x1p-14f ? small : normal, kMaxScale4);
}

// Two codes.  The quotient is off by less than 2^-21 of itself; brought to 18
// mantissa bits, one that is a tie is that again.
__device__ __forceinline__ uint32_t codes_of(float2 x, float inv) {
  const uint32_t lo = (__float_as_uint(x.x * inv) + 0x10u) & 0xffffffe0u;
  const uint32_t hi = (__float_as_uint(x.y * inv) + 0x10u) & 0xffffffe0u;
  uint32_t r;
  asm("{\n\t.reg .b8 b, z;\n\t.reg .b16 w;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %1, %2;\n\t"
      "mov.b16 w, {b, 0};\n\tcvt.u32.u16 %0, w;\n\t}"
      : "=r"(r)
      : "f"(__uint_as_float(hi)), "f"(__uint_as_float(lo)));
  return r;
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) write4_kernel(const __grid_constant__ Params p) {
  pdl_launch_dependents();
  pdl_wait();
  const Side& side = p.side[blockIdx.z];
  const int b = blockIdx.y, n = tokens_of(p, b);
  const int64_t at = p.at ? __ldg(p.at + b) : 0;
  const uint32_t first = blockIdx.x * (kThreads * kItems) + threadIdx.x;
  Place place[kItems];
  uint4 raw[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    place[i] = place_of(p, first + i * kThreads, n, at);
    raw[i] = make_uint4(0, 0, 0, 0);
    if (place[i].there)
      raw[i] = __ldcs(reinterpret_cast<const uint4*>(side.in + offset(side.in_s, b, place[i].t, place[i].h) + 8 * place[i].part));
  }
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
    // magnitudes are in the order of their bits, infinities and NaN above all
    uint32_t top = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
    top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top & 0xffffu, top >> 16);
    const bool fine = top < (BF16 ? 0x7f80u : 0x7c00u);
    const float s = fine ? scale_of(to_float<BF16>(top).x) : 0.f;
    const uint32_t byte = fine ? __half_as_ushort(__float2half_rn(s)) >> 7 : kNaNScale4;
    uint32_t codes = 0;
    if (s > 0.f) {
      const float inv = __frcp_rn(s);
#pragma unroll
      for (int j = 0; j < 4; ++j) codes |= codes_of(to_float<BF16>(w[j]), inv) << (8 * j);
    }
    const Place& x = place[i];
    if (x.held) {
      const sp_kv4& to = side.held;
      *reinterpret_cast<uint32_t*>(to.codes + b * to.batch + x.slot * to.entry + x.h * to.head + 4 * x.part) = codes;
      if (x.part % 2 == 0)
        to.scales[b * to.scales_batch + x.slot * to.scales_entry + x.h * to.scales_head + x.part / 2] = (uint8_t)byte;
    }
    if (x.there && side.out)
      *reinterpret_cast<uint4*>(side.out + offset(side.out_s, b, x.t, x.h) + 8 * x.part) = values_of<BF16>(codes, byte);
  }
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) read4_kernel(const __grid_constant__ Params p) {
  pdl_launch_dependents();
  pdl_wait();
  const Side& side = p.side[blockIdx.z];
  const int b = blockIdx.y, n = tokens_of(p, b);
  const int64_t at = p.at ? __ldg(p.at + b) : 0;
  const uint32_t first = blockIdx.x * (kThreads * kItems) + threadIdx.x;
  Place place[kItems];
  uint32_t codes[kItems], scale[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    place[i] = place_of(p, first + i * kThreads, n, at);
    const Place& x = place[i];
    if (x.held) {
      const sp_kv4& from = side.held;
      codes[i] = __ldg(reinterpret_cast<const uint32_t*>(from.codes + b * from.batch + x.slot * from.entry + x.h * from.head + 4 * x.part));
      scale[i] = __ldg(from.scales + b * from.scales_batch + x.slot * from.scales_entry + x.h * from.scales_head + x.part / 2);
    }
  }
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const Place& x = place[i];
    if (x.held)
      *reinterpret_cast<uint4*>(side.out + offset(side.out_s, b, x.t, x.h) + 8 * x.part) = values_of<BF16>(codes[i], scale[i]);
  }
}

Params params_of(const Cache4Shape& s, int T, const int32_t* at, const int32_t* n) {
  Params p{{}, at, n, T, s.Hkv, s.capacity, (uint32_t)T * s.Hkv * (s.D / 8), Divide(s.D / 8), Divide(s.Hkv)};
  return p;
}
dim3 grid_of(const Params& p, int B) {
  return dim3((p.items + kThreads * kItems - 1) / (kThreads * kItems), (unsigned)B, 2);
}

}  // namespace

cudaError_t launch_write4(const Cache4Shape& s, const sp_write4& c, cudaStream_t stream) {
  Params p = params_of(s, c.T, c.at, c.n);
  p.side[0] = Side{static_cast<const uint16_t*>(c.k), static_cast<uint16_t*>(c.k_out), {c.k_batch, c.k_token, c.k_head},
                   {c.k_out_batch, c.k_out_token, c.k_out_head}, c.k4};
  p.side[1] = Side{static_cast<const uint16_t*>(c.v), static_cast<uint16_t*>(c.v_out), {c.v_batch, c.v_token, c.v_head},
                   {c.v_out_batch, c.v_out_token, c.v_out_head}, c.v4};
  return launch_pdl(s.dtype == SP_BF16 ? write4_kernel<true> : write4_kernel<false>, grid_of(p, c.B), dim3(kThreads), 0, stream, p);
}

cudaError_t launch_read4(const Cache4Shape& s, const sp_read4& c, cudaStream_t stream) {
  Params p = params_of(s, c.T, c.at, c.n);
  p.side[0] = Side{nullptr, static_cast<uint16_t*>(c.k_out), {}, {c.k_out_batch, c.k_out_token, c.k_out_head}, c.k4};
  p.side[1] = Side{nullptr, static_cast<uint16_t*>(c.v_out), {}, {c.v_out_batch, c.v_out_token, c.v_out_head}, c.v4};
  return launch_pdl(s.dtype == SP_BF16 ? read4_kernel<true> : read4_kernel<false>, grid_of(p, c.B), dim3(kThreads), 0, stream, p);
}

}  // namespace sp
