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
// write4_kernel, read4_kernel: a thread has one group of every few tokens, and adds
// up what little of their addresses changes.  Bound by memory: 4 sequences of 32768
// tokens, 8 heads of 128, their values back as well, 1.22 GB in 176 us (7.0 TB/s, 104 %
// of a plain copy's rate; 259 us with 16-byte loads and one group at a time); 48 of up
// to 2047 read back, 258 MB in 38.4 us (6.7 TB/s).  A token of one sequence takes 1.6 us,
// the launch.  Groups, not rows, are a thread's, so that the largest magnitude needs no
// other thread; two are on their way at a time, as 32 bytes each.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "sp_cache4.cuh"
#include "sp_ptx.cuh"

namespace sp {
namespace {

constexpr int kThreads = 256;
constexpr int kItems = 2;                  // groups of a thread on their way at a time
constexpr int kTurns = 2;                  // times that, of a block

struct Strides {
  int64_t batch, token, head;
};
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
  int32_t T, capacity;
  int32_t groups, columns;                 // of a row; of a token (all K/V heads)
  int32_t across, tokens, blocks;          // a block: columns, tokens at a time; blocks for all columns
};

// A thread's column and its tokens t, t + step, ..
struct Place {
  int b, h, group, t, step, end;           // end: tokens of the sequence, at most those of the block
  int64_t at;                              // slot of token 0
};
__device__ __forceinline__ bool place_of(const Params& p, Place* x) {
  const int row = threadIdx.x / p.across, chunk = blockIdx.x / p.blocks;
  const int column = (blockIdx.x - chunk * p.blocks) * p.across + threadIdx.x - row * p.across;
  x->b = blockIdx.y;
  x->h = column / p.groups;
  x->group = column - x->h * p.groups;
  x->step = p.tokens;
  const int first = chunk * (p.tokens * kItems * kTurns);
  x->t = first + row;
  x->end = min(p.n ? min(max(p.n[x->b], 0), p.T) : p.T, first + p.tokens * kItems * kTurns);
  x->at = p.at ? p.at[x->b] : 0;
  return row < p.tokens && column < p.columns && x->t < x->end;
}

template <bool BF16>
__device__ __forceinline__ float2 to_float(uint32_t x) {
  if constexpr (BF16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&x));
}
// 32 bytes, a whole sector of memory.
__device__ __forceinline__ void load8(const void* from, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(from)
               : "memory");
}
__device__ __forceinline__ void store8(void* to, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
// A group's 16 elements; `whole`: they begin on 32 bytes.
__device__ __forceinline__ void load_group(const uint16_t* from, bool whole, uint32_t (&w)[8]) {
  if (whole) return load8(from, w);
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(from + 2 * i);
    w[i] = x.x, w[i + 1] = x.y, w[i + 2] = x.z, w[i + 3] = x.w;
  }
}
__device__ __forceinline__ void store_group(uint16_t* to, bool whole, const uint32_t (&w)[8]) {
  if (whole) return store8(to, w);
#pragma unroll
  for (int i = 0; i < 8; i += 4) *reinterpret_cast<uint4*>(to + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
}

// The values of a group's codes, in the type (both conversions are exact).
template <bool BF16>
__device__ __forceinline__ void values_of(uint2 codes, uint32_t scale, uint32_t (&w)[8]) {
  const uint32_t s = scale_half2(scale);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t v[4];
    codes_to_half(i ? codes.y : codes.x, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = mul_half2(v[j], s);
      if constexpr (BF16) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v[j]));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v[j]) : "f"(f.y), "f"(f.x));
      }
      w[4 * i + j] = v[j];
    }
  }
}

// The scale of a group whose largest magnitude is a (finite): a / 6 to the nearest
// of 3 mantissa bits, below 2^-14 to the nearest multiple of 2^-17, ties to even.
// (The product with 1 / 6, off by 2^-23 of itself, is the quotient again at 18
// mantissa bits where that has so few, as every tie has.)
__device__ __forceinline__ float scale_of(float a) {
  const uint32_t u = (__float_as_uint(a * (1.f / 6.f)) + 0x10u) & 0xffffffe0u;
  const float v = __uint_as_float(u);
  const float normal = __uint_as_float((u + 0x7ffffu + (u >> 20 & 1)) & 0xfff00000u);
  const float small = __fsub_rn(__fadd_rn(v, 96.f), 96.f);     // (96 = 1.5 * 2^23 * 2^-17)
  return fminf(v < 0x1p-14f ? small : normal, kMaxScale4);
}

// The codes of 8 elements, from -1 / s and s.  The quotients are corrected by their
// remainders, so that those that FP32 holds exactly (ties among them) are exact;
// they have the other sign until the end, with which -0 keeps its own.
template <bool BF16>
__device__ __forceinline__ uint32_t codes_of(const uint32_t* w, f32x2 minus_inv, f32x2 s) {
  float2 y[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = to_float<BF16>(w[j]);
    const f32x2 x = pair(f.x, f.y), about = mul2(x, minus_inv);
    y[j] = halves(fma2(fma2(about, s, x), minus_inv, about));
  }
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(y[0].x), "f"(y[0].y), "f"(y[1].x), "f"(y[1].y), "f"(y[2].x), "f"(y[2].y), "f"(y[3].x), "f"(y[3].y));
  return r ^ 0x88888888u;
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) write4_kernel(const __grid_constant__ Params p) {
  pdl_launch_dependents();
  pdl_wait();
  Place x;
  if (!place_of(p, &x)) return;
  const Side& side = p.side[blockIdx.z];
  const sp_kv4& held = side.held;
  const uint16_t* in = side.in + x.b * side.in_s.batch + x.t * side.in_s.token + x.h * side.in_s.head + 16 * x.group;
  uint16_t* out = side.out + x.b * side.out_s.batch + x.t * side.out_s.token + x.h * side.out_s.head + 16 * x.group;
  const int64_t in_step = x.step * side.in_s.token, out_step = x.step * side.out_s.token;
  int64_t slot = x.at + x.t;
  uint8_t* codes = held.codes + x.b * held.batch + slot * held.entry + x.h * held.head + 8 * x.group;
  uint8_t* scales = held.scales + x.b * held.scales_batch + slot * held.scales_entry + x.h * held.scales_head + x.group;
  const int64_t codes_step = x.step * held.entry, scales_step = x.step * held.scales_entry;
  const bool whole_in = ((uintptr_t)in | (uintptr_t)(2 * in_step)) % 32 == 0;
  const bool whole_out = ((uintptr_t)out | (uintptr_t)(2 * out_step)) % 32 == 0;
  for (int t = x.t; t < x.end; t += kItems * x.step) {
    uint32_t w[kItems][8];
#pragma unroll
    for (int i = 0; i < kItems; ++i)
      if (t + i * x.step < x.end) load_group(in + i * in_step, whole_in, w[i]);
    in += kItems * in_step;
#pragma unroll
    for (int i = 0; i < kItems; ++i)
      if (t + i * x.step < x.end) {
        // magnitudes are in the order of their bits, infinities and NaN above all
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = __vmaxu2(top, w[i][j] & 0x7fff7fffu);
        top = max(top & 0xffffu, top >> 16);
        const bool fine = top < (BF16 ? 0x7f80u : 0x7c00u);
        const float s = fine ? scale_of(to_float<BF16>(top).x) : 0.f;
        const uint32_t byte = fine ? __half_as_ushort(__float2half_rn(s)) >> 7 : kNaNScale4;
        uint2 c = make_uint2(0, 0);
        if (s > 0.f) {
          float inv;
          asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
          c.x = codes_of<BF16>(w[i], pair(-inv, -inv), pair(s, s));
          c.y = codes_of<BF16>(w[i] + 4, pair(-inv, -inv), pair(s, s));
        }
        if (slot >= 0 && slot < p.capacity) {
          *reinterpret_cast<uint2*>(codes) = c;
          *scales = (uint8_t)byte;
        }
        if (side.out) {
          uint32_t v[8];
          values_of<BF16>(c, byte, v);
          store_group(out, whole_out, v);
        }
        slot += x.step;
        codes += codes_step;
        scales += scales_step;
        out += out_step;
      }
  }
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) read4_kernel(const __grid_constant__ Params p) {
  pdl_launch_dependents();
  pdl_wait();
  Place x;
  if (!place_of(p, &x)) return;
  const Side& side = p.side[blockIdx.z];
  const sp_kv4& held = side.held;
  uint16_t* out = side.out + x.b * side.out_s.batch + x.t * side.out_s.token + x.h * side.out_s.head + 16 * x.group;
  const int64_t out_step = x.step * side.out_s.token;
  int64_t slot = x.at + x.t;
  const uint8_t* codes = held.codes + x.b * held.batch + slot * held.entry + x.h * held.head + 8 * x.group;
  const uint8_t* scales = held.scales + x.b * held.scales_batch + slot * held.scales_entry + x.h * held.scales_head + x.group;
  const int64_t codes_step = x.step * held.entry, scales_step = x.step * held.scales_entry;
  const bool whole_out = ((uintptr_t)out | (uintptr_t)(2 * out_step)) % 32 == 0;
  constexpr int kAll = kItems * kTurns;
  uint2 c[kAll];
  uint32_t byte[kAll];
  bool there[kAll];
#pragma unroll
  for (int i = 0; i < kAll; ++i) {
    there[i] = x.t + i * x.step < x.end && slot >= 0 && slot < p.capacity;
    if (there[i]) {
      c[i] = *reinterpret_cast<const uint2*>(codes);
      byte[i] = *scales;
    }
    slot += x.step;
    codes += codes_step;
    scales += scales_step;
  }
#pragma unroll
  for (int i = 0; i < kAll; ++i) {
    if (there[i]) {
      uint32_t v[8];
      values_of<BF16>(c[i], byte[i], v);
      store_group(out, whole_out, v);
    }
    out += out_step;
  }
}

Params params_of(const Cache4Shape& s, int T, const int32_t* at, const int32_t* n) {
  Params p{{}, at, n, T, s.capacity};
  p.groups = s.D / kGroup4;
  p.columns = s.Hkv * p.groups;
  p.blocks = ceil_div(p.columns, kThreads);
  p.across = ceil_div(p.columns, p.blocks);
  p.tokens = kThreads / p.across;
  return p;
}
dim3 grid_of(const Params& p, int B) {
  const int chunk = p.tokens * kItems * kTurns;
  return dim3((unsigned)(((int64_t)p.T + chunk - 1) / chunk * p.blocks), (unsigned)B, 2);
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
