// Device helpers of the 8-bit stored form: e4m3 elements (OCP: no infinities,
// NaN is 0x7f, largest finite 448) with one power-of-two scale per block of
// 128, held as the byte e + 127.
//
// The scale of a block is 2^e, e the smallest integer (not below -127) for
// which the block's largest finite magnitude is at most 448 2^e.  A power of
// two costs the elements no relative precision (they are floating point), is
// what the scaled matrix instructions of gfx950 take per 32 of K, and makes an
// element's value independent of the scale except among the subnormals, so
// that a largest magnitude next to a border moves no result.
#pragma once
#include "common.h"

namespace moeca {
namespace {

constexpr int kBlk = 128;  // elements a scale covers

// Bytes of a quantised row of K elements, and of its scales: whole blocks, and
// whole 16-byte chunks of scales (one load instruction brings a row's scales
// of 16 blocks into LDS).
__host__ __device__ constexpr int64_t q8_pitch(int64_t K) { return (K + kBlk - 1) / kBlk * kBlk; }
__host__ __device__ constexpr int64_t q8_spitch(int64_t K) {
  return ((K + kBlk - 1) / kBlk + 15) / 16 * 16;
}

// Magnitudes are compared as bits (sign cleared, their order is the numeric one;
// infinities and NaN come last, from kInfBits on): one instruction for the
// largest of three, where a float maximum would first quieten its operands.
constexpr uint32_t kInfBits = 0x7f800000u;
__device__ __forceinline__ uint32_t q8_mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// The same with 0 for what is not finite: what a block's scale is chosen from.
__device__ __forceinline__ uint32_t q8_finite(float v) {
  const uint32_t b = q8_mag(v);
  return b < kInfBits ? b : 0u;
}

// The scale byte of a block whose largest finite magnitude has the bits `top`:
// m 2^x with 1 <= m < 2 needs e = x - 8, or one more when m > 1.75, which is when
// adding 0x1fffff to the mantissa carries into the exponent.
__device__ __forceinline__ int q8_scale_byte(uint32_t top) {
  const int b = static_cast<int>((top + 0x1fffffu) >> 23) - 8;
  return b > 0 ? b : 0;
}
// 2^-e and 2^e of a scale byte (0..247 as q8_scale_byte gives them; 2^-127 is
// a subnormal).
__device__ __forceinline__ float q8_inv(int byte) {
  return __uint_as_float(static_cast<uint32_t>(254 - byte) << 23);
}
__device__ __forceinline__ float q8_two(int byte) {
  return __uint_as_float(byte > 0 ? static_cast<uint32_t>(byte) << 23 : 0x00400000u);
}

// Four values, already divided by their scale (at most 448, or not finite), to
// e4m3: nearest, ties to even; the conversion makes NaN of NaN and infinities.
__device__ __forceinline__ uint32_t q8_pack4(float a, float b, float c, float d) {
  const int p = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, p, true));
}

typedef __attribute__((ext_vector_type(2))) float q8_f32x2;
__device__ __forceinline__ void q8_unpack4(uint32_t p, float* v) {
  const q8_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(p), false);
  const q8_f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(p), true);
  v[0] = lo[0];
  v[1] = lo[1];
  v[2] = hi[0];
  v[3] = hi[1];
}

// Largest of a 16-lane row's values, in every lane of the row.
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v) {
  auto step = [&](int o) { v = max(v, static_cast<uint32_t>(o)); };
  step(dpp_i32<kDppRow[0]>(static_cast<int>(v)));
  step(dpp_i32<kDppRow[1]>(static_cast<int>(v)));
  step(dpp_i32<kDppRow[2]>(static_cast<int>(v)));
  step(dpp_i32<kDppRow[3]>(static_cast<int>(v)));
  return v;
}

// Eight elements from p (16-byte aligned when VEC), those at or past n as 0.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int n, float* v) {
  if (VEC && n >= 8) {
    if constexpr (sizeof(T) == 2) {
      const uint4 r = *reinterpret_cast<const uint4*>(p);
      const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v[2 * u] = __uint_as_float(w[u] << 16);
        v[2 * u + 1] = __uint_as_float(w[u] & 0xffff0000u);
      }
    } else {
      const float4 a = reinterpret_cast<const float4*>(p)[0];
      const float4 b = reinterpret_cast<const float4*>(p)[1];
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
      v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    return;
  }
#pragma unroll
  for (int u = 0; u < 8; ++u) v[u] = u < n ? Act<T>::to_f32(p[u]) : 0.0f;
}

template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, int n, const float* v) {
  if (VEC && n >= 8) {
    if constexpr (sizeof(T) == 2) {
      uint4 r;
      r.x = f32_to_bf16(v[0]) | (uint32_t(f32_to_bf16(v[1])) << 16);
      r.y = f32_to_bf16(v[2]) | (uint32_t(f32_to_bf16(v[3])) << 16);
      r.z = f32_to_bf16(v[4]) | (uint32_t(f32_to_bf16(v[5])) << 16);
      r.w = f32_to_bf16(v[6]) | (uint32_t(f32_to_bf16(v[7])) << 16);
      *reinterpret_cast<uint4*>(p) = r;
    } else {
      reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
    return;
  }
#pragma unroll
  for (int u = 0; u < 8; ++u)
    if (u < n) p[u] = Act<T>::from_f32(v[u]);
}

// Eight elements of a lane, 16 lanes to a block: the block's scale byte (in
// every lane of the row) and the lane's eight bytes.
__device__ __forceinline__ uint2 q8_quant8(const float* v, int& byte) {
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < 8; ++u) top = max(top, q8_mag(v[u]));
  if (__builtin_expect(__any(top >= kInfBits), 0)) {
    top = 0;
#pragma unroll
    for (int u = 0; u < 8; ++u) top = max(top, q8_finite(v[u]));
  }
  byte = q8_scale_byte(row_max_u32(top));
  const float inv = q8_inv(byte);
  return make_uint2(q8_pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                    q8_pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv));
}

// Sum of squares of eight stored values, in fp64: exact per element (four
// significant bits), 4^e a power of two.
__device__ __forceinline__ double q8_square8(uint2 q, int byte) {
  float f[8];
  q8_unpack4(q.x, f);
  q8_unpack4(q.y, f + 4);
  double d = 0.0;
#pragma unroll
  for (int u = 0; u < 8; ++u) d += static_cast<double>(f[u]) * static_cast<double>(f[u]);
  return ldexp(d, 2 * (byte - 127));
}

}  // namespace
}  // namespace moeca
