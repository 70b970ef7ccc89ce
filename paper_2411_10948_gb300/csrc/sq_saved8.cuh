// Tensors kept in 8 bits: int8 codes q with a power-of-two scale per 32 elements of a row, x~ = q 2^e.
#pragma once

#include "sq_block.cuh"
#include "sq_device.cuh"

namespace sq {

constexpr uint32_t kScaleTop8 = 249;   // 2^122, the largest a finite block has

// x 2^-e rounded to nearest even as bytes: adding 1.5 2^23 leaves the integer in the low bits
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  const float2 i2 = make_float2(inv, inv), shift = make_float2(12582912.0f, 12582912.0f);
  const float2 p = fma2(make_float2(a, b), i2, shift), q = fma2(make_float2(c, d), i2, shift);
  const uint32_t lo = __byte_perm(__float_as_uint(p.x), __float_as_uint(p.y), 0x0040);
  const uint32_t hi = __byte_perm(__float_as_uint(q.x), __float_as_uint(q.y), 0x0040);
  return __byte_perm(lo, hi, 0x5410);
}
__device__ __forceinline__ uint2 codes8_int8(const float (&f)[8], uint32_t scale) {
  if (scale == kScaleNan) return make_uint2(0, 0);
  const float inv = scale_inverse(scale);
  return make_uint2(codes4(f[0], f[1], f[2], f[3], inv), codes4(f[4], f[5], f[6], f[7], inv));
}
// eight codes: a byte q + 128 below the exponent of 2^23 is the float
// 8388608 + 128 + q, so a subtraction gives q (a conversion per code runs at a quarter of the rate)
__device__ __forceinline__ void decode8(uint2 w, float2 (&q)[4]) {
  const uint32_t x = w.x ^ 0x80808080u, y = w.y ^ 0x80808080u;
  const float2 off = make_float2(-8388736.0f, -8388736.0f);
  auto f = [](uint32_t v, uint32_t sel) { return __uint_as_float(__byte_perm(v, 0x4B000000u, sel)); };
  q[0] = add2(make_float2(f(x, 0x7540), f(x, 0x7541)), off);
  q[1] = add2(make_float2(f(x, 0x7542), f(x, 0x7543)), off);
  q[2] = add2(make_float2(f(y, 0x7540), f(y, 0x7541)), off);
  q[3] = add2(make_float2(f(y, 0x7542), f(y, 0x7543)), off);
}
// The value of a kept block's scale byte.  The largest numbers of a type with FP32's range keep as 64 2^122,
// which FP32 does not hold: 2^122 less 2^-24 of it makes that FP32's largest number (an infinity would
// make a derivative NaN that is 0 or 1).
__device__ __forceinline__ float scale_value8(uint32_t byte) {
  if (byte == kScaleNan) return __uint_as_float(0x7FC00000u);
  return __uint_as_float(byte == 0 ? 0x00400000u : (byte << 23) - (byte == kScaleTop8 ? 1u : 0u));
}
__device__ __forceinline__ void decode8(uint2 w, uint32_t scale, float (&f)[8]) {
  const float s = scale_value8(scale);
  float2 q[4];
  decode8(w, q);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    q[i] = mul2(q[i], make_float2(s, s));
    f[2 * i] = q[i].x, f[2 * i + 1] = q[i].y;
  }
}

// the scale byte of the block of 32 that four neighbouring threads hold
__device__ __forceinline__ uint32_t block_scale8(const float (&f)[8]) {
  float m = max_abs(max_abs(max_abs(f[0], f[1]), max_abs(f[2], f[3])), max_abs(max_abs(f[4], f[5]), max_abs(f[6], f[7])));
  m = max_abs(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
  m = max_abs(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
  return scale_of_int8(__float_as_uint(m));
}
__device__ __forceinline__ uint2 ld_codes8(const int8_t* p) {
  uint2 v;
  asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t ld_scale(const uint8_t* p) { return static_cast<uint32_t>(ld_here(p)); }

// Eight elements of a row on their way: aligned rows as they lie, others as a warp's dense loads.
template <typename T, bool kVec>
struct RowIn {
  Raw8<T> raw;
  Dense8 dense;
  __device__ __forceinline__ void load(const T* row, int64_t c, int64_t C, bool in, int lane) {
    if constexpr (kVec) {
      if (!in || c >= C) zero8(raw);
      else if (c + 8 <= C) load8(raw, row + c);
      else load8_tail(raw, row + c, static_cast<int>(C - c));
    } else {
      const int64_t seg = c - 8 * lane;   // the warp's first column
      dense_load(dense, row + seg, in ? C - seg : 0, lane);
    }
  }
  __device__ __forceinline__ void values(float (&f)[8], T* buf, int lane) {
    if constexpr (!kVec) dense_to_raw(raw, dense, buf, lane);
    values8<T>(raw, f);
  }
};
template <typename T, bool kVec>
__device__ __forceinline__ void row_store(T* row, const float (&f)[8], int64_t c, int64_t C, bool in, T* buf, int lane) {
  if constexpr (kVec) {
    if (!in || c >= C) return;
    if (c + 8 <= C) store8(row + c, f);
    else store8_tail(row + c, f, static_cast<int>(C - c));
  } else {
    const int64_t seg = c - 8 * lane;
    dense_store(row + seg, f, in ? C - seg : 0, buf, lane);
  }
}

template <typename T>
inline bool rows16(const void* p, int64_t ld) {   // host: every row is 16-byte aligned
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * static_cast<int64_t>(sizeof(T))) % 16 == 0;
}

}  // namespace sq
