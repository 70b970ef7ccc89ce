// Microscaled 4-bit floats (the OCP MX format with e2m1 elements): quantization of a tensor
// along its rows, its columns or both in one pass, and the expansion back to values.
//
// A block of 32 elements along the contraction shares a power of two 2^e, the smallest with
// max|x| <= 6 2^e; an element is x 2^-e on the grid 0, .5, 1, 1.5, 2, 3, 4, 6, rounded to
// nearest (ties to even) or up with the probability of its fraction of the gap.  Codes of a row
// are packed two per byte, the lower nibble first; scale bytes lie in the order in which the
// tensor cores take them: 512-byte tiles of 128 rows x 4 blocks, the byte of row r, block b of
// a tile at 16 (r mod 32) + 4 (r / 32) + b.
//
// A thread block takes a 128 x 128 tile: its scales are one such tile in each orientation.  The
// rows are encoded from registers as they arrive, 32 bytes of them per thread; for the transposed
// copy the tile (and the draws of the stochastic rounding, so that each is hashed once) goes
// through shared memory, swizzled so that the four row blocks of a column read different banks.
// Stochastic rounding is bound by the integer pipe (the hash of the draws and the encoding); rounding to
// nearest fills no unit (issue slots 66%, integer pipe 59%, DRAM 52% busy at 46% of the warps): maxima are taken of 16-bit pairs as they lie, codes and signs are
// gathered by byte permutations, and what can go through the FP32 pipe does.  Measured, both orientations of
// 16384 x 4096 bf16: nearest 43 us (4.8 TB/s; one orientation 31 us, 5.5), stochastic 76 us (2.7 TB/s, the
// integer pipe 79% busy); fp32 nearest 76 us (4.5 TB/s); expansion of one orientation 33 us (5.2 TB/s).
#include <cuda_runtime.h>

#include <atomic>
#include <cstring>
#include <type_traits>

#include "sq_device.cuh"
#include "sq_block.cuh"
#include "sq_host.h"
#include "sq_quant_dev.cuh"

namespace sq {

constexpr int kMxTile = 128;
constexpr int kMxThreads = 256;

struct MxQuantArgs {
  const void* x;
  int64_t R, C, ld;
  uint64_t seed;
  int64_t row0;
  uint8_t* codes;
  int64_t ld_codes;
  uint8_t* scales;
  uint8_t* codes_t;
  int64_t ld_codes_t;
  uint8_t* scales_t;
  int64_t ktiles, ktiles_t;   // 512-byte scale tiles along a row, of each orientation
  int32_t* status;
};

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) {   // with sign replication (sel + 8)
  uint32_t r;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(sel));
  return r;
}
// byte 3 of four words, and (kSign) the sign of it over the whole byte
template <bool kSign>
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return prmt(prmt(a, b, 0x0073), prmt(c, d, 0x7300), kSign ? 0xFE98 : 0x7610);
}

// Stochastic rounding of v = |x| 2^-e (at most 6) onto the grid by a draw u = (f + 1/2) 2^-16, as a code
// in byte 3.  w = v + max(v, 1) is 2 v above 1, 1 + v below: the grid then has the floats of one
// mantissa bit, two codes per octave from 1 (code 0) on, and the fraction of the gap is the
// other 22 bits F of w's mantissa.  Adding 2^22 - 1 - (64 f + 32) = 64 n + 31, n = 65535 - f, carries
// into the grid's bits exactly where F 2^-22 > u; the sum is rounded upwards, which keeps the
// comparison exact (u is a multiple of 2^-17).  `draw` is 4 (64 n + 31), with a 2 in byte 3 that
// takes the exponent's bias off: 4 w's bits plus draw have the code in byte 3.
__device__ __forceinline__ uint32_t stochastic_code(float v, uint32_t draw) {
  const float a = fabsf(v);
  return __float_as_uint(__fadd_ru(a, fmaxf(a, 1.0f))) * 4u + draw;
}
// draw of the lower / upper half of a word of two n
__device__ __forceinline__ uint32_t draw_lo(uint32_t n) { return prmt(n, 0x0200007Cu, 0x7104); }
__device__ __forceinline__ uint32_t draw_hi(uint32_t n) { return prmt(n, 0x0200007Cu, 0x7324); }
// eight codes (byte 3 of c) and the signs of even and odd elements (whole bytes) as eight nibbles
__device__ __forceinline__ uint32_t pack_codes8(const uint32_t (&c)[8], uint32_t even_signs, uint32_t odd_signs) {
  const uint32_t even = top_bytes<false>(c[0], c[2], c[4], c[6]), odd = top_bytes<false>(c[1], c[3], c[5], c[7]);
  return (odd * 16u + even) | (even_signs & 0x08080808u) | (odd_signs & 0x80808080u);
}

// the draws of a group of four columns, as 65535 - f: the output for state z, inverted
__device__ __forceinline__ uint2 inverted_draws(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  z = ~(z ^ (z >> 31));
  return make_uint2(static_cast<uint32_t>(z), static_cast<uint32_t>(z >> 32));
}

// max |.| of values as they lie in 32-bit words: one float, or two of 16 bits side by side
template <typename T>
__device__ __forceinline__ uint32_t word_max(uint32_t a, uint32_t b) {
  if constexpr (sizeof(T) == 4) return __float_as_uint(max_abs(__uint_as_float(a), __uint_as_float(b)));
  else if constexpr (std::is_same<T, __half>::value) {
    const __half2 m = __hmax2_nan(__habs2(*reinterpret_cast<const __half2*>(&a)), __habs2(*reinterpret_cast<const __half2*>(&b)));
    return *reinterpret_cast<const uint32_t*>(&m);
  } else {
    const __nv_bfloat162 m =
        __hmax2_nan(__habs2(*reinterpret_cast<const __nv_bfloat162*>(&a)), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&b)));
    return *reinterpret_cast<const uint32_t*>(&m);
  }
}
template <typename T>
__device__ __forceinline__ uint32_t raw_max(const Raw8<T>& r) {
  const uint32_t m = word_max<T>(word_max<T>(r.w[0].x, r.w[0].y), word_max<T>(r.w[0].z, r.w[0].w));
  if constexpr (sizeof(T) == 4)
    return word_max<T>(m, word_max<T>(word_max<T>(r.w[1].x, r.w[1].y), word_max<T>(r.w[1].z, r.w[1].w)));
  else
    return m;
}
// the scale byte of a word's maximum (of both halves of a 16-bit pair)
template <typename T>
__device__ __forceinline__ uint32_t word_scale(uint32_t m) {
  if constexpr (sizeof(T) == 4) return scale_of_mx4(m);
  else {
    const float2 v = unpack2<T>(m);
    return scale_of_mx4(__float_as_uint(max_abs(v.x, v.y)));
  }
}

// codes of eight elements by their scale; n0, n1: their inverted draws
template <typename T, bool kSr>
__device__ __forceinline__ uint32_t encode8(const Raw8<T>& raw, uint32_t scale, uint2 n0, uint2 n1) {
  const float inv = scale_inverse(scale);
  float v[8];
  values8<T>(raw, v);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], inv);
  uint32_t r;
  if constexpr (kSr) {
    const uint32_t n[4] = {n0.x, n0.y, n1.x, n1.y};
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = stochastic_code(v[i], (i & 1) ? draw_hi(n[i / 2]) : draw_lo(n[i / 2]));
    uint32_t even, odd;
    if constexpr (sizeof(T) == 4) {
      even = top_bytes<true>(raw.w[0].x, raw.w[0].z, raw.w[1].x, raw.w[1].z);
      odd = top_bytes<true>(raw.w[0].y, raw.w[0].w, raw.w[1].y, raw.w[1].w);
    } else {
      const uint32_t lo = prmt(raw.w[0].x, raw.w[0].y, 0x7351), hi = prmt(raw.w[0].z, raw.w[0].w, 0x7351);
      even = prmt(lo, hi, 0xDC98);
      odd = prmt(lo, hi, 0xFEBA);
    }
    r = pack_codes8(c, even, odd);
  } else {
    r = codes8(v);
  }
  return scale == kScaleNan ? 0u : r;
}

// the swizzled offset (elements) of an even column of the staged tile
template <int kElemBytes>
__device__ __forceinline__ int staged_col(int row, int col) {
  return col ^ (((row >> 5) & 3) * (kElemBytes == 4 ? 8 : 16));
}

// kT: the transposed orientation too (or alone).  kVec: rows of x are 16-byte aligned; else the tile
// is staged element by element first, a warp along a row.
template <typename T, bool kSr, bool kT, bool kVec>
__global__ void __launch_bounds__(kMxThreads) mx4_quantize_kernel(const MxQuantArgs a) {
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ __align__(16) uint8_t srow[512];
  __shared__ __align__(16) uint8_t scol[512];
  T* tile = reinterpret_cast<T*>(dyn);
  uint16_t* draws = reinterpret_cast<uint16_t*>(dyn + sizeof(T) * kMxTile * kMxTile);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t tr = blockIdx.y, tc = blockIdx.x;
  const int64_t r0 = tr * kMxTile, c0 = tc * kMxTile;
  const bool rows_out = a.codes != nullptr && r0 < a.R;
  const bool cols_out = kT && c0 < a.C;
  griddep_wait();
  griddep_launch_dependents();
  const T* x = static_cast<const T*>(a.x);
  bool bad = false;
  if constexpr (!kVec) {
    if constexpr (sizeof(T) == 4) {
      // all of the tile on its way at once, zeros outside (5003 x 1155, nearest: 16.4 us; two rows of each warp
      // at a time through registers 18.5)
      const uint32_t base = smem_u32(dyn);
#pragma unroll 4
      for (int i = 0; i < kMxTile / 8; ++i) {
        const int rl = i * 8 + warp;
        const int64_t r = r0 + rl;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int col = 32 * j + lane;
          const bool in = r < a.R && c0 + col < a.C;
          cp_async_4(base + 4 * (rl * kMxTile + (staged_col<4>(rl, col & ~1) | (col & 1))), x + (in ? r * a.ld + c0 + col : 0), in);
        }
      }
      cp_async_commit();
      cp_async_wait<0>();
    } else {
#pragma unroll 1
      for (int i = 0; i < kMxTile / 8; i += 4) {
        uint32_t e[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int64_t r = r0 + (i + k) * 8 + warp, c = c0 + 32 * j + lane;
            e[k][j] = r < a.R && c < a.C ? ld_bits(x + r * a.ld + c) : 0u;
          }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int rl = (i + k) * 8 + warp, col = 32 * j + lane;
            const int at = rl * kMxTile + (staged_col<sizeof(T)>(rl, col & ~1) | (col & 1));
            reinterpret_cast<uint16_t*>(dyn)[at] = static_cast<uint16_t>(e[k][j]);
          }
      }
    }
    __syncthreads();
  }
  // rows: a thread takes 32 bytes (16 or 8 elements) of a row, four rows on their way at once
  constexpr int kH = sizeof(T) == 4 ? 1 : 2;           // groups of eight elements
  constexpr int kLanes = kMxTile / (8 * kH);           // threads of a row
  constexpr int kRows = 8 * (32 / kLanes);             // rows the block takes at once
  constexpr int kAhead = 4;
  const int t = lane % kLanes, rw = warp * (32 / kLanes) + lane / kLanes;
  const int64_t c = c0 + 8 * kH * t;
  const bool block_in = c0 + (8 * kH * t & ~31) < a.C;
  // the generator's state for the thread's first four columns of its first row, and its row step
  const uint64_t quads = static_cast<uint64_t>((a.C + 31) / 32 * 8);
  uint64_t z = 0;
  if constexpr (kSr)
    z = a.seed + (static_cast<uint64_t>(a.row0 + r0 + rw) * quads + static_cast<uint64_t>(c >> 2) + 1) * kSplitMixGamma;
#pragma unroll 1
  for (int part = 0; part < kMxTile / kRows; part += kAhead) {
    Raw8<T> raw[kAhead][kH];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int rl = (part + i) * kRows + rw;
      const int64_t r = r0 + rl;
#pragma unroll
      for (int h = 0; h < kH; ++h) {
        const int64_t ch = c + 8 * h;
        if constexpr (kVec) {
          if (r >= a.R || ch >= a.C)
            zero8(raw[i][h]);
          else if (ch + 8 <= a.C)
            load8(raw[i][h], x + r * a.ld + ch);
          else
            load8_tail(raw[i][h], x + r * a.ld + ch, static_cast<int>(a.C - ch));
        } else {
          const uint4* src = reinterpret_cast<const uint4*>(tile + rl * kMxTile + staged_col<sizeof(T)>(rl, 8 * (kH * t + h)));
          raw[i][h].w[0] = src[0];
          if constexpr (sizeof(T) == 4) raw[i][h].w[1] = src[1];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int rl = (part + i) * kRows + rw;
      const int64_t r = r0 + rl;
      uint2 n[2 * kH] = {};
      if constexpr (kSr) {
#pragma unroll
        for (int k = 0; k < 2 * kH; ++k) n[k] = inverted_draws(z + static_cast<uint64_t>(k) * kSplitMixGamma);
        z += kRows * quads * kSplitMixGamma;
      }
      if (rows_out) {   // uniform over the block
        uint32_t m = raw_max<T>(raw[i][0]);
        if constexpr (kH == 2) m = word_max<T>(m, raw_max<T>(raw[i][kH - 1]));
        m = word_max<T>(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        if constexpr (kH == 1) m = word_max<T>(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
        const uint32_t sc = word_scale<T>(m);
        bad |= sc == kScaleNan;
        uint32_t code[kH];
#pragma unroll
        for (int h = 0; h < kH; ++h) code[h] = encode8<T, kSr>(raw[i][h], sc, n[2 * h], n[2 * h + 1]);
        if (r < a.R && block_in) {
          uint8_t* dst = a.codes + r * a.ld_codes + (c >> 1);
          if constexpr (kH == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(code[0], code[kH - 1]);
          else *reinterpret_cast<uint32_t*>(dst) = code[0];
        }
        if ((8 * kH * t & 31) == 0) srow[(rl & 31) * 16 + (rl >> 5) * 4 + (8 * kH * t >> 5)] = static_cast<uint8_t>(sc);
      }
      if constexpr (kT) {
#pragma unroll
        for (int h = 0; h < kH; ++h) {
          if constexpr (kVec) {
            uint4* dst = reinterpret_cast<uint4*>(tile + rl * kMxTile + staged_col<sizeof(T)>(rl, 8 * (kH * t + h)));
            dst[0] = raw[i][h].w[0];
            if constexpr (sizeof(T) == 4) dst[1] = raw[i][h].w[1];
          }
          if constexpr (kSr)
            *reinterpret_cast<uint4*>(draws + rl * kMxTile + staged_col<2>(rl, 8 * (kH * t + h))) =
                make_uint4(n[2 * h].x, n[2 * h].y, n[2 * h + 1].x, n[2 * h + 1].y);
        }
      }
    }
  }
  if constexpr (kT) {
    __syncthreads();
    if (cols_out) {
      // a thread's part: two columns x 32 rows
      const int rb = lane & 3, pair = warp * 8 + (lane >> 2);
      const int64_t col = c0 + 2 * pair;
      constexpr int kHeld = sizeof(T) == 4 ? 1 : 32;
      const uint32_t* base = reinterpret_cast<const uint32_t*>(tile + rb * 32 * kMxTile + staged_col<sizeof(T)>(rb * 32, 2 * pair));
      const uint32_t* dbase = reinterpret_cast<const uint32_t*>(draws + rb * 32 * kMxTile + staged_col<2>(rb * 32, 2 * pair));
      uint32_t held[kHeld];   // 16-bit pairs stay in registers for the second pass
      uint32_t m0 = 0, m1 = 0;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        if constexpr (sizeof(T) == 4) {
          const uint2 w = *reinterpret_cast<const uint2*>(base + i * kMxTile);
          m0 = word_max<T>(m0, w.x);
          m1 = word_max<T>(m1, w.y);
        } else {
          held[i] = base[i * kMxTile / 2];
          m0 = word_max<T>(m0, held[i]);
        }
      }
      uint32_t s0, s1;
      if constexpr (sizeof(T) == 4) {
        s0 = scale_of_mx4(m0), s1 = scale_of_mx4(m1);
      } else {
        const float2 m = unpack2<T>(m0);
        s0 = scale_of_mx4(__float_as_uint(m.x)), s1 = scale_of_mx4(__float_as_uint(m.y));
      }
      bad |= s0 == kScaleNan || s1 == kScaleNan;
      const float i0 = scale_inverse(s0), i1 = scale_inverse(s1);
      uint32_t w0[4], w1[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float f0[8], f1[8];
        uint32_t b0[8], b1[8];   // the elements' bits: of fp32, or the pair of 16-bit ones in b0
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float2 v;
          if constexpr (sizeof(T) == 4) {
            v = *reinterpret_cast<const float2*>(base + (q * 8 + i) * kMxTile);
            b0[i] = __float_as_uint(v.x), b1[i] = __float_as_uint(v.y);
          } else {
            b0[i] = held[q * 8 + i];
            v = unpack2<T>(b0[i]);
          }
          f0[i] = __fmul_rn(v.x, i0);
          f1[i] = __fmul_rn(v.y, i1);
        }
        if constexpr (kSr) {
          uint32_t c0q[8], c1q[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t n = dbase[(q * 8 + i) * kMxTile / 2];
            c0q[i] = stochastic_code(f0[i], draw_lo(n));
            c1q[i] = stochastic_code(f1[i], draw_hi(n));
          }
          uint32_t e0, o0, e1, o1;   // signs of even and odd rows of each column
          if constexpr (sizeof(T) == 4) {
            e0 = top_bytes<true>(b0[0], b0[2], b0[4], b0[6]), o0 = top_bytes<true>(b0[1], b0[3], b0[5], b0[7]);
            e1 = top_bytes<true>(b1[0], b1[2], b1[4], b1[6]), o1 = top_bytes<true>(b1[1], b1[3], b1[5], b1[7]);
          } else {
            const uint32_t el = prmt(b0[0], b0[2], 0x7351), eh = prmt(b0[4], b0[6], 0x7351);
            const uint32_t ol = prmt(b0[1], b0[3], 0x7351), oh = prmt(b0[5], b0[7], 0x7351);
            e0 = prmt(el, eh, 0xDC98), e1 = prmt(el, eh, 0xFEBA);
            o0 = prmt(ol, oh, 0xDC98), o1 = prmt(ol, oh, 0xFEBA);
          }
          w0[q] = pack_codes8(c0q, e0, o0);
          w1[q] = pack_codes8(c1q, e1, o1);
        } else {
          w0[q] = codes8(f0);
          w1[q] = codes8(f1);
        }
        if (s0 == kScaleNan) w0[q] = 0u;
        if (s1 == kScaleNan) w1[q] = 0u;
      }
      const int64_t rblock = r0 + 32 * rb;
      if (rblock < a.R) {
        uint8_t* dst = a.codes_t + col * a.ld_codes_t + (rblock >> 1);
        if (col < a.C) *reinterpret_cast<uint4*>(dst) = make_uint4(w0[0], w0[1], w0[2], w0[3]);
        if (col + 1 < a.C)
          *reinterpret_cast<uint4*>(dst + a.ld_codes_t) = make_uint4(w1[0], w1[1], w1[2], w1[3]);
      }
      const int cl = 2 * pair;
      scol[(cl & 31) * 16 + (cl >> 5) * 4 + rb] = static_cast<uint8_t>(s0);
      scol[((cl + 1) & 31) * 16 + (cl >> 5) * 4 + rb] = static_cast<uint8_t>(s1);
    }
  }
  __syncthreads();
  if (tid < 32) {
    if (rows_out)
      reinterpret_cast<uint4*>(a.scales + (tr * a.ktiles + tc) * 512)[tid] = reinterpret_cast<uint4*>(srow)[tid];
    if (cols_out)
      reinterpret_cast<uint4*>(a.scales_t + (tc * a.ktiles_t + tr) * 512)[tid] = reinterpret_cast<uint4*>(scol)[tid];
  }
  if (bad) atomicOr(a.status, kDevNonFinite);
}

// Codes and scales back to values, kDeqRows rows in flight: eight elements per thread, tx threads along a
// row.
constexpr int kDeqRows = 4;

__device__ __forceinline__ int scale_in_tile(int64_t r) {   // of a row, block 0
  const int rl = static_cast<int>(r & 127);
  return (rl & 31) * 16 + (rl >> 5) * 4;
}

__device__ __forceinline__ void values_of_codes8(uint32_t w, float s, float (&f)[8]) {
  uint32_t p[4];
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(p[0]), "=r"(p[1]), "=r"(p[2]), "=r"(p[3])
      : "r"(w));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = unpack2<__half>(p[i]);
    f[2 * i] = v.x * s, f[2 * i + 1] = v.y * s;
  }
}

template <typename T>
__global__ void __launch_bounds__(256)
mx4_dequantize_kernel(const uint8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t R, int64_t C,
                      int64_t ktiles, T* out, int64_t ld) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) * 8;
  if (c >= C) return;
  const int64_t step = static_cast<int64_t>(gridDim.y) * blockDim.y;
  const uint8_t* sbase = scales + (c >> 7) * 512 + (c >> 5 & 3);
  for (int64_t r0 = static_cast<int64_t>(blockIdx.y) * blockDim.y + threadIdx.y; r0 < R; r0 += step * kDeqRows) {
    uint32_t w[kDeqRows], sc[kDeqRows];
#pragma unroll
    for (int k = 0; k < kDeqRows; ++k) {
      const int64_t r = r0 + k * step;
      if (r >= R) continue;
      w[k] = static_cast<uint32_t>(ld_here(reinterpret_cast<const int*>(codes + r * ld_codes + (c >> 1))));
      sc[k] = static_cast<uint32_t>(ld_here(sbase + (r >> 7) * ktiles * 512 + scale_in_tile(r)));
    }
#pragma unroll
    for (int k = 0; k < kDeqRows; ++k) {
      const int64_t r = r0 + k * step;
      if (r >= R) continue;
      float f[8];
      values_of_codes8(w[k], scale_value(sc[k]), f);
      T* o = out + r * ld + c;
      if (c + 8 <= C)
        store8(o, f);
      else
        store8_tail(o, f, static_cast<int>(C - c));
    }
  }
}

// a warp: the 256 elements from its first on, as codes of eight per lane; stored an element per lane
template <typename T>
__global__ void __launch_bounds__(256)
mx4_dequantize_dense_kernel(const uint8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t R, int64_t C,
                            int64_t ktiles, T* out, int64_t ld) {
  __shared__ __align__(16) T exchange[8][256];
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31;
  T* buf = exchange[(threadIdx.y * blockDim.x + threadIdx.x) >> 5];
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) * 8, seg = c - 8 * lane;
  const int64_t cc = c < C ? c : 0;   // codes are read of columns that exist
  const int64_t step = static_cast<int64_t>(gridDim.y) * blockDim.y;
  const uint8_t* sbase = scales + (cc >> 7) * 512 + (cc >> 5 & 3);
  for (int64_t r0 = static_cast<int64_t>(blockIdx.y) * blockDim.y + threadIdx.y; r0 < R; r0 += step * kDeqRows) {   // uniform over a warp
    uint32_t w[kDeqRows], sc[kDeqRows];
#pragma unroll
    for (int k = 0; k < kDeqRows; ++k) {
      const int64_t r = r0 + k * step;
      if (r >= R) continue;
      w[k] = static_cast<uint32_t>(ld_here(reinterpret_cast<const int*>(codes + r * ld_codes + (cc >> 1))));
      sc[k] = static_cast<uint32_t>(ld_here(sbase + (r >> 7) * ktiles * 512 + scale_in_tile(r)));
    }
#pragma unroll
    for (int k = 0; k < kDeqRows; ++k) {
      const int64_t r = r0 + k * step;
      if (r >= R) continue;
      float f[8];
      values_of_codes8(w[k], scale_value(sc[k]), f);
      dense_store(out + r * ld + seg, f, C - seg, buf, lane);
    }
  }
}

// ----------------------------------------------------------------------- host side
static int64_t scale_tiles(int64_t cols) { return (cols + 255) / 256 * 2; }   // along a row
int64_t mx4_scale_ktiles(int64_t cols) { return scale_tiles(cols); }

template <typename T, bool kSr, bool kT, bool kVec>
static int launch_quantize(const MxQuantArgs& a, dim3 grid, cudaStream_t s) {
  constexpr size_t smem = kMxTile * kMxTile * ((kT || !kVec ? sizeof(T) : 0) + (kT && kSr ? 2 : 0));
  static std::atomic<bool> done[64];
  if (smem > 48 * 1024) {
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return cuda_fail(err, "cudaGetDevice");
    if (dev < 0 || dev >= 64 || !done[dev].load(std::memory_order_acquire)) {
      err = cudaFuncSetAttribute(mx4_quantize_kernel<T, kSr, kT, kVec>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 static_cast<int>(smem));
      if (err != cudaSuccess) return cuda_fail(err, "cudaFuncSetAttribute");
      if (dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
    }
  }
  const cudaError_t err = launch_pdl_smem(mx4_quantize_kernel<T, kSr, kT, kVec>, grid, dim3(kMxThreads), smem, s, a);
  return err == cudaSuccess ? SQ_OK : cuda_fail(err, "mx4_quantize_kernel launch");
}

template <typename T, bool kVec>
static int launch_quantize_vec(const MxQuantArgs& a, bool sr, dim3 grid, cudaStream_t s) {
  if (a.codes_t != nullptr)
    return sr ? launch_quantize<T, true, true, kVec>(a, grid, s) : launch_quantize<T, false, true, kVec>(a, grid, s);
  return sr ? launch_quantize<T, true, false, kVec>(a, grid, s) : launch_quantize<T, false, false, kVec>(a, grid, s);
}
template <typename T>
static int launch_quantize_as(const MxQuantArgs& a, bool sr, bool vec, dim3 grid, cudaStream_t s) {
  return vec ? launch_quantize_vec<T, true>(a, sr, grid, s) : launch_quantize_vec<T, false>(a, sr, grid, s);
}

template <typename T>
static cudaError_t launch_dequantize(const uint8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t R, int64_t C,
                                     void* out, int64_t ld, cudaStream_t s) {
  const bool vec = aligned16(out) && (ld * static_cast<int64_t>(sizeof(T))) % 16 == 0;
  const int64_t per_row = (C + 7) / 8;
  unsigned tx = vec ? 8 : 32;   // whole warps of a row, or less than one
  while (tx < 32 && tx < per_row) tx *= 2;
  if (per_row > 32) tx = per_row < 256 ? static_cast<unsigned>((per_row + 31) / 32 * 32) : 256;
  const unsigned ty = 256 / tx;
  const int64_t gy = (R + ty * kDeqRows - 1) / (ty * kDeqRows);
  const dim3 grid(static_cast<unsigned>((per_row + tx - 1) / tx), static_cast<unsigned>(gy < 65535 ? gy : 65535));
  return launch_pdl(vec ? mx4_dequantize_kernel<T> : mx4_dequantize_dense_kernel<T>, grid, dim3(tx, ty), s, codes, ld_codes,
                    scales, R, C, scale_tiles(C), static_cast<T*>(out), ld);
}

}  // namespace sq

using namespace sq;

extern "C" size_t shiftquant_mx4_scale_bytes(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0) return 0;
  return static_cast<size_t>((rows + 127) / 128) * static_cast<size_t>(scale_tiles(cols)) * 512;
}

// rows and columns a quantizer's grid and 64-bit offsets take
static bool mx4_size_ok(int64_t n) { return n <= (int64_t(1) << 31) - 256; }

extern "C" sq_status shiftquant_mx4_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int mode,
                                             uint64_t seed, int64_t row0, uint8_t* codes, int64_t ld_codes,
                                             uint8_t* scales, uint8_t* codes_t, int64_t ld_codes_t, uint8_t* scales_t,
                                             int32_t* dev_status, void* stream) {
  fail(SQ_OK, "");
  if (!dtype_ok(dtype)) return fail(SQ_EINVAL, "mx4_quantize: bad dtype %d", dtype);
  if (mode != SQ_ROUND_NEAREST_EVEN && mode != SQ_ROUND_STOCHASTIC)
    return fail(SQ_EINVAL, "mx4_quantize: bad rounding mode %d", mode);
  if (rows < 0 || cols < 0 || row0 < 0) return fail(SQ_EINVAL, "mx4_quantize: negative size");
  if (rows == 0 || cols == 0) return SQ_OK;
  if (!mx4_size_ok(cols) || rows > int64_t(65534) * kMxTile)
    return fail(SQ_EUNSUPPORTED, "mx4_quantize: more than %lld rows or 2^31 - 256 columns", 65534ll * kMxTile);
  if (x == nullptr || dev_status == nullptr || ld < cols) return fail(SQ_EINVAL, "mx4_quantize: NULL argument or ld < cols");
  if ((codes == nullptr) != (scales == nullptr) || (codes_t == nullptr) != (scales_t == nullptr) ||
      (codes == nullptr && codes_t == nullptr))
    return fail(SQ_EINVAL, "mx4_quantize: codes and scales come in pairs, one pair at least");
  if (reinterpret_cast<uintptr_t>(x) % dtype_bytes(dtype)) return fail(SQ_EALIGN, "mx4_quantize: x is not aligned to its type");
  if (codes != nullptr) {
    if (ld_codes < (cols + 31) / 32 * 16) return fail(SQ_EINVAL, "mx4_quantize: ld_codes < 16 ceil(cols / 32)");
    if (!aligned16(codes) || !aligned16(scales) || ld_codes % 16) return fail(SQ_EALIGN, "mx4_quantize: codes, scales and ld_codes need 16-byte alignment");
  }
  if (codes_t != nullptr) {
    if (ld_codes_t < (rows + 31) / 32 * 16) return fail(SQ_EINVAL, "mx4_quantize: ld_codes_t < 16 ceil(rows / 32)");
    if (!aligned16(codes_t) || !aligned16(scales_t) || ld_codes_t % 16)
      return fail(SQ_EALIGN, "mx4_quantize: codes_t, scales_t and ld_codes_t need 16-byte alignment");
  }
  MxQuantArgs a;
  memset(&a, 0, sizeof(a));
  a.x = x, a.R = rows, a.C = cols, a.ld = ld, a.seed = seed, a.row0 = row0;
  a.codes = codes, a.ld_codes = ld_codes, a.scales = scales;
  a.codes_t = codes_t, a.ld_codes_t = ld_codes_t, a.scales_t = scales_t;
  a.ktiles = scale_tiles(cols), a.ktiles_t = scale_tiles(rows);
  a.status = dev_status;
  const bool vec = aligned16(x) && (ld * dtype_bytes(dtype)) % 16 == 0;
  // the scale tiles of a row come in pairs: the grid runs over the padding's too
  const dim3 grid(static_cast<unsigned>(codes != nullptr ? a.ktiles : (cols + 127) / 128),
                  static_cast<unsigned>(codes_t != nullptr ? a.ktiles_t : (rows + 127) / 128));
  const bool sr = mode == SQ_ROUND_STOCHASTIC;
  cudaStream_t s = as_stream(stream);
  if (dtype == SQ_F32) return launch_quantize_as<float>(a, sr, vec, grid, s);
  if (dtype == SQ_BF16) return launch_quantize_as<__nv_bfloat16>(a, sr, vec, grid, s);
  return launch_quantize_as<__half>(a, sr, vec, grid, s);
}

extern "C" sq_status shiftquant_mx4_dequantize(const uint8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t rows,
                                               int64_t cols, void* out, int dtype, int64_t ld, void* stream) {
  fail(SQ_OK, "");
  if (!dtype_ok(dtype)) return fail(SQ_EINVAL, "mx4_dequantize: bad dtype %d", dtype);
  if (rows < 0 || cols < 0) return fail(SQ_EINVAL, "mx4_dequantize: negative size");
  if (rows == 0 || cols == 0) return SQ_OK;
  if (!mx4_size_ok(cols)) return fail(SQ_EUNSUPPORTED, "mx4_dequantize: more than 2^31 - 256 columns");
  if (codes == nullptr || scales == nullptr || out == nullptr || ld < cols || ld_codes < (cols + 31) / 32 * 16)
    return fail(SQ_EINVAL, "mx4_dequantize: NULL argument or leading dimension too small");
  if (!aligned16(codes) || ld_codes % 16 || reinterpret_cast<uintptr_t>(out) % dtype_bytes(dtype))
    return fail(SQ_EALIGN, "mx4_dequantize: codes need 16-byte rows, out its type's alignment");
  cudaStream_t s = as_stream(stream);
  cudaError_t err;
  if (dtype == SQ_F32) err = launch_dequantize<float>(codes, ld_codes, scales, rows, cols, out, ld, s);
  else if (dtype == SQ_BF16) err = launch_dequantize<__nv_bfloat16>(codes, ld_codes, scales, rows, cols, out, ld, s);
  else err = launch_dequantize<__half>(codes, ld_codes, scales, rows, cols, out, ld, s);
  return err == cudaSuccess ? SQ_OK : cuda_fail(err, "mx4_dequantize_kernel launch");
}
