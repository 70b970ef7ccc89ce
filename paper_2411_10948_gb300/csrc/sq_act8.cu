// Activation functions whose input is kept in 8 bits for the backward pass.
//
// The input x is kept as int8 codes with a power-of-two scale per 32 elements of a row
// (x~ = q 2^e, |q| <= 127, |x - x~| <= 2^(e-1)); the forward output is of x itself, the backward
// pass evaluates its derivative at x~.  All arithmetic is FP32, rounded once on the way out.
//
//   y = f(x), dx = dy f'(x~), with f = x Phi(x) (GELU), its tanh form, or x sigmoid(x);
//   gated: x = [a | u], y = f(a) u, da = dy u~ f'(a~), du = dy f(a~)
//
// Streaming passes, bound by HBM: a thread takes eight consecutive elements (16-byte loads of
// 16-bit types, 8-byte stores of codes), four threads a scale block.  Where rows are not 16-byte
// aligned the accesses are an element per lane, and change hands in shared memory.  Measured at 16384 x 11008
// bf16: gated SiLU forward 236 us (6.2 TB/s), backward 231 us (6.4); SiLU 173 and 168 us (5.3 and 5.4); tanh
// GELU 178 and 174; GELU 208 and 195 us (4.4 and 4.7 TB/s), where no unit is full: issue slots 67% and 61%
// busy, DRAM 48% and 55%, at 44% and 32% of the warps an SM holds.  fp32 GELU of 5003 x 1155, unaligned,
// 21 us either way.
#include <cuda_runtime.h>

#include <cstring>

#include "sq_device.cuh"
#include "sq_block.cuh"
#include "sq_host.h"
#include "sq_saved8.cuh"

namespace sq {

// ------------------------------------------------------------------ activations
// 1 / x (0 for infinity) and 2^x, within two units
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float power2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// |x|, at most 1e30 (an infinity times a tail of 0 would be NaN); NaN stays
__device__ __forceinline__ float bounded_abs(float x) {
  float r;
  asm("{\n\t.reg .f32 a;\n\tabs.f32 a, %1;\n\tmin.NaN.f32 %0, a, 0f7149F2CA;\n\t}" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2e = 1.4426950409f;
// x^2 in the derivative of tanh GELU's argument, which meets f (1 - p) = 0 far out: x^2 is infinite from
// 1.8e19 on, and its product with 0 would be NaN (a NaN x reaches the result by f)
constexpr float kSquareMax = 1e30f;
constexpr float kHalfLog2eLow = -9.62981495e-09f;   // -1 / (2 ln 2) less its FP32 rounding
__device__ constexpr float kExp2[6] = {0.693147182f, 0.240226477f, 0.0555033237f, 0.00961843692f, 0.0013398875f, 0.00015353359f};
__device__ constexpr float kTail[9] = {0.139621302485466f,  0.13986355066299438f, 0.11982102692127228f,
                                       0.10555363446474075f, -0.023215219378471375f, 0.15932410955429077f,
                                       -0.25584304332733154f, 0.14403295516967773f, -0.029158318415284157f};
__device__ constexpr float kTail16[6] = {0.1201210618019104f,    0.11312702298164368f, 0.14712847769260406f,
                                         -0.023300522938370705f, 0.22233377397060394f, -0.07941005378961563f};

// The normal distribution's tail beyond |x| and exp(-x^2 / 2), to about FP32's precision (the tail
// within 10 units of 2^-24 of itself).  x^2 is kept in two parts, so that its rounding does not
// grow into the exponential; 2^f on [-1/2, 1/2] and the tail's factor tail / (t exp(-x^2 / 2)),
// t = 1 / (1 + 0.35 |x|), are polynomials of least relative error fitted on Chebyshev nodes in 64 bits
// (with their FP32 coefficients within 1.6e-8, and 5.9e-8 over |x| < 14.5).  CUDA's normcdff and expf took 157 instructions an element here.
__device__ __forceinline__ void normal_tail(float x, float& tail, float& g) {
  float y;
  asm("{\n\t.reg .f32 a;\n\tabs.f32 a, %1;\n\tmin.NaN.f32 %0, a, 0f41800000;\n\t}" : "=f"(y) : "f"(x));   // at most 16
  const float s = y * y, e = fmaf(y, y, -s);
  const float h = s * -0.72134752f;                                        // y^2 / -(2 ln 2), in two parts
  const float l = fmaf(e, -0.72134752f, fmaf(s, kHalfLog2eLow, fmaf(s, -0.72134752f, -h)));
  const float r = h + 12582912.0f;                                         // 1.5 2^23: the integer in the low bits
  const float f = (h - (r - 12582912.0f)) + l;
  float p = kExp2[5];
#pragma unroll
  for (int i = 4; i >= 0; --i) p = fmaf(p, f, kExp2[i]);
  p = fmaf(p, f, 1.0f);
  g = h < -125.0f ? 0.0f : __int_as_float(__float_as_int(p) + (__float_as_int(r) << 23));
  const float d = fmaf(0.35f, y, 1.0f);
  float t = reciprocal(d);
  t = fmaf(t, fmaf(-d, t, 1.0f), t);
  float q = kTail[8];
#pragma unroll
  for (int i = 7; i >= 0; --i) q = fmaf(q, t, kTail[i]);
  tail = t * g * q;
}

// f(x) and f'(x) in FP32: fp32 tensors.
template <int kAct>
__device__ __forceinline__ void activation_full(float x, float& f, float& df) {
  if constexpr (kAct == SQ_ACT_GELU) {
    float tail, g;
    normal_tail(x, tail, g);
    const float cdf = x < 0.0f ? tail : 1.0f - tail;
    f = x * cdf;
    df = fmaf(x, 0.3989422804f * g, cdf);
  } else {
    // x sigmoid(z): z = x, or 2 sqrt(2 / pi) (x + 0.044715 x^3), as (1 + tanh v) / 2 = sigmoid(2 v)
    float z = x, dz = 1.0f;
    if constexpr (kAct == SQ_ACT_GELU_TANH) {
      const float x2 = x * x;
      z = x * fmaf(0.0713548163f, x2, 1.5957691216f);
      dz = fmaf(0.2140644488f, fminf(x2, kSquareMax), 1.5957691216f);
    }
    const float p = 1.0f / (1.0f + expf(-z));
    f = x * p;
    df = fmaf(f * (1.0f - p), dz, p);
  }
}

// The same for 16-bit tensors, two values at a time, by the exponential and reciprocal units: within about
// 2^-16 of each term of the result (2^-21 but for GELU's tail and exponents far out), where half a unit of
// the types is 2^-9 and 2^-12.
template <int kAct, bool kDeriv>
__device__ __forceinline__ void activation_pair(float2 x, float2& f, float2& df) {
  const float2 one = make_float2(1.0f, 1.0f);
  if constexpr (kAct == SQ_ACT_GELU) {
    // the tail beyond |x| as t exp(-x^2 / 2) Q(t), t = 1 / (1 + 0.3 |x|), Q a polynomial fitted in 64 bits on
    // Chebyshev nodes of |x| < 13.2, beyond which the exponential is below FP32: within 1.3e-5 of the tail
    // itself (2.5e-7 at most), as the types hold the lower tail's outputs to all of their bits
    const float2 x2 = mul2(x, x);
    const float2 h = mul2(x2, make_float2(-0.5f * kLog2e, -0.5f * kLog2e));
    const float2 g = make_float2(power2(h.x), power2(h.y));
    const float2 ax = make_float2(bounded_abs(x.x), bounded_abs(x.y));
    const float2 d = fma2(ax, make_float2(0.3f, 0.3f), one);
    const float2 t = make_float2(reciprocal(d.x), reciprocal(d.y));
    float2 q = make_float2(kTail16[5], kTail16[5]);
#pragma unroll
    for (int i = 4; i >= 0; --i) q = fma2(t, q, make_float2(kTail16[i], kTail16[i]));
    const float2 tail = mul2(mul2(t, g), q);
    // x Phi(x) = max(x, 0) - |x| tail
    f = fma2(make_float2(-ax.x, -ax.y), tail, make_float2(fmaxf(x.x, 0.0f), fmaxf(x.y, 0.0f)));
    if constexpr (kDeriv) {
      // tail below 0, 1 - tail above (and 1/2 where the step is neither 0 nor 1); on the FP32 pipe
      const float2 step = make_float2(__saturatef(x.x * 1e38f), __saturatef(x.y * 1e38f));
      const float2 cdf = fma2(tail, fma2(step, make_float2(-2.0f, -2.0f), one), step);
      df = fma2(mul2(x, g), make_float2(0.3989422804f, 0.3989422804f), cdf);
    }
  } else {
    float2 z, dz = one;   // -z log2(e)
    if constexpr (kAct == SQ_ACT_GELU_TANH) {
      const float2 x2 = mul2(x, x);
      const float a = 1.5957691216f, b = 0.0713548163f;
      z = mul2(x, fma2(x2, make_float2(-b * kLog2e, -b * kLog2e), make_float2(-a * kLog2e, -a * kLog2e)));
      if constexpr (kDeriv)
        dz = fma2(make_float2(fminf(x2.x, kSquareMax), fminf(x2.y, kSquareMax)), make_float2(3.0f * b, 3.0f * b), make_float2(a, a));
    } else {
      z = mul2(x, make_float2(-kLog2e, -kLog2e));
    }
    const float2 e = add2(make_float2(power2(z.x), power2(z.y)), one);
    const float2 p = make_float2(reciprocal(e.x), reciprocal(e.y));
    f = mul2(x, p);
    if constexpr (kDeriv) {
      const float2 w = fma2(f, make_float2(-p.x, -p.y), f);   // f (1 - p)
      df = kAct == SQ_ACT_GELU_TANH ? fma2(w, dz, p) : add2(w, p);
    }
  }
}

// f (and f') of eight values
template <typename T, int kAct, bool kDeriv>
__device__ __forceinline__ void activation8(const float (&x)[8], float (&f)[8], float (&df)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      activation_full<kAct>(x[2 * i], f[2 * i], df[2 * i]);
      activation_full<kAct>(x[2 * i + 1], f[2 * i + 1], df[2 * i + 1]);
    } else {
      float2 a, b = make_float2(0.0f, 0.0f);
      activation_pair<kAct, kDeriv>(make_float2(x[2 * i], x[2 * i + 1]), a, b);
      f[2 * i] = a.x, f[2 * i + 1] = a.y, df[2 * i] = b.x, df[2 * i + 1] = b.y;
    }
  }
}

struct Act8Args {
  const void* in;      // h forward, dy backward
  int64_t ld_in;
  void* out;           // y forward, dh backward
  int64_t ld_out;
  int64_t R, C;        // C: columns of y
  int8_t* codes;
  int64_t ld_codes;
  uint8_t* scales;
  int64_t ld_scales;
  int32_t* status;
};

constexpr int kActRows = 2;   // rows a thread has in flight

// A block's threads: x along a row (whole warps where !kVec), y rows.
template <typename T, int kAct, bool kGated, bool kVec>
__global__ void __launch_bounds__(256, sizeof(T) == 4 ? 2 : (kVec ? 4 : 3)) act8_forward_kernel(const Act8Args a) {
  __shared__ __align__(16) T exchange[kVec ? 1 : 8][kVec ? 8 : 256];
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31;
  T* buf = exchange[kVec ? 0 : (threadIdx.y * blockDim.x + threadIdx.x) >> 5];
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) * 8;
  const int64_t cp = (a.C + 31) & ~int64_t(31), blocks = cp >> 5;
  const T* h = static_cast<const T*>(a.in);
  T* y = static_cast<T*>(a.out);
  bool bad = false;
  const int64_t step = static_cast<int64_t>(gridDim.y) * blockDim.y;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.y) * blockDim.y; r0 < a.R; r0 += step * kActRows) {   // uniform over the block
    RowIn<T, kVec> ia[kActRows], iu[kActRows];
#pragma unroll
    for (int k = 0; k < kActRows; ++k) {
      const int64_t r = r0 + k * step + threadIdx.y;
      ia[k].load(h + r * a.ld_in, c, a.C, r < a.R, lane);
      if constexpr (kGated) iu[k].load(h + r * a.ld_in + a.C, c, a.C, r < a.R, lane);
    }
#pragma unroll
    for (int k = 0; k < kActRows; ++k) {
      const int64_t r = r0 + k * step + threadIdx.y;
      const bool in = r < a.R;
      float x[8], u[8], o[8];
      ia[k].values(x, buf, lane);
      if constexpr (kGated) iu[k].values(u, buf, lane);
      if (a.codes != nullptr) {
        const uint32_t sx = block_scale8(x);
        bad |= sx == kScaleNan;
        if (in && c < a.C) {
          *reinterpret_cast<uint2*>(a.codes + r * a.ld_codes + c) = codes8_int8(x, sx);
          if ((threadIdx.x & 3) == 0) a.scales[r * a.ld_scales + (c >> 5)] = static_cast<uint8_t>(sx);
        }
        if constexpr (kGated) {
          const uint32_t su = block_scale8(u);
          bad |= su == kScaleNan;
          if (in && c < a.C) {
            *reinterpret_cast<uint2*>(a.codes + r * a.ld_codes + cp + c) = codes8_int8(u, su);
            if ((threadIdx.x & 3) == 0) a.scales[r * a.ld_scales + blocks + (c >> 5)] = static_cast<uint8_t>(su);
          }
        }
      }
      float df[8];
      activation8<T, kAct, false>(x, o, df);
      if constexpr (kGated) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] *= u[i];
      }
      row_store<T, kVec>(y + r * a.ld_out, o, c, a.C, in, buf, lane);
    }
  }
  if (bad) atomicOr(a.status, kDevNonFinite);
}

// A thread's row in the backward pass on its way.
template <typename T, bool kGated, bool kVec>
struct ActBack {
  RowIn<T, kVec> dy;
  uint2 qa, qu;
  uint32_t sa, su;
};

// One wave of blocks walks the rows, kActRows of a thread's rows always on their way.
template <typename T, int kAct, bool kGated, bool kVec>
__global__ void __launch_bounds__(256, sizeof(T) == 4 ? 2 : 3) act8_backward_kernel(const Act8Args a) {
  __shared__ __align__(16) T exchange[kVec ? 1 : 8][kVec ? 8 : 256];
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31;
  T* buf = exchange[kVec ? 0 : (threadIdx.y * blockDim.x + threadIdx.x) >> 5];
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) * 8;
  if (kVec && c >= a.C) return;
  const int64_t cp = (a.C + 31) & ~int64_t(31), blocks = cp >> 5;
  const int64_t cc = c < a.C ? c : 0;   // codes are read of columns that exist
  const T* dy = static_cast<const T*>(a.in);
  T* dh = static_cast<T*>(a.out);
  const int64_t step = static_cast<int64_t>(gridDim.y) * blockDim.y;
  const int8_t* codes = a.codes + cc;
  const uint8_t* scales = a.scales + (cc >> 5);
  ActBack<T, kGated, kVec> n[kActRows];
  auto fetch = [&](ActBack<T, kGated, kVec>& b, int64_t r) {   // r: uniform over a warp
    if (r >= a.R) return;
    b.dy.load(dy + r * a.ld_in, c, a.C, true, lane);
    b.qa = ld_codes8(codes + r * a.ld_codes);
    b.sa = ld_scale(scales + r * a.ld_scales);
    if constexpr (kGated) {
      b.qu = ld_codes8(codes + r * a.ld_codes + cp);
      b.su = ld_scale(scales + r * a.ld_scales + blocks);
    }
  };
  int64_t r = static_cast<int64_t>(blockIdx.y) * blockDim.y + threadIdx.y;
#pragma unroll
  for (int k = 0; k < kActRows; ++k) fetch(n[k], r + k * step);
  while (r < a.R) {
#pragma unroll
    for (int k = 0; k < kActRows; ++k, r += step) {
      if (r >= a.R) break;
      float g[8], x[8], u[8], f[8], df[8], da[8], du[8];
      n[k].dy.values(g, buf, lane);
      decode8(n[k].qa, n[k].sa, x);
      if constexpr (kGated) decode8(n[k].qu, n[k].su, u);
      fetch(n[k], r + kActRows * step);
      activation8<T, kAct, true>(x, f, df);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        da[i] = kGated ? g[i] * u[i] * df[i] : g[i] * df[i];
        if constexpr (kGated) du[i] = g[i] * f[i];
      }
      row_store<T, kVec>(dh + r * a.ld_out, da, c, a.C, true, buf, lane);
      if constexpr (kGated) row_store<T, kVec>(dh + r * a.ld_out + a.C, du, c, a.C, true, buf, lane);
    }
  }
}

// ----------------------------------------------------------------------- host side
template <typename T, int kAct, bool kGated, bool kVec>
static cudaError_t launch_act_vec(const Act8Args& a, bool forward, cudaStream_t s) {
  const int64_t threads = (a.C + 31) / 32 * 4;   // of a row: whole scale blocks
  // x threads: whole warps of a row, or less than one
  unsigned tx = kVec ? 8 : 32;
  while (tx < 32 && tx < threads) tx *= 2;
  if (threads > 32) tx = threads < 256 ? static_cast<unsigned>((threads + 31) / 32 * 32) : 256;
  const unsigned ty = 256 / tx;
  const int64_t gx = (threads + tx - 1) / tx;
  int64_t gy = (a.R + kActRows * ty - 1) / (kActRows * ty);
  if (!forward) {
    // one wave: what the SMs hold at once
    const int sms = device_sms(nullptr);
    const int64_t wave = (sms > 0 ? sms : 1) * int64_t((sizeof(T) == 4 ? 512 : 768) / (tx * ty)) / gx;
    if (gy > wave) gy = wave > 0 ? wave : 1;
  }
  const dim3 grid(static_cast<unsigned>(gx), static_cast<unsigned>(gy < 65535 ? gy : 65535)), block(tx, ty);
  return forward ? launch_pdl(act8_forward_kernel<T, kAct, kGated, kVec>, grid, block, s, a)
                 : launch_pdl(act8_backward_kernel<T, kAct, kGated, kVec>, grid, block, s, a);
}
template <typename T, int kAct, bool kGated>
static cudaError_t launch_act(const Act8Args& a, bool forward, cudaStream_t s) {
  const bool vec = rows16<T>(a.in, a.ld_in) && rows16<T>(a.out, a.ld_out) &&
                   (!kGated || (a.C * static_cast<int64_t>(sizeof(T))) % 16 == 0);
  return vec ? launch_act_vec<T, kAct, kGated, true>(a, forward, s) : launch_act_vec<T, kAct, kGated, false>(a, forward, s);
}

template <typename T, bool kGated>
static cudaError_t launch_act_as(const Act8Args& a, int act, bool forward, cudaStream_t s) {
  if (act == SQ_ACT_GELU) return launch_act<T, SQ_ACT_GELU, kGated>(a, forward, s);
  if (act == SQ_ACT_GELU_TANH) return launch_act<T, SQ_ACT_GELU_TANH, kGated>(a, forward, s);
  return launch_act<T, SQ_ACT_SILU, kGated>(a, forward, s);
}

static int run_act(const Act8Args& a, int dtype, int act, int gated, bool forward, void* stream) {
  cudaStream_t s = as_stream(stream);
  cudaError_t err;
  if (dtype == SQ_F32) err = gated ? launch_act_as<float, true>(a, act, forward, s) : launch_act_as<float, false>(a, act, forward, s);
  else if (dtype == SQ_BF16) err = gated ? launch_act_as<__nv_bfloat16, true>(a, act, forward, s) : launch_act_as<__nv_bfloat16, false>(a, act, forward, s);
  else err = gated ? launch_act_as<__half, true>(a, act, forward, s) : launch_act_as<__half, false>(a, act, forward, s);
  return err == cudaSuccess ? SQ_OK : cuda_fail(err, "act8 kernel launch");
}

static int check_act(const char* who, int dtype, int64_t rows, int64_t cols, int act, int gated, const void* in, int64_t ld_in,
                     int64_t in_cols, const void* out, int64_t ld_out, int64_t out_cols, const int8_t* codes, int64_t ld_codes,
                     const uint8_t* scales, int64_t ld_scales) {
  constexpr int64_t kMax = (int64_t(1) << 30);
  if (rows > kMax || cols > kMax) return fail(SQ_EUNSUPPORTED, "%s: more than 2^30 rows or columns", who);
  if (in == nullptr || out == nullptr || ld_in < in_cols || ld_out < out_cols)
    return fail(SQ_EINVAL, "%s: NULL argument or leading dimension too small", who);
  if (reinterpret_cast<uintptr_t>(in) % dtype_bytes(dtype) || reinterpret_cast<uintptr_t>(out) % dtype_bytes(dtype))
    return fail(SQ_EALIGN, "%s: a tensor is not aligned to its type", who);
  if (codes == nullptr) return SQ_OK;
  const int64_t blocks = (cols + 31) / 32 * (gated ? 2 : 1);
  if (ld_codes < 32 * blocks || ld_scales < blocks) return fail(SQ_EINVAL, "%s: ld_codes or ld_scales too small", who);
  if (!aligned16(codes) || ld_codes % 16) return fail(SQ_EALIGN, "%s: codes and ld_codes need 16-byte alignment", who);
  return SQ_OK;
}

}  // namespace sq

using namespace sq;

static bool act_ok(int act) { return act == SQ_ACT_GELU || act == SQ_ACT_GELU_TANH || act == SQ_ACT_SILU; }

extern "C" sq_status shiftquant_act8_forward(const void* h, int dtype, int64_t rows, int64_t cols, int64_t ld_h, int act,
                                             int gated, void* y, int64_t ld_y, int8_t* codes, int64_t ld_codes,
                                             uint8_t* scales, int64_t ld_scales, int32_t* dev_status, void* stream) {
  fail(SQ_OK, "");
  if (!dtype_ok(dtype) || !act_ok(act)) return fail(SQ_EINVAL, "act8_forward: bad dtype or activation");
  if (rows < 0 || cols < 0) return fail(SQ_EINVAL, "act8_forward: negative size");
  if (rows == 0 || cols == 0) return SQ_OK;
  if ((codes == nullptr) != (scales == nullptr) || dev_status == nullptr)
    return fail(SQ_EINVAL, "act8_forward: codes and scales come together, dev_status is required");
  const int st = check_act("act8_forward", dtype, rows, cols, act, gated, h, ld_h, gated ? 2 * cols : cols, y, ld_y, cols, codes,
                           ld_codes, scales, ld_scales);
  if (st != SQ_OK) return st;
  const Act8Args a = {h, ld_h, y, ld_y, rows, cols, codes, ld_codes, scales, ld_scales, dev_status};
  return run_act(a, dtype, act, gated, true, stream);
}

extern "C" sq_status shiftquant_act8_backward(const void* dy, int dtype, int64_t rows, int64_t cols, int64_t ld_dy,
                                              const int8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t ld_scales,
                                              int act, int gated, void* dh, int64_t ld_dh, void* stream) {
  fail(SQ_OK, "");
  if (!dtype_ok(dtype) || !act_ok(act)) return fail(SQ_EINVAL, "act8_backward: bad dtype or activation");
  if (rows < 0 || cols < 0) return fail(SQ_EINVAL, "act8_backward: negative size");
  if (rows == 0 || cols == 0) return SQ_OK;
  if (codes == nullptr || scales == nullptr) return fail(SQ_EINVAL, "act8_backward: NULL codes or scales");
  const int st = check_act("act8_backward", dtype, rows, cols, act, gated, dy, ld_dy, cols, dh, ld_dh, gated ? 2 * cols : cols,
                           codes, ld_codes, scales, ld_scales);
  if (st != SQ_OK) return st;
  const Act8Args a = {dy, ld_dy, dh, ld_dh, rows, cols, const_cast<int8_t*>(codes), ld_codes, const_cast<uint8_t*>(scales),
                      ld_scales, nullptr};
  return run_act(a, dtype, act, gated, false, stream);
}
