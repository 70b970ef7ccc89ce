// Layer and root-mean-square norms whose input is kept in 8 bits for the backward pass.
//
//   s = x + residual (rounded to the type), y = (s - mu) rstd gamma + beta, and with
//   xh = (s~ - mu) rstd, t = dy gamma:
//   dx = rstd (t - mean(t) - xh mean(t xh)) (+ the residual's gradient), mu and mean(t) being 0 for
//   the root-mean-square norm; dgamma = sum dy xh, dbeta = sum dy over rows
//
// s is kept as int8 codes with a power-of-two scale per 32 elements of a row (s~ = q 2^e), its
// statistics in FP32, as is all arithmetic, rounded once on the way out.  The variance is that
// about the mean: a second sweep over registers.
#include <cuda_runtime.h>

#include <atomic>
#include <cstring>

#include "sq_device.cuh"
#include "sq_block.cuh"
#include "sq_host.h"
#include "sq_saved8.cuh"

namespace sq {

// ---------------------------------------------------------------- normalizations
struct Norm8Args {
  const void* x;        // forward: x; backward: dy
  int64_t ld_x;
  const void* res;      // forward: the residual to add; backward: its gradient to add (or null)
  int64_t ld_res;
  void* out;            // y; dx
  int64_t ld_out;
  void* sum;            // forward: x + residual
  int64_t ld_sum;
  int64_t R, C;
  const float* gamma;
  const float* beta;
  float eps;
  int8_t* codes;
  int64_t ld_codes;
  uint8_t* scales;
  int64_t ld_scales;
  float* stats;         // [R][2]: mean, 1 / deviation
  float* part;          // backward: [groups][2 C] partial sums of dgamma, dbeta
  int32_t* status;
};

// The first column of the eight of chunk k that thread t of G holds.
__device__ __forceinline__ int64_t norm_col(int k, int t, int G) { return (static_cast<int64_t>(k) * G + t) * 8; }

// parameters of eight columns (0 past C); kVec: p is 16-byte aligned, else that is looked at here (it mostly
// is where the rows are not)
template <bool kVec>
__device__ __forceinline__ void norm_param(float (&f)[8], const float* p, int64_t c, int64_t C) {
  if ((kVec || (reinterpret_cast<uintptr_t>(p) & 15u) == 0) && c + 8 <= C) {
    const uint4 a = ld_here(reinterpret_cast<const uint4*>(p + c)), b = ld_here(reinterpret_cast<const uint4*>(p + c) + 1);
    f[0] = __uint_as_float(a.x), f[1] = __uint_as_float(a.y), f[2] = __uint_as_float(a.z), f[3] = __uint_as_float(a.w);
    f[4] = __uint_as_float(b.x), f[5] = __uint_as_float(b.y), f[6] = __uint_as_float(b.z), f[7] = __uint_as_float(b.w);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = c + i < C ? ld_here(p + c + i) : 0.0f;
}

// codes and scales of eight elements; true where their block is not finite
__device__ __forceinline__ bool norm_keep(const Norm8Args& a, const float (&f)[8], int64_t r, int64_t c) {
  const uint32_t s = block_scale8(f);
  if (c >= a.C) return false;
  *reinterpret_cast<uint2*>(a.codes + r * a.ld_codes + c) = codes8_int8(f, s);
  if ((c & 31) == 0) a.scales[r * a.ld_scales + (c >> 5)] = static_cast<uint8_t>(s);
  return s == kScaleNan;
}

// eight kept values (0 past C)
__device__ __forceinline__ void norm_kept(const Norm8Args& a, float (&f)[8], int64_t r, int64_t c) {
  if (c >= a.C) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.0f;
    return;
  }
  decode8(ld_codes8(a.codes + r * a.ld_codes + c), ld_scale(a.scales + r * a.ld_scales + (c >> 5)), f);
  if (c + 8 <= a.C) return;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i >= a.C) f[i] = 0.0f;
}

// Sums over the threads of a row of v.x, and where kTwo of v.y: a warp's by shuffles, those of several
// warps (kBlock; blockDim.x threads) through red, the row's own (alternating halves, so one barrier a call),
// in the same order whatever the load.
constexpr int kRowsPerBlock = 8;   // at most
template <bool kTwo>
struct RowRed {
  float4 part[kRowsPerBlock][2][kTwo ? 8 : 4];
};
// kMany: the block may hold several rows of several warps (a barrier each, which keeps all 16 of the block's).
template <bool kBlock, bool kTwo, bool kMany>
__device__ __forceinline__ float2 row_sum(float2 v, RowRed<kTwo>& all, int& half) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
    if constexpr (kTwo) v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
  }
  if constexpr (kBlock) {
    float4* red = all.part[threadIdx.y][half];
    const int warps = blockDim.x >> 5, w = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) {
      if constexpr (kTwo) reinterpret_cast<float2*>(red)[w] = v;
      else reinterpret_cast<float*>(red)[w] = v.x;
    }
    if (!kMany || blockDim.y == 1) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(threadIdx.y + 1), "r"(blockDim.x) : "memory");   // the row's threads
    v = make_float2(0.0f, 0.0f);
    constexpr int kPer = kTwo ? 2 : 4;   // warps per 16 bytes
    for (int i = 0; i < warps; i += kPer) {   // what lies past the last warp's part counts as 0
      const float4 q = red[i / kPer];
      if constexpr (kTwo) {
        v.x += q.x + (i + 1 < warps ? q.z : 0.0f);
        v.y += q.y + (i + 1 < warps ? q.w : 0.0f);
      } else {
        v.x += (q.x + (i + 1 < warps ? q.y : 0.0f)) + ((i + 2 < warps ? q.z : 0.0f) + (i + 3 < warps ? q.w : 0.0f));
      }
    }
    half ^= 1;
  }
  return v;
}
// A row per group of G threads: a warp (kBlock false) or several, blockDim.y groups per block.
// kChunks chunks of 8 elements stay in registers; kChunks = 0: rows beyond them, read again for
// each of the three sweeps.  Bound by HBM (16384 x 4096 bf16 with a residual 90 us, 6.7 TB/s; fp32
// 7.0 TB/s; 100000 x 768 bf16 layer norm 113 us, 6.1 TB/s), by the latency of a block's life where rows are
// fewer (12608 x 768 20.5 us, 4.3 TB/s).  Sums, squares and outputs go two elements per instruction, and the
// rounded sum is stored as it is read back: element by element these took 92, 148 and 25 us.  (One wave of blocks that walk the rows, the next row on its way: 64 registers spill, more
// leave too few warps; 16384 x 4096 bf16 99 us.)  Three blocks per SM are asked for in 16-bit RMS norms of
// two chunks a thread: 16384 x 8192 bf16 181 us for 202, x 4096 89 for 90; layer norms take the same time
// with a bound and without.  Beyond 16384 columns: 4096 x 20000 bf16 RMS with a residual 154 us, fp32
// layer 256 us (4.8 and 5.4 TB/s of what they have to move).
template <typename T, int kChunks, bool kVec, bool kBlock, bool kLayer>
__global__ void __launch_bounds__(512, kVec && kBlock && kChunks == 2 && sizeof(T) == 2 && !kLayer ? 3 : 1) norm8_forward_kernel(const Norm8Args a) {
  __shared__ RowRed<false> red;
  __shared__ __align__(16) T exchange[kVec ? 1 : 16][kVec ? 8 : 256];
  int half = 0;
  griddep_wait();
  griddep_launch_dependents();
  const int G = kBlock ? blockDim.x : 32, t = threadIdx.x, lane = t & 31;
  T* buf = exchange[kVec ? 0 : (threadIdx.y * blockDim.x + t) >> 5];
  const int64_t r = static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y;
  if (r >= a.R) return;   // a whole group
  const T* x = static_cast<const T*>(a.x) + r * a.ld_x;
  const T* res = a.res == nullptr ? nullptr : static_cast<const T*>(a.res) + r * a.ld_res;
  T* sum = a.res == nullptr ? nullptr : static_cast<T*>(a.sum) + r * a.ld_sum;
  T* y = static_cast<T*>(a.out) + r * a.ld_out;
  const int chunks = kChunks > 0 ? kChunks : static_cast<int>((a.C + 8 * G - 1) / (8 * G));
  const float inv_c = 1.0f / static_cast<float>(a.C);
  float v[kChunks > 0 ? kChunks : 1][8];
  auto add = [&](RowIn<T, kVec>& in, float (&f)[8], int64_t c) {   // s = x + residual, rounded to the type
    float g[8];
    in.values(g, buf, lane);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] += g[i];
    Raw8<T> w;
    round8(w, f);
    values8<T>(w, f);
    if (kVec && c + 8 <= a.C) store8(sum + c, w);
    else row_store<T, kVec>(sum, f, c, a.C, true, buf, lane);
  };
  // s of a chunk; after the first sweep the sum is read back (each thread its own elements), as it may have
  // taken the residual's place
  auto fetch = [&](int k, float (&f)[8], bool first) {
    RowIn<T, kVec> in, rr;
    const int64_t c = norm_col(k, t, G);
    const bool adds = res != nullptr && first;
    in.load(res != nullptr && !first ? sum : x, c, a.C, true, lane);
    if (adds) rr.load(res, c, a.C, true, lane);
    in.values(f, buf, lane);
    if (adds) add(rr, f, c);
  };
  float2 acc = make_float2(0.0f, 0.0f);
  if constexpr (kChunks > 0) {
    RowIn<T, kVec> in[kChunks], rr[kChunks];
#pragma unroll
    for (int k = 0; k < kChunks; ++k) in[k].load(x, norm_col(k, t, G), a.C, true, lane);
    if (res != nullptr) {
#pragma unroll
      for (int k = 0; k < kChunks; ++k) rr[k].load(res, norm_col(k, t, G), a.C, true, lane);
    }
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      in[k].values(v[k], buf, lane);
      if (res != nullptr) add(rr[k], v[k], norm_col(k, t, G));
    }
  }
  auto chunk = [&](int k, float (&f)[8], bool first) {
    if constexpr (kChunks > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = v[k][i];
    } else {
      fetch(k, f, first);
    }
  };
  auto pair = [](const float (&f)[8], int i) { return make_float2(f[2 * i], f[2 * i + 1]); };
  // the statistics: the mean first, then the squares about it
#pragma unroll
  for (int k = 0; k < chunks; ++k) {
    float f[8];
    chunk(k, f, true);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = kLayer ? add2(acc, pair(f, i)) : fma2(pair(f, i), pair(f, i), acc);
  }
  float mu = 0.0f;
  acc.x += acc.y;
  acc = row_sum<kBlock, false, false>(acc, red, half);
  if constexpr (kLayer) {
    mu = acc.x * inv_c;
    acc = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < chunks; ++k) {
      float f[8];
      chunk(k, f, false);
      const int64_t c = norm_col(k, t, G);
      if (c + 8 > a.C) {   // what lies past the row counts for nothing
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i >= a.C) f[i] = mu;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 d = add2(pair(f, i), make_float2(-mu, -mu));
        acc = fma2(d, d, acc);
      }
    }
    acc.x += acc.y;
    acc = row_sum<kBlock, false, false>(acc, red, half);
  }
  const float rstd = 1.0f / sqrtf(acc.x * inv_c + a.eps);
  if (a.stats != nullptr && t == 0) reinterpret_cast<float2*>(a.stats)[r] = make_float2(mu, rstd);
  bool bad = false;
#pragma unroll
  for (int k = 0; k < chunks; ++k) {
    float f[8], g[8], b[8], o[8];
    chunk(k, f, false);
    const int64_t c = norm_col(k, t, G);
    norm_param<kVec>(g, a.gamma, c, a.C);
    if constexpr (kLayer) norm_param<kVec>(b, a.beta, c, a.C);
    if (a.codes != nullptr) bad |= norm_keep(a, f, r, c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 r2 = make_float2(rstd, rstd);
      const float2 q = kLayer ? fma2(mul2(add2(pair(f, i), make_float2(-mu, -mu)), r2), pair(g, i), pair(b, i))
                              : mul2(mul2(pair(f, i), r2), pair(g, i));
      o[2 * i] = q.x, o[2 * i + 1] = q.y;
    }
    row_store<T, kVec>(y, o, c, a.C, true, buf, lane);
  }
  if (bad) atomicOr(a.status, kDevNonFinite);
}

// The backward pass of rows that norm8_backward_ring_kernel does not take (any alignment, or longer).
// Rows group by group; the column sums of dgamma and dbeta stay in a thread's registers (in its
// group's row of the workspace for kChunks = 0) until the group's rows are done.  Beyond two chunks the
// sums leave no room for the row, which is read twice.  Bound by the instructions of element-wise accesses
// (5003 x 1155 fp32 35 us for 42 with scalar arithmetic and parameters, 12608 x 767 bf16 48 for 57); for
// kChunks = 0 by the column sums' way through the workspace, two reads and writes per element (4096 x 20000 bf16 RMS
// 864 us, fp32 layer norm 913).
template <typename T, int kChunks, bool kVec, bool kBlock, bool kLayer>
__global__ void __launch_bounds__(512) norm8_backward_kernel(const Norm8Args a) {
  __shared__ RowRed<kLayer> red;
  __shared__ __align__(16) T exchange[kVec ? 1 : 16][kVec ? 8 : 256];
  int half = 0;
  griddep_wait();
  griddep_launch_dependents();
  auto pair = [](const float (&f)[8], int i) { return make_float2(f[i], f[i + 1]); };
  auto put = [](float (&f)[8], int i, float2 v) { f[i] = v.x, f[i + 1] = v.y; };
  const int G = kBlock ? blockDim.x : 32, t = threadIdx.x, lane = t & 31;
  T* buf = exchange[kVec ? 0 : (threadIdx.y * blockDim.x + t) >> 5];
  const int64_t group = static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y;
  const int64_t groups = static_cast<int64_t>(gridDim.x) * blockDim.y;
  const int chunks = kChunks > 0 ? kChunks : static_cast<int>((a.C + 8 * G - 1) / (8 * G));
  const float inv_c = 1.0f / static_cast<float>(a.C);
  float* part = a.part + group * 2 * a.C;
  constexpr int kSums = kChunks > 0 ? kChunks : 1;
  constexpr bool kTwice = kChunks == 0 || kChunks > 2;   // rows are read again for the second sweep
  constexpr int kHeld = kTwice ? 1 : kChunks;
  float dg[kSums][8], db[kSums][8];
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[k][i] = db[k][i] = 0.0f;
  if constexpr (kChunks == 0) {
    for (int k = 0; k < chunks; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t c = norm_col(k, t, G) + i;
        if (c < a.C) part[c] = part[a.C + c] = 0.0f;
      }
  }
  for (int64_t r = group; r < a.R; r += groups) {   // uniform over the group
    const T* dy = static_cast<const T*>(a.x) + r * a.ld_x;
    const T* ds = a.res == nullptr ? nullptr : static_cast<const T*>(a.res) + r * a.ld_res;
    T* dx = static_cast<T*>(a.out) + r * a.ld_out;
    const float2 st = make_float2(ld_here(a.stats + 2 * r), ld_here(a.stats + 2 * r + 1));
    float tv[kHeld][8], xh[kHeld][8];
    RowIn<T, kVec> in[kHeld], rs[kHeld];
    auto fetch = [&](int k, int h) {
      const int64_t c = norm_col(k, t, G);
      in[h].load(dy, c, a.C, true, lane);
      norm_kept(a, xh[h], r, c);
    };
    float2 sum_tx = make_float2(0.0f, 0.0f), sum_t = sum_tx;
    if constexpr (!kTwice) {
#pragma unroll
      for (int k = 0; k < kChunks; ++k) fetch(k, k);
      if (ds != nullptr) {
#pragma unroll
        for (int k = 0; k < kChunks; ++k) rs[k].load(ds, norm_col(k, t, G), a.C, true, lane);
      }
    }
#pragma unroll
    for (int k = 0; k < chunks; ++k) {
      const int h = kTwice ? 0 : k;
      if constexpr (kTwice) fetch(k, 0);
      in[h].values(tv[h], buf, lane);
      const int64_t c = norm_col(k, t, G);
      float g[8];
      norm_param<kVec>(g, a.gamma, c, a.C);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float2 x = mul2(add2(pair(xh[h], i), make_float2(-st.x, -st.x)), make_float2(st.y, st.y));
        const float2 d = pair(tv[h], i);
        if constexpr (kChunks > 0) {
          put(dg[k], i, fma2(d, x, pair(dg[k], i)));
          if (kLayer) put(db[k], i, add2(d, pair(db[k], i)));
        } else {
#pragma unroll
          for (int j = i; j < i + 2; ++j)
            if (c + j < a.C) {
              part[c + j] = fmaf(j == i ? d.x : d.y, j == i ? x.x : x.y, part[c + j]);
              part[a.C + c + j] += j == i ? d.x : d.y;
            }
        }
        const float2 tg = mul2(d, pair(g, i));   // 0 past C
        put(xh[h], i, x);
        put(tv[h], i, tg);
        sum_tx = fma2(tg, x, sum_tx);
        if (kLayer) sum_t = add2(tg, sum_t);
      }
    }
    float2 acc = make_float2(sum_tx.x + sum_tx.y, sum_t.x + sum_t.y);
    acc = row_sum<kBlock, kLayer, true>(acc, red, half);
    const float mx = acc.x * inv_c, mt = kLayer ? acc.y * inv_c : 0.0f;
#pragma unroll
    for (int k = 0; k < chunks; ++k) {
      const int h = kTwice ? 0 : k;
      const int64_t c = norm_col(k, t, G);
      if constexpr (kTwice) {
        float g[8];
        fetch(k, 0);
        norm_param<kVec>(g, a.gamma, c, a.C);
        if (ds != nullptr) rs[0].load(ds, c, a.C, true, lane);
        in[0].values(tv[0], buf, lane);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          put(xh[0], i, mul2(add2(pair(xh[0], i), make_float2(-st.x, -st.x)), make_float2(st.y, st.y)));
          put(tv[0], i, mul2(pair(tv[0], i), pair(g, i)));
        }
      }
      float o[8], s[8];
      if (ds != nullptr) rs[h].values(s, buf, lane);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float2 in_row = fma2(pair(xh[h], i), make_float2(-mx, -mx), add2(pair(tv[h], i), make_float2(-mt, -mt)));
        const float2 r2 = make_float2(st.y, st.y);
        put(o, i, ds != nullptr ? fma2(r2, in_row, pair(s, i)) : mul2(r2, in_row));
      }
      row_store<T, kVec>(dx, o, c, a.C, true, buf, lane);
    }
  }
  if constexpr (kChunks > 0) {
#pragma unroll
    for (int k = 0; k < kChunks; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t c = norm_col(k, t, G) + i;
        if (c < a.C) {
          part[c] = dg[k][i];
          if (kLayer) part[a.C + c] = db[k][i];
        }
      }
  }
}

// The backward pass of aligned rows of up to 8 kChunks elements per thread.  A group takes rows
// group, group + groups, ..; kRing - 1 of them are on their way through the thread's own part of
// shared memory (cp.async; no barrier, as a thread reads what it copied itself), gamma and the
// column sums stay in registers.  FP32 arithmetic goes two elements per instruction.  With four chunks
// (kLean) the sums alone fill the registers: gamma is read, and t and xh formed, once per sweep.
// Bound by the instructions of a row at 16 warps per SM (16384 x 4096 bf16 with dsum 93 us, 5.1 TB/s;
// 124 us with scales and statistics loaded a row ahead by plain loads).  80 registers and 768 threads per SM
// spill: 140 us for 117 then.
template <typename T, int kChunks>   // rows in shared memory: what 512 threads leave room for
constexpr int kRing = kChunks == 3 ? (sizeof(T) == 4 ? 1 : 3) : kChunks > 2 ? (sizeof(T) == 4 ? 1 : 2) : (sizeof(T) == 4 ? 2 : 4);
template <typename T>
constexpr int kRingBytes = 8 * (2 * static_cast<int>(sizeof(T)) + 1) + 4;   // dy, dsum, codes and scale of a chunk

template <typename T, int kChunks, bool kBlock, bool kLayer>
__global__ void __launch_bounds__(512) norm8_backward_ring_kernel(const Norm8Args a) {
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ RowRed<kLayer> red;
  constexpr int D = kRing<T, kChunks>;
  constexpr int kQuads = sizeof(T) / 2;   // 16-byte words of a chunk's elements
  int half = 0;
  griddep_wait();
  griddep_launch_dependents();
  const int G = kBlock ? blockDim.x : 32, t = threadIdx.x;
  const int threads = blockDim.x * blockDim.y, tid = threadIdx.y * blockDim.x + t;
  const int64_t group = static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y;
  const int64_t groups = static_cast<int64_t>(gridDim.x) * blockDim.y;
  const float inv_c = 1.0f / static_cast<float>(a.C);
  const T* dy = static_cast<const T*>(a.x);
  const T* ds = static_cast<const T*>(a.res);
  const uint32_t base = smem_u32(ring);
  // slot (stage d, word w of kChunks (2 kQuads) 16-byte words) of this thread, then the codes
  const uint32_t codes0 = base + static_cast<uint32_t>(D * kChunks * 2 * kQuads * threads) * 16;
  auto slot = [&](int d, int w) { return base + static_cast<uint32_t>((d * kChunks * 2 * kQuads + w) * threads + tid) * 16; };
  auto cslot = [&](int d, int k) { return codes0 + static_cast<uint32_t>((d * kChunks + k) * threads + tid) * 8; };
  // ... the word that holds its scale byte, and the row's statistics
  const uint32_t scales0 = codes0 + static_cast<uint32_t>(D * kChunks * threads) * 8;
  auto wslot = [&](int d, int k) { return scales0 + static_cast<uint32_t>((d * kChunks + k) * threads + tid) * 4; };
  const uint32_t stats0 = scales0 + static_cast<uint32_t>(D * kChunks * threads) * 4;
  auto tslot = [&](int d) { return stats0 + static_cast<uint32_t>(d * threads + tid) * 8; };
  // the next row to copy, from the thread's first column on, and the bytes there are of each word
  const int64_t c0 = norm_col(0, t, G);
  const int chunk = 8 * G;   // columns from a chunk to the next
  const bool sum_too = ds != nullptr;
  int64_t fr = group;
  const T* fdy = dy + group * a.ld_x + c0;
  const T* fds = ds + (sum_too ? group * a.ld_res + c0 : 0);
  const int8_t* fq = a.codes + group * a.ld_codes + c0;
  const uint8_t* fsc = a.scales + group * a.ld_scales + (c0 >> 5);
  const float* fst = a.stats + 2 * group;
  // whole words of scales where rows of them are aligned to such
  const bool words = ((reinterpret_cast<uintptr_t>(a.scales) | static_cast<uintptr_t>(a.ld_scales)) & 3) == 0;
  int have[kChunks];         // bytes of the chunk in the row
#pragma unroll
  for (int k = 0; k < kChunks; ++k) {
    const int64_t left = (a.C - c0 - k * static_cast<int64_t>(chunk)) * static_cast<int64_t>(sizeof(T));
    have[k] = left <= 0 ? 0 : (left < 8 * static_cast<int64_t>(sizeof(T)) ? static_cast<int>(left) : 8 * static_cast<int>(sizeof(T)));
  }
  auto fetch = [&](int d) {
    if (fr < a.R) {
#pragma unroll
      for (int k = 0; k < kChunks; ++k) {
        if (have[k] > 0) {
#pragma unroll
          for (int w = 0; w < kQuads; ++w) {
            // a word wholly past the row reads nothing, from the chunk's own address
            const int bytes = have[k] - 16 * w;
            const int n = bytes <= 0 ? 0 : (bytes < 16 ? bytes : 16);
            const int at = k * chunk + (n > 0 ? w * (16 / static_cast<int>(sizeof(T))) : 0);
            cp_async_16_part(slot(d, (2 * k) * kQuads + w), fdy + at, n);
            if (sum_too) cp_async_16_part(slot(d, (2 * k + 1) * kQuads + w), fds + at, n);
          }
          cp_async_8(cslot(d, k), fq + k * chunk, true);
          const uint8_t* p = fsc + k * (chunk >> 5);
          if (words) cp_async_4(wslot(d, k), reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(3)), true);
          else st_shared_u32(wslot(d, k), static_cast<uint32_t>(ld_here(p)));
        }
      }
      cp_async_8(tslot(d), fst, true);
    }
    cp_async_commit();
    fr += groups;
    fdy += groups * a.ld_x;
    fds += groups * a.ld_res;
    fq += groups * a.ld_codes;
    fsc += groups * a.ld_scales;
    fst += 2 * groups;
  };
  constexpr bool kLean = kChunks > 2;
  constexpr int kKept = kLean ? 1 : kChunks;
  float2 dg[kChunks][4], db[kLayer ? kChunks : 1][4], gamma[kKept][4];
  auto read_gamma = [&](float2 (&to)[4], int k) {
    float g[8];
    norm_param<true>(g, a.gamma, norm_col(k, t, G), a.C);
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = make_float2(g[2 * i], g[2 * i + 1]);
  };
#pragma unroll
  for (int k = 0; k < kChunks; ++k) {
    if (!kLean) read_gamma(gamma[kLean ? 0 : k], k);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      dg[k][i] = make_float2(0.0f, 0.0f);
      if (kLayer) db[k][i] = make_float2(0.0f, 0.0f);
    }
  }
  const int sc_shift = words ? 8 * static_cast<int>((c0 >> 5) & 3) : 0;   // a chunk further on: a multiple of 8 bytes
  T* dx = static_cast<T*>(a.out) + group * a.ld_out;
#pragma unroll
  for (int k = 0; k < kChunks; ++k)   // what no copy reaches reads as zeros
    if (have[k] == 0) {
#pragma unroll
      for (int d = 0; d < D; ++d) {
#pragma unroll
        for (int w = 0; w < 2 * kQuads; ++w) st_shared_v4(slot(d, 2 * k * kQuads + w), 0u, 0u, 0u, 0u);
        st_shared_v2(cslot(d, k), 0u, 0u);
        st_shared_u32(wslot(d, k), 0u);
      }
    }
#pragma unroll
  for (int d = 0; d < D - 1; ++d) fetch(d);
  int d = 0;
  for (int64_t r = group; r < a.R; r += groups) {   // uniform over the group
    fetch(d == 0 ? D - 1 : d - 1);
    cp_async_wait<D - 1>();
    float2 tv[kKept][4], xh[kKept][4];
    float2 sx = make_float2(0.0f, 0.0f), st = make_float2(0.0f, 0.0f);
    const uint2 stat = ld_shared_v2_u32(tslot(d));   // mean, 1 / deviation
    const float rs = __uint_as_float(stat.y), shift = kLayer ? -__uint_as_float(stat.x) * rs : 0.0f;
    float m[kChunks];   // xh = q 2^e rstd - mu rstd
#pragma unroll
    for (int k = 0; k < kChunks; ++k) m[k] = scale_value((ld_shared_u32(wslot(d, k)) >> sc_shift) & 0xFFu) * rs;
    auto form = [&](int k, int h, float2 (&dv)[4]) {   // dy, xh and t of a chunk (t 0 past C)
      Raw8<T> raw;
#pragma unroll
      for (int w = 0; w < kQuads; ++w) raw.w[w] = ld_shared_v4_u32(slot(d, (2 * k) * kQuads + w));
      float g[8];
      values8<T>(raw, g);
      decode8(ld_shared_v2_u32(cslot(d, k)), xh[h]);
      if (kLean) read_gamma(gamma[0], k);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dv[i] = make_float2(g[2 * i], g[2 * i + 1]);
        xh[h][i] = kLayer ? fma2(xh[h][i], make_float2(m[k], m[k]), make_float2(shift, shift)) : mul2(xh[h][i], make_float2(m[k], m[k]));
        tv[h][i] = mul2(dv[i], gamma[h][i]);
      }
    };
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      const int h = kLean ? 0 : k;
      float2 dv[4];
      form(k, h, dv);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dg[k][i] = fma2(dv[i], xh[h][i], dg[k][i]);
        if (kLayer) db[k][i] = add2(db[k][i], dv[i]);
        sx = fma2(tv[h][i], xh[h][i], sx);
        if (kLayer) st = add2(st, tv[h][i]);
      }
    }
    const float2 sum = row_sum<kBlock, kLayer, true>(make_float2(sx.x + sx.y, st.x + st.y), red, half);
    const float mx = -sum.x * inv_c * rs, mt = kLayer ? -sum.y * inv_c * rs : 0.0f;
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      const int h = kLean ? 0 : k;
      if (kLean) {
        float2 dv[4];
        form(k, h, dv);
      }
      float o[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 u = fma2(xh[h][i], make_float2(mx, mx), make_float2(mt, mt));
        const float2 v = fma2(tv[h][i], make_float2(rs, rs), u);
        o[2 * i] = v.x, o[2 * i + 1] = v.y;
      }
      if (sum_too) {
        Raw8<T> raw;
#pragma unroll
        for (int w = 0; w < kQuads; ++w) raw.w[w] = ld_shared_v4_u32(slot(d, (2 * k + 1) * kQuads + w));
        float g[8];
        values8<T>(raw, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] += g[i];
      }
      if (have[k] == 8 * static_cast<int>(sizeof(T))) store8(dx + c0 + k * chunk, o);
      else if (have[k] > 0) store8_tail(dx + c0 + k * chunk, o, have[k] / static_cast<int>(sizeof(T)));
    }
    dx += groups * a.ld_out;
    if (++d == D) d = 0;
  }
  cp_async_wait_all();
  // the block's groups add up, in order, in the ring's place: a row of the workspace per block
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.C;
  if (blockDim.y > 1) {
    __syncthreads();
    float4* mine = reinterpret_cast<float4*>(ring);
    constexpr int kPer = kChunks * (kLayer ? 4 : 2);   // 16-byte words of a thread
    auto at = [&](int y, int w) -> float4& { return mine[(y * kPer + w) * G + t]; };
#pragma unroll
    for (int k = 0; k < kChunks; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        at(threadIdx.y, 2 * k + i) = make_float4(dg[k][2 * i].x, dg[k][2 * i].y, dg[k][2 * i + 1].x, dg[k][2 * i + 1].y);
        if (kLayer) at(threadIdx.y, 2 * kChunks + 2 * k + i) = make_float4(db[k][2 * i].x, db[k][2 * i].y, db[k][2 * i + 1].x, db[k][2 * i + 1].y);
      }
    __syncthreads();
    if (threadIdx.y > 0) return;
    for (int y = 1; y < static_cast<int>(blockDim.y); ++y)
#pragma unroll
      for (int k = 0; k < kChunks; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float4 q = at(y, 2 * k + i);
          dg[k][2 * i] = add2(dg[k][2 * i], make_float2(q.x, q.y));
          dg[k][2 * i + 1] = add2(dg[k][2 * i + 1], make_float2(q.z, q.w));
          if (kLayer) {
            q = at(y, 2 * kChunks + 2 * k + i);
            db[k][2 * i] = add2(db[k][2 * i], make_float2(q.x, q.y));
            db[k][2 * i + 1] = add2(db[k][2 * i + 1], make_float2(q.z, q.w));
          }
        }
  }
#pragma unroll
  for (int k = 0; k < kChunks; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t c = norm_col(k, t, G) + i;
      if (c >= a.C) continue;
      part[c] = (i & 1) ? dg[k][i / 2].y : dg[k][i / 2].x;
      if (kLayer) part[a.C + c] = (i & 1) ? db[k][i / 2].y : db[k][i / 2].x;
    }
}

// the groups' partial sums, in order: 32 columns x 32 parts of the groups per block
__global__ void __launch_bounds__(1024) norm8_columns_kernel(const float* part, int64_t groups, int64_t C, float* dgamma, float* dbeta) {
  __shared__ float red[32][33];
  griddep_wait();
  griddep_launch_dependents();
  const int64_t n = dbeta != nullptr ? 2 * C : C;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + threadIdx.x;
  const int64_t g0 = groups * threadIdx.y / 32, g1 = groups * (threadIdx.y + 1) / 32;
  float s = 0.0f;
  if (c < n) {
    const float* p = part + g0 * 2 * C + c;
#pragma unroll 8
    for (int64_t g = g0; g < g1; ++g, p += 2 * C) s += __ldcg(p);
  }
  red[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y != 0 || c >= n) return;
  s = 0.0f;
#pragma unroll
  for (int k = 0; k < 32; ++k) s += red[k][threadIdx.x];
  (c < C ? dgamma : dbeta)[c < C ? c : c - C] = s;
}

// ----------------------------------------------------------------------- host side
// Threads per row, chunks of eight per thread, and rows per block of a norm: a warp up to 512 columns
// (two chunks a lane), forward up to 768 (three: 12608 x 768 bf16 20.5 us, 22.7 as two warps, which leave
// lanes idle; backward three are no faster, and slower in fp32, 44 us for 37), else two chunks per thread up
// to 8192, four up to 16384, sweeps beyond.  Backward, rows of 8193 to 12288 take three, as four leave one
// block of 272 to 384 threads per SM: 8192 x 11008 bf16 layer norm 246 -> 220 us, RMS norm of 11007 columns
// 470 -> 411, fp32 505 -> 466, bf16 of 8320 157 -> 148, but of 11008 178 -> 191 (from 4097 to 6144 three are
// slower: 5120 79 -> 86).  Blocks are of about 256 threads and add up their rows' column sums (12608 x 768
// bf16 31 -> 27 us); forward several warps of a row are a block (four rows of it per block: 29 us for 25).
struct NormShape {
  int threads, chunks, rows;
};
static NormShape norm_shape(int64_t C, bool forward) {
  if (C <= 512) return {32, C <= 256 ? 1 : 2, kRowsPerBlock};
  if (forward && C <= 768) return {32, 3, kRowsPerBlock};
  if (C > 512 * 32) return {512, 0, 1};
  const int chunks = C > 8192 ? (C > 12288 || forward ? 4 : 3) : 2;
  const int threads = static_cast<int>((C + 8 * chunks - 1) / (8 * chunks) + 31) / 32 * 32;
  return {threads, chunks, threads <= 128 && !forward ? 256 / threads : 1};
}

// blocks of one wave with `threads` threads per SM (or the rows' own)
static int64_t norm_blocks(int64_t R, const NormShape& n, int sms, int threads) {
  const int64_t blocks = (R + n.rows - 1) / n.rows, per_sm = threads / (n.threads * n.rows);
  const int64_t most = (per_sm > 0 ? per_sm : 1) * sms;
  return blocks < most ? blocks : most;
}
constexpr int kBackThreads = 512;   // per SM: the backward pass's registers

template <typename T, int kChunks, bool kBlock, bool kLayer>
static cudaError_t launch_ring(const Norm8Args& a, dim3 grid, dim3 block, cudaStream_t s) {
  const size_t smem = static_cast<size_t>(kRing<T, kChunks>) * (kChunks * kRingBytes<T> + 8) * block.x * block.y;
  static std::atomic<bool> done[64];
  auto kernel = norm8_backward_ring_kernel<T, kChunks, kBlock, kLayer>;
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  if (dev < 0 || dev >= 64 || !done[dev].load(std::memory_order_acquire)) {
    constexpr int most = kRing<T, kChunks> * (kChunks * kRingBytes<T> + 8) * (kBlock ? 512 : 256);
    static_assert(most <= 232448 - 1024, "shared memory beyond a block's");
    err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (err != cudaSuccess) return err;
    if (dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
  }
  return launch_pdl_smem(kernel, grid, block, smem, s, a);
}
template <typename T, bool kLayer>
static cudaError_t launch_backward_ring(const Norm8Args& a, const NormShape& n, unsigned blocks, cudaStream_t s) {
  const dim3 grid(blocks), block(n.threads, n.rows);
  if (n.threads == 32) {
    if (n.chunks == 1) return launch_ring<T, 1, false, kLayer>(a, grid, block, s);
    return launch_ring<T, 2, false, kLayer>(a, grid, block, s);
  }
  if (n.chunks == 2) return launch_ring<T, 2, true, kLayer>(a, grid, block, s);
  if (n.chunks == 3) return launch_ring<T, 3, true, kLayer>(a, grid, block, s);
  return launch_ring<T, 4, true, kLayer>(a, grid, block, s);
}

template <typename T, bool kVec, bool kLayer>
static cudaError_t launch_forward(const Norm8Args& a, const NormShape& n, unsigned blocks, cudaStream_t s) {
  const dim3 grid(blocks), block(n.threads, n.rows);
  if (n.threads == 32) {
    if (n.chunks == 1) return launch_pdl(norm8_forward_kernel<T, 1, kVec, false, kLayer>, grid, block, s, a);
    if (n.chunks == 2) return launch_pdl(norm8_forward_kernel<T, 2, kVec, false, kLayer>, grid, block, s, a);
    return launch_pdl(norm8_forward_kernel<T, 3, kVec, false, kLayer>, grid, block, s, a);
  }
  if (n.chunks == 2) return launch_pdl(norm8_forward_kernel<T, 2, kVec, true, kLayer>, grid, block, s, a);
  if (n.chunks == 4) return launch_pdl(norm8_forward_kernel<T, 4, kVec, true, kLayer>, grid, block, s, a);
  return launch_pdl(norm8_forward_kernel<T, 0, kVec, true, kLayer>, grid, block, s, a);
}

template <typename T, bool kVec, bool kLayer>
static cudaError_t launch_backward(const Norm8Args& a, const NormShape& n, unsigned blocks, cudaStream_t s) {
  const dim3 grid(blocks), block(n.threads, n.rows);
  if (n.chunks == 0) return launch_pdl(norm8_backward_kernel<T, 0, kVec, true, kLayer>, grid, block, s, a);
  if constexpr (kVec) {
    return launch_backward_ring<T, kLayer>(a, n, blocks, s);
  } else {
    if (n.threads == 32) {
      if (n.chunks == 1) return launch_pdl(norm8_backward_kernel<T, 1, false, false, kLayer>, grid, block, s, a);
      return launch_pdl(norm8_backward_kernel<T, 2, false, false, kLayer>, grid, block, s, a);
    }
    if (n.chunks == 2) return launch_pdl(norm8_backward_kernel<T, 2, false, true, kLayer>, grid, block, s, a);
    if (n.chunks == 3) return launch_pdl(norm8_backward_kernel<T, 3, false, true, kLayer>, grid, block, s, a);
    return launch_pdl(norm8_backward_kernel<T, 4, false, true, kLayer>, grid, block, s, a);
  }
}

template <typename T, bool kVec, bool kLayer>
static cudaError_t launch_norm(const Norm8Args& a, const NormShape& n, bool forward, unsigned blocks, cudaStream_t s) {
  return forward ? launch_forward<T, kVec, kLayer>(a, n, blocks, s) : launch_backward<T, kVec, kLayer>(a, n, blocks, s);
}

template <typename T>
static cudaError_t launch_norm_as(const Norm8Args& a, const NormShape& n, bool vec, bool layer, bool forward, unsigned blocks,
                                  cudaStream_t s) {
  if (vec) return layer ? launch_norm<T, true, true>(a, n, forward, blocks, s) : launch_norm<T, true, false>(a, n, forward, blocks, s);
  return layer ? launch_norm<T, false, true>(a, n, forward, blocks, s) : launch_norm<T, false, false>(a, n, forward, blocks, s);
}

// *parts: the rows of partial sums that a backward pass leaves
static int run_norm(const Norm8Args& a, int dtype, bool layer, bool forward, int sms, int64_t* parts, cudaStream_t s) {
  const NormShape n = norm_shape(a.C, forward);
  auto ok = [&](auto tag) {
    using T = decltype(tag);
    return rows16<T>(a.x, a.ld_x) && rows16<T>(a.out, a.ld_out) && (a.res == nullptr || rows16<T>(a.res, a.ld_res)) &&
           (a.res == nullptr || !forward || rows16<T>(a.sum, a.ld_sum)) && aligned16(a.gamma) &&
           (a.beta == nullptr || aligned16(a.beta));
  };
  const bool vec = dtype == SQ_F32 ? ok(float()) : ok(__half());
  const int64_t blocks = forward ? (a.R + n.rows - 1) / n.rows : norm_blocks(a.R, n, sms, kBackThreads);
  const unsigned b = static_cast<unsigned>(blocks);
  if (parts != nullptr) *parts = vec && n.chunks > 0 ? blocks : blocks * n.rows;   // the ring adds up a block's groups
  cudaError_t err;
  if (dtype == SQ_F32) err = launch_norm_as<float>(a, n, vec, layer, forward, b, s);
  else if (dtype == SQ_BF16) err = launch_norm_as<__nv_bfloat16>(a, n, vec, layer, forward, b, s);
  else err = launch_norm_as<__half>(a, n, vec, layer, forward, b, s);
  return err == cudaSuccess ? SQ_OK : cuda_fail(err, "norm8 kernel launch");
}

static int check_norm(const char* who, const Norm8Args& a, int dtype) {
  constexpr int64_t kMax = (int64_t(1) << 30);
  if (a.R > kMax || a.C > kMax) return fail(SQ_EUNSUPPORTED, "%s: more than 2^30 rows or columns", who);
  if (a.x == nullptr || a.out == nullptr || a.gamma == nullptr || a.ld_x < a.C || a.ld_out < a.C)
    return fail(SQ_EINVAL, "%s: NULL argument or leading dimension too small", who);
  if (a.res != nullptr && a.ld_res < a.C) return fail(SQ_EINVAL, "%s: ld of the residual < cols", who);
  const uintptr_t e = dtype_bytes(dtype);
  if (reinterpret_cast<uintptr_t>(a.x) % e || reinterpret_cast<uintptr_t>(a.out) % e || reinterpret_cast<uintptr_t>(a.res) % e ||
      reinterpret_cast<uintptr_t>(a.sum) % e || reinterpret_cast<uintptr_t>(a.gamma) % 4 || reinterpret_cast<uintptr_t>(a.beta) % 4)
    return fail(SQ_EALIGN, "%s: a tensor is not aligned to its type", who);
  if (a.codes == nullptr) return SQ_OK;
  const int64_t nb = (a.C + 31) / 32;
  if (a.ld_codes < 32 * nb || a.ld_scales < nb) return fail(SQ_EINVAL, "%s: ld_codes or ld_scales too small", who);
  if (!aligned16(a.codes) || a.ld_codes % 16 || reinterpret_cast<uintptr_t>(a.stats) % 8)
    return fail(SQ_EALIGN, "%s: codes and ld_codes need 16-byte alignment, stats 8", who);
  return SQ_OK;
}

}  // namespace sq

using namespace sq;

extern "C" sq_status shiftquant_norm8_forward(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld_x,
                                              const void* residual, int64_t ld_residual, void* sum, int64_t ld_sum,
                                              const float* gamma, const float* beta, float eps, void* y, int64_t ld_y,
                                              int8_t* codes, int64_t ld_codes, uint8_t* scales, int64_t ld_scales, float* stats,
                                              int32_t* dev_status, void* stream) {
  fail(SQ_OK, "");
  if (!dtype_ok(dtype)) return fail(SQ_EINVAL, "norm8_forward: bad dtype %d", dtype);
  if (rows < 0 || cols < 0) return fail(SQ_EINVAL, "norm8_forward: negative size");
  if (!(eps >= 0.0f)) return fail(SQ_EINVAL, "norm8_forward: eps is negative or NaN");
  if (rows == 0 || cols == 0) return SQ_OK;
  if ((residual == nullptr) != (sum == nullptr) || (sum != nullptr && ld_sum < cols))
    return fail(SQ_EINVAL, "norm8_forward: residual and sum come together, ld_sum >= cols");
  if ((codes == nullptr) != (scales == nullptr) || (codes == nullptr) != (stats == nullptr) || dev_status == nullptr)
    return fail(SQ_EINVAL, "norm8_forward: codes, scales and stats come together, dev_status is required");
  Norm8Args a;
  memset(&a, 0, sizeof(a));
  a.x = x, a.ld_x = ld_x, a.res = residual, a.ld_res = ld_residual, a.out = y, a.ld_out = ld_y, a.sum = sum, a.ld_sum = ld_sum;
  a.R = rows, a.C = cols, a.gamma = gamma, a.beta = beta, a.eps = eps;
  a.codes = codes, a.ld_codes = ld_codes, a.scales = scales, a.ld_scales = ld_scales, a.stats = stats, a.status = dev_status;
  const int st = check_norm("norm8_forward", a, dtype);
  if (st != SQ_OK) return st;
  const int sms = device_sms(nullptr);
  if (sms <= 0) return fail(SQ_ECUDA, "norm8_forward: no current CUDA device");
  return run_norm(a, dtype, beta != nullptr, true, sms, nullptr, as_stream(stream));
}

extern "C" size_t shiftquant_norm8_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0) return 0;
  const int sms = device_sms(nullptr);
  const NormShape n = norm_shape(cols, false);
  return static_cast<size_t>(norm_blocks(rows, n, sms > 0 ? sms : 152, kBackThreads) * n.rows) * 2 * static_cast<size_t>(cols) * sizeof(float);
}

extern "C" sq_status shiftquant_norm8_backward(const void* dy, int dtype, int64_t rows, int64_t cols, int64_t ld_dy,
                                               const int8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t ld_scales,
                                               const float* stats, const float* gamma, const void* dsum, int64_t ld_dsum,
                                               void* dx, int64_t ld_dx, float* dgamma, float* dbeta, void* workspace,
                                               size_t workspace_bytes, void* stream) {
  fail(SQ_OK, "");
  if (!dtype_ok(dtype)) return fail(SQ_EINVAL, "norm8_backward: bad dtype %d", dtype);
  if (rows < 0 || cols < 0) return fail(SQ_EINVAL, "norm8_backward: negative size");
  if (cols == 0) return SQ_OK;
  if (dgamma == nullptr) return fail(SQ_EINVAL, "norm8_backward: NULL dgamma");
  if (reinterpret_cast<uintptr_t>(dgamma) % 4 || reinterpret_cast<uintptr_t>(dbeta) % 4)
    return fail(SQ_EALIGN, "norm8_backward: dgamma or dbeta is not aligned to its type");
  cudaStream_t s = as_stream(stream);
  if (rows == 0) {   // sums over no rows
    cudaError_t err = cudaMemsetAsync(dgamma, 0, static_cast<size_t>(cols) * sizeof(float), s);
    if (err == cudaSuccess && dbeta != nullptr) err = cudaMemsetAsync(dbeta, 0, static_cast<size_t>(cols) * sizeof(float), s);
    return err == cudaSuccess ? SQ_OK : cuda_fail(err, "cudaMemsetAsync");
  }
  if (codes == nullptr || scales == nullptr || stats == nullptr) return fail(SQ_EINVAL, "norm8_backward: NULL argument");
  Norm8Args a;
  memset(&a, 0, sizeof(a));
  a.x = dy, a.ld_x = ld_dy, a.res = dsum, a.ld_res = ld_dsum, a.out = dx, a.ld_out = ld_dx;
  a.R = rows, a.C = cols, a.gamma = gamma;
  a.codes = const_cast<int8_t*>(codes), a.ld_codes = ld_codes, a.scales = const_cast<uint8_t*>(scales), a.ld_scales = ld_scales;
  a.stats = const_cast<float*>(stats);
  const int st = check_norm("norm8_backward", a, dtype);
  if (st != SQ_OK) return st;
  const int sms = device_sms(nullptr);
  if (sms <= 0) return fail(SQ_ECUDA, "norm8_backward: no current CUDA device");
  if (workspace == nullptr || workspace_bytes < shiftquant_norm8_workspace_bytes(rows, cols))
    return fail(SQ_EINVAL, "norm8_backward: workspace smaller than shiftquant_norm8_workspace_bytes");
  if (!aligned16(workspace)) return fail(SQ_EALIGN, "norm8_backward: the workspace needs 16-byte alignment");
  a.part = static_cast<float*>(workspace);
  int64_t parts = 0;
  const int st2 = run_norm(a, dtype, dbeta != nullptr, false, sms, &parts, s);
  if (st2 != SQ_OK) return st2;
  const int64_t nc = dbeta != nullptr ? 2 * cols : cols;
  const cudaError_t err = launch_pdl(norm8_columns_kernel, dim3(static_cast<unsigned>((nc + 31) / 32)), dim3(32, 32), s,
                                     static_cast<const float*>(a.part), parts, cols, dgamma, dbeta);
  return err == cudaSuccess ? SQ_OK : cuda_fail(err, "norm8_columns_kernel launch");
}
