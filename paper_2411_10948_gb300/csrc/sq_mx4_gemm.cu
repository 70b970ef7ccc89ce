// The product of two microscaled 4-bit tensors on the block-scaled tensor cores:
//   D[m, n] = sum_b 2^(ea[m, b] + eb[n, b]) sum_{k in block b} a[m, k] b[n, k]
// with both operands packed along k (K-major) and the sums held in FP32 (tcgen05.mma
// kind::mxf4, 64 elements of K per instruction, the scale bytes read from tensor memory).  It is
// the forward product (x rows, W columns), loss propagation (dy rows, W rows) and the weight
// gradient (x columns, dy columns) of a linear layer, given the orientation each needs.
//
// Operands and scales arrive by TMA: 256 elements of K per stage, which are one 128-byte
// swizzled row of codes per operand row and two 512-byte scale tiles per 128 rows; the scale
// tiles go on to tensor memory by tcgen05.cp in front of the MMAs that use them.
//
// Two forms.  mx4_pair_kernel: persistent CTA pairs on 256 x 256 tiles.  mx4_split_kernel: tiles
// of 128 columns of D x 16..128 rows, the K loop split over a cluster whose partial tiles are
// summed through distributed shared memory in rank order, for products with too few tiles to
// fill the SMs (a few tokens, small layers); the columns of D are the MMA's M there, so a warp
// writes 32 consecutive outputs of a row.  With up to 32 rows it can take them as floating-point
// values: its epilogue warps then quantize each stage's rows while the weights' copies are on their way.
#include <cuda_runtime.h>

#include <atomic>
#include <cstring>

#include "sq_device.cuh"
#include "sq_block.cuh"
#include "sq_host.h"

namespace sq {

constexpr int kStageK = 256;             // elements of K per stage
constexpr int kOperandRowBytes = 128;    // their codes in one row
constexpr int kScaleBytes = 1024;        // and the scales of 128 rows
constexpr int kScaleCols = 8;            // tensor-memory columns those take

// scale bytes from shared memory to tensor memory, 128 rows x 4 blocks per 512-byte tile: lane l,
// byte b of column j is row 32 j + l, block b, the same in all four lane quarters
template <int kCg>
__device__ __forceinline__ void tc_copy_scales(uint32_t taddr, uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);   // start address
  d |= static_cast<uint64_t>(128 >> 4) << 32;             // 8 rows of 16 bytes per core matrix
  d |= static_cast<uint64_t>(1) << 46;                    // descriptor version (sm_100+)
  if constexpr (kCg == 2)
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(d) : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(d) : "memory");
}

template <int kCg>
__device__ __forceinline__ void tc_mma_mx4(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                           uint32_t sa, uint32_t sb, uint32_t accumulate) {
  if constexpr (kCg == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}

// Instruction descriptor of kind::mxf4: e2m1 operands, e8m0 scales, M x N tile, K = 64; `half`
// says which two of the four scale bytes of a column the instruction takes.
__host__ __device__ constexpr uint32_t mx4_idesc(uint32_t M, uint32_t N, uint32_t half) {
  return (half * 2u << 4)           // scale bytes of B
         | (1u << 7) | (1u << 10)   // A and B: e2m1
         | ((N >> 3) << 17) | (1u << 23) | ((M >> 4) << 24)
         | (half * 2u << 29);       // scale bytes of A
}

// the scales of a stage into tensor memory, then its MMAs: rows of A at a0 (scales sfa),
// rows of B at b0 (sfb: kBTiles tiles of 128 rows).  tsf: 8 columns for A, then 8 per B tile, in
// each the first four blocks' columns of every tile before the last four's.  sfb_off: columns
// by which B's first row lies inside its scale tile.
template <int kCg, uint32_t kM, uint32_t kN, int kBTiles>
__device__ __forceinline__ void mx4_stage(uint32_t d, uint32_t a0, uint32_t b0, uint32_t sfa, uint32_t sfb, uint32_t tsf,
                                          uint32_t sfb_off, bool first) {
  const uint32_t tsfb = tsf + kScaleCols;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    tc_copy_scales<kCg>(tsf + 4 * j, sfa + 512 * j);
#pragma unroll
    for (int t = 0; t < kBTiles; ++t)
      tc_copy_scales<kCg>(tsfb + 4 * (j * kBTiles + t), sfb + t * kScaleBytes + 512 * j);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t idesc = mx4_idesc(kM, kN, k & 1);
    tc_mma_mx4<kCg>(d, make_sdesc_k_sw128(a0 + 32 * k), make_sdesc_k_sw128(b0 + 32 * k), idesc, tsf + 4 * (k >> 1),
                    tsfb + 4 * kBTiles * (k >> 1) + sfb_off, (!first || k > 0) ? 1u : 0u);
  }
}

// The issuing of tcgen05 instructions is what a thread does most of the time here, and its
// operands are uniform registers: a warp's index, rank and tensor-memory base are taken through
// a shuffle, which makes them uniform for the compiler, and the issuing thread is elected.
// With a thread picked by threadIdx instead an instruction took 71 clocks to issue (an MMA of
// 256 columns 128 to run, so that 4 of them with 6 scale copies took 712 clocks for 514) and the
// 16384 x 4096 x 11008 product 302 us.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xFFFFFFFFu, v, 0); }
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}

// Arrive on a barrier of either CTA of a pair after reads of tensor memory (completed, and ordered
// by tc_fence_before): no shared or global memory is handed over, so CTA scope does.  With a
// release at cluster scope the arrival took 1100 clocks.
__device__ __forceinline__ void mbar_arrive_drained(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}

struct Mx4Gemm {
  CUtensorMap a, b;     // codes, boxes of 128 bytes x the rows a CTA holds
  CUtensorMap sa, sb;   // scales, boxes of 1024 bytes x row tiles
  CUtensorMap out;      // 32 rows x 64 bytes (where rows are 16-byte aligned)
  int64_t M, N;
  int kblocks;          // stages of the whole K loop
  int tiles_m, tiles_n; // of the form's tile
  void* d;
  int64_t ldd;
  int tma_out;
  int32_t* status;
};

// ------------------------------------------------------------------ CTA pairs
// 256 x 256 tiles: of the operands of a stage (256 of K) each SM takes 32 KB of codes and 3 KB of scales
// from L2, 560 clocks at 64 bytes a clock, for 512 clocks of MMAs (128 each, measured alone): a smaller tile
// takes more bytes per product, a larger one has no room in tensor memory.  Stages: with an earlier epilogue
// three took 266 us for 16384 x 4096 x 11008 in a loop, four 222, five 205; six are what fits.  Measured (bf16
// out): that product 186-207 us, 7.1-7.9 PFLOP/s; 16384 x 11008 x 4096 207-214 us (6.9-7.1); fp32 out
// 4096 x 11008 x 16384 225 us (6.6, nine tiles a pair and a tenth for four of 76).  The tensor pipe was active
// for 77% of a 16384 x 8192 x 4096 product.  In long runs the power limit takes the clock to 1.7 of 2.07 GHz;
// without copies and outputs the MMAs reached 8.6 PFLOP/s at 2.07.
constexpr int kPM = 128;                   // rows of D per CTA
constexpr int kPN = 256;                   // columns of a tile
constexpr int kPStages = 6;
constexpr int kPABytes = kPM * kOperandRowBytes;
constexpr int kPBBytes = kPN / 2 * kOperandRowBytes;
constexpr int kPStageBytes = kPABytes + kPBBytes + 3 * kScaleBytes;   // A's scales, B's (all 256 rows)
constexpr int kPThreads = 384;             // producer, MMA issuer, 2 idle warps, 8 epilogue warps
constexpr int kPEpiWarp0 = 4;
constexpr int kPEpiWarps = 8;
constexpr int kPBoxBytes = 32 * 64;
constexpr int kPOutOffset = kPStages * kPStageBytes;
constexpr int kPBarOffset = kPOutOffset + kPEpiWarps * kPBoxBytes;
constexpr size_t kPSmem = kPBarOffset + (2 * kPStages + 3) * 8 + 16;
static_assert(kPSmem <= 232448, "shared memory beyond the 227 KB per-CTA limit");
static_assert(kPStageBytes % 1024 == 0 && kPOutOffset % 1024 == 0, "swizzle atoms need 1 KB");
// Tensor memory: 512 columns hold the stages' scales (24 columns each) and two accumulators of
// 256 that share the columns between kPAcc1 and 256: the epilogue drains those first, and the
// next tile's products start while it drains the rest.
constexpr uint32_t kPScaleSlot = 3 * kScaleCols;
constexpr uint32_t kPScale0 = 512 - kPStages * kPScaleSlot;
constexpr uint32_t kPAcc1 = kPScale0 - kPN;
constexpr int kPShared = 192;              // at least the columns the two share
static_assert(kPN - kPAcc1 <= kPShared && kPShared % 64 == 0, "the epilogue hands back whole loads");
constexpr int kPGroupM = 8;                // row tiles that take a column tile in turn

// tile t of the launch: column tiles run inside groups of kPGroupM row tiles
__device__ __forceinline__ void pair_tile(const Mx4Gemm& g, int t, int* tm, int* tn) {
  const int per = kPGroupM * g.tiles_n;
  const int grp = t / per, r = t - grp * per;
  const int rows = min(kPGroupM, g.tiles_m - grp * kPGroupM);
  *tn = r / rows;
  *tm = grp * kPGroupM + r - *tn * rows;
}

// kCols (a multiple of 32) consecutive columns of the warp's 32 lanes
template <int kCols>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&v)[kCols]) {
  static_assert(kCols % 32 == 0, "whole loads");
#pragma unroll
  for (int c = 0; c < kCols; c += 32) tmem_ld_32x32b_x32(taddr + c, reinterpret_cast<uint32_t (&)[32]>(v[c]));
}

// 16-byte quad of a row of a staged box (64-byte rows, 64-byte swizzle)
__device__ __forceinline__ uint32_t box_quad(uint32_t buf, int row, int quad) {
  return buf + row * 64 + ((quad ^ ((row >> 1) & 3)) << 4);
}

// 32 rows x 64 bytes of D from FP32 sums, a lane a row: through shared memory by TMA, or where rows
// are not 16-byte aligned an element per lane and row
template <typename T>
__device__ __forceinline__ void write_box(const Mx4Gemm& g, const uint32_t* v, uint32_t buf, int64_t row0, int64_t col0,
                                          int lane) {
  if (row0 >= g.M || col0 >= g.N) return;   // warp-uniform
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if constexpr (sizeof(T) == 4) w[i] = v[i];
    else w[i] = pack2<T>(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
  }
  if (lane == 0) bulk_wait_read<0>();       // the box's last store has read it
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) st_shared_v4(box_quad(buf, lane, i), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  if (g.tma_out) {
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_2d(&g.out, buf, static_cast<int32_t>(col0), static_cast<int32_t>(row0));
      bulk_commit();
    }
    return;
  }
  __syncwarp();
  constexpr int kPerRow = 64 / sizeof(T);    // elements: 16 or 32
  constexpr int kStep = 32 / kPerRow;        // rows at a time
  const int c = lane % kPerRow, r0 = lane / kPerRow;
  T* d = static_cast<T*>(g.d) + (row0 + r0) * g.ldd + col0 + c;
  const int64_t step = kStep * g.ldd;
  const int left = col0 + c < g.N ? static_cast<int>(g.M - row0 < 32 ? g.M - row0 : 32) - r0 : 0;   // rows, from the lane's first on
  const bool whole = row0 + 32 <= g.M && col0 + kPerRow <= g.N;
#pragma unroll
  for (int h = 0; h < kPerRow; h += 8) {
    uint32_t x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // row r = (h + i) kStep + r0 of the box: its swizzle is the same for all lanes
      constexpr int kShift = kStep == 2 ? 0 : 1;
      const int quad = (c * static_cast<int>(sizeof(T)) / 16) ^ (((h + i) >> kShift) & 3);
      x[i] = ld_shared_u32(buf + ((h + i) * kStep + r0) * 64 + quad * 16 + (c * sizeof(T) & 12));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (whole || (h + i) * kStep < left) {
        if constexpr (sizeof(T) == 4) *d = __uint_as_float(x[i]);
        else *reinterpret_cast<uint16_t*>(d) = static_cast<uint16_t>((c & 1) ? x[i] >> 16 : x[i]);
      }
      d += step;
    }
  }
  __syncwarp();
}

template <typename T>
__global__ void __launch_bounds__(kPThreads, 1) mx4_pair_kernel(const __grid_constant__ Mx4Gemm g) {
  extern __shared__ __align__(1024) uint8_t smem[];
  if ((smem_u32(smem) & 1023u) != 0) {  // the swizzled layouts need 1 KB alignment
    if (threadIdx.x == 0) atomicOr(g.status, kDevInternal);
    return;
  }
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + kPBarOffset);
  uint64_t* empty = full + kPStages;
  uint64_t* tfull = empty + kPStages;   // a tile's products are complete (in each CTA)
  uint64_t* tempty = tfull + 1;         // the leader's: both epilogues have drained the shared columns
  uint64_t* drain = tempty + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = static_cast<int>(uniform(threadIdx.x >> 5)), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kPStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    mbar_init(tfull, 1);
    mbar_init(tempty, 2 * kPEpiWarps);
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane == 0) {
    tma_prefetch_desc(&g.a);
    tma_prefetch_desc(&g.b);
    tma_prefetch_desc(&g.sa);
    tma_prefetch_desc(&g.sb);
  }
  if (warp == 1) {
    tmem_alloc<2>(smem_u32(tmem_slot), 512);
    tmem_relinquish<2>();
  }
  tc_fence_before();
  cluster_sync();
  tc_fence_after();
  griddep_wait();
  griddep_launch_dependents();
  const uint32_t tmem = uniform(*tmem_slot);
  const uint32_t rank = uniform(cluster_ctarank());
  const int pair = static_cast<int>(blockIdx.x) >> 1, npairs = static_cast<int>(gridDim.x) >> 1;
  const int tiles = g.tiles_m * g.tiles_n;
  const uint32_t peer_abort = mapa_shared(smem_u32(const_cast<int*>(abort_flag)), rank ^ 1u);

  if (warp == 0) {
    if (elect_one()) {
      // producer: each CTA loads its 128 rows of A with their scales, its half of B's rows, and
      // the scales of all of B's; the bytes of both CTAs count on the leader's barrier
      const uint32_t full_c = mapa_shared(smem_u32(full), 0);
      int s = 0;
      uint32_t ph = 0;
      long long issued = 0;
      bool ok = true;
      for (int t = pair; t < tiles && ok; t += npairs) {
        int tm, tn;
        pair_tile(g, t, &tm, &tn);
        for (int kb = 0; kb < g.kblocks; ++kb) {
          if (!mbar_wait(&empty[s], ph ^ 1u, abort_flag)) {
            ok = false;
            break;
          }
          const uint32_t a0 = smem_u32(smem + s * kPStageBytes);
          const uint32_t bar = full_c + s * 8;
          if (rank == 0) mbar_arrive_expect_tx(&full[s], 2 * kPStageBytes);
          tma_load_2d_pair(a0, &g.a, bar, kb * kOperandRowBytes, tm * 2 * kPM + static_cast<int>(rank) * kPM);
          tma_load_2d_pair(a0 + kPABytes, &g.b, bar, kb * kOperandRowBytes, tn * kPN + static_cast<int>(rank) * (kPN / 2));
          tma_load_2d_pair(a0 + kPABytes + kPBBytes, &g.sa, bar, kb * (kScaleBytes / 4), tm * 2 + static_cast<int>(rank));
          tma_load_2d_pair(a0 + kPABytes + kPBBytes + kScaleBytes, &g.sb, bar, kb * (kScaleBytes / 4), tn * 2);
          ++issued;
          if (++s == kPStages) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      if (!ok) {
        atomicOr(g.status, kDevTimeout);
        *abort_flag = 1;
        st_cluster_u32(peer_abort, 1);
      }
      // every issued copy has landed before the CTAs may exit: the leader's barriers count the
      // bytes of both; after a timeout the peer gives its own copies time instead
      if (rank == 0) {
        for (long long i = issued > kPStages ? issued - kPStages : 0; i < issued; ++i)
          mbar_wait(&full[i % kPStages], static_cast<uint32_t>((i / kPStages) & 1), nullptr);
      } else if (!ok) {
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) {
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0 && elect_one()) {
      // MMA issuer (the leader's)
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      int it = 0;
      for (int t = pair; t < tiles && ok; t += npairs, ++it) {
        if (it > 0 && !mbar_wait(tempty, static_cast<uint32_t>(it - 1) & 1u, abort_flag)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t d = tmem + ((it & 1) ? kPAcc1 : 0u);
        for (int kb = 0; kb < g.kblocks; ++kb) {
          if (!mbar_wait(&full[s], ph, abort_flag)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t a0 = smem_u32(smem + s * kPStageBytes);
          const uint32_t sf = a0 + kPABytes + kPBBytes;
          mx4_stage<2, 2 * kPM, kPN, 2>(d, a0, a0 + kPABytes, sf, sf + kScaleBytes, tmem + kPScale0 + s * kPScaleSlot, 0u,
                                        kb == 0);
          tc_commit<2>(smem_u32(&empty[s]), 0x3);
          if (++s == kPStages) {
            s = 0;
            ph ^= 1u;
          }
        }
        if (ok) tc_commit<2>(smem_u32(tfull), 0x3);
      }
      if (!ok) {
        atomicOr(g.status, kDevTimeout);
        *abort_flag = 1;
        st_cluster_u32(peer_abort, 1);
      }
      tc_commit<2>(smem_u32(drain), 0x1);  // every MMA issued has completed
      mbar_wait(drain, 0, nullptr);
    }
  } else if (warp >= kPEpiWarp0) {
    // epilogue: half h takes kPShared / 2 of the shared columns into registers at once, hands them
    // back and writes them, then its part of the others; boxes of 32 rows x 64 bytes
    constexpr int kBox = 64 / sizeof(T);          // columns of a box
    const int q = warp & 3, h = (warp - kPEpiWarp0) >> 2;
    const uint32_t buf = smem_u32(smem + kPOutOffset + (warp - kPEpiWarp0) * kPBoxBytes);
    const uint32_t tempty_c = mapa_shared(smem_u32(tempty), 0);
    bool ok = true;
    int it = 0;
    for (int t = pair; t < tiles; t += npairs, ++it) {
      int tm, tn;
      pair_tile(g, t, &tm, &tn);
      if (!__all_sync(0xFFFFFFFFu, mbar_wait(tfull, static_cast<uint32_t>(it) & 1u, abort_flag))) {
        ok = false;
        break;
      }
      tc_fence_after();
      const int64_t row0 = static_cast<int64_t>(tm) * 2 * kPM + rank * kPM + q * 32;
      const int64_t n0 = static_cast<int64_t>(tn) * kPN;
      const uint32_t acc = tmem + (static_cast<uint32_t>(q * 32) << 16) + ((it & 1) ? kPAcc1 : 0u);
      // buffer 0 shares its upper columns, buffer 1 its lower ones
      const int first = ((it & 1) ? 0 : kPN - kPShared) + h * (kPShared / 2);
      const int second = ((it & 1) ? kPShared : 0) + h * ((kPN - kPShared) / 2);
      {
        uint32_t v[kPShared / 2];
        tmem_ld_cols<kPShared / 2>(acc + first, v);
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_drained(tempty_c);
#pragma unroll
        for (int c = 0; c < kPShared / 2; c += kBox) write_box<T>(g, v + c, buf, row0, n0 + first + c, lane);
      }
      {
        uint32_t v[(kPN - kPShared) / 2];
        tmem_ld_cols<(kPN - kPShared) / 2>(acc + second, v);
        tmem_ld_wait();
#pragma unroll
        for (int c = 0; c < (kPN - kPShared) / 2; c += kBox) write_box<T>(g, v + c, buf, row0, n0 + second + c, lane);
      }
      tc_fence_before();   // these reads precede the arrival for the next tile
    }
    if (!ok) {
      atomicOr(g.status, kDevTimeout);
      *abort_flag = 1;
      st_cluster_u32(peer_abort, 1);
    }
    if (lane == 0) bulk_wait_read<0>();  // no store still reads shared memory at exit
  }
  tc_fence_before();
  cluster_sync();   // neither CTA leaves while the other may reach its barriers, memory or TMEM
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc<2>(tmem, 512);
  }
}

// ------------------------------------------------------- split K over a cluster
// Bound by latency: set-up 0.2 us, the first stage's copy and MMAs 1.1 us, the partial tiles' exchange and the
// outputs' way out 2 us and more, and by the weights' bytes where there are many.  One token (graph replays,
// weights from HBM) through 4096 x 4096 4.9 us, 4096 x 11008 7.3 us (3.3 TB/s); 64 rows through 4096 x 4096
// 10.1 us with their quantization; a 256 x 512 x 512 product 4.6 us.
constexpr int kSplitBlocks = 2;  // blocks per SM that a split of K may reach (3: a token through 4096 x 11008 12.4 us for 9.9 then)
constexpr int kSThreads = 192;   // 4 epilogue warps, producer, MMA issuer

template <int kN>
struct Split {
  static constexpr int stages = kN == 128 ? 3 : kN == 64 ? 4 : 5;
  static constexpr int a_bytes = 128 * kOperandRowBytes;
  static constexpr int b_bytes = kN * kOperandRowBytes;
  static constexpr int stage_bytes = a_bytes + b_bytes + 2 * kScaleBytes;
  static constexpr int bar_offset = stages * stage_bytes;
  static constexpr size_t bytes = bar_offset + (2 * stages + 2) * 8 + 16;
  static constexpr uint32_t acc_cols = kN < 32 ? 32 : kN;
  static constexpr uint32_t cols = acc_cols + stages * 2 * kScaleCols > 128 ? 256 : 128;
  static_assert(128 * kN * 4 <= bar_offset, "the partial tile takes the stages' place");
  static_assert(stage_bytes % 1024 == 0, "swizzle atoms need 1 KB");
};

__device__ __forceinline__ float4 ld_cluster_v4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}

// The sum of kSize partial tiles [m][n] at `part` of each rank's shared memory, in rank order, into D: the
// rank's part of the tile, four consecutive columns of a row per thread and item, eight loads on their way
// at once.  (All loads at once, and the ranks parting before the stores: 256 x 512 x 512 alike, but a token
// through 4096 x 4096, eight ranks, 5.8 us for 4.8.)
template <typename T, int kN, int kSize>
__device__ __forceinline__ void sum_ranks(const Mx4Gemm& g, uint32_t part, uint32_t rank, int m0, int n0) {
  constexpr int kAtOnce = 8 / kSize;
  T* d = static_cast<T*>(g.d);
  for (int i0 = static_cast<int>(rank) * kSThreads + static_cast<int>(threadIdx.x); i0 < 32 * kN; i0 += kAtOnce * kSize * kSThreads) {
    float4 v[kAtOnce][kSize];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = i0 + k * kSize * kSThreads;
      if (i >= 32 * kN) continue;
#pragma unroll
      for (int r = 0; r < kSize; ++r)
        v[k][r] = kSize == 1 ? ld_shared_v4_f32(part + i * 16) : ld_cluster_v4(mapa_shared(part + i * 16, r));
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = i0 + k * kSize * kSThreads, m = i >> 5, n = (i & 31) * 4;
      if (i >= 32 * kN || m0 + m >= g.M || n0 + n >= g.N) continue;
      float4 sum = v[k][0];
#pragma unroll
      for (int r = 1; r < kSize; ++r) {
        sum.x += v[k][r].x, sum.y += v[k][r].y;
        sum.z += v[k][r].z, sum.w += v[k][r].w;
      }
      T* o = d + static_cast<int64_t>(m0 + m) * g.ldd + n0 + n;
      if (g.tma_out && n0 + n + 4 <= g.N) {   // aligned rows: four at once
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(o) = sum;
        else *reinterpret_cast<uint2*>(o) = make_uint2(pack2<T>(sum.x, sum.y), pack2<T>(sum.z, sum.w));
      } else {
        const float q[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (n0 + n + j < g.N) o[j] = from_f32<T>(q[j]);
      }
    }
  }
  if constexpr (kSize > 1) cluster_sync();   // no CTA leaves while another may read its tile
}

// The rows' operand as floating-point values [M, ld], K of them a row (vec: 16-byte aligned rows).
struct Mx4Rows {
  const void* x;
  int64_t ld, K;
  int vec;
  // at most four rows: a stage is one warp's (eight blocks of each row), and the warps take the stages in turn.
  // One row through 4096 x 11008 7.5 us, 10.0 where all four warps share each stage; 4096 x 4096 5.0 and 5.2
  int by_warp;
};

// A block of 32 elements of a row on its way to a thread.
template <typename T>
struct Block32 {
  Raw8<T> raw[4];
  __device__ __forceinline__ void load(const Mx4Rows& rows, int64_t m, int64_t M, int64_t k) {
    const T* p = static_cast<const T*>(rows.x) + m * rows.ld + k;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t left = m < M ? rows.K - k - 8 * i : 0;
      if (left <= 0) zero8(raw[i]);
      else if (rows.vec && left >= 8) load8(raw[i], p + 8 * i);
      else load8_tail(raw[i], p + 8 * i, left < 8 ? static_cast<int>(left) : 8);
    }
  }
  // the block's scale byte, and its codes
  __device__ __forceinline__ uint32_t quantize(uint4& codes) const {
    float f[4][8], m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      values8<T>(raw[i], f[i]);
      m[i] = max_abs(max_abs(max_abs(f[i][0], f[i][1]), max_abs(f[i][2], f[i][3])),
                     max_abs(max_abs(f[i][4], f[i][5]), max_abs(f[i][6], f[i][7])));
    }
    const uint32_t scale = scale_of_mx4(__float_as_uint(max_abs(max_abs(m[0], m[1]), max_abs(m[2], m[3]))));
    const float inv = scale_inverse(scale);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] *= inv;
      w[i] = scale == kScaleNan ? 0u : codes8(f[i]);
    }
    codes = make_uint4(w[0], w[1], w[2], w[3]);
    return scale;
  }
};

// blockIdx.x: rank in the cluster (a K range); y: tile of 128 columns of D; z: tile of kN rows.
// g.a holds the columns' operand (D's n), g.b the rows' (D's m), which kQuant takes from `rows` instead.
template <typename T, int kN, bool kQuant>
__global__ void __launch_bounds__(kSThreads) mx4_split_kernel(const __grid_constant__ Mx4Gemm g, const Mx4Rows rows) {
  using L = Split<kN>;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::bar_offset);
  uint64_t* empty = full + L::stages;
  uint64_t* tfull = empty + L::stages;
  uint64_t* drain = tfull + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = static_cast<int>(uniform(threadIdx.x >> 5)), lane = threadIdx.x & 31;
  const bool aligned = (smem_u32(smem) & 1023u) == 0;   // the swizzled layouts need 1 KB alignment
  if (threadIdx.x == 0) {
    for (int s = 0; s < L::stages; ++s) {
      mbar_init(&full[s], kQuant ? (rows.by_warp ? 2 : 5) : 1);   // the copies, and the warps that quantize
      mbar_init(&empty[s], 1);
    }
    mbar_init(tfull, 1);
    mbar_init(drain, 1);
    *abort_flag = aligned ? 0 : 1;
    if (!aligned) atomicOr(g.status, kDevInternal);
    fence_mbar_init();
    tma_prefetch_desc(&g.a);
    tma_prefetch_desc(&g.sa);
    if (!kQuant) {
      tma_prefetch_desc(&g.b);
      tma_prefetch_desc(&g.sb);
    }
  }
  if (warp == 5) {
    tmem_alloc<1>(smem_u32(tmem_slot), L::cols);
    tmem_relinquish<1>();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_wait();
  griddep_launch_dependents();
  const uint32_t tmem = uniform(*tmem_slot);
  const uint32_t rank = uniform(cluster_ctarank());
  const uint32_t size = gridDim.x;
  const int kb0 = static_cast<int>(static_cast<int64_t>(g.kblocks) * rank / size);
  const int kb1 = static_cast<int>(static_cast<int64_t>(g.kblocks) * (rank + 1) / size);
  const int n0 = static_cast<int>(blockIdx.y) * 128, m0 = static_cast<int>(blockIdx.z) * kN;
  if (warp == 4) {
    if (elect_one()) {
      int s = 0;
      uint32_t ph = 0;
      int issued = 0;
      bool ok = aligned;
      for (int kb = kb0; kb < kb1 && ok; ++kb) {
        if (!mbar_wait(&empty[s], ph ^ 1u, abort_flag)) {
          ok = false;
          break;
        }
        const uint32_t a0 = smem_u32(smem + s * L::stage_bytes);
        const uint32_t bar = smem_u32(&full[s]);
        mbar_arrive_expect_tx(&full[s], kQuant ? L::a_bytes + kScaleBytes : L::stage_bytes);
        tma_load_2d(a0, &g.a, bar, kb * kOperandRowBytes, n0);
        tma_load_2d(a0 + L::a_bytes + L::b_bytes, &g.sa, bar, kb * (kScaleBytes / 4), n0 >> 7);
        if (!kQuant) {
          tma_load_2d(a0 + L::a_bytes, &g.b, bar, kb * kOperandRowBytes, m0);
          tma_load_2d(a0 + L::a_bytes + L::b_bytes + kScaleBytes, &g.sb, bar, kb * (kScaleBytes / 4), m0 >> 7);
        }
        ++issued;
        if (++s == L::stages) {
          s = 0;
          ph ^= 1u;
        }
      }
      if (!ok && aligned) {
        atomicOr(g.status, kDevTimeout);
        *abort_flag = 1;
      }
      for (int i = issued > L::stages ? issued - L::stages : 0; i < issued; ++i)   // landed before exit
        mbar_wait(&full[i % L::stages], static_cast<uint32_t>((i / L::stages) & 1), nullptr);
    }
  } else if (warp == 5) {
    if (elect_one()) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = aligned;
      for (int kb = kb0; kb < kb1 && ok; ++kb) {
        if (!mbar_wait(&full[s], ph, abort_flag)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t a0 = smem_u32(smem + s * L::stage_bytes);
        const uint32_t sf = a0 + L::a_bytes + L::b_bytes;
        mx4_stage<1, 128, kN, 1>(tmem, a0, a0 + L::a_bytes, sf, sf + kScaleBytes,
                                 tmem + L::acc_cols + s * 2 * kScaleCols, static_cast<uint32_t>(m0 & 127) >> 5, kb == kb0);
        tc_commit<1>(smem_u32(&empty[s]), 0);
        if (++s == L::stages) {
          s = 0;
          ph ^= 1u;
        }
      }
      if (ok) {
        tc_commit<1>(smem_u32(tfull), 0);
      } else if (aligned) {
        atomicOr(g.status, kDevTimeout);
        *abort_flag = 1;
      }
      tc_commit<1>(smem_u32(drain), 0);
      mbar_wait(drain, 0, nullptr);
    }
  } else if (warp < 4) {
    if constexpr (kQuant) {
      // a thread a block of 32 of each 16th row: codes at their swizzled place, the scale byte in its tile
      constexpr int kPer = kN / 16;
      const int b = threadIdx.x & 7;
      const int row = rows.by_warp ? lane >> 3 : static_cast<int>(threadIdx.x) >> 3;
      const int first = rows.by_warp ? warp : 0, step = rows.by_warp ? 4 : 1;
      Block32<T> next[kPer];
      bool ok = aligned, bad = false;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (kb0 + first < kb1) next[i].load(rows, m0 + row + 16 * i, g.M, static_cast<int64_t>(kb0 + first) * kStageK + 32 * b);
      for (int it = first; kb0 + it < kb1; it += step) {
        const int kb = kb0 + it, s = it % L::stages;
        uint4 codes[kPer];
        uint32_t scale[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          scale[i] = next[i].quantize(codes[i]);
          bad |= scale[i] == kScaleNan;
          if (kb + step < kb1) next[i].load(rows, m0 + row + 16 * i, g.M, static_cast<int64_t>(kb + step) * kStageK + 32 * b);
        }
        if (!__all_sync(0xFFFFFFFFu, ok && mbar_wait(&empty[s], (static_cast<uint32_t>(it / L::stages) & 1u) ^ 1u, abort_flag))) {
          ok = false;
          break;
        }
        uint8_t* stage = smem + s * L::stage_bytes + L::a_bytes;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int r = row + 16 * i;
          *reinterpret_cast<uint4*>(stage + r * kOperandRowBytes + ((b ^ (r & 7)) << 4)) = codes[i];
          stage[L::b_bytes + kScaleBytes + (b >> 2) * 512 + r * 16 + (b & 3)] = static_cast<uint8_t>(scale[i]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&full[s]);
      }
      if (bad) atomicOr(g.status, kDevNonFinite);
      if (!ok && aligned && lane == 0) {
        atomicOr(g.status, kDevTimeout);
        *abort_flag = 1;
      }
    }
    // the partial tile, [m][n], in the place of the stages (every MMA has read them)
    if (__all_sync(0xFFFFFFFFu, mbar_wait(tfull, 0, abort_flag))) {
      tc_fence_after();
      float* part = reinterpret_cast<float*>(smem);
      const uint32_t acc = tmem + (static_cast<uint32_t>(warp * 32) << 16);
      constexpr int kC = kN < 32 ? 16 : 32;
#pragma unroll 1
      for (int c = 0; c < kN; c += kC) {
        uint32_t v[kC];
        if constexpr (kC == 16) tmem_ld_32x32b_x16(acc + c, v);
        else tmem_ld_32x32b_x32(acc + c, v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < kC; ++i) part[(c + i) * 128 + warp * 32 + lane] = __uint_as_float(v[i]);
      }
    } else if (lane == 0 && aligned) {
      atomicOr(g.status, kDevTimeout);
      *abort_flag = 1;
    }
    tc_fence_before();
  }
  if (size > 1) cluster_sync();   // every CTA's partial tile is in place
  else __syncthreads();
  if (warp == 5) {
    tc_fence_after();
    tmem_dealloc<1>(tmem, L::cols);
  }
  if (size == 1) sum_ranks<T, kN, 1>(g, smem_u32(smem), rank, m0, n0);
  else if (size == 2) sum_ranks<T, kN, 2>(g, smem_u32(smem), rank, m0, n0);
  else if (size == 4) sum_ranks<T, kN, 4>(g, smem_u32(smem), rank, m0, n0);
  else sum_ranks<T, kN, 8>(g, smem_u32(smem), rank, m0, n0);
}

// ----------------------------------------------------------------------- host side
int64_t mx4_scale_ktiles(int64_t cols);

static int make_map(CUtensorMap* map, CUtensorMapDataType dt, const void* base, int64_t inner, int64_t rows, int64_t pitch,
                    int box_inner, int box_rows, CUtensorMapSwizzle swizzle) {
  auto fn = tensor_map_encoder();
  if (!fn) return fail(SQ_ECUDA, "cuTensorMapEncodeTiled is not available from the driver");
  cuuint64_t gdim[2] = {static_cast<cuuint64_t>(inner), static_cast<cuuint64_t>(rows)};
  cuuint64_t gstride[1] = {static_cast<cuuint64_t>(pitch)};
  cuuint32_t box[2] = {static_cast<cuuint32_t>(box_inner), static_cast<cuuint32_t>(box_rows)};
  cuuint32_t estride[2] = {1, 1};
  const CUresult r = fn(map, dt, 2, const_cast<void*>(base), gdim, gstride, box, estride, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SQ_OK : fail(SQ_ECUDA, "cuTensorMapEncodeTiled failed (%d)", static_cast<int>(r));
}

// an operand's codes [rows, K] and scales; `held` rows of codes and `tiles` row tiles of scales per copy
static int operand_maps(CUtensorMap* codes_map, CUtensorMap* scales_map, const uint8_t* codes, int64_t ld,
                        const uint8_t* scales, int64_t rows, int64_t K, int held, int tiles) {
  int st = make_map(codes_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, (K + 31) / 32 * 16, rows, ld, kOperandRowBytes, held,
                    CU_TENSOR_MAP_SWIZZLE_128B);
  if (st != SQ_OK) return st;
  const int64_t words = mx4_scale_ktiles(K) * 128;
  return make_map(scales_map, CU_TENSOR_MAP_DATA_TYPE_INT32, scales, words, (rows + 127) / 128, words * 4,
                  kScaleBytes / 4, tiles, CU_TENSOR_MAP_SWIZZLE_NONE);
}

// a kernel's shared memory, set once per device
template <typename K>
static int allow_smem(K kernel, size_t bytes, std::atomic<bool>* done, int dev) {
  if (dev >= 0 && dev < 64 && done[dev].load(std::memory_order_acquire)) return SQ_OK;
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
  if (err != cudaSuccess) return cuda_fail(err, "cudaFuncSetAttribute");
  if (dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
  return SQ_OK;
}

template <typename K, typename... Args>
static int launch_clusters(K kernel, dim3 grid, int threads, size_t smem, unsigned cluster, cudaStream_t s, const char* what,
                           const Args&... args) {
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, args...);
  return err == cudaSuccess ? SQ_OK : cuda_fail(err, what);
}

struct Mx4Operand {
  const uint8_t* codes;
  int64_t ld;
  const uint8_t* scales;
};

template <typename T>
static int launch_pair(Mx4Gemm& g, const Mx4Operand& a, const Mx4Operand& b, int64_t K, int dev, int sms, cudaStream_t s) {
  static std::atomic<bool> done[64];
  int st = allow_smem(mx4_pair_kernel<T>, kPSmem, done, dev);
  if (st == SQ_OK) st = operand_maps(&g.a, &g.sa, a.codes, a.ld, a.scales, g.M, K, kPM, 1);
  if (st == SQ_OK) st = operand_maps(&g.b, &g.sb, b.codes, b.ld, b.scales, g.N, K, kPN / 2, 2);
  if (st == SQ_OK && g.tma_out)
    st = make_map(&g.out, sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, g.d, g.N, g.M,
                  g.ldd * static_cast<int64_t>(sizeof(T)), 64 / sizeof(T), 32, CU_TENSOR_MAP_SWIZZLE_64B);
  if (st != SQ_OK) return st;
  g.tiles_m = static_cast<int>((g.M + 2 * kPM - 1) / (2 * kPM));
  g.tiles_n = static_cast<int>((g.N + kPN - 1) / kPN);
  const int64_t tiles = static_cast<int64_t>(g.tiles_m) * g.tiles_n;
  const int pairs = static_cast<int>(tiles < sms / 2 ? tiles : sms / 2);
  return launch_clusters(mx4_pair_kernel<T>, dim3(2 * pairs), kPThreads, kPSmem, 2, s, "mx4_pair_kernel launch", g);
}

// Rows that a product quantizes itself: what one scale operand's first 32 rows hold, for callers without room
// for their codes.  Against the quantizer and the product as two launches (us a call, graphs, weights from
// HBM): 1 row through 4096 x 11008 7.5 for 9.1, 4096 x 4096 5.0 for 7.1; 5 rows 10.9 for 9.4 and 5.9 for 7.7,
// 16 rows 11.4 for 9.6 and 6.3 for 8.0, 32 rows 15.3 for 10.0 and 7.9 for 8.4, 17 rows through 1155 x 1001
// 12.6 for 7.1: one launch is the faster one up to four rows, and further on for some weights alone.
constexpr int kQuantRows = 32;
// whether a product takes the form of few rows: its column tiles are the grid's y
static bool few_rows(int64_t M, int64_t N) { return M <= kQuantRows && (N + 127) / 128 <= 65535; }

// rows: null where both operands are mx4
template <typename T, int kN, bool kQuant>
static int launch_split(Mx4Gemm& g, const Mx4Operand& a, const Mx4Rows* rows, const Mx4Operand& b, int64_t K, int dev, int sms,
                        cudaStream_t s) {
  using L = Split<kN>;
  static std::atomic<bool> done[64];
  int st = allow_smem(mx4_split_kernel<T, kN, kQuant>, L::bytes, done, dev);
  if (st == SQ_OK) st = operand_maps(&g.a, &g.sa, b.codes, b.ld, b.scales, g.N, K, 128, 1);
  if (st == SQ_OK && !kQuant) st = operand_maps(&g.b, &g.sb, a.codes, a.ld, a.scales, g.M, K, kN, 1);
  if (st != SQ_OK) return st;
  g.tiles_n = static_cast<int>((g.N + 127) / 128);
  g.tiles_m = static_cast<int>((g.M + kN - 1) / kN);
  if (kN < 64 && g.tiles_m > 1) return fail(SQ_EUNSUPPORTED, "mx4_split_kernel: %d rows per tile, several tiles", kN);
  const int64_t tiles = static_cast<int64_t>(g.tiles_m) * g.tiles_n;
  unsigned split = 1;
  while (split < 8 && 2 * split <= static_cast<unsigned>(g.kblocks) && tiles * split * 2 <= kSplitBlocks * sms) split *= 2;
  const Mx4Rows none = {nullptr, 0, 0, 0, 0};
  return launch_clusters(mx4_split_kernel<T, kN, kQuant>, dim3(split, g.tiles_n, g.tiles_m), kSThreads, L::bytes, split, s,
                         "mx4_split_kernel launch", g, rows != nullptr ? *rows : none);
}

template <typename T>
static int run_mx4(Mx4Gemm& g, const Mx4Operand& a, const Mx4Operand& b, int64_t K, int dev, int sms, cudaStream_t s) {
  // few rows in the form, and so with the order of sums, of rows that the product quantizes itself; as CTA
  // pairs 32 rows through 4096 x 11008 took 16.4 us for 14.3 (a call alone), 4096 x 65536 43 for 37, 16 rows
  // through 512 x 131072 18.4 for 20.4
  if (few_rows(g.M, g.N)) {
    if (g.M <= 16) return launch_split<T, 16, false>(g, a, nullptr, b, K, dev, sms, s);
    return launch_split<T, 32, false>(g, a, nullptr, b, K, dev, sms, s);
  }
  // CTA pairs from a quarter of the SMs in tiles on.  Pairs and split, us (bf16 out): M x K x N = 1536 x 4096 x 1792 (42
  // tiles) 9.4 and 11.6, 2048 x 11008 x 1280 16.6 and 22.2, 256 x 4096 x 11008 10.3 and 12.4, but 33 x 4096 x
  // 11008 10.6 and 9.4; below, 512 x 4096 x 512 8.4 and 6.9, 128 x 11008 x 4096 16.2 and 12.9, but 1024 x 1024 x 1024
  // (16 tiles) 5.6 and 8.6, 1536 x 4096 x 1536 9.1 and 11.0: the best threshold falls with K
  const int64_t tiles = ((g.M + 255) / 256) * ((g.N + 255) / 256);
  if (tiles >= sms / 4) return launch_pair<T>(g, a, b, K, dev, sms, s);
  // 128 rows where their blocks, each with a K range of a stage at least, fill the SMs, else 64.  No fewer
  // where there are several tiles: a scale operand starts at an even column of tensor memory
  // (32 rows each), so a tile of 16 or 32 rows can only be its scale tile's first.
  const int64_t columns = (g.N + 127) / 128, ranges = g.kblocks < 8 ? g.kblocks : 8;
  if (g.M > 64 && (g.M + 127) / 128 * columns * ranges >= sms) return launch_split<T, 128, false>(g, a, nullptr, b, K, dev, sms, s);
  return launch_split<T, 64, false>(g, a, nullptr, b, K, dev, sms, s);
}

template <typename T>
static int run_mx4_rows(Mx4Gemm& g, const Mx4Rows& rows, const Mx4Operand& b, int dev, int sms, cudaStream_t s) {
  const Mx4Operand none = {nullptr, 0, nullptr};
  return g.M <= 16 ? launch_split<T, 16, true>(g, none, &rows, b, rows.K, dev, sms, s)
                   : launch_split<T, 32, true>(g, none, &rows, b, rows.K, dev, sms, s);
}

// what both products check of their weights and their output
static int check_mx4(const char* who, const uint8_t* b_codes, int64_t ldb, const uint8_t* b_scales, int64_t M, int64_t N,
                     int64_t K, const void* d, int dtype, int64_t ldd, const int32_t* dev_status) {
  constexpr int64_t kMax = (int64_t(1) << 31) - 256;
  if (M > kMax || N > kMax || K > kMax || ((M + 255) / 256) * ((N + 255) / 256) > kMax)
    return fail(SQ_EUNSUPPORTED, "%s: a size is above 2^31 - 256, or more than 2^31 - 256 tiles", who);
  if (d == nullptr || dev_status == nullptr || ldd < N) return fail(SQ_EINVAL, "%s: NULL argument, or the output's ld < N", who);
  if (reinterpret_cast<uintptr_t>(d) % dtype_bytes(dtype)) return fail(SQ_EALIGN, "%s: the output is not aligned to its type", who);
  if (K == 0) return SQ_OK;
  if (b_codes == nullptr || b_scales == nullptr) return fail(SQ_EINVAL, "%s: NULL argument", who);
  if (ldb < (K + 31) / 32 * 16) return fail(SQ_EINVAL, "%s: a leading dimension < 16 ceil(K / 32)", who);
  if (!aligned16(b_codes) || !aligned16(b_scales) || ldb % 16)
    return fail(SQ_EALIGN, "%s: codes, scales and leading dimensions need 16-byte alignment", who);
  return SQ_OK;
}

static Mx4Gemm gemm_args(int64_t M, int64_t N, int64_t K, void* d, int esize, int64_t ldd, int32_t* dev_status) {
  Mx4Gemm g;
  memset(&g, 0, sizeof(g));
  g.M = M, g.N = N, g.d = d, g.ldd = ldd, g.status = dev_status;
  g.kblocks = static_cast<int>((K + kStageK - 1) / kStageK);
  g.tma_out = aligned16(d) && (ldd * esize) % 16 == 0;
  return g;
}

static int zero_output(void* d, int64_t M, int64_t N, int64_t ldd, int esize, cudaStream_t s) {   // the empty sum
  const cudaError_t err = cudaMemset2DAsync(d, static_cast<size_t>(ldd) * esize, 0, static_cast<size_t>(N) * esize, static_cast<size_t>(M), s);
  return err == cudaSuccess ? SQ_OK : cuda_fail(err, "cudaMemset2DAsync");
}

}  // namespace sq

using namespace sq;

extern "C" sq_status shiftquant_mx4_gemm(const uint8_t* a_codes, int64_t lda, const uint8_t* a_scales, const uint8_t* b_codes,
                                         int64_t ldb, const uint8_t* b_scales, int64_t M, int64_t N, int64_t K, void* d,
                                         int dtype, int64_t ldd, int32_t* dev_status, void* stream) {
  fail(SQ_OK, "");
  if (!dtype_ok(dtype)) return fail(SQ_EINVAL, "mx4_gemm: bad dtype %d", dtype);
  if (M < 0 || N < 0 || K < 0) return fail(SQ_EINVAL, "mx4_gemm: negative size");
  if (M == 0 || N == 0) return SQ_OK;
  const int st = check_mx4("mx4_gemm", b_codes, ldb, b_scales, M, N, K, d, dtype, ldd, dev_status);
  if (st != SQ_OK) return st;
  const int esize = dtype_bytes(dtype);
  cudaStream_t s = as_stream(stream);
  if (K == 0) return zero_output(d, M, N, ldd, esize, s);
  if (a_codes == nullptr || a_scales == nullptr) return fail(SQ_EINVAL, "mx4_gemm: NULL argument");
  if (lda < (K + 31) / 32 * 16) return fail(SQ_EINVAL, "mx4_gemm: lda < 16 ceil(K / 32)");
  if (!aligned16(a_codes) || !aligned16(a_scales) || lda % 16)
    return fail(SQ_EALIGN, "mx4_gemm: codes, scales and leading dimensions need 16-byte alignment");
  int dev = 0;
  const int sms = device_sms(&dev);
  if (sms <= 0) return fail(SQ_ECUDA, "mx4_gemm: no current CUDA device");
  Mx4Gemm g = gemm_args(M, N, K, d, esize, ldd, dev_status);
  const Mx4Operand a = {a_codes, lda, a_scales}, b = {b_codes, ldb, b_scales};
  if (dtype == SQ_F32) return run_mx4<float>(g, a, b, K, dev, sms, s);
  if (dtype == SQ_BF16) return run_mx4<__nv_bfloat16>(g, a, b, K, dev, sms, s);
  return run_mx4<__half>(g, a, b, K, dev, sms, s);
}

extern "C" sq_status shiftquant_mx4_linear(const void* x, int dtype, int64_t M, int64_t K, int64_t ld_x, const uint8_t* w_codes_t,
                                           int64_t ld_w, const uint8_t* w_scales_t, int64_t N, void* y, int64_t ld_y,
                                           uint8_t* x_codes, int64_t ld_x_codes, uint8_t* x_scales, int32_t* dev_status,
                                           void* stream) {
  fail(SQ_OK, "");
  if (!dtype_ok(dtype)) return fail(SQ_EINVAL, "mx4_linear: bad dtype %d", dtype);
  if (M < 0 || N < 0 || K < 0) return fail(SQ_EINVAL, "mx4_linear: negative size");
  if (M == 0 || N == 0) return SQ_OK;
  int st = check_mx4("mx4_linear", w_codes_t, ld_w, w_scales_t, M, N, K, y, dtype, ld_y, dev_status);
  if (st != SQ_OK) return st;
  const int esize = dtype_bytes(dtype);
  cudaStream_t s = as_stream(stream);
  if (K == 0) return zero_output(y, M, N, ld_y, esize, s);
  if (x == nullptr || ld_x < K) return fail(SQ_EINVAL, "mx4_linear: NULL x or ld_x < K");
  if (reinterpret_cast<uintptr_t>(x) % esize) return fail(SQ_EALIGN, "mx4_linear: x is not aligned to its type");
  if (!few_rows(M, N)) {
    if (x_codes == nullptr || x_scales == nullptr)
      return fail(SQ_EINVAL, "mx4_linear: more than %d rows need x_codes and x_scales", kQuantRows);
    st = shiftquant_mx4_quantize(x, dtype, M, K, ld_x, SQ_ROUND_NEAREST_EVEN, 0, 0, x_codes, ld_x_codes, x_scales, nullptr, 0,
                                 nullptr, dev_status, stream);
    if (st != SQ_OK) return st;
    return shiftquant_mx4_gemm(x_codes, ld_x_codes, x_scales, w_codes_t, ld_w, w_scales_t, M, N, K, y, dtype, ld_y, dev_status,
                               stream);
  }
  int dev = 0;
  const int sms = device_sms(&dev);
  if (sms <= 0) return fail(SQ_ECUDA, "mx4_linear: no current CUDA device");
  Mx4Gemm g = gemm_args(M, N, K, y, esize, ld_y, dev_status);
  const Mx4Operand b = {w_codes_t, ld_w, w_scales_t};
  const Mx4Rows rows = {x, ld_x, K, aligned16(x) && (ld_x * esize) % 16 == 0, M <= 4};
  if (dtype == SQ_F32) return run_mx4_rows<float>(g, rows, b, dev, sms, s);
  if (dtype == SQ_BF16) return run_mx4_rows<__nv_bfloat16>(g, rows, b, dev, sms, s);
  return run_mx4_rows<__half>(g, rows, b, dev, sms, s);
}
