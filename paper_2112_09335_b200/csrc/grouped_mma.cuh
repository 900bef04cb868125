// Products on the 5th-generation tensor cores for matrices of many kinds: the loop that all kernels of grouped.cu share.
//
// A block owns one SM and walks over work items, each a tile of 128 rows x kBN columns of some D = A B with a reduction of any length.
//   warps 0-7    epilogue: tensor memory -> registers -> sums of segments -> result
//   warp 8       matrix instructions (one lane issues)
//   warp 9       copies of operand tiles by TMA, or warps 9-16: operand tiles through registers
// Operand tiles are 64 steps of the reduction wide and lie in shared memory with the 128-byte swizzle, K-major (a row of the tile is
// 128 bytes of the reduction) or MN-major (a row is one step of the reduction, 128 bytes of the tile's rows or columns; tiles of more than 64 are
// groups of 64, 8192 bytes apart), whichever way the matrix lies in memory: nothing is ever transposed by hand.
//
// Operands have kParts parts of 16 bits:
//   1   the operand itself
//   2   x = hi + 2^-11 lo, halves (orthogonalised updates: entries bounded, fixed scales)
//   3   x = b0 + b1 + b2, bf16, each part what the last ones leave, cut after 8 bits: 24 bits in all, so the sum is x exactly, with the
//       exponents of fp32 (no scales to keep, nothing for one large element to drown).  Products: b0 b0 and, apart, b0 b1 + b1 b0 + b1 b1 + b0 b2 + b2 b0;
//       what is left out is below 2^-21 of |x||y|, 2^-24 in the mean.
// The main product and the corrections have accumulators of their own.  The tensor core cuts an accumulator toward zero at every
// instruction; an error that grows with the length of the reduction is kept out by taking the accumulator into registers after
// every segment of 256 steps, where segments are added in fp32 (rounded to nearest).  Two accumulators alternate, so that instructions of a segment run
// beside the reading of the one before it.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gemm_tc.cuh"
#include "grouped_plan.hpp"

namespace gcn_admm_grouped {

using gtc::smem_u32;

constexpr int kBM = 128, kBK = 64;   // rows of a tile; reduction steps of a chunk
constexpr int kATile = kBM * kBK * 2;              // bytes of one part of an operand tile of A
constexpr int kGroup64 = kBK * 128;                // bytes between groups of 64 in an MN-major tile
constexpr int kEpiWarps = 8, kMmaWarp = kEpiWarps, kFirstProducer = kMmaWarp + 1;
constexpr int kBuffer = 2048;                      // bytes of an epilogue warp's buffer: 32 rows of 64

template <int PARTS, int BN, bool TMA>
struct Geometry {
  static constexpr int kBTile = BN * kBK * 2;
  static constexpr int kStage = PARTS * (kATile + kBTile);
  static constexpr int kStages = 196608 / kStage < 8 ? 196608 / kStage : 8;
  static constexpr int kProducers = TMA ? 1 : 8;               // warps
  static constexpr int kThreads = (kFirstProducer + kProducers) * 32;
  static constexpr int kAccs = PARTS > 1 ? 2 : 1;              // accumulators of a set
  static constexpr uint32_t kTmemCols = 2 * kAccs * BN;
  static constexpr int kBuffersAt = kStages * kStage, kTablesAt = kBuffersAt + kEpiWarps * kBuffer;
  static_assert(kTmemCols >= 32 && kTmemCols <= 512, "tensor memory");
};

// Byte offsets of the 16-byte unit `u` (eight elements) of a tile's row.
__device__ __forceinline__ uint32_t unit_k(int row, int u) { return (uint32_t)row * 128u + (uint32_t)((u ^ (row & 7)) << 4); }
__device__ __forceinline__ uint32_t unit_mn(int step, int u) { return (uint32_t)(u >> 3) * kGroup64 + (uint32_t)step * 128u + (uint32_t)(((u & 7) ^ (step & 7)) << 4); }

// Operand descriptors, version 1, SWIZZLE_128B.  Low word: address and leading byte offset (MN-major: between groups of 64; K-major: unused); high
// word: stride byte offset, between groups of eight 128-byte rows.  Both kinds have the same high word.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
template <bool MN>
__device__ __forceinline__ uint32_t desc_lo(uint32_t address) { return ((address >> 4) & 0x3fffu) | ((MN ? kGroup64 >> 4 : 1u) << 16); }
// 16 steps of the reduction, in units of 16 bytes: 32 bytes of a row, or two groups of eight rows
template <bool MN>
constexpr uint32_t kStep16 = MN ? 2048u >> 4 : 32u >> 4;

// Instruction descriptor: D fp32, A and B both of bf16 or both of fp16, M = 128; N is added per item.
template <bool A_MN, bool B_MN>
__device__ __forceinline__ uint32_t instruction(bool bf16) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | ((uint32_t)(kBM >> 4) << 24);
}
__device__ __forceinline__ void mma(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %6};\n\t"
      "mov.b64 db, {%2, %6};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, {%5, %5, %5, %5}, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(0u), "r"(kDescHi)
      : "memory");
}
__device__ __forceinline__ void copy_2d(uint32_t to, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void copy_3d(uint32_t to, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}

// What a block needs beside its operands.
struct Bars {
  uint64_t full[8], empty[8], acc_full[2], acc_empty[2], drain;
};

// NC columns of 32 rows, one row a lane, to `out` (element (0, 0) of the warp's part), the first rows_left rows and cols_left columns of them.
// Through a buffer, so that what leaves a warp at once are 64 bytes of each of eight rows, whole sectors.  vec: rows of `out` start on 16-byte boundaries.
template <int NC>
__device__ __forceinline__ void store_rows(const float (&acc)[NC], uint8_t* buf, void* out, long long ld, int out_type, bool vec, int rows_left, int cols_left) {
  const int lane = threadIdx.x & 31, q = lane & 3;
  uint8_t* const mine = buf + lane * 64;
  const int turn = (lane >> 1) & 3;
  if (out_type == kF32) {
#pragma unroll
    for (int c0 = 0; c0 < NC; c0 += 16) {
      if (c0 < cols_left) {
#pragma unroll
        for (int u = 0; u < 4; ++u) *reinterpret_cast<float4*>(mine + ((u ^ turn) << 4)) = make_float4(acc[c0 + 4 * u], acc[c0 + 4 * u + 1], acc[c0 + 4 * u + 2], acc[c0 + 4 * u + 3]);
        __syncwarp();
        const int col = c0 + 4 * q, some = cols_left - col;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 8 * i + (lane >> 2);
          const float4 v = *reinterpret_cast<const float4*>(buf + r * 64 + ((q ^ ((r >> 1) & 3)) << 4));
          float* const at = static_cast<float*>(out) + r * ld + col;
          if (r < rows_left && some > 0) {
            if (vec && some >= 4) {
              *reinterpret_cast<float4*>(at) = v;
            } else {
              at[0] = v.x;
              if (some > 1) at[1] = v.y;
              if (some > 2) at[2] = v.z;
              if (some > 3) at[3] = v.w;
            }
          }
        }
        __syncwarp();
      }
    }
  } else {
#pragma unroll
    for (int c0 = 0; c0 < NC; c0 += 32) {
      if (c0 < cols_left) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = acc[c0 + 8 * u + 2 * e], y = acc[c0 + 8 * u + 2 * e + 1];
            if (out_type == kBf16) {
              const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
              w[e] = *reinterpret_cast<const uint32_t*>(&b);
            } else {
              const __half2 b = __floats2half2_rn(x, y);
              w[e] = *reinterpret_cast<const uint32_t*>(&b);
            }
          }
          *reinterpret_cast<uint4*>(mine + ((u ^ turn) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        __syncwarp();
        const int col = c0 + 8 * q, some = cols_left - col;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 8 * i + (lane >> 2);
          const uint4 v = *reinterpret_cast<const uint4*>(buf + r * 64 + ((q ^ ((r >> 1) & 3)) << 4));
          unsigned short* const at = static_cast<unsigned short*>(out) + r * ld + col;
          if (r < rows_left && some > 0) {
            if (vec && some >= 8) {
              *reinterpret_cast<uint4*>(at) = v;
            } else {
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (e < some) at[e] = (unsigned short)(w[e >> 1] >> (16 * (e & 1)));
            }
          }
        }
        __syncwarp();
      }
    }
  }
}

// Eight elements of a row on their way from memory to an operand tile, those from `valid` on zero.  vec: the row's units are 16-byte aligned.
template <typename T>
struct Raw;
template <>
struct Raw<float> {
  float x[8];
  __device__ __forceinline__ void load(const float* p, int valid, bool vec) {
    if (vec && valid >= 8) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = e < valid ? __ldg(p + e) : 0.f;
    }
  }
  // The three parts, `part` bytes apart: each the upper half of what the last ones leave (differences are exact).
  __device__ __forceinline__ void store(uint8_t* at, int part) const {
    uint32_t w[3][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float u = x[2 * e], v = x[2 * e + 1];
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        w[k][e] = __byte_perm(__float_as_uint(u), __float_as_uint(v), 0x7632);
        u -= __uint_as_float(__float_as_uint(u) & 0xffff0000u);
        v -= __uint_as_float(__float_as_uint(v) & 0xffff0000u);
      }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(at + k * part) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
  }
};
template <>
struct Raw<unsigned short> {
  uint4 x;
  __device__ __forceinline__ void load(const unsigned short* p, int valid, bool vec) {
    if (vec && valid >= 8) {
      x = __ldg(reinterpret_cast<const uint4*>(p));
    } else {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = (2 * e < valid ? (uint32_t)__ldg(p + 2 * e) : 0u) | (2 * e + 1 < valid ? (uint32_t)__ldg(p + 2 * e + 1) << 16 : 0u);
      x = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  __device__ __forceinline__ void store(uint8_t* at, int) const { *reinterpret_cast<uint4*>(at) = x; }
};

// The shared loop.  A job J says what the items are, where operand tiles come from and what becomes of a tile's sums:
//   J::Args, kParts, kBN, kAMn, kBMn, kTma, kSegment (chunks), kMeets (finish() has barriers of the epilogue warps)
//   J(args, tables)                   built by every thread; setup(): tables in shared memory, by the whole block, between barriers
//   bool item(unsigned i, Item&)      the i-th item, false behind the last; Item has chunks (of the reduction, maybe none), n (columns) and tail
//                                     (steps of the last chunk that count, where rows behind them hold other data; else 64)
//   copy(item, chunk, tile, bar)      kTma: issues the copies of a chunk and announces their bytes
//   load(item, chunk, thread, raw_a, raw_b)   otherwise
//   finish(item, acc, buf, warp)      the sums of this warp's rows and columns; by all epilogue warps
template <class J>
__global__ void __launch_bounds__(Geometry<J::kParts, J::kBN, J::kTma>::kThreads, 1) k_products(const __grid_constant__ typename J::Args args) {
  using G = Geometry<J::kParts, J::kBN, J::kTma>;
  constexpr int S = G::kStages, BN = J::kBN, PARTS = J::kParts, kSegment = J::kSegment;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) Bars bars;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t base = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t full = smem_u32(bars.full), empty = smem_u32(bars.empty), acc_full = smem_u32(bars.acc_full), acc_empty = smem_u32(bars.acc_empty);
  if (tid == 0) {
    for (int s = 0; s < S; ++s) {
      gtc::mbar_init(full + 8 * s, G::kProducers);
      gtc::mbar_init(empty + 8 * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      gtc::mbar_init(acc_full + 8 * a, 1);
      gtc::mbar_init(acc_empty + 8 * a, kEpiWarps);
    }
    gtc::mbar_init(smem_u32(&bars.drain), 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(G::kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  gtc::enter_kernel();
  J job(args, smem + G::kTablesAt);
  job.setup();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  volatile int* const abortp = &abort_flag;
  int copies = 0;   // stages this thread has started copies into
  typename J::Item it;

  if (warp >= kFirstProducer) {
    int slot = 0;
    uint32_t parity = 1;   // a fresh barrier passes a wait on parity 1
    if constexpr (J::kTma) {
      if (lane == 0) {
        bool ok = true;
        for (unsigned i = blockIdx.x; ok && job.item(i, it); i += gridDim.x) {
          for (int c = 0; c < it.chunks; ++c) {
            ok = gtc::mbar_wait_abortable(empty + 8 * slot, parity, abortp);
            if (!ok) break;
            job.copy(it, c, base + (uint32_t)slot * G::kStage, full + 8 * slot);
            ++copies;
            if (++slot == S) { slot = 0; parity ^= 1u; }
          }
        }
      }
    } else {
      using R = Raw<typename J::T>;
      R a[kBM * 8 / 256], b[BN * 8 / 256];
      const int t = tid - kFirstProducer * 32;
      unsigned i = blockIdx.x;
      int c = 0;
      bool more = job.item(i, it);
      const auto settle = [&] {   // on to the next item where this one has no chunk left
        while (more && c >= it.chunks) {
          i += gridDim.x;
          c = 0;
          more = job.item(i, it);
        }
      };
      settle();
      if (more) job.load(it, c, t, a, b);
      while (more) {
        if (!__all_sync(0xffffffffu, gtc::mbar_wait_abortable(empty + 8 * slot, parity, abortp))) break;
        uint8_t* const st = smem + (size_t)slot * G::kStage;
#pragma unroll
        for (int u = 0; u < kBM * 8 / 256; ++u) {
          const int at = t + 256 * u;
          a[u].store(st + (J::kAMn ? unit_mn(at / (kBM / 8), at % (kBM / 8)) : unit_k(at >> 3, at & 7)), kATile);
        }
#pragma unroll
        for (int u = 0; u < BN * 8 / 256; ++u) {
          const int at = t + 256 * u;
          b[u].store(st + PARTS * kATile + (J::kBMn ? unit_mn(at / (BN / 8), at % (BN / 8)) : unit_k(at >> 3, at & 7)), G::kBTile);
        }
        ++c;
        settle();
        if (more) job.load(it, c, t, a, b);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        gtc::mbar_arrive_warp(full + 8 * slot);
        if (++slot == S) { slot = 0; parity ^= 1u; }
      }
    }
  } else if (warp == kMmaWarp) {
    const uint32_t kind = instruction<J::kAMn, J::kBMn>(job.bf16());
    int slot = 0, set = 0;
    uint32_t parity = 0, acc_parity = 1;
    bool ok = true;
    for (unsigned i = blockIdx.x; ok && job.item(i, it); i += gridDim.x) {
      const uint32_t idesc = kind | (uint32_t)((min(it.n, BN) + 15) / 16 * 2) << 17;
      for (int c = 0; c < it.chunks; ++c) {
        const bool first = c % kSegment == 0, last = c + 1 == it.chunks;
        ok = __all_sync(0xffffffffu, (!first || gtc::mbar_wait_abortable(acc_empty + 8 * set, acc_parity, abortp)) &&
                                         gtc::mbar_wait_abortable(full + 8 * slot, parity, abortp));
        if (!ok) break;
        const uint32_t at = base + (uint32_t)slot * G::kStage;
        int steps = kBK / 16;
        if (J::kTma && J::kAMn && last && it.tail < kBK) {
          // rows of the next group came with the copy: the steps that are still read are cleared in both operands
          steps = (it.tail + 15) / 16;
          const int clear = steps * 16 - it.tail, groups = kBM / 64 + BN / 64;
          for (int u = lane; u < clear * groups * 8; u += 32) {
            const int row = it.tail + (u >> 3) % clear, group = (u >> 3) / clear;
            *reinterpret_cast<uint4*>(smem + (size_t)slot * G::kStage + group * kGroup64 + row * 128 + (u & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (lane == 0) {
          const uint32_t a = desc_lo<J::kAMn>(at), b = desc_lo<J::kBMn>(at + PARTS * kATile);
          constexpr uint32_t pa = kATile >> 4, pb = G::kBTile >> 4, oa = kStep16<J::kAMn>, ob = kStep16<J::kBMn>;
          const uint32_t d = tmem + (uint32_t)(set * G::kAccs * BN);
          for (int k = 0; k < steps; ++k) {
            const uint32_t ak = a + k * oa, bk = b + k * ob, go_on = !first || k > 0;
            mma(d, ak, bk, idesc, go_on);
            if constexpr (PARTS > 1) {
              mma(d + BN, ak, bk + pb, idesc, go_on);
              mma(d + BN, ak + pa, bk, idesc, 1u);
            }
            if constexpr (PARTS > 2) {
              mma(d + BN, ak + pa, bk + pb, idesc, 1u);
              mma(d + BN, ak, bk + 2 * pb, idesc, 1u);
              mma(d + BN, ak + 2 * pa, bk, idesc, 1u);
            }
          }
          gtc::mma_commit(empty + 8 * slot);
          if (last || c % kSegment == kSegment - 1) gtc::mma_commit(acc_full + 8 * set);
        }
        __syncwarp();
        if (last || c % kSegment == kSegment - 1) {
          if (set == 1) acc_parity ^= 1u;
          set ^= 1;
        }
        if (++slot == S) { slot = 0; parity ^= 1u; }
      }
    }
  } else {
    constexpr int NC = BN / 2;   // columns of a warp
    constexpr float kCorrection = PARTS == 2 ? 0x1p-11f : 1.f;
    uint8_t* const buf = smem + G::kBuffersAt + warp * kBuffer;
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)((warp >> 2) * NC);
    int set = 0;
    uint32_t parity = 0;
    bool ok = true;
    for (unsigned i = blockIdx.x; ok && job.item(i, it); i += gridDim.x) {
      float acc[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[c] = 0.f;
      const bool mine = (warp >> 2) * NC < it.n;   // whether any of the warp's columns are asked for
      for (int c = 0; c < it.chunks; c += kSegment) {
        ok = __all_sync(0xffffffffu, gtc::mbar_wait_abortable(acc_full + 8 * set, parity, abortp));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (mine) {
          const uint32_t from = lanes + (uint32_t)(set * G::kAccs * BN);
#pragma unroll
          for (int c0 = 0; c0 < NC; c0 += 16) {
            uint32_t v[16], w[16];
            GTC_TMEM_LD16(v, from + c0);
            if (PARTS > 1) GTC_TMEM_LD16(w, from + BN + c0);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[c0 + e] += PARTS > 1 ? fmaf(__uint_as_float(w[e]), kCorrection, __uint_as_float(v[e])) : __uint_as_float(v[e]);
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        gtc::mbar_arrive_warp(acc_empty + 8 * set);
        if (set == 1) parity ^= 1u;
        set ^= 1;
      }
      // where epilogue warps meet in finish(), those that gave up and those that did not leave together
      if constexpr (J::kMeets) ok = gtc::all_agree(ok, kEpiWarps * 32);
      if (ok) job.finish(it, acc, buf, warp);
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (abort_flag) {   // what is still in flight is waited for before shared and tensor memory are let go
    if (tid == 0) atomicOr(job.error_flag(), 1);
    if (warp == kFirstProducer && lane == 0 && J::kTma) gtc::drain_copies(full, S, copies);
    if (warp == kMmaWarp && lane == 0) gtc::drain_mmas(smem_u32(&bars.drain));
    __syncthreads();
  }
  if (warp == kMmaWarp) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(G::kTmemCols) : "memory");
  }
}

}  // namespace gcn_admm_grouped
