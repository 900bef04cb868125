// Products on the 5th-generation tensor cores for matrices of many kinds: the loop that all kernels of grouped.cu share.
//
// A block owns one SM and walks over work items, each a tile of 128 rows x kBN columns of some D = A B with a reduction of any length.
//   warps 0-7    epilogue: tensor memory -> registers -> sums of segments -> result
//   warp 8       matrix instructions (one lane issues)
//   warp 9       copies of operand tiles by TMA;  warp 10: clears what they bring from behind the end of a group
//   warps 12-19  where an operand has to be split or does not lie on 16-byte boundaries: its tiles, through registers
// (Issuing behind a producer's part of a chunk, in 16 warps, held up that warp and with it all others: 24 instructions take 2600 clocks to
// be accepted.)
// Operand tiles are 64 steps of the reduction wide and lie in shared memory with the 128-byte swizzle, K-major (a row of the tile is
// 128 bytes of the reduction) or MN-major (a row is one step of the reduction, 128 bytes of the tile's rows or columns; tiles of more than 64 are
// groups of 64, 8192 bytes apart), whichever way the matrix lies in memory: nothing is ever transposed by hand.
//
// kPair: two blocks on neighbouring SMs (a cluster) work on one tile of 256 rows, each with 128 of the rows of A, half the columns of B and the
// sums of its rows; one of them issues instructions for both.  A block alone moves 48 KB into shared memory and 48 KB out of it for the
// 512 clocks of a chunk's instructions (128 x 256), 192 bytes a clock where it has 128; in a pair it is 32 and 32.
//
// Operands have kParts parts of 16 bits:
//   1   the operand itself
//   2   x = hi + 2^-11 lo, halves (orthogonalised updates: entries bounded, a scale for every matrix)
//   3   x = b0 + b1 + b2, bf16, each part what the last ones leave, cut after 8 bits: 24 bits in all, with the exponents of fp32 (no scales to
//       keep, nothing for one large element to drown): the sum is x exactly from 2^-110 on; below, parts end at 2^-133, the last bit of a bf16.
//       Products: b0 b0 and, apart, b0 b1 + b1 b0 + b1 b1 + b0 b2 + b2 b0; what is left out, b1 b2 + b2 b1 and b2 b2, has the sign of the product and is
//       below 2^-21 of |x||y|, 2^-24 in the mean.
// The main product and the corrections have accumulators of their own.  The tensor core cuts an accumulator toward zero at every
// instruction; an error that grows with the length of the reduction is kept out by taking the accumulator into registers after
// every segment of 256 steps or fewer (1024 where a result of 16 bits would not show it), where segments are added in fp32, rounded to nearest.  Two accumulators alternate, so that instructions of a segment run
// beside the reading of the one before it.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gemm_tc.cuh"
#include "grouped_plan.hpp"
#include "grouped_words.hpp"

namespace gcn_admm_grouped {

using gtc::smem_u32;

constexpr int kBM = 128, kBK = 64;   // rows of a tile; reduction steps of a chunk
constexpr int kATile = kBM * kBK * 2;              // bytes of one part of an operand tile of A
constexpr int kGroup64 = kBK * 128;                // bytes between groups of 64 in an MN-major tile
constexpr int kEpiWarps = 8, kMmaWarp = kEpiWarps, kFirstLoader = kMmaWarp + 4;
constexpr int kBuffer = 2048;                      // bytes of an epilogue warp's buffer: 32 rows of 64

template <int PARTS, int BN, bool TMA, bool PAIR>
struct Geometry {
  static constexpr int kBCols = PAIR ? BN / 2 : BN;            // columns of B that this block's shared memory holds
  static constexpr int kBTile = kBCols * kBK * 2;
  static constexpr int kStage = PARTS * (kATile + kBTile);
  static constexpr int kStages = 196608 / kStage < 8 ? 196608 / kStage : 8;
  static constexpr int kProducers = TMA ? 1 : 8;               // warps
  static constexpr int kThreads = (kMmaWarp + 4 + (TMA ? 0 : kProducers)) * 32;
  static constexpr int kAccs = PARTS > 1 ? 2 : 1;              // accumulators of a set
  static constexpr uint32_t kTmemCols = 2 * kAccs * BN;
  static constexpr int kBuffersAt = kStages * kStage, kTablesAt = kBuffersAt + kEpiWarps * kBuffer;
  static_assert(kTmemCols >= 32 && kTmemCols <= 512, "tensor memory");
  static_assert(PARTS == 1 || 2 * BN <= 256, "columns of an instruction");
  static_assert(!PAIR || (PARTS == 1 && TMA && BN == 256), "the pair has one layout");
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

// Instruction descriptor: D fp32, A and B both of bf16 or both of fp16, M = 128 (of a pair 256); N is added per item.
template <bool A_MN, bool B_MN, bool PAIR>
__device__ __forceinline__ uint32_t instruction(bool bf16) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | ((uint32_t)((PAIR ? 2 * kBM : kBM) >> 4) << 24);
}
__device__ __forceinline__ void mma(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %5};\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHi)
      : "memory");
}
// The same for a pair of blocks, M = 256: by one thread of the first block, for both.
__device__ __forceinline__ void mma_pair(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %5};\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHi)
      : "memory");
}
// Arrives at the barrier of this address in both blocks when all instructions issued so far are done.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((unsigned short)3) : "memory");
}
__device__ __forceinline__ uint32_t of_first_block(uint32_t address) {
  uint32_t there;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(there) : "r"(address));
  return there;
}
__device__ __forceinline__ void meet_pair() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// One arrival for the whole warp at a barrier of the pair's first block.  What it orders are reads of tensor memory (tcgen05 fences) or, `wrote`, stores
// to shared memory that the other block's instructions will read.  (Release and acquire at cluster scope cost hundreds of clocks: with them on every arrival and
// wait, 32768 x 2048 x 2048 took 540 us instead of 296.)
__device__ __forceinline__ void arrive_at_first(uint32_t there, bool wrote) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) {
    if (wrote) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(there) : "memory");
    else asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(there) : "memory");
  }
}
// Of a phase that is known to be over: what the other block stored before it arrived is seen.
__device__ __forceinline__ void acquire_cluster(uint32_t bar, uint32_t parity) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%0], %1;\n\t}"
      ::"r"(bar), "r"(parity)
      : "memory");
}
// Announces `bytes` at `bar` and arrives there; where THERE, the first block's.
template <bool THERE>
__device__ __forceinline__ void expect(uint32_t bar, uint32_t bytes) {
  if constexpr (THERE) asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
  else asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Copies of a box into this block's shared memory; where PAIR, `bar` may be the first block's.
template <bool PAIR>
__device__ __forceinline__ void copy_2d(uint32_t to, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if constexpr (PAIR)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void copy_3d(uint32_t to, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if constexpr (PAIR)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}

struct Nothing {};

// What a block needs beside its operands.
struct Bars {
  uint64_t full[8], empty[8], acc_full[2], acc_empty[2], tail[8], drain;
};

// Rows of what a warp leaves, one row a lane, 64 bytes of each at a time.  Where rows lie on 32-byte boundaries every lane writes whole sectors of its own row, at
// once.  Otherwise they go through a buffer in shared memory, so that what leaves a warp at once are 64 bytes of each of eight rows; where they
// do not lie on 16-byte boundaries either, or end inside of 16 bytes, a warp writes 16 columns (fp32) or 32 of two rows at once, halves two by
// two in whichever way they are aligned (13752 x 767 halves, with their product: 87 us where each lane wrote eight halves one by one, 42 us
// so).  Whole
// sectors are not kept in L1 (weight gradients of 16384 x 2048 x 1024 to fp32: 111 -> 101 us); what goes through the buffer leaves by ordinary stores.  The buffer is not for all: while a pair multiplies, its operands alone take 128 bytes a clock from and to shared memory, all there are.
__device__ __forceinline__ void store32(void* at, const uint4& a, const uint4& b) {
  asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}
__device__ __forceinline__ void load32(const void* at, uint32_t* w) {
  asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(at)
               : "memory");
}
__device__ __forceinline__ uint32_t pack(int type, float x, float y) {
  if (type == kBf16) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&b);
  }
  const __half2 b = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&b);
}
__device__ __forceinline__ uint4 words(float x, float y, float z, float w) {
  return make_uint4(__float_as_uint(x), __float_as_uint(y), __float_as_uint(z), __float_as_uint(w));
}
struct RowStore {
  uint8_t* buf;
  uint8_t* out;
  long long ld;
  int size, rows_left, cols_left;   // size: bytes of an element
  bool direct, units;               // rows of whole sectors of 32 bytes, of whole units of 16
  // boundary: bytes that every row starts at a multiple of, 32, 16 or less
  __device__ __forceinline__ RowStore(uint8_t* buf_, void* out_, long long ld_, int size_, int boundary, int rows_left_, int cols_left_)
      : buf(buf_), out(static_cast<uint8_t*>(out_)), ld(ld_), size(size_), rows_left(rows_left_), cols_left(cols_left_),
        direct(boundary >= 32 && (cols_left_ * size_ & 31) == 0), units(boundary >= 16 && (cols_left_ * size_ & 15) == 0) {}
  __device__ __forceinline__ uint8_t* unit(int r, int u) const { return buf + r * 64 + ((u ^ ((r >> 1) & 3)) << 4); }
  // 64 bytes of this lane's row, from column c0 on.
  __device__ __forceinline__ void put(int c0, const uint4& w0, const uint4& w1, const uint4& w2, const uint4& w3) const {
    const int lane = threadIdx.x & 31, q = lane & 3, r0 = lane >> 2;
    if (direct) {
      uint8_t* const at = out + (lane * ld + c0) * size;
      if (lane < rows_left) store32(at, w0, w1);
      if (lane < rows_left && c0 * size + 32 < cols_left * size) store32(at + 32, w2, w3);
      return;
    }
    *reinterpret_cast<uint4*>(unit(lane, 0)) = w0;
    *reinterpret_cast<uint4*>(unit(lane, 1)) = w1;
    *reinterpret_cast<uint4*>(unit(lane, 2)) = w2;
    *reinterpret_cast<uint4*>(unit(lane, 3)) = w3;
    __syncwarp();
    const uint8_t* const from = unit(r0, q);         // rows 8 apart have the same turn: 512 bytes apart
    if (units) {
      uint8_t* const at = out + (r0 * ld + c0) * size + 16 * q;
      const long long down = 8 * ld * size;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (8 * i + r0 < rows_left && c0 * size + 16 * q < cols_left * size) *reinterpret_cast<uint4*>(at + i * down) = *reinterpret_cast<const uint4*>(from + 512 * i);
    } else if (size == 4) {
      const int c = lane & 15;
      float* at = reinterpret_cast<float*>(out) + (lane >> 4) * ld + c0 + c;
#pragma unroll 4
      for (int r = lane >> 4; r < 32; r += 2, at += 2 * ld)
        if (r < rows_left && c0 + c < cols_left) *at = reinterpret_cast<const float*>(unit(r, c >> 2))[c & 3];
    } else {
      // word j of a row holds columns 2 j and 2 j + 1, or, where the row starts in the middle of a word, 2 j - 1 and 2 j: then the first and
      // the last column of the step go alone
      const int j = lane & 15, some = cols_left - c0;
      unsigned short* row = reinterpret_cast<unsigned short*>(out) + (lane >> 4) * ld + c0;
#pragma unroll 4
      for (int r = lane >> 4; r < 32; r += 2, row += 2 * ld) {
        const uint32_t word = reinterpret_cast<const uint32_t*>(unit(r, j >> 2))[j & 3], before = __shfl_up_sync(0xffffffffu, word, 1, 16);
        const bool odd = (reinterpret_cast<uintptr_t>(row) & 2) != 0, there = r < rows_left;
        const int c = odd ? 2 * j - 1 : 2 * j;
        const uint32_t w = odd ? __byte_perm(before, word, 0x5432) : word;
        if (there && c >= 0 && c + 1 < some) *reinterpret_cast<uint32_t*>(row + c) = w;
        if (there && c >= 0 && c + 1 == some) row[c] = (unsigned short)w;
        if (there && c < 0) row[0] = (unsigned short)word;
        if (there && odd && j == 15 && 31 < some) row[31] = (unsigned short)(word >> 16);
      }
    }
    __syncwarp();
  }
};
template <int NC>
__device__ __forceinline__ void store_rows(const float (&acc)[NC], uint8_t* buf, void* out, long long ld, int out_type, int boundary, int rows_left, int cols_left) {
  const RowStore to(buf, out, ld, out_type == kF32 ? 4 : 2, boundary, rows_left, cols_left);
  if (out_type == kF32) {
#pragma unroll
    for (int c0 = 0; c0 < NC; c0 += 16) {
      if (c0 < cols_left) {
        uint4 w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          w[u] = words(acc[c0 + 4 * u], acc[c0 + 4 * u + 1], acc[c0 + 4 * u + 2], acc[c0 + 4 * u + 3]);
        to.put(c0, w[0], w[1], w[2], w[3]);
      }
    }
  } else {
#pragma unroll
    for (int c0 = 0; c0 < NC; c0 += 32) {
      if (c0 < cols_left) {
        uint4 w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float* const x = acc + c0 + 8 * u;
          w[u] = make_uint4(pack(out_type, x[0], x[1]), pack(out_type, x[2], x[3]), pack(out_type, x[4], x[5]), pack(out_type, x[6], x[7]));
        }
        to.put(c0, w[0], w[1], w[2], w[3]);
      }
    }
  }
}

// Eight elements of a row on their way from memory to an operand tile, those from `valid` on zero.
template <typename T>
struct Raw;
__device__ __forceinline__ float4 load16(const float* at) {   // read once by this SM
  float4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(at));
  return v;
}
template <>
struct Raw<float> {
  float x[8];
  // VEC: quads are 16-byte aligned and lie inside or outside as a whole
  template <bool VEC>
  __device__ __forceinline__ void load(const float* p, int valid) {
    if constexpr (VEC) {
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
      if (valid > 0) a = load16(p);
      if (valid > 4) b = load16(p + 4);
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = e < valid ? __ldg(p + e) : 0.f;
    }
  }
  // The three parts, `part` bytes apart: each the upper half of what the last ones leave (differences are exact).
  __device__ __forceinline__ void store(uint8_t* at, long long part) const {
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
    for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(at + part_at(k, part)) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
  }
};
// Halves on any boundary: the aligned words that hold them, as they are, until they are stored (124576 x 211 x 156 in 20 groups: 123 us; with a
// load for every half, put together as it came, about 20 % more).  A word that holds an element of a matrix lies in the matrix's allocation; other words are not touched.
template <>
struct Raw<unsigned short> {
  uint32_t v[5];
  int valid;   // elements, negative where the first is in the middle of a word
  template <bool>
  __device__ __forceinline__ void load(const unsigned short* p, int valid_) {
    const HalfWords words(reinterpret_cast<uintptr_t>(p), valid_);
    const uint32_t* const q = reinterpret_cast<const uint32_t*>(words.first);
    valid = words.odd ? -words.some : words.some;
#pragma unroll
    for (int k = 0; k < 5; ++k) v[k] = words.holds(k) ? __ldg(q + k) : 0u;
  }
  __device__ __forceinline__ void store(uint8_t* at, long long) const {
    const int some = abs(valid);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      w[k] = valid < 0 ? __funnelshift_r(v[k], v[k + 1], 16) : v[k];
      if (2 * k + 1 >= some) w[k] = 2 * k < some ? w[k] & 0xffffu : 0u;
    }
    *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// The shared loop.  A job J says what the items are, where operand tiles come from and what becomes of a tile's sums:
//   J::Args, kParts, kBN, kAMn, kBMn, kTma, kTmaB (of operands that go through registers B still comes by TMA), kPair, kTailed (copies bring rows from behind the end of an item), kMeets (finish() has barriers of the epilogue warps)
//   segment()                         chunks of a segment, a power of two
//   J(args, tables, rank)             built by every thread (rank: of the block in its pair); setup(): tables in shared memory, by the whole
//                                     block, between barriers
//   J::Walk start(worker, workers)    where this block's (pair's) items begin
//   bool next(Walk&, Item&)           the next of them, false behind the last; Item has chunks (of the reduction, maybe none), n (columns) and tail
//                                     (steps of the last chunk that count, where rows behind them hold other data; else 64)
//   copy(item, chunk, tile, bar)      kTma: announces the bytes of this block's copies of a chunk at `bar` and issues them; template argument: whether `bar` is
//                                     the first block's
//   load_a, load_b(item, chunk, unit, raw)   otherwise: eight elements of a tile; copy_b(item, chunk, tile, bar) where kTmaB
//   early(item, warp, Early&)         loads of what finish() reads, issued before the sums are there
//   finish(item, acc, Early&, buf, warp)   the sums of this warp's rows and columns; by all epilogue warps
template <class J>
using GeometryOf = Geometry<J::kParts, J::kBN, J::kTma, J::kPair>;

template <class J>
__global__ void __launch_bounds__(GeometryOf<J>::kThreads, 1) k_products(const __grid_constant__ typename J::Args args) {
  using G = GeometryOf<J>;
  constexpr int S = G::kStages, BN = J::kBN, PARTS = J::kParts;
  constexpr bool PAIR = J::kPair;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) Bars bars;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t base = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t full = smem_u32(bars.full), empty = smem_u32(bars.empty), acc_full = smem_u32(bars.acc_full), acc_empty = smem_u32(bars.acc_empty);
  const uint32_t drain = smem_u32(&bars.drain), tail = smem_u32(bars.tail);
  // of the pair: its first block (rank 0) issues the instructions, and the barriers that it waits on for both are its own
  const int rank = PAIR ? (int)(blockIdx.x & 1) : 0;
  const unsigned worker = PAIR ? blockIdx.x >> 1 : blockIdx.x, workers = PAIR ? gridDim.x >> 1 : gridDim.x;
  const uint32_t full_there = PAIR ? of_first_block(full) : full, acc_empty_there = PAIR ? of_first_block(acc_empty) : acc_empty;
  if (tid == 0) {
    for (int s = 0; s < S; ++s) {
      gtc::mbar_init(full + 8 * s, PAIR ? 2 : G::kProducers + (J::kTmaB ? 1 : 0));
      gtc::mbar_init(empty + 8 * s, 1);
      gtc::mbar_init(tail + 8 * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      gtc::mbar_init(acc_full + 8 * a, 1);
      gtc::mbar_init(acc_empty + 8 * a, PAIR ? 2 * kEpiWarps : kEpiWarps);
    }
    gtc::mbar_init(drain, 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(G::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(G::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  if (tid == kMmaWarp * 32 + 32) {
    if constexpr (J::kTma) asm volatile("prefetch.tensormap [%0];" ::"l"(&args.a) : "memory");
    if constexpr (J::kTma || J::kTmaB) asm volatile("prefetch.tensormap [%0];" ::"l"(&args.b) : "memory");
  }
  gtc::enter_kernel();
  J job(args, smem + G::kTablesAt, rank);
  job.setup();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if constexpr (PAIR) meet_pair();   // both blocks' barriers are there
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  volatile int* const abortp = &abort_flag;
  const int segment = job.segment();
  CopyLog copies;   // of this thread
  typename J::Item it;
  typename J::Walk walk = job.start(worker, workers);

  // Registers go where they are needed.  384 threads start with 168 each: the epilogue's eight warps get 208, the four others 80 (256 x 208 + 128 x 80 = 63488
  // of 64512).  640 threads start with 96: the epilogue gets 104, the eight loading warps 112 and the four others 48 (256 x 104 + 256 x 112 + 128 x 48 = 61440,
  // all there are).
  if (warp >= kMmaWarp && warp < kFirstLoader) {
  if constexpr (J::kTma) asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
  else asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
  if (warp == kMmaWarp + 2 && J::kTma) {
    if constexpr (J::kTailed) {
      // Rows of the next group come with the last chunk of a tile: the steps that are still read are cleared in both operands, in a pair by each
      // block in its own.  A warp of its own does it while chunks before this one are multiplied, and then arrives where
      // copies of other chunks arrive.  (Where the issuing warp did it, chunks behind waited.)
      int slot = 0;
      uint32_t parities = 0;   // of the slots, a bit each
      bool ok = true;
      while (ok && job.next(walk, it)) {
        slot = (slot + it.chunks) % S;
        if (it.chunks == 0 || it.tail == kBK) continue;
        const int at = (slot + S - 1) % S, steps = (it.tail + 15) / 16, clear = steps * 16 - it.tail, groups = kBM / 64 + G::kBCols / 64;
        ok = __all_sync(0xffffffffu, gtc::mbar_wait_abortable(tail + 8 * at, parities >> at & 1u, abortp));
        if (!ok) break;
        parities ^= 1u << at;
        for (int u = lane; u < clear * groups * 8; u += 32) {
          const int row = it.tail + (u >> 3) % clear, group = (u >> 3) / clear;
          *reinterpret_cast<uint4*>(smem + (size_t)at * G::kStage + group * kGroup64 + row * 128 + (u & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if constexpr (PAIR) arrive_at_first(full_there + 8 * at, true);
        else gtc::mbar_arrive_warp(full + 8 * at);
      }
    }
  } else if (warp == kMmaWarp + 1 && (J::kTma || J::kTmaB)) {
    int slot = 0;
    uint32_t parity = 1;   // a fresh barrier passes a wait on parity 1
    if constexpr (J::kTma || J::kTmaB) {
      if (lane == 0) {
        bool ok = true;
        while (ok && job.next(walk, it)) {
          for (int c = 0; c < it.chunks; ++c) {
            ok = gtc::mbar_wait_abortable(empty + 8 * slot, parity, abortp);
            if (!ok) break;
            const uint32_t tile = base + (uint32_t)slot * G::kStage;
            if constexpr (J::kTmaB) job.copy_b(it, c, tile + PARTS * kATile, full + 8 * slot);
            // a chunk with rows to clear is announced to the warp that does it
            else if (J::kTailed && it.tail < kBK && c + 1 == it.chunks) job.template copy<false>(it, c, tile, tail + 8 * slot);
            else job.template copy<PAIR>(it, c, tile, full_there + 8 * slot);
            copies.add(slot, J::kTailed && it.tail < kBK && c + 1 == it.chunks);
            if (++slot == S) { slot = 0; parity ^= 1u; }
          }
        }
      }
    }
  } else if (warp == kMmaWarp) {
    // One thread waits and issues, with as little as possible between a chunk's last instruction and the next one's first: what the loop takes beyond the
    // 512 clocks of a chunk's instructions (256 x 256 by a pair) is time that the tensor core stands still.  So what a chunk needs is kept in
    // counters that are added to, and decisions are per segment.  (A chunk took 710 clocks with all of them made for every chunk.)
    if (lane == 0 && rank == 0) {
      const uint32_t kind = instruction<J::kAMn, J::kBMn, PAIR>(job.bf16());
      constexpr uint32_t pa = kATile >> 4, pb = G::kBTile >> 4, oa = kStep16<J::kAMn>, ob = kStep16<J::kBMn>, kStride = G::kStage >> 4;
      const uint32_t a0 = desc_lo<J::kAMn>(base), b_behind = desc_lo<J::kBMn>(base + PARTS * kATile) - a0;   // fields do not carry into each other
      uint32_t a = a0, at = 0, parity = 0, set = 0, acc_parity = 1;   // descriptor of A, offset of the barriers
      bool ok = true;
      while (ok && job.next(walk, it)) {
        const uint32_t idesc = kind | (uint32_t)((PAIR ? BN : (min(it.n, BN) + 15) / 16 * 16) >> 3) << 17;
        [[maybe_unused]] const uint32_t both = kind | (uint32_t)(2 * BN >> 3) << 17;
        const int chunks = it.chunks, tail_steps = J::kTailed ? (it.tail + 15) / 16 : kBK / 16;
        for (int c = 0; c < chunks && ok;) {
          const int stop = min(chunks, c + segment);
          const uint32_t d = tmem + set * (G::kAccs * BN);
          ok = gtc::mbar_wait_abortable(acc_empty + 8 * set, acc_parity, abortp);
          if (!ok) break;
          uint32_t go_on = 0;
          for (; c < stop; ++c) {
            ok = gtc::mbar_wait_abortable(full + at, parity, abortp);
            if (!ok) break;
            if (PAIR && J::kTailed && c + 1 == chunks) acquire_cluster(full + at, parity);   // what the other block has cleared
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t b = a + b_behind;
            const auto step = [&](int k, uint32_t more) {
              const uint32_t ak = a + k * oa, bk = b + k * ob;
              if constexpr (PAIR) {
                mma_pair(d, ak, bk, idesc, more);
              } else {
                // Part 0 of A with parts 0 and 1 of B, which lie one behind the other as do main sums and corrections: one instruction of 2 BN
                // columns, which reads A once
                mma(d, ak, bk, PARTS > 1 ? both : idesc, more);
                if constexpr (PARTS > 1) mma(d + BN, ak + pa, bk, idesc, 1u);
                if constexpr (PARTS > 2) {
                  mma(d + BN, ak + pa, bk + pb, idesc, 1u);
                  mma(d + BN, ak, bk + 2 * pb, idesc, 1u);
                  mma(d + BN, ak + 2 * pa, bk, idesc, 1u);
                }
              }
            };
            step(0, go_on);
            if (J::kTailed && c + 1 == chunks) {
              for (int k = 1; k < tail_steps; ++k) step(k, 1u);
            } else {
#pragma unroll
              for (int k = 1; k < kBK / 16; ++k) step(k, 1u);
            }
            go_on = 1;
            if constexpr (PAIR) commit_pair(empty + at);
            else gtc::mma_commit(empty + at);
            a += kStride;
            at += 8;
            if (at == 8 * S) { a = a0; at = 0; parity ^= 1u; }
          }
          if (!ok) break;
          if constexpr (PAIR) commit_pair(acc_full + 8 * set);
          else gtc::mma_commit(acc_full + 8 * set);
          acc_parity ^= set;
          set ^= 1u;
        }
      }
    }
  }
  } else if (warp >= kFirstLoader) {
    if constexpr (!J::kTma) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
      // Elements are loaded kAhead chunks before they go to shared memory (two where B comes by TMA and leaves the registers).
      constexpr int kAhead = J::kTmaB ? 2 : 1, kUnitsA = kBM * 8 / 256, kUnitsB = J::kTmaB ? 0 : BN * 8 / 256;
      using R = Raw<typename J::T>;
      R a[kAhead][kUnitsA], b[kAhead][kUnitsB > 0 ? kUnitsB : 1];
      const int t = tid - kFirstLoader * 32;
      int slot = 0, c = 0, held = 0;   // held: chunks in registers
      uint32_t parity = 1;
      it.chunks = 0;
      const auto load = [&](R (&to_a)[kUnitsA], R (&to_b)[kUnitsB > 0 ? kUnitsB : 1]) {
        while (c >= it.chunks) {   // on to the next item where this one has no chunk left
          c = 0;
          if (!job.next(walk, it)) {
            it.chunks = 0;
            return;
          }
        }
#pragma unroll
        for (int u = 0; u < kUnitsA; ++u) job.load_a(it, c, t + 256 * u, to_a[u]);
#pragma unroll
        for (int u = 0; u < kUnitsB; ++u) job.load_b(it, c, t + 256 * u, to_b[u]);
        ++c;
        ++held;
      };
#pragma unroll
      for (int d = 0; d < kAhead; ++d) load(a[d], b[d]);
      bool ok = true;
      while (ok && held > 0) {
#pragma unroll
        for (int d = 0; d < kAhead; ++d) {
          if (held == 0) break;
          ok = __all_sync(0xffffffffu, gtc::mbar_wait_abortable(empty + 8 * slot, parity, abortp));
          if (!ok) break;
          uint8_t* const st = smem + (size_t)slot * G::kStage;
#pragma unroll
          for (int u = 0; u < kUnitsA; ++u) {
            const int at = t + 256 * u;
            a[d][u].store(st + (J::kAMn ? unit_mn(at / (kBM / 8), at % (kBM / 8)) : unit_k(at >> 3, at & 7)), kATile);
          }
#pragma unroll
          for (int u = 0; u < kUnitsB; ++u) {
            const int at = t + 256 * u;
            b[d][u].store(st + PARTS * kATile + (J::kBMn ? unit_mn(at / (BN / 8), at % (BN / 8)) : unit_k(at >> 3, at & 7)), G::kBTile);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          gtc::mbar_arrive_warp(full + 8 * slot);
          --held;
          load(a[d], b[d]);
          if (++slot == S) { slot = 0; parity ^= 1u; }
        }
      }
    }
  } else {
    if constexpr (J::kTma) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    constexpr int NC = BN / 2;   // columns of a warp
    constexpr float kCorrection = PARTS == 2 ? 0x1p-11f : 1.f;
    uint8_t* const buf = smem + G::kBuffersAt + warp * kBuffer;
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)((warp >> 2) * NC);
    int set = 0;
    uint32_t parity = 0;
    bool ok = true;
    while (ok && job.next(walk, it)) {
      float acc[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[c] = 0.f;
      const bool mine = (warp >> 2) * NC < it.n;   // whether any of the warp's columns are asked for
      typename J::Early early;
      job.early(it, warp, early);
      for (int c = 0; c < it.chunks; c += segment) {
        ok = __all_sync(0xffffffffu, gtc::mbar_wait_abortable(acc_full + 8 * set, parity, abortp));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (mine) {
          const uint32_t from = lanes + (uint32_t)(set * G::kAccs * BN);
          // 16 columns are added while the next 16 are on their way
          uint32_t v[2][16], w[PARTS > 1 ? 2 : 1][16];
          GTC_TMEM_LD16(v[0], from);
          if constexpr (PARTS > 1) GTC_TMEM_LD16(w[0], from + BN);
#pragma unroll
          for (int c0 = 0; c0 < NC; c0 += 16) {
            constexpr int kLast = NC - 16;
            const int now = c0 / 16 & 1;
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            if (c0 < kLast) {
              GTC_TMEM_LD16(v[now ^ 1], from + c0 + 16);
              if constexpr (PARTS > 1) GTC_TMEM_LD16(w[now ^ 1], from + BN + c0 + 16);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              if constexpr (PARTS > 1) acc[c0 + e] += fmaf(__uint_as_float(w[now][e]), kCorrection, __uint_as_float(v[now][e]));
              else acc[c0 + e] += __uint_as_float(v[now][e]);
            }
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        if constexpr (PAIR) arrive_at_first(acc_empty_there + 8 * set, false);
        else gtc::mbar_arrive_warp(acc_empty + 8 * set);
        if (set == 1) parity ^= 1u;
        set ^= 1;
      }
      // where epilogue warps meet in finish(), those that gave up and those that did not leave together
      if constexpr (J::kMeets) ok = gtc::all_agree(ok, kEpiWarps * 32);
      if (ok) job.finish(it, acc, early, buf, warp);
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (abort_flag) {
    // What is still in flight is waited for before shared and tensor memory are let go: each copy at the barrier that it reports to, with a bound (a phase
    // that also waits for what never came does not end).  Copies of a pair's second block report to the first one's barriers, on which
    // only that one can wait: there the bound itself, a thousand times what a copy takes, has to do.  A block of a pair that has not given up has
    // seen the end of every copy and instruction, its own and those that the other block issued for it.
    if (tid == 0) atomicOr(job.error_flag(), 1);
    if (warp == kMmaWarp + 1 && lane == 0 && (J::kTma || J::kTmaB)) {
      bool unseen = false;
      for (int i = max(0, copies.started - S); i < copies.started; ++i) {
        const int slot = i % S;
        if (J::kTailed && copies.is_tail(slot)) gtc::drain_wait(tail + 8 * slot, copies.tail_parity(slot));
        else if (rank == 0) gtc::drain_wait(full + 8 * slot, CopyLog::full_parity(i, S));
        else unseen = true;
      }
      if (PAIR && unseen)
        for (const long long t0 = clock64(); clock64() - t0 < gtc::kDrainClocks;) {}
    }
    if (warp == kMmaWarp && lane == 0 && rank == 0) {
      if constexpr (PAIR) {
        commit_pair(drain);
        gtc::drain_wait(drain, 0);
      } else {
        gtc::drain_mmas(drain);
      }
    }
    __syncthreads();
  }
  if constexpr (PAIR) meet_pair();   // neither block's memory is used by the other any more
  if (warp == kMmaWarp) {
    __syncwarp();
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(G::kTmemCols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(G::kTmemCols) : "memory");
  }
}

}  // namespace gcn_admm_grouped
