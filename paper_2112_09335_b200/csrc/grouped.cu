// Products grouped by expert, their gradients, and orthogonalised updates.
#include "grouped.hpp"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace gcn_admm_grouped {
namespace {

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void put(float* at, float x) { *at = x; }
__device__ __forceinline__ void put(__nv_bfloat16* at, float x) { *at = __float2bfloat16_rn(x); }
__device__ __forceinline__ void put(__half* at, float x) { *at = __float2half_rn(x); }

// Rows of a group: offsets[g] .. offsets[g+1] cut to 0 .. rows, none where they descend.  Whatever the offsets hold, no row outside of
// the matrices is touched.
__device__ __forceinline__ int2 group_rows(const int* __restrict__ offsets, int g, int rows) {
  const int lo = min(max(__ldg(offsets + g), 0), rows);
  return make_int2(lo, max(lo, min(__ldg(offsets + g + 1), rows)));
}

constexpr int kTile = 64, kStep = 16;

// One 64 x 64 tile of sum over c < K of a(i, c) b(c, j), by 256 threads of 4 x 4 elements.  `a` and `b` give an element, zero outside.
template <typename GetA, typename GetB, typename Put>
__device__ void tile_product(int K, const GetA& a, const GetB& b, const Put& put_at) {
  __shared__ float sa[kStep][kTile + 1], sb[kStep][kTile + 1];
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  float acc[4][4] = {};
  for (int c0 = 0; c0 < K; c0 += kStep) {
    for (int e = tid; e < kStep * kTile; e += 256) {
      sa[e & 15][e >> 4] = c0 + (e & 15) < K ? a(e >> 4, c0 + (e & 15)) : 0.f;
      sb[e >> 6][e & 63] = c0 + (e >> 6) < K ? b(c0 + (e >> 6), e & 63) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kStep; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[c][ty + 16 * i], sb[c][tx + 16 * j], acc[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) put_at(ty + 16 * i, tx + 16 * j, acc[i][j]);
}

template <typename T, typename O>
__global__ void __launch_bounds__(256) k_grouped(const Product p) {
  __shared__ int s_g, s_row, s_end;
  const int rows = (int)p.rows;
  if (threadIdx.x == 0) {
    int tile = blockIdx.x, g = 0;
    for (; g < p.groups; ++g) {
      const int2 r = group_rows(p.offsets, g, rows);
      const int tiles = (r.y - r.x + kTile - 1) / kTile;
      if (tile < tiles) { s_row = r.x + tile * kTile; s_end = r.y; break; }
      tile -= tiles;
    }
    s_g = g;
  }
  __syncthreads();
  if (s_g == p.groups) return;
  const int row0 = s_row, left = s_end - row0, col0 = blockIdx.y * kTile;
  const T* const x = static_cast<const T*>(p.x) + row0 * p.ldx;
  const T* const w = static_cast<const T*>(p.w) + s_g * p.stride_w;
  O* const y = static_cast<O*>(p.y) + row0 * p.ldy;
  tile_product(
      p.k, [&](int i, int c) { return i < left ? to_float(x[i * p.ldx + c]) : 0.f; },
      [&](int c, int j) { return col0 + j < p.n ? to_float(p.transposed ? w[(col0 + j) * p.ldw + c] : w[c * p.ldw + col0 + j]) : 0.f; },
      [&](int i, int j, float v) { if (i < left && col0 + j < p.n) put(y + i * p.ldy + col0 + j, v); });
}

template <typename T, typename O>
__global__ void __launch_bounds__(256) k_grouped_tn(const ProductTn p) {
  const int2 r = group_rows(p.offsets, blockIdx.z, (int)p.rows);
  const int i0 = blockIdx.x * kTile, j0 = blockIdx.y * kTile;
  const T* const x = static_cast<const T*>(p.x) + r.x * p.ldx;
  const T* const y = static_cast<const T*>(p.y) + r.x * p.ldy;
  O* const dw = static_cast<O*>(p.dw) + blockIdx.z * p.stride_dw;
  tile_product(
      r.y - r.x, [&](int i, int c) { return i0 + i < p.ka ? to_float(x[c * p.ldx + i0 + i]) : 0.f; },
      [&](int c, int j) { return j0 + j < p.nb ? to_float(y[c * p.ldy + j0 + j]) : 0.f; },
      [&](int i, int j, float v) { if (i0 + i < p.ka && j0 + j < p.nb) put(dw + (i0 + i) * p.lddw + j0 + j, v); });
}

// X = G / (||G|| + eps), a block for every matrix; rows are the shorter side.  The norm is summed in fp64: squares of fp32 numbers leave
// the range of fp32.
template <typename T>
__global__ void __launch_bounds__(256) k_normalise(const Orthogonal p, float* __restrict__ x, int m, int n) {
  __shared__ double s_sum[256];
  const bool turn = p.rows > p.cols;
  const T* const g = static_cast<const T*>(p.g) + blockIdx.x * p.stride_g;
  const auto at = [&](long long e) { return (double)to_float(turn ? g[(e % n) * p.ldg + e / n] : g[(e / n) * p.ldg + e % n]); };
  double sum = 0.0;
  for (long long e = threadIdx.x; e < (long long)m * n; e += 256) sum += at(e) * at(e);
  s_sum[threadIdx.x] = sum;
  __syncthreads();
  for (int d = 128; d > 0; d >>= 1) {
    if (threadIdx.x < d) s_sum[threadIdx.x] += s_sum[threadIdx.x + d];
    __syncthreads();
  }
  const double norm = sqrt(s_sum[0]) + (double)p.eps, inverse = norm > 0.0 ? 1.0 / norm : 0.0;
  for (long long e = threadIdx.x; e < (long long)m * n; e += 256) x[(long long)blockIdx.x * m * n + e] = (float)(at(e) * inverse);
}

// C = A B (B transposed where `bt`), matrices of a batch one after the other; where `d` is given, C = a I + b D + c A B.
__global__ void __launch_bounds__(256) k_batch_product(const float* A, const float* B, float* C, int m, int n, int k, bool bt, const float* D, float a, float b, float c) {
  const long long z = blockIdx.z;
  A += z * m * k; B += z * n * k; C += z * m * n;
  if (D != nullptr) D += z * m * n;
  const int i0 = blockIdx.x * kTile, j0 = blockIdx.y * kTile;
  tile_product(
      k, [&](int i, int q) { return i0 + i < m ? A[(long long)(i0 + i) * k + q] : 0.f; },
      [&](int q, int j) { return j0 + j < n ? bt ? B[(long long)(j0 + j) * k + q] : B[(long long)q * n + j0 + j] : 0.f; },
      [&](int i, int j, float v) {
        i += i0; j += j0;
        if (i < m && j < n) C[(long long)i * n + j] = D != nullptr ? (i == j ? a : 0.f) + b * D[(long long)i * n + j] + c * v : v;
      });
}
template <typename O>
__global__ void __launch_bounds__(256) k_leave(const Orthogonal p, const float* __restrict__ x, int m, int n) {
  const bool turn = p.rows > p.cols;
  O* const out = static_cast<O*>(p.out) + blockIdx.z * p.stride_o;
  for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < (long long)m * n; e += (long long)gridDim.x * 256) {
    const long long i = e / n, j = e % n;
    put(turn ? out + j * p.ldo + i : out + i * p.ldo + j, p.scale * x[(long long)blockIdx.z * m * n + e]);
  }
}

template <typename F>
void with_type(int type, const F& f) {
  switch (type) {
    case kBf16: f(__nv_bfloat16()); break;
    case kF16: f(__half()); break;
    default: f(float());
  }
}
template <typename F>
void with_types(int type, int out_type, const F& f) {
  with_type(type, [&](auto in) {
    if (out_type == type) f(in, in);
    else f(in, float());
  });
}

}  // namespace

std::size_t space_bytes(const ProductTn&) { return 0; }
std::size_t tickets_of(const ProductTn&) { return 0; }
std::size_t space_bytes(const Orthogonal& p) {
  const std::size_t m = std::min(p.rows, p.cols), n = std::max(p.rows, p.cols);
  return (std::size_t)p.batch * (2 * m * n + 2 * m * m) * sizeof(float);
}

cudaError_t enqueue(const Product& p, const Room& room) {
  if (p.rows == 0) return cudaSuccess;
  const dim3 grid((unsigned)(cdiv(p.rows, kTile) + p.groups), (unsigned)cdiv(p.n, kTile));
  with_types(p.type, p.out_type, [&](auto in, auto out) { k_grouped<decltype(in), decltype(out)><<<grid, 256, 0, room.stream>>>(p); });
  ++*room.launches;
  return cudaGetLastError();
}

cudaError_t enqueue(const ProductTn& p, const Room& room) {
  const dim3 grid((unsigned)cdiv(p.ka, kTile), (unsigned)cdiv(p.nb, kTile), (unsigned)p.groups);
  with_types(p.type, p.out_type, [&](auto in, auto out) { k_grouped_tn<decltype(in), decltype(out)><<<grid, 256, 0, room.stream>>>(p); });
  ++*room.launches;
  return cudaGetLastError();
}

cudaError_t enqueue(const Orthogonal& p, const Room& room) {
  const int m = std::min(p.rows, p.cols), n = std::max(p.rows, p.cols);
  float* x = static_cast<float*>(room.space);
  float* y = x + (std::size_t)p.batch * m * n;
  float *const s = y + (std::size_t)p.batch * m * n, *const f = s + (std::size_t)p.batch * m * m;
  with_type(p.type, [&](auto in) { k_normalise<decltype(in)><<<p.batch, 256, 0, room.stream>>>(p, x, m, n); });
  const dim3 square((unsigned)cdiv(m, kTile), (unsigned)cdiv(m, kTile), (unsigned)p.batch), wide((unsigned)cdiv(m, kTile), (unsigned)cdiv(n, kTile), (unsigned)p.batch);
  for (int i = 0; i < p.steps; ++i) {
    const float* const c = p.coefficients + 3 * i;
    k_batch_product<<<square, 256, 0, room.stream>>>(x, x, s, m, m, n, true, nullptr, 0.f, 0.f, 0.f);
    k_batch_product<<<square, 256, 0, room.stream>>>(s, s, f, m, m, m, false, s, c[0], c[1], c[2]);
    k_batch_product<<<wide, 256, 0, room.stream>>>(f, x, y, m, n, m, false, nullptr, 0.f, 0.f, 0.f);
    std::swap(x, y);
  }
  const dim3 grid((unsigned)std::min<long long>(1024, cdiv((long long)m * n, 256)), 1, (unsigned)p.batch);
  with_type(p.out_type, [&](auto out) { k_leave<decltype(out)><<<grid, 256, 0, room.stream>>>(p, x, m, n); });
  *room.launches += 2 + 3 * p.steps;
  return cudaGetLastError();
}

}  // namespace gcn_admm_grouped
