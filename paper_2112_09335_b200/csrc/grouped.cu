// Products grouped by expert, their gradients, and orthogonalised updates.
#include "grouped.hpp"

#include <atomic>
#include <climits>

#include "grouped_mma.cuh"
#include "tensor_map.hpp"

namespace gcn_admm_grouped {
namespace {

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void put(float* at, float x) { *at = x; }
__device__ __forceinline__ void put(__nv_bfloat16* at, float x) { *at = __float2bfloat16_rn(x); }
__device__ __forceinline__ void put(__half* at, float x) { *at = __float2half_rn(x); }

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

// ---- groups of rows ----------------------------------------------------------------------------------
// Rows of a group: offsets[g] .. offsets[g+1] cut to 0 .. rows, none where they descend.  Whatever the offsets hold, no row outside of
// the matrices is touched.  Offsets are read as they are when the kernel runs.
__device__ __forceinline__ int2 group_rows(const int* offsets, int g, int rows) {
  const volatile int* const at = offsets + g;
  const int lo = min(max(at[0], 0), rows);
  return make_int2(lo, max(lo, min(at[1], rows)));
}

// Which item belongs to which group: every block counts for itself (1024 groups are 4 loads a thread and a scan by one warp; a launch
// that wrote the table down would cost more than all blocks' counting).
struct Groups {
  unsigned* ends;     // [groups] items of this group and all before it
  int *begin, *end;   // [groups] rows
  int count;
  __device__ __forceinline__ Groups(uint8_t* tables, int count_)
      : ends(reinterpret_cast<unsigned*>(tables)), begin(reinterpret_cast<int*>(tables) + kMaxGroups), end(reinterpret_cast<int*>(tables) + 2 * kMaxGroups), count(count_) {}
  // ends[g] = items of group g alone before, of all up to g afterwards, and the total.  By one warp.
  __device__ __forceinline__ static void scan(unsigned* v, int count) {
    const int lane = threadIdx.x & 31;
    unsigned long long before = 0;
    for (int g0 = 0; g0 < count; g0 += 32) {
      unsigned long long x = g0 + lane < count ? v[g0 + lane] : 0u;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const unsigned long long y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
      x += before;
      before = __shfl_sync(0xffffffffu, x, 31);
      if (g0 + lane < count) v[g0 + lane] = (unsigned)min(x, (unsigned long long)INT_MAX);   // more than any memory has room for
    }
  }
  // The group of item i < ends[count - 1], from `g` on; `before`: items ahead of it.
  __device__ __forceinline__ int find(unsigned i, unsigned& before) const {
    int lo = 0, hi = count - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (ends[mid] > i) hi = mid;
      else lo = mid + 1;
    }
    before = lo > 0 ? ends[lo - 1] : 0u;
    return lo;
  }
};
constexpr int kTableBytes = 4 * kMaxGroups * 4 + 16;

// ---- y = x W_g ---------------------------------------------------------------------------------------
struct ProductArgs {
  CUtensorMap a, b;      // of x and of the weights, where tiles are copied by TMA
  Product p;
  int* error_flag;
  bool vec_x, vec_w, vec_y;   // 16-byte boundaries
};

template <typename T_, int PARTS, int BN, bool TRANSPOSED, bool TMA>
struct ProductJob {
  using T = T_;
  using Args = ProductArgs;
  static constexpr int kParts = PARTS, kBN = BN;
  static constexpr bool kAMn = false, kBMn = !TRANSPOSED, kTma = TMA, kMeets = false;
  struct Item {
    int chunks, n, tail, g, row0, left, col0;
  };
  const Args& a;
  Groups groups;
  int tiles_n;
  __device__ __forceinline__ ProductJob(const Args& args, uint8_t* tables) : a(args), groups(tables, args.p.groups), tiles_n((args.p.n + BN - 1) / BN) {}
  __device__ __forceinline__ bool bf16() const { return PARTS > 1 || a.p.type == kBf16; }
  __device__ __forceinline__ int* error_flag() const { return a.error_flag; }
  __device__ __forceinline__ void setup() {
    for (int g = threadIdx.x; g < groups.count; g += blockDim.x) {
      const int2 r = group_rows(a.p.offsets, g, (int)a.p.rows);
      groups.begin[g] = r.x;
      groups.end[g] = r.y;
      groups.ends[g] = (unsigned)min((unsigned long long)((r.y - r.x + kBM - 1) / kBM) * tiles_n, (unsigned long long)INT_MAX);
    }
    __syncthreads();
    if (threadIdx.x < 32) Groups::scan(groups.ends, groups.count);
  }
  __device__ __forceinline__ bool item(unsigned i, Item& it) const {
    if (i >= groups.ends[groups.count - 1]) return false;
    unsigned before;
    it.g = groups.find(i, before);
    const unsigned local = i - before, tile = local / tiles_n;
    it.row0 = groups.begin[it.g] + (int)tile * kBM;
    it.left = groups.end[it.g] - it.row0;
    it.col0 = (int)(local - tile * tiles_n) * BN;
    it.n = a.p.n - it.col0;
    it.chunks = (a.p.k + kBK - 1) / kBK;
    it.tail = kBK;
    return true;
  }
  __device__ __forceinline__ void copy(const Item& it, int c, uint32_t tile, uint32_t bar) const {
    const int boxes = TRANSPOSED ? BN / 64 : min(BN / 64, (it.n + 63) / 64);   // columns behind the last are left out: they meet no result
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)(kATile + boxes * kGroup64)) : "memory");
    copy_2d(tile, &a.a, c * kBK, it.row0, bar);
    if constexpr (TRANSPOSED) {
      copy_3d(tile + kATile, &a.b, c * kBK, it.col0, it.g, bar);
    } else {
      for (int b = 0; b < boxes; ++b) copy_3d(tile + kATile + b * kGroup64, &a.b, it.col0 + 64 * b, c * kBK, it.g, bar);
    }
  }
  template <int NA, int NB>
  __device__ __forceinline__ void load(const Item& it, int c, int t, Raw<T> (&ra)[NA], Raw<T> (&rb)[NB]) const {
    const T* const x = static_cast<const T*>(a.p.x) + (long long)it.row0 * a.p.ldx;
    const T* const w = static_cast<const T*>(a.p.w) + (long long)it.g * a.p.stride_w;
#pragma unroll
    for (int u = 0; u < NA; ++u) {
      const int at = t + 256 * u, row = at >> 3, k = c * kBK + (at & 7) * 8;
      ra[u].load(x + row * a.p.ldx + k, row < it.left ? a.p.k - k : 0, a.vec_x);
    }
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      const int at = t + 256 * u;
      if constexpr (TRANSPOSED) {
        const int col = at >> 3, k = c * kBK + (at & 7) * 8;
        rb[u].load(w + (it.col0 + col) * a.p.ldw + k, col < it.n ? a.p.k - k : 0, a.vec_w);
      } else {
        const int k = c * kBK + at / (BN / 8), col = at % (BN / 8) * 8;
        rb[u].load(w + k * a.p.ldw + it.col0 + col, k < a.p.k ? it.n - col : 0, a.vec_w);
      }
    }
  }
  template <int NC>
  __device__ __forceinline__ void finish(const Item& it, const float (&acc)[NC], uint8_t* buf, int warp) const {
    const int row = (warp & 3) * 32, col = (warp >> 2) * NC;
    const long long at = (it.row0 + row) * a.p.ldy + it.col0 + col;
    void* const y = a.p.out_type == kF32 ? (void*)(static_cast<float*>(a.p.y) + at) : (void*)(static_cast<unsigned short*>(a.p.y) + at);
    store_rows<NC>(acc, buf, y, a.p.ldy, a.p.out_type, a.vec_y, it.left - row, it.n - col);
  }
};

// ---- dw_g = x_g^T y_g --------------------------------------------------------------------------------
// A group's rows are cut into pieces of at most `piece` chunks where it has more, so that few tiles still fill the chip and no long group is
// walked by one block while the others wait.  The pieces' sums go to the workspace, and the block that finishes a tile's last piece adds
// them up, always in the order of the pieces.
struct ProductTnArgs {
  CUtensorMap a, b;
  ProductTn p;
  int* error_flag;
  bool vec_x, vec_y, vec_w;
  int piece;            // chunks
  unsigned slots;       // tiles of sums the workspace has room for
  float* space;
  unsigned* tickets;
};

template <typename T_, int PARTS, int BN, bool TMA>
struct ProductTnJob {
  using T = T_;
  using Args = ProductTnArgs;
  static constexpr int kParts = PARTS, kBN = BN;
  static constexpr bool kAMn = true, kBMn = true, kTma = TMA, kMeets = true;
  struct Item {
    int chunks, n, tail, g, row0, end, m0, col0;
    int pieces;
    unsigned piece, tile;
  };
  const Args& a;
  Groups groups;
  unsigned* slots;   // [groups] first of the group's tiles of sums
  int* last;
  int tiles_n, tiles, longest;   // longest: chunks of a piece
  __device__ __forceinline__ ProductTnJob(const Args& args, uint8_t* tables)
      : a(args), groups(tables, args.p.groups), slots(reinterpret_cast<unsigned*>(tables) + 3 * kMaxGroups), last(reinterpret_cast<int*>(tables) + 4 * kMaxGroups),
        tiles_n((args.p.nb + BN - 1) / BN), tiles(tiles_n * ((args.p.ka + kBM - 1) / kBM)), longest(args.piece) {}
  __device__ __forceinline__ bool bf16() const { return PARTS > 1 || a.p.type == kBf16; }
  __device__ __forceinline__ int* error_flag() const { return a.error_flag; }
  __device__ __forceinline__ static int pieces_of(int rows, int piece, int& per) {
    const int chunks = (rows + kBK - 1) / kBK, want = chunks > piece ? (chunks + piece - 1) / piece : 1;
    per = want > 1 ? (chunks + want - 1) / want : chunks;
    return want > 1 ? (chunks + per - 1) / per : 1;
  }
  __device__ __forceinline__ void setup() {
    count_items();
    __syncthreads();
    if (slots[groups.count - 1] > a.slots) {   // groups that overlap: nothing is cut then
      longest = INT_MAX;
      __syncthreads();
      count_items();
    }
  }
  __device__ __forceinline__ void count_items() {
    for (int g = threadIdx.x; g < groups.count; g += blockDim.x) {
      const int2 r = group_rows(a.p.offsets, g, (int)a.p.rows);
      int per;
      const unsigned long long items = (unsigned long long)pieces_of(r.y - r.x, longest, per) * tiles;
      groups.begin[g] = r.x;
      groups.end[g] = r.y;
      groups.ends[g] = (unsigned)min(items, (unsigned long long)INT_MAX);
      slots[g] = items > (unsigned)tiles ? groups.ends[g] : 0u;
    }
    __syncthreads();
    if (threadIdx.x < 32) Groups::scan(groups.ends, groups.count);
    else if (threadIdx.x < 64) Groups::scan(slots, groups.count);
  }
  __device__ __forceinline__ bool item(unsigned i, Item& it) const {
    if (i >= groups.ends[groups.count - 1]) return false;
    unsigned before;
    it.g = groups.find(i, before);
    const unsigned local = i - before;
    const int begin = groups.begin[it.g], end = groups.end[it.g];
    int per;
    it.pieces = pieces_of(end - begin, longest, per);
    it.piece = local / tiles;
    it.tile = local - it.piece * tiles;
    it.m0 = (int)(it.tile / tiles_n) * kBM;
    it.col0 = (int)(it.tile % tiles_n) * BN;
    it.n = a.p.nb - it.col0;
    it.row0 = begin + (int)it.piece * per * kBK;
    it.end = (int)it.piece + 1 < it.pieces ? it.row0 + per * kBK : end;
    it.chunks = (it.end - it.row0 + kBK - 1) / kBK;
    it.tail = it.end - it.row0 - (it.chunks - 1) * kBK;
    return true;
  }
  __device__ __forceinline__ void copy(const Item& it, int c, uint32_t tile, uint32_t bar) const {
    const int boxes_a = min(kBM / 64, (a.p.ka - it.m0 + 63) / 64), boxes_b = min(BN / 64, (it.n + 63) / 64), row = it.row0 + c * kBK;
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)((boxes_a + boxes_b) * kGroup64)) : "memory");
    for (int b = 0; b < boxes_a; ++b) copy_2d(tile + b * kGroup64, &a.a, it.m0 + 64 * b, row, bar);
    for (int b = 0; b < boxes_b; ++b) copy_2d(tile + kATile + b * kGroup64, &a.b, it.col0 + 64 * b, row, bar);
  }
  template <int NA, int NB>
  __device__ __forceinline__ void load(const Item& it, int c, int t, Raw<T> (&ra)[NA], Raw<T> (&rb)[NB]) const {
    const T* const x = static_cast<const T*>(a.p.x) + it.m0;
    const T* const y = static_cast<const T*>(a.p.y) + it.col0;
#pragma unroll
    for (int u = 0; u < NA; ++u) {
      const int at = t + 256 * u, col = at % (kBM / 8) * 8;
      const long long row = it.row0 + c * kBK + at / (kBM / 8);
      ra[u].load(x + row * a.p.ldx + col, row < it.end ? a.p.ka - it.m0 - col : 0, a.vec_x);
    }
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      const int at = t + 256 * u, col = at % (BN / 8) * 8;
      const long long row = it.row0 + c * kBK + at / (BN / 8);
      rb[u].load(y + row * a.p.ldy + col, row < it.end ? it.n - col : 0, a.vec_y);
    }
  }
  template <int NC>
  __device__ __forceinline__ void finish(const Item& it, float (&acc)[NC], uint8_t* buf, int warp) const {
    const int lane = threadIdx.x & 31;
    if (it.pieces > 1) {
      const unsigned first = it.g > 0 ? slots[it.g - 1] : 0u;   // (scanned)
      float* const sums = a.space + (size_t)(first + it.tile) * (kBM * BN) + (size_t)warp * NC * 32 + lane;
      const size_t step = (size_t)tiles * (kBM * BN);
      float* const mine = sums + it.piece * step;
#pragma unroll
      for (int c = 0; c < NC; ++c) __stcg(mine + c * 32, acc[c]);
      __threadfence();
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (threadIdx.x == 0) {
        unsigned* const ticket = a.tickets + first + it.tile;
        const unsigned done = atomicAdd(ticket, 1u);
        *last = done + 1 == (unsigned)it.pieces;
        if (*last) *ticket = 0u;
        __threadfence();
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (!*last) return;
      __threadfence();
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[c] = 0.f;
      for (int s = 0; s < it.pieces; ++s)
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[c] += __ldcg(sums + s * step + c * 32);
    }
    const int row = it.m0 + (warp & 3) * 32, col = it.col0 + (warp >> 2) * NC;
    const long long at = it.g * a.p.stride_dw + row * a.p.lddw + col;
    void* const dw = a.p.out_type == kF32 ? (void*)(static_cast<float*>(a.p.dw) + at) : (void*)(static_cast<unsigned short*>(a.p.dw) + at);
    store_rows<NC>(acc, buf, dw, a.p.lddw, a.p.out_type, a.vec_w, a.p.ka - row, a.p.nb - col);
  }
};

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

constexpr int kSms = 148;

// Whether every row of a matrix starts on a 16-byte boundary.
bool even(const void* p, long long ld, int size) { return reinterpret_cast<std::uintptr_t>(p) % 16 == 0 && ld * size % 16 == 0; }

// Tensor map of `depth` row-major matrices of 16-bit elements, rows x cols, for tiles of box_rows rows and 64 columns with the 128-byte swizzle;
// elements outside of a matrix read as zero.  False where there is no such map (the operand then goes through registers).
bool make_map(CUtensorMap* map, int type, const void* p, long long cols, long long rows, long long ld, long long depth, long long stride, int box_rows) {
  const auto fn = gcn_admm_host::encode_tiled();
  if (fn == nullptr) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)depth};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, depth > 1 ? (cuuint64_t)stride * 2 : (cuuint64_t)ld * 2};
  const cuuint32_t box[3] = {kBK, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
  return fn(map, type == kBf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, stride > 0 ? 3 : 2, const_cast<void*>(p), dims, strides, box, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A kernel that waits for its predecessor on the stream itself (gtc::enter_kernel), so that its launch runs beside that one's end.
template <class J>
cudaError_t launch(const typename J::Args& args, unsigned grid, const Room& room) {
  using G = Geometry<J::kParts, J::kBN, J::kTma>;
  constexpr size_t smem = 1024 + G::kTablesAt + kTableBytes;
  static_assert(smem + 1024 <= 232448, "shared memory of an SM");
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  static std::atomic<unsigned long long> allowed{0};   // devices whose limit for this kernel is raised
  if (device > 63 || !(allowed.load() >> device & 1)) {
    e = cudaFuncSetAttribute(k_products<J>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    if (device <= 63) allowed.fetch_or(1ull << device);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(G::kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = room.stream;
  cudaLaunchAttribute behind{};
  behind.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  behind.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &behind;
  cfg.numAttrs = 1;
  ++*room.launches;
  return cudaLaunchKernelEx(&cfg, k_products<J>, args);
}

}  // namespace

// Pieces of a weight gradient: the longest whose items give every SM one of about equal length.
struct TnPlan {
  int bn, piece;
  long long slots;
};
TnPlan plan(const ProductTn& p) {
  const bool wide = p.type != kF32;
  TnPlan t;
  t.bn = p.nb <= 64 ? 64 : p.nb <= 128 || !wide ? 128 : 256;
  const long long tiles = cdiv(p.ka, kBM) * cdiv(p.nb, t.bn), chunks = cdiv(p.rows, kBK);
  t.piece = (int)std::max<long long>(8, cdiv(chunks * tiles, kSms));
  // A group of c > piece >= 8 chunks has at most 2 c / piece pieces, and such groups together at most 9/8 of the chunks of all rows.
  t.slots = std::min<long long>(cdiv(9 * chunks, 4 * t.piece) * tiles, INT_MAX);
  if (chunks <= t.piece) t.slots = 0;
  return t;
}
std::size_t space_bytes(const ProductTn& p) {
  const TnPlan t = plan(p);
  return (std::size_t)t.slots * kBM * t.bn * sizeof(float);
}
std::size_t tickets_of(const ProductTn& p) { return (std::size_t)plan(p).slots; }
std::size_t space_bytes(const Orthogonal& p) {
  const std::size_t m = std::min(p.rows, p.cols), n = std::max(p.rows, p.cols);
  return (std::size_t)p.batch * (2 * m * n + 2 * m * m) * sizeof(float);
}

cudaError_t enqueue(const Product& p, const Room& room) {
  if (p.rows == 0) return cudaSuccess;
  ProductArgs a{};
  a.p = p;
  a.error_flag = room.error_flag;
  const int size = size_of(p.type);
  a.vec_x = even(p.x, p.ldx, size);
  a.vec_w = even(p.w, p.ldw, size) && (p.groups == 1 || p.stride_w * size % 16 == 0);
  a.vec_y = even(p.y, p.ldy, size_of(p.out_type));
  const long long tiles_m = std::min<long long>(p.rows, cdiv(p.rows, kBM) + p.groups);   // at most, wherever the groups begin
  const auto pick = [&](auto tma) {
    // The widest tile that still gives every SM one
    const auto enough = [&](int bn) { return p.n > bn / 2 && tiles_m * cdiv(p.n, bn) >= kSms; };
    const int bn = decltype(tma)::value && enough(256) ? 256 : enough(128) ? 128 : 64;
    const unsigned grid = (unsigned)std::min<long long>(kSms, tiles_m * cdiv(p.n, bn));
    if (decltype(tma)::value) {
      const long long w_rows = p.transposed ? p.n : p.k, w_cols = p.transposed ? p.k : p.n;
      if (!make_map(&a.a, p.type, p.x, p.k, p.rows, p.ldx, 1, 0, kBM) ||
          !make_map(&a.b, p.type, p.w, w_cols, w_rows, p.ldw, p.groups, p.stride_w, p.transposed ? bn : kBK))
        return cudaErrorNotSupported;
    }
    const auto go = [&](auto width, auto turned) {
      constexpr int BN = decltype(width)::value;
      constexpr bool T = decltype(turned)::value;
      if constexpr (decltype(tma)::value) return launch<ProductJob<unsigned short, 1, BN, T, true>>(a, grid, room);
      else if constexpr (BN == 256) return cudaErrorNotSupported;
      else if (p.type == kF32) return launch<ProductJob<float, 3, BN, T, false>>(a, grid, room);
      else return launch<ProductJob<unsigned short, 1, BN, T, false>>(a, grid, room);
    };
    const auto turn = [&](auto width) { return p.transposed ? go(width, std::true_type()) : go(width, std::false_type()); };
    return bn == 256 ? turn(std::integral_constant<int, 256>()) : bn == 128 ? turn(std::integral_constant<int, 128>()) : turn(std::integral_constant<int, 64>());
  };
  if (p.type != kF32 && a.vec_x && a.vec_w) {
    const cudaError_t e = pick(std::true_type());
    if (e != cudaErrorNotSupported) return e;
  }
  return pick(std::false_type());
}

cudaError_t enqueue(const ProductTn& p, const Room& room) {
  ProductTnArgs a{};
  a.p = p;
  a.error_flag = room.error_flag;
  const int size = size_of(p.type);
  a.vec_x = even(p.x, p.ldx, size);
  a.vec_y = even(p.y, p.ldy, size);
  a.vec_w = even(p.dw, p.lddw, size_of(p.out_type)) && (p.groups == 1 || p.stride_dw * size_of(p.out_type) % 16 == 0);
  const TnPlan t = plan(p);
  a.piece = t.piece;
  a.slots = (unsigned)t.slots;
  a.space = static_cast<float*>(room.space);
  a.tickets = room.tickets;
  const long long items = cdiv(p.ka, kBM) * cdiv(p.nb, t.bn) * p.groups + t.slots;
  const unsigned grid = (unsigned)std::min<long long>(kSms, items);
  const auto width = [&](const auto& f) {
    return t.bn == 256 ? f(std::integral_constant<int, 256>()) : t.bn == 128 ? f(std::integral_constant<int, 128>()) : f(std::integral_constant<int, 64>());
  };
  if (p.type == kF32)
    return width([&](auto w) {
      if constexpr (decltype(w)::value == 256) return cudaErrorNotSupported;
      else return launch<ProductTnJob<float, 3, decltype(w)::value, false>>(a, grid, room);
    });
  if (p.rows > 0 && a.vec_x && a.vec_y && make_map(&a.a, p.type, p.x, p.ka, p.rows, p.ldx, 1, 0, kBK) && make_map(&a.b, p.type, p.y, p.nb, p.rows, p.ldy, 1, 0, kBK))
    return width([&](auto w) { return launch<ProductTnJob<unsigned short, 1, decltype(w)::value, true>>(a, grid, room); });
  return width([&](auto w) { return launch<ProductTnJob<unsigned short, 1, decltype(w)::value, false>>(a, grid, room); });
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
