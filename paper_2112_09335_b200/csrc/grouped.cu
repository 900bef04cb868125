// Products grouped by expert, their gradients, and orthogonalised updates.
#include "grouped.hpp"

#include <atomic>
#include <climits>
#include <type_traits>

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

// Eight elements of a row, those from `valid` on zero.
template <typename T>
__device__ __forceinline__ void load8(const T* at, int valid, bool vec, float (&v)[8]) {
  if (vec && valid >= 8) {
    uint4 w[sizeof(T) / 2];
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) w[k] = *(reinterpret_cast<const uint4*>(at) + k);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = to_float(reinterpret_cast<const T*>(w)[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < valid ? to_float(at[k]) : 0.f;
  }
}

constexpr int kSms = 148;

// ---- groups of rows ----------------------------------------------------------------------------------
// Rows of a group: offsets[g] .. offsets[g+1] cut to 0 .. rows, none where they descend.  Whatever the offsets hold, no row outside of
// the matrices is touched.  Offsets are read as they are when the kernel runs.
__device__ __forceinline__ int2 group_rows(const int* offsets, int g, int rows) {
  const volatile int* const at = offsets + g;
  const int lo = min(max(at[0], 0), rows);
  return make_int2(lo, max(lo, min(at[1], rows)));
}

// v[g] = the sum of v up to g.  By one warp.
template <typename V>
__device__ __forceinline__ void scan(V* v, int count) {
  const int lane = threadIdx.x & 31;
  unsigned long long before = 0;
  for (int g0 = 0; g0 < count; g0 += 32) {
    unsigned long long x = g0 + lane < count ? (unsigned long long)v[g0 + lane] : 0ull;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const unsigned long long y = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += y;
    }
    x += before;
    before = __shfl_sync(0xffffffffu, x, 31);
    if (g0 + lane < count) v[g0 + lane] = sizeof(V) == 4 ? (V)min(x, (unsigned long long)INT_MAX) : (V)x;   // more tiles than that no memory has room for
  }
}

// Rows of the groups, and tiles of rows: every block counts for itself (1024 groups are 4 loads a thread and a scan by one warp; a launch
// that wrote the table down would cost more than all blocks' counting).
struct Groups {
  unsigned* ends;     // [groups] tiles of rows of this group and all before it
  int *begin, *end;   // [groups] rows
  int count;
  __device__ __forceinline__ Groups(uint8_t* tables, int count_)
      : ends(reinterpret_cast<unsigned*>(tables)), begin(reinterpret_cast<int*>(tables) + kMaxGroups), end(reinterpret_cast<int*>(tables) + 2 * kMaxGroups), count(count_) {}
  __device__ __forceinline__ unsigned tiles() const { return ends[count - 1]; }
  // The group of tile i < tiles(), from g on.
  __device__ __forceinline__ int find(unsigned i, int g) const {
    for (int k = 0; k < 3; ++k, ++g)   // mostly this group or one of the next
      if (ends[g] > i) return g;
    int lo = g, hi = count - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (ends[mid] > i) hi = mid;
      else lo = mid + 1;
    }
    return lo;
  }
};
constexpr int kTableBytes = 4 * kMaxGroups * 4 + 16 + (kSms + 1) * 8;

// ---- y = x W_g ---------------------------------------------------------------------------------------
struct ProductArgs {
  CUtensorMap a, b, few;   // of x and of the weights, where tiles are copied by TMA; of x in boxes of kFewRows rows
  Product p;
  int* error_flag;
  bool vec_x, vec_w;     // rows start on 16-byte boundaries
  int boundary;          // of the rows of y
};

// The weights of a product of many rows, fp32, as the three parts of their elements: images of part 0 of all matrices, then part 1 and 2, rows padded to 16
// bytes, from which tiles are copied by TMA.  Otherwise every tile of 128 rows would split them again.
struct SplitWeights {
  const float* w;
  long long ldw, stride_w;
  int rows, cols, ld, groups;
  bool vec;
  unsigned short* to;
};
__global__ void __launch_bounds__(256) k_split_weights(const SplitWeights p) {
  gtc::enter_kernel();
  const unsigned units = p.ld / 8, count = (unsigned)p.rows * units;   // checked: below 2^31
  const long long part = (long long)p.groups * p.rows * p.ld;
  const float* const w = p.w + (long long)blockIdx.y * p.stride_w;
  unsigned short* const to = p.to + (long long)blockIdx.y * p.rows * p.ld;
  for (unsigned e = blockIdx.x * 256 + threadIdx.x; e < count; e += gridDim.x * 256) {
    const unsigned row = e / units, col = (e - row * units) * 8;
    Raw<float> x;
    load8(w + row * p.ldw + col, p.cols - (int)col, p.vec, x.x);
    x.store(reinterpret_cast<uint8_t*>(to + (long long)row * p.ld + col), part * 2);
  }
}

constexpr int kFewRows = 16;   // (whole groups of eight rows of a tile)

template <typename T_, int PARTS, int BN, bool TRANSPOSED, bool TMA, bool PAIR = false, bool VEC = false, bool SPLIT = false>
struct ProductJob {
  using T = T_;
  using Args = ProductArgs;
  static constexpr int kParts = PARTS, kBN = BN;
  static constexpr bool kAMn = false, kBMn = !TRANSPOSED, kTma = TMA, kTmaB = SPLIT, kTailed = false, kMeets = false, kPair = PAIR;
  static constexpr int kTileRows = PAIR ? 2 * kBM : kBM;
  struct Item {
    int chunks, n, tail, g, row0, left, col0;
  };
  const Args& a;
  Groups groups;
  int tiles_n, rank;
  __device__ __forceinline__ ProductJob(const Args& args, uint8_t* tables, int rank_)
      : a(args), groups(tables, args.p.groups), tiles_n((args.p.n + BN - 1) / BN), rank(rank_) {}
  __device__ __forceinline__ bool bf16() const { return PARTS > 1 || a.p.type == kBf16; }
  __device__ __forceinline__ int segment() const { return a.p.out_type == kF32 ? 4 : 16; }
  __device__ __forceinline__ int* error_flag() const { return a.error_flag; }
  __device__ __forceinline__ void setup() {
    for (int g = threadIdx.x; g < groups.count; g += blockDim.x) {
      const int2 r = group_rows(a.p.offsets, g, (int)a.p.rows);
      groups.begin[g] = r.x;
      groups.end[g] = r.y;
      groups.ends[g] = (unsigned)((r.y - r.x + kTileRows - 1) / kTileRows);
    }
    __syncthreads();
    if (threadIdx.x < 32) scan(groups.ends, groups.count);
  }
  // Tiles in turn, those of a row of tiles one after the other.  The next is step tiles on: step_rows rows of tiles and step_cols of the row.  (With the group searched for and
  // divisions on every step it took a thousand clocks.)
  struct Walk {
    unsigned row, col, step_rows, step_cols;
    int g;
  };
  __device__ __forceinline__ Walk start(unsigned worker, unsigned workers) const {
    const unsigned n = (unsigned)tiles_n;
    return Walk{worker / n, worker % n, workers / n, workers % n, 0};
  }
  __device__ __forceinline__ bool next(Walk& at, Item& it) const {
    if (at.row >= groups.tiles()) return false;
    at.g = groups.find(at.row, at.g);
    const unsigned before = at.g > 0 ? groups.ends[at.g - 1] : 0u;
    it.g = at.g;
    it.row0 = groups.begin[at.g] + (int)(at.row - before) * kTileRows + rank * kBM;
    it.left = groups.end[at.g] - it.row0;
    it.col0 = (int)at.col * BN;
    it.n = a.p.n - it.col0;
    it.chunks = (a.p.k + kBK - 1) / kBK;
    it.tail = kBK;
    at.row += at.step_rows;
    at.col += at.step_cols;
    if (at.col >= (unsigned)tiles_n) {
      at.col -= tiles_n;
      ++at.row;
    }
    return true;
  }
  template <bool THERE>
  __device__ __forceinline__ void copy(const Item& it, int c, uint32_t tile, uint32_t bar) const {
    constexpr int kBCols = PAIR ? BN / 2 : BN;
    const int col0 = it.col0 + rank * kBCols;
    const int boxes = TRANSPOSED ? kBCols / 64 : min(kBCols / 64, max(0, (a.p.n - col0 + 63) / 64));   // columns behind the last are left out: they meet no result
    // a group's last rows, of single tokens all it has, come without the rows behind them; what else is in the tile meets no result
    const int few = PAIR ? kBM : (it.left + kFewRows - 1) / kFewRows;
    if (few * kFewRows <= kBM / 2) {
      expect<THERE>(bar, (uint32_t)(few * kFewRows * 128 + boxes * kGroup64));
      for (int i = 0; i < few; ++i) copy_2d<THERE>(tile + i * kFewRows * 128, &a.few, c * kBK, it.row0 + i * kFewRows, bar);
    } else {
      expect<THERE>(bar, (uint32_t)(kATile + boxes * kGroup64));
      copy_2d<THERE>(tile, &a.a, c * kBK, it.row0, bar);
    }
    if constexpr (TRANSPOSED) {
      copy_3d<THERE>(tile + kATile, &a.b, c * kBK, col0, it.g, bar);
    } else {
      for (int b = 0; b < boxes; ++b) copy_3d<THERE>(tile + kATile + b * kGroup64, &a.b, col0 + 64 * b, c * kBK, it.g, bar);
    }
  }
  __device__ __forceinline__ void copy_b(const Item& it, int c, uint32_t tile, uint32_t bar) const {
    const int boxes = TRANSPOSED ? BN / 64 : min(BN / 64, (it.n + 63) / 64);
    expect<false>(bar, (uint32_t)(PARTS * boxes * kGroup64));
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      const uint32_t to = tile + part * (BN * kBK * 2);
      const int z = part * groups.count + it.g;
      if constexpr (TRANSPOSED) {
        copy_3d<false>(to, &a.b, c * kBK, it.col0, z, bar);
      } else {
        for (int b = 0; b < boxes; ++b) copy_3d<false>(to + b * kGroup64, &a.b, it.col0 + 64 * b, c * kBK, z, bar);
      }
    }
  }
  __device__ __forceinline__ void load_a(const Item& it, int c, int at, Raw<T>& raw) const {
    const int row = at >> 3, k = c * kBK + (at & 7) * 8;
    raw.template load<VEC>(static_cast<const T*>(a.p.x) + (long long)(it.row0 + row) * a.p.ldx + k, row < it.left ? a.p.k - k : 0);
  }
  __device__ __forceinline__ void load_b(const Item& it, int c, int at, Raw<T>& raw) const {
    const T* const w = static_cast<const T*>(a.p.w) + (long long)it.g * a.p.stride_w;
    if constexpr (TRANSPOSED) {
      const int col = at >> 3, k = c * kBK + (at & 7) * 8;
      raw.template load<VEC>(w + (long long)(it.col0 + col) * a.p.ldw + k, col < it.n ? a.p.k - k : 0);
    } else {
      const int k = c * kBK + at / (BN / 8), col = at % (BN / 8) * 8;
      raw.template load<VEC>(w + (long long)k * a.p.ldw + it.col0 + col, k < a.p.k ? it.n - col : 0);
    }
  }
  using Early = Nothing;
  __device__ __forceinline__ void early(const Item&, int, Early&) const {}
  template <int NC>
  __device__ __forceinline__ void finish(const Item& it, const float (&acc)[NC], Early&, uint8_t* buf, int warp) const {
    const int row = (warp & 3) * 32, col = (warp >> 2) * NC;
    const long long at = (it.row0 + row) * a.p.ldy + it.col0 + col;
    void* const y = a.p.out_type == kF32 ? (void*)(static_cast<float*>(a.p.y) + at) : (void*)(static_cast<unsigned short*>(a.p.y) + at);
    store_rows<NC>(acc, buf, y, a.p.ldy, a.p.out_type, a.boundary, it.left - row, it.n - col);
  }
};

// ---- dw_g = x_g^T y_g --------------------------------------------------------------------------------
// Tiles of groups of unequal length do not share out evenly.  Workers (blocks, or pairs of blocks) take whole tiles in turn while
// there is more than one round of them left (all of them, from kWholeRounds on), so that those at work at the same time read the same group's rows; what remains, up to two rounds, is seen as one
// stretch of chunks (group, tile, chunk of rows in this order), of which every worker gets what brings it to the mean.  So few
// tiles still fill the chip, and with fewer than kWholeRounds rounds a long group is not walked by one worker while the others wait.  From there on tiles are dealt by
// their number alone: a group far longer than the others keeps the workers of its tiles (600 groups of 64 x 64, one of 150000 rows and the others of ten: 810 us;
// as many rows in equal groups: 20).  (169343 x 256 x 40 in 32 groups, 64 tiles: 143 us in
// pieces of a length fixed beforehand, 88 us so; all work as one stretch took 259 us for 16384 x 2048 x 1024 in 16 groups, where each worker read rows of its
// own, instead of 118.)
// A tile that several workers share is put together from their sums, which they leave in the workspace: whoever comes last of up
// to kJoin workers adds theirs up, in the order of the work; where there are more, whoever comes last of these adds those up in turn.
struct ProductTnArgs {
  CUtensorMap a, b;
  ProductTn p;
  int* error_flag;
  bool vec_x, vec_y;    // rows start on 16-byte boundaries
  int boundary;         // of the rows of dw
  float* space;         // two tiles of sums for every block
  unsigned* tickets;    // three for every block
};
constexpr int kJoin = 12;        // one block reads the sums of all, one after the other: 148 of them took 148 us
constexpr int kWholeRounds = 4;  // of whole tiles, from which no stretch is made: its sums, at the end of all work, cost as much as the last round's gaps
constexpr int kLeastChunks = 4;  // of a worker: below, the sums cost more than what they spread

template <typename T_, int PARTS, int BN, bool TMA, bool PAIR = false, bool VEC = false>
struct ProductTnJob {
  using T = T_;
  using Args = ProductTnArgs;
  using Size = unsigned long long;
  static constexpr int kParts = PARTS, kBN = BN;
  static constexpr bool kAMn = true, kBMn = true, kTma = TMA, kTmaB = false, kTailed = TMA, kMeets = true, kPair = PAIR;
  static constexpr int kTileRows = PAIR ? 2 * kBM : kBM, kRanks = PAIR ? 2 : 1;
  struct Item {
    int chunks, n, tail, g, row0, end, m0, col0;
    unsigned from, pieces, piece;   // first worker of the tile, number of them, which of them this one is
  };
  struct Walk {
    Size at, end;      // of the stretch
    unsigned round, worker;
  };
  const Args& a;
  Size* ends;          // [groups] chunks of this group and all before it
  int *begin, *end;    // [groups] rows
  int* last;
  Size* shares;        // [workers + 1] where each worker's part of the stretch begins
  int count, tiles_n, tiles, rank;
  unsigned workers, rounds;
  __device__ __forceinline__ ProductTnJob(const Args& args, uint8_t* tables, int rank_)
      : a(args), ends(reinterpret_cast<Size*>(tables)), begin(reinterpret_cast<int*>(tables) + 2 * kMaxGroups), end(reinterpret_cast<int*>(tables) + 3 * kMaxGroups),
        last(reinterpret_cast<int*>(tables) + 4 * kMaxGroups), shares(reinterpret_cast<Size*>(tables) + 2 * kMaxGroups + 2), count(args.p.groups), tiles_n((args.p.nb + BN - 1) / BN),
        tiles(tiles_n * ((args.p.ka + kTileRows - 1) / kTileRows)), rank(rank_) {}
  __device__ __forceinline__ bool bf16() const { return PARTS > 1 || a.p.type == kBf16; }
  __device__ __forceinline__ int segment() const { return a.p.out_type == kF32 ? 4 : 16; }
  __device__ __forceinline__ int* error_flag() const { return a.error_flag; }
  // Chunks of a tile of group g; a group without rows has one, which writes zeros.
  __device__ __forceinline__ unsigned chunks_of(int g) const { return (unsigned)max(1, (end[g] - begin[g] + kBK - 1) / kBK); }
  __device__ __forceinline__ void setup() {
    for (int g = threadIdx.x; g < count; g += blockDim.x) {
      const int2 r = group_rows(a.p.offsets, g, (int)a.p.rows);
      begin[g] = r.x;
      end[g] = r.y;
      ends[g] = (Size)chunks_of(g) * tiles;
    }
    __syncthreads();
    if (threadIdx.x < 32) scan(ends, count);
    __syncthreads();
    const Size total = ends[count - 1], all = (Size)count * tiles;
    workers = (unsigned)min((Size)gridDim.x / kRanks, max((Size)1, total / kLeastChunks));
    rounds = (unsigned)(all / workers >= kWholeRounds ? (all + workers - 1) / workers : all / workers >= 2 ? all / workers - 1 : 0);
    if (all / workers >= kWholeRounds) return;
    // what a worker is short of the mean after its rounds, and of the stretch as much in proportion (and one chunk, so that none is left out)
    if (threadIdx.x < workers) {
      Size load = 0;
      for (unsigned r = 0; r < rounds; ++r) load += chunks_of((int)(((Size)r * workers + threadIdx.x) / tiles));
      shares[threadIdx.x] = total / workers > load ? total / workers - load : 1;
    }
    __syncthreads();
    if (threadIdx.x < 32) {
      scan(shares, (int)workers);
      __syncwarp();
      const Size stretch = total - first_of_stretch(), sum = shares[workers - 1];
      for (int p = (int)((workers - 1) / 32 * 32); p >= 0; p -= 32) {   // from behind: share p goes to place p + 1
        const unsigned w = (unsigned)p + threadIdx.x;
        const Size to = w < workers ? w + 1 + (Size)((double)(stretch - workers) * ((double)shares[w] / (double)sum)) : 0;
        __syncwarp();
        if (w < workers) shares[w + 1] = w + 1 == workers ? stretch : to;
        __syncwarp();
      }
      if (threadIdx.x == 0) shares[0] = 0;
    }
  }
  // Chunks ahead of the stretch, which begins with a whole tile.
  __device__ __forceinline__ Size first_of_stretch() const {
    const Size tile = (Size)rounds * workers;
    const int g = (int)(tile / tiles);
    return (g > 0 ? ends[g - 1] : 0) + (tile - (Size)g * tiles) * chunks_of(g);
  }
  __device__ __forceinline__ unsigned owner(Size at) const {
    unsigned lo = 0, hi = workers - 1;
    while (lo < hi) {
      const unsigned mid = (lo + hi) >> 1;
      if (shares[mid + 1] > at) hi = mid;
      else lo = mid + 1;
    }
    return lo;
  }
  __device__ __forceinline__ Walk start(unsigned worker, unsigned) const {
    if (worker >= workers) return Walk{0, 0, rounds, worker};
    if ((Size)rounds * workers >= (Size)count * tiles) return Walk{0, 0, 0, worker};   // no stretch
    return Walk{shares[worker], shares[worker + 1], 0, worker};
  }
  __device__ __forceinline__ bool next(Walk& w, Item& it) const {
    it.pieces = 1;
    it.piece = 0;
    it.from = w.worker;
    unsigned tile, c0 = 0, per, c1;
    if (w.round < rounds) {
      const Size i = (Size)w.round * workers + w.worker;
      if (i >= (Size)count * tiles) return false;
      ++w.round;
      it.g = (int)(i / tiles);
      tile = (unsigned)(i - (Size)it.g * tiles);
      c1 = per = chunks_of(it.g);
    } else {
      if (w.at >= w.end) return false;
      const Size ahead = first_of_stretch(), at = ahead + w.at;
      int lo = 0, hi = count - 1;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] > at) hi = mid;
        else lo = mid + 1;
      }
      it.g = lo;
      per = chunks_of(lo);
      const Size local = at - (lo > 0 ? ends[lo - 1] : 0);
      tile = (unsigned)(local / per);
      c0 = (unsigned)(local - (Size)tile * per);
      c1 = (unsigned)min((Size)per, c0 + (w.end - w.at));
      if (c0 > 0 || c1 < per) {
        const Size begins = w.at - c0;
        it.from = owner(begins);
        it.pieces = owner(begins + per - 1) - it.from + 1;
        it.piece = w.worker - it.from;
      }
      w.at += c1 - c0;
    }
    it.m0 = (int)(tile / tiles_n) * kTileRows + rank * kBM;
    it.col0 = (int)(tile % tiles_n) * BN;
    it.n = a.p.nb - it.col0;
    it.row0 = begin[it.g] + (int)c0 * kBK;
    it.end = c1 < per ? begin[it.g] + (int)c1 * kBK : end[it.g];
    it.chunks = (it.end - it.row0 + kBK - 1) / kBK;
    it.tail = it.end - it.row0 - (it.chunks - 1) * kBK;
    return true;
  }
  template <bool THERE>
  __device__ __forceinline__ void copy(const Item& it, int c, uint32_t tile, uint32_t bar) const {
    constexpr int kBCols = PAIR ? BN / 2 : BN;
    const int col0 = it.col0 + rank * kBCols, row = it.row0 + c * kBK;
    const int boxes_a = min(kBM / 64, max(0, (a.p.ka - it.m0 + 63) / 64)), boxes_b = min(kBCols / 64, max(0, (a.p.nb - col0 + 63) / 64));
    expect<THERE>(bar, (uint32_t)((boxes_a + boxes_b) * kGroup64));
    for (int b = 0; b < boxes_a; ++b) copy_2d<THERE>(tile + b * kGroup64, &a.a, it.m0 + 64 * b, row, bar);
    for (int b = 0; b < boxes_b; ++b) copy_2d<THERE>(tile + kATile + b * kGroup64, &a.b, col0 + 64 * b, row, bar);
  }
  __device__ __forceinline__ void load_a(const Item& it, int c, int at, Raw<T>& raw) const {
    const int col = it.m0 + at % (kBM / 8) * 8, row = it.row0 + c * kBK + at / (kBM / 8);
    raw.template load<VEC>(static_cast<const T*>(a.p.x) + (long long)row * a.p.ldx + col, row < it.end ? a.p.ka - col : 0);
  }
  __device__ __forceinline__ void load_b(const Item& it, int c, int at, Raw<T>& raw) const {
    const int col = it.col0 + at % (BN / 8) * 8, row = it.row0 + c * kBK + at / (BN / 8);
    raw.template load<VEC>(static_cast<const T*>(a.p.y) + (long long)row * a.p.ldy + col, row < it.end ? a.p.nb - col : 0);
  }
  // The sums of a worker: of the tile it begins (but does not end) or of the one it continues.  It has at most one of each.
  template <int NC>
  __device__ __forceinline__ float* sums(unsigned worker, bool begins, int warp) const {
    return a.space + (((size_t)worker * 2 + begins) * kRanks + rank) * (kBM * BN) + (size_t)warp * NC * 32 + (threadIdx.x & 31);
  }
  // Leaves acc with the others' and says, to all epilogue warps, whether all `of` are there.
  template <int NC>
  __device__ __forceinline__ bool leave(const float (&acc)[NC], float* at, unsigned* ticket, unsigned of, int columns) const {
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (c < columns) __stcg(at + c * 32, acc[c]);
    __threadfence();
    asm volatile("bar.sync 1, 256;" ::: "memory");
    if (threadIdx.x == 0) {
      *last = atomicAdd(ticket, 1u) + 1 == of;
      if (*last) *ticket = 0u;
      __threadfence();
    }
    asm volatile("bar.sync 1, 256;" ::: "memory");
    const bool all = *last != 0;
    asm volatile("bar.sync 1, 256;" ::: "memory");
    return all;
  }
  using Early = Nothing;
  __device__ __forceinline__ void early(const Item&, int, Early&) const {}
  template <int NC>
  __device__ __forceinline__ void finish(const Item& it, float (&acc)[NC], Early&, uint8_t* buf, int warp) const {
    const int row = it.m0 + (warp & 3) * 32, col = it.col0 + (warp >> 2) * NC;
    if (it.pieces > 1) {
      const int columns = a.p.ka - row > 0 ? a.p.nb - col : 0;   // that come to anything
      const auto of_piece = [&](unsigned piece) { return sums<NC>(it.from + piece, piece == 0, warp); };
      const auto add_up = [&](unsigned from, unsigned to, unsigned step) {
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[c] = 0.f;
        for (unsigned q = from; q < to; q += step) {
          const float* const at = of_piece(q);
#pragma unroll
          for (int c = 0; c < NC; ++c)
            if (c < columns) acc[c] += __ldcg(at + c * 32);
        }
      };
      const unsigned join = it.piece / kJoin, first = join * kJoin, behind = min(it.pieces, first + kJoin);
      // tickets of the blocks that begin a tile, that begin a later join of one, and of the joins of a tile
      const unsigned all = gridDim.x, mine = (it.from + first) * kRanks + rank;
      if (!leave<NC>(acc, of_piece(it.piece), a.tickets + (join > 0 ? all : 0u) + mine, behind - first, columns)) return;
      add_up(first, behind, 1);
      if (it.pieces > kJoin) {
        if (!leave<NC>(acc, of_piece(first), a.tickets + 2 * all + it.from * kRanks + rank, (it.pieces + kJoin - 1) / kJoin, columns)) return;
        add_up(0, it.pieces, kJoin);
      }
    }
    const long long at = it.g * a.p.stride_dw + row * a.p.lddw + col;
    void* const dw = a.p.out_type == kF32 ? (void*)(static_cast<float*>(a.p.dw) + at) : (void*)(static_cast<unsigned short*>(a.p.dw) + at);
    store_rows<NC>(acc, buf, dw, a.p.lddw, a.p.out_type, a.boundary, a.p.ka - row, a.p.nb - col);
  }
};

// ---- orthogonalised updates --------------------------------------------------------------------------
// X <- P X with P = a I + b S + c S S, S = X X^T; for matrices taller than wide X <- X P with S = X^T X.  Three products a step, of pairs of halves (three matrix
// instructions for one, 22 bits of each operand), whatever the type of the result.  (Single halves are enough for the rounding of a bf16 result as long as it lasts a few
// steps, but steps lift small singular values, and what they are off, by |a| each: ten steps of a matrix of a hundred strong directions over a floor of
// 1e-3 ended 4e-2 off, coefficients whose curve is steep at 1 nowhere near.)
// Matrices between products are images: part hi of all matrices, then part lo, rows padded to 32 bytes, under a power of two that comes from
// the bounds of the singular values (step_factors(), for each matrix from its own norm: beside eps it may be tiny): entries stay below 2^15 and
// far above the smallest half.  S and P are symmetric: only
// tiles that reach the diagonal are formed, the others are written turned.  X keeps its own orientation throughout, so nothing is transposed.
struct Image {
  __half* at;
  int rows, ld;            // ld: columns rounded up to 16, so that rows are whole sectors
  long long part;          // from hi to lo
  __device__ __forceinline__ __half* matrix(int b) const { return at + (long long)b * rows * ld; }
};

constexpr int kNormBlocks = 256;   // partial sums of a norm, at most

// Partial sums of squares of every matrix; in fp64: squares of fp32 numbers leave the range of fp32.  (One load a thread and 64 blocks took 520 us
// of 4096 x 4096 halves, eight elements a load and as many blocks as there is work for 24.)
template <typename T>
__global__ void __launch_bounds__(256) k_norm(const Orthogonal p, bool vec, double* __restrict__ partial) {
  gtc::enter_kernel();
  __shared__ double s_sum[8];
  const T* const g = static_cast<const T*>(p.g) + (long long)blockIdx.y * p.stride_g;
  const unsigned units = (p.cols + 7) / 8, count = (unsigned)p.rows * units;
  double sum = 0.0;
  for (unsigned e = blockIdx.x * 256 + threadIdx.x; e < count; e += gridDim.x * 256) {
    const unsigned row = e / units, col = (e - row * units) * 8;
    float v[8];
    load8(g + row * p.ldg + col, p.cols - (int)col, vec, v);
    double part[2] = {0.0, 0.0};
#pragma unroll
    for (int k = 0; k < 8; ++k) part[k & 1] = fma((double)v[k], (double)v[k], part[k & 1]);
    sum += part[0] + part[1];
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) sum += s_sum[w];
    partial[blockIdx.y * kNormBlocks + blockIdx.x] = sum;
  }
}

struct Steps {
  int count;
  float c[3 * kMaxSteps];
};
// What the three products of each step multiply with, for every matrix: StepFactors, a float4 each: of the sums; of S (X: of the result); of the diagonal.
struct Factors {
  float4* at;
  int batch;
  __host__ __device__ __forceinline__ float4* of(int step, int stage) const { return at + ((size_t)step * 3 + stage) * batch; }
};

// X_0 = G / (||G|| + eps), to its image; with no steps to take, p.scale times it, to the result.  A thread has eight elements of a row at a time.  The last
// block of each matrix follows the scales through the steps meanwhile.
constexpr int kStartBlocks = 8 * kSms;   // of all matrices together, or one for each: finding out a scale costs a block more than 2048 elements (16 of
// 1024 x 2048: 60 us with a block for every 2048 elements, 38 so)
template <typename T, typename O>
__global__ void __launch_bounds__(256) k_start(const Orthogonal p, bool vec, const double* __restrict__ partial, int partials, const Image x, const __grid_constant__ Steps steps,
                                               const Factors factors) {
  gtc::enter_kernel();
  __shared__ double s_sum[8];
  __shared__ Stationary s_at[kMaxSteps];
  __shared__ double s_most[kMaxSteps];
  const unsigned blocks = gridDim.x - 1;
  if (blockIdx.x == blocks && (int)threadIdx.x < steps.count) {
    const float* const c = steps.c + 3 * threadIdx.x;
    s_at[threadIdx.x] = stationary(c[0], c[1], c[2]);
  }
  double sum = (int)threadIdx.x < partials ? partial[blockIdx.y * kNormBlocks + threadIdx.x] : 0.0;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  sum = 0.0;
  for (int w = 0; w < 8; ++w) sum += s_sum[w];
  const double norm = sqrt(sum) + (double)p.eps;
  // a zero matrix stays zero, one that is not finite becomes NaN
  const double inverse = !(norm > 0.0) ? (sum == 0.0 ? 0.0 : nan("")) : norm < INFINITY ? 1.0 / norm : nan("");
  const double first = first_bound(sqrt(sum) * inverse);
  if (blockIdx.x == blocks) {
    double most = first;
    for (int i = 0; threadIdx.x == 0 && i < steps.count; ++i) {
      s_most[i] = most;
      most = bound_behind(grow(most, steps.c[3 * i], steps.c[3 * i + 1], steps.c[3 * i + 2], s_at[i]));
    }
    __syncthreads();
    const int i = (int)threadIdx.x;
    if (i < steps.count) {
      const float* const c = steps.c + 3 * i;
      const StepFactors f = step_factors(s_most[i], grow(s_most[i], c[0], c[1], c[2], s_at[i]), c[0], c[1], c[2], i + 1 == steps.count, p.scale);
      factors.of(i, 0)[blockIdx.y] = make_float4(f.gram, 0.f, 0.f, 0.f);
      factors.of(i, 1)[blockIdx.y] = make_float4(f.square, f.linear, f.diagonal, 0.f);
      factors.of(i, 2)[blockIdx.y] = make_float4(f.move, f.scale, 0.f, 0.f);
    }
    return;
  }
  const double by = x.at != nullptr ? ldexp(inverse, scale_for(first)) : inverse;
  const float scale = x.at != nullptr ? 1.f : p.scale;
  const T* const g = static_cast<const T*>(p.g) + (long long)blockIdx.y * p.stride_g;
  const unsigned units = x.ld / 8, count = (unsigned)p.rows * units;
  for (unsigned e = blockIdx.x * 256 + threadIdx.x; e < count; e += blocks * 256) {
    const unsigned row = e / units, col = (e - row * units) * 8;
    float v[8];
    load8(g + row * p.ldg + col, p.cols - (int)col, vec, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)((double)v[k] * by) * scale;
    if (x.at != nullptr) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const __half2 h = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
        const float2 f = __half22float2(h);
        const __half2 l = __floats2half2_rn((v[2 * k] - f.x) * 0x1p11f, (v[2 * k + 1] - f.y) * 0x1p11f);
        hi[k] = *reinterpret_cast<const uint32_t*>(&h);
        lo[k] = *reinterpret_cast<const uint32_t*>(&l);
      }
      __half* const at = x.matrix(blockIdx.y) + (long long)row * x.ld + col;
      *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(at + x.part) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    } else {
      O* const at = static_cast<O*>(p.out) + (long long)blockIdx.y * p.stride_o + row * p.ldo + col;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if ((int)col + k < p.cols) put(at + k, v[k]);
    }
  }
}

// Matrices whose shorter side is at most 32, all steps in one launch: a block has a matrix in its shared memory, in fp32 and with fp32 FMA.  (Through the tensor cores
// every step is three launches of tiles that are nearly empty: eight matrices of 128 x 16 took 73 us, 16 us so.)
// X lies as [n][M], its shorter side, padded to M, contiguous.  S: every warp adds up the products of its part of the n steps, a lane the M / 8 x M / 4
// entries at its place, and the warps' sums are added in order.  X <- P X: a thread has columns of its own and reads P, the same for all.
constexpr int kSmallSide = 32, kSmallThreads = 512, kSmallBytes = 160 * 1024;
template <int M>
constexpr size_t small_bytes(int n) {
  return ((size_t)n * M + (kSmallThreads / 32) * M * M + 2 * M * M) * sizeof(float);
}
template <int M, typename T, typename O>
__global__ void __launch_bounds__(kSmallThreads) k_small(const Orthogonal p, const __grid_constant__ Steps steps) {
  gtc::enter_kernel();
  constexpr int kWarps = kSmallThreads / 32, TI = M / 8, TJ = M / 4;
  extern __shared__ __align__(16) float small_smem[];
  __shared__ double s_sum[kWarps];
  const bool tall = p.rows > p.cols;
  const int m = tall ? p.cols : p.rows, n = tall ? p.rows : p.cols, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  float* const x = small_smem;
  float* const part = x + (size_t)n * M;               // [kWarps][M][M]
  float *const s = part + kWarps * M * M, *const f = s + M * M;
  const T* const g = static_cast<const T*>(p.g) + (long long)blockIdx.x * p.stride_g;
  const auto index = [&](int e, int& i, int& k) {      // of the e-th element as it lies in memory
    const int row = e / p.cols, col = e - row * p.cols;
    i = tall ? col : row;
    k = tall ? row : col;
    return row * p.ldg + col;
  };
  for (int e = tid; e < n * M; e += kSmallThreads) x[e] = 0.f;
  __syncthreads();
  double sum = 0.0;
  for (int e = tid; e < m * n; e += kSmallThreads) {
    int i, k;
    const float v = to_float(g[index(e, i, k)]);
    x[k * M + i] = v;
    sum = fma((double)v, (double)v, sum);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) s_sum[warp] = sum;
  __syncthreads();
  sum = 0.0;
  for (int w = 0; w < kWarps; ++w) sum += s_sum[w];
  const double norm = sqrt(sum) + (double)p.eps;
  const double inverse = !(norm > 0.0) ? (sum == 0.0 ? 0.0 : nan("")) : norm < INFINITY ? 1.0 / norm : nan("");   // as k_start
  for (int e = tid; e < n * M; e += kSmallThreads) x[e] = (float)((double)x[e] * (e % M < m ? inverse : 0.0));
  __syncthreads();
  for (int step = 0; step < steps.count; ++step) {
    const float a = steps.c[3 * step], b = steps.c[3 * step + 1], c = steps.c[3 * step + 2];
    {
      const int i0 = (lane & 7) * TI, j0 = (lane >> 3) * TJ;
      float acc[TI][TJ] = {};
      for (int k = warp; k < n; k += kWarps) {
        float u[TI], v[TJ];
#pragma unroll
        for (int i = 0; i < TI; ++i) u[i] = x[k * M + i0 + i];
#pragma unroll
        for (int j = 0; j < TJ; ++j) v[j] = x[k * M + j0 + j];
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
          for (int j = 0; j < TJ; ++j) acc[i][j] = fmaf(u[i], v[j], acc[i][j]);
      }
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) part[warp * M * M + (i0 + i) * M + j0 + j] = acc[i][j];
    }
    __syncthreads();
    for (int e = tid; e < M * M; e += kSmallThreads) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) v += part[w * M * M + e];
      s[e] = v;
    }
    __syncthreads();
    for (int e = tid; e < M * M; e += kSmallThreads) {
      const int i = e / M, j = e % M;
      float v = 0.f;
#pragma unroll
      for (int q = 0; q < M; ++q) v = fmaf(s[i * M + q], s[q * M + j], v);
      f[e] = fmaf(c, v, fmaf(b, s[e], i == j ? a : 0.f));
    }
    __syncthreads();
    for (int k = tid; k < n; k += kSmallThreads) {
      float v[M];
#pragma unroll
      for (int q = 0; q < M; q += 4) {
        const float4 w = *reinterpret_cast<const float4*>(x + k * M + q);
        v[q] = w.x; v[q + 1] = w.y; v[q + 2] = w.z; v[q + 3] = w.w;
      }
#pragma unroll 4
      for (int i = 0; i < M; ++i) {
        float w[4] = {};
#pragma unroll
        for (int q = 0; q < M; q += 4) {
          const float4 h = *reinterpret_cast<const float4*>(f + i * M + q);
          w[0] = fmaf(h.x, v[q], w[0]);
          w[1] = fmaf(h.y, v[q + 1], w[1]);
          w[2] = fmaf(h.z, v[q + 2], w[2]);
          w[3] = fmaf(h.w, v[q + 3], w[3]);
        }
        x[k * M + i] = (w[0] + w[1]) + (w[2] + w[3]);
      }
    }
    __syncthreads();
  }
  O* const out = static_cast<O*>(p.out) + (long long)blockIdx.x * p.stride_o;
  for (int e = tid; e < m * n; e += kSmallThreads) {
    int i, k;
    index(e, i, k);
    const int row = tall ? k : i, col = tall ? i : k;
    put(out + row * p.ldo + col, p.scale * x[k * M + i]);
  }
}

enum Stage { kGram, kPolynomial, kMove };
struct OrthogonalArgs {
  CUtensorMap a, b;
  int* error_flag;
  int batch, rows, cols, k;     // of the products: D is rows x cols, the reduction has k steps
  const float4* factors;        // of every matrix, for this stage
  Image s, to;                  // kPolynomial: S; where the result goes
  void* out;                    // last kMove: the caller's matrix
  int out_type;
  long long ldo, stride_o;
  int boundary;                 // of its rows
};

template <Stage STAGE, int BN, bool A_MN, bool B_MN>
struct OrthogonalJob {
  using Args = OrthogonalArgs;
  static constexpr int kParts = 2, kBN = BN;
  static constexpr bool kAMn = A_MN, kBMn = B_MN, kTma = true, kTmaB = false, kTailed = false, kMeets = false, kPair = false, kSymmetric = STAGE != kMove;
  struct Item {
    int chunks, n, tail, matrix, row0, col0;
    bool turn;
  };
  const Args& a;
  __device__ __forceinline__ OrthogonalJob(const Args& args, uint8_t*, int) : a(args) {}
  __device__ __forceinline__ bool bf16() const { return false; }
  // results show where sums are cut (1000 x 767 in fp32: 4.7e-6 off with segments of 4 chunks, 1.4e-6 with one)
  __device__ __forceinline__ int segment() const { return 2; }
  __device__ __forceinline__ int* error_flag() const { return a.error_flag; }
  __device__ __forceinline__ void setup() {}
  // Tiles of a matrix: all, or for a symmetric one those of row block i whose columns do not lie behind it: kBM / BN (i + 1)
  __host__ __device__ static long long tiles(int rows, int cols) {
    const long long m = (rows + kBM - 1) / kBM;
    return kSymmetric ? kBM / BN * (m * (m + 1) / 2) : m * ((cols + BN - 1) / BN);
  }
  struct Walk {
    unsigned i, step;
  };
  __device__ __forceinline__ Walk start(unsigned worker, unsigned workers) const { return Walk{worker, workers}; }
  __device__ __forceinline__ bool next(Walk& at, Item& it) const {
    const unsigned per = (unsigned)tiles(a.rows, a.cols), i = at.i;
    it.matrix = (int)(i / per);
    if (it.matrix >= a.batch) return false;
    at.i += at.step;
    const unsigned t = i - (unsigned)it.matrix * per;
    unsigned row, col;
    if constexpr (kSymmetric) {
      constexpr unsigned kAcross = kBM / BN;
      const unsigned u = t / kAcross;   // in blocks of kBM columns
      row = (unsigned)((sqrtf(8.f * (float)u + 1.f) - 1.f) * 0.5f);
      while (row * (row + 1) / 2 > u) --row;
      while ((row + 1) * (row + 2) / 2 <= u) ++row;
      col = t - kAcross * (row * (row + 1) / 2);
    } else {
      const unsigned across = (unsigned)((a.cols + BN - 1) / BN);
      row = t / across;
      col = t - row * across;
    }
    it.col0 = (int)col * BN;
    it.turn = kSymmetric && it.col0 + BN <= (int)row * kBM;
    it.row0 = (int)row * kBM;
    it.n = a.cols - it.col0;
    it.chunks = it.n > 0 ? (a.k + kBK - 1) / kBK : 0;   // (a symmetric matrix's last row block may reach past its columns)
    it.tail = kBK;
    return true;
  }
  template <bool THERE>
  __device__ __forceinline__ void copy(const Item& it, int c, uint32_t tile, uint32_t bar) const {
    constexpr int kBTile = BN * kBK * 2;
    const int col0 = it.col0;
    const int boxes_a = A_MN ? min(kBM / 64, max(0, (a.rows - it.row0 + 63) / 64)) : kBM / 64, boxes_b = B_MN ? min(BN / 64, max(0, (a.cols - col0 + 63) / 64)) : BN / 64;
    expect<THERE>(bar, (uint32_t)(kParts * (boxes_a + boxes_b) * kGroup64));
#pragma unroll
    for (int part = 0; part < kParts; ++part) {
      const int z = part * a.batch + it.matrix;
      const uint32_t ta = tile + part * kATile, tb = tile + kParts * kATile + part * kBTile;
      if constexpr (A_MN) {
        for (int b = 0; b < boxes_a; ++b) copy_3d<THERE>(ta + b * kGroup64, &a.a, it.row0 + 64 * b, c * kBK, z, bar);
      } else {
        copy_3d<THERE>(ta, &a.a, c * kBK, it.row0, z, bar);
      }
      if constexpr (B_MN) {
        for (int b = 0; b < boxes_b; ++b) copy_3d<THERE>(tb + b * kGroup64, &a.b, col0 + 64 * b, c * kBK, z, bar);
      } else {
        copy_3d<THERE>(tb, &a.b, c * kBK, col0, z, bar);
      }
    }
  }
  // 32 elements of this lane's row of an image, two sectors of each part.  On their way while the columns before are worked on, the first while the
  // tile's products are formed.
  static constexpr bool kReads = STAGE == kPolynomial;
  struct Block {
    uint32_t hi[16], lo[16];
  };
  struct Early : std::conditional_t<kReads, Block, Nothing> {
    float4 factors;   // of the matrix, on their way while its products are formed
  };
  __device__ __forceinline__ void fetch(const Item& it, int row, int col, Block& b) const {
    const __half* const at = a.s.matrix(it.matrix) + (long long)row * a.s.ld + col;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (row < a.s.rows && col + 16 * h < a.s.ld) {
        load32(at + 16 * h, b.hi + 8 * h);
        load32(at + 16 * h + a.s.part, b.lo + 8 * h);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) b.hi[8 * h + e] = b.lo[8 * h + e] = 0u;
      }
    }
  }
  __device__ __forceinline__ void early(const Item& it, int warp, Early& b) const {
    b.factors = __ldg(a.factors + it.matrix);
    if constexpr (kReads) fetch(it, it.row0 + (warp & 3) * 32 + (threadIdx.x & 31), it.col0 + (warp >> 2) * (BN / 2), b);
  }
  __device__ __forceinline__ static float2 floats(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
  // 32 rows x 32 columns of halves, a row a lane, as columns x rows of the turned matrix at `out`: 64 bytes of a row at once.
  __device__ __forceinline__ static void put_turned(const uint32_t (&w)[16], __half* out, long long ld, int rows_left, int cols_left) {
    const int lane = threadIdx.x & 31;
    if (lane >= rows_left) return;
#pragma unroll
    for (int c = 0; c < 32; ++c)
      if (c < cols_left) reinterpret_cast<unsigned short*>(out)[c * ld + lane] = (unsigned short)(w[c >> 1] >> (16 * (c & 1)));
  }
  // 32 columns at a time from sums to what is stored of them: few registers beside the sums
  template <int NC>
  __device__ __forceinline__ void finish(const Item& it, float (&acc)[NC], Early& next, uint8_t* buf, int warp) const {
    const int row0 = it.row0 + (warp & 3) * 32, col0 = it.col0 + (warp >> 2) * NC, lane = threadIdx.x & 31, row = row0 + lane;
    const int rows_left = a.rows - row0, cols_left = a.cols - col0;
    if (rows_left <= 0 || cols_left <= 0) return;
    const float4 factors = next.factors;
    const float factor = factors.x, linear = factors.y, on_diagonal = factors.z;
    const bool diagonal = STAGE == kPolynomial && row0 < col0 + NC && col0 < row0 + 32;   // whether the warp holds some of it
    const bool out = STAGE == kMove && a.out != nullptr;
    const int out_size = a.out_type == kF32 ? 4 : 2;
    __half* const to = a.to.matrix(it.matrix);
    // images have room up to their leading dimension, and whole units there
    const RowStore hi_to = out ? RowStore(buf, static_cast<uint8_t*>(a.out) + ((long long)it.matrix * a.stride_o + row0 * a.ldo + col0) * out_size, a.ldo, out_size, a.boundary, rows_left, cols_left)
                               : RowStore(buf, to + (long long)row0 * a.to.ld + col0, a.to.ld, 2, 32, rows_left, a.to.ld - col0);
#pragma unroll
    for (int c0 = 0; c0 < NC; c0 += 32) {
      if (c0 < cols_left) {
        float x[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) x[c] = STAGE == kMove ? acc[c0 + c] * factor * linear : acc[c0 + c] * factor;
        if constexpr (kReads) {
          const Block now = static_cast<const Block&>(next);
          if (c0 + 32 < NC) fetch(it, row, col0 + c0 + 32, next);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float2 v = floats(now.hi[e]), low = floats(now.lo[e]);
            x[2 * e] = fmaf(linear, fmaf(low.x, 0x1p-11f, v.x), x[2 * e]);
            x[2 * e + 1] = fmaf(linear, fmaf(low.y, 0x1p-11f, v.y), x[2 * e + 1]);
          }
        }
        if (diagonal) {
#pragma unroll
          for (int c = 0; c < 32; ++c)
            if (row == col0 + c0 + c) x[c] += on_diagonal;
        }
        if (out && a.out_type == kF32) {
#pragma unroll
          for (int half = 0; half < 32; half += 16)
            if (c0 + half < cols_left)
              hi_to.put(c0 + half, words(x[half], x[half + 1], x[half + 2], x[half + 3]), words(x[half + 4], x[half + 5], x[half + 6], x[half + 7]),
                        words(x[half + 8], x[half + 9], x[half + 10], x[half + 11]), words(x[half + 12], x[half + 13], x[half + 14], x[half + 15]));
        } else {
          const int type = out ? a.out_type : (int)kF16;
          uint32_t h[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) h[e] = pack(type, x[2 * e], x[2 * e + 1]);
          hi_to.put(c0, make_uint4(h[0], h[1], h[2], h[3]), make_uint4(h[4], h[5], h[6], h[7]), make_uint4(h[8], h[9], h[10], h[11]), make_uint4(h[12], h[13], h[14], h[15]));
          if (!out) {
            __half* const turned = to + (long long)(col0 + c0) * a.to.ld + row0;
            if (it.turn) put_turned(h, turned, a.to.ld, rows_left, cols_left - c0);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float2 v = floats(h[e]);
              h[e] = pack(kF16, (x[2 * e] - v.x) * 0x1p11f, (x[2 * e + 1] - v.y) * 0x1p11f);
            }
            RowStore lo_to = hi_to;
            lo_to.out += 2 * a.to.part;
            lo_to.put(c0, make_uint4(h[0], h[1], h[2], h[3]), make_uint4(h[4], h[5], h[6], h[7]), make_uint4(h[8], h[9], h[10], h[11]), make_uint4(h[12], h[13], h[14], h[15]));
            if (it.turn) put_turned(h, turned + a.to.part, a.to.ld, rows_left, cols_left - c0);
          }
        }
      }
    }
  }
};

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

// Whether tiles of 256 columns are well filled: pairs have no narrower ones.
bool fits_pairs(int n) { return cdiv(n, 256) * 256 * 4 <= 5LL * n; }

// Whether every row of a matrix starts on a 16-byte boundary.
bool even(const void* p, long long ld, int size) { return reinterpret_cast<std::uintptr_t>(p) % 16 == 0 && ld * size % 16 == 0; }

// Bytes, 32, 16 or 1, that every row of every matrix starts at a multiple of.
int boundary_of(const void* p, long long ld, long long stride, int size) {
  const unsigned long long low = reinterpret_cast<std::uintptr_t>(p) | (unsigned long long)ld * size | (unsigned long long)stride * size;
  return low % 32 == 0 ? 32 : low % 16 == 0 ? 16 : 1;
}

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
  using G = GeometryOf<J>;
  constexpr size_t smem = 1024 + G::kTablesAt + kTableBytes;
  static_assert(smem + 512 <= 232448, "shared memory of an SM");
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  static std::atomic<unsigned long long> allowed{0};   // devices whose limit for this kernel is raised
  if (device > 63 || !(allowed.load() >> device & 1)) {
    e = cudaFuncSetAttribute(k_products<J>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    cudaFuncAttributes built;
    e = cudaFuncGetAttributes(&built, k_products<J>);
    if (e != cudaSuccess) return e;
    if (built.numRegs < (J::kTma ? 168 : 96)) return cudaErrorInvalidConfiguration;   // the registers that its warps share out (see k_products)
    if (device <= 63) allowed.fetch_or(1ull << device);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(G::kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = room.stream;
  cudaLaunchAttribute with[2]{};
  with[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  with[0].val.programmaticStreamSerializationAllowed = 1;
  with[1].id = cudaLaunchAttributeClusterDimension;
  with[1].val.clusterDim.x = 2;
  with[1].val.clusterDim.y = with[1].val.clusterDim.z = 1;
  cfg.attrs = with;
  cfg.numAttrs = J::kPair ? 2 : 1;
  ++*room.launches;
  return cudaLaunchKernelEx(&cfg, k_products<J>, args);
}

// The small kernels, launched the same way.
template <typename... P, typename... Q>
cudaError_t launch_plain_of(void (*kernel)(P...), dim3 grid, int threads, size_t smem, const Room& room, const Q&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = room.stream;
  cudaLaunchAttribute behind{};
  behind.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  behind.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &behind;
  cfg.numAttrs = 1;
  ++*room.launches;
  return cudaLaunchKernelEx(&cfg, kernel, std::remove_reference_t<P>(args)...);
}
template <typename... P, typename... Q>
cudaError_t launch_plain(void (*kernel)(P...), dim3 grid, const Room& room, const Q&... args) {
  return launch_plain_of(kernel, grid, 256, 0, room, args...);
}
template <typename T>
struct Tag {
  using Type = T;
};

}  // namespace

// Tiles of a weight gradient: 256 x 256 by pairs of blocks where both widths fill them, else 128 rows by what the columns need and the registers of a
// block that loads through them allow.
struct TnPlan {
  int bn, ranks;     // ranks: blocks of a tile
  bool tma;
  unsigned grid;
};
TnPlan plan(const ProductTn& p) {
  const bool wide = p.type != kF32;
  const int size = size_of(p.type);
  const bool tma = wide && p.rows > 0 && even(p.x, p.ldx, size) && even(p.y, p.ldy, size) && gcn_admm_host::encode_tiled() != nullptr;
  const bool pair = tma && fits_pairs(p.ka) && fits_pairs(p.nb);
  TnPlan t{p.nb <= 64 ? 64 : p.nb <= 128 || !tma ? 128 : 256, pair ? 2 : 1, tma, kSms};
  // no more than there is work for: chunks at most, wherever the groups begin, and not fewer than tiles
  const long long tiles = cdiv(p.ka, t.ranks * kBM) * cdiv(p.nb, t.bn), chunks = tiles * (cdiv(p.rows, kBK) + p.groups);
  t.grid = (unsigned)std::min<long long>(kSms, t.ranks * std::max<long long>(1, chunks / kLeastChunks));
  return t;
}
std::size_t space_bytes(const ProductTn& p) {
  const TnPlan t = plan(p);
  return 2ull * t.grid * kBM * t.bn * sizeof(float);
}
std::size_t tickets_of(const ProductTn& p) { return 3ull * plan(p).grid; }

// The images of a call in its workspace.
struct OrthogonalSpace {
  double* partial;
  Image x[2], s, p;
  Factors factors;
  std::size_t bytes;
  OrthogonalSpace(const Orthogonal& o, void* space) {
    const int m = std::min(o.rows, o.cols);
    std::size_t used = 0;
    const auto take = [&](std::size_t size) {
      void* const at = static_cast<char*>(space) + used;
      used += (size + 255) / 256 * 256;
      return at;
    };
    partial = static_cast<double*>(take((std::size_t)o.batch * kNormBlocks * sizeof(double)));
    const auto image = [&](int rows, int cols) {
      const int ld = (cols + 15) / 16 * 16;
      const long long part = (long long)o.batch * rows * ld;
      return Image{static_cast<__half*>(take(2 * part * sizeof(__half))), rows, ld, part};
    };
    x[0] = image(o.rows, o.cols);
    x[1] = image(o.rows, o.cols);
    s = image(m, m);
    p = image(m, m);
    factors = Factors{static_cast<float4*>(take((std::size_t)o.steps * 3 * o.batch * sizeof(float4))), o.batch};
    bytes = used;
  }
};
bool is_small(const Orthogonal& p);
std::size_t space_bytes(const Orthogonal& p) { return is_small(p) ? 0 : OrthogonalSpace(p, nullptr).bytes; }

// Whether the weights are split beforehand: where there are at least two tiles of rows to a group they would be split again for every one.
bool splits_weights(const Product& p) {
  const long long w_rows = p.transposed ? p.n : p.k, w_cols = p.transposed ? p.k : p.n;
  return p.type == kF32 && !p.unsplit && p.rows >= 2LL * kBM * p.groups && w_rows * cdiv(w_cols, 8) < INT_MAX && gcn_admm_host::encode_tiled() != nullptr;
}
std::size_t space_bytes(const Product& p) {
  if (!splits_weights(p)) return 0;
  const std::size_t rows = p.transposed ? p.n : p.k, ld = cdiv(p.transposed ? p.k : p.n, 8) * 8;
  return 3 * (std::size_t)p.groups * rows * ld * 2;
}

cudaError_t enqueue(const Product& p, const Room& room) {
  if (p.rows == 0) return cudaSuccess;
  ProductArgs a{};
  a.p = p;
  a.error_flag = room.error_flag;
  const int size = size_of(p.type);
  a.vec_x = even(p.x, p.ldx, size);
  a.vec_w = even(p.w, p.ldw, size) && (p.groups == 1 || p.stride_w * size % 16 == 0);
  a.boundary = boundary_of(p.y, p.ldy, 0, size_of(p.out_type));
  const long long tiles_m = std::min<long long>(p.rows, cdiv(p.rows, kBM) + p.groups);   // at most, wherever the groups begin
  if (p.type != kF32 && a.vec_x && a.vec_w && fits_pairs(p.n) && std::min<long long>(p.rows, cdiv(p.rows, 2 * kBM) + p.groups) * cdiv(p.n, 256) >= kSms / 2) {
    const long long w_rows = p.transposed ? p.n : p.k, w_cols = p.transposed ? p.k : p.n;
    if (make_map(&a.a, p.type, p.x, p.k, p.rows, p.ldx, 1, 0, kBM) && make_map(&a.b, p.type, p.w, w_cols, w_rows, p.ldw, p.groups, p.stride_w, p.transposed ? 128 : kBK))
      return p.transposed ? launch<ProductJob<unsigned short, 1, 256, true, true, true>>(a, kSms, room) : launch<ProductJob<unsigned short, 1, 256, false, true, true>>(a, kSms, room);
  }
  const bool split = splits_weights(p);
  const bool x_quads = a.vec_x && p.k % 4 == 0, quads = x_quads && a.vec_w && (p.transposed || p.n % 4 == 0);   // rows of the operands are whole quads
  const auto pick = [&](auto tma) {
    // A tile costs its columns, and its 128 rows as much as 64 columns; what counts are the tiles that one SM has.  (Eight rows of 64 groups, 1024 x 2048: 256 tiles of
    // 64 columns, two for some SMs, 18 us, 128 of 128 columns 11.)
    const auto cost = [&](int bn) { return cdiv(tiles_m * cdiv(p.n, bn), kSms) * (std::min(bn, p.n) + 64); };
    int bn = cost(128) <= cost(64) ? 128 : 64;
    if (decltype(tma)::value && cost(256) <= cost(bn)) bn = 256;
    if (p.n <= bn / 2) bn = p.n <= 64 ? 64 : 128;
    const unsigned grid = (unsigned)std::min<long long>(kSms, tiles_m * cdiv(p.n, bn));
    if (split) {
      const int w_rows = p.transposed ? p.n : p.k, w_cols = p.transposed ? p.k : p.n, ld = (w_cols + 7) / 8 * 8;
      const SplitWeights sw{static_cast<const float*>(p.w), p.ldw, p.stride_w, w_rows, w_cols, ld, p.groups, a.vec_w, static_cast<unsigned short*>(room.space)};
      const cudaError_t e = launch_plain(k_split_weights, dim3((unsigned)std::min<long long>(256, cdiv((long long)w_rows * (ld / 8), 256)), (unsigned)p.groups), room, sw);
      if (e != cudaSuccess) return e;
      if (!make_map(&a.b, kBf16, room.space, w_cols, w_rows, ld, 3LL * p.groups, (long long)w_rows * ld, p.transposed ? bn : kBK)) return cudaErrorNotSupported;
    }
    if (decltype(tma)::value) {
      const long long w_rows = p.transposed ? p.n : p.k, w_cols = p.transposed ? p.k : p.n;
      if (!make_map(&a.a, p.type, p.x, p.k, p.rows, p.ldx, 1, 0, kBM) || !make_map(&a.few, p.type, p.x, p.k, p.rows, p.ldx, 1, 0, kFewRows) ||
          !make_map(&a.b, p.type, p.w, w_cols, w_rows, p.ldw, p.groups, p.stride_w, p.transposed ? bn : kBK))
        return cudaErrorNotSupported;
    }
    const auto go = [&](auto width, auto turned) {
      constexpr int BN = decltype(width)::value;
      constexpr bool T = decltype(turned)::value;
      if constexpr (decltype(tma)::value) return launch<ProductJob<unsigned short, 1, BN, T, true>>(a, grid, room);
      else if constexpr (BN == 256) return cudaErrorNotSupported;
      else if (split && x_quads) return launch<ProductJob<float, 3, BN, T, false, false, true, true>>(a, grid, room);
      else if (split) return launch<ProductJob<float, 3, BN, T, false, false, false, true>>(a, grid, room);
      else if (p.type == kF32 && quads) return launch<ProductJob<float, 3, BN, T, false, false, true>>(a, grid, room);
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
  a.boundary = boundary_of(p.dw, p.lddw, p.groups > 1 ? p.stride_dw : 0, size_of(p.out_type));
  const TnPlan t = plan(p);
  a.space = static_cast<float*>(room.space);
  a.tickets = room.tickets;
  if (t.ranks == 2) {
    if (!make_map(&a.a, p.type, p.x, p.ka, p.rows, p.ldx, 1, 0, kBK) || !make_map(&a.b, p.type, p.y, p.nb, p.rows, p.ldy, 1, 0, kBK)) return cudaErrorNotSupported;
    return launch<ProductTnJob<unsigned short, 1, 256, true, true>>(a, t.grid, room);
  }
  const unsigned grid = t.grid;
  const auto width = [&](const auto& f) {
    return t.bn == 256 ? f(std::integral_constant<int, 256>()) : t.bn == 128 ? f(std::integral_constant<int, 128>()) : f(std::integral_constant<int, 64>());
  };
  if (t.tma) {
    if (!make_map(&a.a, p.type, p.x, p.ka, p.rows, p.ldx, 1, 0, kBK) || !make_map(&a.b, p.type, p.y, p.nb, p.rows, p.ldy, 1, 0, kBK)) return cudaErrorNotSupported;
    return width([&](auto w) { return launch<ProductTnJob<unsigned short, 1, decltype(w)::value, true>>(a, grid, room); });
  }
  return width([&](auto w) {
    constexpr int BN = decltype(w)::value;
    if constexpr (BN == 256) return cudaErrorNotSupported;
    else if (p.type != kF32) return launch<ProductTnJob<unsigned short, 1, BN, false>>(a, grid, room);
    else if (a.vec_x && a.vec_y && p.ka % 4 == 0 && p.nb % 4 == 0) return launch<ProductTnJob<float, 3, BN, false, false, true>>(a, grid, room);
    else return launch<ProductTnJob<float, 3, BN, false>>(a, grid, room);
  });
}

Steps steps_of(const Orthogonal& p) {
  Steps s{};
  s.count = p.steps;
  if (p.steps > 0) std::copy(p.coefficients, p.coefficients + 3 * p.steps, s.c);
  return s;
}

// One block a matrix, where it fits (see k_small).
bool is_small(const Orthogonal& p) {
  const int m = std::min(p.rows, p.cols), n = std::max(p.rows, p.cols);
  return m <= kSmallSide && (m <= 8 ? small_bytes<8>(n) : m <= 16 ? small_bytes<16>(n) : small_bytes<32>(n)) <= (size_t)kSmallBytes;
}
template <int M>
cudaError_t enqueue_small(const Orthogonal& p, const Room& room) {
  const Steps steps = steps_of(p);
  const size_t smem = small_bytes<M>(std::max(p.rows, p.cols));
  cudaError_t e = cudaSuccess;
  with_types(p.type, p.out_type, [&](auto in, auto out) {
    const auto kernel = k_small<M, decltype(in), decltype(out)>;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallBytes);
    if (e == cudaSuccess) e = launch_plain_of(kernel, dim3((unsigned)p.batch), kSmallThreads, smem, room, p, steps);
  });
  return e;
}

cudaError_t enqueue(const Orthogonal& p, const Room& room) {
  const int m = std::min(p.rows, p.cols);
  if (is_small(p)) return m <= 8 ? enqueue_small<8>(p, room) : m <= 16 ? enqueue_small<16>(p, room) : enqueue_small<32>(p, room);
  const bool tall = p.rows > p.cols;
  const OrthogonalSpace at(p, room.space);
  const Image none{nullptr, p.rows, at.x[0].ld, 0};
  const long long elements = (long long)p.rows * p.cols;
  const int partials = (int)std::min<long long>(kNormBlocks, cdiv(elements, 4096));
  const bool vec = even(p.g, p.ldg, size_of(p.type)) && (p.batch == 1 || p.stride_g * size_of(p.type) % 16 == 0);
  cudaError_t e = cudaSuccess;
  with_type(p.type, [&](auto in) { e = launch_plain(k_norm<decltype(in)>, dim3((unsigned)partials, (unsigned)p.batch), room, p, vec, at.partial); });
  if (e != cudaSuccess) return e;
  const unsigned start_blocks = (unsigned)std::min<long long>(cdiv(kStartBlocks, p.batch), cdiv(elements, 2048));
  with_types(p.type, p.out_type, [&](auto in, auto out) {
    e = launch_plain(k_start<decltype(in), decltype(out)>, dim3(start_blocks + 1, (unsigned)p.batch), room, p, vec, at.partial, partials,
                     p.steps > 0 ? at.x[0] : none, steps_of(p), at.factors);
  });
  const auto map = [&](CUtensorMap* t, const Image& im, int cols, int box_rows) {
    return make_map(t, kF16, im.at, cols, im.rows, im.ld, 2LL * p.batch, (long long)im.rows * im.ld, box_rows);
  };
  // the widest tile that every SM gets one of
  const int bn = p.batch * (cdiv(m, kBM) * (cdiv(m, kBM) + 1) / 2) >= kSms ? 128 : 64;
  for (int i = 0; i < p.steps && e == cudaSuccess; ++i) {
    const bool last = i + 1 == p.steps;
    const Image &x = at.x[i & 1], &y = at.x[(i + 1) & 1];
    const auto product = [&](auto tag, OrthogonalArgs& a) {
      using J = typename decltype(tag)::Type;
      a.error_flag = room.error_flag;
      a.batch = p.batch;
      const long long items = J::tiles(a.rows, a.cols) * p.batch;
      if (items > INT_MAX) return cudaErrorInvalidValue;
      return launch<J>(a, (unsigned)std::min<long long>(kSms, items), room);
    };
    OrthogonalArgs gram{}, poly{}, move{};
    gram.rows = gram.cols = m;
    gram.k = tall ? p.rows : p.cols;
    gram.factors = at.factors.of(i, 0);
    gram.to = at.s;
    poly.rows = poly.cols = poly.k = m;
    poly.factors = at.factors.of(i, 1);
    poly.s = at.s;
    poly.to = at.p;
    move.rows = p.rows;
    move.cols = p.cols;
    move.k = m;
    move.factors = at.factors.of(i, 2);
    move.to = y;
    if (last) {
      move.out = p.out;
      move.out_type = p.out_type;
      move.ldo = p.ldo;
      move.stride_o = p.stride_o;
      move.boundary = boundary_of(p.out, p.ldo, p.batch > 1 ? p.stride_o : 0, size_of(p.out_type));
    }
    const auto step = [&](auto width) {
      constexpr int BN = decltype(width)::value;
      const bool maps = map(&poly.a, at.s, m, kBM) && map(&poly.b, at.s, m, BN) &&
                        (tall ? map(&gram.a, x, p.cols, kBK) && map(&gram.b, x, p.cols, kBK) && map(&move.a, x, p.cols, kBM) && map(&move.b, at.p, m, BN)
                              : map(&gram.a, x, p.cols, kBM) && map(&gram.b, x, p.cols, BN) && map(&move.a, at.p, m, kBM) && map(&move.b, x, p.cols, kBK));
      if (!maps) return cudaErrorNotSupported;
      cudaError_t q = tall ? product(Tag<OrthogonalJob<kGram, BN, true, true>>(), gram) : product(Tag<OrthogonalJob<kGram, BN, false, false>>(), gram);
      if (q == cudaSuccess) q = product(Tag<OrthogonalJob<kPolynomial, BN, false, false>>(), poly);
      if (q == cudaSuccess) q = tall ? product(Tag<OrthogonalJob<kMove, BN, false, false>>(), move) : product(Tag<OrthogonalJob<kMove, BN, false, true>>(), move);
      return q;
    };
    e = bn == 64 ? step(std::integral_constant<int, 64>()) : step(std::integral_constant<int, 128>());
  }
  return e;
}

}  // namespace gcn_admm_grouped
