// Grouped products of an expert's matrix, for any size, stride and alignment:
// forward, gradient in the rows, gradient in the weights, and the forward in
// 8-bit integers (grouped.h states the three products in one frame).
//
// A workgroup of four waves computes a tile of 128 x 128 results; a wave holds
// 64 x 64 of them as 2 x 2 blocks of v_mfma_f32_32x32x16_bf16 (8-bit integers:
// v_mfma_i32_32x32x32_i8).  Tiles of both operands, 16 KiB each, pass through
// registers into LDS: loads into registers take any byte alignment, and what lies
// past an edge is replaced by zeros there.  The next tile's loads are in flight
// while a tile is multiplied; three workgroups to a CU cover the rest of their time
// (one LDS stage each: with two stages and two workgroups the products of odd sizes
// ran a third slower).  An operand that lies along the sum is kept as rows of 128 bytes
// and read back 16 bytes a lane; one that lies across it is kept as it comes, 64
// rows of 128 columns, and read with the transposing LDS load, which hands each
// lane four elements of its column.
//
// What bounds it: loads that straddle lines (a wave's 16-byte loads take 7.6 ns on
// aligned rows, 13.8 where rows start on any dword, 27 on any 2 bytes), then LDS.
// 8 experts of 1024 rows, 4097 x 8191: forward 0.90 ms (608 TFLOP/s), dx 0.96, dW
// 0.94; 8-bit integers 0.54 (1025 TOP/s).
#include <algorithm>

#include "grouped_fast.h"

namespace eaas {
namespace {

constexpr int kBI = 128, kBJ = 128, kThreads = 256;
constexpr int kStage = 16384;  // bytes of one operand's tile

// 16 bytes at an address of element alignment.
__device__ __forceinline__ u32x4 load16(const char* p) {
  u32x4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}

// The first n >= 1 elements of 16 bytes, zeros after them.  (Every lane loads as
// many elements as fit, the last one repeatedly: loads under a condition each would
// be waited for one by one.)
template <int ESZ>
__device__ __forceinline__ u32x4 load_some(const char* p, int n) {
  constexpr int EPC = 16 / ESZ;
  uint32_t e[EPC];
#pragma unroll
  for (int c = 0; c < EPC; ++c) {
    const char* at = p + min(c, n - 1) * ESZ;
    e[c] = ESZ == 2 ? *reinterpret_cast<const uint16_t*>(at) : *reinterpret_cast<const uint8_t*>(at);
  }
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int c = 0; c < EPC; ++c) v[c * ESZ / 4] |= (c < n ? e[c] : 0u) << (8 * (c * ESZ % 4));
  return v;
}

// One operand's tile on its way from memory to LDS.
//   ACROSS: rows are the sum's index [s0, s0 + 64) up to s_end, columns
//           [c0, c0 + 128) of `width`
//   else:   128 rows (pointers fixed for the whole sum), 128 bytes of the sum
template <bool ACROSS, int ESZ>
struct Loader {
  static constexpr int EPC = 16 / ESZ;  // elements of a chunk
  const char* row[4];                   // along: this thread's rows
  int chunk, r0;
  u32x4 v[4];

  template <class RowPtr>
  __device__ __forceinline__ void init(RowPtr rp) {
    const int tid = threadIdx.x;
    if constexpr (ACROSS) {
      chunk = tid & 15;
      r0 = tid >> 4;
    } else {
      chunk = tid & 7;
      r0 = tid >> 3;
#pragma unroll
      for (int q = 0; q < 4; ++q) row[q] = rp(q, r0 + 32 * q);
    }
  }
  // s0: the sum's index where the tile starts; s_end: where the sum ends.  (One
  // branch around all of a tile's loads: with one around each they were waited for
  // one by one, 8 round trips a tile.)
  template <class RowPtr>
  __device__ __forceinline__ void load(RowPtr rp, int s0, int s_end, int c0, int width) {
    const int c = ACROSS ? c0 + chunk * EPC : 0, s_first = ACROSS ? s0 + r0 : s0 + chunk * EPC;
    auto at = [&](int q) {
      return ACROSS ? rp(q, s_first + 16 * q) + (size_t)c * ESZ
                    : row[ACROSS ? 0 : q] + (size_t)s_first * ESZ;
    };
    const bool inside = ACROSS ? s0 + 64 <= s_end && c0 + 128 <= width : s0 + 8 * EPC <= s_end;
    if (__builtin_amdgcn_readfirstlane(inside)) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = load16(at(q));
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v[q] = u32x4{0, 0, 0, 0};
        const int n = ACROSS ? (s_first + 16 * q < s_end ? width - c : 0) : s_end - s_first;
        if (n >= EPC) v[q] = load16(at(q));
        else if (n > 0) v[q] = load_some<ESZ>(at(q), n);
      }
    }
  }
  __device__ __forceinline__ void store(LDS_AS char* stage) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (ACROSS) {
        const int r = r0 + 16 * q;
        *reinterpret_cast<LDS_AS u32x4*>(stage + r * 256 + ((chunk ^ swz_across(r)) << 4)) = v[q];
      } else {
        const int r = r0 + 32 * q;
        *reinterpret_cast<LDS_AS u32x4*>(stage + r * 128 + ((chunk ^ swz_along(r)) << 4)) = v[q];
      }
    }
  }
};

// Fragment of k-step kk for the 32 rows (along) or columns (across) from c0: lane
// l holds element l % 32 and 16 bytes of the sum, the half l / 32 of the step.
template <bool ACROSS>
__device__ __forceinline__ u32x4 fragment(const LDS_AS char* stage, int c0, int kk) {
  const int lane = threadIdx.x & (kWave - 1);
  if constexpr (ACROSS) {
    const int g = lane >> 4, i = lane & 15;
    const int c = c0 + (g & 1) * 16 + (i & 3) * 4;
    u32x4 f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int s = kk * 16 + (g >> 1) * 8 + h * 4 + (i >> 2);
      const LDS_AS char* at = stage + s * 256 + (((c >> 3) ^ swz_across(s)) << 4) + (c & 7) * 2;
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)at);
      const u32x2 w = __builtin_bit_cast(u32x2, t);
      f[2 * h] = w[0];
      f[2 * h + 1] = w[1];
    }
    return f;
  } else {
    const int r = c0 + (lane & 31);
    return *reinterpret_cast<const LDS_AS u32x4*>(stage + r * 128 +
                                                  (((2 * kk + (lane >> 5)) ^ swz_along(r)) << 4));
  }
}

template <int DIR, bool I8>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3, 3)))
void grouped_any_kernel(GroupedParams p) {
  constexpr bool A_ACROSS = DIR == kGradWeights, B_ACROSS = DIR != kForward;
  constexpr int ESZ = I8 ? 1 : 2;
  constexpr int SUM = 128 / ESZ;  // the sum's elements in a tile
  static_assert(!I8 || DIR == kForward, "8-bit integers: forward only");
  constexpr int kWaves = kThreads / kWave;
  constexpr int kLds = std::max(2 * kStage, kWaves * kWayOutBytes);
  __shared__ __attribute__((aligned(16))) char smem[kLds];
  __shared__ int s_find[kThreads / kWave + 4];
  GroupedTile t;
  if (!find_tile<DIR, kBI, kBJ, kThreads>(p, s_find, t)) return;

  const int cols = columns<DIR>(p);
  const int sum_end = DIR == kForward ? p.K : DIR == kGradRows ? p.N : t.end - t.beg;
  const int tiles = ceil_div(sum_end, SUM);
  const int split = blockIdx.y;
  const int first = (int)((long long)tiles * split / p.splits);
  const int last = (int)((long long)tiles * (split + 1) / p.splits);

  const char* w = p.b + (DIR == kGradWeights ? 0 : (size_t)t.e * p.N * p.K * ESZ);
  // rows past the tile's repeat one that exists; their results are not stored
  auto a_row = [&](int, int i) {
    if (DIR == kGradWeights) return p.a + (size_t)(t.beg + i) * p.lda * ESZ;
    const int r = t.i0 + min(i, t.i_valid - 1);
    return p.a + (size_t)(DIR == kForward ? source_row(p, r) : r) * p.lda * ESZ;
  };
  int src[4];  // kGradWeights: this thread's rows of x in the next tile to load
  auto b_row = [&](int q, int j) {
    if (DIR == kForward) return w + (size_t)min(t.j0 + j, cols - 1) * p.ldb * ESZ;
    if (DIR == kGradRows) return w + (size_t)j * p.ldb * ESZ;
    return w + (size_t)src[q] * p.ldb * ESZ;
  };
  auto find_rows = [&](int kt) {
    if constexpr (DIR == kGradWeights) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        src[q] = source_row(p, min(t.beg + kt * SUM + (int)threadIdx.x / 16 + 16 * q, t.end - 1));
    }
  };
  Loader<A_ACROSS, ESZ> la;
  Loader<B_ACROSS, ESZ> lb;
  la.init(a_row);
  lb.init(b_row);
  auto load = [&](int kt) {
    la.load(a_row, kt * SUM, sum_end, t.i0, p.N);
    lb.load(b_row, kt * SUM, sum_end, t.j0, cols);
    if (kt + 1 < last) find_rows(kt + 1);
  };

  typedef typename std::conditional<I8, i32x16, f32x16>::type Acc;
  Acc acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = Acc{};
  const int wave = threadIdx.x / kWave;
  const int wi = (wave & 1) * 64, wj = (wave >> 1) * 64;
  LDS_AS char* lds = (LDS_AS char*)smem;

  if (first < last) {
    find_rows(first);
    load(first);
    for (int kt = first; kt < last; ++kt) {
      la.store(lds);
      lb.store(lds + kStage);
      __syncthreads();
      if (kt + 1 < last) load(kt + 1);
      const LDS_AS char *sa = lds, *sb = lds + kStage;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        u32x4 fa[2], fb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) fa[i] = fragment<A_ACROSS>(sa, wi + 32 * i, kk);
#pragma unroll
        for (int j = 0; j < 2; ++j) fb[j] = fragment<B_ACROSS>(sb, wj + 32 * j, kk);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if constexpr (I8)
              acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(
                  __builtin_bit_cast(i32x4, fb[j]), __builtin_bit_cast(i32x4, fa[i]), acc[i][j], 0,
                  0, 0);
            else
              acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                  __builtin_bit_cast(bf16x8, fb[j]), __builtin_bit_cast(bf16x8, fa[i]), acc[i][j],
                  0, 0, 0);
          }
      }
      __syncthreads();
    }
  }

  // (the last barrier is behind every wave's fragment reads)
  way_out<DIR, I8>(p, t, split, wi, t.j0 + wj, acc,
                   (LDS_AS float*)(smem + wave * kWayOutBytes));
}

// The parts of a split sum joined, in ascending order: one thread for four
// columns of one row (VEC: rows of whole quads, 16 bytes a part).  Parts are loaded
// eight at a time.
template <int DIR, bool I8, bool VEC>
__global__ __launch_bounds__(256) void grouped_join_kernel(GroupedParams p) {
  typedef typename std::conditional<I8, i32x4, f32x4>::type Quad;
  typedef typename std::conditional<I8, int, float>::type One;
  const int cols = columns<DIR>(p);
  const int quads = ceil_div(cols, 4);
  const long long rows = DIR == kGradWeights ? (long long)p.E * p.N
                                             : min(max(p.offsets[p.E], 0), p.R);
  const long long first = DIR == kGradWeights ? 0 : min(max(p.offsets[0], 0), p.R);
  const size_t stride = (DIR == kGradWeights ? (size_t)p.E * p.N : (size_t)p.R) * cols;
  for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < (rows - first) * quads;
       u += (long long)gridDim.x * 256) {
    const long long row = first + u / quads;
    const int j = (int)(u % quads) * 4;
    const One* part = static_cast<const One*>(p.part) + (size_t)row * cols + j;
    Quad v = {0, 0, 0, 0};
    for (int s0 = 0; s0 < p.splits; s0 += 8) {
      Quad t[8];
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const One* at = part + (size_t)min(s0 + s, p.splits - 1) * stride;
        if constexpr (VEC) {
          t[s] = *reinterpret_cast<const Quad*>(at);
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c) t[s][c] = at[min(c, cols - 1 - j)];
        }
      }
#pragma unroll
      for (int s = 0; s < 8; ++s)
        if (s0 + s < p.splits) v += t[s];
    }
    const int e = DIR == kGradWeights ? (int)(row / p.N) : 0;
    const int i = DIR == kGradWeights ? (int)(row % p.N) : (int)row;
    if constexpr (I8) {
      // the group whose rows hold i: the last that starts at or before it
      int lo = 0, hi = p.E - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.offsets[mid] <= i) lo = mid; else hi = mid - 1;
      }
      store4<DIR>(p, lo, i, j, scaled(p, lo, p.row_scale[source_row(p, i)], j, v));
    } else {
      store4<DIR>(p, e, i, j, v);
    }
  }
}

// Row tiles of all groups together, at most: every group may end in a part tile.
long long most_row_tiles(const GroupedArgs& a, int bi) {
  return a.R / bi + std::min(a.R, a.E);
}

long long out_tiles(const GroupedArgs& a, int bi, int bj) {
  if (a.dir == kForward) return most_row_tiles(a, bi) * ceil_div(a.N, bj);
  if (a.dir == kGradRows) return most_row_tiles(a, bi) * ceil_div(a.K, bj);
  return (long long)a.E * ceil_div(a.N, bi) * ceil_div(a.K, bj);
}

// Whether the loads that go straight to LDS may be used: everything they read in
// multiples of 16 bytes (rows of W: K elements; the sum of kGradRows: N), and what
// one descriptor covers below 2 GiB: 256 rows, or with perm all tokens.
bool in_16_bytes(const GroupedArgs& a) {
  const int m = a.i8 ? 16 : 8, esz = a.i8 ? 1 : 2;
  if (a.K % m || a.lda % m || (uintptr_t)a.a % 16 || (uintptr_t)a.b % 16) return false;
  const long long ldb = a.dir == kGradWeights ? a.ldb : a.K, most = 1LL << 31;
  if (256 * esz * std::max(a.lda, ldb) >= most) return false;
  if (a.perm && a.R / a.k * (a.dir == kGradWeights ? ldb : a.lda) * esz >= most) return false;
  if (a.dir == kForward) return true;
  return a.N % m == 0 && (a.dir == kGradRows || ldb % m == 0);
}

// Which kernel computes a product, on which tiles, and in how many parts.
enum GroupedKernel { kAny, kFew, kLarge };
struct GroupedPlan {
  GroupedKernel kernel;
  int bi, bj;
  int splits;
};

// The time of a product on one kernel in us, which the choice below compares: a
// fixed part, what a tile's steps of the sum (64, or 128 in 8 bits) take on a CU of
// its own, and how workgroups that share a CU slow one another (three of the any
// kernel's fit, of which 0.65 of a step each comes out).  Splitting a sum adds a
// launch that joins its parts.  The constants are fitted to 88 of 254 shapes (groups
// of 1 to 4000 rows, 1 to 63 groups, N and K of 64 to 13000) x 4 products x up to 13
// ways of computing each, all timed: 10% off on average, and over all shapes what
// they choose takes 2% longer than the fastest way (thresholds on sizes alone: 10%
// forward, 9% 8-bit, 7% dx, 4% dW).
constexpr int kCUs = 256;

double join_us(double out, int splits) {  // (a thread's loads of its parts are a chain)
  return splits == 1 ? 0 : 3.5 + (0.06 + 1.4e-6 * out) * splits;
}

double any_us(double tiles, int steps, int splits) {
  return 6 + std::max(1.0, 0.65 * tiles * splits / kCUs) * ceil_div(steps, splits);
}

double few_us(double tiles, int steps, int bi, int splits) {  // 4 waves share the steps
  return 5 + std::max(1.0, 1.25 * tiles * splits / kCUs) *
                 (3 + (bi == 64 ? 0.6 : 0.4) * ceil_div(ceil_div(steps, splits), 4));
}

double large_us(double tiles, int steps) {
  return std::max(1.0, tiles / kCUs) * (10 + 0.92 * steps);
}

// Parts of the sum: the fewest that the estimate finds best.
template <typename F>
int best_parts(int steps, double out, F&& us, double* time) {
  int best = 1;
  *time = us(1);
  for (int s = 2; s <= steps && s <= 2 * kCUs; s += 1 + s / 8) {
    const double t = us(s) + join_us(out, s);
    if (t < *time) *time = t, best = s;
  }
  return best;
}

// The choice.  Two regions are taken before the estimates, which know no memory
// traffic; both sides measured (us, rows of each group x E groups, N x K, bf16 results):
//   Large tiles on every CU, groups of some rows and a sum of some steps: they read
//   the weights as fast as the few-rows kernel, and each byte once.  dx 24 x 32, 4096
//   x 7168: 349 large, 367 few; 16 x 128, 1536 x 2048: 148, 175; 8-bit 24 x 32: 165,
//   183; forward 64 x 32: 318, 369, but 32 x 128: 190, 177.  2500 x 16, 4096 x 512
//   (8 steps): 172 large, 238 any; but 482 x 19, 2208 x 160 (3 steps): 32, 22.
//   dW 128 x 32, 2048 x 2048: 68 large, 83 any; 64 x 128, 1536 x 2048: 147 large, 172
//   any (fp32: 274, 257); on fewer large tiles than CUs 4096 x 1, 1024 x 4096 (64 tiles):
//   75 large, 79 any in one part (61 in two: the rule looks at neither sums that long
//   nor parts; 131072 x 1, 1792 x 1792: 2172, in two parts 1598); 4096 x 8, 256 x 256 (8
//   tiles): 72 large, 22 any in 8 parts.
//   Groups of one to 24 rows, a sum of some steps: tiles of 16 or 32 rows, which the
//   others would leave mostly empty.  20 x 8, 4096 x 4096, forward: 43 few, 53 any in 3 parts,
//   63 large; 14 x 53, 160 x 3600, dx (3 steps): 49 few, 23 any.
// What the estimates decide: forward 200 x 1, 1024 x 1024: 8 few in one part, 11 in
// 4; 215 x 3, 464 x 12176: 38 few in 2 parts, 34 any in 16, 45 few in 4; 2500 x 4, 512 x
// 8192: 127 large, 130 any in 2 parts, 132 few.
// A group's rows are the mean over the groups that could have any: rows that fall on
// few of many groups take tiles for the mean.  Forward, 256 rows on 1 of 32, 4096 x
// 7168: 56 on tiles of 16 rows, 31 on 64; 96 rows on each of 16 of 128, 2048 x 2048: 63,
// large 39; but 64 on each of 8 of 128, 1536 x 2048: 20, 21 on 64, 29 large.
GroupedPlan grouped_plan(const GroupedArgs& a, bool in16) {
  const long long rows = a.R / std::max(1, std::min(a.R, a.E));  // of a group that has any
  const long long sum = a.dir == kForward ? a.K : a.dir == kGradRows ? a.N : rows;
  const int steps = ceil_div((int)sum, a.i8 ? 128 : 64);
  const double out = a.dir == kGradWeights ? (double)a.E * a.N * a.K
                                           : (double)a.R * (a.dir == kForward ? a.N : a.K);
  const double tiles = (double)out_tiles(a, kBI, kBJ);
  const long long large = out_tiles(a, 256, 256);
  const GroupedPlan on_large{kLarge, 256, 256, 1};
  GroupedPlan any{kAny, kBI, kBJ, 1};
  double t_any;
  any.splits = best_parts(steps, out, [&](int s) { return any_us(tiles, steps, s); }, &t_any);
  if (!in16) return any;
  if (a.dir == kGradWeights) return rows >= 128 && large >= 48 ? on_large : any;
  const int some = a.dir == kForward && !a.i8 ? 48 : 16;
  if (rows >= some && large >= 192 && steps >= 4) return on_large;
  GroupedPlan few{kFew, rows <= 12 ? 16 : rows <= 24 ? 32 : 64, 64, 1};
  const double cells = (double)out_tiles(a, few.bi, few.bj);
  double t_few;
  few.splits = best_parts(steps, out, [&](int s) { return few_us(cells, steps, few.bi, s); },
                          &t_few);
  if (rows <= 24 && steps >= 4) return few;
  const double t_large = large_us((double)large, steps);
  return t_large < std::min(t_any, t_few) ? on_large : t_few < t_any ? few : any;
}

// Workspace: the parts of a split sum, or the large tiles' table of row tiles.
size_t plan_bytes(const GroupedArgs& a, const GroupedPlan& g) {
  if (g.kernel == kLarge && a.dir != kGradWeights) return 16 * (1 + most_row_tiles(a, g.bi));
  if (g.splits == 1) return 0;
  const size_t rows = a.dir == kGradWeights ? (size_t)a.E * a.N : (size_t)a.R;
  return (size_t)g.splits * rows * (a.dir == kForward ? a.N : a.K) * 4;
}

template <int DIR, bool I8>
hipError_t launch_product(GroupedParams p, const GroupedArgs& a, hipStream_t stream) {
  const GroupedPlan g = grouped_plan(a, in_16_bytes(a));
  const long long tiles = out_tiles(a, g.bi, g.bj);
  if (tiles <= 0) return hipSuccess;
  if (tiles > 0x7fffffffLL) return hipErrorInvalidValue;
  p.splits = g.splits;
  hipError_t e = hipSuccess;
  if (g.kernel == kLarge) {
    e = launch_grouped_pp<DIR, I8>(p, tiles, stream);
  } else if (g.kernel == kFew) {
    if constexpr (DIR != kGradWeights) e = launch_grouped_few<DIR, I8>(p, g.bi, tiles, stream);
  } else {
    hipLaunchKernelGGL((grouped_any_kernel<DIR, I8>), tile_grid(tiles, p.splits), dim3(kThreads),
                       0, stream, p);
    e = hipGetLastError();
  }
  if (e != hipSuccess || p.splits == 1) return e;
  const int cols = DIR == kForward ? a.N : a.K;
  const long long rows = DIR == kGradWeights ? (long long)a.E * a.N : a.R;
  const long long blocks = (rows * ceil_div(cols, 4) + 255) / 256;
  const dim3 grid((unsigned)std::min<long long>(blocks, 4096)), block(256);
  if (cols % 4 == 0)
    hipLaunchKernelGGL((grouped_join_kernel<DIR, I8, true>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((grouped_join_kernel<DIR, I8, false>), grid, block, 0, stream, p);
  return hipGetLastError();
}

}  // namespace

size_t grouped_workspace(const GroupedArgs& a) {
  return plan_bytes(a, grouped_plan(a, in_16_bytes(a)));
}

size_t grouped_workspace_most(const GroupedArgs& a) {
  return std::max(plan_bytes(a, grouped_plan(a, true)), plan_bytes(a, grouped_plan(a, false)));
}

int grouped_plan_code(const GroupedArgs& a, bool in16) {
  const GroupedPlan g = grouped_plan(a, in16);
  return g.kernel + 4 * g.bi + 4096 * g.splits;
}

hipError_t launch_grouped(const GroupedArgs& a, hipStream_t stream) {
  GroupedParams p{};
  p.a = static_cast<const char*>(a.a);
  p.lda = a.lda;
  p.b = static_cast<const char*>(a.b);
  p.ldb = a.dir == kGradWeights ? a.ldb : a.K;
  p.perm = a.perm;
  p.k = a.k;
  p.offsets = a.offsets;
  p.R = a.R;
  p.E = a.E;
  p.N = a.N;
  p.K = a.K;
  p.out = a.out;
  p.ldo = a.ldo;
  p.out_fp32 = a.out_fp32;
  p.accumulate = a.accumulate;
  p.vec = a.ldo % 4 == 0 && (uintptr_t)a.out % (a.out_fp32 ? 16 : 8) == 0;
  p.vec16 = a.ldo * (a.out_fp32 ? 4 : 2) % 16 == 0 && (uintptr_t)a.out % 16 == 0;
  int shift = 0;
  while ((1LL << shift) < a.k) ++shift;
  p.k_mul = (uint32_t)(((1ULL << (31 + shift)) + a.k - 1) / a.k);
  p.k_shift = shift - 1;
  p.row_scale = a.row_scale;
  p.col_scale = a.col_scale;
  p.part = a.ws;
  p.row_tiles = static_cast<i32x4*>(a.ws);
  if (a.i8) return launch_product<kForward, true>(p, a, stream);
  if (a.dir == kForward) return launch_product<kForward, false>(p, a, stream);
  if (a.dir == kGradRows) return launch_product<kGradRows, false>(p, a, stream);
  return launch_product<kGradWeights, false>(p, a, stream);
}

}  // namespace eaas
