// Device-side parts shared by the grouped product kernels (grouped.hip, grouped_few.hip,
// grouped_pp.h and grouped_fp8.hip): parameters, the tile a workgroup works on, and stores.
//
// One frame holds the three products of an expert's matrix W [N,K]:
//   kForward   y[r,n]   = sum_k x[r,k] W[n,k]     i = r, j = n, sum over k
//   kGradRows  dx[r,k]  = sum_n dy[r,n] W[n,k]    i = r, j = k, sum over n
//   kGradWeights dW[n,k] = sum_r dy[r,n] x[r,k]   i = n, j = k, sum over r
// Operand A holds the i side and operand B the j side.  An operand lies either
// along the sum (its memory rows are i or j) or across it (its memory rows are
// the sum's index): A across in kGradWeights, B across in both gradients.
//
// Two products have an epilogue that is not the identity:
//   kSwiglu (kForward)       W is [W_gate; W_up] by rows, N = 2I.  A column tile holds as
//                            many gate rows of W as up rows, those of the same columns
//                            of h, so that the two sums a value of h needs meet in one
//                            lane.  Columns of the result are those of h, 0 .. I-1.
//   kSwigluGrad (kGradRows)  the sums are dh, which is not stored: gate and up are read
//                            and their gradients written (and h, for the gradient of
//                            the matrix that h went into).
// Operands of 8 bits are kInt8 (sums in int32, scaled once at the end) or kFp8, whose
// scales change every 128 elements of the sum: the sum over such a block is taken by
// itself and then added, scaled, to the sum at hand.
#pragma once

#include <algorithm>

#include "common.h"
#include "gemm_common.h"
#include "internal.h"
#include "swiglu.h"

namespace eaas {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

struct GroupedParams {
  const char* a;          // x | dy | dy
  long long lda;          // elements
  const char* b;          // W | W | x
  long long ldb;
  const int32_t* perm;    // kForward: rows of a; kGradWeights: rows of b; or nullptr
  int k;                  // slots per token (with perm)
  uint32_t k_mul;         // slot / k as (slot * k_mul >> 32) >> k_shift, for k > 1
  int k_shift;
  const int32_t* offsets; // [E+1]
  int R, E, N, K;
  void* out;              // y | dx | dW
  long long ldo;
  bool out_fp32;
  bool vec;               // out may be stored four columns at a time
  bool vec16;             // and 16 bytes at a time
  bool accumulate;        // kGradWeights: out += (fp32)
  const float* row_scale; // kInt8: of x's rows; kFp8: [rows, ceil(K/128)]
  const float* col_scale; // kInt8: [E,N]; kFp8: [E, ceil(N/128), ceil(K/128)]
  uint16_t* gu;           // kSwiglu: gets the sums, or nullptr; kSwigluGrad: read
  long long ldgu;
  uint16_t* h;            // kSwigluGrad: written, or nullptr
  long long ldh;
  int splits;             // the sum in this many parts, to `part` if more than one
  i32x4* row_tiles;       // large tiles: the row tiles of all groups (in the workspace)
  void* part;             // [splits][rows of out][columns] fp32 (8-bit: int32)
};

// Columns of the result (kSwiglu: of h; kSwigluGrad: of dh).
template <int DIR, int EPI = kPlain>
__device__ __forceinline__ int columns(const GroupedParams& p) {
  return DIR != kForward ? p.K : EPI == kSwiglu ? p.N / 2 : p.N;
}

__device__ __forceinline__ void group_range(const GroupedParams& p, int e, int& beg, int& end) {
  beg = min(max(p.offsets[e], 0), p.R);
  end = min(max(p.offsets[e + 1], beg), p.R);
}

// The token of a slot.
__device__ __forceinline__ int token_of(const GroupedParams& p, int slot) {
  slot = min(max(slot, 0), p.R - 1);
  return p.k == 1 ? slot : (int)(__umulhi((uint32_t)slot, p.k_mul) >> p.k_shift);
}

__device__ __forceinline__ int source_row(const GroupedParams& p, int r) {
  return p.perm ? token_of(p, p.perm[r]) : r;
}

// Two fp32 to bf16, to the nearest, ties to even (one instruction here).
__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}

// The part of a product that a workgroup computes.
struct GroupedTile {
  int e, beg, end;  // group and its rows
  int i0, j0;       // first row of out (kGradWeights: of dW[e]) and column
  int i_valid;      // rows of the tile inside the group (or N)
};

constexpr int kGroupedRun = 4;  // row tiles that share a column tile, one after the other

// Tile `local` of a group of `mt` row tiles and nt column tiles: runs of
// kGroupedRun row tiles, column tile by column tile inside a run, so tiles that
// are worked on together share both operands.
__device__ __forceinline__ void tile_of(int local, int mt, int nt, int& tm, int& tn) {
  const int run = local / (kGroupedRun * nt);
  const int here = min(kGroupedRun, mt - run * kGroupedRun);
  const int in = local - run * kGroupedRun * nt;
  tn = in / here;
  tm = run * kGroupedRun + in - tn * here;
}

// The grid of a launch over `tiles` tiles, each in `splits` parts.  (A dimension of a
// grid holds less than 2^32 threads, so many tiles lie along z too.)
constexpr long long kGridX = 1 << 22;
inline dim3 tile_grid(long long tiles, int splits) {
  return dim3((unsigned)std::min(tiles, kGridX), (unsigned)splits,
              (unsigned)((tiles + kGridX - 1) / kGridX));
}

// The tile of this workgroup; false if there is none.  kForward and kGradRows:
// the groups' row tiles are counted from the offsets (on the device), NT threads
// take consecutive groups each, and the thread whose groups hold the tile
// publishes it.  `lds` holds NT / 64 + 4 ints.  (Ends with a barrier.)
template <int DIR, int BI, int BJ, int NT, int EPI = kPlain>
__device__ __forceinline__ bool find_tile(const GroupedParams& p, int* lds, GroupedTile& t) {
  const int tile = blockIdx.x + blockIdx.z * (int)kGridX;
  if constexpr (DIR == kGradWeights) {
    const int mt = ceil_div(p.N, BI), nt = ceil_div(p.K, BJ);
    if (tile >= p.E * mt * nt) return false;
    const int id = xcd_window_remap(tile, p.E * mt * nt);
    t.e = id / (mt * nt);
    int tm, tn;
    tile_of(id - t.e * mt * nt, mt, nt, tm, tn);
    group_range(p, t.e, t.beg, t.end);
    t.i0 = tm * BI;
    t.j0 = tn * BJ;
    t.i_valid = min(BI, p.N - t.i0);
    return true;
  } else {
    constexpr int PER = ceil_div(kMaxExperts, NT);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int per = ceil_div(p.E, NT);
    int count[PER], sum = 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const int e = tid * per + q;
      count[q] = 0;
      if (q < per && e < p.E) {
        int beg, end;
        group_range(p, e, beg, end);
        count[q] = ceil_div(end - beg, BI);
      }
      sum += count[q];
    }
    int incl = sum;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const int o = __shfl_up(incl, d, kWave);
      if (lane >= d) incl += o;
    }
    int* found = lds + NT / kWave;
    if (lane == kWave - 1) lds[wave] = incl;
    if (tid == 0) found[0] = -1;
    __syncthreads();
    int before = incl - sum, total = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) {
      before += w < wave ? lds[w] : 0;
      total += lds[w];
    }
    const int nt = ceil_div(columns<DIR, EPI>(p), BJ);
    total *= nt;
    if (tile < total) {
      const int id = xcd_window_remap(tile, total);
#pragma unroll
      for (int q = 0; q < PER; ++q) {
        if (id >= before * nt && id < (before + count[q]) * nt) {
          found[0] = tid * per + q;
          found[1] = id - before * nt;
          found[2] = count[q];
        }
        before += count[q];
      }
    }
    __syncthreads();
    if (found[0] < 0) return false;
    t.e = __builtin_amdgcn_readfirstlane(found[0]);
    int tm, tn;
    tile_of(__builtin_amdgcn_readfirstlane(found[1]), __builtin_amdgcn_readfirstlane(found[2]), nt,
            tm, tn);
    group_range(p, t.e, t.beg, t.end);
    t.i0 = t.beg + tm * BI;
    t.j0 = tn * BJ;
    t.i_valid = min(BI, t.end - t.i0);
    __syncthreads();  // lds is free again
    return true;
  }
}

// Column j of row i of the result.
template <int DIR>
__device__ __forceinline__ void store1(const GroupedParams& p, int e, int i, int j, float v) {
  const size_t at = (DIR == kGradWeights ? ((size_t)e * p.N + i) : (size_t)i) * p.ldo + j;
  if (p.out_fp32) {
    float* o = static_cast<float*>(p.out) + at;
    *o = DIR == kGradWeights && p.accumulate ? *o + v : v;
  } else {
    static_cast<uint16_t*>(p.out)[at] = (uint16_t)to_bf16x2(v, 0.0f);
  }
}

// Four consecutive columns j.. of row i of the result (row of y or dx, or row n
// of dW[e]); cols: columns that exist.
template <int DIR>
__device__ __forceinline__ void store4(const GroupedParams& p, int e, int i, int j, f32x4 v) {
  const int cols = columns<DIR>(p);
  const size_t at = (DIR == kGradWeights ? ((size_t)e * p.N + i) : (size_t)i) * p.ldo + j;
  if (p.vec && j + 4 <= cols) {
    if (p.out_fp32) {
      f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at);
      *o = DIR == kGradWeights && p.accumulate ? *o + v : v;
    } else {
      u32x2 o;
      o[0] = to_bf16x2(v[0], v[1]);
      o[1] = to_bf16x2(v[2], v[3]);
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + at) = o;
    }
    return;
  }
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (j + c < cols) store1<DIR>(p, e, i, j + c, v[c]);
}

// Scales of the 8-bit product at row i and columns j..: the sum rounded to fp32,
// times the row's scale, times the columns'.
__device__ __forceinline__ f32x4 scaled(const GroupedParams& p, int e, float rs, int j, i32x4 v) {
  f32x4 o;
#pragma unroll
  for (int c = 0; c < 4; ++c)
    o[c] = (float)v[c] * rs * (j + c < p.N ? p.col_scale[(size_t)e * p.N + j + c] : 0.0f);
  return o;
}

// Columns j.. of row i of a product with an epilogue, eight or the n < 8 that exist, at
// any alignment.  kSwiglu: h, and the sums where they are kept.
__device__ __forceinline__ void store_swiglu(const GroupedParams& p, size_t i, int j, int n,
                                             const float (&g)[8], const float (&u)[8]) {
  float h[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) h[c] = gated(g[c], u[c]);
  store8(static_cast<uint16_t*>(p.out) + i * p.ldo + j, n, h);
  if (p.gu) {
    uint16_t* at = p.gu + i * p.ldgu + j;
    store8(at, n, g);
    store8(at + p.N / 2, n, u);
  }
}

// kSwigluGrad: gate and up of eight columns as they come, and what dh makes of them.  (The
// result may lie over gate and up, so the compiler keeps their loads behind earlier stores:
// where several are to be in flight, they are all taken first.)
struct GateUp {
  u32x4 gate, up;
};
__device__ __forceinline__ u32x4 load8_raw(const uint16_t* p, int n) {
  u32x4 v = {0, 0, 0, 0};
  if (n >= 8) {
    __builtin_memcpy(&v, p, 16);
  } else if (n > 0) {
    // (every element is loaded, the last one repeatedly: loads under a condition each would
    // be waited for one by one)
    uint32_t e[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) e[c] = p[min(c, n - 1)];
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c / 2] |= (c < n ? e[c] : 0u) << (16 * (c & 1));
  }
  return v;
}
__device__ __forceinline__ GateUp load_gate_up(const GroupedParams& p, size_t i, int j, int n) {
  const uint16_t* from = p.gu + i * p.ldgu + j;
  return {load8_raw(from, n), load8_raw(from + p.K, n)};
}
// (far: past the caches, for results of large products)
typedef uint32_t any4 __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void store8_raw(uint16_t* at, int n, u32x4 v, bool far) {
  if (n >= 8) {
    if (far) __builtin_nontemporal_store(v, reinterpret_cast<any4*>(at));
    else __builtin_memcpy(at, &v, 16);
  } else {
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (c < n) at[c] = (uint16_t)(v[c / 2] >> (16 * (c & 1)));
  }
}
__device__ __forceinline__ void store_swiglu_grad(const GroupedParams& p, size_t i, int j, int n,
                                                  const GateUp& x, const float (&dh)[8], bool far) {
  u32x4 dg, du, h;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const float g0 = __uint_as_float(x.gate[c] << 16), u0 = __uint_as_float(x.up[c] << 16);
    const float g1 = __uint_as_float(x.gate[c] & 0xffff0000u);
    const float u1 = __uint_as_float(x.up[c] & 0xffff0000u);
    const SwigluGrad t0 = swiglu_grad(g0, u0, dh[2 * c]), t1 = swiglu_grad(g1, u1, dh[2 * c + 1]);
    dg[c] = to_bf16x2(t0.gate, t1.gate);
    du[c] = to_bf16x2(t0.up, t1.up);
    h[c] = to_bf16x2(gated(g0, u0), gated(g1, u1));
  }
  uint16_t* to = static_cast<uint16_t*>(p.out) + i * p.ldo + j;
  store8_raw(to, n, dg, far);
  store8_raw(to + p.K, n, du, far);
  if (p.h) store8_raw(p.h + i * p.ldh + j, n, h, far);
}

// Column j of row i alone: from the sums of gate and up, or dh.
template <int EPI>
__device__ __forceinline__ void store_one(const GroupedParams& p, size_t i, int j, float a, float b) {
  uint16_t* to = static_cast<uint16_t*>(p.out) + i * p.ldo + j;
  auto bits = [](float v) { return (uint16_t)to_bf16x2(v, 0.0f); };
  if constexpr (EPI == kSwiglu) {
    *to = bits(gated(a, b));
    if (p.gu) {
      p.gu[i * p.ldgu + j] = bits(a);
      p.gu[i * p.ldgu + j + p.N / 2] = bits(b);
    }
  } else {
    const uint16_t* from = p.gu + i * p.ldgu + j;
    const float g = __uint_as_float((uint32_t)from[0] << 16);
    const float u = __uint_as_float((uint32_t)from[p.K] << 16);
    const SwigluGrad t = swiglu_grad(g, u, a);
    to[0] = bits(t.gate);
    to[p.K] = bits(t.up);
    if (p.h) p.h[i * p.ldh + j] = bits(gated(g, u));
  }
}

// grouped_pp.h (compiled in grouped_fast.hip): 256 x 256 tiles, sizes and addresses in
// multiples of 16 bytes.
template <int DIR, bool I8>
hipError_t launch_grouped_pp(const GroupedParams& p, long long tiles, hipStream_t stream);

// grouped_swiglu.hip: the same with an epilogue.
hipError_t launch_grouped_swiglu_pp(const GroupedParams& p, long long tiles, hipStream_t stream);
hipError_t launch_grouped_swiglu_grad_pp(const GroupedParams& p, long long tiles,
                                         hipStream_t stream);

// grouped_fp8.hip: the same for block-scaled e4m3, bf16 results, short sums.
hipError_t launch_grouped_fp8_pp(const GroupedParams& p, long long tiles, hipStream_t stream);

// The same operands on 128 x 128 tiles, fp32 sums of exact products.
hipError_t launch_grouped_fp8_mid(const GroupedParams& p, long long tiles, hipStream_t stream);

// grouped_few.hip: tiles of `rows` (16, 32 or 64) x 64 under the same condition.
template <int DIR, int TYPE, int EPI>
hipError_t launch_grouped_few(const GroupedParams& p, int rows, long long tiles,
                              hipStream_t stream);

// Where a partial sum of row i, column j goes (kGradWeights: row n of group e).
template <int DIR>
__device__ __forceinline__ size_t part_at(const GroupedParams& p, int split, int e, int i, int j) {
  const size_t rows = DIR == kGradWeights ? (size_t)p.E * p.N : (size_t)p.R;
  const size_t row = DIR == kGradWeights ? (size_t)e * p.N + i : (size_t)i;
  return ((size_t)split * rows + row) * columns<DIR>(p) + j;
}

}  // namespace eaas
