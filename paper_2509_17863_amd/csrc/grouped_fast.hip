// Grouped products whose sizes, strides and bases are multiples of 16 bytes, for
// groups of many rows (grouped.h states the products; grouped.hip has the kernels
// for everything else).
//
// A workgroup of eight waves computes 256 x 256 results; the sum advances by
// tiles of 128 bytes (64 bf16 or 128 8-bit values) of both operands, 32 KiB each,
// which go from memory to LDS without passing through registers.  The waves form
// two groups of four, one wave of each to a SIMD.  Group 0 holds result rows 0-127
// and loads operand A, group 1 rows 128-255 and operand B; a wave has 128 x 64
// results.  The groups walk the same tiles one phase apart: in an M phase a wave
// issues its share of the loads and reads the fragments of one tile into
// registers, in a C phase it issues their 32 MFMAs, so that each SIMD's matrix
// pipe is fed by one wave while the other reads:
//   group 0, phase 2t:   M(t): load A tile t+1 (t >= 1), fragments of tile t
//   group 0, phase 2t+1: C(t), then wait until A tile t+1 has landed
//   group 1, phase 2t+1: M(t): load B tile t+2, fragments of tile t, wait until B
//                        tile t+1 has landed
//   group 1, phase 2t+2: C(t)
// A has two LDS stages, B three; a stage is filled again only after both groups
// have read it.
//
// One workgroup stays on each CU and goes from tile to tile: the first two tiles of
// the sum of its next results are on their way before the results at hand are
// stored, and nothing waits for those stores before the third.  (A workgroup to a
// tile spent 4 us of 38 on starting and waited 8 for its stores to end, at 1024
// rows of the sum in dW.)  Row tiles come from a table that a small kernel makes
// from the groups' offsets.
//
// What bounds it: long sums the power limit (8192^3: 0.80 ms forward, 0.81 dx, 0.83
// dW, 1.37 PFLOP/s, at 1.44 GHz with the matrix pipes busy 83% of cycles; 8-bit
// integers 0.44 ms, 2.5 POP/s); short ones the 7 us a tile that are left of start,
// way out and stores (8 experts of 1024 rows, 4096 x 14336, dW fp32: 0.94 ms, 1.02
// PFLOP/s; 1.5 us for each 64 rows of the sum).
//
// An operand that lies along the sum is kept as 256 rows of 128 bytes; one that
// lies across it as 64 rows of 512 bytes, read with the transposing LDS load.  The
// loads are bounds-checked buffer loads: whatever lies past the sum's end or past
// the last row arrives as zeros.
#include <algorithm>

#include "grouped_fast.h"

namespace eaas {
namespace {

#define INLINE __attribute__((always_inline))

constexpr int kB = 256;               // result rows and columns of a tile
constexpr int kThreads = 512;
constexpr int kStage = 32768;         // bytes of one operand's tile
constexpr int kSA = 2, kSB = 3;       // stages of A and B
constexpr int kLds = (kSA + kSB) * kStage;
constexpr int kInst = 8;              // loads of one wave per tile of its operand

// The kernel's parameters, read again from where the launch put them.  (What only the
// step from tile to tile needs would otherwise be held in scalar registers through
// the main loop, which has none to spare.)
__device__ __forceinline__ GroupedParams fresh_params() {
  auto at = (const CONST_AS GroupedParams*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return *(const GroupedParams*)at;
}
// A scalar that the compiler takes for a new one here, so that what is computed
// from it is computed again instead of being held across the main loop.
__device__ __forceinline__ uint32_t opaque(uint32_t v) {
  v = __builtin_amdgcn_readfirstlane(v);
  asm volatile("" : "+s"(v));
  return v;
}

// A value that is the same in all lanes, kept as one (a quotient is not by itself).
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Row tiles of all groups, in order: rows[0][0] is their number, rows[1 + n] row
// tile n as (group, first row, rows of it that exist, 0).
__global__ __launch_bounds__(1024) void row_tiles_kernel(GroupedParams p) {
  __shared__ int s_before[kMaxExperts + 1];
  __shared__ int s_wave[16];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  int beg = 0, end = 0;
  if (tid < p.E) group_range(p, tid, beg, end);
  int incl = ceil_div(end - beg, kB);
  const int mine = incl;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int o = __shfl_up(incl, d, kWave);
    if (lane >= d) incl += o;
  }
  if (lane == kWave - 1) s_wave[wave] = incl;
  __syncthreads();
  for (int w = 0; w < wave; ++w) incl += s_wave[w];
  s_before[tid] = incl - mine;
  if (tid == 1023) s_before[1024] = incl;
  __syncthreads();
  // (offsets that do not ascend can name more tiles than the table holds)
  const int total = min(s_before[1024], p.R / kB + min(p.R, p.E));
  if (tid == 0) p.row_tiles[0] = i32x4{total, 0, 0, 0};
  for (int n = tid; n < total; n += 1024) {
    // the last group whose tiles start at or before n (groups without rows share
    // their successor's start and are passed over)
    int lo = 0, hi = p.E - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_before[mid] <= n) lo = mid; else hi = mid - 1;
    }
    group_range(p, lo, beg, end);
    const int r0 = beg + (n - s_before[lo]) * kB;
    p.row_tiles[1 + n] = i32x4{lo, r0, min(kB, end - r0), 0};
  }
}

// A wave's 128 x 64 results to memory through 4 KiB of LDS of its own, so that
// whole 128-byte segments of rows are stored: rows row0.. of the tile, columns
// col0.. of the result.  acc[i][j][v]: row i*32 + lane % 32, column j*32 + 8*(v/4) +
// 4*(lane/32) + v % 4.  `before_stores` runs once, ahead of the first store.  (A
// wave's own LDS accesses complete in order.)
template <int DIR, bool I8, class Acc, class F>
__device__ __forceinline__ void store_results(const GroupedParams& p, const GroupedTile& t, int row0,
                                              int col0, const Acc (&acc)[4][2], LDS_AS char* buf,
                                              F before_stores) {
  const int lane = __lane_id();
  const int lrow = lane & 31, khalf = lane >> 5;
  const int cols = columns<DIR>(p);
  if (row0 >= t.i_valid || col0 >= cols ||
      (DIR == kGradWeights && p.accumulate && t.end == t.beg)) {
    before_stores();
    return;
  }
  float rs[4];
  f32x4 cs[2][4];
  if constexpr (I8) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      rs[i] = p.row_scale[source_row(p, t.i0 + min(row0 + i * 32 + lrow, t.i_valid - 1))];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          cs[j][q][c] = p.col_scale[(size_t)t.e * p.N +
                                    min(col0 + j * 32 + 8 * q + 4 * khalf + c, p.N - 1)];
    // all of them here and now: a load left for later would be waited for in the
    // next results' main loop, together with the loads ahead of it
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(rs[i]));
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) asm volatile("" : "+v"(cs[j][q]));
  }
  auto quad = [&](int i, int j, int q) INLINE {
    f32x4 o;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const auto v = acc[i][j][4 * q + c];
      if constexpr (I8) o[c] = (float)v * rs[i] * cs[j][q][c];
      else o[c] = v;
    }
    return o;
  };
  const size_t row_base = DIR == kGradWeights ? (size_t)t.e * p.N + t.i0 : (size_t)t.i0;
  // whole 16-byte pieces everywhere in this wave's columns
  const bool whole = p.vec16 && !p.accumulate && col0 + 64 <= cols;
  const int m8 = lane >> 3, c8 = lane & 7;  // on the way out 8 lanes take a row of 128 bytes
  if (p.vec16 && !p.out_fp32) {
    // bf16: 64 columns are 128 bytes
    const int col = col0 + c8 * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 v = quad(i, j, q);
          *reinterpret_cast<LDS_AS u32x2*>(buf + lrow * 128 + (((j * 4 + q) ^ (lrow & 7)) << 4) +
                                           khalf * 8) =
              u32x2{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
        }
      if (whole) {
        u32x4 o[4];
#pragma unroll
        for (int s = 0; s < 4; ++s)
          o[s] = *reinterpret_cast<const LDS_AS u32x4*>(buf + (s * 8 + m8) * 128 +
                                                        ((c8 ^ m8) << 4));
        if (i == 0) before_stores();
        uint16_t* at = static_cast<uint16_t*>(p.out) + (row_base + row0 + i * 32 + m8) * p.ldo + col;
        // (results of large products are read after they have left the caches)
#pragma unroll
        for (int s = 0; s < 4; ++s)
          if (row0 + i * 32 + s * 8 + m8 < t.i_valid)
            __builtin_nontemporal_store(o[s], reinterpret_cast<u32x4*>(at + s * 8 * p.ldo));
      } else {
        if (i == 0) before_stores();
#pragma unroll 1
        for (int s = 0; s < 4; ++s) {
          const int ri = row0 + i * 32 + s * 8 + m8;
          const LDS_AS uint16_t* from =
              (const LDS_AS uint16_t*)(buf + (s * 8 + m8) * 128 + ((c8 ^ m8) << 4));
          uint16_t* at = static_cast<uint16_t*>(p.out) + (row_base + ri) * p.ldo + col;
          if (ri < t.i_valid)
#pragma unroll
            for (int c = 0; c < 8; ++c)
              if (col + c < cols) at[c] = from[c];
        }
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      // 32 x 32 results, 128 bytes to a row
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<LDS_AS f32x4*>(buf + lrow * 128 + (((2 * q + khalf) ^ (lrow & 7)) << 4)) =
            quad(i, j, q);
      const int col = col0 + j * 32 + c8 * 4;
      const LDS_AS char* from = buf + m8 * 128 + ((c8 ^ m8) << 4);
      if (whole) {
        f32x4 o[4];
#pragma unroll
        for (int s = 0; s < 4; ++s)
          o[s] = *reinterpret_cast<const LDS_AS f32x4*>(from + s * 1024);
        if (i == 0 && j == 0) before_stores();
        float* at = static_cast<float*>(p.out) + (row_base + row0 + i * 32 + m8) * p.ldo + col;
#pragma unroll
        for (int s = 0; s < 4; ++s)
          if (row0 + i * 32 + s * 8 + m8 < t.i_valid)
            __builtin_nontemporal_store(o[s], reinterpret_cast<f32x4*>(at + s * 8 * p.ldo));
      } else {
        if (i == 0 && j == 0) before_stores();
#pragma unroll 1
        for (int s = 0; s < 4; ++s) {
          const int ri = row0 + i * 32 + s * 8 + m8;
          const f32x4 v = *reinterpret_cast<const LDS_AS f32x4*>(from + s * 1024);
          if (ri < t.i_valid && col < cols) store4<DIR>(p, t.e, t.i0 + ri, col, v);
        }
      }
    }
}

// GATHER: rows of x come through perm.
template <int DIR, bool I8, bool GATHER>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void grouped_pp_kernel(GroupedParams p) {
  constexpr bool A_ACROSS = DIR == kGradWeights, B_ACROSS = DIR != kForward;
  constexpr int ESZ = I8 ? 1 : 2;
  constexpr int SUM = 128 / ESZ;
  constexpr int MBW = 4, NBW = 2, KK = 4;
  __shared__ __attribute__((aligned(1024))) char smem_raw[kLds];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int grp = wave >> 2, w4 = wave & 3;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)smem_raw);
  const int cols = columns<DIR>(p);
  const long long a_row = p.lda * ESZ, b_row = p.ldb * ESZ;  // bytes of a row

  // the tiles of results, and this workgroup's
  const int mt = DIR == kGradWeights ? ceil_div(p.N, kB)
                                     : ((const CONST_AS i32x4*)p.row_tiles)[0][0];
  const int nt = ceil_div(cols, kB);
  const int total = DIR == kGradWeights ? p.E * mt * nt : mt * nt;
  GroupedTile t;
  int sum_end = 0, nk = 0;  // of the sum: its length and its tiles

  // Loads of an operand by the four waves of its group, chunks of 16 bytes swapped
  // within the row as the fragment reads expect them:
  //   along:  instruction q of wave w moves rows (w + 4q)*8 .. +8 (lane l: row l/8,
  //           chunk l%8)
  //   across: instruction q of wave w moves sum rows w*16 + 2q .. +2 (lane l: row
  //           l/32, chunk l%32)
  const char* along_base = nullptr;   // along the sum: rows i or j
  // (of every instruction; in kGradRows, short of registers, of the first)
  constexpr int kOffs = DIR == kForward ? kInst : 1;
  uint32_t along_off[kOffs], along_bytes = 0;
  const char* across_base = nullptr;  // across it: columns from i0 or j0
  uint32_t across_off[2], across_bytes = 0;  // (bytes: gathered rows)
  // the chunk of the sum that this lane loads (along)
  const int my_chunk = (lane & 7) ^ swz_along(w4 * 8 + (lane >> 3));

  auto locate = [&](int id) INLINE {
    const GroupedParams p = fresh_params();
    const long long a_row = p.lda * ESZ, b_row = p.ldb * ESZ;
    id = xcd_window_remap(id, total);
    int tm, tn;
    if constexpr (DIR == kGradWeights) {
      t.e = uniform(id / (mt * nt));
      tile_of(id - t.e * mt * nt, mt, nt, tm, tn);
      tm = uniform(tm);
      t.beg = min(max(((const CONST_AS int32_t*)p.offsets)[t.e], 0), p.R);
      t.end = min(max(((const CONST_AS int32_t*)p.offsets)[t.e + 1], t.beg), p.R);
      t.i0 = tm * kB;
      t.i_valid = min(kB, p.N - t.i0);
      sum_end = t.end - t.beg;
    } else {
      tile_of(id, mt, nt, tm, tn);
      tm = uniform(tm);
      const i32x4 r = ((const CONST_AS i32x4*)p.row_tiles)[1 + tm];
      t.e = r[0];
      t.beg = t.end = 0;
      t.i0 = r[1];
      t.i_valid = r[2];
      sum_end = DIR == kForward ? p.K : p.N;
    }
    t.j0 = uniform(tn) * kB;
    nk = ceil_div(sum_end, SUM);
    const char* w = p.b + (DIR == kGradWeights ? 0 : (size_t)t.e * p.N * p.K * ESZ);
    if (grp == 0 ? !A_ACROSS : !B_ACROSS) {
      const int row0 = lane >> 3;
      if (grp == 0) {
        // (gathered: rows past the tile's repeat one that exists; their results are not stored)
        constexpr bool gather = DIR == kForward && GATHER;
        along_base = gather ? p.a : p.a + t.i0 * a_row;
        along_bytes = (uint32_t)(((gather ? p.R / p.k : t.i_valid) - 1) * a_row +
                                 (long long)sum_end * ESZ);
#pragma unroll
        for (int q = 0; q < kOffs; ++q) {
          const int row = (w4 + 4 * q) * 8 + row0;
          const int src = gather ? source_row(p, t.i0 + min(row, t.i_valid - 1)) : row;
          along_off[q] = (uint32_t)(src * a_row) + my_chunk * 16;
        }
      } else {
        along_base = w + t.j0 * b_row;
        along_bytes = (uint32_t)(min(kB, cols - t.j0) * b_row);
#pragma unroll
        for (int q = 0; q < kOffs; ++q)
          along_off[q] = (uint32_t)(((w4 + 4 * q) * 8 + row0) * b_row) + my_chunk * 16;
      }
    } else {
      const int h = lane >> 5;
      const long long row = grp == 0 ? a_row : b_row;
      // rows w4*16 + 2q + h; q even and odd differ in the chunks' order
#pragma unroll
      for (int odd = 0; odd < 2; ++odd) {
        const int r = 2 * odd + h;
        across_off[odd] = (uint32_t)((grp == 0 ? t.i0 : t.j0) * ESZ +
                                     ((lane & 31) ^ swz_across(r)) * 16);
        if (!(DIR == kGradWeights && GATHER && grp == 1))
          across_off[odd] += (uint32_t)((w4 * 16 + r) * row);
      }
      if (DIR == kGradWeights && GATHER && grp == 1)
        across_bytes = (uint32_t)((p.R / p.k - 1) * row + (long long)cols * ESZ);
      if (grp == 0) across_base = p.a + t.beg * row;
      else if (DIR == kGradRows) across_base = w;
      else across_base = GATHER ? p.b : p.b + t.beg * row;
    }
  };

  auto issue_along = [&](int kt, uint32_t lds, long long row) INLINE {
    lds = opaque(lds);
    const uint32_t step = opaque((uint32_t)row * 32);
    const i32x4 d = descriptor(along_base + (size_t)kt * 128, along_bytes - (uint32_t)kt * 128);
    const bool in = kt * 8 + my_chunk < ceil_div(sum_end * ESZ, 16);
#pragma unroll
    for (int q = 0; q < kInst; ++q)
      load_lds16(d, in ? along_off[q % kOffs] + (kOffs == 1 ? q * step : 0) : kNowhere,
                 lds + (w4 + 4 * q) * 1024);
  };
  auto issue_across = [&](int kt, uint32_t lds, long long row_bytes, int width) INLINE {
    lds = opaque(lds);
    const long long row = opaque((uint32_t)row_bytes);
    const int left = min(64, sum_end - kt * 64);
    const i32x4 d = descriptor(across_base + (long long)kt * 64 * row,
                               (uint32_t)((left - 1) * row + (long long)width * ESZ));
#pragma unroll
    for (int q = 0; q < kInst; ++q)
      load_lds16(d, across_off[q & 1] + (uint32_t)((q & ~1) * 2 * row),
                 lds + (w4 * 16 + 2 * q) * 512);
  };
  // Gathered rows of x: their slots come through the scalar cache (a vector load
  // here would make the compiler wait for the loads it does not know about), one
  // tile before they are used.
  int slots[2 * kInst];
  auto fetch_slots = [&](int kt) INLINE {
    const CONST_AS int32_t* perm = (const CONST_AS int32_t*)p.perm;
    const int s0 = t.beg + kt * 64 + w4 * 16;
    if (s0 + 2 * kInst <= p.R) {
#pragma unroll
      for (int i = 0; i < 2 * kInst; ++i) slots[i] = perm[s0 + i];
    } else {
#pragma unroll
      for (int i = 0; i < 2 * kInst; ++i) slots[i] = perm[min(s0 + i, p.R - 1)];
    }
  };
  auto issue_gathered = [&](int kt, uint32_t lds) INLINE {
    lds = opaque(lds);
    const uint32_t b_row = opaque((uint32_t)p.ldb * ESZ);
    const int left = sum_end - kt * 64 - w4 * 16;
    const i32x4 d = descriptor(
        across_base, across_bytes);
    // lane i works out row i of the sixteen
    int slot = 0;
#pragma unroll
    for (int i = 0; i < 2 * kInst; ++i)
      asm("v_writelane_b32 %0, %1, %2" : "+v"(slot) : "s"(slots[i]), "n"(i));
    const int at = lane < left ? (int)((uint32_t)token_of(p, slot) * b_row) : (int)kNowhere;
#pragma unroll
    for (int q = 0; q < kInst; ++q) {
      const uint32_t even = __builtin_amdgcn_readlane(at, 2 * q);
      const uint32_t odd = __builtin_amdgcn_readlane(at, 2 * q + 1);
      const uint32_t base = lane < 32 ? even : odd;
      load_lds16(d, base == kNowhere ? kNowhere : base + across_off[q & 1],
                 lds + (w4 * 16 + 2 * q) * 512);
    }
    if (kt + 1 < nk) fetch_slots(kt + 1);
  };
  auto issue = [&](int kt) INLINE {
    if (grp == 0) {
      const uint32_t dst = lds0 + (kt % kSA) * kStage;
      if constexpr (A_ACROSS) issue_across(kt, dst, a_row, p.N);
      else issue_along(kt, dst, a_row);
    } else {
      const uint32_t dst = lds0 + (kSA + kt % kSB) * kStage;
      if constexpr (!B_ACROSS) issue_along(kt, dst, b_row);
      else if constexpr (DIR == kGradWeights && GATHER) issue_gathered(kt, dst);
      else issue_across(kt, dst, b_row, cols);
    }
  };

  // fragment addresses: lane l holds row or column l % 32 of a block and 16 bytes
  // of the sum, half l / 32 of the k-step.  One address for each operand: blocks and
  // k-steps differ from it by a constant or in address bits that the order of
  // chunks exchanges (and are derived from it anew for every tile, which spares the
  // registers that holding them would take).
  auto first_fragment = [&](bool across, int c0) {
    if (across) {
      const int tg = lane >> 4, ti = lane & 15;  // transposing load: group of 16, lane in it
      const int row = (tg >> 1) * 8 + (ti >> 2);
      const int chunk = (c0 >> 3) + (tg & 1) * 2 + ((ti & 3) >> 1);
      return row * 512 + ((chunk ^ swz_across(ti >> 2)) << 4) + (ti & 1) * 8;
    }
    const int row = c0 + (lane & 31);
    return row * 128 + (((lane >> 5) ^ swz_along(row)) << 4);
  };
  const int a_at = first_fragment(A_ACROSS, grp * 128), b_at = first_fragment(B_ACROSS, w4 * 64);
  typedef typename std::conditional<I8, i32x16, f32x16>::type Acc;
  Acc acc[MBW][NBW];
  const LDS_AS char* smem = (const LDS_AS char*)smem_raw;

  struct Frags {
    u32x4 a[KK][MBW], b[KK][NBW];
  };
  auto fragment = [&](auto across, const LDS_AS char* stage, int at, int block, int kk) INLINE {
    if constexpr (decltype(across)::value) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      const LDS_AS char* src = stage + (at ^ (block << 6)) + kk * 8192;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                     (LDS_AS s16x4*)(src)));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                     (LDS_AS s16x4*)(src + 2048)));
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      return *reinterpret_cast<const LDS_AS u32x4*>(stage + (at ^ (kk << 5)) + block * 4096);
    }
  };
  // mb: row blocks of this wave that hold rows of the result
  auto load_frags = [&](auto mb, int kt, Frags& f) INLINE {
    const LDS_AS char* sa = smem + (kt % kSA) * kStage;
    const LDS_AS char* sb = smem + (kSA + kt % kSB) * kStage;
    int a0 = a_at, b0 = b_at;
    asm volatile("" : "+v"(a0), "+v"(b0));
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
#pragma unroll
      for (int j = 0; j < NBW; ++j)
        f.b[kk][j] = fragment(std::integral_constant<bool, B_ACROSS>{}, sb, b0, j, kk);
#pragma unroll
      for (int i = 0; i < decltype(mb)::value; ++i)
        f.a[kk][i] = fragment(std::integral_constant<bool, A_ACROSS>{}, sa, a0, i, kk);
    }
    // the stage may be filled again right after the next barrier
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  auto mfmas = [&](auto mb, const Frags& f) INLINE {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int i = 0; i < decltype(mb)::value; ++i)
#pragma unroll
        for (int j = 0; j < NBW; ++j) {
          if constexpr (I8)
            acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(
                __builtin_bit_cast(i32x4, f.b[kk][j]), __builtin_bit_cast(i32x4, f.a[kk][i]),
                acc[i][j], 0, 0, 0);
          else
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                __builtin_bit_cast(bf16x8, f.b[kk][j]), __builtin_bit_cast(bf16x8, f.a[kk][i]),
                acc[i][j], 0, 0, 0);
        }
    __builtin_amdgcn_s_setprio(0);
  };
  auto phase_end = [&]() INLINE {
    __builtin_amdgcn_sched_barrier(0);
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };


  // the first two tiles of the sum, of both operands
  auto start = [&]() INLINE {
    if (nk == 0) return;
    if (DIR == kGradWeights && GATHER && grp == 1) fetch_slots(0);
    issue(0);
    if (nk > 1) issue(1);
  };
  // The sum of one tile of results.  Both groups pass 2*nk barriers: group 1 idles in
  // the first phase, and group 0 goes on to the next results while group 1 has its
  // last MFMAs to issue.  Tiles 0 and 1 have landed: the waits start with tile 2.
  auto walk = [&](auto mb) INLINE {
    constexpr bool LIVE = decltype(mb)::value > 0;
    if (grp == 0) {
#pragma unroll 1
      for (int kt = 0; kt < nk; ++kt) {
        if (kt >= 1 && kt + 1 < nk) issue(kt + 1);
        Frags f;
        if constexpr (LIVE) load_frags(mb, kt, f);
        phase_end();
        if constexpr (LIVE) mfmas(mb, f);
        if (kt >= 1) wait_vmcnt<0>();
        phase_end();
      }
    } else {
      phase_end();
#pragma unroll 1
      for (int kt = 0; kt < nk; ++kt) {
        if (kt + 2 < nk) issue(kt + 2);
        Frags f;
        if constexpr (LIVE) load_frags(mb, kt, f);
        if (kt >= 1) {
          if (kt + 2 < nk) wait_vmcnt<kInst>();
          else wait_vmcnt<0>();
        }
        phase_end();
        if constexpr (LIVE) mfmas(mb, f);
        if (kt + 1 < nk) phase_end();
      }
    }
  };
  int id = blockIdx.x;
  if (id >= total) return;
  locate(id);
  start();
  wait_vmcnt<0>();
  for (;;) {
#pragma unroll
    for (int i = 0; i < MBW; ++i)
#pragma unroll
      for (int j = 0; j < NBW; ++j) acc[i][j] = Acc{};
    if (nk > 0) {
      // The stores' passes through B's third stage end here: a wave whose rows do not
      // all exist need not have waited for its last ones, and group 1 loads into that
      // stage two barriers from here.
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      phase_end();
      // a wave multiplies the row blocks that exist (rounded up to 0, 2 or 4), and
      // loads its share for the others in any case
      const int rows = t.j0 + w4 * 64 < cols ? t.i_valid - grp * 128 : 0;
      if (rows > 64) walk(std::integral_constant<int, 4>{});
      else if (rows > 0) walk(std::integral_constant<int, 2>{});
      else walk(std::integral_constant<int, 0>{});
    }
    // The next results' operands go ahead of the stores (the last barrier is behind
    // every wave's fragment reads; the stores pass through B's third stage), and
    // have landed when the stores start, so that no wait for them meets a store.
    const GroupedTile done = t;
    id += gridDim.x;
    const bool more = id < total;
    if (more) {
      locate(id);
      start();
    }
    store_results<DIR, I8>(fresh_params(), done, grp * 128, done.j0 + w4 * 64, acc,
                           (LDS_AS char*)smem_raw + 4 * kStage + wave * 4096,
                           [&]() { wait_vmcnt<0>(); });
    if (!more) break;
  }
}

}  // namespace

template <int DIR, bool I8>
hipError_t launch_grouped_pp(const GroupedParams& p, long long tiles, hipStream_t stream) {
  if (tiles > 0x7fffffffLL || p.splits != 1) return hipErrorInvalidValue;
  if (DIR != kGradWeights) {
    hipLaunchKernelGGL(row_tiles_kernel, dim3(1), dim3(1024), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // one workgroup to a CU
  const dim3 grid((unsigned)std::min<long long>(tiles, 256)), block(kThreads);
  if (DIR != kGradRows && p.perm)
    hipLaunchKernelGGL((grouped_pp_kernel<DIR, I8, DIR != kGradRows>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((grouped_pp_kernel<DIR, I8, false>), grid, block, 0, stream, p);
  return hipGetLastError();
}

template hipError_t launch_grouped_pp<kForward, false>(const GroupedParams&, long long, hipStream_t);
template hipError_t launch_grouped_pp<kForward, true>(const GroupedParams&, long long, hipStream_t);
template hipError_t launch_grouped_pp<kGradRows, false>(const GroupedParams&, long long, hipStream_t);
template hipError_t launch_grouped_pp<kGradWeights, false>(const GroupedParams&, long long, hipStream_t);

}  // namespace eaas
