// Parts shared by the grouped product kernels: loads straight into LDS, the order
// of chunks there, and the way out of the results.
#pragma once

#include <type_traits>

#include "grouped.h"

namespace eaas {

// One wave-wide load of 16 bytes a lane from memory into LDS: lane l reads at
// rsrc.base + voff(l), or zeros if that is past the descriptor's size, and the
// bytes land at lds + 16 * l.  Inline assembly, so that the compiler adds no waits
// of its own; completion is counted with vmcnt.
__device__ __forceinline__ void load_lds16(const i32x4& rsrc, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :: "v"(voff), "s"(rsrc), "s"(lds) : "memory");
}

// Raw buffer descriptor of `bytes` bytes from `base` (both wave-uniform).
__device__ __forceinline__ i32x4 descriptor(const char* base, uint32_t bytes) {
  const uint64_t v = reinterpret_cast<uint64_t>(base);
  i32x4 d;
  d[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)v);
  d[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32) & 0xffff);
  d[2] = __builtin_amdgcn_readfirstlane((int)bytes);
  d[3] = 0x00020000;
  return d;
}

// An offset past every descriptor's end: the arrays that a descriptor covers here
// end below it, so offset and size together never wrap.
constexpr uint32_t kNowhere = 0x80000000u;

__device__ __forceinline__ int swz_along(int row) { return (row & 7) ^ ((row >> 3) & 1); }
// The transposing load's 16 lanes take 4 rows x 32 bytes, its 32 lanes 4 rows x 64
// bytes: the four rows' chunks go to distinct banks in both views (32 banks or 64).
__device__ __forceinline__ int swz_across(int row) {
  return ((row & 1) << 2) | (((row >> 1) & 1) * 10);
}

// A wave's results, MBW x 2 blocks of 32 x 32, to memory: rows row0.. of the tile,
// columns col0.. of the result.  They pass through `buf`, kWayOutBytes of LDS that
// this wave alone uses, 32 rows x 64 columns at a time, so that whole row segments
// are stored.  acc[i][j][v]: row i*32 + lane % 32, column
// j*32 + 8*(v/4) + 4*(lane/32) + v % 4.  (A wave's own LDS accesses complete in
// order.)
constexpr int kWayOutLd = 68;  // floats: a pad of 16 bytes against bank conflicts
constexpr int kWayOutBytes = 32 * kWayOutLd * 4;

template <int DIR, bool I8, int MBW, class Acc>
__device__ __forceinline__ void way_out(const GroupedParams& p, const GroupedTile& t, int split,
                                        int row0, int col0, const Acc (&acc)[MBW][2],
                                        LDS_AS float* buf) {
  constexpr int LD = kWayOutLd;
  const int lane = __lane_id();
  const int lrow = lane & 31, khalf = lane >> 5;
  const int cols = columns<DIR>(p);
  if (col0 >= cols) return;
  if (DIR == kGradWeights && p.accumulate && p.splits == 1 && t.end == t.beg) return;  // + 0
  // how rows are stored: as bf16 or fp32, 16 bytes a lane, or an element a lane
  // where the result's rows are not in multiples of 16 bytes
  const bool loose = p.splits == 1 ? !p.vec16 : cols % 4 != 0;
  const bool narrow = !loose && p.splits == 1 && !p.out_fp32;
  const int cl = loose ? lane : narrow ? (lane & 7) * 8 : (lane & 15) * 4, col = col0 + cl;
  // 8-bit integers: rows are scaled on the way into LDS, columns on the way out
  const bool scale = I8 && p.splits == 1;
  float rs[MBW], cs[8];
  if (scale) {
#pragma unroll
    for (int i = 0; i < MBW; ++i)
      rs[i] = p.row_scale[source_row(p, t.i0 + min(row0 + i * 32 + lrow, t.i_valid - 1))];
#pragma unroll
    for (int c = 0; c < 8; ++c)
      cs[c] = p.col_scale[(size_t)t.e * p.N + min(col + c, p.N - 1)];
  }
  auto stage = [&](int i) {
    LDS_AS float* at = buf + lrow * LD + 4 * khalf;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 o;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const auto v = acc[i][j][4 * q + c];
          if constexpr (I8) o[c] = scale ? (float)v * rs[i] : __int_as_float(v);
          else o[c] = v;
        }
        *reinterpret_cast<LDS_AS f32x4*>(at + j * 32 + 8 * q) = o;
      }
  };
#pragma unroll
  for (int i = 0; i < MBW; ++i) {
    stage(i);
    const LDS_AS float* from = buf + cl;
    if (narrow) {
      // 8 lanes to a row of 64 results
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int m = s * 8 + (lane >> 3);
        const int ri = row0 + i * 32 + m, row = t.i0 + ri;
        f32x4 lo = *reinterpret_cast<const LDS_AS f32x4*>(from + m * LD);
        f32x4 hi = *reinterpret_cast<const LDS_AS f32x4*>(from + m * LD + 4);
        if (ri >= t.i_valid || col >= cols) continue;
        if constexpr (I8) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            lo[c] *= cs[c];
            hi[c] *= cs[4 + c];
          }
        }
        if (col + 8 <= cols) {
          u32x4 o;
          o[0] = to_bf16x2(lo[0], lo[1]);
          o[1] = to_bf16x2(lo[2], lo[3]);
          o[2] = to_bf16x2(hi[0], hi[1]);
          o[3] = to_bf16x2(hi[2], hi[3]);
          const size_t at = (DIR == kGradWeights ? (size_t)t.e * p.N + row : (size_t)row) * p.ldo;
          // (results of large products are read after they have left the caches)
          __builtin_nontemporal_store(
              o, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.out) + at + col));
        } else {
          store4<DIR>(p, t.e, row, col, lo);
          if (col + 4 < cols) store4<DIR>(p, t.e, row, col + 4, hi);
        }
      }
    } else if (loose) {
      // 64 lanes to a row; rows that exist are a prefix
      const int live = min(32, t.i_valid - (row0 + i * 32));
      const int row = t.i0 + row0 + i * 32;
      if (col < cols && live > 0) {
        auto rows = [&](auto* out, size_t ld, auto convert) {
#pragma unroll 1
          for (int m0 = 0; m0 < live; m0 += 8) {
            float v[8];
#pragma unroll
            for (int m = 0; m < 8; ++m) v[m] = from[(m0 + m) * LD];
#pragma unroll
            for (int m = 0; m < 8; ++m)
              if (m0 + m < live) convert(out + (m0 + m) * ld, v[m]);
          }
        };
        if (p.splits > 1) {
          rows(static_cast<float*>(p.part) + part_at<DIR>(p, split, t.e, row, col), cols,
               [](float* o, float v) { *o = v; });
        } else {
          const size_t at =
              (DIR == kGradWeights ? (size_t)t.e * p.N + row : (size_t)row) * p.ldo + col;
          const float c = I8 ? cs[0] : 1.0f;
          if (!p.out_fp32)
            rows(static_cast<uint16_t*>(p.out) + at, p.ldo,
                 [c](uint16_t* o, float v) { *o = (uint16_t)to_bf16x2(I8 ? v * c : v, 0.0f); });
          else if (p.accumulate)
            rows(static_cast<float*>(p.out) + at, p.ldo, [](float* o, float v) { *o += v; });
          else
            rows(static_cast<float*>(p.out) + at, p.ldo,
                 [c](float* o, float v) { *o = I8 ? v * c : v; });
        }
      }
    } else {
      // 16 lanes to a row
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const int m = s * 4 + (lane >> 4);
        const int ri = row0 + i * 32 + m, row = t.i0 + ri;
        f32x4 v = *reinterpret_cast<const LDS_AS f32x4*>(from + m * LD);
        if (ri >= t.i_valid || col >= cols) continue;
        if (p.splits > 1) {
          *reinterpret_cast<f32x4*>(static_cast<float*>(p.part) +
                                    part_at<DIR>(p, split, t.e, row, col)) = v;
          continue;
        }
        if constexpr (I8) {
#pragma unroll
          for (int c = 0; c < 4; ++c) v[c] *= cs[c];
        }
        if (col + 4 <= cols && !p.accumulate) {
          const size_t at = (DIR == kGradWeights ? (size_t)t.e * p.N + row : (size_t)row) * p.ldo;
          __builtin_nontemporal_store(
              v, reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at + col));
        } else {
          store4<DIR>(p, t.e, row, col, v);
        }
      }
    }
  }
}

}  // namespace eaas
