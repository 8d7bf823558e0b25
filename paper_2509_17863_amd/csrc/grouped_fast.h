// Parts shared by the grouped product kernels: loads straight into LDS, the order
// of chunks there, fragments, and the way out of the results.
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

// The same with 4 bytes a lane, landing at lds + 4 * l.
__device__ __forceinline__ void load_lds4(const i32x4& rsrc, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds"
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

// The sums over a block of 128 e4m3 elements for 64 rows from a0 and 64 columns from b0:
// codes go to bf16, which holds them exactly, products of those are exact in fp32 and are
// summed there.  (The 8-bit floating matrix instructions keep less: see grouped_fp8.hip.)
// A lane's 16 codes make two steps of the sum, whose order both operands share.
__device__ __forceinline__ void fp8_block(const LDS_AS char* sa, int a0, const LDS_AS char* sb,
                                          int b0, f32x16 (&part)[2][2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) part[i][j] = f32x16{};
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    u32x4 a[2], b[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      a[i] = fragment<false>(sa, a0 + 32 * i, kk);
      b[i] = fragment<false>(sb, b0 + 32 * i, kk);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x8 fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[i] = fp8x8_to_bf16(u32x2{a[i][2 * h], a[i][2 * h + 1]});
        fb[i] = fp8x8_to_bf16(u32x2{b[i][2 * h], b[i][2 * h + 1]});
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          part[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j], fa[i], part[i][j], 0, 0, 0);
    }
  }
}

// kFp8: the sums of a block go to the accumulators times the scales of their row and columns,
// whose product is taken first.  Where that lies past fp32's largest number or below its
// normal range, the result need not (sums of a block reach 2^25, and down to 2^-18): such rows
// take zero for the product, and, if a wave has any, their sums are added behind the others',
// multiplied by the larger scale first, which stays in range wherever the result does.
// (Scales that are zero or no number give the same either way.  A branch for each block of
// results instead keeps their sums from going beside the next ones' instructions: 12% of the
// 128 x 128 tiles' time.)
__device__ __forceinline__ bool out_of_range(float rs, float cs) {
  constexpr int kNormalOrNaN = 0x10b;  // v_cmp_class
  return !__builtin_amdgcn_classf(rs * cs, kNormalOrNaN) && rs != 0.0f && cs != 0.0f;
}
__device__ __forceinline__ float scale_of(float rs, float cs, bool& far) {
  const bool out = out_of_range(rs, cs);
  far |= out;
  return out ? 0.0f : rs * cs;
}
__device__ __forceinline__ float add_far(float sum, float rs, float cs, float acc) {
  const bool row_first = fabsf(rs) > fabsf(cs);
  const float out = fmaf(sum * (row_first ? rs : cs), row_first ? cs : rs, acc);
  return out_of_range(rs, cs) ? out : acc;
}

// A wave's results, MBW x 2 blocks of 32 x 32, to memory: rows row0.. of the tile,
// columns col0.. of the result.  They pass through `buf`, kWayOutBytes of LDS that
// this wave alone uses, 32 rows x 64 columns at a time, so that whole row segments
// are stored.  acc[i][j][v]: row i*32 + lane % 32, column
// j*32 + 8*(v/4) + 4*(lane/32) + v % 4.  (A wave's own LDS accesses complete in
// order.)
constexpr int kWayOutLd = 68;  // floats: a pad of 16 bytes against bank conflicts
constexpr int kWayOutBytes = 32 * kWayOutLd * 4;

template <int DIR, int TYPE, int MBW, class Acc>
__device__ __forceinline__ void way_out(const GroupedParams& p, const GroupedTile& t, int split,
                                        int row0, int col0, const Acc (&acc)[MBW][2],
                                        LDS_AS float* buf) {
  constexpr int LD = kWayOutLd;
  constexpr bool I8 = TYPE == kInt8;
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

// The same for a product with an epilogue.  kSwiglu: block 0 of a wave holds gate and
// block 1 up of the 32 columns from col0; kSwigluGrad: 64 columns of dh.  Parts of a split
// sum are stored as they come, those of kSwiglu at their columns of the matrix.
template <int DIR, int EPI, int MBW>
__device__ __forceinline__ void way_out_swiglu(const GroupedParams& p, const GroupedTile& t,
                                               int split, int row0, int col0,
                                               const f32x16 (&acc)[MBW][2], LDS_AS float* buf) {
  constexpr int LD = kWayOutLd;
  const int lane = __lane_id();
  const int lrow = lane & 31, khalf = lane >> 5;
  const int cols = columns<DIR, EPI>(p);
  if (col0 >= cols) return;
  // a lane takes eight columns: four or eight lanes to a row
  constexpr int PER = EPI == kSwiglu ? 4 : 8, ROWS = kWave / PER;
  const int c = (lane & (PER - 1)) * 8, n = cols - (col0 + c);
#pragma unroll
  for (int i = 0; i < MBW; ++i) {
    GateUp gate_up[32 / ROWS];
    if constexpr (EPI == kSwigluGrad) {
      if (p.splits == 1) {
#pragma unroll
        for (int s = 0; s < 32 / ROWS; ++s) {
          const int ri = row0 + i * 32 + s * ROWS + lane / PER;
          gate_up[s] = load_gate_up(p, t.i0 + ri, col0 + c, ri < t.i_valid ? n : 0);
        }
      }
    }
    LDS_AS float* at = buf + lrow * LD + 4 * khalf;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<LDS_AS f32x4*>(at + j * 32 + 8 * q) =
            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2],
                  acc[i][j][4 * q + 3]};
#pragma unroll
    for (int s = 0; s < 32 / ROWS; ++s) {
      const int m = s * ROWS + lane / PER, ri = row0 + i * 32 + m;
      float a[8], b[8];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f32x4 x = *reinterpret_cast<const LDS_AS f32x4*>(buf + m * LD + c + 4 * q);
        const f32x4 y = *reinterpret_cast<const LDS_AS f32x4*>(
            buf + m * LD + (EPI == kSwiglu ? 32 : 0) + c + 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a[4 * q + e] = x[e];
          b[4 * q + e] = y[e];
        }
      }
      if (ri >= t.i_valid || n <= 0) continue;
      const int row = t.i0 + ri;
      if (p.splits > 1) {
        const int wide = columns<DIR>(p);
        float* o = static_cast<float*>(p.part) + ((size_t)split * p.R + row) * wide + col0 + c;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < n) {
            o[e] = a[e];
            if constexpr (EPI == kSwiglu) o[cols + e] = b[e];
          }
      } else if constexpr (EPI == kSwiglu) {
        store_swiglu(p, row, col0 + c, n, a, b);
      } else {
        store_swiglu_grad(p, row, col0 + c, n, gate_up[s], a, false);
      }
    }
  }
}

}  // namespace eaas
