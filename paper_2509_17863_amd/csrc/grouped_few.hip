// Grouped products (forward and gradient in the rows) for groups of a few rows,
// with sizes and addresses in multiples of 16 bytes (grouped.h states the
// products).
//
// Such a product is bound by reading the weights once.  A workgroup of four waves
// computes 16 * MB rows x 64 columns; the waves share out the sum, a quarter each,
// and add their results in LDS at the end.  Until then a wave works alone, without
// barriers: it loads tiles of 128 bytes of the sum (64 bf16, 128 8-bit values) of
// its 64 weight rows (kGradRows: 64 rows of the sum x 64 columns) and of the rows,
// 8 + 2 * MB KiB, straight into its own two LDS stages, whole 128-byte lines at a
// time, and refills a stage as soon as it has read it.  (Two stages and two workgroups
// to a CU for 16 rows; three stages for 32 and two for 64, one workgroup: 96 to 150
// KiB in flight on a CU, several times what the memory's latency asks for.)
//
// kSwiglu: the 64 weight rows are 32 gate rows and the up rows of the same columns.  kFp8:
// a tile of the sum is one block of scales; the rows' scales travel in the stage, and codes
// go to bf16 as they are read (as in grouped_fast.h, fp8_block), which memory leaves time for.
//
// Measured, reading the weights once:
//   bf16, 4 rows of each of 128 experts, 2048 x 768: forward 76 us (5.3 TB/s), dx 71 (5.6),
//   the gated product's way back 73 (5.5); gated, 32 rows of 8 experts, 28672 x 4096: 300 (6.3)
//   8-bit integers, one token on 8 experts, 4096 x 7168: 37 us (6.4); 8 tokens on 128 experts,
//   1536 x 2048: 50 (6.3)
//   e4m3, the same two: 37 to 39 us (6.0 to 6.3), 29 to 30 (5.0)
#include "grouped_fast.h"

namespace eaas {
namespace {

constexpr int kJ = 64;             // columns of a tile
constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kWBytes = kJ * 128;  // weights of a stage

// Order of the eight 16-byte chunks of a 128-byte row of the sum's index, for the
// transposing load (16 lanes: 4 rows x 32 bytes).
__device__ __forceinline__ int swz_sum(int row) { return (((row & 3) ^ ((row >> 3) & 1)) << 1); }

template <int DIR, int TYPE, int EPI, int MB, int STAGES>
__global__ __launch_bounds__(kThreads) void grouped_few_kernel(GroupedParams p) {
  constexpr bool B_ACROSS = DIR == kGradRows;
  constexpr bool I8 = TYPE == kInt8, FP8 = TYPE == kFp8;
  constexpr int ESZ = TYPE == kBf16 ? 2 : 1, SUM = 128 / ESZ;
  constexpr int BI = 16 * MB, NB = kJ / 16;
  constexpr int kOutJ = EPI == kSwiglu ? kJ / 2 : kJ;  // columns of a result tile
  // kFp8: the rows' scales travel in the stage, or, where they would keep a second workgroup
  // off the CU, in a register: four tiles' at a time, one for each quarter of the wave
  constexpr bool S_STAGE = FP8 && MB > 1, S_REG = FP8 && MB == 1;
  constexpr int kXBytes = BI * 128, kSBytes = S_STAGE ? 256 : 0, kStage = kWBytes + kXBytes + kSBytes;
  constexpr int W_INST = kWBytes / 1024, X_INST = kXBytes / 1024;
  constexpr int INST = W_INST + X_INST + (S_STAGE ? 1 : 0);
  constexpr int LD = kJ + 4;
  constexpr int kRing = kWaves * STAGES * kStage, kParts = kWaves * BI * LD * 4;
  __shared__ __attribute__((aligned(1024))) char smem_raw[kRing > kParts ? kRing : kParts];
  GroupedTile t;
  if (!find_tile<DIR, BI, kOutJ, kThreads, EPI>(p, reinterpret_cast<int*>(smem_raw), t)) return;

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const uint32_t lds0 =
      __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)smem_raw) + wave * STAGES * kStage;
  const int cols = columns<DIR, EPI>(p);
  const int sum_end = DIR == kForward ? p.K : p.N;
  const int tiles = ceil_div(sum_end, SUM);
  const int parts = p.splits * kWaves, part = blockIdx.y * kWaves + wave;
  const int first = (int)((long long)tiles * part / parts);
  const int nk = (int)((long long)tiles * (part + 1) / parts) - first;
  const char* w = p.b + (size_t)t.e * p.N * p.K * ESZ;
  const long long a_row = p.lda * ESZ, b_row = p.ldb * ESZ;

  // loads: instruction q moves rows 8q .. 8q + 7 (lane l: row l/8, chunk l%8)
  const int r8 = lane >> 3, c8 = lane & 7;
  const bool gather = DIR == kForward && p.perm;
  const char* x_base = gather ? p.a : p.a + t.i0 * a_row;
  const uint32_t x_bytes =
      (uint32_t)(((gather ? p.R / p.k : t.i_valid) - 1) * a_row + (long long)sum_end * ESZ);
  uint32_t x_off[X_INST];
#pragma unroll
  for (int q = 0; q < X_INST; ++q) {
    const int row = min(8 * q + r8, t.i_valid - 1);
    const int src = gather ? source_row(p, t.i0 + row) : row;
    x_off[q] = (uint32_t)(src * a_row) + ((c8 ^ swz_along(8 * q + r8)) * 16);
  }
  uint32_t w_off[2];  // q even and odd differ in the chunks' order
#pragma unroll
  for (int odd = 0; odd < 2; ++odd) {
    const int row = 8 * odd + r8;
    w_off[odd] = (uint32_t)(row * b_row) +
                 (B_ACROSS ? t.j0 * ESZ + ((c8 ^ swz_sum(row)) * 16) : (c8 ^ swz_along(row)) * 16);
  }
  const char* w_base = B_ACROSS ? w : w + t.j0 * b_row;
  const uint32_t w_bytes = (uint32_t)(min(kOutJ, cols - t.j0) * b_row);
  const int chunks = ceil_div(sum_end * ESZ, 16);  // of the sum

  // kFp8: a lane's row of x has its scales there, and the columns, which lie in one block
  // of 128, have theirs at col_scale
  const int kb = FP8 ? ceil_div(p.K, 128) : 0;
  const char* s_base = nullptr;
  uint32_t s_bytes = 0, s_off = 0;
  const CONST_AS float* col_scale = nullptr;
  const float* row_scale = nullptr;
  if constexpr (S_REG) {
    const int row = min(lane & 15, t.i_valid - 1);
    row_scale = p.row_scale + (size_t)source_row(p, t.i0 + row) * kb;
  }
  if constexpr (S_STAGE) {
    const int row = min(lane, t.i_valid - 1);
    s_base = reinterpret_cast<const char*>(p.row_scale + (gather ? 0 : (size_t)t.i0 * kb));
    s_bytes = (uint32_t)((gather ? p.R / p.k : t.i_valid) * 4LL * kb);
    s_off = (uint32_t)((gather ? source_row(p, t.i0 + row) : row) * 4LL * kb);
  }
  if constexpr (FP8) {
    col_scale = (const CONST_AS float*)(p.col_scale +
                                        ((size_t)t.e * ceil_div(p.N, 128) + t.j0 / 128) * kb);
  }
  auto issue = [&](int kt) {
    const int at = first + kt;
    const uint32_t dst = lds0 + (kt % STAGES) * kStage;
    // the chunk of the sum that this lane loads (swz_along: q's parity matters)
    const bool even = at * 8 + (c8 ^ swz_along(r8)) < chunks;
    const bool odd = at * 8 + (c8 ^ swz_along(8 + r8)) < chunks;
    if constexpr (B_ACROSS) {
      const int left = min(64, sum_end - at * 64);
      const i32x4 d = descriptor(w_base + (long long)at * 64 * b_row,
                                 (uint32_t)((left - 1) * b_row + (long long)cols * ESZ));
#pragma unroll
      for (int q = 0; q < W_INST; ++q)
        load_lds16(d, w_off[q & 1] + (uint32_t)((q & ~1) * 8 * b_row), dst + q * 1024);
    } else {
      const char* from = w_base + (size_t)at * 128;
      const uint32_t bytes = w_bytes - (uint32_t)at * 128;
      // (kSwiglu: gate rows, then up rows)
      constexpr int HALF = EPI == kSwiglu ? W_INST / 2 : W_INST;
#pragma unroll
      for (int first_q = 0; first_q < W_INST; first_q += HALF) {
        const i32x4 d = descriptor(from + (first_q ? cols * b_row : 0), bytes);
#pragma unroll
        for (int q = 0; q < HALF; ++q)
          load_lds16(d, (q & 1 ? odd : even) ? w_off[q & 1] + (uint32_t)((q & ~1) * 8 * b_row)
                                             : kNowhere, dst + (first_q + q) * 1024);
      }
    }
    const i32x4 d = descriptor(x_base + (size_t)at * 128, x_bytes - (uint32_t)at * 128);
#pragma unroll
    for (int q = 0; q < X_INST; ++q)
      load_lds16(d, (q & 1 ? odd : even) ? x_off[q] : kNowhere, dst + kWBytes + q * 1024);
    if constexpr (S_STAGE)
      load_lds4(descriptor(s_base + (size_t)at * 4, s_bytes - (uint32_t)at * 4), s_off,
                dst + kWBytes + kXBytes);
  };

  // fragments of v_mfma_*_16x16: lane l holds row or column l % 16 and 16 bytes of
  // the sum, quarter l / 16 of the k-step
  const int l16 = lane & 15, g = lane >> 4;
  typedef typename std::conditional<I8, i32x4, f32x4>::type Acc;
  Acc acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = Acc{};
  const LDS_AS char* ring = (const LDS_AS char*)smem_raw + wave * STAGES * kStage;
  // (cs: the columns' scale, row: the rows' where a register has it)
  auto multiply = [&](const LDS_AS char* stage, float row, float cs) {
    f32x4 part[FP8 ? MB : 1][FP8 ? NB : 1];
    if constexpr (FP8) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) part[i][j] = f32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      u32x4 fw[NB], fx[MB];
      const int chunk = 4 * ks + g;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        if constexpr (B_ACROSS) {
          typedef short s16x4 __attribute__((ext_vector_type(4)));
          u32x2 h2[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int row = ks * 32 + g * 8 + h * 4 + (l16 >> 2);
            const int c = (j * 2 + ((l16 & 3) >> 1)) ^ swz_sum(row);
            h2[h] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (LDS_AS s16x4*)(stage + row * 128 + c * 16 + (l16 & 1) * 8)));
          }
          fw[j] = u32x4{h2[0][0], h2[0][1], h2[1][0], h2[1][1]};
        } else {
          const int row = j * 16 + l16;
          fw[j] = *reinterpret_cast<const LDS_AS u32x4*>(stage + row * 128 +
                                                         ((chunk ^ swz_along(row)) << 4));
        }
      }
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const int row = i * 16 + l16;
        fx[i] = *reinterpret_cast<const LDS_AS u32x4*>(stage + kWBytes + row * 128 +
                                                       ((chunk ^ swz_along(row)) << 4));
      }
      if constexpr (FP8) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8 bx[MB];
#pragma unroll
          for (int i = 0; i < MB; ++i) bx[i] = fp8x8_to_bf16(u32x2{fx[i][2 * h], fx[i][2 * h + 1]});
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            const bf16x8 bw = fp8x8_to_bf16(u32x2{fw[j][2 * h], fw[j][2 * h + 1]});
#pragma unroll
            for (int i = 0; i < MB; ++i)
              part[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw, bx[i], part[i][j], 0, 0, 0);
          }
        }
        continue;
      }
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          if constexpr (I8)
            acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
                __builtin_bit_cast(i32x4, fw[j]), __builtin_bit_cast(i32x4, fx[i]), acc[i][j], 0,
                0, 0);
          else
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, fw[j]), __builtin_bit_cast(bf16x8, fx[i]), acc[i][j], 0,
                0, 0);
        }
    }
    if constexpr (FP8) {
      float rs[MB];
      bool far = false;
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        rs[i] = S_REG ? row : *reinterpret_cast<const LDS_AS float*>(stage + kWBytes + kXBytes +
                                                                     (i * 16 + l16) * 4);
        const float f = scale_of(rs[i], cs, far);
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int v = 0; v < 4; ++v) acc[i][j][v] = fmaf(part[i][j][v], f, acc[i][j][v]);
      }
      if (__builtin_expect(__any(far), false)) {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v)
              acc[i][j][v] = add_far(part[i][j][v], rs[i], cs, acc[i][j][v]);
      }
    }
  };

#pragma unroll
  for (int s = 0; s < STAGES; ++s)
    if (s < nk) issue(s);
  float col = FP8 && nk > 0 ? col_scale[first] : 0.0f;
  // (a load that the compiler waits for waits for the ring as well: once in four tiles)
  float four = 0.0f, coming = S_REG && nk > 0 ? row_scale[min(first + g, kb - 1)] : 0.0f;
  for (int kt = 0; kt < nk; ++kt) {
    if constexpr (S_REG) {
      if ((kt & 3) == 0) {
        four = coming;
        if (kt + 4 < nk) coming = row_scale[min(first + kt + 4 + g, kb - 1)];
      }
    }
    const float next = FP8 ? col_scale[first + min(kt + 1, nk - 1)] : 0.0f;
    // (past the last full ring the count is not known here: wait for all)
    if (kt + STAGES <= nk) wait_vmcnt<(STAGES - 1) * INST>();
    else wait_vmcnt<0>();
    asm volatile("" ::: "memory");
    multiply(ring + (kt % STAGES) * kStage, S_REG ? __shfl(four, (kt & 3) * 16 + l16, kWave) : 0.0f,
             col);
    col = next;
    // the stage is read: it may be filled again
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (kt + STAGES < nk) issue(kt + STAGES);
  }

  // the waves' results through LDS, added in ascending order of the sum
  __syncthreads();
  LDS_AS char* sums = (LDS_AS char*)smem_raw;
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
      *reinterpret_cast<LDS_AS Acc*>(sums + ((wave * BI + i * 16 + l16) * LD + j * 16 + 4 * g) * 4) =
          acc[i][j];
  __syncthreads();
  if constexpr (EPI != kPlain) {
    // eight columns of the result a thread
    constexpr int PER = kOutJ / 8;
    for (int u = threadIdx.x; u < BI * PER; u += kThreads) {
      const int ri = u / PER, c = (u % PER) * 8, col0 = t.j0 + c, n = cols - col0;
      if (ri >= t.i_valid || n <= 0) continue;
      const int row = t.i0 + ri;
      float a[8] = {}, b[8] = {};
#pragma unroll
      for (int s = 0; s < kWaves; ++s)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const LDS_AS char* from = sums + ((s * BI + ri) * LD + c + 4 * q) * 4;
          const f32x4 x = *reinterpret_cast<const LDS_AS f32x4*>(from);
          f32x4 y = x;
          if constexpr (EPI == kSwiglu)
            y = *reinterpret_cast<const LDS_AS f32x4*>(from + kOutJ * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            a[4 * q + e] += x[e];
            b[4 * q + e] += y[e];
          }
        }
      if (p.splits > 1) {
        const int wide = columns<DIR>(p);
        float* o = static_cast<float*>(p.part) + ((size_t)blockIdx.y * p.R + row) * wide + col0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < n) {
            o[e] = a[e];
            if constexpr (EPI == kSwiglu) o[cols + e] = b[e];
          }
      } else if constexpr (EPI == kSwiglu) {
        store_swiglu(p, row, col0, n, a, b);
      } else {
        store_swiglu_grad(p, row, col0, n, load_gate_up(p, row, col0, n), a, false);
      }
    }
    return;
  }
#pragma unroll
  for (int u = 0; u < MB; ++u) {
    const int ri = u * 16 + (int)threadIdx.x / 16, c = (threadIdx.x & 15) * 4;
    const int col = t.j0 + c, row = t.i0 + ri;
    if (ri >= t.i_valid || col >= cols) continue;
    Acc v = Acc{};
#pragma unroll
    for (int s = 0; s < kWaves; ++s)
      v += *reinterpret_cast<const LDS_AS Acc*>(sums + ((s * BI + ri) * LD + c) * 4);
    if (p.splits > 1) {
      auto* o = static_cast<typename std::conditional<I8, int, float>::type*>(p.part) +
                part_at<DIR>(p, blockIdx.y, t.e, row, col);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (col + q < cols) o[q] = v[q];
    } else if constexpr (I8) {
      store4<DIR>(p, t.e, row, col, scaled(p, t.e, p.row_scale[source_row(p, row)], col, v));
    } else {
      store4<DIR>(p, t.e, row, col, v);
    }
  }
}

template <int DIR, int TYPE, int EPI, int MB, int STAGES>
hipError_t launch(const GroupedParams& p, long long tiles, hipStream_t stream) {
  hipLaunchKernelGGL((grouped_few_kernel<DIR, TYPE, EPI, MB, STAGES>), tile_grid(tiles, p.splits),
                     dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

template <int DIR, int TYPE, int EPI>
hipError_t launch_grouped_few(const GroupedParams& p, int rows, long long tiles,
                              hipStream_t stream) {
  if (tiles > 0x7fffffffLL) return hipErrorInvalidValue;
  if (rows == 16) return launch<DIR, TYPE, EPI, 1, 2>(p, tiles, stream);
  if (rows == 32) return launch<DIR, TYPE, EPI, 2, 3>(p, tiles, stream);
  return launch<DIR, TYPE, EPI, 4, 2>(p, tiles, stream);
}

template hipError_t launch_grouped_few<kForward, kBf16, kPlain>(const GroupedParams&, int, long long, hipStream_t);
template hipError_t launch_grouped_few<kForward, kInt8, kPlain>(const GroupedParams&, int, long long, hipStream_t);
template hipError_t launch_grouped_few<kForward, kFp8, kPlain>(const GroupedParams&, int, long long, hipStream_t);
template hipError_t launch_grouped_few<kForward, kBf16, kSwiglu>(const GroupedParams&, int, long long, hipStream_t);
template hipError_t launch_grouped_few<kGradRows, kBf16, kPlain>(const GroupedParams&, int, long long, hipStream_t);
template hipError_t launch_grouped_few<kGradRows, kBf16, kSwigluGrad>(const GroupedParams&, int, long long, hipStream_t);

}  // namespace eaas
