// e4m3 codes with fp32 scales, one for each 128 columns of a row or each 128 x 128
// block of a matrix.
//
// Activation quantization for the fp8-weight, fp8-activation step: per row
// and per block of 128 channels, s = amax / 448 (1 for an all-zero block)
// and q = e4m3fn(x / s), rounded to nearest even and saturated at 448.  The
// scale and the quotient are correctly rounded fp32, so the codes are the
// ones a plain fp32 evaluation of that definition gives.  (The paper's
// grouped-GEMM engine, §4.1, consumes block-scaled fp8 operands; the
// blocking follows the weights' 128-channel K blocks.)
#include <algorithm>

#include "internal.h"
#include "swiglu.h"

namespace eaas {
namespace {

constexpr int kQuantThreads = 256;

// One lane: 8 consecutive values (16 bytes of bf16); 16 lanes: one block of
// 128.  Blocks never straddle rows (K is a multiple of 128), and the chunk
// count is a multiple of 16, so a 16-lane group is always wholly active.
__global__ __launch_bounds__(kQuantThreads) void quantize_rows_kernel(
    const uint16_t* __restrict__ x, long long n_chunks, uint8_t* __restrict__ q,
    float* __restrict__ s) {
  for (long long c = (long long)blockIdx.x * kQuantThreads + threadIdx.x; c < n_chunks;
       c += (long long)gridDim.x * kQuantThreads) {
    const u32x4 raw = *reinterpret_cast<const u32x4*>(x + c * 8);
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(raw[i] << 16);
      v[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
    }
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(v[i]));
#pragma unroll
    for (int m = 8; m >= 1; m >>= 1) amax = fmaxf(amax, __shfl_xor(amax, m, 16));
    const float sc = amax > 0.0f ? amax / 448.0f : 1.0f;
    u32x2 o;
    o[0] = pack_e4m3x4(v[0] / sc, v[1] / sc, v[2] / sc, v[3] / sc);
    o[1] = pack_e4m3x4(v[4] / sc, v[5] / sc, v[6] / sc, v[7] / sc);
    *reinterpret_cast<u32x2*>(q + c * 8) = o;
    if ((c & 15) == 0) s[c >> 4] = sc;
  }
}

// (Measured: rows of 32768 x 2048 in 46 us, 4.4 TB/s; weights of 32 x 4096 x 7168 in 0.66 ms,
// 4.2; gated rows of 32768 x 2048 in 99, 3.4, bound by their instructions.)

// The largest magnitude among 16 lanes of values, as integers: NaN above infinity
// above every finite one.
__device__ __forceinline__ uint32_t largest8(const float (&v)[8], uint32_t m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
}
__device__ __forceinline__ uint32_t largest16(uint32_t m) {
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d, 16));
  return m;
}

// The scale of a block: its largest magnitude times 1/448 rounded to fp32, or 1 where that
// is zero (a block of zeros, or next to fp32's least); NaN if the block holds an infinity or
// a NaN.
__device__ __forceinline__ float block_scale(uint32_t m) {
  if (m >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  const float s = __uint_as_float(m) * (1.0f / 448.0f);
  return s == 0.0f ? 1.0f : s;
}

// n of eight codes to q, which may start on any byte.  (Zeros where the scale is NaN.)
__device__ __forceinline__ void store_codes(uint8_t* q, int n, const float (&v)[8], float sc) {
  uint32_t w[2] = {0, 0};
  if (sc == sc) {
    w[0] = pack_e4m3x4(v[0] / sc, v[1] / sc, v[2] / sc, v[3] / sc);
    w[1] = pack_e4m3x4(v[4] / sc, v[5] / sc, v[6] / sc, v[7] / sc);
  }
  if (n >= 8) {
    __builtin_memcpy(q, w, 8);
  } else {
    for (int i = 0; i < n; ++i) q[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

template <bool FP32>
__device__ __forceinline__ void load_values(const void* x, long long at, int n, float (&v)[8]) {
  if constexpr (FP32) {
    const float* p = static_cast<const float*>(x) + at;
    if (n >= 8) {
      __builtin_memcpy(v, p, 32);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.0f;
      if (n > 0) {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = p[min(i, n - 1)];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? e[i] : 0.0f;
      }
    }
  } else {
    load8(static_cast<const uint16_t*>(x) + at, n, v);
  }
}

// The row of unit u, kb units to a row.  (A 64-bit quotient costs as much as the rest of a
// unit.)
__device__ __forceinline__ long long row_of(long long u, int kb) {
  return u >> 32 ? u / kb : (long long)((uint32_t)u / (uint32_t)kb);
}

// Rows of any length, stride and alignment, a scale for each 128 columns: 16 lanes
// take a block.
template <bool FP32>
__global__ __launch_bounds__(kQuantThreads) void quantize_row_blocks_kernel(
    const void* __restrict__ x, long long ldx, long long rows, int K, uint8_t* __restrict__ q,
    float* __restrict__ s) {
  const int kb = ceil_div(K, 128);
  const long long total = rows * kb;
  const int l = threadIdx.x & 15;
  for (long long u = ((long long)blockIdx.x * kQuantThreads + threadIdx.x) >> 4; u < total;
       u += (long long)gridDim.x * (kQuantThreads / 16)) {
    const long long r = row_of(u, kb);
    const int b = (int)(u - r * kb), c = b * 128 + l * 8, n = K - c;
    float v[8];
    load_values<FP32>(x, r * ldx + c, n, v);
    const float sc = block_scale(largest16(largest8(v, 0)));
    store_codes(q + r * K + c, n, v, sc);
    if (l == 0) s[u] = sc;
  }
}

// Matrices [rows, K] with a scale for each 128 x 128 block: a workgroup takes a block,
// thread t columns 8 (t % 16) .. +7 of rows t / 16 + 16 i.
template <bool FP32>
__global__ __launch_bounds__(kQuantThreads) void quantize_blocks_kernel(
    const void* __restrict__ x, long long ldx, long long mats, long long rows, int K,
    uint8_t* __restrict__ q, float* __restrict__ s) {
  __shared__ uint32_t s_max[kQuantThreads / kWave];
  const int kb = ceil_div(K, 128);
  const long long nb = (rows + 127) / 128, total = mats * nb * kb;
  const int col = (threadIdx.x & 15) * 8, row = threadIdx.x >> 4;
  for (long long u = blockIdx.x; u < total; u += gridDim.x) {
    const int b = (int)(u % kb);
    const long long bi = u / kb % nb, m = u / kb / nb;
    const int c = b * 128 + col, n = K - c;
    float v[8][8];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const long long r = bi * 128 + row + 16 * i;
      load_values<FP32>(x, (m * rows + min(r, rows - 1)) * ldx + c, r < rows ? n : 0, v[i]);
      most = largest8(v[i], most);
    }
    most = largest16(most);
    most = max(most, (uint32_t)__shfl_xor((int)most, 16));
    most = max(most, (uint32_t)__shfl_xor((int)most, 32));
    __syncthreads();  // (the last block's maxima are read)
    if ((threadIdx.x & (kWave - 1)) == 0) s_max[threadIdx.x / kWave] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kQuantThreads / kWave; ++w) most = max(most, s_max[w]);
    const float sc = block_scale(most);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const long long r = bi * 128 + row + 16 * i;
      if (r < rows) store_codes(q + (m * rows + r) * K + c, n, v[i], sc);
    }
    if (threadIdx.x == 0) s[u] = sc;
  }
}

// Finite values to e4m3 codes.
__device__ __forceinline__ float within_448(float v) {
  return __builtin_amdgcn_fmed3f(v, -448.0f, 448.0f);
}
__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// silu(gate) * up in 64 bits, rounded once to fp32.
__device__ __noinline__ float silu_up_64(float g, float up) {
  return (float)((double)g / (1.0 + exp(-(double)g)) * (double)up);
}

// g / (1 + exp(-g)) from a gate of kFar or more, to four units in the last place: exp(-g)
// is two to the power of -g log2(e), whose product is kept with its remainder, hi + lo, and
// 2^lo = 1 + lo ln(2) to fp32.  (Six instructions where the full exponential has fourteen;
// 32768 rows of 2048: 109 -> 99 us.)
__device__ __forceinline__ float silu_near(float g) {
  constexpr double kLog2e = 1.4426950408889634;
  constexpr float kHi = (float)kLog2e, kLo = (float)(kLog2e - (double)kHi);
  const float hi = -g * kHi;
  const float lo = fmaf(-g, kLo, fmaf(-g, kHi, -hi));
  const float z = __builtin_amdgcn_exp2f(hi);
  const float d = 1.0f + fmaf(z, lo * 0.693147181f, z);
  const float y = __builtin_amdgcn_rcpf(d);
  const float q = g * y;
  return fmaf(fmaf(-q, d, g), y, q);
}

// Rows of [gate | up] to h = silu(gate) * up as e4m3 codes, a scale for each 128 columns;
// 16 lanes take a block.  Scale and codes are those of h rounded once to fp32: where a
// value falls next to the middle between two codes, an error in its last place costs a
// whole step (with plain fp32 values, about one code in 10^6, the results of a following
// fp32 product were 1.7e-4 of their norm off).  So h is computed in fp32, to a few units
// in its last place, and again in 64 bits where that matters: for the values next to the
// block's largest, and for a lane's codes if moving a quotient by 2^-20 of itself changes
// one.  (Blocks near either end of fp32's range, where such bounds do not hold, take 64
// bits throughout.)
__global__ __launch_bounds__(kQuantThreads) void swiglu_fp8_kernel(
    const uint16_t* __restrict__ gu, long long rows, int I, const int32_t* n_rows,
    uint8_t* __restrict__ q, float* __restrict__ s) {
  const int kb = ceil_div(I, 128);
  const long long total = live_rows(rows, n_rows) * kb;
  const int l = threadIdx.x & 15;
  for (long long u = ((long long)blockIdx.x * kQuantThreads + threadIdx.x) >> 4; u < total;
       u += (long long)gridDim.x * (kQuantThreads / 16)) {
    const long long r = row_of(u, kb);
    const int b = (int)(u - r * kb), c = b * 128 + l * 8, n = I - c;
    const uint16_t* row = gu + r * 2 * I + c;
    float g[8], up[8], v[8];
    load8(row, n, g);
    load8(row + I, n, up);
    bool far = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = silu_near(g[i]) * up[i];
      far |= g[i] < kFar;
    }
    if (far) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (g[i] < kFar) v[i] = silu_far_up(g[i], up[i]);
    }
    const uint32_t mine = largest8(v, 0), m = largest16(mine);
    const bool ends = m - 0x0d000000u >= 0x70000000u;  // below 2^-101 or from 2^123 on
    // the values that may be the block's largest, in 64 bits: one, as a rule
    uint32_t most = 0;
    const uint32_t near = ends ? 0 : m - 16;
    if (m != 0 && mine >= near) {
      uint32_t left = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        left |= (__float_as_uint(v[i]) & 0x7fffffffu) >= near ? 1u << i : 0u;
      do {
        const int at = __builtin_ctz(left);
        float ga = g[0], ua = up[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) {
          ga = at == i ? g[i] : ga;
          ua = at == i ? up[i] : ua;
        }
        most = max(most, __float_as_uint(silu_up_64(ga, ua)) & 0x7fffffffu);
        left &= left - 1;
      } while (left);
    }
    most = largest16(most);
    const float sc = block_scale(most);
    uint32_t w[2] = {0, 0};
    if (sc == sc) {
      const float lo = __builtin_amdgcn_rcpf(sc) * (1.0f - 0x1p-20f);
      const float hi = __builtin_amdgcn_rcpf(sc) * (1.0f + 0x1p-20f);
      uint32_t w2[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // (the smaller quotients are at most 448 by themselves)
        const float* x = v + 4 * h;
        w[h] = pack_codes(x[0] * lo, x[1] * lo, x[2] * lo, x[3] * lo);
        w2[h] = pack_codes(within_448(x[0] * hi), within_448(x[1] * hi), within_448(x[2] * hi),
                           within_448(x[3] * hi));
      }
      if (ends || w[0] != w2[0] || w[1] != w2[1]) {
#pragma unroll 1
        for (int i = 0; i < 8; ++i) v[i] = silu_up_64(g[i], up[i]);
        w[0] = pack_e4m3x4(v[0] / sc, v[1] / sc, v[2] / sc, v[3] / sc);
        w[1] = pack_e4m3x4(v[4] / sc, v[5] / sc, v[6] / sc, v[7] / sc);
      }
    }
    uint8_t* o = q + r * I + c;
    if (n >= 8) {
      __builtin_memcpy(o, w, 8);
    } else {
      for (int i = 0; i < n; ++i) o[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
    }
    if (l == 0) s[u] = sc;
  }
}

// Workgroups of a pass over `units` of 16 lanes each.
unsigned unit_grid(long long units) {
  return (unsigned)std::min<long long>((units + kQuantThreads / 16 - 1) / (kQuantThreads / 16),
                                       8192);
}

}  // namespace

hipError_t launch_quantize_blocks(const void* x, bool fp32, long long ldx, long long mats,
                                  long long rows, int K, int block_rows, uint8_t* q, float* s,
                                  hipStream_t stream) {
  if (mats * rows <= 0) return hipSuccess;
  const long long kb = ceil_div(K, 128);
  if (block_rows == 1) {
    const dim3 grid(unit_grid(mats * rows * kb));
    if (fp32)
      hipLaunchKernelGGL(quantize_row_blocks_kernel<true>, grid, dim3(kQuantThreads), 0, stream, x,
                         ldx, mats * rows, K, q, s);
    else
      hipLaunchKernelGGL(quantize_row_blocks_kernel<false>, grid, dim3(kQuantThreads), 0, stream, x,
                         ldx, mats * rows, K, q, s);
  } else {
    const dim3 grid((unsigned)std::min<long long>(mats * ((rows + 127) / 128) * kb, 1 << 16));
    if (fp32)
      hipLaunchKernelGGL(quantize_blocks_kernel<true>, grid, dim3(kQuantThreads), 0, stream, x, ldx,
                         mats, rows, K, q, s);
    else
      hipLaunchKernelGGL(quantize_blocks_kernel<false>, grid, dim3(kQuantThreads), 0, stream, x,
                         ldx, mats, rows, K, q, s);
  }
  return hipGetLastError();
}

hipError_t launch_swiglu_fp8(const uint16_t* gu, long long rows, int I, const int32_t* n_rows,
                             uint8_t* q, float* s, hipStream_t stream) {
  if (rows <= 0) return hipSuccess;
  hipLaunchKernelGGL(swiglu_fp8_kernel, dim3(unit_grid(rows * ceil_div(I, 128))),
                     dim3(kQuantThreads), 0, stream, gu, rows, I, n_rows, q, s);
  return hipGetLastError();
}

hipError_t launch_quantize_rows(const uint16_t* x, long long rows, int K, uint8_t* q, float* s,
                                hipStream_t stream) {
  const long long n_chunks = rows * (K / 8);
  if (n_chunks <= 0) return hipSuccess;
  const long long blocks = (n_chunks + kQuantThreads - 1) / kQuantThreads;
  const unsigned grid = (unsigned)(blocks < 8192 ? blocks : 8192);
  hipLaunchKernelGGL(quantize_rows_kernel, dim3(grid), dim3(kQuantThreads), 0, stream, x,
                     n_chunks, q, s);
  return hipGetLastError();
}

}  // namespace eaas
