// What stands between and around the grouped products of an expert layer: the
// activation h = silu(gate) * up and its gradient, rows in 8-bit integers, and
// the gradient of the weighted combine.  All of it is bound by memory: each value
// is read once and written once, 16 bytes a lane, and what a row needs as a whole
// (its largest magnitude, its inner product) is reduced while the row stays in
// registers.  32768 rows of 2048: h in 73 us (5.5 TB/s), its gradient 118 (5.7), as
// 8-bit rows 77 (4.4: 41 vector instructions a value, which take 82% of the cycles), bf16
// rows to 8 bits 39 (5.1); the combine's gradient, 4096 tokens of 8 slots, 7168 wide:
// 296 (5.0).
#include <algorithm>

#include "common.h"
#include "internal.h"

namespace eaas {
namespace {

constexpr int kThreads = 256;

// Eight bf16 at an address of 2-byte alignment, n of them valid (zeros after).
__device__ __forceinline__ void load8(const uint16_t* p, int n, float (&v)[8]) {
  if (n >= 8) {
    u32x4 raw;
    __builtin_memcpy(&raw, p, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(raw[i] << 16);
      v[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? __uint_as_float((uint32_t)p[i] << 16) : 0.0f;
  }
}

__device__ __forceinline__ void store8(uint16_t* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i)  // (one instruction a pair)
      o[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]});
    __builtin_memcpy(p, &o, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (uint16_t)f32_to_bf16_bits(v[i]);
  }
}

// 1 / (1 + exp(-g)) as a product hi * lo: with z = exp(-|g| / 2) it is z * (z / (1 +
// z^2)) for g < 0 and 1 * (1 / (1 + z^2)) otherwise, so a gate far below zero,
// whose sigmoid alone is under the normal range of fp32, keeps its precision
// until the product with the gate is taken.  The hardware exponential and
// reciprocal err by a few units in the last place of fp32, far below the rounding
// of the results to bf16.
struct Sigmoid {
  float hi, lo;
};
__device__ __forceinline__ Sigmoid sigmoid(float g) {
  const float z = __expf(-0.5f * fabsf(g));
  const float r = __builtin_amdgcn_rcpf(1.0f + z * z);
  return g < 0.0f ? Sigmoid{z, z * r} : Sigmoid{1.0f, r};
}

__device__ __forceinline__ float silu_up(float g, float up) {
  const Sigmoid t = sigmoid(g);
  return (g * t.hi) * t.lo * up;
}

// g / (1 + exp(-g)) from a gate of kFar or more, to about two units in the last place:
// the full exponential and its sum with 1 are rounded, the quotient is corrected by
// its remainder.  (The reciprocal is a normal number there.)
constexpr float kFar = -86.0f;
__device__ __forceinline__ float silu_full(float g) {
  const float d = 1.0f + expf(-g);
  const float y = __builtin_amdgcn_rcpf(d);
  const float q = g * y;
  return fmaf(fmaf(-q, d, g), y, q);
}

// The same times up, below kFar: the quotient is g exp(g) to fp32, whose exponential
// leaves the normal range from -87.3 on; two factors exp(g / 2) do not, and each takes
// its share of the product.
__device__ __forceinline__ float silu_far_up(float g, float up) {
  const float z = expf(0.5f * g);
  return (g * z) * (z * up);
}

__device__ __forceinline__ long long live_rows(long long rows, const int32_t* n_rows) {
  return n_rows ? min(rows, (long long)max(*n_rows, 0)) : rows;
}

// One thread: eight columns of a row.
template <bool BACKWARD>
__global__ __launch_bounds__(kThreads) void swiglu_kernel(const uint16_t* gu, const uint16_t* dh,
                                                          long long rows, int I,
                                                          const int32_t* n_rows, uint16_t* out) {
  const int chunks = ceil_div(I, 8);
  const long long total = live_rows(rows, n_rows) * chunks;
  for (long long u = (long long)blockIdx.x * kThreads + threadIdx.x; u < total;
       u += (long long)gridDim.x * kThreads) {
    const long long r = u / chunks;
    const int c = (int)(u - r * chunks) * 8;
    const int n = I - c;
    const uint16_t* row = gu + r * 2 * I + c;
    float g[8], up[8], o[8];
    load8(row, n, g);
    load8(row + I, n, up);
    if constexpr (!BACKWARD) {
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = silu_up(g[i], up[i]);
      store8(out + r * I + c, n, o);
    } else {
      float d[8], o2[8];
      load8(dh + r * I + c, n, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const Sigmoid t = sigmoid(g[i]);
        o[i] = d[i] * up[i] * t.hi * (t.lo * (1.0f + g[i] * (1.0f - t.hi * t.lo)));
        o2[i] = (d[i] * g[i] * t.hi) * t.lo;
      }
      store8(out + r * 2 * I + c, n, o);
      store8(out + r * 2 * I + I + c, n, o2);
    }
  }
}

// Rows in 8-bit integers: TPR threads to a row, each with up to HELD chunks of
// eight values in registers between the row's largest magnitude and its codes
// (HELD = 0: any length; the values are computed again for the codes).
// SWIGLU: the values are silu(gate) * up of a row [gate | up] of 2K, with the
// exponential and the quotient of full precision: where a value falls next to the
// middle between two codes, an error in its last place costs a whole step.
template <bool SWIGLU, int TPR, int HELD>
__global__ __launch_bounds__(kThreads) void quantize_int8_kernel(const uint16_t* x, long long ldx,
                                                                 long long rows, int K,
                                                                 const int32_t* n_rows, int8_t* q,
                                                                 float* s) {
  __shared__ uint32_t s_max[kThreads / kWave];
  const int tid = threadIdx.x % TPR;
  const int chunks = ceil_div(K, 8);
  const long long live = live_rows(rows, n_rows);
  auto value = [&](const uint16_t* row, int c, float (&v)[8]) {
    load8(row + c, K - c, v);
    if constexpr (SWIGLU) {
      float up[8], o[8];
      load8(row + K + c, K - c, up);
      bool far = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        o[i] = silu_full(v[i]) * up[i];
        far |= v[i] < kFar;
      }
      if (far) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (v[i] < kFar) o[i] = silu_far_up(v[i], up[i]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = o[i];
    }
  };
  // magnitudes as integers: NaN above infinity above every finite one
  auto largest = [](const float (&v)[8], uint32_t m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
  };
  constexpr int RPB = kThreads / TPR;
  for (long long r0 = (long long)blockIdx.x * RPB; r0 < live; r0 += (long long)gridDim.x * RPB) {
    const long long r = r0 + threadIdx.x / TPR;
    const bool on = r < live;
    const uint16_t* row = x + (on ? r : r0) * ldx;
    float held[HELD > 0 ? HELD : 1][8];
    uint32_t m = 0;
    if constexpr (HELD > 0) {
#pragma unroll
      for (int h = 0; h < HELD; ++h) {
        const int ch = tid + h * TPR;
        if (ch < chunks) {
          value(row, ch * 8, held[h]);
          m = largest(held[h], m);
        }
      }
    } else {
      for (int ch = tid; ch < chunks; ch += TPR) {
        value(row, ch * 8, held[0]);
        m = largest(held[0], m);
      }
    }
#pragma unroll
    for (int d = 1; d < (TPR < kWave ? TPR : kWave); d <<= 1)
      m = max(m, (uint32_t)__shfl_xor((int)m, d, kWave));
    if constexpr (TPR > kWave) {
      __syncthreads();
      if ((threadIdx.x & (kWave - 1)) == 0) s_max[threadIdx.x / kWave] = m;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kThreads / kWave; ++w) m = max(m, s_max[w]);
    }
    const bool finite = m < 0x7f800000u;
    const float amax = __uint_as_float(m);
    // (the product is zero for a row of zeros, and below 2^-143 too)
    const float step = amax * (1.0f / 127.0f);
    const float sc = !finite ? __uint_as_float(0x7fc00000u) : step == 0.0f ? 1.0f : step;
    const float inv = __builtin_amdgcn_rcpf(sc);
    auto emit = [&](int ch, const float (&v)[8]) {
      // A product with the reciprocal is within 1e-4 of the quotient (at most 128, a
      // few units in the last place): it gives the same code unless that close to
      // the middle between two, where the quotient itself decides.  (So it does
      // where the product is not a number: a scale below the normal range, or NaN.)
      float code[8];
      bool close = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float t = v[i] * inv;
        code[i] = rintf(t);
        close |= !(fabsf(t - code[i]) < 0.4999f);
      }
      if (close) {
        // (a scale below the normal range is coarse: keep its quotients in range)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          code[i] = finite ? fminf(fmaxf(rintf(v[i] / sc), -127.0f), 127.0f) : 0.0f;
      }
      uint32_t w[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i / 4] |= (uint32_t)((int)code[i] & 0xff) << (8 * (i % 4));
      int8_t* o = q + r * K + ch * 8;
      if (K - ch * 8 >= 8) {
        __builtin_memcpy(o, w, 8);
      } else {
        for (int i = 0; i < K - ch * 8; ++i) o[i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
      }
    };
    if (on) {
      if constexpr (HELD > 0) {
#pragma unroll
        for (int h = 0; h < HELD; ++h)
          if (tid + h * TPR < chunks) emit(tid + h * TPR, held[h]);
      } else {
        for (int ch = tid; ch < chunks; ch += TPR) {
          value(row, ch * 8, held[0]);
          emit(ch, held[0]);
        }
      }
      if (tid == 0) s[r] = sc;
    }
  }
}

template <bool SWIGLU>
hipError_t launch_int8(const uint16_t* x, long long ldx, long long rows, int K,
                       const int32_t* n_rows, int8_t* q, float* s, hipStream_t stream) {
  if (rows <= 0) return hipSuccess;
  auto go = [&](auto kernel, int tpr) {
    const long long blocks = (rows + kThreads / tpr - 1) / (kThreads / tpr);
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<long long>(blocks, 1 << 16)),
                       dim3(kThreads), 0, stream, x, ldx, rows, K, n_rows, q, s);
    return hipGetLastError();
  };
  // A wave to a row where there are rows enough to fill the chip with them (no
  // barrier, and a lane's chunks are loaded together): 65536 rows of 768 in 59 us
  // against 102 with a workgroup to a row, 32768 of 2048 in 77 against 82; else a
  // workgroup to a row.
  if (rows >= 2048 && K <= 2048) {
    if (K <= 512) return go(quantize_int8_kernel<SWIGLU, 64, 1>, 64);
    if (K <= 1024) return go(quantize_int8_kernel<SWIGLU, 64, 2>, 64);
    return go(quantize_int8_kernel<SWIGLU, 64, 4>, 64);
  }
  if (K <= 2048) return go(quantize_int8_kernel<SWIGLU, 256, 1>, 256);
  if (K <= 8192) return go(quantize_int8_kernel<SWIGLU, 256, 4>, 256);
  if (K <= 16384) return go(quantize_int8_kernel<SWIGLU, 256, 8>, 256);
  return go(quantize_int8_kernel<SWIGLU, 256, 0>, 256);
}

// Gradient of the combine: TPS threads take a slot.
template <int TPS, bool FP32>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(
    const void* dout, const float* y, const int32_t* inv, const float* w, int R, int H, int k,
    uint16_t* dy, float* dw) {
  __shared__ float s_sum[kThreads / kWave];
  const int tid = threadIdx.x % TPS;
  const int slot = blockIdx.x * (kThreads / TPS) + threadIdx.x / TPS;
  const int row = slot < R ? inv[slot] : -1;
  const bool on = row >= 0 && row < R;
  float sum = 0.0f;
  if (on) {
    const float ws = w[slot];
    const size_t src = (size_t)(slot / k) * H, dst = (size_t)row * H;
    for (int c = tid * 8; c < H; c += TPS * 8) {
      float d[8], o[8];
      if constexpr (FP32) {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(dout) + src + c);
        const f32x4 lo = p[0], hi = p[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          d[i] = lo[i];
          d[4 + i] = hi[i];
        }
      } else {
        load8(static_cast<const uint16_t*>(dout) + src + c, 8, d);
      }
      const f32x4* py = reinterpret_cast<const f32x4*>(y + dst + c);
      const f32x4 lo = __builtin_nontemporal_load(py), hi = __builtin_nontemporal_load(py + 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum += d[i] * lo[i] + d[4 + i] * hi[i];
        o[i] = ws * d[i];
        o[4 + i] = ws * d[4 + i];
      }
      store8(dy + dst + c, 8, o);
    }
  }
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) sum += __shfl_xor(sum, m, kWave);
  if constexpr (TPS > kWave) {
    if ((threadIdx.x & (kWave - 1)) == 0) s_sum[threadIdx.x / kWave] = sum;
    __syncthreads();
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kThreads / kWave; ++i) sum += s_sum[i];
  }
  if (tid == 0 && slot < R) dw[slot] = on ? sum : 0.0f;
}

unsigned swiglu_grid(long long rows, int I) {
  const long long n = rows * ceil_div(I, 8);
  return (unsigned)std::min<long long>((n + kThreads - 1) / kThreads, 1 << 16);
}

}  // namespace

hipError_t launch_swiglu(const uint16_t* gu, long long rows, int I, const int32_t* n_rows,
                         uint16_t* h, hipStream_t stream) {
  if (rows <= 0) return hipSuccess;
  hipLaunchKernelGGL(swiglu_kernel<false>, dim3(swiglu_grid(rows, I)), dim3(kThreads), 0, stream,
                     gu, nullptr, rows, I, n_rows, h);
  return hipGetLastError();
}

hipError_t launch_swiglu_backward(const uint16_t* gu, const uint16_t* dh, long long rows, int I,
                                  const int32_t* n_rows, uint16_t* dgu, hipStream_t stream) {
  if (rows <= 0) return hipSuccess;
  hipLaunchKernelGGL(swiglu_kernel<true>, dim3(swiglu_grid(rows, I)), dim3(kThreads), 0, stream,
                     gu, dh, rows, I, n_rows, dgu);
  return hipGetLastError();
}

hipError_t launch_quantize_int8(const uint16_t* x, long long ldx, long long rows, int K, int8_t* q,
                                float* s, hipStream_t stream) {
  return launch_int8<false>(x, ldx, rows, K, nullptr, q, s, stream);
}

hipError_t launch_swiglu_int8(const uint16_t* gu, long long rows, int I, const int32_t* n_rows,
                              int8_t* q, float* s, hipStream_t stream) {
  return launch_int8<true>(gu, 2LL * I, rows, I, n_rows, q, s, stream);
}

hipError_t launch_combine_backward(const void* dout, bool dout_fp32, const float* y,
                                   const int32_t* inv, const float* w, int T, int H, int k,
                                   uint16_t* dy, float* dw, hipStream_t stream) {
  const int R = T * k;
  if (R <= 0) return hipSuccess;
  // few slots: a workgroup each; many: a wave each, which needs no barrier
  auto go = [&](auto kernel, int tps) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(R, kThreads / tps)), dim3(kThreads), 0,
                       stream, dout, y, inv, w, R, H, k, dy, dw);
    return hipGetLastError();
  };
  if (R <= 4096)
    return dout_fp32 ? go(combine_backward_kernel<256, true>, 256)
                     : go(combine_backward_kernel<256, false>, 256);
  return dout_fp32 ? go(combine_backward_kernel<64, true>, 64)
                   : go(combine_backward_kernel<64, false>, 64);
}

}  // namespace eaas
