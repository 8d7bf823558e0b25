// The activation h = silu(gate) * up and its gradient, value by value, and the
// 16-byte accesses of the kernels that pass over rows of them (activation.hip,
// quant.hip) or compute them from a product's sums (grouped.hip and its parts).
#pragma once

#include "common.h"

namespace eaas {

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
  } else if (n > 0) {
    // (every element is loaded, the last one repeatedly: loads under a condition each would
    // be waited for one by one)
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = p[min(i, n - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? __uint_as_float(e[i] << 16) : 0.0f;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
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

// The same from a product's sums, in an order that keeps its precision for any up: the gate
// times its sigmoid alone leaves the normal range below -93, and may be wanted times 10^30.
__device__ __forceinline__ float gated(float g, float up) {
  const Sigmoid t = sigmoid(g);
  return (g * t.hi) * (t.lo * up);
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

// The gradient of a gate and its up value from that of h, and h itself.
struct SwigluGrad {
  float gate, up;
};
__device__ __forceinline__ SwigluGrad swiglu_grad(float g, float up, float dh) {
  const Sigmoid t = sigmoid(g);
  return {dh * up * t.hi * (t.lo * (1.0f + g * (1.0f - t.hi * t.lo))), (dh * g * t.hi) * t.lo};
}

__device__ __forceinline__ long long live_rows(long long rows, const int32_t* n_rows) {
  return n_rows ? min(rows, (long long)max(*n_rows, 0)) : rows;
}

}  // namespace eaas
