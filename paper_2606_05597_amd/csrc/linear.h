// What the products of grpo_linear.h share: activations, the epilogue, and the launch of the tiled product.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>

#include "device.h"
#include "grpo_linear.h"

namespace grpo {

// ---- activations ----------------------------------------------------------------
// On the hardware's exp2 and reciprocal (an ulp each): in a tile's epilogue nothing runs beside them, and the library's
// erff, expf and division took 20 us of a 100 us tile.
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -kLog2e));
}

// (1 + tanh u) / 2 = sigmoid(2u) of u = sqrt(2 / pi) (z + 0.044715 z^3), which for negative z is small and has no 1 to cancel.
__device__ __forceinline__ float twice_u(float z) { return (2.f * 0.79788456f) * fmaf(0.044715f * z * z, z, z); }

// The normal distribution's function at z and e^(-z^2 / 2).  For x >= 0, erfc(x) = (a1 t + .. + a8 t^8) e^(-x^2), t = 1 / (1 +
// 0.33 x): coefficients fitted here for the least largest relative error over 0 <= x <= 9.4 (repeatedly reweighted least
// squares, Lawson's method), 8.2e-8, so that the tail below zero keeps its bits.  Five terms reach 2.8e-5.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.33f * 0.70710678f, fabsf(z), 1.f));
  e = __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2e));
  float p = fmaf(-0.135928795f, t, 0.462688237f);
  p = fmaf(p, t, -0.355438948f);
  p = fmaf(p, t, 0.412541598f);
  p = fmaf(p, t, 0.0450106487f);
  p = fmaf(p, t, 0.201923817f);
  p = fmaf(p, t, 0.182837248f);
  p = fmaf(p, t, 0.186366111f);
  const float half = 0.5f * p * t * e;  // of the tail beyond |z|
  return z >= 0.f ? 1.f - half : half;
}

template <int ACT>
__device__ __forceinline__ float act_of(float z) {
  if constexpr (ACT == GRPO_ACT_RELU) return z > 0.f || isnan(z) ? z : 0.f;
  if constexpr (ACT == GRPO_ACT_GELU) {
    float e;
    return z * normal_cdf(z, e);
  }
  if constexpr (ACT == GRPO_ACT_GELU_TANH) return z * sigmoid(twice_u(z));
  if constexpr (ACT == GRPO_ACT_SILU) return z * sigmoid(z);
  return z;
}

template <int ACT>
__device__ __forceinline__ float slope_of(float z) {
  if constexpr (ACT == GRPO_ACT_RELU) return z > 0.f ? 1.f : isnan(z) ? z : 0.f;
  if constexpr (ACT == GRPO_ACT_GELU) {
    float e;
    const float c = normal_cdf(z, e);
    return fmaf(0.39894228f * z, e, c);
  }
  if constexpr (ACT == GRPO_ACT_GELU_TANH) {
    // s + z s (1 - s) d(2u)/dz, with 1 - s = e s and e held below infinity
    const float e = __builtin_amdgcn_exp2f(fminf(twice_u(z) * -kLog2e, 127.f)), s = __builtin_amdgcn_rcpf(1.f + e);
    const float q = fminf(fabsf(z), 1e6f);  // beyond, s (1 - s) is 0 and z^2 may be infinite
    return fmaf(copysignf(q, z) * (s * (e * s)), (2.f * 0.79788456f) * fmaf(3.f * 0.044715f * q, q, 1.f), s);
  }
  if constexpr (ACT == GRPO_ACT_SILU) {
    const float g = sigmoid(z);
    return g * fmaf(z, 1.f - g, 1.f);
  }
  return 1.f;
}

__device__ __forceinline__ float load_any(const void* p, int64_t i, bool bf16) {
  return bf16 ? bf16_to_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_any(void* p, int64_t i, float v, bool bf16) {
  if (bf16) store_elem(static_cast<uint16_t*>(p) + i, v);
  else static_cast<float*>(p)[i] = v;
}

// ---- the products ---------------------------------------------------------------
struct Epilogue {
  void* out;  // [M, N], rows ldo apart
  int64_t ldo;
  const void* bias;      // [N] or NULL
  const void* residual;  // [M, N] of out's type, rows ldr apart, or NULL
  int64_t ldr;
  float* z;  // [M, N] or NULL
  int act;
  bool out_bf16, bias_bf16, accumulate;
};

// 8 columns of a row, at any alignment of their elements.
__device__ __forceinline__ void load8(const void* p, int64_t i, bool bf16, float (&v)[8]) {
  if (bf16) {
    const u32x4 x = *reinterpret_cast<const u32x4_a2*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = elem<uint16_t>(x, q);
  } else {
    const u32x4_a4* x = reinterpret_cast<const u32x4_a4*>(static_cast<const float*>(p) + i);
    const u32x4 a = x[0], b = x[1];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[q] = __uint_as_float(a[q]);
      v[q + 4] = __uint_as_float(b[q]);
    }
  }
}
__device__ __forceinline__ void store8(void* p, int64_t i, bool bf16, const float (&v)[8]) {
  if (bf16) {
    u32x4 x;
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = pack_bf16(v[2 * q], v[2 * q + 1]);
    *reinterpret_cast<u32x4_a2*>(static_cast<uint16_t*>(p) + i) = x;
  } else {
    u32x4 a, b;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      a[q] = __float_as_uint(v[q]);
      b[q] = __float_as_uint(v[q + 4]);
    }
    u32x4_a4* x = reinterpret_cast<u32x4_a4*>(static_cast<float*>(p) + i);
    x[0] = a;
    x[1] = b;
  }
  asm volatile("s_nop 1" ::: "memory");  // the stores have read their data before their registers are reused
}

// 8 columns as they lie in memory.
struct Raw8 {
  u32x4 a, b;  // bf16: a alone
  __device__ __forceinline__ void load(const void* p, int64_t i, bool bf16) {
    if (bf16) {
      a = *reinterpret_cast<const u32x4_a2*>(static_cast<const uint16_t*>(p) + i);
    } else {
      const u32x4_a4* x = reinterpret_cast<const u32x4_a4*>(static_cast<const float*>(p) + i);
      a = x[0];
      b = x[1];
    }
  }
  __device__ __forceinline__ float at(int q, bool bf16) const {
    return bf16 ? elem<uint16_t>(a, q) : __uint_as_float(q < 4 ? a[q] : b[q - 4]);
  }
};

// The epilogue of 8 sums v of row m, columns n .. n + 7, all of them below N; r: what is added last, or NULL.
template <int ACT>
__device__ __forceinline__ void finish_whole8(const Epilogue& e, int m, int n, int N, const float (&bias)[8], const Raw8* r,
                                              float (&v)[8]) {
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] += bias[q];
  if (e.z) store8(e.z, (int64_t)m * N + n, false, v);
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = act_of<ACT>(v[q]);
  if (r) {
    if (e.out_bf16) {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] += r->at(q, true);
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] += r->at(q, false);
    }
  }
  store8(e.out, (int64_t)m * e.ldo + n, e.out_bf16, v);
}

// The same of the columns below N.
template <int ACT>
__device__ __forceinline__ void finish8(const Epilogue& e, int m, int n, int N, const float (&bias)[8], float (&v)[8]) {
  const bool all = n + 8 <= N;
  const int k = all ? 8 : N - n;
  const int64_t o = (int64_t)m * e.ldo + n;
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] += bias[q];
  if (e.z) {
    const int64_t oz = (int64_t)m * N + n;
    if (all) store8(e.z, oz, false, v);
    else
      for (int q = 0; q < 8; ++q)
        if (q < k) e.z[oz + q] = v[q];
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = act_of<ACT>(v[q]);
  const void* more = e.residual ? e.residual : e.accumulate ? e.out : nullptr;
  if (more) {
    const int64_t om = e.residual ? (int64_t)m * e.ldr + n : o;
    float r[8];
    if (all) load8(more, om, e.out_bf16, r);
    else
#pragma unroll
      for (int q = 0; q < 8; ++q) r[q] = q < k ? load_any(more, om + q, e.out_bf16) : 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] += r[q];
  }
  if (all) store8(e.out, o, e.out_bf16, v);
  else
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < k) store_any(e.out, o + q, v[q], e.out_bf16);
}

// An operand of a tiled product, of `rows` rows, as it lies: with the summed dimension contiguous ([rows, K], rows ld apart),
// or (turned) with the rows contiguous ([K, rows], K's ld apart).  Vectors of 16 bytes: p and ld, and K or (turned) rows,
// are multiples of 8 elements; K's end may be padded with zeros by one operand alone.
struct TileOperand {
  const uint16_t* p;
  int64_t ld;
  bool turned;
};

struct TileArgs {
  TileOperand a, b;
  int M, N, K;
  int splits, split_k;  // > 1: the sums of split_k of K each, to part [splits][M][N]
  float* part;
  Epilogue e;
};

// Tiles of the shapes below.
struct TileShape {
  int m, n;
};
constexpr TileShape kTileShapes[] = {{256, 256}, {128, 128}, {64, 128}, {192, 256}};

// C [M, N] = A B^T, with the epilogue where it is not split.
void launch_tiles(const TileArgs& t, int shape, hipStream_t s);

}  // namespace grpo
