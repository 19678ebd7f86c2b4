// Internal: element types and store steps shared by the kernels of the training path.
#pragma once
#include "plain.h"
#include <type_traits>

namespace ffsplit {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;  // native vector: stays in registers
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;

// silu(z) = z s with s = 1 / (1 + e^-z); its derivative is s (1 + z (1 - s)).  bf16 layers: exp2 and
// a reciprocal, both within 1 ulp; fp32 layers: expf and a division.
template <typename T>
__device__ __forceinline__ float sigmoid_of(float z) {
  if (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * z));
  return 1.0f / (1.0f + expf(-z));
}

// gelu(z) = z Phi(z) and gelu'(z) = Phi(z) + z phi(z).  bf16 layers: Phi(-a) = e^(-a^2/2) / 2 * p(t),
// t = 1 / (1 + 0.3275911 a / sqrt 2), the rational form 7.1.26 of Abramowitz and Stegun (absolute
// error 1.5e-7 of erf): its exponential is phi's, so that both cost one exponential and one
// reciprocal.  fp32 layers: erfcf and expf.
template <typename T>
__device__ __forceinline__ void gelu_and_slope(float z, float& h, float& d) {
  if (sizeof(T) == 2) {
    const float a = fabsf(z);
    const float t = __builtin_amdgcn_rcpf(fmaf(a, 0.23164190f, 1.0f));
    const float e = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
    float q = fmaf(t, 0.53070271f, -0.72657601f);
    q = fmaf(t, q, 0.71070687f);
    q = fmaf(t, q, -0.14224837f);
    q = fmaf(t, q, 0.12741480f);
    const float tail = t * q * e;   // Phi(-a)
    const float cdf = z > 0.f ? 1.0f - tail : tail;
    h = z * cdf;
    d = fmaf(z * 0.39894228f, e, cdf);
  } else {
    const float cdf = 0.5f * erfcf(z * -0.70710678118654752f);   // (1 + erf cancels below 0: nothing is left at -5.6)
    h = z * cdf;
    d = cdf + z * (0.39894228040143268f * expf(-0.5f * z * z));
  }
}

// The kept derivatives of a bf16 layer in 16 bits: sign and root, sqrt(65536 |D|), in fp16.  In bf16 they would cost as much
// precision as each of the roundings that the products force on H, dU and dG (relative error of a gradient 2.9e-3, so 2.4e-3);
// as they are, fp16 would lose the factors of small tokens or weights (2.5 % at 1e-6, all of them below 3e-8).  A root has half the
// octaves: the relative error is at most 2^-10 from 2^-44 to 65504, 2^-8 down to 2^-48, and zero is left below 2^-66.  One
// beyond 65504 is kept as infinity and makes the gradient say so.  (In time 0.2 to 0.9 % of a step: 4096 tokens of 4096 x 11008
// 2563 -> 2570 us, 256 tokens 375 -> 378.)
struct Root16 { _Float16 root; };

// Storage types: float, uint16_t (bf16 bits) and Root16.
template <typename T>
__device__ __forceinline__ void load8(const void* base, int64_t at, float (&v)[8]) {
  if constexpr (std::is_same<T, float>::value) {
    const f32x4_t a = *(const f32x4_t*)((const char*)base + at * 4), b = *(const f32x4_t*)((const char*)base + at * 4 + 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
  } else if constexpr (std::is_same<T, Root16>::value) {
    const f16x8_t h = *(const f16x8_t*)((const char*)base + at * 2);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float r = (float)h[e];
      v[e] = r * 0x1p-16f * fabsf(r);
    }
  } else {
    const u32x4_t u = *(const u32x4_t*)((const char*)base + at * 2);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(u[e] << 16);
      v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
  }
}
// eight of them as loaded
template <typename T>
struct Raw8 {
  u32x4_t u[sizeof(T) / 2];
  __device__ __forceinline__ void load(const void* base, int64_t at) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) u[i] = *(const u32x4_t*)((const char*)base + at * (int)sizeof(T) + 16 * i);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const { load8<T>(u, 0, v); }
};
template <typename T>
__device__ __forceinline__ void store8(void* base, int64_t at, const float (&v)[8]) {
  if constexpr (std::is_same<T, float>::value) {
    *(f32x4_t*)((char*)base + at * 4) = f32x4_t{v[0], v[1], v[2], v[3]};
    *(f32x4_t*)((char*)base + at * 4 + 16) = f32x4_t{v[4], v[5], v[6], v[7]};
  } else if constexpr (std::is_same<T, Root16>::value) {
    f16x8_t h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (_Float16)copysignf(__builtin_amdgcn_sqrtf(fabsf(v[e]) * 65536.0f), v[e]);
    *(f16x8_t*)((char*)base + at * 2) = h;
  } else {
    *(u32x4_t*)((char*)base + at * 2) = u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                                                pack_bf16x2(v[6], v[7])};
  }
}
template <typename T>
using kept_t = typename std::conditional<std::is_same<T, float>::value, float, Root16>::type;
__device__ __forceinline__ float load1(const void* base, int64_t at, bool f32) {
  return f32 ? ((const float*)base)[at] : bf16_to_f32(((const bf16_t*)base)[at]);
}
__device__ __forceinline__ void store1(void* base, int64_t at, bool f32, float v) {
  if (f32) ((float*)base)[at] = v;
  else ((bf16_t*)base)[at] = f32_to_bf16(v);
}

// where an activation's element lies, and how many rows of it are stored
template <typename T>
__device__ __forceinline__ int64_t act_at(int64_t row, int col, int64_t ldi) {
  return sizeof(T) == 2 ? blocked_at(row, col, ldi) : row * ldi + col;
}
template <typename T, int EPI>
inline __host__ __device__ int stored_rows(const PlainArgs& p) {
  return sizeof(T) == 2 && EPI != EPI_OUT ? (p.M + 15) / 16 * 16 : p.M;
}

// EPI_GRAD: dH in v, the kept derivatives in a and b
template <typename T>
__device__ __forceinline__ void grad8(const PlainArgs& p, int64_t row, int col, const float (&v)[8], float (&a)[8], float (&b)[8]) {
  const int64_t at = act_at<T>(row, col, p.ldi);
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = col + e < p.N ? v[e] * a[e] : 0.f;
  store8<T>(p.O1, at, a);
  if (p.D2 != nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = col + e < p.N ? v[e] * b[e] : 0.f;
    store8<T>(p.O2, at, b);
  }
}

// The store step of eight columns col .. col + 7 (a multiple of 8, below n_store; EPI_OUT: below N) of
// one row.  v: the sums (EPI_GLU: the gate's, u the up columns'); which: the destination of EPI_OUT.
template <typename T, int EPI>
__device__ __forceinline__ void emit8(const PlainArgs& p, int which, int64_t row, int col, float (&v)[8], float (&u)[8]) {
  if (EPI == EPI_OUT) {
    void* const C = which ? p.C[1] : p.C[0];
    const int64_t at = row * p.ldc + col;
    if (p.resid != nullptr) {
      float r[8];
      load8<float>(p.resid, at, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    }
    const bool f32 = sizeof(T) == 4 || p.out_f32;
    if ((p.ldc & 7) == 0) {
      if (p.accumulate) {
        float w[8];
        if (f32) load8<float>(C, at, w);
        else load8<T>(C, at, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += w[e];
      }
      if (f32) store8<float>(C, at, v);
      else store8<T>(C, at, v);
    } else {   // rows that are not aligned: element by element
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < p.N) {
          const float w = p.accumulate ? load1(C, at + e, f32) : 0.f;
          store1(C, at + e, f32, v[e] + w);
        }
    }
    return;
  }
  const int64_t at = row * p.ldi + col;
  float a[8], b[8];
  if (EPI == EPI_GRAD) {
    load8<kept_t<T>>(p.D1, at, a);
    if (p.D2 != nullptr) load8<kept_t<T>>(p.D2, at, b);
    grad8<T>(p, row, col, v, a, b);
    return;
  }
  float h[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (EPI == EPI_GLU) {
      const float s = sigmoid_of<T>(v[e]);
      a[e] = v[e] * s;
      h[e] = a[e] * u[e];
      b[e] = u[e] * s * fmaf(v[e], 1.0f - s, 1.0f);
    } else {
      gelu_and_slope<T>(v[e], h[e], a[e]);
    }
    if (col + e >= p.N) { h[e] = 0.f; a[e] = 0.f; b[e] = 0.f; }
  }
  store8<T>(p.H, act_at<T>(row, col, p.ldi), h);
  if (p.D1 != nullptr) {
    store8<kept_t<T>>((void*)p.D1, at, a);
    if (EPI == EPI_GLU) store8<kept_t<T>>((void*)p.D2, at, b);
  }
}

}  // namespace ffsplit
