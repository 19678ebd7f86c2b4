// Gradient kernels beside the products: backward pass of the per-token RMS norm, the norm over all
// gradients and clipping.  All of them are bound by memory traffic.
#include "grad.h"
#include "plain_epi.h"
#include "../../include/ffsplit.h"
#include <algorithm>

namespace ffsplit {

namespace {

// n = r x with r = (mean(x^2) + eps)^(-1/2), so dx = r (dn - (r x) (r mean(x dn))): two sums over the row,
// then one pass.  (r x is of order one and r mean(x dn) of the order of dn, so that the gradient is right wherever n
// is; r^3 alone leaves fp32 for tokens of 1e13 or 1e-13.)
// TPR threads per row, which keep it in registers (one read of everything): rows of up to 1024 elements in a wavefront,
// 8192 in a workgroup, where longer ones are read a second time.  4096 rows of 5120, bf16 with the residual, 294 MB: 49 us
// (6.0 TB/s) in traces, 50 to 56 a call back to back.
template <bool BF16, int TPR>
__global__ void __launch_bounds__(256) rmsnorm_backward_kernel(const float* x, const void* dn, int64_t T, int d, float eps,
                                                               const float* residual, float* dx, void* cast) {
  constexpr int NV = TPR == 64 ? 2 : 4, RPB = 256 / TPR, WPR = TPR / 64;
  __shared__ float sums[4][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int t = tid % TPR;
  for (int64_t first = (int64_t)blockIdx.x * RPB; first < T; first += (int64_t)gridDim.x * RPB) {
    const int64_t row = first + tid / TPR;
    const int64_t at = row * d;
    const bool on = row < T;
    float v[NV][8], g[NV][8];
    float s2 = 0.f, sx = 0.f;
    auto load = [&](int c, float (&a)[8], float (&b)[8]) {
      load8<float>(x, at + c, a);
      if (BF16) load8<uint16_t>(dn, at + c, b);
      else load8<float>(dn, at + c, b);
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) { v[i][e] = 0.f; g[i][e] = 0.f; }
      if (on && c < d) load(c, v[i], g[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) { s2 = fmaf(v[i][e], v[i][e], s2); sx = fmaf(v[i][e], g[i][e], sx); }
    if (TPR == 256 && on)
      for (int c = (t + NV * TPR) * 8; c < d; c += TPR * 8) {
        float a[8], b[8];
        load(c, a, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) { s2 = fmaf(a[e], a[e], s2); sx = fmaf(a[e], b[e], sx); }
      }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) { s2 += __shfl_xor(s2, o); sx += __shfl_xor(sx, o); }
    if (WPR > 1) {
      __syncthreads();   // (the sums of the row before have been read)
      if (lane == 0) { sums[wave][0] = s2; sums[wave][1] = sx; }
      __syncthreads();
      s2 = 0.f; sx = 0.f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) { s2 += sums[w][0]; sx += sums[w][1]; }
    }
    const float r = 1.0f / sqrtf(s2 / (float)d + eps);
    const float k = r * (sx / (float)d);
    auto emit = [&](int c, const float (&a)[8], const float (&b)[8]) {
      float o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (residual != nullptr) load8<float>(residual, at + c, o);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = fmaf(r, fmaf(-k, r * a[e], b[e]), o[e]);
      store8<float>(dx, at + c, o);
      if (cast != nullptr) {
        if (BF16) store8<uint16_t>(cast, at + c, o);
        else store8<float>(cast, at + c, o);
      }
    };
    if (on) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TPR) * 8;
        if (c < d) emit(c, v[i], g[i]);
      }
      if (TPR == 256)
        for (int c = (t + NV * TPR) * 8; c < d; c += TPR * 8) {
          float a[8], b[8];
          load(c, a, b);
          emit(c, a, b);
        }
    }
  }
}

template <bool BF16>
__global__ void __launch_bounds__(256) cast_kernel(const float* src, int64_t n8, void* dst) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n8; i += (int64_t)gridDim.x * 256) {
    float v[8];
    load8<float>(src, i * 8, v);
    if (BF16) store8<uint16_t>(dst, i * 8, v);
    else store8<float>(dst, i * 8, v);
  }
}

// A group of tensors whose description travels as kernel arguments, cut into chunks of 32 KiB (eight
// 16-byte loads a thread).
constexpr int GROUP = 56;
constexpr int CHUNK = 32768;
constexpr int MAX_BLOCKS = 2048;
struct Group {
  const void* src[GROUP];
  void* dst[GROUP];
  int64_t bytes[GROUP];
  int32_t first[GROUP + 1];   // first chunk of each tensor
  uint64_t f32;               // bit i: tensor i is fp32
  int32_t n;
};
static_assert(sizeof(Group) + 64 <= 4096, "kernel arguments");

__device__ __forceinline__ int tensor_of(const Group& g, int chunk) {
  int lo = 0, hi = g.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (g.first[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double wave_sum(double s) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
  return s;
}
__device__ __forceinline__ double block_sum_256(double s, double* w) {
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  return (w[0] + w[1]) + (w[2] + w[3]);
}

// Squares are formed and added in 64 bits: no overflow for any finite gradient, and the sum over 10^9
// elements is exact to far below fp32.  The conversions hide behind the loads: 541 MB in 85 us (6.3 TB/s).
__global__ void __launch_bounds__(256) grad_norm_kernel(const Group g, double* partial) {
  __shared__ double w[4];
  const int chunks = g.first[g.n];
  double s = 0.0;
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int i = tensor_of(g, c);
    const int64_t at = (int64_t)(c - g.first[i]) * CHUNK;
    const char* const src = (const char*)g.src[i] + at;
    const int left = (int)min((int64_t)CHUNK, g.bytes[i] - at);
    const bool f32 = (g.f32 >> i) & 1;
    auto add = [&](uint32_t u) {
      if (f32) {
        const double a = __uint_as_float(u);
        s = fma(a, a, s);
      } else {
        const double a = __uint_as_float(u << 16), b = __uint_as_float(u & 0xffff0000u);
        s = fma(a, a, s);
        s = fma(b, b, s);
      }
    };
    if (left == CHUNK) {
      u32x4_t v[CHUNK / 4096];
#pragma unroll
      for (int k = 0; k < CHUNK / 4096; ++k) v[k] = *(const u32x4_t*)(src + (k * 256 + threadIdx.x) * 16);
#pragma unroll
      for (int k = 0; k < CHUNK / 4096; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) add(v[k][e]);
    } else {
      const int whole = left & ~15;
      for (int o = threadIdx.x * 16; o < whole; o += 4096) {
        const u32x4_t v = *(const u32x4_t*)(src + o);
#pragma unroll
        for (int e = 0; e < 4; ++e) add(v[e]);
      }
      // the last elements of the tensor
      const int esz = f32 ? 4 : 2;
      for (int o = whole + threadIdx.x * esz; o < left; o += 256 * esz)
        add(f32 ? *(const uint32_t*)(src + o) : (uint32_t)*(const uint16_t*)(src + o));
    }
  }
  s = block_sum_256(s, w);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ void __launch_bounds__(256) grad_norm_finish_kernel(const double* partial, int n, float* norm, int32_t* nonfinite) {
  __shared__ double w[4];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) s += partial[i];
  s = block_sum_256(s, w);
  if (threadIdx.x == 0) {
    const float r = (float)sqrt(s);
    *norm = r;
    if (nonfinite != nullptr) *nonfinite = __builtin_isfinite(r) ? 0 : FFSPLIT_E_NONFINITE;
  }
}

// The chunks are walked from the last to the first: what the norm read last is still in cache.  Stores go past the caches,
// so that it stays there: 541 MB read and written in 185 us, norm and clipping together 312 -> 280.
__global__ void __launch_bounds__(256) grad_clip_kernel(const Group g, const float* norm, float max_norm) {
  const float n = *norm;
  float k = __builtin_isfinite(n) && n > max_norm ? max_norm / n : 1.0f, p = 1.0f;
  if (k < 0x1p-126f) {   // a subnormal factor has lost its last bits: in two parts, the first a power of two near 1 / n
    p = ldexpf(1.0f, -min(ilogbf(n), 126));
    k = max_norm / (n * p);
  }
  const int chunks = g.first[g.n];
  for (int r = blockIdx.x; r < chunks; r += gridDim.x) {
    const int c = chunks - 1 - r;
    const int i = tensor_of(g, c);
    const int64_t at = (int64_t)(c - g.first[i]) * CHUNK;
    const char* const src = (const char*)g.src[i] + at;
    char* const dst = (char*)g.dst[i] + at;
    if (k == 1.0f && p == 1.0f && src == dst) continue;   // in place, nothing to scale
    const int left = (int)min((int64_t)CHUNK, g.bytes[i] - at);
    const bool f32 = (g.f32 >> i) & 1;
    auto scale = [&](uint32_t u) -> uint32_t {
      if (k == 1.0f && p == 1.0f) return u;   // (a copy, NaN payloads and all)
      if (f32) return __float_as_uint(__uint_as_float(u) * p * k);
      return pack_bf16x2(__uint_as_float(u << 16) * p * k, __uint_as_float(u & 0xffff0000u) * p * k);
    };
    if (left == CHUNK) {
      u32x4_t v[CHUNK / 4096];
#pragma unroll
      for (int q = 0; q < CHUNK / 4096; ++q) v[q] = *(const u32x4_t*)(src + (q * 256 + threadIdx.x) * 16);
#pragma unroll
      for (int q = 0; q < CHUNK / 4096; ++q) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[q][e] = scale(v[q][e]);
        __builtin_nontemporal_store(v[q], (u32x4_t*)(dst + (q * 256 + threadIdx.x) * 16));
      }
    } else {
      const int whole = left & ~15;
      for (int o = threadIdx.x * 16; o < whole; o += 4096) {
        u32x4_t v = *(const u32x4_t*)(src + o);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = scale(v[e]);
        *(u32x4_t*)(dst + o) = v;
      }
      const int esz = f32 ? 4 : 2;
      for (int o = whole + threadIdx.x * esz; o < left; o += 256 * esz) {
        if (f32) *(uint32_t*)(dst + o) = scale(*(const uint32_t*)(src + o));
        else *(uint16_t*)(dst + o) = (uint16_t)scale(*(const uint16_t*)(src + o));
      }
    }
  }
}

// Calls f(group) for groups of at most GROUP non-empty tensors; chunks of a group fit 31 bits.
template <typename F>
int for_groups(const GradSet& set, F f) {
  Group g = {};
  for (int i = 0; i <= set.n; ++i) {
    if (i == set.n || g.n == GROUP) {
      if (g.n > 0 && f(g) != 0) return -1;
      g = {};
    }
    if (i == set.n) break;
    const bool one = set.n_mats == 0;
    const int64_t count = one ? set.counts[i] : set.count;
    if (count == 0) continue;
    const bool f32 = one ? set.dtypes[i] == FFSPLIT_F32 : set.f32 != 0;
    const int64_t bytes = count * (f32 ? 4 : 2);
    const int64_t chunks = (bytes + CHUNK - 1) / CHUNK;
    if (g.first[g.n] + chunks > 0x3fffffff) return -1;
    g.src[g.n] = one ? set.src[i] : set.mats[i % set.n_mats][i / set.n_mats];
    g.dst[g.n] = one ? (set.dst ? set.dst[i] : nullptr) : set.mats[i % set.n_mats][i / set.n_mats];
    g.bytes[g.n] = bytes;
    if (f32) g.f32 |= 1ull << g.n;
    g.first[g.n + 1] = g.first[g.n] + (int32_t)chunks;
    ++g.n;
  }
  return 0;
}

}  // namespace

int launch_rmsnorm_backward(const float* x, const void* dn, int64_t T, int d, float eps, int bf16, const float* residual,
                            float* dx, void* dx_cast, hipStream_t st) {
  if (T <= 0) return 0;
  // a wavefront per row up to 1024 elements (no more: see the kernel), a workgroup beyond (us with a wavefront / a workgroup, bf16, 16384 rows of
  // 512 22 / 35, 1024 40 / 45, 1536 64 / 63, 2048 99 / 91, 8192 500 / 390; 64 rows of 512 4.2 / 3.7, 8192 11 / 4.9)
  const bool wide = d > 1024;
  const int64_t blocks = wide ? T : (T + 3) / 4;
  const dim3 grid((unsigned)std::min<int64_t>(blocks, 1 << 20));
#define FFS_GO(B, N) hipLaunchKernelGGL((rmsnorm_backward_kernel<B, N>), grid, dim3(256), 0, st, x, dn, T, d, eps, residual, dx, dx_cast)
  if (bf16) { if (wide) FFS_GO(true, 256); else FFS_GO(true, 64); }
  else { if (wide) FFS_GO(false, 256); else FFS_GO(false, 64); }
#undef FFS_GO
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_cast(const float* src, int64_t n, int bf16, void* dst, hipStream_t st) {
  const int64_t n8 = n / 8;
  if (n8 <= 0) return 0;
  const dim3 grid((unsigned)std::min<int64_t>((n8 + 255) / 256, 4096));
  if (bf16) hipLaunchKernelGGL(cast_kernel<true>, grid, dim3(256), 0, st, src, n8, dst);
  else hipLaunchKernelGGL(cast_kernel<false>, grid, dim3(256), 0, st, src, n8, dst);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

size_t grad_norm_ws_bytes(int64_t n) { return (size_t)((n + GROUP - 1) / GROUP) * MAX_BLOCKS * 8 + 256; }

int launch_grad_norm(const GradSet& set, float* norm, int32_t* nonfinite, double* ws, hipStream_t st) {
  int partials = 0;
  if (for_groups(set, [&](const Group& g) {
        const int blocks = std::min(g.first[g.n], MAX_BLOCKS);
        hipLaunchKernelGGL(grad_norm_kernel, dim3(blocks), dim3(256), 0, st, g, ws + partials);
        partials += blocks;
        return hipGetLastError() == hipSuccess ? 0 : -1;
      }))
    return -1;
  hipLaunchKernelGGL(grad_norm_finish_kernel, dim3(1), dim3(256), 0, st, ws, partials, norm, nonfinite);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_grad_clip(const GradSet& set, const float* norm, float max_norm, hipStream_t st) {
  return for_groups(set, [&](const Group& g) {
    hipLaunchKernelGGL(grad_clip_kernel, dim3(std::min(g.first[g.n], MAX_BLOCKS)), dim3(256), 0, st, g, norm, max_norm);
    return hipGetLastError() == hipSuccess ? 0 : -1;
  });
}

}  // namespace ffsplit
