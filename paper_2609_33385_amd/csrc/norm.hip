// Norms before and behind an MoE block.
//
//  in   n = x * rsqrt(mean(x^2) + eps) * w, rounded to x's dtype for the gate, and
//       the unrounded n in 8 bits for the experts: e4m3 with a scale
//       s = max(amax, 2^-100) / 448 for each 128 consecutive values, rounded from the
//       fp32 product n (1 / s) (one reciprocal for 8 values of a lane; a quotient
//       each would differ at midpoints alone).
//  out  f_t = sum_j weight[t][j] O[inv_perm[t k + j]] (or a dense row f_t),
//       y_t = alpha x_t + gate o (f_t * rsqrt(mean(f_t^2) + eps) * w).
//
// One pass: a row stays in registers between its sum of squares and its
// output. All sums are fp32. TPR threads take a row, 8 consecutive values a
// thread and step (16 bytes of bf16), so 16 lanes hold a block of 128. Bound by
// memory, each value read and written once: 16384 rows of 4096 bf16 to bf16 and 8
// bits 67.6 us (5.0 TB/s, of the 5.06 that a large copy reaches), 16384 tokens of 8
// routes of 4096 258 us (5.0 TB/s). A few rows are a launch and two latencies, 3.2
// and 5.5 us of the device for 32 rows of 2048 (8 routes each).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kernels.h"
#include "oled.h"

namespace oled {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kNormThreads = 256;
constexpr int kNormMaxHidden = 16384;
constexpr float kF8Max = 448.f;                     // largest e4m3 value
constexpr float kF8Least = 7.88860905221011805e-31f; // 2^-100: least amax that is scaled

__device__ __forceinline__ uint32_t to_bf16(float f) {   // nearest even; NaN stays NaN
  const uint32_t u = __float_as_uint(f);
  return __builtin_isnan(f) ? 0x7FC0u : (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

template <class T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <>
__device__ __forceinline__ void load8<uint16_t>(const uint16_t* p, float (&v)[8]) {
  const u32x4_t r = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r[i] << 16);
    v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
  }
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float4 r = *reinterpret_cast<const float4*>(p + 4 * i);
    v[4 * i] = r.x;
    v[4 * i + 1] = r.y;
    v[4 * i + 2] = r.z;
    v[4 * i + 3] = r.w;
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  u32x4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = to_bf16(v[2 * i]) | (to_bf16(v[2 * i + 1]) << 16);
  *reinterpret_cast<u32x4_t*>(p) = r;
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// Sum over the TPR threads of a row (a row's wavefronts share a workgroup).
template <int TPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if constexpr (TPR > 64) {
    __shared__ float part[kNormThreads / 64];
    const int wave = threadIdx.x >> 6, first = threadIdx.x / TPR * (TPR / 64);
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i) v += part[first + i];
  }
  return v;
}

// 1 / sqrt(mean square + eps) of a row; 0 where that is 1 / 0 (eps 0 and a row of zeros, a
// token without routes among them): such a row stays zeros.
__device__ __forceinline__ float row_factor(float sum, int H, float eps) {
  const float m = sum / static_cast<float>(H) + eps;
  return m == 0.f ? 0.f : rsqrtf(m);
}

struct NormIn {
  const void* x;
  int64_t ldx;
  const float* w;
  float eps;
  int T, H;
  void* n;
  uint8_t* q;
  float* qs;
  uint32_t t0;   // first row of the launch
};

template <class X, int TPR, int NC>
__global__ __launch_bounds__(kNormThreads) void k_norm_in(NormIn a) {
  const uint32_t t = a.t0 + blockIdx.x * (kNormThreads / TPR) + threadIdx.x / TPR, T = a.T;
  const int sub = threadIdx.x % TPR;
  const X* row = static_cast<const X*>(a.x) + static_cast<size_t>(min(t, T - 1)) * a.ldx;
  float v[NC][8];
  float ss = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int h = 8 * (sub + TPR * c);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] = 0.f;
    if (h < a.H) load8(row + h, v[c]);
#pragma unroll
    for (int i = 0; i < 8; ++i) ss += v[c][i] * v[c][i];
  }
  if (a.w) {
    const float r = row_factor(row_sum<TPR>(ss), a.H, a.eps);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int h = 8 * (sub + TPR * c);
      if (h < a.H) {
        float w[8];
        load8(a.w + h, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] * r * w[i];
      }
    }
  }
  if (t >= T) return;
  const size_t out = static_cast<size_t>(t) * a.H;
  const int blocks = (a.H + 127) / 128;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int h = 8 * (sub + TPR * c);
    if (a.q) {   // 16 lanes hold the 128 values of a scale (those past H are zero)
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[c][i]));
#pragma unroll
      for (int d = 1; d < 16; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
      const float s = fmaxf(m, kF8Least) / kF8Max, inv = 1.f / s;
      if (h < a.H) {
        int p[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          p[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[c][4 * i] * inv, v[c][4 * i + 1] * inv, 0, false);
          p[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[c][4 * i + 2] * inv, v[c][4 * i + 3] * inv, p[i], true);
        }
        *reinterpret_cast<int2*>(a.q + out + h) = make_int2(p[0], p[1]);
        if ((sub & 15) == 0) a.qs[static_cast<size_t>(t) * blocks + h / 128] = s;
      }
    }
    if (a.n && h < a.H) store8(static_cast<X*>(a.n) + out + h, v[c]);
  }
}

struct NormOut {
  const void* f;
  const float* weights;    // [T][k]
  const int32_t* inv_perm; // [T][k], -1: no route
  int k;                   // 0: f has one row a token
  int T, H;
  const float* w;
  float eps;
  const float* gate;
  int gate_tokens;
  const void* x;
  float alpha;
  void* y;
  uint32_t t0;   // first token of the launch
};

// A token's routes in the order of its choice, one row read at a time by all of its
// threads. Routes without a row add nothing: neither their weight nor a row is read.
template <class F, class Y, int TPR, int NC>
__global__ __launch_bounds__(kNormThreads) void k_norm_out(NormOut a) {
  const uint32_t t = a.t0 + blockIdx.x * (kNormThreads / TPR) + threadIdx.x / TPR, T = a.T;
  const int sub = threadIdx.x % TPR;
  const uint32_t tt = min(t, T - 1);
  const F* f = static_cast<const F*>(a.f);
  float v[NC][8];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] = 0.f;
  if (a.k == 0) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int h = 8 * (sub + TPR * c);
      if (h < a.H) load8(f + static_cast<size_t>(tt) * a.H + h, v[c]);
    }
  } else {
    const size_t r0 = static_cast<size_t>(tt) * a.k;
    for (int j = 0; j < a.k; ++j) {
      const int pos = a.inv_perm[r0 + j];
      if (pos < 0) continue;
      const float g = a.weights[r0 + j];
      const F* row = f + static_cast<size_t>(pos) * a.H;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int h = 8 * (sub + TPR * c);
        if (h < a.H) {
          float o[8];
          load8(row + h, o);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[c][i] += g * o[i];
        }
      }
    }
  }
  if (a.w) {
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += v[c][i] * v[c][i];
    const float r = row_factor(row_sum<TPR>(ss), a.H, a.eps);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int h = 8 * (sub + TPR * c);
      if (h < a.H) {
        float w[8];
        load8(a.w + h, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] * r * w[i];
      }
    }
  }
  if (t >= T) return;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int h = 8 * (sub + TPR * c);
    if (h >= a.H) continue;
    if (a.gate) {
      float g[8];
      load8(a.gate + static_cast<size_t>(a.gate_tokens ? t / static_cast<uint32_t>(a.gate_tokens) : 0u) * a.H + h, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] *= g[i];
    }
    const size_t at = static_cast<size_t>(t) * a.H + h;
    if (a.x) {
      float x[8];
      load8(static_cast<const Y*>(a.x) + at, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] += a.alpha * x[i];
    }
    store8(static_cast<Y*>(a.y) + at, v[c]);
  }
}

// A launch takes fewer than 2^32 threads (the grid of a larger one wraps, without an error):
// more rows are several launches.
constexpr int64_t kNormGrid = 1 << 23;
template <int TPR, int NC, class Fn>
hipError_t norm_launches(int64_t T, Fn&& launch) {
  constexpr int64_t rows = kNormThreads / TPR;
  for (int64_t t0 = 0; t0 < T; t0 += kNormGrid * rows) {
    const int64_t blocks = (T - t0 + rows - 1) / rows;
    launch(std::integral_constant<int, TPR>{}, std::integral_constant<int, NC>{}, static_cast<uint32_t>(t0),
           static_cast<uint32_t>(blocks < kNormGrid ? blocks : kNormGrid));
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

// Threads of a row and steps by the row's length: a wavefront up to one step, then a
// workgroup, whose many wavefronts keep more in flight. us, a wavefront against a
// workgroup, in and out: 16384 x 512 10.2 : 16.3 and 39.6 : 80.8; 16384 x 2048 40.0 : 36.4
// and 140.8 : 141.9, 4096 x 2048 11.0 : 10.2 and 45.5 : 39.4, 32 x 2048 out 10.3 : 8.1;
// 16384 x 4096 82.1 : 67.7 and 313 : 268.
template <class Fn>
hipError_t norm_form(int T, int H, Fn&& launch) {
  if (H <= 512) return norm_launches<64, 1>(T, launch);
  if (H <= 2048) return norm_launches<256, 1>(T, launch);
  if (H <= 4096) return norm_launches<256, 2>(T, launch);
  if (H <= 8192) return norm_launches<256, 4>(T, launch);
  return norm_launches<256, 8>(T, launch);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool known(int32_t dtype) { return dtype == OLED_F32 || dtype == OLED_BF16; }

}  // namespace
}  // namespace oled

extern "C" oled_status oled_norm_in(const void* x_dev, int32_t dtype, int64_t ldx, int32_t T,
                                    int32_t H, const float* weight_dev, float eps, void* n_dev,
                                    void* q_dev, float* q_scale_dev, void* stream) {
  using namespace oled;
  if (!x_dev || (!n_dev && !q_dev) || (!q_dev != !q_scale_dev)) {
    set_noctx_error("oled_norm_in: NULL input, no output, or only one of q and its scales");
    return OLED_ERR_INVALID_ARG;
  }
  if (T < 1 || H < 1 || !known(dtype) || ldx < H || !(eps >= 0.f)) {
    set_noctx_error("oled_norm_in: T and H must be >= 1, ldx >= H, eps >= 0, dtype F32 or BF16");
    return OLED_ERR_INVALID_ARG;
  }
  if (H % 8 != 0 || H > kNormMaxHidden || ldx % 8 != 0) {
    set_noctx_error("oled_norm_in: H and ldx must be multiples of 8 and H at most 16384");
    return OLED_ERR_UNSUPPORTED;
  }
  if (!aligned16(x_dev) || !aligned16(weight_dev) || !aligned16(n_dev) || !aligned16(q_dev)) {
    set_noctx_error("oled_norm_in: x, weight, n and q must be on 16-byte boundaries");
    return OLED_ERR_INVALID_ARG;
  }
  NormIn a{x_dev, ldx, weight_dev, eps, T, H, n_dev, static_cast<uint8_t*>(q_dev), q_scale_dev, 0};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = norm_form(T, H, [&](auto tpr, auto nc, uint32_t t0, uint32_t blocks) {
    constexpr int TPR = decltype(tpr)::value, NC = decltype(nc)::value;
    a.t0 = t0;
    if (dtype == OLED_F32)
      hipLaunchKernelGGL((k_norm_in<float, TPR, NC>), dim3(blocks), dim3(kNormThreads), 0, s, a);
    else
      hipLaunchKernelGGL((k_norm_in<uint16_t, TPR, NC>), dim3(blocks), dim3(kNormThreads), 0, s, a);
  });
  if (e != hipSuccess) {
    set_noctx_error("oled_norm_in: launch failed");
    return OLED_ERR_HIP;
  }
  return OLED_OK;
}

extern "C" oled_status oled_norm_out(const void* f_dev, int32_t f_dtype, const float* weights_dev,
                                     const int32_t* inv_perm_dev, int32_t k, int32_t T, int32_t H,
                                     const float* norm_weight_dev, float eps,
                                     const float* gate_dev, int32_t gate_tokens,
                                     const void* x_dev, float residual_scale, void* y_dev,
                                     int32_t y_dtype, void* stream) {
  using namespace oled;
  if (!f_dev || !y_dev || (k > 0 && (!weights_dev || !inv_perm_dev))) {
    set_noctx_error("oled_norm_out: NULL f, y, or (k > 0) weights or inv_perm");
    return OLED_ERR_INVALID_ARG;
  }
  if (T < 1 || H < 1 || k < 0 || gate_tokens < 0 || !known(f_dtype) || !known(y_dtype) ||
      !(eps >= 0.f)) {
    set_noctx_error("oled_norm_out: T and H must be >= 1, k, gate_tokens and eps >= 0, dtypes F32 "
                    "or BF16");
    return OLED_ERR_INVALID_ARG;
  }
  if (H % 8 != 0 || H > kNormMaxHidden || k > kMaxTopK) {
    set_noctx_error("oled_norm_out: H must be a multiple of 8 up to 16384, k at most 16");
    return OLED_ERR_UNSUPPORTED;
  }
  if (!aligned16(f_dev) || !aligned16(norm_weight_dev) || !aligned16(gate_dev) ||
      !aligned16(x_dev) || !aligned16(y_dev)) {
    set_noctx_error("oled_norm_out: f, norm_weight, gate, x and y must be on 16-byte boundaries");
    return OLED_ERR_INVALID_ARG;
  }
  NormOut a{f_dev, weights_dev, inv_perm_dev, k, T, H, norm_weight_dev, eps, gate_dev,
            gate_tokens, x_dev, residual_scale, y_dev, 0};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = norm_form(T, H, [&](auto tpr, auto nc, uint32_t t0, uint32_t blocks) {
    constexpr int TPR = decltype(tpr)::value, NC = decltype(nc)::value;
    a.t0 = t0;
    const dim3 grid(blocks), block(kNormThreads);
    if (f_dtype == OLED_F32) {
      if (y_dtype == OLED_F32)
        hipLaunchKernelGGL((k_norm_out<float, float, TPR, NC>), grid, block, 0, s, a);
      else
        hipLaunchKernelGGL((k_norm_out<float, uint16_t, TPR, NC>), grid, block, 0, s, a);
    } else {
      if (y_dtype == OLED_F32)
        hipLaunchKernelGGL((k_norm_out<uint16_t, float, TPR, NC>), grid, block, 0, s, a);
      else
        hipLaunchKernelGGL((k_norm_out<uint16_t, uint16_t, TPR, NC>), grid, block, 0, s, a);
    }
  });
  if (e != hipSuccess) {
    set_noctx_error("oled_norm_out: launch failed");
    return OLED_ERR_HIP;
  }
  return OLED_OK;
}
