// Residual add, RMSNorm and rounding to 8 bits in one pass over the rows (specvla_rmsnorm_q8), and the
// rounding alone (specvla_quantize_rows). For a row x, its residual r and gain g, with C = 127 (int8) or
// 448 (e4m3):
//   s = x + r, rounded to the type it is stored in        t = s * g        amax = max |t|
//   code = round-half-even(t * C / amax)                  scale = amax / C * rsqrt(mean(s^2) + eps)
// The norm's factor is common to the row, so it cancels in the codes: they need the row's largest |t| only,
// and are decided as 64-bit arithmetic decides them. What 32 bits give is off by less than 2^-21 of itself, so
// only values that near to the middle between two codes (about one in 10,000) are done again in 64 bits.
//
// One CTA per row, the row in registers between the reduction and the rounding: every input is read once and
// every output written once. Bound by HBM at many rows, by launch and two dependent loads at few.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace norm_q8 {

enum Code { CODE_I8 = 0, CODE_E4M3 = 1 };

struct Args {
  const void *x, *r;         // [rows][ldx], [rows][ldr]; r may be NULL
  const float *gain;         // [d] or NULL: ones
  void *s;                   // [rows][lds] sum of x and r, or NULL
  unsigned char *q;          // [rows][ldq] codes
  float *scale;              // [rows]
  int d;
  long long ldx, ldr, lds, ldq;
  float eps;
  int norm;                  // 0: codes and scale of x itself
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float v) { return __float2bfloat16(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half(v); }

template <typename T, int V> struct alignas(sizeof(T) * V) Vec { T e[V]; };

template <int CODE> __device__ __forceinline__ constexpr double top() { return CODE == CODE_I8 ? 127.0 : 448.0; }

// The code of v in 64 bits, as a float.
template <int CODE> __device__ __noinline__ float round_exact(double v) {
  if (CODE == CODE_I8) return (float)rint(v);
  // e4m3: three bits after the leading one, a step of 2^-9 below 2^-6
  const double a = fabs(v);
  const int e = a < 0.015625 ? -6 : ilogb(a);
  return (float)(rint(scalbn(v, 3 - e)) * scalbn(1.0, e - 3));
}
// Codes of two values that are off by less than 2^-21 of themselves; true: both are certain, since the values a
// little above and a little below round alike.
constexpr float ABOVE = 1.f + 4.76837158e-7f, BELOW = 1.f - 4.76837158e-7f;     // 1 +- 2^-21
template <int CODE> __device__ __forceinline__ bool encode2(float f0, float f1, uint16_t &codes) {
  if (CODE == CODE_I8) {
    // 1.5 * 2^23 + f has the rounded f in its low bits
    constexpr float MAGIC = 12582912.f;
    const uint32_t a0 = __float_as_uint(fmaf(f0, ABOVE, MAGIC)), b0 = __float_as_uint(fmaf(f0, BELOW, MAGIC));
    const uint32_t a1 = __float_as_uint(fmaf(f1, ABOVE, MAGIC)), b1 = __float_as_uint(fmaf(f1, BELOW, MAGIC));
    codes = (uint16_t)__byte_perm(a0, a1, 0x0040);
    return a0 == b0 && a1 == b1;
  }
  const __nv_fp8x2_storage_t a = __nv_cvt_float2_to_fp8x2(make_float2(f0 * ABOVE, f1 * ABOVE), __NV_SATFINITE, __NV_E4M3);
  const __nv_fp8x2_storage_t b = __nv_cvt_float2_to_fp8x2(make_float2(f0 * BELOW, f1 * BELOW), __NV_SATFINITE, __NV_E4M3);
  codes = a;
  return a == b;
}
template <int CODE> __device__ __forceinline__ unsigned char encode(float f) {
  if (CODE == CODE_I8) return (unsigned char)(signed char)(int)rintf(f);
  return (unsigned char)__nv_cvt_float_to_fp8(f, __NV_SATFINITE, __NV_E4M3);
}
// Maximum in which a NaN wins.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Vectors of a row that a thread keeps in registers (16 elements; 1024 threads leave 64 registers each): what
// does not fit, rows of more than 16384 elements, is read again.
__host__ __device__ constexpr int cached(int V) { return 16 / V; }

// V elements at a time (16 bytes of x; 1: rows that no 16-byte load fits).
template <typename T, int CODE, int V>
__global__ void __launch_bounds__(1024) norm_q8_kernel(const Args a) {
  constexpr int CACHE = cached(V);
  pdl_wait();
  pdl_launch();
  const long long row = blockIdx.x;
  const T *x = static_cast<const T *>(a.x) + row * a.ldx;
  const T *r = a.r ? static_cast<const T *>(a.r) + row * a.ldr : nullptr;
  T *so = a.s ? static_cast<T *>(a.s) + row * a.lds : nullptr;
  unsigned char *q = a.q + row * a.ldq;
  const int stride = (int)blockDim.x * V, i0 = (int)threadIdx.x * V;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;

  auto load_sum = [&](int i, float (&s)[V]) {
    const Vec<T, V> vx = *reinterpret_cast<const Vec<T, V> *>(x + i);
#pragma unroll
    for (int e = 0; e < V; e++) s[e] = to_float(vx.e[e]);
    if (r) {
      const Vec<T, V> vr = *reinterpret_cast<const Vec<T, V> *>(r + i);
#pragma unroll
      for (int e = 0; e < V; e++) s[e] = to_float(from_float<T>(s[e] + to_float(vr.e[e])));
    }
  };
  auto load_gain = [&](int i, float (&g)[V]) {
#pragma unroll
    for (int e = 0; e < V; e++) g[e] = 1.f;
    if (!a.gain) return;
    if constexpr (V % 4 == 0) {
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        const float4 v = *reinterpret_cast<const float4 *>(a.gain + i + e);
        g[e] = v.x, g[e + 1] = v.y, g[e + 2] = v.z, g[e + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < V; e++) g[e] = a.gain[i + e];
    }
  };
  auto store_sum = [&](int i, const float (&s)[V]) {
    if (!so) return;
    Vec<T, V> v;
#pragma unroll
    for (int e = 0; e < V; e++) v.e[e] = from_float<T>(s[e]);
    *reinterpret_cast<Vec<T, V> *>(so + i) = v;
  };

  // ---- the row's sum of squares and its largest |t|, in 32 bits
  float ct[CACHE][V];
  float ss = 0.f, best = 0.f;
  auto take = [&](const float (&s)[V], const float (&g)[V], float (&t)[V]) {
#pragma unroll
    for (int e = 0; e < V; e++) {
      t[e] = s[e] * g[e];
      ss = fmaf(s[e], s[e], ss);
      best = max_nan(best, fabsf(t[e]));
    }
  };
  {
    float cs[CACHE][V], cg[CACHE][V];
#pragma unroll
    for (int j = 0; j < CACHE; j++) {
      const int i = i0 + j * stride;
#pragma unroll
      for (int e = 0; e < V; e++) cs[j][e] = cg[j][e] = 0.f;
      if (i < a.d) {
        load_sum(i, cs[j]);
        load_gain(i, cg[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < CACHE; j++) {
      if (i0 + j * stride < a.d) store_sum(i0 + j * stride, cs[j]);
      take(cs[j], cg[j], ct[j]);
    }
  }
  for (int i = i0 + CACHE * stride; i < a.d; i += stride) {
    float s[V], g[V], t[V];
    load_sum(i, s);
    load_gain(i, g);
    store_sum(i, s);
    take(s, g, t);
  }
  __shared__ float s_ss[32], s_best[32];
  __shared__ unsigned long long s_amax;
  __shared__ double s_max[32], s_sq[32];
  __shared__ int s_bad[32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    ss += __shfl_xor_sync(0xffffffffu, ss, o);
    best = max_nan(best, __shfl_xor_sync(0xffffffffu, best, o));
  }
  if (lane == 0) s_ss[warp] = ss, s_best[warp] = best;
  if (threadIdx.x == 0) s_amax = 0;
  __syncthreads();
  ss = lane < warps ? s_ss[lane] : 0.f;
  best = lane < warps ? s_best[lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    ss += __shfl_xor_sync(0xffffffffu, ss, o);
    best = max_nan(best, __shfl_xor_sync(0xffffffffu, best, o));
  }
  double sq = ss, amax = 0.0;

  // element i of the row again: the sum from where it was stored (x or r may have been overwritten by it)
  auto sum_at = [&](int i) { return so ? to_float(so[i]) : r ? to_float(from_float<T>(to_float(x[i]) + to_float(r[i]))) : to_float(x[i]); };
  auto gain_at = [&](int i) { return a.gain ? a.gain[i] : 1.f; };
  auto t_of = [&](int i, float (&t)[V]) {
    float g[V];
    load_gain(i, g);
#pragma unroll
    for (int e = 0; e < V; e++) t[e] = sum_at(i + e) * g[e];
  };

  // ---- rows outside the range of 32-bit squares and products (the same for every thread): all in 64 bits
  const bool wide = !(ss < 1e37f) || ss < 1e-30f || !(best < 1e37f) || best < 1e-30f;
  bool finite = true;
  if (wide) {
    double m = 0.0, z = 0.0;
    int bad = 0;
    for (int i = i0; i < a.d; i += stride)
#pragma unroll
      for (int e = 0; e < V; e++) {
        const float s = sum_at(i + e), g = gain_at(i + e);
        bad |= !(fabsf(s) < INFINITY) || !(fabsf(g) < INFINITY);
        z += (double)s * s;
        m = fmax(m, fabs((double)s * g));
      }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      z += __shfl_xor_sync(0xffffffffu, z, o);
      m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
      bad |= __shfl_xor_sync(0xffffffffu, bad, o);
    }
    if (lane == 0) s_sq[warp] = z, s_max[warp] = m, s_bad[warp] = bad;
    __syncthreads();
    sq = 0.0, bad = 0;
    for (int w = 0; w < warps; w++) {
      sq += s_sq[w];
      amax = fmax(amax, s_max[w]);
      bad |= s_bad[w];
    }
    finite = !bad;
  } else {
    // the largest product in 64 bits: among those that 32 bits call the largest
    auto tie = [&](int i, const float (&t)[V]) {
#pragma unroll
      for (int e = 0; e < V; e++)
        if (fabsf(t[e]) == best)
          atomicMax(&s_amax, (unsigned long long)__double_as_longlong(fabs((double)sum_at(i + e) * gain_at(i + e))));
    };
#pragma unroll
    for (int j = 0; j < CACHE; j++)
      if (i0 + j * stride < a.d) tie(i0 + j * stride, ct[j]);
    for (int i = i0 + CACHE * stride; i < a.d; i += stride) {
      float t[V];
      t_of(i, t);
      tie(i, t);
    }
    __syncthreads();
    amax = __longlong_as_double((long long)s_amax);
  }
  if (threadIdx.x == 0) {
    double scale = amax / top<CODE>();
    if (a.norm) scale = scale / sqrt(sq / a.d + (double)a.eps);
    if (amax == 0.0) scale = 1.0;                      // a row of zeros
    a.scale[row] = finite ? (float)scale : __int_as_float(0x7fffffff);   // a NaN spoils its own row only
  }

  // ---- codes
  const bool none = !finite || amax == 0.0;
  const float c = (float)top<CODE>() / (float)amax;
  auto exact = [&](int i) -> unsigned char {
    return encode<CODE>(none ? 0.f : round_exact<CODE>((double)sum_at(i) * gain_at(i) * top<CODE>() / amax));
  };
  auto emit = [&](int i, const float (&t)[V]) {
    Vec<unsigned char, V> o;
    bool sure = !wide;
    if constexpr (V > 1) {
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        uint16_t two;
        sure &= encode2<CODE>(t[e] * c, t[e + 1] * c, two);
        o.e[e] = (unsigned char)two;
        o.e[e + 1] = (unsigned char)(two >> 8);
      }
    } else {
      uint16_t two;
      sure &= encode2<CODE>(t[0] * c, 0.f, two);
      o.e[0] = (unsigned char)two;
    }
    if (!sure) {
#pragma unroll 1
      for (int e = 0; e < V; e++) q[i + e] = exact(i + e);
    } else {
      *reinterpret_cast<Vec<unsigned char, V> *>(q + i) = o;
    }
  };
#pragma unroll
  for (int j = 0; j < CACHE; j++)
    if (i0 + j * stride < a.d) emit(i0 + j * stride, ct[j]);
  for (int i = i0 + CACHE * stride; i < a.d; i += stride) {
    float t[V];
    t_of(i, t);
    emit(i, t);
  }
}

}  // namespace norm_q8
