// Residual add, RMSNorm and rounding to 8 bits in one pass over the rows (specvla_rmsnorm_q8), and the
// rounding alone (specvla_quantize_rows). For a row x, its residual r and gain g, with C = 127 (int8) or
// 448 (e4m3):
//   s = x + r, rounded to the type it is stored in        t = s * g        amax = max |t|
//   code = round-half-even(t * C / amax)                  scale = amax / C * rsqrt(mean(s^2) + eps)
// The norm's factor is common to the row, so it cancels in the codes: they need the row's largest |t| only,
// and are decided as 64-bit arithmetic decides them. A product in 32 bits is off by at most 2^-22 of itself,
// so only values that near to the middle between two codes (about one in 10,000) are done again in 64 bits.
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
template <int CODE> __device__ __forceinline__ float round_exact(double v) {
  if (CODE == CODE_I8) return (float)rint(v);
  // e4m3: three bits after the leading one, a step of 2^-9 below 2^-6
  const double a = fabs(v);
  const int e = a < 0.015625 ? -6 : ilogb(a);
  return (float)(rint(scalbn(v, 3 - e)) * scalbn(1.0, e - 3));
}
// Whether f, off by at most 2^-22 of itself, may round to another code than the value it stands for.
template <int CODE> __device__ __forceinline__ bool near_border(float f) {
  if (CODE == CODE_I8) return fabsf(f - rintf(f)) > 0.49995f;           // 127 * 2^-22 = 3e-5
  const float g = f * 512.f;                                            // subnormal codes: steps of 2^-9
  if (fabsf(f) < 0.0157f && fabsf(g - rintf(g)) > 0.49999f) return true;
  return ((__float_as_uint(f) & 0xfffffu) - 0x7fff0u) <= 0x20u;         // 20 bits below the kept ones, half = 0x80000
}
template <int CODE> __device__ __forceinline__ unsigned char encode(float f) {
  if (CODE == CODE_I8) return (unsigned char)(signed char)(int)rintf(f);
  return (unsigned char)__nv_cvt_float_to_fp8(f, __NV_SATFINITE, __NV_E4M3);
}

// Vectors of a row that a thread keeps in registers (16 elements; 1024 threads leave 64 registers each): what
// does not fit, rows of more than 16384 elements, is read again.
__host__ __device__ constexpr int cached(int V) { return V == 1 ? 4 : 16 / V; }

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

  // ---- the row's sum of squares and its largest |t|: compared in 32 bits, equal ones in 64
  float cs[CACHE][V], cg[CACHE][V];
  float ss = 0.f, best = 0.f, bs = 0.f, bg = 0.f;
  bool odd = false;                                    // a product that 32 bits do not hold
  auto take = [&](const float (&s)[V], const float (&g)[V]) {
#pragma unroll
    for (int e = 0; e < V; e++) {
      const float t = fabsf(s[e] * g[e]);
      ss = fmaf(s[e], s[e], ss);
      odd |= !(t < INFINITY);
      if (t > best || (t == best && fabs((double)s[e] * g[e]) > fabs((double)bs * bg))) best = t, bs = s[e], bg = g[e];
    }
  };
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
    const int i = i0 + j * stride;
    if (i < a.d) store_sum(i, cs[j]);
    take(cs[j], cg[j]);
  }
  for (int i = i0 + CACHE * stride; i < a.d; i += stride) {
    float s[V], g[V];
    load_sum(i, s);
    load_gain(i, g);
    store_sum(i, s);
    take(s, g);
  }
  __shared__ float s_ss[32];
  __shared__ double s_max[32], s_sq[32];
  __shared__ int s_odd[32];
  double amax = fabs((double)bs * bg);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    ss += __shfl_xor_sync(0xffffffffu, ss, o);
    amax = fmax(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  }
  odd = __any_sync(0xffffffffu, odd);
  if (lane == 0) {
    s_ss[warp] = ss;
    s_max[warp] = amax;
    s_odd[warp] = odd;
  }
  __syncthreads();
  ss = lane < warps ? s_ss[lane] : 0.f;
  amax = lane < warps ? s_max[lane] : 0.0;
  odd = __any_sync(0xffffffffu, lane < warps && s_odd[lane]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    ss += __shfl_xor_sync(0xffffffffu, ss, o);
    amax = fmax(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  }
  double sq = ss;

  // the sums again, from registers or from where they were stored
  auto again = [&](int j, int i, float (&s)[V], float (&g)[V]) {
    if (j < CACHE) {
#pragma unroll
      for (int c = 0; c < CACHE; c++)
        if (c == j) {
#pragma unroll
          for (int e = 0; e < V; e++) s[e] = cs[c][e], g[e] = cg[c][e];
        }
      return;
    }
    if (so) {                                          // (x or r may have been overwritten by it)
      const Vec<T, V> v = *reinterpret_cast<const Vec<T, V> *>(so + i);
#pragma unroll
      for (int e = 0; e < V; e++) s[e] = to_float(v.e[e]);
    } else {
      load_sum(i, s);
    }
    load_gain(i, g);
  };

  // ---- rows outside the range of 32-bit squares and products (the same for every thread): all in 64 bits
  const bool wide = odd || !(sq < 1e37) || sq < 1e-30 || amax < 1e-30;
  bool finite = true;
  if (wide) {
    double m = 0.0, z = 0.0;
    int bad = 0;
    for (int j = 0, i = i0; i < a.d; j++, i += stride) {
      float s[V], g[V];
      again(j, i, s, g);
#pragma unroll
      for (int e = 0; e < V; e++) {
        bad |= !(fabsf(s[e]) < INFINITY) || !(fabsf(g[e]) < INFINITY);
        z += (double)s[e] * s[e];
        m = fmax(m, fabs((double)s[e] * g[e]));
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      z += __shfl_xor_sync(0xffffffffu, z, o);
      m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
      bad |= __shfl_xor_sync(0xffffffffu, bad, o);
    }
    __syncthreads();                                   // (everyone has read the first round's values)
    if (lane == 0) {
      s_sq[warp] = z;
      s_max[warp] = m;
      s_odd[warp] = bad;
    }
    __syncthreads();
    sq = 0.0, amax = 0.0, bad = 0;
    for (int w = 0; w < warps; w++) {
      sq += s_sq[w];
      amax = fmax(amax, s_max[w]);
      bad |= s_odd[w];
    }
    finite = !bad;
  }
  if (threadIdx.x == 0) {
    double scale = amax / top<CODE>();
    if (a.norm) scale = scale / sqrt(sq / a.d + (double)a.eps);
    if (amax == 0.0) scale = 1.0;                      // a row of zeros
    a.scale[row] = finite ? (float)scale : __int_as_float(0x7fffffff);   // a NaN spoils its own row only
  }

  // ---- codes
  const bool none = !finite || amax == 0.0;
  const float c = (float)(top<CODE>() / amax);
  auto code_of = [&](float s, float g) -> unsigned char {
    float f = s * g * c;
    if (wide || near_border<CODE>(f)) f = none ? 0.f : round_exact<CODE>((double)s * g * top<CODE>() / amax);
    return encode<CODE>(f);
  };
  auto emit = [&](int i, const float (&s)[V], const float (&g)[V]) {
    Vec<unsigned char, V> o;
#pragma unroll
    for (int e = 0; e < V; e++) o.e[e] = code_of(s[e], g[e]);
    *reinterpret_cast<Vec<unsigned char, V> *>(q + i) = o;
  };
#pragma unroll
  for (int j = 0; j < CACHE; j++)
    if (i0 + j * stride < a.d) emit(i0 + j * stride, cs[j], cg[j]);
  for (int i = i0 + CACHE * stride; i < a.d; i += stride) {
    float s[V], g[V];
    again(CACHE, i, s, g);
    emit(i, s, g);
  }
}

}  // namespace norm_q8
