// Residual add, RMSNorm and rounding to 8 bits in one pass over the rows (specvla_rmsnorm_q8), and the
// rounding alone (specvla_quantize_rows). For a row x, its residual r and gain g, with C = 127 (int8) or
// 448 (e4m3):
//   s = x + r, rounded to the type it is stored in        t = s * g        amax = max |t|
//   code = round-half-even(t * C / amax)                  scale = amax / C * rsqrt(mean(s^2) + eps)
// The norm's factor is common to the row, so it cancels in the codes: they need the row's largest |t| only,
// and are decided as 64-bit arithmetic decides them. What 32 bits give is off by less than 2^-21 of itself, so
// only values that near to the middle between two codes (about one in 10,000) are done again in 64 bits.
//
// The row is in registers between the reduction and the rounding: every input is read once and every output written once.
// What a row costs beside its bytes is a chain: loads, a reduction over the CTA, the factor, the codes. So it has one
// block barrier and no 64-bit arithmetic on its way (the codes that stay open are settled afterwards by their warp alone:
// with the row's largest value in 64 bits and a second barrier, 4764 rows of 4096 took 69 us, with both but fewer
// instructions 57), 32 elements a thread (51 with 16) and the next row's copies in flight (47). 4764 x 4096 f32 with a residual
// to e4m3: 46 to 47 us, 5.4 TB/s, bound by HBM; bf16 to int8: 27 us. 27 x 4096 bf16: 4.0 us, a launch and three dependent loads. 777 x 4095
// f16, whose rows no 16-byte load fits: 10 us, one element per load.
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
  int rows, d;
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

template <int V> __device__ __forceinline__ void load_gain(const float *gain, float (&g)[V]) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const float4 v = *reinterpret_cast<const float4 *>(gain + e);
      g[e] = v.x, g[e + 1] = v.y, g[e + 2] = v.z, g[e + 3] = v.w;
    }
  } else {
    g[0] = *gain;
  }
}

// The code of v in 64 bits, as a float.
template <int CODE> __device__ __noinline__ float round_exact(double v) {
  if (CODE == CODE_I8) return (float)rint(v);
  // e4m3: three bits after the leading one, a step of 2^-9 below 2^-6
  const double a = fabs(v);
  const int e = a < 0.015625 ? -6 : ilogb(a);
  return (float)(rint(scalbn(v, 3 - e)) * scalbn(1.0, e - 3));
}
// Codes of four values t * c, of which 32 bits give less than 2^-21 too much or too little: with c a little larger and a
// little smaller (above, below) both round alike, or the value's byte in `unsure` is not 0.
template <int CODE> __device__ __forceinline__ uint32_t encode4(const float (&t)[4], float above, float below, uint32_t &unsure) {
  if (CODE == CODE_I8) {
    // 1.5 * 2^23 + f has the rounded f in its low bits
    constexpr float MAGIC = 12582912.f;
    uint32_t a[4], b[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
      a[e] = __float_as_uint(fmaf(t[e], above, MAGIC));
      b[e] = __float_as_uint(fmaf(t[e], below, MAGIC));
    }
    const uint32_t wa = __byte_perm(__byte_perm(a[0], a[1], 0x0040), __byte_perm(a[2], a[3], 0x0040), 0x5410);
    unsure = wa ^ __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    return wa;
  }
  auto pack = [&](float c) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(t[0] * c, t[1] * c), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(t[2] * c, t[3] * c), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
  };
  const uint32_t wa = pack(above);
  unsure = wa ^ pack(below);
  return wa;
}
template <int CODE> __device__ __forceinline__ unsigned char encode(float f) {
  if (CODE == CODE_I8) return (unsigned char)(signed char)(int)rintf(f);
  return (unsigned char)__nv_cvt_float_to_fp8(f, __NV_SATFINITE, __NV_E4M3);
}
// Shared memory of a CTA's reductions; words of warps that are not there stay 0.
struct Shared {
  alignas(16) float ss[2][32];
  alignas(16) uint32_t best[2][32];
  uint32_t tied[2][32];      // the warp's lanes that have its largest
  double max64[32], sq[32];
  int bad[32];
};
__device__ __forceinline__ void clear(Shared &sh) {
  for (int w = threadIdx.x; w < 64; w += blockDim.x) (&sh.ss[0][0])[w] = 0.f, (&sh.best[0][0])[w] = 0;
  __syncthreads();
}

// A row as its threads see it: thread i has the vectors i, i + threads, ... of V elements.
template <typename T> struct Row {
  const T *x, *r;            // r: NULL without a residual
  T *s;                      // NULL: the sum is not wanted
  const float *gain;         // NULL: ones
  unsigned char *q;
  float *scale;
  // element i again, from where the sum was stored (x or r may have been overwritten by it)
  __device__ __forceinline__ float sum(int i) const {
    return s ? to_float(s[i]) : r ? to_float(from_float<T>(to_float(x[i]) + to_float(r[i]))) : to_float(x[i]);
  }
  __device__ __forceinline__ float gain_at(int i) const { return gain ? gain[i] : 1.f; }
};
template <typename T>
__device__ __forceinline__ Row<T> row_of(const Args &a, long long row) {
  return {static_cast<const T *>(a.x) + row * a.ldx, a.r ? static_cast<const T *>(a.r) + row * a.ldr : nullptr,
          a.s ? static_cast<T *>(a.s) + row * a.lds : nullptr, a.gain, a.q + row * a.ldq, a.scale + row};
}

// A row outside the range of 32-bit squares and products: all of it in 64 bits. Every thread of the CTA comes here.
template <typename T, int CODE, int V>
__device__ __noinline__ void wide_row(Shared &sh, const Row<T> row, int d, float eps, int norm) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, stride = blockDim.x * V, i0 = threadIdx.x * V;
  double m = 0.0, z = 0.0;
  int bad = 0;
  for (int i = i0; i < d; i += stride)
#pragma unroll 1
    for (int e = 0; e < V; e++) {
      const float s = row.sum(i + e), g = row.gain_at(i + e);
      bad |= !(fabsf(s) < INFINITY) || !(fabsf(g) < INFINITY);
      z += (double)s * s;
      m = fmax(m, fabs((double)s * g));
    }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    z += __shfl_xor_sync(0xffffffffu, z, o);
    bad |= __shfl_xor_sync(0xffffffffu, bad, o);
    m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  if (lane == 0) sh.sq[warp] = z, sh.max64[warp] = m, sh.bad[warp] = bad;
  __syncthreads();
  double sq = 0.0, amax = 0.0;
  bad = 0;
  for (int w = 0; w < warps; w++) {
    sq += sh.sq[w];
    amax = fmax(amax, sh.max64[w]);
    bad |= sh.bad[w];
  }
  const bool none = bad || amax == 0.0;
  for (int i = i0; i < d; i += stride)
#pragma unroll 1
    for (int e = 0; e < V; e++)
      row.q[i + e] = encode<CODE>(none ? 0.f : round_exact<CODE>((double)row.sum(i + e) * row.gain_at(i + e) * top<CODE>() / amax));
  if (threadIdx.x == 0) {
    float scale = (float)(amax / top<CODE>() / (norm ? sqrt(sq / d + (double)eps) : 1.0));
    if (amax == 0.0) scale = 1.f;                      // a row of zeros
    *row.scale = bad ? __int_as_float(0x7fffffff) : scale;   // what is not finite spoils its own row only
  }
  __syncthreads();                                     // (the words of this part are read before another row's are written)
}

// A warp's codes that 32 bits leave open, in 64: open has a bit for each of a thread's first E elements; more: all that
// follow them are looked at. The row's largest |t| is that of the elements which 32 bits call the largest: the words of
// this turn say which threads have them.
template <typename T, int CODE, int V, int E>
__device__ __noinline__ void settle(const Shared &sh, int turn, const Row<T> row, int d, float top_t, uint32_t open, bool more) {
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5, stride = blockDim.x * V;
  double amax = 0.0;
  for (int w = 0; w < warps; w++) {
    if (sh.best[turn][w] != __float_as_uint(top_t)) continue;
    for (uint32_t left = sh.tied[turn][w]; left; left &= left - 1) {
      const int first = (w * 32 + __ffs(left) - 1) * V;
      for (int k = lane; first + k / V * stride < d; k += 32) {            // the lanes share that thread's elements
        const int i = first + k / V * stride + k % V;
        const float s = row.sum(i), g = row.gain_at(i);
        if (fabsf(s * g) == top_t) amax = fmax(amax, fabs((double)s * g));
      }
      __syncwarp();
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) amax = fmax(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  auto exact = [&](int k) {
    const int i = (int)threadIdx.x * V + k / V * stride + k % V;
    if (i >= d) return false;
    row.q[i] = encode<CODE>(round_exact<CODE>((double)row.sum(i) * row.gain_at(i) * top<CODE>() / amax));
    return true;
  };
  for (; open; open &= open - 1) exact(__ffs(open) - 1);
  if (more)
    for (int k = E; exact(k); k++) {}
}

// From a thread's products t (N vectors), its sum of squares and its largest |t| (as an unsigned word: a NaN is larger than
// any number) to codes and scale. rest(above, below): codes of vectors past the N first; true if one is not certain.
template <typename T, int CODE, int V, int N, typename Rest>
__device__ __forceinline__ void finish_row(Shared &sh, int turn, const Args &a, const Row<T> &row, const float (&t)[N][V], float ss,
                                           uint32_t best, bool full, int stride, int warps, Rest rest) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i0 = threadIdx.x * V;
  const uint32_t own = best;
  ss = warp_sum(ss);
  best = __reduce_max_sync(0xffffffffu, best);
  const uint32_t tied = __ballot_sync(0xffffffffu, own == best);
  if (lane == 0) sh.ss[turn][warp] = ss, sh.best[turn][warp] = best, sh.tied[turn][warp] = tied;
  __syncthreads();
  // (the other turn's words may still be read)
  ss = 0.f, best = 0;
  for (int w = 0; w < warps; w += 4) {
    const float4 vs = *reinterpret_cast<const float4 *>(&sh.ss[turn][w]);
    const uint4 vb = *reinterpret_cast<const uint4 *>(&sh.best[turn][w]);
    ss += (vs.x + vs.y) + (vs.z + vs.w);
    best = max(max(best, max(vb.x, vb.y)), max(vb.z, vb.w));
  }
  const float top_t = __uint_as_float(best);
  if (!(ss < 1e37f) || ss < 1e-30f || !(top_t < 1e37f) || top_t < 1e-30f) {       // (the same for every thread)
    wide_row<T, CODE, V>(sh, row, a.d, a.eps, a.norm);
    return;
  }
  if (threadIdx.x == 0) {
    const float scale = top_t * (1.f / (float)top<CODE>());
    *row.scale = a.norm ? scale * rsqrtf(ss / (float)a.d + a.eps) : scale;
  }
  // (a factor off by 2^-23, a product by 2^-24, the largest |t| and the others by 2^-24 each: less than 6 * 2^-24)
  const float c = __frcp_rn(top_t) * (float)top<CODE>(), above = c * (1.f + 3.6e-7f), below = c * (1.f - 3.6e-7f);
  uint32_t open = 0;                                   // (zeros past the row's end are certain)
#pragma unroll
  for (int j = 0; j < N; j++) {
    const int i = i0 + j * stride;
    if constexpr (V == 1) {
      const float u[4] = {t[j][0], 0.f, 0.f, 0.f};
      uint32_t x;
      const uint32_t w = encode4<CODE>(u, above, below, x);
      if (i < a.d) row.q[i] = (unsigned char)w;
      if (x) open |= 1u << j;
    } else {
      uint32_t w[V / 4];
#pragma unroll
      for (int k = 0; k < V / 4; k++) {
        const float u[4] = {t[j][4 * k], t[j][4 * k + 1], t[j][4 * k + 2], t[j][4 * k + 3]};
        uint32_t x;
        w[k] = encode4<CODE>(u, above, below, x);
        if (x) {
          const uint32_t bits = (x & 0xff ? 1u : 0u) | (x & 0xff00 ? 2u : 0u) | (x & 0xff0000 ? 4u : 0u) | (x >> 24 ? 8u : 0u);
          open |= bits << (j * V + 4 * k);
        }
      }
      if (full || i < a.d) {
        if constexpr (V == 4) *reinterpret_cast<uint32_t *>(row.q + i) = w[0];
        else *reinterpret_cast<uint2 *>(row.q + i) = make_uint2(w[0], w[1]);
      }
    }
  }
  const bool more = rest(above, below);
  if (__any_sync(0xffffffffu, open != 0 || more)) settle<T, CODE, V, N * V>(sh, turn, row, a.d, top_t, open, more);
}

// One row per CTA, 16 elements a thread in registers, V at a time (16 bytes of x; 1: rows that no 16-byte load fits); of
// rows of more than 16384 elements the rest is read again. Loads first and without branches: past the row's end they read
// its last elements, which are not counted.
template <typename T, int CODE, int V>
__global__ void __launch_bounds__(1024) norm_q8_kernel(const Args a) {
  constexpr int N = 16 / V;
  __shared__ Shared sh;
  clear(sh);
  pdl_wait();
  pdl_launch();
  const Row<T> row = row_of<T>(a, blockIdx.x);
  const int stride = (int)blockDim.x * V, i0 = (int)threadIdx.x * V;
  float t[N][V], ss = 0.f;
  {
    Vec<T, V> v[N], u[N];
    float g[N][V];
#pragma unroll
    for (int j = 0; j < N; j++) v[j] = *reinterpret_cast<const Vec<T, V> *>(row.x + min(i0 + j * stride, a.d - V));
    if (row.r) {
#pragma unroll
      for (int j = 0; j < N; j++) u[j] = *reinterpret_cast<const Vec<T, V> *>(row.r + min(i0 + j * stride, a.d - V));
    }
    if (a.gain) {
#pragma unroll
      for (int j = 0; j < N; j++) load_gain<V>(a.gain + min(i0 + j * stride, a.d - V), g[j]);
    }
#pragma unroll
    for (int j = 0; j < N; j++) {
      const bool in = i0 + j * stride < a.d;
#pragma unroll
      for (int e = 0; e < V; e++) {
        if (row.r) v[j].e[e] = from_float<T>(to_float(v[j].e[e]) + to_float(u[j].e[e]));
        const float s = in ? to_float(v[j].e[e]) : 0.f;
        ss = fmaf(s, s, ss);
        t[j][e] = a.gain && in ? s * g[j][e] : s;
      }
      if (row.s && in) *reinterpret_cast<Vec<T, V> *>(row.s + i0 + j * stride) = v[j];
    }
  }
  uint32_t best = 0;
#pragma unroll
  for (int j = 0; j < N; j++)
#pragma unroll
    for (int e = 0; e < V; e++) best = max(best, __float_as_uint(t[j][e]) & 0x7fffffffu);
  for (int i = i0 + N * stride; i < a.d; i += stride)
#pragma unroll 1
    for (int e = i; e < i + V; e++) {
      const T sum = row.r ? from_float<T>(to_float(row.x[e]) + to_float(row.r[e])) : row.x[e];
      const float s = to_float(sum);
      if (row.s) row.s[e] = sum;
      ss = fmaf(s, s, ss);
      best = max(best, __float_as_uint(s * row.gain_at(e)) & 0x7fffffffu);
    }
  finish_row<T, CODE, V, N>(sh, 0, a, row, t, ss, best, false, stride, blockDim.x >> 5, [&](float above, float below) {
    bool open = false;
    for (int i = i0 + N * stride; i < a.d; i += stride)
#pragma unroll 1
      for (int e = i; e < i + V; e++) {
        const float u[4] = {row.sum(e) * row.gain_at(e), 0.f, 0.f, 0.f};
        uint32_t any;
        row.q[e] = (unsigned char)encode4<CODE>(u, above, below, any);
        open |= any != 0;
      }
    return open;
  });
}

// Many rows: a CTA of NT threads takes every gridDim.x-th row, and copies the next one to shared memory as soon as the present
// one is in registers, 32 elements a thread (what is done once per row and warp weighs half of what it does at 16). A
// thread reads back what it copied itself, so the copies need no barrier.
template <typename T, int CODE, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) norm_q8_rows_kernel(const Args a) {
  constexpr int V = 16 / (int)sizeof(T), N = 32 / V, STRIDE = NT * V;
  __shared__ Shared sh;
  extern __shared__ __align__(16) unsigned char smem_raw[];   // [x, r][N][NT] of 16 bytes
  const bool full = a.d == N * STRIDE;
  const int i0 = (int)threadIdx.x * V;
  auto slot = [&](int which, int j) { return smem_raw + (uint32_t)((which * N + j) * NT + (int)threadIdx.x) * 16; };
  auto copy_row = [&](long long row) {
    const T *x = static_cast<const T *>(a.x) + row * a.ldx + i0;
    const T *r = static_cast<const T *>(a.r) + row * a.ldr + i0;
#pragma unroll
    for (int j = 0; j < N; j++)
      if (full || i0 + j * STRIDE < a.d) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(slot(0, j))),
                     "l"(x + j * STRIDE) : "memory");
        if (a.r)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(slot(1, j))),
                       "l"(r + j * STRIDE) : "memory");
      }
  };
  clear(sh);
  pdl_wait();
  pdl_launch();
  copy_row(blockIdx.x);
  int turn = 0;
  for (long long n = blockIdx.x; n < a.rows; n += gridDim.x, turn ^= 1) {
    const Row<T> row = row_of<T>(a, n);
    float t[N][V], ss = 0.f;
    uint32_t best = 0;
    asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
    for (int j = 0; j < N; j++) {
      const bool in = full || i0 + j * STRIDE < a.d;
      Vec<T, V> v = *reinterpret_cast<const Vec<T, V> *>(slot(0, j));
      if (a.r) {
        const Vec<T, V> u = *reinterpret_cast<const Vec<T, V> *>(slot(1, j));
#pragma unroll
        for (int e = 0; e < V; e++) v.e[e] = from_float<T>(to_float(v.e[e]) + to_float(u.e[e]));
      }
      if (row.s && in) *reinterpret_cast<Vec<T, V> *>(row.s + i0 + j * STRIDE) = v;
      float g[V];
      if (a.gain) load_gain<V>(a.gain + (full ? i0 + j * STRIDE : min(i0 + j * STRIDE, a.d - V)), g);
#pragma unroll
      for (int e = 0; e < V; e++) {
        const float s = in ? to_float(v.e[e]) : 0.f;
        ss = fmaf(s, s, ss);
        t[j][e] = a.gain && in ? s * g[e] : s;
        best = max(best, __float_as_uint(t[j][e]) & 0x7fffffffu);
      }
    }
    if (n + gridDim.x < a.rows) copy_row(n + gridDim.x);
    finish_row<T, CODE, V, N>(sh, turn, a, row, t, ss, best, full, STRIDE, NT / 32, [](float, float) { return false; });
  }
}

}  // namespace norm_q8
