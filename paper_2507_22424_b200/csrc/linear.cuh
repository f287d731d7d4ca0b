// Linear layer with its epilogue (specvla_linear):
//   Y[t][n] = act(sx[t] sw[n] sum_k X[t][k] W[n][k] + bias[n]) + R[t][n]
// of bf16 or f16 operands, or of int8 codes or e4m3 values with a scale per row of X and of W. int8 sums are exact (32-bit
// integers); the others are exact products added up in the tensor cores' fp32 accumulator, which cuts off instead of
// rounding, and for fp32 results in parts of K (in_parts, below). Everything after them is fp32 and is rounded once, on the
// way out.
//
// The tensor cores take W on their M axis (128 rows a tile) and the rows of X on N, so that a few rows cost a narrow
// MMA and one pass over W. A K block is 128 bytes of every row (64 or 128 elements): one swizzled row of
// shared memory and four MMAs, whatever the type.
#pragma once
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "tc_ptx.cuh"

namespace linear {

using namespace gemm_tc;

enum Kind { KIND_16 = 0, KIND_I8 = 1, KIND_E4M3 = 2 };
enum Act { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4 };

constexpr int BM = 128;                    // rows of W per tile
constexpr int KBYTES = 128;                // bytes of a row per K block
constexpr int W_BYTES = BM * KBYTES;
constexpr int MAX_TN = 256;                // rows of X per tile
constexpr int MAX_S = 8;                   // K slices (CTAs of a cluster)
constexpr int MAX_STAGES = 10;
constexpr int RING = 208 * 1024;
constexpr int SMEM = RING + 1024;
constexpr int THREADS = 192;               // warp 0 copies, warp 1 MMAs, warps 2-5 epilogue

struct Args {
  int T, N, KB;                            // K blocks
  int tn;                                  // rows per chunk = rows of an X box, a multiple of 16
  int act;
  int part;                                // K blocks per accumulator (in_parts)
  uint32_t idesc;
  int pairs;                               // N is even, and Y and R take two columns at a time
  const float *x_scale, *w_scale, *bias;   // NULL: ones / ones / zeros
  const void *res;                         // NULL: none
  void *y;
  long long ldr, ldy;
  unsigned long long wait_ns;
  int withhold;                            // test hook: > 0: the K block (withhold - 1) of every CTA is never loaded
  int *status;                             // waits that gave up add to it
};

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float as_float(__half v) { return __half2float(v); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16 *p, float v) { *p = __float2bfloat16(v); }
__device__ __forceinline__ void put(__half *p, float v) { *p = __float2half(v); }
__device__ __forceinline__ void put2(float *p, float a, float b) { *reinterpret_cast<float2 *>(p) = make_float2(a, b); }
__device__ __forceinline__ void put2(bf16 *p, float a, float b) { *reinterpret_cast<__nv_bfloat162 *>(p) = __floats2bfloat162_rn(a, b); }
__device__ __forceinline__ void put2(__half *p, float a, float b) { *reinterpret_cast<__half2 *>(p) = __floats2half2_rn(a, b); }

// v / (1 + exp(-z)) through exp(-|z|), which never overflows: small results are numbers as long as exp is one. FAST: for results
// that are rounded to 16 bits, exp2 and the reciprocal of the special-function unit (2^-22 relative) in place of expf and a
// division. tanh goes through this sum too, which cancels nothing.
template <bool FAST> __device__ __forceinline__ float sigmoid_times(float v, float z) {
  float e;
  if (FAST) {
    float r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(-1.442695041f * fabsf(z)));
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return (z < 0.f ? v * e : v) * r;
  }
  e = expf(-fabsf(z));
  return (z < 0.f ? v * e : v) / (1.f + e);
}
// GELU: max(v, 0) - m / 2 erfc(m / sqrt 2), m = |v|; negative v take the small product itself, so that nothing cancels. It is
// m p(t) exp(-m^2 / 2), t = 1 / (1 + C m), where p is a polynomial of degree 8 without a constant term, fitted to
// erfcx(m / sqrt 2) / 2 over 0 <= m <= 14 so that its largest relative error is smallest (9e-8; Lawson's reweighted least
// squares): right relative to itself, as far down as it is a number. |v| stops at 64, where the product is long 0, so that
// everything stays in range, and 0 v keeps the NaN of a NaN and of -infinity. No branch on v: 15 us instead of 11 for
// 1001 x 4331 x 128.
constexpr float GELU_C = 0.304595530f;
__device__ __forceinline__ float gelu_poly(float t) {
  float p = fmaf(t, 0.0367648005f, -0.153923899f);
  p = fmaf(p, t, 0.188323691f);
  p = fmaf(p, t, -0.0400405787f);
  p = fmaf(p, t, 0.122031376f);
  p = fmaf(p, t, 0.10302265f);
  p = fmaf(p, t, 0.122346029f);
  return fmaf(p, t, 0.12147598f) * t;
}
// For 16-bit results, two at a time: both reciprocals come from the one of their product (the special-function unit takes 8
// clocks an instruction), and the exponent keeps its roundings (a product off by 1.5e-6 of itself at most, and 3 * 2^-24 m^2 / 2 more:
// 2e-6 where f16 ends, 1e-5 at -13).
__device__ __forceinline__ void fast_gelu(float &v0, float &v1) {
  const float m[2] = {fminf(fabsf(v0), 64.f), fminf(fabsf(v1), 64.f)};
  const float d0 = fmaf(GELU_C, m[0], 1.f), d1 = fmaf(GELU_C, m[1], 1.f);
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(d0 * d1));
  const float t[2] = {r * d1, r * d0};
#pragma unroll
  for (int k = 0; k < 2; k++) {
    float &v = k ? v1 : v0;
    float e;
    asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(-0.72134752f * m[k] * m[k]));
    const float flat = 0.f * v, base = v > 0.f ? v : flat;
    v = fmaf(-(gelu_poly(t[k]) * m[k]), e, base);
  }
}
// For fp32 results the roundings of m^2 and of the exponent are put back: the product is right to ten 2^-23 of itself at
// worst. (v / 2 (1 + erf) cancels below -2: 4 % off at -5, and 0 from -5.6 on.)
__device__ __forceinline__ float exact_gelu(float v) {
  const float m = fminf(fabsf(v), 64.f);
  float t, e;
  asm("rcp.approx.f32 %0, %1;" : "=f"(t) : "f"(fmaf(GELU_C, m, 1.f)));
  constexpr float H = 0.7213475108f, HL = 9.6298e-9f;        // log2(e) / 2 = H + HL
  const float sq = m * m, y = H * sq;
  const float lost = fmaf(HL, sq, fmaf(H, fmaf(m, m, -sq), fmaf(H, sq, -y)));
  asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(-y));
  e = fmaf(e, -0.693147181f * lost, e);
  const float flat = 0.f * v, base = v > 0.f ? v : flat;
  return fmaf(-(gelu_poly(t) * m), e, base);
}
template <bool FAST, int M> __device__ __forceinline__ void activate(float (&v)[M], int act) {
  switch (act) {
    case ACT_RELU:
#pragma unroll
      for (int j = 0; j < M; j++) v[j] = v[j] < 0.f ? 0.f : v[j];         // (a NaN stays one)
      break;
    case ACT_GELU:
      if constexpr (FAST) {
#pragma unroll
        for (int j = 0; j < M; j += 2) fast_gelu(v[j], v[j + 1]);
      } else {
#pragma unroll
        for (int j = 0; j < M; j++) v[j] = exact_gelu(v[j]);
      }
      break;
    case ACT_GELU_TANH:
      // (1 + tanh z) / 2 = 1 / (1 + exp(-2 z)), z = sqrt(2 / pi) (v + 0.044715 v^3)
#pragma unroll
      for (int j = 0; j < M; j++) v[j] = sigmoid_times<FAST>(v[j], v[j] * (1.595769122f + 0.0713548163f * v[j] * v[j]));
      break;
    case ACT_SILU:
#pragma unroll
      for (int j = 0; j < M; j++) v[j] = sigmoid_times<FAST>(v[j], v[j]);
      break;
    default: break;
  }
}

// One MMA of 32 bytes of K.
template <int KIND>
__device__ __forceinline__ void mma(uint32_t d, uint64_t ad, uint64_t bd, uint32_t idesc, uint32_t acc) {
  if constexpr (KIND == KIND_16) {
    tc_mma(d, ad, bd, idesc, acc);
  } else if constexpr (KIND == KIND_I8) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(ad), "l"(bd), "r"(idesc), "r"(acc) : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(ad), "l"(bd), "r"(idesc), "r"(acc) : "memory");
  }
}
// Accumulator: fp32 (1) or int32 (2); operands: f16 0, bf16 1 / signed 8-bit 1 / e4m3 0; M, N.
inline uint32_t make_idesc(int kind, bool is_bf16, int m, int n) {
  const uint32_t fmt = kind == KIND_16 ? (is_bf16 ? 1u : 0u) : kind == KIND_I8 ? 1u : 0u;
  return ((kind == KIND_I8 ? 2u : 1u) << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <int KIND> __device__ __forceinline__ uint32_t add_acc(uint32_t a, uint32_t b) {
  return KIND == KIND_I8 ? a + b : __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
}
template <int KIND> __device__ __forceinline__ float acc_value(uint32_t r) {
  return KIND == KIND_I8 ? (float)(int)r : __uint_as_float(r);
}
__host__ __device__ constexpr int stage_bytes(int tn) { return W_BYTES + tn * KBYTES; }
__host__ __device__ constexpr int stages_of(int tn) { return RING / stage_bytes(tn) < MAX_STAGES ? RING / stage_bytes(tn) : MAX_STAGES; }
__host__ __device__ constexpr int tmem_cols(int tn) { return tn <= 32 ? 32 : tn <= 64 ? 64 : tn <= 128 ? 128 : 256; }
// The tensor cores' fp32 additions cut off, which costs a sum 0.15 * 2^-23 of its size per MMA: 4.4e-6 (root mean square, over the
// results' size) for 290 bf16 rows of 4096 in one accumulator, 12e-6 for 11008, where torch's fp32 product has 0.6e-6 and 1.2e-6. So
// for fp32 results parts of K are summed by the tensor cores, and the parts in fp32: a quarter of K each, at most 4 K blocks (16
// MMAs) in slices and 8 in pairs, 0.24e-6 and 0.47e-6 whatever K. Slices keep a part in each of as many accumulators as tensor
// memory has; pairs add every part to sums in registers, of at most PART_TN rows, while the next one is under way: 290 x 11008 x
// 4096 31.4 -> 32.2 us (parts of 4 33.9), 4096^3 100 -> 105 (115), 27 x 32064 x 4096 43.7 as before, 1001 x 4332 x 2056 in f16 22 -> 29
// (two rounds of tiles). (PART_TN 160 or 192 spill: 290 rows 36 and 45 us. 16-bit results stay as they are: their rounding
// is 2e-4 (f16) or 1.7e-3 (bf16), the cut-off a sixteenth of it at most.)
template <int KIND, typename OUT> __host__ __device__ constexpr bool in_parts() { return KIND != KIND_I8 && sizeof(OUT) == 4; }
constexpr int SLICE_PART = 4, PAIR_PART = 8;
constexpr int PART_TN = 128;

template <typename OUT> struct alignas(2 * sizeof(OUT)) Two { OUT a, b; };
// One element, or two side by side, into the low bits of r (two floats: r and r1); r keeps its value where p is false. A
// predicated load, not a branch: behind a branch, every load would wait for the one before it (1001 x 4332 x 2056 in f16:
// 54 us instead of 24).
template <int BYTES> __device__ __forceinline__ void load_if(uint32_t &r, uint32_t &r1, const void *q, bool p) {
  if constexpr (BYTES == 2)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %2, 0;\n\t@p ld.global.u16 %0, [%1];\n\t}" : "+r"(r) : "l"(q), "r"((int)p));
  else if constexpr (BYTES == 4)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %2, 0;\n\t@p ld.global.u32 %0, [%1];\n\t}" : "+r"(r) : "l"(q), "r"((int)p));
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %3, 0;\n\t@p ld.global.v2.u32 {%0, %1}, [%2];\n\t}"
                 : "+r"(r), "+r"(r1) : "l"(q), "r"((int)p));
}
__device__ __forceinline__ uint32_t pack2(bf16, float a, float b) { const __nv_bfloat162 v = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t *>(&v); }
__device__ __forceinline__ uint32_t pack2(__half, float a, float b) { const __half2 v = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t *>(&v); }
__device__ __forceinline__ float2 unpack2(bf16, uint32_t r) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&r)); }
__device__ __forceinline__ float2 unpack2(__half, uint32_t r) { return __half22float2(*reinterpret_cast<const __half2 *>(&r)); }
template <typename OUT> __device__ __forceinline__ float unpack1(uint32_t r) {
  if constexpr (sizeof(OUT) == 4) return __uint_as_float(r);
  else return unpack2(OUT{}, r).x;
}

// The residual of 16 accumulator columns (rows t0 .. t0 + 15 of the chunk) of this lane's output column n, asked for ahead of
// the accumulator. In pairs: of the row t0 + 2 p + (n & 1) two columns, r[p] (floats: r[2 p], r[2 p + 1]).
template <typename OUT>
__device__ __forceinline__ void residual16(const Args &a, uint32_t (&r)[16], int n, int t0, int T, long long row0) {
  if (!a.res) return;
  const OUT *q = static_cast<const OUT *>(a.res);
  if (a.pairs) {
    const int odd = n & 1, ne = n & ~1, left = ne < a.N ? T - t0 - odd : 0;
    q += (row0 + t0 + odd) * a.ldr + ne;
#pragma unroll
    for (int p = 0; p < 8; p++, q += 2 * a.ldr) load_if<2 * sizeof(OUT)>(r[sizeof(OUT) == 2 ? p : 2 * p], r[2 * p + 1], q, 2 * p < left);
  } else {
    const int left = n < a.N ? T - t0 : 0;
    q += (row0 + t0) * a.ldr + n;
#pragma unroll
    for (int j = 0; j < 16; j++, q += a.ldr) load_if<sizeof(OUT)>(r[j], r[j], q, j < left);
  }
}
// Asks for the residual of a tile's 128 columns from n0 in L2, long before it is added: thread i of `threads` takes rows
// i, i + threads, ...; only addresses of elements that exist are formed.
template <typename OUT>
__device__ __forceinline__ void prefetch_residual(const Args &a, int i, int threads, int n0, int T, long long row0) {
  if (!a.res || n0 >= a.N) return;
  const int last = min(n0 + BM, a.N) - 1;
  for (int t = i; t < T; t += threads) {
    const OUT *q = static_cast<const OUT *>(a.res) + (row0 + t) * a.ldr;
    for (int n = n0; n <= last; n += 128 / (int)sizeof(OUT)) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + n));
    asm volatile("prefetch.global.L2 [%0];" ::"l"(q + last));
  }
}
// Values that are not looked at before this point: without it their use moves up to the loads, and each waits for its own.
__device__ __forceinline__ void hold(uint32_t (&r)[16]) {
#pragma unroll
  for (int k = 0; k < 16; k++) asm volatile("" : "+r"(r[k]));
}
__device__ __forceinline__ void hold(float (&r)[16]) {
#pragma unroll
  for (int k = 0; k < 16; k++) asm volatile("" : "+f"(r[k]));
}
// 16 accumulator columns (rows t0 .. t0 + 15) of one output column: scales and bias. `acc` is free afterwards, for the next columns.
template <int KIND>
__device__ __forceinline__ void scale16(const Args &a, const uint32_t (&acc)[16], float (&v)[16], float sw, float b, const float *s_scale) {
  if (a.x_scale) {
#pragma unroll
    for (int j = 0; j < 16; j += 4) {
      const float4 sx = *reinterpret_cast<const float4 *>(s_scale + j);
      v[j] = fmaf(acc_value<KIND>(acc[j]), sw * sx.x, b);
      v[j + 1] = fmaf(acc_value<KIND>(acc[j + 1]), sw * sx.y, b);
      v[j + 2] = fmaf(acc_value<KIND>(acc[j + 2]), sw * sx.z, b);
      v[j + 3] = fmaf(acc_value<KIND>(acc[j + 3]), sw * sx.w, b);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 16; j++) v[j] = fmaf(acc_value<KIND>(acc[j]), sw, b);
  }
}
// Finishes and stores them. In pairs, neighbouring lanes exchange their values of every second row, so that both store two
// columns of one row: half as many stores. 16-bit results are exchanged rounded, two rows in one register; their residual,
// read in the order of the stores, goes the other way first (one exchange and one byte permutation are their own inverse).
template <typename OUT>
__device__ __forceinline__ void finish16(const Args &a, float (&v)[16], const uint32_t (&r)[16], int n, int t0, int T, long long row0) {
  activate<sizeof(OUT) == 2>(v, a.act);
  OUT *y = static_cast<OUT *>(a.y);
  if (a.pairs) {
    const int odd = n & 1, ne = n & ~1, left = ne < a.N ? T - t0 - odd : 0;
    OUT *q = y + (row0 + t0 + odd) * a.ldy + ne;
    if constexpr (sizeof(OUT) == 2) {
      const uint32_t order = odd ? 0x3276 : 0x5410;
      if (a.res) {
#pragma unroll
        for (int p = 0; p < 8; p++) {
          const float2 f = unpack2(OUT{}, __byte_perm(r[p], __shfl_xor_sync(0xffffffffu, r[p], 1), order));
          v[2 * p] += f.x;
          v[2 * p + 1] += f.y;
        }
      }
#pragma unroll
      for (int p = 0; p < 8; p++, q += 2 * a.ldy) {
        const uint32_t w = pack2(OUT{}, v[2 * p], v[2 * p + 1]);
        const uint32_t w2 = __byte_perm(w, __shfl_xor_sync(0xffffffffu, w, 1), order);
        if (2 * p < left) *reinterpret_cast<uint32_t *>(q) = w2;
      }
    } else {
#pragma unroll
      for (int p = 0; p < 8; p++, q += 2 * a.ldy) {
        const float other = __shfl_xor_sync(0xffffffffu, odd ? v[2 * p] : v[2 * p + 1], 1);
        float lo = odd ? other : v[2 * p], hi = odd ? v[2 * p + 1] : other;
        if (a.res) lo += unpack1<OUT>(r[2 * p]), hi += unpack1<OUT>(r[2 * p + 1]);
        if (2 * p < left) put2(q, lo, hi);
      }
    }
  } else {
    const int left = n < a.N ? T - t0 : 0;
    OUT *q = y + (row0 + t0) * a.ldy + n;
    if (a.res) {
#pragma unroll
      for (int j = 0; j < 16; j++) v[j] += unpack1<OUT>(r[j]);
    }
#pragma unroll
    for (int j = 0; j < 16; j++, q += a.ldy)
      if (j < left) put(q, v[j]);
  }
}

// Few rows: bound by the weights. One row by 4096 x 4096 in bf16 9.7 us (32 tiles of four CTAs; 5.1 us of weights, the rest start,
// first loads and the hand-over between CTAs), 27 x 11008 x 4096 18.2 us (86 CTAs, 5.0 TB/s).
// One tile of 128 columns by one chunk of rows per cluster of S CTAs, which share its K blocks. S = 1: finished from
// tensor memory. S > 1: every CTA leaves its partial tile in its own shared memory, and after one cluster barrier
// finishes the rows rank, rank + S, ... from all of them, in rank order (the result does not depend on timing).
template <int KIND, typename OUT>
static __global__ void __launch_bounds__(THREADS, 1)
linear_slice_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const Args a, const int S) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t s_bar[2 * MAX_STAGES + 1];
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail, s_done;
  __shared__ __align__(16) float s_scale[MAX_TN];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int stages = stages_of(a.tn), stage = stage_bytes(a.tn);
  const uint32_t bars = smem_u32(s_bar);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (MAX_STAGES + s); };
  const uint32_t acc_bar = bars + 8u * (2 * MAX_STAGES);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int tile = (int)blockIdx.x / S, rank = (int)blockIdx.x - tile * S, chunk = blockIdx.y;
  const int kb0 = (int)((long long)rank * a.KB / S), n_kb = (int)((long long)(rank + 1) * a.KB / S) - kb0;
  const long long row0 = (long long)chunk * a.tn;
  const int T = min(a.T - chunk * a.tn, a.tn);
  constexpr bool PARTS = in_parts<KIND, OUT>();
  const int width = tmem_cols(a.tn), parts = PARTS ? (n_kb + a.part - 1) / a.part : 1;
  int cols = width;                                            // a power of two
  while (PARTS && cols < parts * width) cols *= 2;
  auto fail = [&]() {
    atomicAdd(a.status, 1);
    s_fail = 1;
  };
  if (threadIdx.x == 0) {
    prefetch_tensormap(&tmW);
    prefetch_tensormap(&tmX);
    for (int s = 0; s < stages; s++) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(acc_bar, 1);
    s_fail = 0;
    s_done = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    tc_alloc(smem_u32(&s_tmem), cols);
    tc_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
  grid_dep_wait();
  grid_dep_launch();

  if (warp == 0) {
    const uint64_t pol_w = gridDim.y == 1 ? policy_evict_first() : policy_evict_last(), pol_x = policy_evict_last();
    const bool lead = elect_one();
    for (int it = 0, st = 0, ph = 1; it < n_kb; it++) {
      const bool ok = mbar_wait(empty_bar(st), ph, a.wait_ns);
      if (!__all_sync(0xffffffffu, ok)) {
        if (lead) fail();
        break;
      }
      if (lead && it != a.withhold - 1) {
        const uint32_t s = base + st * stage;
        mbar_expect_tx(full_bar(st), stage);
        tma_load_2d(s, &tmW, (kb0 + it) * KBYTES, tile * BM, full_bar(st), pol_w);
        tma_load_2d(s + W_BYTES, &tmX, (kb0 + it) * KBYTES, (int)row0, full_bar(st), pol_x);
      }
      __syncwarp();
      if (++st == stages) {
        st = 0;
        ph ^= 1;
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    const bool lead = elect_one();
    uint32_t d = tmem;
    for (int it = 0, st = 0, ph = 0, in = 0; it < n_kb; it++) {
      const bool ok = mbar_wait(full_bar(st), ph, a.wait_ns);
      if (!__all_sync(0xffffffffu, ok)) {
        if (lead) fail();
        break;
      }
      tc_fence_after();
      const uint64_t ad = smem_desc(base + st * stage), bd = smem_desc(base + st * stage + W_BYTES);
      if (lead) {
#pragma unroll
        for (int k = 0; k < KBYTES / 32; k++) mma<KIND>(d, ad + 2 * k, bd + 2 * k, a.idesc, in > 0 || k > 0);
        tc_commit(empty_bar(st));
        if (it == n_kb - 1) tc_commit(acc_bar);
      }
      __syncwarp();
      in++;
      if (PARTS && in == a.part) {
        in = 0;
        d += width;
      }
      if (++st == stages) {
        st = 0;
        ph ^= 1;
      }
    }
    __syncwarp();
  } else {
    const int et = threadIdx.x - 64, q = warp & 3;
    for (int t = et; t < a.tn; t += 128) s_scale[t] = a.x_scale && t < T ? a.x_scale[row0 + t] : 1.f;
    const int n = tile * BM + q * 32 + lane;
    const float sw = a.w_scale && n < a.N ? a.w_scale[n] : 1.f, b = a.bias && n < a.N ? a.bias[n] : 0.f;
    if (rank == 0) prefetch_residual<OUT>(a, et, 128, tile * BM, T, row0);
    if (et == 0) {                                             // one thread polls, the others sleep
      const bool ok = mbar_wait(acc_bar, 0, a.wait_ns);
      s_done = ok;
      if (!ok) fail();
    }
    asm volatile("bar.sync 1, 128;" ::: "memory");
    tc_fence_after();
    if (s_done) {
      const uint32_t ta = tmem + ((uint32_t)(q * 32) << 16);
      for (int t0 = 0; t0 < T; t0 += 16) {
        uint32_t v[16];
        tc_ld16(ta + t0, v);
        for (int p = 1; PARTS && p < parts; p++) {
          uint32_t more[16];
          tc_ld16(ta + p * width + t0, more);
          tc_wait_ld();
          hold(v);
          hold(more);
#pragma unroll
          for (int j = 0; j < 16; j++) v[j] = add_acc<KIND>(v[j], more[j]);
        }
        if (S == 1) {
          uint32_t r[16] = {};
          residual16<OUT>(a, r, n, t0, T, row0);
          tc_wait_ld();
          hold(v);
          hold(r);
          float f[16];
          scale16<KIND>(a, v, f, sw, b, s_scale + t0);
          finish16<OUT>(a, f, r, n, t0, T, row0);
        } else {
          tc_wait_ld();
#pragma unroll
          for (int j = 0; j < 16; j++)                         // (the ring is idle: every MMA has read its operands)
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(base + (uint32_t)(((t0 + j) * BM + q * 32 + lane) * 4)), "r"(v[j]) : "memory");
        }
      }
    }
  }
  if (S > 1) {
    namespace cg = cooperative_groups;
    cg::cluster_group cl = cg::this_cluster();
    __syncwarp();
    cl.sync();
    if (warp >= 2) {
      const int et = threadIdx.x - 64;
      const int c = (et & 63) * 2, n = tile * BM + c;
      const bool one = n < a.N, two = n + 1 < a.N;
      const OUT *res = static_cast<const OUT *>(a.res);
      float sw[2] = {1.f, 1.f}, b[2] = {0.f, 0.f};
      for (int e = 0; e < 2; e++)
        if (n + e < a.N) {
          if (a.w_scale) sw[e] = a.w_scale[n + e];
          if (a.bias) b[e] = a.bias[n + e];
        }
      const unsigned char *p0 = smem_raw + (base - smem_u32(smem_raw));
      // four rows at a time, so that their loads (residual, then the S partial sums) are in flight together; past the last
      // row and column the nearest element inside is read
      for (int t0 = rank + S * (et >> 6); t0 < T; t0 += 8 * S) {
        int t[4];
        Two<OUT> r[4] = {};
#pragma unroll
        for (int u = 0; u < 4; u++) t[u] = min(t0 + 2 * S * u, T - 1);
        if (res) {
#pragma unroll
          for (int u = 0; u < 4; u++) {
            const OUT *q = res + (row0 + t[u]) * a.ldr;
            if (a.pairs) r[u] = *reinterpret_cast<const Two<OUT> *>(q + min(n, a.N - 2));
            else r[u].a = q[min(n, a.N - 1)], r[u].b = q[min(n + 1, a.N - 1)];
          }
        }
        uint2 sum[4];
        for (int o = 0; o < S; o++) {
          const unsigned char *peer = cl.map_shared_rank(p0, o);
          uint2 part[4];
#pragma unroll
          for (int u = 0; u < 4; u++) part[u] = *reinterpret_cast<const uint2 *>(peer + (t[u] * BM + c) * 4);
#pragma unroll
          for (int u = 0; u < 4; u++)
            sum[u] = o == 0 ? part[u] : make_uint2(add_acc<KIND>(sum[u].x, part[u].x), add_acc<KIND>(sum[u].y, part[u].y));
        }
        float v[8];
#pragma unroll
        for (int u = 0; u < 4; u++) {
          v[2 * u] = fmaf(acc_value<KIND>(sum[u].x), sw[0] * s_scale[t[u]], b[0]);
          v[2 * u + 1] = fmaf(acc_value<KIND>(sum[u].y), sw[1] * s_scale[t[u]], b[1]);
        }
        activate<sizeof(OUT) == 2>(v, a.act);
#pragma unroll
        for (int u = 0; u < 4; u++) {
          if (!one || t0 + 2 * S * u >= T) continue;
          OUT *y = static_cast<OUT *>(a.y) + (row0 + t[u]) * a.ldy + n;
          if (res) v[2 * u] += as_float(r[u].a), v[2 * u + 1] += as_float(r[u].b);
          if (two && a.pairs) {
            put2(y, v[2 * u], v[2 * u + 1]);
          } else {
            put(y, v[2 * u]);
            if (two) put(y + 1, v[2 * u + 1]);
          }
        }
      }
    }
    __syncwarp();
    cl.sync();                                                 // nobody leaves while a peer reads its shared memory
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (s_fail) {                                                // copies may be in flight: let them land
    const uint64_t t0 = global_ns();
    while (global_ns() - t0 < 200000ull) __nanosleep(1000);
  }
  if (warp == 1) tc_dealloc(tmem, cols);
}

// ------------------------------------------------------------------------- many rows
// Tiles of 256 columns by up to 256 rows, each by a pair of CTAs: one MMA of M = 256 runs on both SMs and reads W (128
// rows) and X (half the rows) from the shared memory of the CTA that holds them, so that an SM fetches 32 KB per K block
// where a tile of its own would cost it 48 KB (L2 bounds the products, not the tensor cores). Persistent: a pair takes
// every n-th tile; the accumulator has two buffers in tensor memory, and eight warps finish one tile while the
// tensor cores work on the next. A K block of tn rows takes 256 + tn clocks, its bytes at 64 a clock and SM; its MMAs take
// 2 tn. 4764 x 22016 x 4096 in e4m3 293 us, 2.93 PFLOP/s (the tensor pipe 88 % of the time, clocks at the power limit);
// 4096^3 in bf16 93 us, 1.47 PFLOP/s; 290 x 11008 x 4096 in bf16 30 us (32 with GELU; 129 tiles on 74 pairs, bound by L2);
// the int8 head of 27 rows (32064 x 4096) 23.7 us, 5.7 TB/s. Where K is short the finishing loop counts: 2000 x 4096 x 512 in
// bf16 12.0 us, 2368 x 4096 x 128 11.7 us.
constexpr int PAIR_THREADS = 320;          // warp 0 copies, warp 1 MMAs (of the pair's first CTA), warps 2-9 epilogue
constexpr int PAIR_STAGES = 8;
__host__ __device__ constexpr int pair_stage(int tn) { return W_BYTES + tn / 2 * KBYTES; }
__host__ __device__ constexpr int pair_stages(int tn) { return RING / pair_stage(tn) < PAIR_STAGES ? RING / pair_stage(tn) : PAIR_STAGES; }

__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *tm, int x, int y, uint32_t bar, uint64_t pol) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint "
      "[%0], [%1, {%2, %3}], [%4], %5;"
      ::"r"(dst), "l"(tm), "r"(x), "r"(y), "r"(bar), "l"(pol) : "memory");
}
template <int KIND>
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t ad, uint64_t bd, uint32_t idesc, uint32_t acc) {
  if constexpr (KIND == KIND_16)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(ad), "l"(bd), "r"(idesc), "r"(acc) : "memory");
  else if constexpr (KIND == KIND_I8)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(ad), "l"(bd), "r"(idesc), "r"(acc) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(ad), "l"(bd), "r"(idesc), "r"(acc) : "memory");
}
// The barrier at this offset in both CTAs receives one arrival when every MMA issued so far has finished.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// Says that this warp has read its part of an accumulator. Relaxed: what it orders is tensor memory, which the fences before it and
// after the wait do; a release would also wait for the warp's stores of results (1000 to 3600 clocks).
__device__ __forceinline__ void arrive_peer(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

struct PairTiles {
  int tiles, chunks, raster;               // tiles of 256 columns, chunks of a.tn rows, chunks side by side
};
// Position i of the order in which tiles are taken: groups of `raster` chunks, within a group tile after tile with its
// chunks side by side, so that what runs at the same time shares W and X in L2.
__device__ __forceinline__ void tile_at(const PairTiles &p, int i, int &tile, int &chunk) {
  const int grp = i / (p.raster * p.tiles), in = i - grp * p.raster * p.tiles;
  const int width = min(p.raster, p.chunks - grp * p.raster);
  tile = in / width;
  chunk = grp * p.raster + in - tile * width;
}

template <int KIND, typename OUT>
static __global__ void __launch_bounds__(PAIR_THREADS, 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const Args a, const PairTiles p) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t s_bar[2 * PAIR_STAGES + 4];
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail, s_done[2];
  __shared__ __align__(16) float s_scale[2][MAX_TN];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int stages = pair_stages(a.tn), stage = pair_stage(a.tn);
  const uint32_t bars = smem_u32(s_bar);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (PAIR_STAGES + s); };
  auto acc_bar = [&](int b) { return bars + 8u * (2 * PAIR_STAGES + b); };         // buffer b holds a tile
  auto free_bar = [&](int b) { return bars + 8u * (2 * PAIR_STAGES + 2 + b); };    // ... has been read by both CTAs
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  uint32_t rank;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;
  const int total = p.tiles * p.chunks;
  constexpr bool PARTS = in_parts<KIND, OUT>();
  // a wait that gave up: both CTAs of the pair leave in the same way
  auto fail = [&]() {
    atomicAdd(a.status, 1);
    for (uint32_t r = 0; r < 2; r++)
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_addr(smem_u32(&s_fail), r)), "r"(1) : "memory");
  };
  if (threadIdx.x == 0) {
    prefetch_tensormap(&tmW);
    prefetch_tensormap(&tmX);
    for (int s = 0; s < stages; s++) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; b++) {
      mbar_init(acc_bar(b), 1);
      mbar_init(free_bar(b), 16);                              // the epilogue warps of both CTAs
    }
    s_fail = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cooperative_groups::this_cluster().sync();                   // the peer's barriers and tensor memory are there too
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
  grid_dep_wait();
  grid_dep_launch();

  if (warp == 0) {
    const uint64_t pol = policy_evict_last();
    const bool lead = elect_one();
    const uint32_t x_bytes = (uint32_t)(a.tn / 2 * KBYTES);
    int st = 0, ph = 1, n = 0;
    bool ok = true;
    for (int i = pair; ok && i < total; i += pairs) {
      int tile, chunk;
      tile_at(p, i, tile, chunk);
      const int yw = tile * 2 * BM + (int)rank * BM, yx = chunk * a.tn + (int)rank * (a.tn / 2);
      for (int kb = 0; kb < a.KB; kb++, n++) {
        ok = __all_sync(0xffffffffu, mbar_wait(empty_bar(st), ph, a.wait_ns));
        if (!ok) {
          if (lead) fail();
          break;
        }
        if (lead && n != a.withhold - 1) {
          const uint32_t s = base + st * stage, bar = peer_addr(full_bar(st), 0);
          if (rank == 0) mbar_expect_tx(full_bar(st), 2 * (W_BYTES + x_bytes));
          tma_load_pair(s, &tmW, kb * KBYTES, yw, bar, pol);
          tma_load_pair(s + W_BYTES, &tmX, kb * KBYTES, yx, bar, pol);
        }
        __syncwarp();
        if (++st == stages) {
          st = 0;
          ph ^= 1;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      const bool lead = elect_one();
      int st = 0, ph = 0, buf = 0, fph = 1;
      bool ok = true;
      const int per_tile = PARTS ? (a.KB + a.part - 1) / a.part : 1;
      // (tiles, or their parts of K, one after the other)
      for (int i = pair, part = 0; ok && i < total; part + 1 < per_tile ? part++ : (part = 0, i += pairs)) {
        ok = __all_sync(0xffffffffu, mbar_wait(free_bar(buf), fph, a.wait_ns));
        if (!ok) {
          if (lead) fail();
          break;
        }
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)(buf * MAX_TN);
        const int n_kb = PARTS ? min(a.part, a.KB - part * a.part) : a.KB;
        for (int kb = 0; kb < n_kb; kb++) {
          ok = __all_sync(0xffffffffu, mbar_wait(full_bar(st), ph, a.wait_ns));
          if (!ok) {
            if (lead) fail();
            break;
          }
          tc_fence_after();
          const uint64_t ad = smem_desc(base + st * stage), bd = smem_desc(base + st * stage + W_BYTES);
          if (lead) {
#pragma unroll
            for (int k = 0; k < KBYTES / 32; k++) mma_pair<KIND>(d, ad + 2 * k, bd + 2 * k, a.idesc, kb > 0 || k > 0);
            commit_pair(empty_bar(st));
            if (kb == n_kb - 1) commit_pair(acc_bar(buf));
          }
          __syncwarp();
          if (++st == stages) {
            st = 0;
            ph ^= 1;
          }
        }
        if (++buf == 2) {
          buf = 0;
          fph ^= 1;
        }
      }
    }
    __syncwarp();
  } else {
    const int et = threadIdx.x - 64, q = warp & 3, half = (warp - 2) >> 2, cols = a.tn / 2;
    int buf = 0, ph = 0;
    // every thread learns whether buffer `buf` holds its sums
    auto wait_sums = [&]() {
      if (et == 0) {
        const bool ok = mbar_wait(acc_bar(buf), ph, a.wait_ns);
        s_done[buf] = ok;
        if (!ok) fail();
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
      return s_done[buf] != 0;
    };
    auto free_sums = [&]() {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_peer(peer_addr(free_bar(buf), 0));
      if (++buf == 2) {
        buf = 0;
        ph ^= 1;
      }
    };
    for (int i = pair, tile_no = 0; i < total; i += pairs, tile_no++) {
      int tile, chunk;
      tile_at(p, i, tile, chunk);
      const long long row0 = (long long)chunk * a.tn;
      const int T = min(a.T - chunk * a.tn, a.tn), n = tile * 2 * BM + (int)rank * BM + q * 32 + lane;
      const float sw = a.w_scale && n < a.N ? a.w_scale[n] : 1.f, b = a.bias && n < a.N ? a.bias[n] : 0.f;
      const int turn = PARTS ? tile_no & 1 : buf;
      if (a.x_scale && et < a.tn) s_scale[turn][et] = et < T ? a.x_scale[row0 + et] : 1.f;
      prefetch_residual<OUT>(a, et, 256, tile * 2 * BM + (int)rank * BM, T, row0);
      const int t_begin = half * cols, t_end = min((half + 1) * cols, T);
      if constexpr (PARTS) {
        constexpr int G = PART_TN / 32;
        float sum[G][16];
        bool ok = true;
        for (int kb = 0; kb < a.KB; kb += a.part) {
          ok = wait_sums();
          if (!ok) break;
          tc_fence_after();
          const uint32_t ta = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * MAX_TN + t_begin);
#pragma unroll
          for (int g = 0; g < G; g++) {
            if (t_begin + 16 * g >= t_end) break;
            uint32_t acc[16];
            tc_ld16(ta + 16 * g, acc);
            tc_wait_ld();
            hold(acc);
#pragma unroll
            for (int j = 0; j < 16; j++) sum[g][j] = kb == 0 ? __uint_as_float(acc[j]) : sum[g][j] + __uint_as_float(acc[j]);
          }
          free_sums();
        }
        if (!ok) break;
        uint32_t next[16] = {};
        residual16<OUT>(a, next, n, t_begin, T, row0);
#pragma unroll
        for (int g = 0; g < G; g++) {
          const int t0 = t_begin + 16 * g;
          if (t0 >= t_end) break;
          uint32_t acc[16], r[16];
          float v[16];
#pragma unroll
          for (int k = 0; k < 16; k++) acc[k] = __float_as_uint(sum[g][k]);
          scale16<KIND>(a, acc, v, sw, b, s_scale[turn] + t0);
#pragma unroll
          for (int k = 0; k < 16; k++) r[k] = next[k];
          hold(v);
          hold(r);
          if (t0 + 16 < t_end) residual16<OUT>(a, next, n, t0 + 16, T, row0);
          finish16<OUT>(a, v, r, n, t0, T, row0);
        }
      } else {
        if (!wait_sums()) break;
        tc_fence_after();
        const uint32_t ta = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * MAX_TN);
        uint32_t acc[16], next[16] = {};                        // accumulator and residual, 16 rows ahead
        residual16<OUT>(a, next, n, t_begin, T, row0);
        if (t_begin < t_end) tc_ld16(ta + t_begin, acc);
        for (int t0 = t_begin; t0 < t_end; t0 += 16) {
          uint32_t r[16];
          float v[16];
          tc_wait_ld();
          hold(acc);
          scale16<KIND>(a, acc, v, sw, b, s_scale[turn] + t0);
#pragma unroll
          for (int k = 0; k < 16; k++) r[k] = next[k];
          hold(v);
          hold(r);
          if (t0 + 16 < t_end) {
            tc_ld16(ta + t0 + 16, acc);
            residual16<OUT>(a, next, n, t0 + 16, T, row0);
          }
          finish16<OUT>(a, v, r, n, t0, T, row0);
        }
        free_sums();
      }
    }
    __syncwarp();
  }
  // nobody leaves while the pair's MMAs may read its shared memory or its peer may signal it
  tc_fence_before();
  __syncthreads();
  cooperative_groups::this_cluster().sync();
  tc_fence_after();
  if (s_fail) {
    const uint64_t t0 = global_ns();
    while (global_ns() - t0 < 200000ull) __nanosleep(1000);
    cooperative_groups::this_cluster().sync();                 // (the flag is the same in both CTAs)
  }
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// ------------------------------------------------------------------------- host side
// Rows of `bytes` bytes, `ld` bytes apart: boxes of `rows` rows of 128 bytes. What lies past the matrix reads as zero.
inline bool make_map(CUtensorMap *tm, const void *p, long long n_rows, long long bytes, long long ld, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)bytes, (cuuint64_t)n_rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld};
  cuuint32_t box[2] = {KBYTES, (cuuint32_t)box_rows};
  cuuint32_t es[2] = {1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(p), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace linear
