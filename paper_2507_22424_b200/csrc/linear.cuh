// Linear layer with its epilogue (specvla_linear):
//   Y[t][n] = act(sx[t] sw[n] sum_k X[t][k] W[n][k] + bias[n]) + R[t][n]
// of bf16 or f16 operands, or of int8 codes or e4m3 values with a scale per row of X and of W. Products are exact
// in the accumulator's type (int8: 32-bit integers; else fp32), everything after them is fp32 and is rounded once,
// on the way out.
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

#define SV_ERR_LINEAR_EMPTY 11
#define SV_ERR_LINEAR_FULL 12
#define SV_ERR_LINEAR_ACC 13

struct Args {
  int T, N, KB;                            // K blocks
  int tn;                                  // rows per chunk = rows of an X box, a multiple of 16
  int act;
  uint32_t idesc;
  int pairs;                               // Y (and R) take two columns at a time
  const float *x_scale, *w_scale, *bias;   // NULL: ones / ones / zeros
  const void *res;                         // NULL: none
  void *y;
  long long ldr, ldy;
  unsigned long long wait_ns;
  int withhold;                            // test hook: > 0: the K block (withhold - 1) of every CTA is never loaded
  int *status;
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
__device__ __forceinline__ float2 get2(const float *p) { return *reinterpret_cast<const float2 *>(p); }
__device__ __forceinline__ float2 get2(const bf16 *p) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(p)); }
__device__ __forceinline__ float2 get2(const __half *p) { return __half22float2(*reinterpret_cast<const __half2 *>(p)); }

__device__ __forceinline__ float activate(float v, int act) {
  switch (act) {
    case ACT_RELU: return v < 0.f ? 0.f : v;                               // (a NaN stays one)
    case ACT_GELU: return 0.5f * v * (1.f + erff(v * 0.70710678f));
    case ACT_GELU_TANH: return 0.5f * v * (1.f + tanhf(0.79788456f * (v + 0.044715f * v * v * v)));
    case ACT_SILU: return v / (1.f + expf(-v));
    default: return v;
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
template <int KIND> __device__ __forceinline__ float acc_value(uint32_t r) {
  return KIND == KIND_I8 ? (float)(int)r : __uint_as_float(r);
}
__host__ __device__ constexpr int stage_bytes(int tn) { return W_BYTES + tn * KBYTES; }
__host__ __device__ constexpr int stages_of(int tn) { return RING / stage_bytes(tn) < MAX_STAGES ? RING / stage_bytes(tn) : MAX_STAGES; }
__host__ __device__ constexpr int tmem_cols(int tn) { return tn <= 32 ? 32 : tn <= 64 ? 64 : tn <= 128 ? 128 : 256; }

// Finishes and stores 16 accumulator columns (rows t0 .. t0 + 15 of the chunk) of this lane's output column n: v is
// the accumulator. In pairs, neighbouring lanes exchange a value each per two rows, so that both store two columns
// of one row: half as many stores.
template <int KIND, typename OUT>
__device__ __forceinline__ void finish16(const Args &a, const uint32_t (&v)[16], int n, int t0, int T, long long row0,
                                         float sw, float b, const float *s_scale) {
  OUT *y = static_cast<OUT *>(a.y);
  const OUT *res = static_cast<const OUT *>(a.res);
  const bool odd = n & 1;
  if (a.pairs) {
    const int ne = n & ~1;
    const bool one = ne < a.N, two = ne + 1 < a.N;
    float2 rr[8];
#pragma unroll
    for (int p = 0; p < 8; p++) {
      const int t = t0 + 2 * p + (odd ? 1 : 0);
      rr[p] = make_float2(0.f, 0.f);
      if (res && t < T && one) {
        const OUT *q = res + (row0 + t) * a.ldr + ne;
        if (two) rr[p] = get2(q);
        else rr[p].x = as_float(*q);
      }
    }
#pragma unroll
    for (int p = 0; p < 8; p++) {
      const float y0 = activate(acc_value<KIND>(v[2 * p]) * (sw * s_scale[t0 + 2 * p]) + b, a.act);
      const float y1 = activate(acc_value<KIND>(v[2 * p + 1]) * (sw * s_scale[t0 + 2 * p + 1]) + b, a.act);
      const float other = __shfl_xor_sync(0xffffffffu, odd ? y0 : y1, 1);
      const int t = t0 + 2 * p + (odd ? 1 : 0);
      if (t < T && one) {
        OUT *q = y + (row0 + t) * a.ldy + ne;
        const float lo = (odd ? other : y0) + rr[p].x, hi = (odd ? y1 : other) + rr[p].y;
        if (two) put2(q, lo, hi);
        else put(q, lo);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 16; j++) {
      const int t = t0 + j;
      if (t < T && n < a.N) {
        float o = activate(acc_value<KIND>(v[j]) * (sw * s_scale[t]) + b, a.act);
        if (res) o += as_float(res[(row0 + t) * a.ldr + n]);
        put(y + (row0 + t) * a.ldy + n, o);
      }
    }
  }
}

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
  __shared__ float s_scale[MAX_TN];
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
  const int cols = tmem_cols(a.tn);
  auto fail = [&](int code) {
    atomicExch(a.status, code);
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
        if (lead) fail(SV_ERR_LINEAR_EMPTY);
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
    for (int it = 0, st = 0, ph = 0; it < n_kb; it++) {
      const bool ok = mbar_wait(full_bar(st), ph, a.wait_ns);
      if (!__all_sync(0xffffffffu, ok)) {
        if (lead) fail(SV_ERR_LINEAR_FULL);
        break;
      }
      tc_fence_after();
      const uint64_t ad = smem_desc(base + st * stage), bd = smem_desc(base + st * stage + W_BYTES);
      if (lead) {
#pragma unroll
        for (int k = 0; k < KBYTES / 32; k++) mma<KIND>(tmem, ad + 2 * k, bd + 2 * k, a.idesc, it > 0 || k > 0);
        tc_commit(empty_bar(st));
        if (it == n_kb - 1) tc_commit(acc_bar);
      }
      __syncwarp();
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
    if (et == 0) {                                             // one thread polls, the others sleep
      const bool ok = mbar_wait(acc_bar, 0, a.wait_ns);
      s_done = ok;
      if (!ok) fail(SV_ERR_LINEAR_ACC);
    }
    asm volatile("bar.sync 1, 128;" ::: "memory");
    tc_fence_after();
    if (s_done) {
      const uint32_t ta = tmem + ((uint32_t)(q * 32) << 16);
      for (int t0 = 0; t0 < T; t0 += 16) {
        uint32_t v[16];
        tc_ld16(ta + t0, v);
        tc_wait_ld();
        if (S == 1) {
          finish16<KIND, OUT>(a, v, n, t0, T, row0, sw, b, s_scale);
        } else {
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
      float sw[2] = {1.f, 1.f}, b[2] = {0.f, 0.f};
      for (int e = 0; e < 2; e++)
        if (n + e < a.N) {
          if (a.w_scale) sw[e] = a.w_scale[n + e];
          if (a.bias) b[e] = a.bias[n + e];
        }
      const unsigned char *p0 = smem_raw + (base - smem_u32(smem_raw));
      for (int t = rank + S * (et >> 6); t < T && one; t += 2 * S) {
        float v[2];
        if (KIND == KIND_I8) {
          int s[2] = {0, 0};
          for (int r = 0; r < S; r++) {
            const int2 p = *reinterpret_cast<const int2 *>(cl.map_shared_rank(p0, r) + (t * BM + c) * 4);
            s[0] += p.x, s[1] += p.y;
          }
          v[0] = (float)s[0], v[1] = (float)s[1];
        } else {
          v[0] = v[1] = 0.f;
          for (int r = 0; r < S; r++) {
            const float2 p = *reinterpret_cast<const float2 *>(cl.map_shared_rank(p0, r) + (t * BM + c) * 4);
            v[0] += p.x, v[1] += p.y;
          }
        }
        const OUT *res = static_cast<const OUT *>(a.res);
        OUT *y = static_cast<OUT *>(a.y) + (row0 + t) * a.ldy + n;
        for (int e = 0; e < 2; e++) {
          v[e] = activate(v[e] * (sw[e] * s_scale[t]) + b[e], a.act);
          if (res && n + e < a.N) v[e] += as_float(res[(row0 + t) * a.ldr + n + e]);
        }
        if (two && a.pairs) {
          put2(y, v[0], v[1]);
        } else {
          put(y, v[0]);
          if (two) put(y + 1, v[1]);
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
