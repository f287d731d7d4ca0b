// Verification of drafted tokens by given random numbers (specvla_verify_sampled, specvla_verify_tree_sampled).
//
// p_i = softmax(logits_i / temperature) over the ids [lo, hi). The walk starts at the root; at a row a, with
// beta = 0 and S = 1, its children c are looked at in ascending order, x = token of c:
//   draft probabilities q_a given:  r(x) = max(p_a(x) - beta q_a(x), 0);  c is accepted when u_c q_a(x) S < r(x);
//                                   else beta += S, S = sum over all ids of max(p_a - beta q_a, 0)
//   none given:                     r = p_a without the tokens refused at a, S = its sum;  accepted when u_c S < r(x)
// The walk goes on at an accepted child. Where no child is accepted, the token after the path is the first id
// whose cumulative r exceeds u_0 times its sum. (Multi-round speculative sampling: tokens have the target's
// distribution when siblings were drawn independently from q_a, or, without q, whatever they are.)
//
// All of it is 64-bit: a cumulative sum over 32064 ids in 32 bits would put the drawn token next to its border
// in about one call of a hundred. exp is a table of 64 powers of two and a polynomial (Tang 1989), 10
// 64-bit operations, so that a pass over logits stays near the rate at which they are read.
//
// Two launches, or the second alone (LAZY, below). stats: a warp per (row, 512 ids) leaves their maximum and their sum of exponentials, all rows at once:
// 22 us for 13.5 M f32 logits (816 rows of 32064 ids, half of them in ragged trees), 20 us for 12.3 M bf16 ones. Its bytes
// take 8 and 4 us; it is bound by its instructions, eleven 64-bit ones a logit among them. walk: per tree one
// CTA, or with draft probabilities a cluster of up to eight that shares the passes over the vocabulary which refused children
// ask for; rows' sums and the children's weights are gathered in parallel, and without draft probabilities every child is
// decided at once, so that the walk itself runs from shared memory; the drawn token takes a search over the sums of 512
// ids and one warp's scan. One tree: 5 to 10 us, nearly all of it latency (dependent loads, 64-bit reductions). Both
// together: 27 rows x 256 ids 11 us, 51 x 32064 15 us, 64 chains of 6 rows 36 us. Where the trees have many more rows than a walk
// visits, the cluster sums a row when the walk comes to it: 16 trees of 51 rows with draft probabilities 39 us instead of 46 (39 to 46
// on other inputs: the longest path counts).
#pragma once
#include <cooperative_groups.h>
#include <algorithm>
#include <cuda_fp16.h>

#include "common.cuh"

namespace sampled {

constexpr int SUB = 512;                  // ids that one warp sums
constexpr int STATS_THREADS = 256;
constexpr int WALK_THREADS = 512;
constexpr int CLUSTER = 8;                // largest
constexpr int MAX_IDS = 1 << 20;          // ids that may take part
constexpr float MAX_TEMPERATURE = 1e30f;   // (300 temperatures below any logit is still a number)
inline double exp_factor(float temperature) { return 92.332482616893657 / (double)temperature; }
inline int pieces_of(int ids) { return (ids + SUB - 1) / SUB; }

struct Args {
  const void *logits;                     // [rows][ld] of f32 / bf16 / f16
  long long ld;
  const float *probs;                     // [rows][ld_probs] or NULL
  long long ld_probs;
  int lo, hi;
  int n_sub;                              // pieces of SUB ids
  int per_cta;                            // ... that a CTA of the first launch takes
  int kept;                               // ... whose probabilities a warp of the second keeps between passes over a row
  float temperature;
  double factor;                          // 64 / (ln 2 temperature)
  const float *u;                         // [rows], in the order of the logits' rows
  // trees, as arrays ...
  const int *tokens, *parent, *n_rows;    // [n_seq][rows]; n_rows [n_seq] or NULL
  int rows;
  // ... or as the context keeps them
  const DevTree *trees;
  // workspace
  float *sub_max;                         // [rows][n_sub]
  double *sub_sum;                        // [rows][n_sub] sum of exp((z - sub_max) / temperature)
  // answers
  int *out_m, *out_tok, *out_path;        // [n_seq], [n_seq][out_width] twice, -1 behind the last
  int out_width;
};

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<bf16>(bf16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f<__half>(__half v) { return __half2float(v); }

// 2^(i / 64), copied to shared memory by a kernel's first threads.
static __device__ const double EXP2_64[64] = {
    1, 1.0108892860517005, 1.0218971486541166, 1.0330248790212284,
    1.0442737824274138, 1.0556451783605572, 1.0671404006768237, 1.0787607977571199,
    1.0905077326652577, 1.1023825833078409, 1.1143867425958924, 1.1265216186082418,
    1.1387886347566916, 1.1511892299529827, 1.1637248587775775, 1.1763969916502812,
    1.189207115002721, 1.2021567314527031, 1.215247359980469, 1.22848053610687,
    1.241857812073484, 1.2553807570246911, 1.2690509571917332, 1.2828700160787783,
    1.2968395546510096, 1.3109612115247644, 1.3252366431597413, 1.3396675240533029,
    1.3542555469368927, 1.3690024229745905, 1.383909881963832, 1.3989796725383112,
    1.4142135623730951, 1.42961333839197, 1.4451808069770467, 1.460917794180647,
    1.4768261459394993, 1.4929077282912648, 1.5091644275934228, 1.5255981507445384,
    1.5422108254079407, 1.5590044002378369, 1.5759808451078865, 1.593142151342267,
    1.6104903319492543, 1.6280274218573478, 1.6457554781539649, 1.6636765803267364,
    1.681792830507429, 1.7001063537185235, 1.7186192981224779, 1.7373338352737062,
    1.7562521603732995, 1.7753764925265212, 1.7947090750031072, 1.8142521755003989,
    1.8340080864093424, 1.8539791250833855, 1.8741676341103, 1.8945759815869656,
    1.9152065613971474, 1.9360617934922943, 1.9571441241754002, 1.9784560263879509,
};
struct ExpTable { double t[64]; };
__device__ __forceinline__ void fill(ExpTable &tab) {
  if (threadIdx.x < 64) tab.t[threadIdx.x] = EXP2_64[threadIdx.x];
}
// Weights of one row: exp((z - zmax) / temperature) = 2^(y / 64) with y = (z - zmax) 64 / (ln 2 temperature) = n + r,
// n whole, |r| <= 1/2: a table entry, a power of two and a polynomial of degree 4 in r (the first term left out is
// below 4e-14). Ten 64-bit operations with the sum. zmax has 1, an infinite one too; a NaN, and what lies below e^-300, 0.
struct RowExp {
  float zmax, low;
  double k;
  __device__ __forceinline__ RowExp(float zm, float temperature, double k_)
      : zmax(zm), low(fmaxf(zm - 300.f * temperature, -3.4028235e38f)), k(k_) {}
  // zmax finite, low <= z <= zmax (low is rounded: twice the distance at most)
  __device__ __forceinline__ double inner(float z, const ExpTable &tab) const {
    constexpr double MAGIC = 6755399441055744.0;               // 1.5 * 2^52
    const double d = (double)z - (double)zmax;
    const double m = fma(d, k, MAGIC);
    const int n = __double2loint(m);
    const double r = fma(d, k, MAGIC - m);
    double p = fma(r, 5.7328516886404019e-10, 2.1173137155464776e-07);                               // (ln 2 / 64)^j / j!
    p = fma(p, r, 5.86490495505617e-05);
    p = fma(p, r, 0.010830424696249145);
    p = fma(p, r, 1.0);
    const double t = tab.t[n & 63];
    return p * __hiloint2double(__double2hiint(t) + ((n >> 6) << 20), __double2loint(t));
  }
  __device__ __forceinline__ double operator()(float z, const ExpTable &tab) const {
    return z == zmax ? 1.0 : finite(z, tab);
  }
  __device__ __forceinline__ double finite(float z, const ExpTable &tab) const {
    const double p = inner(z, tab);
    return z >= low ? p : 0.0;
  }
  // the same for a sum that zmax is part of (zmax finite, low < zmax): what counts as 0 gives e^-300 at most
  __device__ __forceinline__ double summand(float z, const ExpTable &tab) const { return inner(fmaxf(z, low), tab); }
};

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// 16 ids of a lane: ids 128 j + 4 lane + e of the piece that starts at `first`, or (RUN) 16 lane + 4 j + e; -inf past
// `end`. Loads first, selections after: behind a branch each load would wait for the one before it.
template <bool RUN, typename T> __device__ __forceinline__ void load_piece(const T *row, int first, int end, bool vec, float (&z)[16]) {
  const int lane = threadIdx.x & 31, base = first + (RUN ? 16 : 4) * lane, step = RUN ? 4 : 128;
  if (vec && first + SUB <= end) {
    struct alignas(4 * sizeof(T)) Four { T e[4]; };
    Four v[4];
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] = *reinterpret_cast<const Four *>(row + base + step * j);
#pragma unroll
    for (int k = 0; k < 16; k++) z[k] = to_f(v[k >> 2].e[k & 3]);
  } else {
    T v[16];
#pragma unroll
    for (int k = 0; k < 16; k++) v[k] = row[min(base + step * (k >> 2) + (k & 3), end - 1)];
#pragma unroll
    for (int k = 0; k < 16; k++) z[k] = base + step * (k >> 2) + (k & 3) < end ? to_f(v[k]) : -INFINITY;
  }
}
// Whether four elements at a multiple of four ids after lo are aligned.
template <typename T> __device__ __forceinline__ bool aligned4(const T *p) {
  return reinterpret_cast<uintptr_t>(p) % (4 * sizeof(T)) == 0;
}

// Maximum and sum of exponentials of a piece (whole warp).
template <typename T>
__device__ __forceinline__ void sum_piece(const Args &a, const T *z0, int sub, int width, bool vec, const ExpTable &tab, float &m, double &s) {
  float z[16];
  load_piece<false>(z0, sub * SUB, width, vec, z);
  m = -INFINITY;
#pragma unroll
  for (int k = 0; k < 16; k++) m = fmaxf(m, z[k]);             // (a NaN loses)
  m = warp_max(m);
  const RowExp weight(m, a.temperature, a.factor);
  s = 0.0;
  if (m < INFINITY && weight.low < m) {
#pragma unroll
    for (int k = 0; k < 16; k++) s += weight.summand(z[k], tab);
  } else if (m > -INFINITY) {                                  // infinite logits share the row, or the temperature is next to 0
#pragma unroll
    for (int k = 0; k < 16; k++) s += weight(z[k], tab);
  }
  s = warp_sum64(s);
}

// CTX: row numbers of a context's call (no rows are left out). A CTA takes a.per_cta pieces of one row, its warps in turn.
template <typename T, bool CTX>
static __global__ void __launch_bounds__(STATS_THREADS, 6) stats_kernel(const Args a) {
  __shared__ ExpTable tab;
  fill(tab);
  pdl_wait();
  pdl_launch();
  const int row = blockIdx.x, lane = threadIdx.x & 31;
  if (!CTX && a.n_rows) {
    const int seq = row / a.rows;
    if (row - seq * a.rows >= max(a.n_rows[seq], 1)) return;
  }
  const int end = min(a.n_sub, ((int)blockIdx.y + 1) * a.per_cta), width = a.hi - a.lo;
  int sub = (int)blockIdx.y * a.per_cta + (threadIdx.x >> 5);
  const T *z0 = static_cast<const T *>(a.logits) + row * a.ld + a.lo;
  const bool vec = aligned4(z0);
  __syncthreads();
  for (; sub < end; sub += STATS_THREADS / 32) {
    float m;
    double s;
    sum_piece(a, z0, sub, width, vec, tab, m, s);
    if (lane == 0) {
      a.sub_max[(size_t)row * a.n_sub + sub] = m;
      a.sub_sum[(size_t)row * a.n_sub + sub] = s;
    }
  }
}

struct Walk {
  float zmax[SV_MAX_TREE];                // of a row with children
  double z[SV_MAX_TREE];                  // its sum of weights; 0: nothing to draw from, the lowest id has all
  double w[SV_MAX_TREE];                  // weight of the row's token in its parent's row (PROBS: over its sum)
  float q[SV_MAX_TREE], u[SV_MAX_TREE];
  int tok[SV_MAX_TREE];
  int inner[SV_MAX_TREE];                 // the row has children
  alignas(16) int parent[SV_MAX_TREE];    // -1 past the last row
  int yes[SV_MAX_TREE];                   // no PROBS: the row is accepted if the walk comes to it; 2: not yet decided
  int again[SV_MAX_TREE];                 // no PROBS: an elder sibling has the same token
  int path[SV_MAX_TREE];
  int refused[SV_MAX_TREE];               // tokens refused at the row where the walk ends, each once
  int n_refused, cur, next, m, want;      // want: the walk waits for a pass over the vocabulary
  double beta, S;
  double part[2][CLUSTER * WALK_THREADS / 32];   // sums of the cluster's warps, by turns
  float part_max[2][CLUSTER * WALK_THREADS / 32];
  double left[WALK_THREADS / 32];
};

// The children that put_yes left open (of row `of`, or of all rows where it is -1), from the sums of their parents' rows without
// the tokens refused before them (whole CTA). z0: the tree's first row.
template <typename T>
static __device__ __noinline__ void settle_yes(Walk &w, const ExpTable &tab, const T *z0, long long ld, int n, int width, int n_sub,
                                               float temperature, double factor, int of) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int j = 1; j < n; j++) {
    const int i = w.parent[j];
    if (i < 0 || (of >= 0 && i != of) || w.yes[j] != 2) continue;
    const T *z1 = z0 + i * ld;
    const RowExp weight(w.zmax[i], temperature, factor);
    double s = 0.0;
    for (int k = warp; k < n_sub; k += WALK_THREADS / 32) {
      float z[16];
      load_piece<false>(z1, k * SUB, width, aligned4(z1), z);
      uint32_t out = 0;                                          // this lane's refused ones
      for (int r = i + 1; r < j; r++) {
        const int at = w.parent[r] == i ? w.tok[r] - k * SUB : -1;
        if (at >= 0 && at < SUB && (at >> 2 & 31) == lane) out |= 1u << (at >> 7 << 2 | (at & 3));
      }
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const double v = weight(z[e], tab);                      // (past the last id: -inf)
        s += out >> e & 1 ? 0.0 : v;
      }
    }
    s = warp_sum64(s);
    if (lane == 0) w.left[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
      double S = 0.0;
      for (int k = 0; k < WALK_THREADS / 32; k++) S += w.left[k];
      w.yes[j] = (double)w.u[j] * S < w.w[j];
    }
    __syncthreads();
  }
}

// The piece at `target` of n sums (whole warp), and the cumulative sum before it; the last piece that has any weight
// where none reaches it, -1: none has.
__device__ __forceinline__ int search_sums(int n, double target, const double *sums, double *before) {
  const int lane = threadIdx.x & 31;
  double base = 0.0, last_base = 0.0;
  int last = -1;
  for (int k0 = 0; k0 < n; k0 += 32) {
    const double v = k0 + lane < n ? sums[k0 + lane] : 0.0;
    double incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    const double excl = base + (incl - v);
    const unsigned hit = __ballot_sync(0xffffffffu, v > 0.0 && base + incl > target);
    if (hit) {
      const int l = __ffs(hit) - 1;
      *before = __shfl_sync(0xffffffffu, excl, l);
      return k0 + l;
    }
    const unsigned some = __ballot_sync(0xffffffffu, v > 0.0);
    if (some) {
      const int l = 31 - __clz(some);
      last = k0 + l;
      last_base = __shfl_sync(0xffffffffu, excl, l);
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  *before = last_base;
  return last;
}
// The same among 16 consecutive ids a lane, which begin at the cumulative sum `before`: the first id whose cumulative
// weight exceeds `target`, else the last that has any.
__device__ __forceinline__ int search_ids(double before, double target, int first, const double (&wt)[16]) {
  const int lane = threadIdx.x & 31;
  double mine = 0.0;
#pragma unroll
  for (int e = 0; e < 16; e++) mine += wt[e];
  double incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  double c = before + (incl - mine);
  int found = -1, any = -1;
#pragma unroll
  for (int e = 0; e < 16; e++) {
    c += wt[e];
    if (wt[e] > 0.0) {
      any = first + 16 * lane + e;
      if (found < 0 && c > target) found = any;
    }
  }
  const unsigned hit = __ballot_sync(0xffffffffu, found >= 0);
  if (hit) return __shfl_sync(0xffffffffu, found, __ffs(hit) - 1);
  const unsigned some = __ballot_sync(0xffffffffu, any >= 0);
  return some ? __shfl_sync(0xffffffffu, any, 31 - __clz(some)) : -1;
}

// LAZY: without the first launch; the cluster sums a row when the walk comes to it.
// Dynamic shared memory: [n_sub] doubles, the sums of the pieces of the row where the walk ends; LAZY: [n_sub] floats, their
// maxima; PROBS: then p and q of the first a.kept pieces of every warp.
template <typename T, bool PROBS, bool LAZY, bool CTX>
static __global__ void __launch_bounds__(WALK_THREADS, PROBS || LAZY ? 2 : 1) walk_kernel(const Args a, const EpArgs ea) {
  namespace cg = cooperative_groups;
  constexpr bool CLUSTERED = PROBS || LAZY;
  __shared__ ExpTable tab;
  __shared__ Walk w;
  extern __shared__ double s_sub[];
  fill(tab);
  if (CLUSTERED) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // (that every CTA has started)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int WARPS = WALK_THREADS / 32;
  if (tid < SV_MAX_TREE) w.inner[tid] = 0, w.parent[tid] = -1;
  int rank = 0, ranks = 1;
  if (CLUSTERED) {
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  }
  const int seq = (int)blockIdx.x / ranks;
  pdl_wait();
  pdl_launch();
  const DevTree *tr = CTX ? a.trees + ea.eps[seq] : nullptr;
  const long long row0 = CTX ? ea.row0[seq] : (long long)seq * a.rows;
  const int n = CTX ? min(tr->n_rows, ea.nrows[seq]) : a.n_rows ? min(max(a.n_rows[seq], 1), a.rows) : a.rows;
  const int width = a.hi - a.lo;
  auto logits_of = [&](int i) { return static_cast<const T *>(a.logits) + (row0 + i) * a.ld + a.lo; };
  auto probs_of = [&](int i) { return a.probs + (row0 + i) * a.ld_probs + a.lo; };
  auto maxima_of = [&](int i) { return a.sub_max + (size_t)(row0 + i) * a.n_sub; };
  auto sums_of = [&](int i) { return a.sub_sum + (size_t)(row0 + i) * a.n_sub; };
  auto row_max = [&](const float *sm) {                          // (whole warp)
    float m = -INFINITY;
    for (int k = lane; k < a.n_sub; k += 32) m = fmaxf(m, sm[k]);
    return warp_max(m);
  };

  float *s_max = reinterpret_cast<float *>(s_sub + a.n_sub);
  double *s_kept = s_sub + a.n_sub + (LAZY ? (a.n_sub + 1) / 2 : 0);

  // ---- the tree; a thread keeps its row's parent and token
  __syncthreads();
  int my_parent = -1, my_x = -1;
  float my_z = 0.f, my_q = 0.f;
  uint32_t elder[4];
  if (tid < n) {
    my_x = (int)((unsigned)(CTX ? tr->tok[tid] : a.tokens[row0 + tid]) - (unsigned)a.lo);
    my_parent = CTX ? tr->parent[tid] : a.parent[row0 + tid];
    if (tid == 0 || my_parent < 0 || my_parent >= tid) my_parent = -1;   // no row's child
    w.u[tid] = a.u[row0 + tid];
    w.tok[tid] = my_x;
    w.parent[tid] = my_parent;
    if (my_parent >= 0) w.inner[my_parent] = 1;
  }
  const bool inside = my_parent >= 0 && my_x >= 0 && my_x < width;
  if (inside) {
    my_z = to_f(logits_of(my_parent)[my_x]);
    if (PROBS) my_q = fmaxf(probs_of(my_parent)[my_x], 0.f);
  }
  __syncthreads();
  // ---- rows with children: maximum and sum from the pieces, a warp per row
  for (int i = warp; !LAZY && i < n; i += WARPS) {
    if (!w.inner[i]) continue;
    const float *sm = maxima_of(i);
    const double *su = sums_of(i);
    // (the first 64 pieces' values are asked for together)
    const int k0 = min(lane, a.n_sub - 1), k1 = min(lane + 32, a.n_sub - 1);
    const float m0 = sm[k0], m1 = sm[k1];
    const double s0 = su[k0], s1 = su[k1];
    float m = fmaxf(m0, m1);
    for (int k = lane + 64; k < a.n_sub; k += 32) m = fmaxf(m, sm[k]);
    m = warp_max(m);
    const RowExp weight(m, a.temperature, a.factor);
    double z = 0.0;
    if (m > -INFINITY) {
      if (lane < a.n_sub && m0 > -INFINITY) z = s0 * weight(m0, tab);
      if (lane + 32 < a.n_sub && m1 > -INFINITY) z += s1 * weight(m1, tab);
      for (int k = lane + 64; k < a.n_sub; k += 32)
        if (sm[k] > -INFINITY) z += su[k] * weight(sm[k], tab);
    }
    z = warp_sum64(z);
    if (lane == 0) w.zmax[i] = m, w.z[i] = z;
  }
  if (tid == 0) {
    w.cur = 0, w.next = 1, w.m = 0, w.n_refused = 0, w.path[0] = 0;
    w.beta = 0.0, w.S = 1.0;
  }
  __syncthreads();
  // weight of id x of a row with children, and the sum of its row
  auto weight_of = [&](int i, float z, int x) {
    return w.z[i] > 0.0 ? RowExp(w.zmax[i], a.temperature, a.factor)(z, tab) : x == 0 ? 1.0 : 0.0;
  };
  auto sum_of = [&](int i) { return w.z[i] > 0.0 ? w.z[i] : 1.0; };
  // weight of the thread's token in its parent's row
  auto put_weight = [&]() {
    const double v = inside ? weight_of(my_parent, my_z, my_x) : 0.0;
    w.w[tid] = PROBS ? (inside ? v / sum_of(my_parent) : 0.0) : v;
  };
  // no PROBS: whether the thread's row is accepted if the walk comes to it; S: what is left of the parent's row then. The
  // subtraction leaves an error of up to 2^-40 of the whole in S (the weights' 4e-14 each, roundings); where that could turn the
  // decision, S is summed without the refused tokens (settle_yes). true: that is to be done.
  auto put_yes = [&]() {
    int yes = 0;
    if (inside && !w.again[tid] && w.w[tid] > 0.0) {
      const double whole = sum_of(my_parent), u = w.u[tid];
      double S = whole;
#pragma unroll
      for (int k = 0; k < 4; k++)
        for (uint32_t left = elder[k]; left; left &= left - 1) {
          const int j = 32 * k + __ffs(left) - 1;
          if (!w.again[j]) S -= w.w[j];
        }
      const double off = S < whole ? 0x1p-40 * whole : 0.0;
      yes = u * (S + off) < w.w[tid] ? 1 : u * (S - off) < w.w[tid] ? 2 : 0;
    }
    w.yes[tid] = yes;
    return yes == 2;
  };
  auto decide = [&](bool mine, int of) {
    const bool open = mine && put_yes();
    if (__syncthreads_or(open))
      settle_yes(w, tab, logits_of(0), a.ld, n, width, a.n_sub, a.temperature, a.factor, of);
  };
  if (tid < n) {
    w.q[tid] = my_q;
    if (!PROBS) {
      // the row's elder siblings, a bit each
#pragma unroll
      for (int k = 0; k < 4; k++) {
        elder[k] = 0;
        if (32 * k < tid && my_parent >= 0) {
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            const int4 p = *reinterpret_cast<const int4 *>(&w.parent[32 * k + j]);
            elder[k] |= (uint32_t)((p.x == my_parent) | (p.y == my_parent) << 1 | (p.z == my_parent) << 2 | (p.w == my_parent) << 3) << j;
          }
          if (32 * k + 31 >= tid) elder[k] &= (1u << (tid & 31)) - 1;
        }
      }
      bool again = false;
#pragma unroll
      for (int k = 0; k < 4; k++)
        for (uint32_t left = elder[k]; left; left &= left - 1) again |= w.tok[32 * k + __ffs(left) - 1] == my_x;
      w.again[tid] = again;
    }
    if (!LAZY) put_weight();
  }
  __syncthreads();
  if (!PROBS && !LAZY) {                                         // every child is decided at once
    decide(tid < n, -1);
  }
  if (CLUSTERED) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");

  // ---- the walk: a warp runs it from shared memory, everybody joins for a pass over the vocabulary
  int turn = 0;
  // Hands a value of this warp to the cluster's CTAs; all have all of them when it returns (the words of a turn are written
  // again after the next hand-over, which every CTA comes to when it has read them).
  auto hand_over = [&](double sum, float max) {
    if (lane < ranks) {
      cg::cluster_group cl = cg::this_cluster();
      *cl.map_shared_rank(&w.part[turn][rank * WARPS + warp], lane) = sum;
      if (LAZY) *cl.map_shared_rank(&w.part_max[turn][rank * WARPS + warp], lane) = max;
    }
    if (ranks > 1) cg::this_cluster().sync();
    else __syncthreads();
  };
  bool fresh = true;                                             // LAZY: the walk has just come to its row
  for (;;) {
    if constexpr (LAZY) {
      if (fresh) {
        const int cur = w.cur;
        const T *z0 = logits_of(cur);
        const bool vz = aligned4(z0);
        float M = -INFINITY;
        double S = 0.0;
        for (int k = warp * ranks + rank; k < a.n_sub; k += WARPS * ranks) {
          float m;
          double s;
          sum_piece(a, z0, k, width, vz, tab, m, s);
          if (lane == 0) s_sub[k] = s, s_max[k] = m;
          if (m > M) {
            S = (M > -INFINITY ? S * RowExp(m, a.temperature, a.factor)(M, tab) : 0.0) + s;
            M = m;
          } else if (m > -INFINITY) {
            S += s * RowExp(M, a.temperature, a.factor)(m, tab);
          }
        }
        hand_over(S, M);
        M = -INFINITY;
        for (int k = lane; k < ranks * WARPS; k += 32) M = fmaxf(M, w.part_max[turn][k]);
        M = warp_max(M);
        const RowExp weight(M, a.temperature, a.factor);
        S = 0.0;
        for (int k = lane; k < ranks * WARPS; k += 32)
          if (w.part_max[turn][k] > -INFINITY) S += w.part[turn][k] * weight(w.part_max[turn][k], tab);
        S = warp_sum64(S);
        turn ^= 1;
        if (tid == 0) w.zmax[cur] = M, w.z[cur] = S;
        __syncthreads();
        if (tid < n && my_parent == cur) put_weight();
        __syncthreads();
        if (!PROBS) decide(tid < n && my_parent == cur, cur);
      }
    }
    if (warp == 0) {
      int cur = w.cur, m = w.m;
      if constexpr (PROBS) {
        double beta = w.beta, S = w.S;
        int want = 0, i0 = w.next;
        while (i0 < n && !want) {
          const unsigned kids = __ballot_sync(0xffffffffu, i0 + lane < n && w.parent[i0 + lane] == cur);
          if (!kids) {
            i0 += 32;
            continue;
          }
          const int c = i0 + __ffs(kids) - 1;
          i0 = c + 1;
          const double q = w.q[c], r = w.w[c] - beta * q;
          if (r > 0.0 && (double)w.u[c] * q * S < r) {
            cur = c;
            m++;
            beta = 0.0, S = 1.0;
            if (lane == 0) w.path[m] = c;
            if (LAZY) want = 4;                                  // its row's sum
          } else {
            // the sum of what is left: the row's first (1), with another child to come (3), a later one (2)
            unsigned others = 0;
            for (int i1 = i0; i1 < n && !others; i1 += 32)
              others = __ballot_sync(0xffffffffu, i1 + lane < n && w.parent[i1 + lane] == cur);
            want = beta > 0.0 ? 2 : others ? 3 : 1;
            beta += S;
          }
        }
        if (lane == 0) w.cur = cur, w.m = m, w.next = i0, w.beta = beta, w.S = S, w.want = want;
      } else {
        int want = 0;
        for (int i0 = cur + 1; i0 < n && !want;) {
          const unsigned kids = __ballot_sync(0xffffffffu, i0 + lane < n && w.parent[i0 + lane] == cur && w.yes[i0 + lane]);
          if (!kids) {
            i0 += 32;
            continue;
          }
          cur = i0 + __ffs(kids) - 1;
          i0 = cur + 1;
          m++;
          if (lane == 0) w.path[m] = cur;
          if (LAZY) want = 4;
        }
        // the children refused there
        int nref = 0;
        for (int i0 = cur + 1; i0 < n; i0 += 32) {
          const int i = i0 + lane;
          const bool no = i < n && w.parent[i] == cur && !w.again[i] && w.tok[i] >= 0 && w.tok[i] < width;
          const unsigned all = __ballot_sync(0xffffffffu, no);
          if (no) w.refused[nref + __popc(all & ((1u << lane) - 1))] = w.tok[i];
          nref += __popc(all);
        }
        if (lane == 0) w.cur = cur, w.m = m, w.n_refused = nref, w.want = want;
      }
    }
    __syncthreads();
    if (!CLUSTERED || !w.want) break;
    fresh = w.want == 4;
    if (LAZY && fresh) {
      __syncthreads();                                           // (everyone has read what is wanted)
      continue;
    }
    if constexpr (PROBS) {
      // S = sum of max(p - beta q, 0): pieces go round the cluster's warps; their sums stay for the search, and p and q in
      // shared memory for the row's next pass
      const int cur = w.cur;
      const bool none = !(w.z[cur] > 0.0), first = w.want != 2, keep = w.want == 3;
      const double beta = w.beta, inv_z = 1.0 / sum_of(cur);
      const RowExp weight(w.zmax[cur], a.temperature, a.factor);
      const T *z0 = logits_of(cur);
      const float *q0 = probs_of(cur);
      const bool vz = aligned4(z0), vq = aligned4(q0);
      double mine = 0.0;
      for (int k = warp * ranks + rank, n = 0; k < a.n_sub; k += WARPS * ranks, n++) {
        double p[16], s = 0.0;
        float q[16];
        double *kp = s_kept + ((size_t)n * WARPS + warp) * 768 + lane;   // 16 x 32 of p, then of q
        if (first || n >= a.kept) {
          float z[16];
          load_piece<false>(z0, k * SUB, width, vz, z);
          load_piece<false>(q0, k * SUB, width, vq, q);
#pragma unroll
          for (int e = 0; e < 16; e++) {
            const int x = k * SUB + 128 * (e >> 2) + 4 * lane + (e & 3);
            p[e] = none ? (x == 0 ? 1.0 : 0.0) : weight(z[e], tab) * inv_z;      // (past the last id: -inf)
            q[e] = fmaxf(q[e], 0.f);
          }
          if (keep && n < a.kept) {
            float *kq = reinterpret_cast<float *>(kp + 512 - lane) + lane;
#pragma unroll
            for (int e = 0; e < 16; e++) kp[32 * e] = p[e], kq[32 * e] = q[e];
          }
        } else {
          const float *kq = reinterpret_cast<const float *>(kp + 512 - lane) + lane;
#pragma unroll
          for (int e = 0; e < 16; e++) p[e] = kp[32 * e], q[e] = kq[32 * e];
        }
#pragma unroll
        for (int e = 0; e < 16; e++) s += fmax(fma(-beta, (double)q[e], p[e]), 0.0);
        s = warp_sum64(s);
        if (lane == 0) s_sub[k] = s;
        mine += s;
      }
      hand_over(mine, 0.f);
      if (warp == 0) {
        double s = 0.0;
        for (int k = lane; k < ranks * WARPS; k += 32) s += w.part[turn][k];
        s = warp_sum64(s);
        if (lane == 0) w.S = s;
        __syncwarp();
      }
      turn ^= 1;
    }
  }

  // ---- the token after the path, from what is left of its last row
  const int cur = w.cur, m = w.m;
  const bool residual = PROBS && w.beta > 0.0 && w.S > 0.0;      // (the last pass was made with this beta)
  if (CLUSTERED && ranks > 1) {
    // every CTA has its own pieces' sums: the first one collects them
    cg::cluster_group cl = cg::this_cluster();
    if ((residual || LAZY) && rank != 0)
      for (int k = warp * ranks + rank; k < a.n_sub; k += WARPS * ranks)
        if (lane == 0) {
          cl.map_shared_rank(s_sub, 0)[k] = s_sub[k];
          if (LAZY) cl.map_shared_rank(s_max, 0)[k] = s_max[k];
        }
    cl.sync();
    if (rank != 0) return;
  }
  const float *sm = maxima_of(cur);
  const double *su = sums_of(cur);
  const float zm = LAZY || w.inner[cur] ? w.zmax[cur] : row_max(sm);
  const RowExp weight(zm, a.temperature, a.factor);
  const bool none = !(zm > -INFINITY);
  // the sums of p itself over the pieces first, first + step, ... (by warps, LAZY, from the logits; else by threads)
  auto plain_sums = [&](int first, int step) {
    if (LAZY) {
      const T *z0 = logits_of(cur);
      for (int k = first; k < a.n_sub; k += step) {
        float m;
        double s;
        sum_piece(a, z0, k, width, aligned4(z0), tab, m, s);
        if (lane == 0) s_sub[k] = m > -INFINITY ? s * weight(m, tab) : 0.0;
      }
    } else {
      for (int k = first; k < a.n_sub; k += step) s_sub[k] = sm[k] > -INFINITY ? su[k] * weight(sm[k], tab) : 0.0;
    }
  };
  if (!residual) {
    if (!LAZY) plain_sums(tid, WALK_THREADS);
    else if (PROBS && w.beta > 0.0) plain_sums(warp, WARPS);     // (what was left there is nothing: the sums are gone)
    else
      for (int k = tid; k < a.n_sub; k += WALK_THREADS) s_sub[k] = s_max[k] > -INFINITY ? s_sub[k] * weight(s_max[k], tab) : 0.0;
    // pieces that hold a refused token are summed again without it
    for (int k0 = 0; !PROBS && k0 < w.n_refused; k0 += WARPS) {
      const int k = k0 + warp, piece = k < w.n_refused ? w.refused[k] / SUB : -1;
      double s = 0.0;
      if (piece >= 0) {
        float z[16];
        const T *z0 = logits_of(cur);
        load_piece<false>(z0, piece * SUB, width, aligned4(z0), z);
        uint32_t out = 0;                                        // this lane's refused ones
        for (int j = 0; j < w.n_refused; j++) {
          const int at = w.refused[j] - piece * SUB;
          if (at >= 0 && at < SUB && (at >> 2 & 31) == lane) out |= 1u << (at >> 7 << 2 | (at & 3));
        }
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const double v = weight(z[e], tab);                    // (past the last id: -inf)
          s += out >> e & 1 ? 0.0 : v;
        }
        s = warp_sum64(s);
      }
      __syncthreads();                                           // (after the plain sums)
      if (piece >= 0 && lane == 0) s_sub[piece] = s;             // (twice in the same piece: the same sum)
    }
    __syncthreads();
  }
  if (warp == 0) {
    int drop = PROBS ? 0 : w.n_refused;
    auto sum_all = [&]() {
      double t = 0.0;
      for (int k = lane; k < a.n_sub; k += 32) t += s_sub[k];
      return warp_sum64(t);
    };
    double total = sum_all();
    if (!none && !(total > 0.0) && drop) {                       // nothing is left: from p itself
      drop = 0;
      if (LAZY) plain_sums(0, 1);
      else plain_sums(lane, 32);
      __syncwarp();
      total = sum_all();
    }
    int token = 0;                                               // a row without a number gives its lowest id
    if (!none || residual) {
      const double target = (double)w.u[0] * total;
      double before = 0.0;
      const int piece = search_sums(a.n_sub, target, s_sub, &before);
      if (piece >= 0) {
        const T *z0 = logits_of(cur);
        const double inv_z = residual && !none ? 1.0 / w.z[cur] : 1.0;
        float z[16], q[16];
        load_piece<true>(z0, piece * SUB, width, aligned4(z0), z);
        if (residual) load_piece<true>(probs_of(cur), piece * SUB, width, aligned4(probs_of(cur)), q);
        double wt[16];
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const int x = piece * SUB + 16 * lane + e;
          double v = none ? (x == 0 ? 1.0 : 0.0) : weight(z[e], tab) * inv_z;
          if (residual) v = fmax(v - w.beta * (double)fmaxf(q[e], 0.f), 0.0);
          wt[e] = x < width ? v : 0.0;
        }
        for (int j = 0; j < drop; j++) {
          const int at = w.refused[j] - (piece * SUB + 16 * lane);
#pragma unroll
          for (int e = 0; e < 16; e++) wt[e] = at == e ? 0.0 : wt[e];
        }
        token = max(search_ids(before, target, piece * SUB, wt), 0);
      }
    }
    int *om = a.out_m + seq, *ot = a.out_tok + (size_t)seq * a.out_width, *op = a.out_path + (size_t)seq * a.out_width;
    for (int k = lane; k < a.out_width; k += 32) {
      op[k] = k <= m ? w.path[k] : -1;
      ot[k] = a.lo + (k < m ? w.tok[w.path[k + 1]] : token);
      if (k > m) ot[k] = -1;
    }
    if (lane == 0) *om = m;
  }
}

// Both launches. CTX: a context's call, which has its rows in ea and its trees in a.trees.
template <typename T, bool CTX>
inline cudaError_t enqueue(Args a, const EpArgs &ea, int n_seq, int total_rows, cudaStream_t st) {
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = CLUSTER;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  // All rows at once (a microsecond per 1150 pieces), unless they are many more than the walks visit: then row by row as they come
  // to them, which is counted as six rows of every tree at 2.5 us beside their pieces. 16 trees of 51 rows of 32064 ids: 39 us, all at
  // once 46; 64 chains of 6 rows: 47 and 36. What is accepted is not known here, so that deep paths lose: 16 chains of 60 rows, none
  // accepted 13 us and 47, 52 accepted on average 279 and 53; 64 chains of 64 rows, 4 accepted 35 and 142, 54 accepted 359 and 148;
  // 4 chains of 128 rows, 66 accepted 477 and 47. A context's trees are few and small.
  const bool lazy = !CTX && (long long)total_rows * a.n_sub > 6 * (2900 + (long long)n_seq * a.n_sub);
  cudaError_t err = cudaSuccess;
  if (!lazy) {
    // one piece a warp while there are few, up to three (816 rows of 32064 ids with their walk: 55 us, with one 58, with eight
    // 61; 51 rows: 15, with two 16, with eight 22)
    constexpr int WARPS = STATS_THREADS / 32;
    const long long all = (long long)total_rows * a.n_sub, room = 148 * 128;
    a.per_cta = WARPS * (int)std::min(3ll, std::max(1ll, (all + room - 1) / room));
    cfg.gridDim = dim3(total_rows, (a.n_sub + a.per_cta - 1) / a.per_cta);
    cfg.blockDim = dim3(STATS_THREADS);
    if ((err = cudaLaunchKernelEx(&cfg, stats_kernel<T, CTX>, a)) != cudaSuccess) return err;
  }
  cfg.blockDim = dim3(WALK_THREADS);
  cfg.dynamicSmemBytes = a.n_sub * sizeof(double) + (lazy ? (a.n_sub + 1) / 2 * sizeof(double) : 0);
  // a pass over the vocabulary is shared by as many CTAs as run at once, two on an SM
  int ranks = 1;
  while ((a.probs || lazy) && ranks < CLUSTER && 2 * ranks * n_seq <= 2 * 148 && 2 * ranks <= a.n_sub) ranks *= 2;
  constexpr size_t KEPT = WALK_THREADS / 32 * 768 * sizeof(double);   // bytes of one piece per warp
  a.kept = a.probs && a.n_sub <= WALK_THREADS / 32 * ranks ? 1 : 0;
  cfg.dynamicSmemBytes += a.kept * KEPT;
  cfg.gridDim = dim3(ranks * n_seq);
  at[1].val.clusterDim.x = ranks;
  if (a.probs || lazy) cfg.numAttrs = 2;
  auto go = [&](auto kernel) {
    if (a.kept && (err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                              (int)(MAX_IDS / SUB * 12 + KEPT))) != cudaSuccess)
      return err;
    return cudaLaunchKernelEx(&cfg, kernel, a, ea);
  };
  if constexpr (CTX) {                                           // (a context has no draft probabilities)
    return go(walk_kernel<T, false, false, true>);
  } else {
    if (lazy) return a.probs ? go(walk_kernel<T, true, true, false>) : go(walk_kernel<T, false, true, false>);
    return a.probs ? go(walk_kernel<T, true, false, false>) : go(walk_kernel<T, false, false, false>);
  }
}

}  // namespace sampled
