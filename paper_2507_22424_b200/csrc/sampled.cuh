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
// Two launches. stats: a warp per (row, 512 ids) leaves their maximum and their sum of exponentials: all rows at
// once, bound by HBM. walk: per tree one CTA (a cluster of eight, when a refused child asks for a pass over the
// vocabulary); rows' sums and the children's weights are gathered in parallel, so that the walk itself runs from
// shared memory, and the drawn token takes a search over the sums of 512 ids and one warp's scan.
#pragma once
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace sampled {

constexpr int SUB = 512;                  // ids that one warp sums
constexpr int STATS_THREADS = 256;
constexpr int WALK_THREADS = 512;
constexpr int CLUSTER = 8;
constexpr int MAX_IDS = 1 << 20;          // ids that may take part
inline int pieces_of(int ids) { return (ids + SUB - 1) / SUB; }

struct Args {
  const void *logits;                     // [rows][ld] of f32 / bf16 / f16
  long long ld;
  const float *probs;                     // [rows][ld_probs] or NULL
  long long ld_probs;
  int lo, hi;
  int n_sub;                              // pieces of SUB ids
  float temperature;
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

// 2^(i / 64) for the exponential below, filled by the kernel's first threads.
struct ExpTable { double t[64]; };
__device__ __forceinline__ void fill(ExpTable &tab) {
  if (threadIdx.x < 64) tab.t[threadIdx.x] = exp2((double)threadIdx.x * 0.015625);
}
// exp(x) for x <= 0: x = n ln2 / 64 + r, |r| <= ln2 / 128, exp(x) = 2^(n / 64) (1 + r + ... + r^5 / 120); the first
// term left out is below 4e-17. Below -700: 0.
__device__ __forceinline__ double exp_neg(double x, const ExpTable &tab) {
  constexpr double INV = 92.332482616893656877;              // 64 / ln 2
  constexpr double LN2_HI = 0.010830424667801708, LN2_LO = 2.8447437476627285e-11;   // ln 2 / 64 in two parts
  constexpr double MAGIC = 6755399441055744.0;               // 1.5 * 2^52
  const double m = fma(x, INV, MAGIC);
  const int n = (int)(unsigned)__double_as_longlong(m);
  const double nd = m - MAGIC;
  const double r = fma(nd, -LN2_LO, fma(nd, -LN2_HI, x));
  double p = fma(r, 1.0 / 120, 1.0 / 24);
  p = fma(p, r, 1.0 / 6);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.0);
  p = fma(p, r, 1.0);
  const double t = tab.t[n & 63];
  const double s = __hiloint2double(__double2hiint(t) + ((n >> 6) << 20), __double2loint(t));
  return x < -700.0 ? 0.0 : p * s;
}
// exp((z - max) / temperature), 0 for a NaN; max itself (an infinite one too) has 1.
__device__ __forceinline__ double weight(float z, float zmax, double inv_t, const ExpTable &tab) {
  if (z == zmax) return 1.0;
  const double x = ((double)z - (double)zmax) * inv_t;
  return x < 0.0 ? exp_neg(x, tab) : 0.0;                     // (NaN compares false)
}

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// 16 ids of a lane: ids 128 j + 4 lane + e of the piece that starts at `first`; -inf past `end`.
template <typename T> __device__ __forceinline__ void load_piece(const T *row, int first, int end, bool vec, float (&z)[16]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < 4; j++) {
    const int i = first + 128 * j + 4 * lane;
    if (vec && i + 4 <= end) {
      struct alignas(4 * sizeof(T)) Four { T e[4]; };
      const Four v = *reinterpret_cast<const Four *>(row + i);
#pragma unroll
      for (int e = 0; e < 4; e++) z[4 * j + e] = to_f(v.e[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; e++) z[4 * j + e] = i + e < end ? to_f(row[i + e]) : -INFINITY;
    }
  }
}
// Whether four elements at a multiple of four ids after lo are aligned.
template <typename T> __device__ __forceinline__ bool aligned4(const T *p) {
  return reinterpret_cast<uintptr_t>(p) % (4 * sizeof(T)) == 0;
}

// CTX: row numbers of a context's call (no rows are left out).
template <typename T, bool CTX>
static __global__ void __launch_bounds__(STATS_THREADS) stats_kernel(const Args a, int total_rows) {
  __shared__ ExpTable tab;
  fill(tab);
  pdl_wait();
  pdl_launch();
  __syncthreads();
  const int lane = threadIdx.x & 31;
  const long long piece = (long long)blockIdx.x * (STATS_THREADS / 32) + (threadIdx.x >> 5);
  if (piece >= (long long)total_rows * a.n_sub) return;
  const int row = (int)(piece / a.n_sub), sub = (int)(piece - (long long)row * a.n_sub);
  if (!CTX && a.n_rows) {
    const int seq = row / a.rows;
    if (row - seq * a.rows >= max(a.n_rows[seq], 1)) return;
  }
  const T *z0 = static_cast<const T *>(a.logits) + row * a.ld + a.lo;
  float z[16];
  load_piece(z0, sub * SUB, a.hi - a.lo, aligned4(z0), z);
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < 16; k++) m = fmaxf(m, z[k]);             // (a NaN loses)
  m = warp_max(m);
  const double inv_t = 1.0 / (double)a.temperature;
  double s = 0.0;
  if (m > -INFINITY) {
#pragma unroll
    for (int k = 0; k < 16; k++) s += weight(z[k], m, inv_t, tab);
  }
  s = warp_sum64(s);
  if (lane == 0) {
    a.sub_max[(size_t)row * a.n_sub + sub] = m;
    a.sub_sum[(size_t)row * a.n_sub + sub] = s;
  }
}

struct Walk {
  float zmax[SV_MAX_TREE];                // of every row
  double z[SV_MAX_TREE];                  // its sum of weights; 0: nothing to draw from, the lowest id has all
  double w[SV_MAX_TREE];                  // weight of the row's token in its parent's row
  float q[SV_MAX_TREE], u[SV_MAX_TREE];
  int tok[SV_MAX_TREE], parent[SV_MAX_TREE];
  int path[SV_MAX_TREE];
  int refused[SV_MAX_TREE];                // tokens refused at the row where the walk stands, each once
  int n_refused, cur, next, m, want;      // want: the walk waits for a pass over the vocabulary
  double beta, S;
  double part[2][CLUSTER];                // sums of the cluster's CTAs, by turns
  double warp_part[WALK_THREADS / 32];
};

// The token at `target` within a piece that begins at the cumulative sum `before` (whole warp): the first id
// whose cumulative weight exceeds it, else the last one that has any.
__device__ __forceinline__ int search_piece(double before, double target, int first, const double (&wt)[16]) {
  const int lane = threadIdx.x & 31;
  int last = -1;
#pragma unroll
  for (int j = 0; j < 4; j++) {
    const double mine = ((wt[4 * j] + wt[4 * j + 1]) + wt[4 * j + 2]) + wt[4 * j + 3];
    double incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    double c = before + (incl - mine);
    int found = -1, any = -1;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      c += wt[4 * j + e];
      if (wt[4 * j + e] > 0.0) {
        any = first + 128 * j + 4 * lane + e;
        if (found < 0 && c > target) found = any;
      }
    }
    const unsigned hit = __ballot_sync(0xffffffffu, found >= 0);
    if (hit) return __shfl_sync(0xffffffffu, found, __ffs(hit) - 1);
    const unsigned some = __ballot_sync(0xffffffffu, any >= 0);
    if (some) last = __shfl_sync(0xffffffffu, any, 31 - __clz(some));
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
  return last;
}

// The piece at `target` of n sums (whole warp): sums[k] is given by `at`; returns the piece, or the last one that has
// any weight, and the cumulative sum before it. -1: none has.
template <typename F> __device__ __forceinline__ int search_sums(int n, double target, F at, double *before) {
  const int lane = threadIdx.x & 31;
  double base = 0.0, last_base = 0.0;
  int last = -1;
  for (int k0 = 0; k0 < n; k0 += 32) {
    const double v = k0 + lane < n ? at(k0 + lane) : 0.0;
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

// Dynamic shared memory: [n_sub] doubles, the sums of the pieces of the row where the walk ends.
template <typename T, bool PROBS, bool CTX>
static __global__ void __launch_bounds__(WALK_THREADS, 1) walk_kernel(const Args a, const EpArgs ea) {
  namespace cg = cooperative_groups;
  __shared__ ExpTable tab;
  __shared__ Walk w;
  extern __shared__ double s_sub[];
  fill(tab);
  if (PROBS) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // (that every CTA has started)
  __syncthreads();
  pdl_wait();
  pdl_launch();
  const int rank = PROBS ? (int)(blockIdx.x % CLUSTER) : 0, ranks = PROBS ? CLUSTER : 1;
  const int seq = PROBS ? (int)(blockIdx.x / CLUSTER) : (int)blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int WARPS = WALK_THREADS / 32;
  const DevTree *tr = CTX ? a.trees + ea.eps[seq] : nullptr;
  const long long row0 = CTX ? ea.row0[seq] : (long long)seq * a.rows;
  const int n = CTX ? tr->n_rows : a.n_rows ? min(max(a.n_rows[seq], 1), a.rows) : a.rows;
  const int width = a.hi - a.lo;
  const double inv_t = 1.0 / (double)a.temperature;
  auto logits_of = [&](int i) { return static_cast<const T *>(a.logits) + (row0 + i) * a.ld + a.lo; };
  auto probs_of = [&](int i) { return a.probs + (row0 + i) * a.ld_probs + a.lo; };

  // ---- all rows: maximum and sum from the pieces, a warp per row
  for (int i = tid; i < n; i += WALK_THREADS) {
    w.tok[i] = CTX ? tr->tok[i] : a.tokens[row0 + i];
    w.parent[i] = CTX ? tr->parent[i] : a.parent[row0 + i];
    w.u[i] = a.u[row0 + i];
  }
  for (int i = warp; i < n; i += WARPS) {
    const float *sm = a.sub_max + (size_t)(row0 + i) * a.n_sub;
    const double *su = a.sub_sum + (size_t)(row0 + i) * a.n_sub;
    float m = -INFINITY;
    for (int k = lane; k < a.n_sub; k += 32) m = fmaxf(m, sm[k]);
    m = warp_max(m);
    __syncwarp();
    double z = 0.0;
    if (m > -INFINITY)
      for (int k = lane; k < a.n_sub; k += 32)
        if (sm[k] > -INFINITY) z += su[k] * weight(sm[k], m, inv_t, tab);
    z = warp_sum64(z);
    if (lane == 0) w.zmax[i] = m, w.z[i] = z;
  }
  if (tid == 0) {
    w.cur = 0, w.next = 1, w.m = 0, w.n_refused = 0, w.path[0] = 0;
    w.beta = 0.0, w.S = 1.0;
  }
  __syncthreads();
  // weight (in units of the row's sum) of id x of row i
  auto p_of = [&](int i, float z, int x) -> double {
    if (!(w.z[i] > 0.0)) return x == 0 ? 1.0 : 0.0;
    return weight(z, w.zmax[i], inv_t, tab) / w.z[i];
  };
  for (int i = 1 + tid; i < n; i += WALK_THREADS) {
    const int p = w.parent[i], x = w.tok[i] - a.lo;
    const bool ok = p >= 0 && p < i && x >= 0 && x < width;
    w.w[i] = ok ? p_of(p, to_f(logits_of(p)[x]), x) : 0.0;
    w.q[i] = PROBS && ok ? fmaxf(probs_of(p)[x], 0.f) : 0.f;
    if (!ok && (p < 0 || p >= i)) w.parent[i] = -1;              // no row's child
  }
  __syncthreads();

  if (PROBS) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");

  // ---- the walk: a warp runs it from shared memory, everybody joins for a pass over the vocabulary
  int turn = 0;
  for (;;) {
    if (warp == 0) {
      int cur = w.cur, m = w.m, nref = w.n_refused;
      double beta = w.beta, S = w.S;
      int want = 0;
      for (int i0 = w.next; i0 < n && !want;) {
        const int i = i0 + lane;
        const unsigned kids = __ballot_sync(0xffffffffu, i < n && w.parent[i] == cur);
        if (!kids) {
          i0 += 32;
          continue;
        }
        const int c = i0 + __ffs(kids) - 1;
        i0 = c + 1;
        const int x = w.tok[c] - a.lo;
        bool take;
        if (PROBS) {
          const double q = w.q[c], r = w.w[c] - beta * q;
          take = r > 0.0 && (double)w.u[c] * q * S < r;
        } else {
          bool twice = false;
          for (int k = lane; k < nref; k += 32) twice |= w.refused[k] == x;
          twice = __any_sync(0xffffffffu, twice);
          const double r = twice ? 0.0 : w.w[c];
          take = r > 0.0 && (double)w.u[c] * S < r;
          if (!take && !twice && x >= 0 && x < width) {
            __syncwarp();
            if (lane == 0) w.refused[nref] = x;
            nref++;
            S -= r;
            __syncwarp();
          }
        }
        if (take) {
          cur = c;
          m++;
          nref = 0;
          beta = 0.0, S = 1.0;
          if (lane == 0) w.path[m] = c;
        } else if (PROBS) {
          beta += S;
          want = 1;                                              // S of the next beta
        }
        if (lane == 0) w.next = i0;
      }
      __syncwarp();
      if (lane == 0) w.cur = cur, w.m = m, w.n_refused = nref, w.beta = beta, w.S = S, w.want = want;
    }
    __syncthreads();
    if (!PROBS || !w.want) break;
    if constexpr (PROBS) {
      // S = sum of max(p - beta q, 0): pieces go round the cluster's warps; their sums stay for the search
      const int cur = w.cur;
      const double beta = w.beta, inv_z = w.z[cur] > 0.0 ? 1.0 / w.z[cur] : 0.0;
      const T *z0 = logits_of(cur);
      const float *q0 = probs_of(cur);
      const bool vz = aligned4(z0), vq = aligned4(q0);
      double mine = 0.0;
      for (int k = warp * ranks + rank; k < a.n_sub; k += WARPS * ranks) {
        float z[16], q[16];
        load_piece(z0, k * SUB, width, vz, z);
        load_piece(q0, k * SUB, width, vq, q);
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const int x = k * SUB + 128 * (e >> 2) + 4 * lane + (e & 3);
          const double p = inv_z > 0.0 ? weight(z[e], w.zmax[cur], inv_t, tab) * inv_z : x == 0 ? 1.0 : 0.0;
          if (x < width) s += fmax(p - beta * (double)fmaxf(q[e], 0.f), 0.0);
        }
        s = warp_sum64(s);
        if (lane == 0) s_sub[k] = s;
        mine += s;
      }
      if (lane == 0) w.warp_part[warp] = mine;
      __syncthreads();
      if (tid == 0) {
        double s = 0.0;
        for (int k = 0; k < WARPS; k++) s += w.warp_part[k];
        cg::cluster_group cl = cg::this_cluster();
        for (int k = 0; k < ranks; k++) *cl.map_shared_rank(&w.part[turn][rank], k) = s;
      }
      cg::this_cluster().sync();
      if (tid == 0) {
        double s = 0.0;
        for (int k = 0; k < ranks; k++) s += w.part[turn][k];
        w.S = s;
      }
      turn ^= 1;
      __syncthreads();
    }
  }

  // ---- the token after the path
  const int cur = w.cur, m = w.m;
  const bool residual = PROBS && w.beta > 0.0 && w.S > 0.0;      // (the last pass was made with this beta)
  if constexpr (PROBS) {
    // every CTA has its own pieces' sums: the first one collects them
    cg::cluster_group cl = cg::this_cluster();
    if (residual && rank != 0)
      for (int k = warp * ranks + rank; k < a.n_sub; k += WARPS * ranks)
        if (lane == 0) cl.map_shared_rank(s_sub, 0)[k] = s_sub[k];
    cl.sync();
    if (rank != 0) return;
  }
  const bool none = !(w.z[cur] > 0.0);
  if (!residual) {
    // what is left is p, without the refused tokens: the sums of the pieces that hold one are made again
    const float zm = w.zmax[cur];
    const float *sm = a.sub_max + (size_t)(row0 + cur) * a.n_sub;
    const double *su = a.sub_sum + (size_t)(row0 + cur) * a.n_sub;
    for (int k = tid; k < a.n_sub; k += WALK_THREADS) {
      const float km = sm[k];
      s_sub[k] = km > -INFINITY ? su[k] * weight(km, zm, inv_t, tab) : 0.0;
    }
    __syncthreads();
    if (!PROBS) {
      for (int k = warp; k < w.n_refused; k += WARPS) {
        const int piece = w.refused[k] / SUB;
        bool first = true;                                       // once per piece
        for (int j = 0; j < k; j++) first &= w.refused[j] / SUB != piece;
        if (!first) continue;
        float z[16];
        const T *z0 = logits_of(cur);
        load_piece(z0, piece * SUB, width, aligned4(z0), z);
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const int x = piece * SUB + 128 * (e >> 2) + 4 * lane + (e & 3);
          bool out = false;
          for (int j = 0; j < w.n_refused; j++) out |= w.refused[j] == x;
          if (!out && x < width) s += weight(z[e], zm, inv_t, tab);
        }
        s = warp_sum64(s);
        if (lane == 0) s_sub[piece] = s;
      }
      __syncthreads();
    }
  }
  if (warp == 0) {
    int drop = PROBS ? 0 : w.n_refused;
    double total = 0.0;
    for (int k = lane; k < a.n_sub; k += 32) total += s_sub[k];
    total = warp_sum64(total);
    if (!none && !(total > 0.0) && drop) {                       // nothing is left: from p itself
      drop = 0;
      const float zm = w.zmax[cur];
      const float *sm = a.sub_max + (size_t)(row0 + cur) * a.n_sub;
      const double *su = a.sub_sum + (size_t)(row0 + cur) * a.n_sub;
      for (int k = lane; k < a.n_sub; k += 32) {
        const float km = sm[k];
        s_sub[k] = km > -INFINITY ? su[k] * weight(km, zm, inv_t, tab) : 0.0;
      }
      total = w.z[cur];
      __syncwarp();
    }
    int token = 0;                                               // a row without a number gives its lowest id
    if (!none || residual) {
      const double target = (double)w.u[0] * total;
      double before = 0.0;
      const int piece = search_sums(a.n_sub, target, [&](int k) { return s_sub[k]; }, &before);
      if (piece >= 0) {
        float z[16], q[16];
        const T *z0 = logits_of(cur);
        load_piece(z0, piece * SUB, width, aligned4(z0), z);
        if (residual) load_piece(probs_of(cur), piece * SUB, width, aligned4(probs_of(cur)), q);
        double wt[16];
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const int x = piece * SUB + 128 * (e >> 2) + 4 * lane + (e & 3);
          double v = none ? (x == 0 ? 1.0 : 0.0) : weight(z[e], w.zmax[cur], inv_t, tab);
          if (residual) v = fmax((none ? v : v * (1.0 / w.z[cur])) - w.beta * (double)fmaxf(q[e], 0.f), 0.0);
          for (int j = 0; j < drop; j++)
            if (w.refused[j] == x) v = 0.0;
          wt[e] = x < width ? v : 0.0;
        }
        token = search_piece(before, target, piece * SUB, wt);
        if (token < 0) token = 0;
      }
    }
    int *om = a.out_m + seq, *ot = a.out_tok + (size_t)seq * a.out_width, *op = a.out_path + (size_t)seq * a.out_width;
    for (int k = lane; k < a.out_width; k += 32) {
      op[k] = k <= m ? w.path[k] : -1;
      ot[k] = k < m ? w.tok[w.path[k + 1]] : k == m ? a.lo + token : -1;
    }
    if (lane == 0) *om = m;
  }
}

// Both launches; type: of the logits (f32, bf16, f16). A context's call has its rows in ea and its trees in a.trees.
template <typename T, bool CTX>
inline cudaError_t enqueue_t(const Args &a, const EpArgs &ea, int n_seq, int total_rows, cudaStream_t st) {
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
  const long long pieces = (long long)total_rows * a.n_sub;
  cfg.gridDim = dim3((unsigned)((pieces + STATS_THREADS / 32 - 1) / (STATS_THREADS / 32)));
  cfg.blockDim = dim3(STATS_THREADS);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, stats_kernel<T, CTX>, a, total_rows);
  if (e != cudaSuccess) return e;
  cfg.blockDim = dim3(WALK_THREADS);
  cfg.dynamicSmemBytes = a.n_sub * sizeof(double);
  cfg.gridDim = dim3(a.probs ? n_seq * CLUSTER : n_seq);
  if (a.probs) cfg.numAttrs = 2;
  return a.probs ? cudaLaunchKernelEx(&cfg, walk_kernel<T, true, CTX>, a, ea) : cudaLaunchKernelEx(&cfg, walk_kernel<T, false, CTX>, a, ea);
}
template <bool CTX>
inline cudaError_t enqueue(const Args &a, const EpArgs &ea, int type, int n_seq, int total_rows, cudaStream_t st) {
  switch (type) {
    case 0: return enqueue_t<float, CTX>(a, ea, n_seq, total_rows, st);
    case 1: return enqueue_t<bf16, CTX>(a, ea, n_seq, total_rows, st);
    default: return enqueue_t<__half, CTX>(a, ea, n_seq, total_rows, st);
  }
}

}  // namespace sampled
