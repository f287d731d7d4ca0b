// Entry points of the stand-alone operators (see include/specvla.h): RMSNorm to 8 bits, the linear layer with its
// epilogue, verification of drafted tokens by random numbers.
#include "../../include/specvla.h"

#include <string.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <mutex>

#include "linear.cuh"
#include "norm_q8.cuh"
#include "sampled.cuh"

namespace {

size_t bytes_of(int type) {
  switch (type) {
    case SPECVLA_F32: return 4;
    case SPECVLA_BF16: case SPECVLA_F16: return 2;
    case SPECVLA_I8: case SPECVLA_E4M3: return 1;
    default: return 0;
  }
}
bool is_float(int type) { return type == SPECVLA_F32 || type == SPECVLA_BF16 || type == SPECVLA_F16; }
bool is_code(int type) { return type == SPECVLA_I8 || type == SPECVLA_E4M3; }
bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// Every kernel here may start beside its predecessor and waits for it before it touches memory. A launch that is
// refused fails this call and no other.
template <typename... P, typename... A>
int launch(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, int cluster, void *stream, A... args) {
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) == cudaSuccess) return SPECVLA_OK;
  cudaGetLastError();
  return SPECVLA_ERR_CUDA;
}

// ------------------------------------------------------------------ RMSNorm to 8 bits
template <typename T, int CODE>
int norm_launch(const norm_q8::Args &a, int rows, void *stream) {
  constexpr int V = 16 / (int)sizeof(T);
  const bool vec = a.d % V == 0 && aligned(a.x, 16) && a.ldx % V == 0 && (!a.r || (aligned(a.r, 16) && a.ldr % V == 0)) &&
                   (!a.s || (aligned(a.s, 16) && a.lds % V == 0)) && (!a.gain || aligned(a.gain, 16)) &&
                   aligned(a.q, V) && a.ldq % V == 0;
  // as many vectors a thread as it keeps; with fewer rows than SMs one, so that all loads are in flight at once
  const int step = vec ? V : 1, keep = 16 / step;
  const long long n = (a.d + step - 1) / step, per = rows <= 148 ? 1 : keep;
  const int threads = (int)std::min(1024ll, std::max(64ll, (n + 32 * per - 1) / (32 * per) * 32));
  // many rows: CTAs that copy ahead, 1024 threads on an SM
  if (vec && rows > 148 * 4) {
    auto go = [&](auto kernel, int nt) {
      const size_t smem = (size_t)(a.r ? 2 : 1) * nt * 32 * sizeof(T);
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
        cudaGetLastError();
        return (int)SPECVLA_ERR_CUDA;
      }
      const int ctas = (int)std::min<size_t>(1024 / nt, 200 * 1024 / smem);
      return launch(kernel, dim3(std::min(rows, 148 * ctas)), dim3(nt), smem, 1, stream, a);
    };
    if (a.d <= 64 * 32) return go(norm_q8::norm_q8_rows_kernel<T, CODE, 64>, 64);
    if (a.d <= 128 * 32) return go(norm_q8::norm_q8_rows_kernel<T, CODE, 128>, 128);
    if (a.d <= 256 * 32) return go(norm_q8::norm_q8_rows_kernel<T, CODE, 256>, 256);
    if (a.d <= 512 * 32) return go(norm_q8::norm_q8_rows_kernel<T, CODE, 512>, 512);
  }
  return launch(vec ? norm_q8::norm_q8_kernel<T, CODE, V> : norm_q8::norm_q8_kernel<T, CODE, 1>, dim3(rows), dim3(threads), 0, 1,
                stream, a);
}
int norm_entry(const norm_q8::Args &a, int rows, int type, int code_type, void *stream) {
  const bool i8 = code_type == SPECVLA_I8;
  using namespace norm_q8;
  switch (type) {
    case SPECVLA_F32: return i8 ? norm_launch<float, CODE_I8>(a, rows, stream) : norm_launch<float, CODE_E4M3>(a, rows, stream);
    case SPECVLA_BF16: return i8 ? norm_launch<bf16, CODE_I8>(a, rows, stream) : norm_launch<bf16, CODE_E4M3>(a, rows, stream);
    default: return i8 ? norm_launch<__half, CODE_I8>(a, rows, stream) : norm_launch<__half, CODE_E4M3>(a, rows, stream);
  }
}

// ------------------------------------------------------------------ linear layer
constexpr int MAX_DEVICES = 64;
std::mutex g_mutex;
struct Fit { bool known; int clusters[linear::MAX_S + 1]; } g_fit[MAX_DEVICES];

// Clusters of S CTAs that are resident at once, per device; 0: unknown.
const Fit *cluster_fit() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return nullptr;
  std::lock_guard<std::mutex> lock(g_mutex);
  Fit &f = g_fit[dev];
  if (f.known) return &f;
  auto kernel = linear::linear_slice_kernel<linear::KIND_16, float>;
  cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, linear::SMEM);
  for (int S = 1; S <= linear::MAX_S; S++) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(S * 64);
    cfg.blockDim = dim3(linear::THREADS);
    cfg.dynamicSmemBytes = linear::SMEM;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = S;
    at.val.clusterDim.y = 1;
    at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess) f.clusters[S] = n;
  }
  cudaGetLastError();
  f.known = true;
  return &f;
}

// How a call is cut. pair: tiles of 256 columns by pairs of CTAs; else tiles of 128 columns by clusters of S CTAs.
struct Plan {
  bool pair;
  int tn, tiles, chunks, S, grid, raster;
  int part;                                // K blocks per accumulator (linear::in_parts)
};
// parts: fp32 results of parts of K (linear::in_parts).
Plan plan_linear(int T, int N, int KB, bool parts, const Fit *fit) {
  Plan best = {};
  // few rows: one pass over W, every K block by one CTA; as many slices as run at once, four K blocks each at least
  Plan p = {};
  p.tiles = (N + linear::BM - 1) / linear::BM;
  p.chunks = (T + linear::MAX_TN - 1) / linear::MAX_TN;
  p.tn = ((T + p.chunks - 1) / p.chunks + 15) / 16 * 16;
  p.chunks = (T + p.tn - 1) / p.tn;
  p.S = 1;
  for (int s = 2; fit && s <= linear::MAX_S; s++)
    if ((long long)fit->clusters[s] >= (long long)p.tiles * p.chunks && KB / s >= 4) p.S = s;
  const int slice = (KB + p.S - 1) / p.S, held = 512 / linear::tmem_cols(p.tn), quarter = std::max(1, KB / 4);
  p.part = std::max(std::min(quarter, linear::SLICE_PART), (slice + held - 1) / held);
  best = p;
  // Clocks of a choice: K blocks, whose bytes come from L2 at 64 a clock and SM (slices: 256 + 2 tn, pairs: 256 + tn a block);
  // start, accumulator and exit; slices' hand-over. Neither is done before the weights have been read, at 3440 bytes a clock.
  const double read = (double)N * KB * linear::KBYTES / 3440 + 8000;
  const long long rounds = p.S > 1 ? 1 : ((long long)p.tiles * p.chunks + std::max(1, fit ? fit->clusters[1] : 1) - 1) / std::max(1, fit ? fit->clusters[1] : 1);
  double cost = rounds * (((KB + p.S - 1) / p.S) * (256. + 2 * p.tn) + 8000 + 24 * p.tn);
  if (p.S > 1) cost += 2500 + (p.tn / (8 * p.S) + 1) * 1000;
  cost = std::max(cost, read);
  if (p.chunks > 65535) cost = 1e300;      // (more than a grid's second dimension holds)
  // (tensor memory holds too few accumulators for parts of K about as short as a pair's)
  const bool coarse = parts && p.part > linear::PAIR_PART * 3 / 2;
  if (fit && fit->clusters[2] > 0 && (T > 16 || coarse)) {
    // Slices in several rounds start each anew, with nothing under way meanwhile; pairs stay resident and go on reading. 17 to 64 rows,
    // 22016 to 128256 columns, K 1024 to 8192: as slices int8 2 to 25 % longer, bf16 2 % shorter to 31 % longer; K 64 to 288 with 46 to
    // 526 rows: 33 to 57 % longer.
    if (rounds > 1 || coarse) cost = 1e300;
    const int pairs = fit->clusters[2], tiles = (N + 2 * linear::BM - 1) / (2 * linear::BM);
    for (int tn = parts ? linear::PART_TN : linear::MAX_TN; tn >= 32; tn -= 32) {
      const int chunks = (T + tn - 1) / tn;
      if (((T + chunks - 1) / chunks + 31) / 32 * 32 != tn) continue;    // (narrower chunks are no more)
      const long long waves = ((long long)tiles * chunks + pairs - 1) / pairs;
      const double k = std::max(read, waves * (KB * (256. + tn) + 8000 + 24 * tn));
      if (k < cost) {
        cost = k;
        best = {true, tn, tiles, chunks, 1, (int)std::min<long long>(pairs, (long long)tiles * chunks) * 2, 0, std::min(quarter, linear::PAIR_PART)};
      }
    }
  }
  // chunks side by side: 32 MB of X stay in L2 while W streams past (4764 x 22016 x 4096 in e4m3: 290 MB read from memory with
  // eight, 116 with all nineteen)
  best.raster = (int)std::min<long long>(best.chunks, std::max<long long>(4, (32ll << 20) / ((long long)best.tn * KB * linear::KBYTES)));
  return best;
}

template <int KIND, typename OUT>
int linear_launch(const CUtensorMap &mw, const CUtensorMap &mx, const linear::Args &a, const Plan &p, void *stream) {
  auto slice = linear::linear_slice_kernel<KIND, OUT>;
  auto pair = linear::linear_pair_kernel<KIND, OUT>;
  if ((p.pair ? cudaFuncSetAttribute(pair, cudaFuncAttributeMaxDynamicSharedMemorySize, linear::SMEM)
              : cudaFuncSetAttribute(slice, cudaFuncAttributeMaxDynamicSharedMemorySize, linear::SMEM)) != cudaSuccess) {
    cudaGetLastError();
    return SPECVLA_ERR_CUDA;
  }
  if (p.pair)
    return launch(pair, dim3(p.grid), dim3(linear::PAIR_THREADS), linear::SMEM, 2, stream, mw, mx, a,
                  linear::PairTiles{p.tiles, p.chunks, p.raster});
  return launch(slice, dim3(p.tiles * p.S, p.chunks), dim3(linear::THREADS), linear::SMEM, p.S, stream, mw, mx, a, p.S);
}
template <int KIND>
int linear_out(int out_type, const CUtensorMap &mw, const CUtensorMap &mx, const linear::Args &a, const Plan &p, void *stream) {
  switch (out_type) {
    case SPECVLA_F32: return linear_launch<KIND, float>(mw, mx, a, p, stream);
    case SPECVLA_BF16: return linear_launch<KIND, bf16>(mw, mx, a, p, stream);
    default: return linear_launch<KIND, __half>(mw, mx, a, p, stream);
  }
}

std::atomic<unsigned long long> g_linear_wait_ns{gemm_tc::WAIT_LIMIT_NS};   // of the next call (specvla_linear_fault_test)
std::atomic<int> g_linear_withhold{0};
constexpr int MAX_ROW = 1 << 30;         // elements of a row: offsets within one are 32-bit

}  // namespace

int specvla_rmsnorm_q8(const specvla_norm_args *n, void *stream) {
  if (!n || !n->x || !n->codes || !n->scale || n->rows < 1 || n->d < 1 || n->d > MAX_ROW || !is_float(n->type) || !is_code(n->code_type))
    return SPECVLA_ERR_INVALID_ARG;
  if (n->ldx < n->d || n->ld_codes < n->d || (n->residual && n->ld_residual < n->d) || (n->sum && n->ld_sum < n->d) || !(n->eps >= 0.f))
    return SPECVLA_ERR_INVALID_ARG;
  const size_t e = bytes_of(n->type);
  if (!aligned(n->x, e) || !aligned(n->residual, e) || !aligned(n->sum, e) || !aligned(n->gain, 4) || !aligned(n->scale, 4))
    return SPECVLA_ERR_INVALID_ARG;
  const norm_q8::Args a = {n->x, n->residual, n->gain, n->sum, static_cast<unsigned char *>(n->codes), n->scale, n->rows,
                           n->d, n->ldx, n->ld_residual, n->ld_sum, n->ld_codes, n->eps, 1};
  return norm_entry(a, n->rows, n->type, n->code_type, stream);
}

int specvla_quantize_rows(const void *X, int type, int rows, int d, long long ldx, void *codes, int code_type,
                          long long ld_codes, float *scale, void *stream) {
  if (!X || !codes || !scale || rows < 1 || d < 1 || d > MAX_ROW || ldx < d || ld_codes < d || !is_float(type) || !is_code(code_type) ||
      !aligned(X, bytes_of(type)) || !aligned(scale, 4))
    return SPECVLA_ERR_INVALID_ARG;
  const norm_q8::Args a = {X, nullptr, nullptr, nullptr, static_cast<unsigned char *>(codes), scale, rows, d, ldx, 0, 0, ld_codes, 0.f, 0};
  return norm_entry(a, rows, type, code_type, stream);
}

int specvla_linear_fault_test(long long wait_limit_ns, int withhold_k_block) {
  if (wait_limit_ns < 1000 || withhold_k_block < -1) return SPECVLA_ERR_INVALID_ARG;
  g_linear_wait_ns = (unsigned long long)wait_limit_ns;
  g_linear_withhold = withhold_k_block + 1;
  return SPECVLA_OK;
}

int specvla_linear(const specvla_linear_args *l, void *stream) {
  if (!l || !l->X || !l->W || !l->Y || !l->status || l->T < 1 || l->N < 1 || l->K < 1) return SPECVLA_ERR_INVALID_ARG;
  const bool codes = is_code(l->type);
  if (!(codes || l->type == SPECVLA_BF16 || l->type == SPECVLA_F16) || !is_float(l->out_type)) return SPECVLA_ERR_INVALID_ARG;
  if (l->act < SPECVLA_ACT_NONE || l->act > SPECVLA_ACT_SILU) return SPECVLA_ERR_INVALID_ARG;
  if (!codes && (l->x_scale || l->w_scale)) return SPECVLA_ERR_INVALID_ARG;
  if (l->K > MAX_ROW / 2 || l->N > MAX_ROW || l->T > MAX_ROW) return SPECVLA_ERR_INVALID_ARG;   // (coordinates of copies are 32-bit)
  if (l->type == SPECVLA_I8 && l->K > 131071) return SPECVLA_ERR_INVALID_ARG;       // 2^14 K must fit 31 bits
  const long long e = (long long)bytes_of(l->type), eo = (long long)bytes_of(l->out_type);
  // (a single row has no distance to the next)
  const long long bytes = l->K * e, one = (bytes + 15) / 16 * 16;
  const long long ldx = l->T == 1 ? one : l->ldx * e, ldw = l->N == 1 ? one : l->ldw * e;
  if ((l->T > 1 && l->ldx < l->K) || (l->N > 1 && l->ldw < l->K) || ldx % 16 || ldw % 16 || !aligned(l->X, 16) || !aligned(l->W, 16))
    return SPECVLA_ERR_INVALID_ARG;
  if ((l->T > 1 && (l->ldy < l->N || (l->residual && l->ld_residual < l->N))) || !aligned(l->Y, eo) || !aligned(l->residual, eo) ||
      !aligned(l->x_scale, 4) || !aligned(l->w_scale, 4) || !aligned(l->bias, 4) || !aligned(l->status, 4))
    return SPECVLA_ERR_INVALID_ARG;
  linear::Args a = {};
  a.T = l->T, a.N = l->N;
  a.KB = (int)((bytes + linear::KBYTES - 1) / linear::KBYTES);
  a.act = l->act;
  a.pairs = l->N % 2 == 0 && aligned(l->Y, 2 * eo) && (l->T == 1 || l->ldy % 2 == 0) &&
            (!l->residual || (aligned(l->residual, 2 * eo) && (l->T == 1 || l->ld_residual % 2 == 0)));
  a.x_scale = l->x_scale, a.w_scale = l->w_scale, a.bias = l->bias;
  a.res = l->residual, a.ldr = l->ld_residual;
  a.y = l->Y, a.ldy = l->ldy;
  a.status = l->status;
  a.wait_ns = g_linear_wait_ns.exchange(gemm_tc::WAIT_LIMIT_NS);  // the test hook holds for one call
  a.withhold = g_linear_withhold.exchange(0);
  const int kind = l->type == SPECVLA_I8 ? linear::KIND_I8 : l->type == SPECVLA_E4M3 ? linear::KIND_E4M3 : linear::KIND_16;
  const Plan p = plan_linear(l->T, l->N, a.KB, kind != linear::KIND_I8 && l->out_type == SPECVLA_F32, cluster_fit());
  if (!p.pair && p.chunks > 65535) return SPECVLA_ERR_INVALID_ARG;
  a.tn = p.tn;
  a.part = p.part;
  a.idesc = linear::make_idesc(kind, l->type == SPECVLA_BF16, p.pair ? 2 * linear::BM : linear::BM, a.tn);
  CUtensorMap mw, mx;
  if (!linear::make_map(&mw, l->W, l->N, bytes, ldw, linear::BM) || !linear::make_map(&mx, l->X, l->T, bytes, ldx, p.pair ? a.tn / 2 : a.tn)) {
    cudaGetLastError();
    return SPECVLA_ERR_CUDA;
  }
  switch (kind) {
    case linear::KIND_16: return linear_out<linear::KIND_16>(l->out_type, mw, mx, a, p, stream);
    case linear::KIND_I8: return linear_out<linear::KIND_I8>(l->out_type, mw, mx, a, p, stream);
    default: return linear_out<linear::KIND_E4M3>(l->out_type, mw, mx, a, p, stream);
  }
}

// ------------------------------------------------------------------ verification by random numbers
size_t specvla_verify_sampled_scratch_bytes(int n_seq, int rows, int lo, int hi) {
  if (n_seq < 1 || rows < 1 || rows > SPECVLA_MAX_TREE_ROWS || lo < 0 || hi <= lo || hi - lo > sampled::MAX_IDS ||
      n_seq > INT_MAX / (rows * sampled::CLUSTER))
    return 0;
  const size_t pieces = (size_t)n_seq * rows * sampled::pieces_of(hi - lo);
  return pieces * (sizeof(double) + sizeof(float));
}

int specvla_verify_sampled(const specvla_verify_args *v, void *scratch, size_t scratch_bytes, void *stream) {
  if (!v || !v->logits || !v->tokens || !v->parent || !v->u || !v->accept_len || !v->path || !v->tokens_out || !scratch)
    return SPECVLA_ERR_INVALID_ARG;
  const size_t need = specvla_verify_sampled_scratch_bytes(v->n_seq, v->rows, v->lo, v->hi);
  if (need == 0 || v->hi > v->vocab || v->ld_logits < v->vocab || (v->draft_probs && v->ld_draft < v->vocab) || !is_float(v->logits_type) ||
      !(v->temperature > 0.f) || v->temperature > sampled::MAX_TEMPERATURE)
    return SPECVLA_ERR_INVALID_ARG;
  if (!aligned(scratch, 8) || !aligned(v->logits, bytes_of(v->logits_type)) || !aligned(v->draft_probs, 4) || !aligned(v->tokens, 4) ||
      !aligned(v->parent, 4) || !aligned(v->n_rows, 4) || !aligned(v->u, 4) || !aligned(v->accept_len, 4) || !aligned(v->path, 4) ||
      !aligned(v->tokens_out, 4))
    return SPECVLA_ERR_INVALID_ARG;
  if (scratch_bytes < need) return SPECVLA_ERR_CAPACITY;
  sampled::Args a = {};
  a.logits = v->logits, a.ld = v->ld_logits;
  a.probs = v->draft_probs, a.ld_probs = v->ld_draft;
  a.lo = v->lo, a.hi = v->hi;
  a.n_sub = sampled::pieces_of(v->hi - v->lo);
  a.temperature = v->temperature;
  a.factor = sampled::exp_factor(v->temperature);
  a.u = v->u;
  a.tokens = v->tokens, a.parent = v->parent, a.n_rows = v->n_rows;
  a.rows = v->rows;
  a.sub_sum = static_cast<double *>(scratch);
  a.sub_max = reinterpret_cast<float *>(a.sub_sum + (size_t)v->n_seq * v->rows * a.n_sub);
  a.out_m = v->accept_len, a.out_tok = v->tokens_out, a.out_path = v->path;
  a.out_width = v->rows;
  const EpArgs none = {};
  const int total = v->n_seq * v->rows;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t err = v->logits_type == SPECVLA_F32    ? sampled::enqueue<float, false>(a, none, v->n_seq, total, st)
                          : v->logits_type == SPECVLA_BF16 ? sampled::enqueue<bf16, false>(a, none, v->n_seq, total, st)
                                                           : sampled::enqueue<__half, false>(a, none, v->n_seq, total, st);
  if (err == cudaSuccess) return SPECVLA_OK;
  cudaGetLastError();
  return SPECVLA_ERR_CUDA;
}
