// Log-probabilities of given tokens and the losses over them (post-training of the
// model: a preference loss over pairs of sequences, a clipped policy loss), with the
// gradient at the logits.
//
// Row t of the logits z and its target y give lp = z_y - m - log S, m = max_v z_v,
// S = sum_v exp(z_v - m); a target outside [0, V) makes the row not count: lp = 0,
// nothing of the row is read and its gradient is zero.  A loss is a function of the
// lp, so its gradient is dz_v = c ([v = y] - p_v) with c = dloss / dlp and p_v =
// exp(z_v - m) / S.  Everything but the passes over the logits is a few operations
// per token, done in float64 by one workgroup (a ratio of probabilities shows every
// digit of their logarithms, and a sequence's sum of them cancels against the
// reference's).
//
//   logit_part_kernel   reads the rows: (m, S) of every slice of a row
//   *_finish_kernel     merges a row's slices; loss, statistics, c of every token
//   logit_grad_kernel   reads the rows again and writes the gradient
//
// All three are HBM bound (V 4 or 2 bytes a row against a few exponentials).  No
// atomics: every sum has one order.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace axon {

constexpr int PART_THREADS = 256;
constexpr int PART_RUNS = 4;  // groups of 8 logits a thread holds at once
constexpr int GRAD_RUNS = 4;

// (m, s) joined with (m2, s2), both the sum of exp(value - maximum); a side that has
// seen nothing is (-inf, 0)
AXON_DEV void join_part(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  const float a = top == -INFINITY ? 0.f : top;  // -inf - (-inf) is not a number
  s = s * __expf(m - a) + s2 * __expf(m2 - a);
  m = top;
}

// exp(v - m) for many v and one m as 2^(v log2 e - m log2 e): one fused multiply-add
// and the hardware exponential.  m log2 e is rounded, which scales every result by
// the same 2^d; ``fix`` = 2^-d undoes it once, on the sum.  Where m log2 e may
// overflow (``low``: a row or slice of nothing but the type's lowest values, or
// -infinity), the difference is taken first.
struct ExpFrom {
  static constexpr float L = 1.4426950408889634f;
  float m, base, fix;
  bool low;
  AXON_DEV explicit ExpFrom(float top) {
    m = top == -INFINITY ? 0.f : top;  // -inf - (-inf) is not a number
    low = m < -2e38f;
    base = low ? 0.f : m * L;
    fix = low ? 1.f : 1.f - fmaf(m, L, -base) * 0.6931471805599453f;
  }
  template <int N>
  AXON_DEV void operator()(float (&v)[N]) const {
    if (!low) {
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = __builtin_amdgcn_exp2f(fmaf(v[j], L, -base));
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = __builtin_amdgcn_exp2f((v[j] - m) * L);
    }
  }
};

// N groups of 8 logits into a thread's (m, s)
template <int N>
AXON_DEV void take_runs(float& m, float& s, float (&v)[N][8]) {
  float top = m;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, v[k][j]);
  const ExpFrom e(top);
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    e(v[k]);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += v[k][j];
  }
  s = s * __expf(m - (top == -INFINITY ? 0.f : top)) + sum * e.fix;
  m = top;
}

// One slice (of ``slices``, ``cols`` wide) of one row a workgroup: its maximum and
// sum of exponentials.  Rows that do not count are skipped.
template <typename T>
__global__ void __launch_bounds__(PART_THREADS) logit_part_kernel(const T* __restrict__ z, int64_t ld, int V,
                                                                  const int32_t* __restrict__ targets, int64_t items,
                                                                  int slices, int cols, float2* __restrict__ part,
                                                                  float* __restrict__ logps) {
  __shared__ float red[2][PART_THREADS / 64];
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t t = it / slices;
    const int c0 = (int)(it % slices) * cols, c1 = min(V, c0 + cols);
    const int tg = targets[t];
    if (tg < 0 || tg >= V) {  // uniform over the workgroup
      if (logps && threadIdx.x == 0) logps[t] = 0.f;
      continue;
    }
    const T* row = z + t * ld;
    float m = -INFINITY, s = 0.f;
    for (int c = c0 + threadIdx.x * 8; c < c1; c += PART_THREADS * 8 * PART_RUNS) {
      float v[PART_RUNS][8];
#pragma unroll
      for (int k = 0; k < PART_RUNS; ++k) load_run8(row, c + k * PART_THREADS * 8, c1, v[k], -INFINITY);
      take_runs(m, s, v);
    }
    // over the workgroup: the common maximum first, then the sums scaled to it
    const float wm = wave_max(m);
    s = wave_sum(s * __expf(m - (wm == -INFINITY ? 0.f : wm)));
    __syncthreads();  // the last item's values have been read
    if ((threadIdx.x & 63) == 0) {
      red[0][threadIdx.x >> 6] = wm;
      red[1][threadIdx.x >> 6] = s;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      float M = red[0][0], S = red[1][0];
#pragma unroll
      for (int w = 1; w < PART_THREADS / 64; ++w) join_part(M, S, red[0][w], red[1][w]);
      if (part) part[it] = float2{M, S};
      if (logps) logps[t] = (float)((double)to_f32(row[tg]) - (double)M - log((double)S));
    }
  }
}

// (m, S) of row t from its slices, and its target's log-probability
template <typename T>
AXON_DEV double merge_row(const T* z, int64_t ld, const float2* part, int slices, int64_t t, int tg, float2& st) {
  const float2* p = part + t * slices;
  float m = p[0].x, s = p[0].y;
  for (int i = 1; i < slices; ++i) join_part(m, s, p[i].x, p[i].y);
  st = float2{m, s};
  return (double)to_f32(z[t * ld + tg]) - (double)m - log((double)s);
}

template <typename T>
__global__ void __launch_bounds__(256) logps_finish_kernel(const T* __restrict__ z, int64_t ld, int V,
                                                           const int32_t* __restrict__ targets, int64_t tokens,
                                                           const float2* __restrict__ part, int slices,
                                                           float* __restrict__ logps,
                                                           const float* __restrict__ dlogps, float2* __restrict__ stat,
                                                           float* __restrict__ coef) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= tokens) return;
  const int tg = targets[t];
  const bool ok = tg >= 0 && tg < V;
  float2 st = {0.f, 1.f};
  const double lp = ok ? merge_row(z, ld, part, slices, t, tg, st) : 0.0;
  if (logps) logps[t] = (float)lp;
  if (coef) {
    stat[t] = st;
    coef[t] = ok ? dlogps[t] : 0.f;
  }
}

AXON_DEV double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// sum over a workgroup of 1024 threads, in every thread
AXON_DEV double block_sum_f64(double v, double* red /* 16 */) {
  v = wave_sum_f64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
  for (int i = 0; i < 16; ++i) s += red[i];
  return s;
}

// log(1 + exp(v)) without overflow
AXON_DEV double softplus_f64(double v) { return fmax(v, 0.0) + log1p(exp(-fabs(v))); }

// Pairs (chosen 2i, rejected 2i + 1): s_j the sum of sequence j's lp, u_i = beta
// ((s_2i - ref_2i) - (s_2i+1 - ref_2i+1)), loss = mean of (1 - e) softplus(-u) + e
// softplus(u); dloss / ds_2i = beta / pairs (e sigmoid(u) - (1 - e) sigmoid(-u)).
// One workgroup: tokens, then sequences, then pairs.
template <typename T>
__global__ void __launch_bounds__(1024) preference_finish_kernel(
    const T* __restrict__ z, int64_t ld, int V, const int32_t* __restrict__ targets, int tokens,
    const float2* part /* may be stat */, int slices, const int32_t* __restrict__ cu, int seqs,
    const float* __restrict__ ref, float beta, float smoothing, float* __restrict__ loss,
    float* __restrict__ seq_logps, float* __restrict__ margins, double* __restrict__ lps, double* __restrict__ sums,
    float2* stat, float* __restrict__ coef) {
  __shared__ double red[16];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  for (int t = tid; t < tokens; t += 1024) {
    const int tg = targets[t];
    float2 st = {0.f, 1.f};
    lps[t] = tg >= 0 && tg < V ? merge_row(z, ld, part, slices, t, tg, st) : 0.0;
    stat[t] = st;
  }
  __syncthreads();
  for (int j = wave; j < seqs; j += 16) {
    const int t1 = min(tokens, cu[j + 1]);
    double s = 0.0;
    for (int t = max(0, cu[j]) + lane; t < t1; t += 64) s += lps[t];
    s = wave_sum_f64(s);
    if (lane == 0) {
      sums[j] = s;
      seq_logps[j] = (float)s;
    }
  }
  __syncthreads();
  const int pairs = seqs / 2;
  double total = 0.0;
  for (int i = tid; i < pairs; i += 1024) {
    double r0 = sums[2 * i], r1 = sums[2 * i + 1];
    if (ref) {
      r0 -= (double)ref[2 * i];
      r1 -= (double)ref[2 * i + 1];
    }
    const double u = (double)beta * (r0 - r1), e = (double)smoothing;
    margins[i] = (float)u;
    total += (1.0 - e) * softplus_f64(-u) + e * softplus_f64(u);
    const double yes = 1.0 / (1.0 + exp(-u)), no = 1.0 / (1.0 + exp(u));
    const double d = (double)beta / pairs * (e * yes - (1.0 - e) * no);
    sums[2 * i] = d;
    sums[2 * i + 1] = -d;
  }
  total = block_sum_f64(total, red);
  if (tid == 0) loss[0] = pairs > 0 ? (float)(total / pairs) : 0.f;
  __syncthreads();
  if (!coef) return;
  for (int t = tid; t < tokens; t += 1024) {
    const int tg = targets[t];
    coef[t] = tg >= 0 && tg < V ? (float)sums[seq_of_token(cu, seqs, t)] : 0.f;
  }
}

// Tokens with ratio q = exp(lp - old) and advantage A: -min(q A, clip(q, 1 - lo, 1 +
// hi) A) + k (exp(g) - g - 1), g = ref - lp, weighted by w: 1 / counted tokens or
// (per sequence) 1 / (sequences with counted tokens x the sequence's counted tokens).
// dloss / dlp = w (-(not clipped) q A + k (1 - exp(g))).  stats: the weighted means of
// the clipped term, of exp(g) - g - 1 and of the clipped tokens.
template <typename T>
__global__ void __launch_bounds__(1024) policy_finish_kernel(
    const T* __restrict__ z, int64_t ld, int V, const int32_t* __restrict__ targets, int tokens,
    const float2* part /* may be stat */, int slices, const int32_t* __restrict__ cu, int seqs,
    const float* __restrict__ old, const float* __restrict__ ref, const float* __restrict__ adv, float lo, float hi,
    float kl_coef, float* __restrict__ loss, float* __restrict__ stats, float* __restrict__ logps,
    double* __restrict__ weights, float2* stat, float* __restrict__ coef) {
  __shared__ double red[16];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  // the weights: counted tokens of all, or of each sequence
  double n = 0.0;
  if (cu) {
    for (int j = wave; j < seqs; j += 16) {
      const int t1 = min(tokens, cu[j + 1]);
      int own = 0;
      for (int t = max(0, cu[j]) + lane; t < t1; t += 64) own += targets[t] >= 0 && targets[t] < V;
      const double c = wave_sum_f64((double)own);
      if (lane == 0) weights[j] = c;
      n += lane == 0 && c > 0.0 ? 1.0 : 0.0;
    }
  } else {
    for (int t = tid; t < tokens; t += 1024) n += targets[t] >= 0 && targets[t] < V ? 1.0 : 0.0;
  }
  n = block_sum_f64(n, red);  // and the sequences' counts are visible
  double sum_l = 0.0, sum_s = 0.0, sum_k = 0.0, sum_c = 0.0;
  for (int t = tid; t < tokens; t += 1024) {
    const int tg = targets[t];
    const bool ok = tg >= 0 && tg < V;
    float2 st = {0.f, 1.f};
    double lp = 0.0, c = 0.0;
    if (ok) {
      lp = merge_row(z, ld, part, slices, t, tg, st);
      const double w = 1.0 / (cu ? n * weights[seq_of_token(cu, seqs, t)] : n);
      const double A = (double)adv[t], q = exp(lp - (double)old[t]);
      const double held = fmin(fmax(q, 1.0 - (double)lo), 1.0 + (double)hi);
      // A = 0: no term, also where the ratio overflows
      const double free_term = A == 0.0 ? 0.0 : q * A, held_term = A == 0.0 ? 0.0 : held * A;
      const bool clipped = free_term > held_term;
      const double surrogate = -(clipped ? held_term : free_term);
      double kl = 0.0, dkl = 0.0;
      if (ref) {
        const double g = (double)ref[t] - lp;
        dkl = -expm1(g);
        kl = -dkl - g;
      }
      const double k = (double)kl_coef;
      c = w * ((clipped ? 0.0 : -free_term) + (ref ? k * dkl : 0.0));
      sum_l += w * (surrogate + (ref ? k * kl : 0.0));
      sum_s += w * surrogate;
      sum_k += w * kl;
      sum_c += clipped ? w : 0.0;
    }
    logps[t] = (float)lp;
    if (coef) {
      stat[t] = st;
      coef[t] = (float)c;
    }
  }
  sum_l = block_sum_f64(sum_l, red);
  sum_s = block_sum_f64(sum_s, red);
  sum_k = block_sum_f64(sum_k, red);
  sum_c = block_sum_f64(sum_c, red);
  if (tid == 0) {
    loss[0] = (float)sum_l;
    stats[0] = (float)sum_s;
    stats[1] = (float)sum_k;
    stats[2] = (float)sum_c;
  }
}

// 8 logits to their gradients f exp(v - m), f = -c / S, and c more at the target, the
// ``at``-th of them if it is one
AXON_DEV void grad_run(float (&v)[8], const ExpFrom& e, float f, float c, int at) {
  e(v);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= f;
  if ((unsigned)at < 8u)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += j == at ? c : 0.f;
}

// dz of one slice of a row a workgroup.  z and dz may be one buffer: a thread reads
// what it then writes.
template <typename T, typename TO>
__global__ void __launch_bounds__(256) logit_grad_kernel(const T* z, int64_t ld, int V,
                                                         const int32_t* __restrict__ targets, int64_t items, int slices,
                                                         const float2* __restrict__ stat,
                                                         const float* __restrict__ coef, TO* dz, int64_t lddz) {
  constexpr int COLS = 256 * 8 * GRAD_RUNS;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t t = it / slices;
    const int c0 = (int)(it % slices) * COLS + threadIdx.x * 8;
    const float w = coef[t];
    const T* row = z + t * ld;
    TO* out = dz + t * lddz;
    float v[GRAD_RUNS][8];
    if (w == 0.f) {
#pragma unroll
      for (int k = 0; k < GRAD_RUNS; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[k][j] = 0.f;
    } else {
      const float2 st = stat[t];
      const int tg = targets[t];
      const ExpFrom e(st.x);
      const float f = -w / st.y * e.fix;
#pragma unroll
      for (int k = 0; k < GRAD_RUNS; ++k) load_run8(row, c0 + k * 2048, V, v[k], 0.f);
#pragma unroll
      for (int k = 0; k < GRAD_RUNS; ++k) grad_run(v[k], e, f, w, tg - (c0 + k * 2048));
    }
#pragma unroll
    for (int k = 0; k < GRAD_RUNS; ++k)
      if (c0 + k * 2048 < V) store_run8(out, c0 + k * 2048, V, v[k]);
  }
}

// ---------------------------------------------------------------- within a training step

// (m, S) of a row from the np (largest, sum) partials of its 64-column pieces, a
// workgroup a row; rows that do not count are skipped
__global__ void __launch_bounds__(256) piece_merge_kernel(const float2* __restrict__ pieces, int np, int V,
                                                          const int32_t* __restrict__ targets,
                                                          float2* __restrict__ stat) {
  __shared__ float red[2][4];
  const int t = blockIdx.x, tg = targets[t];
  if (tg < 0 || tg >= V) return;
  float m = -INFINITY, s = 0.f;
  for (int i = threadIdx.x; i < np; i += 256) {
    const float2 p = pieces[(int64_t)t * np + i];
    join_part(m, s, p.x, p.y);
  }
  const float wm = wave_max(m);
  s = wave_sum(s * __expf(m - (wm == -INFINITY ? 0.f : wm)));
  if ((threadIdx.x & 63) == 0) {
    red[0][threadIdx.x >> 6] = wm;
    red[1][threadIdx.x >> 6] = s;
  }
  __syncthreads();
  if (threadIdx.x) return;
  m = red[0][0];
  s = red[1][0];
#pragma unroll
  for (int w = 1; w < 4; ++w) join_part(m, s, red[0][w], red[1][w]);
  stat[t] = float2{m, s};
}

// The gradient as the training step's GEMM operand: bf16 in the row-pair layout,
// columns V .. ldl - 1 zero.  8 columns per thread (ldl % 32 == 0), every load
// unconditional (the padding columns hold whatever the buffer held and are not used);
// 8 lanes fill one 128-byte line of a row pair.
__global__ void __launch_bounds__(256) logit_grad_pair_kernel(const float* __restrict__ z, int ldl, int V, int T,
                                                              const int32_t* __restrict__ targets,
                                                              const float2* __restrict__ stat,
                                                              const float* __restrict__ coef, bf16* __restrict__ dlog) {
  const int tid = threadIdx.x;
  const int t = blockIdx.y * 2 + ((tid >> 2) & 1);
  const int v0 = (blockIdx.x * 32 + (tid >> 3)) * 32 + (tid & 3) * 8;
  if (t >= T || v0 >= ldl) return;
  float v[8];
  load_run8(z + (int64_t)t * ldl, v0, ldl, v, 0.f);
  const float w = coef[t];
  const float2 st = stat[t];
  const int tg = targets[t];
  const float f = -w / st.y;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    v[j] = w == 0.f || v0 + j >= V ? 0.f : __expf(v[j] - st.x) * f + (v0 + j == tg ? w : 0.f);
  Run8<bf16>::store(dlog + xp_off(t, v0, ldl), v);
}

// ---------------------------------------------------------------- launchers

namespace {

constexpr int64_t MAX_WGS = 1 << 20;  // more items than this: the workgroups loop

// Slices of a row for the statistics pass: whole rows once there are enough of
// them to fill the chip (8 workgroups on each of the 256 CUs), else as many slices
// as give that, of at least one group of 8 per thread
void part_shape(int64_t tokens, int V, int& slices, int& cols) {
  const int most = (V + PART_THREADS * 8 - 1) / (PART_THREADS * 8);
  const int want = (int)std::min<int64_t>(most, std::max<int64_t>(1, 2048 / std::max<int64_t>(tokens, 1)));
  const int runs = (most + want - 1) / want;
  cols = runs * PART_THREADS * 8;
  slices = (V + cols - 1) / cols;
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

// the workspace of a call
struct LossWs {
  float2* part;
  float2* stat;
  float* coef;
  double* lps;   // preference: [tokens]
  double* seq;   // [seqs]
};
size_t carve(int64_t tokens, int V, int64_t seqs, char* base, LossWs* ws) {
  int slices, cols;
  part_shape(tokens, V, slices, cols);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* p = base + at;
    at += up(bytes);
    return p;
  };
  LossWs w;
  w.part = (float2*)take((size_t)tokens * slices * sizeof(float2));
  w.stat = (float2*)take((size_t)tokens * sizeof(float2));
  w.coef = (float*)take((size_t)tokens * sizeof(float));
  w.lps = (double*)take((size_t)tokens * sizeof(double));
  w.seq = (double*)take((size_t)seqs * sizeof(double));
  if (ws) *ws = w;
  return at;
}

template <typename T>
int run_parts(const LogitRows& r, float2* part, float* logps, hipStream_t s) {
  int slices, cols;
  part_shape(r.tokens, r.V, slices, cols);
  const int64_t items = r.tokens * slices;
  logit_part_kernel<T><<<(unsigned)std::min(items, MAX_WGS), PART_THREADS, 0, s>>>(
      (const T*)r.z, r.ld, r.V, r.targets, items, slices, cols, part, slices == 1 ? logps : nullptr);
  return slices;
}

template <typename T>
void run_grad(const LogitRows& r, const LossWs& w, hipStream_t s) {
  const int slices = (r.V + 2048 * GRAD_RUNS - 1) / (2048 * GRAD_RUNS);
  const int64_t items = r.tokens * slices;
  const unsigned wgs = (unsigned)std::min(items, MAX_WGS);
  if (r.dz_bf16)
    logit_grad_kernel<T, bf16><<<wgs, 256, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets, items, slices, w.stat, w.coef,
                                                   (bf16*)r.dz, r.lddz);
  else
    logit_grad_kernel<T, float><<<wgs, 256, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets, items, slices, w.stat, w.coef,
                                                    (float*)r.dz, r.lddz);
}

template <typename T>
void logprobs(const LogitRows& r, float* logps, const float* dlogps, void* wsp, hipStream_t s) {
  if (r.tokens <= 0) return;
  LossWs w;
  carve(r.tokens, r.V, 0, (char*)wsp, &w);
  const int slices = run_parts<T>(r, w.part, logps, s);
  if (logps && slices == 1) return;
  logps_finish_kernel<T><<<(unsigned)((r.tokens + 255) / 256), 256, 0, s>>>(
      (const T*)r.z, r.ld, r.V, r.targets, r.tokens, w.part, slices, logps, dlogps, w.stat, dlogps ? w.coef : nullptr);
  if (dlogps) run_grad<T>(r, w, s);
}

template <typename T>
void preference(const LogitRows& r, const PreferenceArgs& a, void* wsp, hipStream_t s) {
  LossWs w;
  carve(r.tokens, r.V, a.seqs, (char*)wsp, &w);
  const int slices = r.tokens > 0 ? run_parts<T>(r, w.part, nullptr, s) : 1;
  preference_finish_kernel<T><<<1, 1024, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets, (int)r.tokens, w.part, slices,
                                                 a.cu, a.seqs, a.ref, a.beta, a.smoothing, a.loss, a.seq_logps,
                                                 a.margins, w.lps, w.seq, w.stat, r.dz ? w.coef : nullptr);
  if (r.dz && r.tokens > 0) run_grad<T>(r, w, s);
}

template <typename T>
void policy(const LogitRows& r, const PolicyArgs& a, void* wsp, hipStream_t s) {
  LossWs w;
  carve(r.tokens, r.V, a.seqs, (char*)wsp, &w);
  const int slices = r.tokens > 0 ? run_parts<T>(r, w.part, nullptr, s) : 1;
  policy_finish_kernel<T><<<1, 1024, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets, (int)r.tokens, w.part, slices, a.cu,
                                             a.seqs, a.old, a.ref, a.adv, a.lo, a.hi, a.kl_coef, a.loss, a.stats,
                                             a.logps, w.seq, w.stat, r.dz ? w.coef : nullptr);
  if (r.dz && r.tokens > 0) run_grad<T>(r, w, s);
}

}  // namespace

size_t loss_workspace_bytes(int64_t tokens, int V, int64_t seqs) { return carve(tokens, V, seqs, nullptr, nullptr); }

void launch_token_logps(const LogitRows& r, float* logps, void* ws, hipStream_t s) {
  if (r.z_bf16) logprobs<bf16>(r, logps, nullptr, ws, s);
  else logprobs<float>(r, logps, nullptr, ws, s);
}
void launch_token_logps_bwd(const LogitRows& r, const float* dlogps, void* ws, hipStream_t s) {
  if (r.z_bf16) logprobs<bf16>(r, nullptr, dlogps, ws, s);
  else logprobs<float>(r, nullptr, dlogps, ws, s);
}
void launch_preference_loss(const LogitRows& r, const PreferenceArgs& a, void* ws, hipStream_t s) {
  if (r.z_bf16) preference<bf16>(r, a, ws, s);
  else preference<float>(r, a, ws, s);
}
void launch_policy_loss(const LogitRows& r, const PolicyArgs& a, void* ws, hipStream_t s) {
  if (r.z_bf16) policy<bf16>(r, a, ws, s);
  else policy<float>(r, a, ws, s);
}

namespace {

void train_stat(const TrainLogits& r, hipStream_t s) {
  piece_merge_kernel<<<r.T, 256, 0, s>>>(r.lse_part, (r.V + LSE_COLS - 1) / LSE_COLS, r.V, r.targets, r.stat);
}

void train_grad(const TrainLogits& r, hipStream_t s) {
  logit_grad_pair_kernel<<<dim3((r.ldl / 32 + 31) / 32, (r.T + 1) / 2), 256, 0, s>>>(r.z, r.ldl, r.V, r.T, r.targets,
                                                                                     r.stat, r.coef, r.dlog);
}

}  // namespace

void launch_preference_train(const TrainLogits& r, const PreferenceArgs& a, hipStream_t s) {
  train_stat(r, s);
  preference_finish_kernel<float><<<1, 1024, 0, s>>>(r.z, r.ldl, r.V, r.targets, r.T, r.stat, 1, a.cu, a.seqs, a.ref,
                                                     a.beta, a.smoothing, a.loss, a.seq_logps, a.margins, r.lps, r.seq,
                                                     r.stat, r.coef);
  train_grad(r, s);
}

void launch_policy_train(const TrainLogits& r, const PolicyArgs& a, hipStream_t s) {
  train_stat(r, s);
  policy_finish_kernel<float><<<1, 1024, 0, s>>>(r.z, r.ldl, r.V, r.targets, r.T, r.stat, 1, a.cu, a.seqs, a.old, a.ref,
                                                 a.adv, a.lo, a.hi, a.kl_coef, a.loss, a.stats, a.logps, r.seq, r.stat,
                                                 r.coef);
  train_grad(r, s);
}

}  // namespace axon
