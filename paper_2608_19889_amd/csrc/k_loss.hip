// Log-probabilities of given tokens and the losses over them (post-training of the
// model: a preference loss over pairs of sequences, a clipped policy loss), with the
// gradient at the logits.
//
// Row t of the logits z and its target y give lp = z_y - m - log S, m = max_v z_v,
// S = sum_v exp(z_v - m); a target outside [0, V) makes the row not count: lp = 0,
// nothing of the row is read and its gradient is zero.  A loss is a function of the
// lp, so its gradient is dz_v = c ([v = y] - p_v) with c = dloss / dlp and p_v =
// exp(z_v - m) / S.  S is a float32 sum of float32 exponentials.  What follows is a few
// operations per token: log-probabilities are joined and sums over tokens added in
// float64 (a sequence's cancels against the reference's); a policy token's own terms are
// float32 (see policy_token).
//
//   logit_part_kernel       reads the rows: (m, S) of every slice of a row
//   *_finish_kernel         one workgroup joins the rows' slices; loss, statistics, c of
//                           every token (the policy's: the loss alone, and in a step)
//   preference_few_kernel   the same and the gradient, for few tokens, by every workgroup
//   logit_grad_kernel       reads the rows again and writes the gradient
// where c depends on the row alone (the policy loss, a caller's own):
//   policy_weights_kernel   the tokens' weights (of few tokens: by each row's workgroup)
//   logit_row_kernel        a row's (m, S), terms, c and gradient in one pass
//   policy_terms_kernel     the terms from logit_part_kernel's (m, S): many tokens' loss
//                           alone
//   policy_sum_kernel       adds up the loss's terms
//
// All are HBM bound (V 4 or 2 bytes a row against a few exponentials).  No atomics:
// every sum has one order.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace axon {

constexpr int PART_THREADS = 256;
constexpr int PART_RUNS = 4;  // groups of 8 logits a thread holds at once
constexpr int GRAD_RUNS = 4;
constexpr int FEW = 256;  // tokens that every workgroup goes through by itself, one a thread

// exp(x) of the joins, x <= 0, with log2 e in two parts: as one float it is 1.3e-8 of
// itself too small, and x may be most of a logit's distance from the row's maximum, so
// every sum came out too large by the same share, which a sequence's log-probability adds
// up.  Mean error of log S, normal logits of deviation 2, 32000 float32: -4.7e-8 ->
// -2e-10; 128256 bf16: -8.0e-8 -> -2.3e-8.
AXON_DEV float exp_join(float x) { return __builtin_amdgcn_exp2f(fmaf(x, 1.442695022f, x * 1.925963e-8f)); }

// (m, s) joined with (m2, s2), both the sum of exp(value - maximum); a side that has
// seen nothing is (-inf, 0)
AXON_DEV void join_part(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  const float a = top == -INFINITY ? 0.f : top;  // -inf - (-inf) is not a number
  s = s * exp_join(m - a) + s2 * exp_join(m2 - a);
  m = top;
}

// the sum of a single logit, as its own maximum
AXON_DEV float one_exp(float v) { return v == -INFINITY ? 0.f : v - v + 1.f; }  // (infinity or NaN: NaN)

// 1 where a row's wide accesses would be off by 2 bytes (they take 20% longer than any
// multiple of 4): its first logit goes alone then, the groups of 8 start after it
AXON_DEV int odd_head(const float*) { return 0; }
AXON_DEV int odd_head(const bf16* row) { return (int)((uintptr_t)row >> 1 & 1); }

// exp(v - m) for many v <= m as 2^((v - m) log2 e).  The difference comes first: of equal
// values it is 0 and the power 1, and its rounding grows with |v - m| alone.  (One
// operation less, 2^(v log2 e - m log2 e) with a rounded m log2 e, is off by that
// rounding, which grows with |m| and overflows the power.)
struct ExpFrom {
  float m;
  AXON_DEV explicit ExpFrom(float top) : m(top == -INFINITY ? 0.f : top) {}  // -inf - (-inf) is not a number
  AXON_DEV float operator()(float v) const { return __builtin_amdgcn_exp2f((v - m) * 1.4426950408889634f); }
};

// N groups of 8 logits into a thread's (m, s)
template <int N>
AXON_DEV void take_runs(float& m, float& s, const float (&v)[N][8]) {
  float top = m;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, v[k][j]);
  const ExpFrom e(top);
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += e(v[k][j]);
  s = s * exp_join(m - e.m) + sum;
  m = top;
}

// N groups of 8 of the columns c, c + stride, .. of [0, n), n >= 8, into a thread's (m, s).
// CUT: groups at the end, read whole at its last columns and counted where they are
// still to come.  (Every load is unconditional: one under a branch whose other arm fills
// the same registers is waited for at once.)
template <int N, bool CUT, typename T>
AXON_DEV void read_runs(const T* row, int c, int stride, int n, float& m, float& s) {
  Run8<T> r[N];
#pragma unroll
  for (int k = 0; k < N; ++k) r[k].load(row + (CUT ? min(c + k * stride, n - 8) : c + k * stride));
  float v[N][8];
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[k][j] = !CUT || min(c + k * stride, n - 8) + j >= c + k * stride ? r[k][j] : -INFINITY;
  take_runs(m, s, v);
}

// (m, s) over a workgroup of PART_THREADS, in every thread
AXON_DEV void join_block(float& m, float& s, float (*red)[PART_THREADS / 64]) {
  const float wm = wave_max(m);
  s = wave_sum(s * exp_join(m - (wm == -INFINITY ? 0.f : wm)));
  __syncthreads();  // the last values have been read
  if ((threadIdx.x & 63) == 0) {
    red[0][threadIdx.x >> 6] = wm;
    red[1][threadIdx.x >> 6] = s;
  }
  __syncthreads();
  m = red[0][0];
  s = red[1][0];
#pragma unroll
  for (int w = 1; w < PART_THREADS / 64; ++w) join_part(m, s, red[0][w], red[1][w]);
}

// A token's log-probability, for whichever is asked for; 0 where it does not count
template <typename T>
AXON_DEV void put_logp(bool counts, const T* chosen, float m, float s, float* logp, double* lp) {
  if (!logp && !lp) return;
  const double v = counts ? (double)to_f32(*chosen) - (double)m - log((double)s) : 0.0;
  if (logp) *logp = (float)v;
  if (lp) *lp = v;
}

// One slice (of ``slices``, ``cols`` wide) of one row a workgroup: its maximum and
// sum of exponentials, and, of whole rows, the target's log-probability.  Rows that do
// not count are skipped.  chosen: the targets' logits too.
template <typename T>
__global__ void __launch_bounds__(PART_THREADS, 8) logit_part_kernel(const T* __restrict__ z, int64_t ld, int V,
                                                                  const int32_t* __restrict__ targets, int64_t items,
                                                                  int slices, int cols, float2* __restrict__ part,
                                                                  float* __restrict__ logps, double* __restrict__ lps,
                                                                  float* __restrict__ chosen) {
  constexpr int STRIDE = PART_THREADS * 8, BLOCK = STRIDE * PART_RUNS;
  __shared__ float red[2][PART_THREADS / 64];
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t t = it / slices;
    const int tg = targets[t];
    if (tg < 0 || tg >= V) {  // uniform over the workgroup
      if (threadIdx.x == 0) put_logp(false, z, 0.f, 1.f, logps ? logps + t : nullptr, lps ? lps + t : nullptr);
      continue;
    }
    const T* row = z + t * ld;
    const int h = odd_head(row), c0 = (int)(it % slices) * cols, n = min(V - h - c0, cols);
    float m = -INFINITY, s = 0.f;
    if (h && c0 == 0 && threadIdx.x == 0) join_part(m, s, to_f32(row[0]), one_exp(to_f32(row[0])));
    row += h + c0;
    if (n >= 8) {
      int c = 0;
      for (; c + BLOCK <= n; c += BLOCK) read_runs<PART_RUNS, false>(row, c + threadIdx.x * 8, STRIDE, n, m, s);
      for (; c < n; c += STRIDE) read_runs<1, true>(row, c + threadIdx.x * 8, STRIDE, n, m, s);
    } else if ((int)threadIdx.x < n) {
      const float v = to_f32(row[threadIdx.x]);
      join_part(m, s, v, one_exp(v));
    }
    join_block(m, s, red);
    if (threadIdx.x == 0) {
      if (part) part[it] = float2{m, s};
      if (chosen && c0 == 0) chosen[t] = to_f32(z[t * ld + tg]);
      put_logp(true, z + t * ld + tg, m, s, logps ? logps + t : nullptr, lps ? lps + t : nullptr);
    }
  }
}

// (m, s) of token t from its slices, at most 16, all under way together
AXON_DEV float2 join_slices(const float2* part, int64_t t, int slices) {
  float2 p[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) p[i] = part[t * slices + min(i, slices - 1)];
  float m = p[0].x, s = p[0].y;
#pragma unroll
  for (int i = 1; i < 16; ++i)
    if (i < slices) join_part(m, s, p[i].x, p[i].y);
  return float2{m, s};
}

// log-probabilities from the rows' slices
template <typename T>
__global__ void __launch_bounds__(256) logps_finish_kernel(const T* __restrict__ z, int64_t ld, int V,
                                                           const int32_t* __restrict__ targets, int64_t tokens,
                                                           const float2* __restrict__ part, int slices,
                                                           float* __restrict__ logps) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= tokens) return;
  const int tg = targets[t];
  const bool counts = tg >= 0 && tg < V;
  const float2 st = counts ? join_slices(part, t, slices) : float2{0.f, 1.f};
  put_logp(counts, z + t * ld + tg, st.x, st.y, logps + t, nullptr);
}

AXON_DEV double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// N sums over a workgroup of THREADS, in every thread
template <int THREADS = 1024, int N>
AXON_DEV void block_sums_f64(double (&v)[N], double (*red)[16]) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = wave_sum_f64(v[k]);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k)
    if ((threadIdx.x & 63) == 0) red[k][threadIdx.x >> 6] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] = 0.0;
    for (int i = 0; i < THREADS / 64; ++i) v[k] += red[k][i];
  }
}

// The sequence of a token, for a workgroup of 1024 threads that look up many: the
// boundaries of up to CU_HELD sequences are kept in LDS (a search in memory waits for
// every step).  A barrier between hold() and of().
constexpr int CU_HELD = 1024;
struct SeqLookup {
  const int32_t* cu;
  int seqs;
  AXON_DEV void hold(int32_t* held) const {
    if (cu && seqs <= CU_HELD)
      for (int i = threadIdx.x; i < seqs; i += 1024) held[i] = cu[i];
  }
  AXON_DEV int of(const int32_t* held, int t) const {
    return seqs <= CU_HELD ? seq_of_token(held, seqs, t) : seq_of_token(cu, seqs, t);
  }
};

// log(1 + exp(v)) without overflow
AXON_DEV double softplus_f64(double v) { return fmax(v, 0.0) + log1p(exp(-fabs(v))); }

// Pairs (chosen 2i, rejected 2i + 1): s_j the sum of sequence j's lp, u_i = beta
// ((s_2i - ref_2i) - (s_2i+1 - ref_2i+1)), loss = mean of (1 - e) softplus(-u) + e
// softplus(u); dloss / ds_2i = beta / pairs (e sigmoid(u) - (1 - e) sigmoid(-u)).
// One workgroup, from the tokens' lps: sums [seqs] in, dloss / ds out; the
// results only where ``write``.
struct PairOut {
  float *loss, *seq_logps, *margins;
};
template <int THREADS>
AXON_DEV void pair_coefs(const double* lps, int tokens, const int32_t* cu, int seqs, const float* ref, float beta,
                         float smoothing, double* sums, double (*red)[16], bool write, PairOut out) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  for (int j = wave; j < seqs; j += THREADS / 64) {
    const int t1 = min(tokens, cu[j + 1]);
    double s = 0.0;
#pragma unroll 8
    for (int t = max(0, cu[j]) + lane; t < t1; t += 64) s += lps[t];
    s = wave_sum_f64(s);
    if (lane == 0) {
      sums[j] = s;
      if (write) out.seq_logps[j] = (float)s;
    }
  }
  __syncthreads();
  const int pairs = seqs / 2;
  double total[1] = {};
  for (int i = tid; i < pairs; i += THREADS) {
    double r0 = sums[2 * i], r1 = sums[2 * i + 1];
    if (ref) {
      r0 -= (double)ref[2 * i];
      r1 -= (double)ref[2 * i + 1];
    }
    const double u = (double)beta * (r0 - r1), e = (double)smoothing;
    if (write) out.margins[i] = (float)u;
    total[0] += (1.0 - e) * softplus_f64(-u) + (e > 0.0 ? e * softplus_f64(u) : 0.0);  // (u may be infinite)
    const double yes = 1.0 / (1.0 + exp(-u)), no = 1.0 / (1.0 + exp(u));
    const double d = (double)beta / pairs * (e * yes - (1.0 - e) * no);
    sums[2 * i] = d;
    sums[2 * i + 1] = -d;
  }
  block_sums_f64<THREADS>(total, red);  // (its barriers make the sequences' coefficients visible)
  if (write && tid == 0) out.loss[0] = pairs > 0 ? (float)(total[0] / pairs) : 0.f;
}

// slices > 1: the tokens' lps and stat first (else the rows' pass has left them)
template <typename T>
__global__ void __launch_bounds__(1024) preference_finish_kernel(
    const T* __restrict__ z, int64_t ld, int V, const int32_t* __restrict__ targets, int tokens,
    const float2* __restrict__ part, int slices, const int32_t* __restrict__ cu, int seqs,
    const float* __restrict__ ref, float beta, float smoothing, PairOut out, double* __restrict__ lps,
    double* __restrict__ sums, float2* __restrict__ stat, float* __restrict__ coef) {
  __shared__ double red[1][16];
  __shared__ int32_t held[CU_HELD];
  const SeqLookup seq{cu, seqs};
  const int tid = threadIdx.x;
  seq.hold(held);
  if (slices > 1)
    for (int64_t t = tid; t < tokens; t += 1024) {
      const int tg = targets[t];
      const bool counts = tg >= 0 && tg < V;
      const float2 st = counts ? join_slices(part, t, slices) : float2{0.f, 1.f};
      put_logp(counts, z + t * ld + tg, st.x, st.y, nullptr, lps + t);
      stat[t] = st;
    }
  __syncthreads();
  pair_coefs<1024>(lps, tokens, cu, seqs, ref, beta, smoothing, sums, red, true, out);
  if (!coef) return;
#pragma unroll 4
  for (int t = tid; t < tokens; t += 1024) {
    const int tg = targets[t];
    const double d = sums[seq.of(held, t)];
    coef[t] = tg >= 0 && tg < V ? (float)d : 0.f;
  }
}

// exp(x) - x - 1, from e = exp(x) - 1.  The difference of the two cancels as x does (a
// policy that has hardly moved from its reference), so up to 1/2 it is the series
// x^2 (1/2! + x/3! + .. + x^8/10!), whose rest is below 2^-31 of it.
AXON_DEV float kl_term(float x, float e) {
  if (!(fabsf(x) < 0.5f)) return x == INFINITY ? x : e - x;
  float s = 2.75573192e-7f;
  const float over[8] = {2.75573192e-6f, 2.48015873e-5f, 1.98412698e-4f, 1.38888889e-3f,
                         8.33333333e-3f, 4.16666667e-2f, 1.66666667e-1f, 0.5f};
#pragma unroll
  for (int i = 0; i < 8; ++i) s = fmaf(s, x, over[i]);
  return x * x * s;
}

struct PolicyTerms {
  float lp, c;  // log-probability; dloss / dlp of weight 1
  float surrogate, kl;
  bool clipped;
};
// one token (see policy_finish_kernel), from its logit and its row's (m, S), in float32:
// where one workgroup does a batch's tokens, float64 exponentials took longer than
// everything else there.  The log-probability's three terms and the other policy's are
// added with their rounding errors kept (Knuth's two-sum), so the ratio is off by the
// last digits of S and of a logarithm below 1/2, and by its own exponential's.
AXON_DEV PolicyTerms policy_token(float z, float m, float s, float old, float A, bool has_ref, float ref, float lo,
                                  float hi, float kl_coef) {
  auto sum = [](float a, float b, float& low) {  // a + b, its rounding error added to low
    const float r = a + b, bb = r - a;
    low += (a - (r - bb)) + (b - bb);
    return r;
  };
  PolicyTerms p;
  // log s = k log 2 + log f, s = 2^k f, f within a factor of root 2 of 1 (Cody and Waite's
  // split: k times the first 16 bits of log 2 is exact, k times the rest goes to low): log
  // f is small, and so is its rounding, where log s as one float is off by up to 5e-7
  const float k = (float)__builtin_amdgcn_frexp_expf(s * 0.70710678f);
  float low = k * -1.42860682e-6f;
  const float f = __builtin_amdgcn_ldexpf(s, (int)-k);
  const float lp = sum(sum(sum(z, -m, low), k * -0.693145752f, low), -logf(f), low);
  p.lp = fabsf(lp) < INFINITY ? lp + low : lp;  // (an infinite sum's error is not a number)
  float el = low;
  const float d = sum(lp, -old, el), e = expf(d);
  const float q = fabsf(d) < 100.f ? e * (1.f + el) : e;  // (beyond, 0 or infinity, and el may be a whole term)
  const float held = fminf(fmaxf(q, 1.f - lo), 1.f + hi);
  // A = 0: no term, also where the ratio overflows
  const float free_term = A == 0.f ? 0.f : q * A, held_term = A == 0.f ? 0.f : held * A;
  p.clipped = free_term > held_term;
  p.surrogate = -(p.clipped ? held_term : free_term);
  p.c = p.clipped ? 0.f : -free_term;
  p.kl = 0.f;
  if (has_ref) {
    float er = -low;
    const float g = sum(ref, -lp, er), x = fabsf(g) < INFINITY ? g + er : g, dkl = -expm1f(x);
    p.kl = kl_term(x, -dkl);
    if (kl_coef > 0.f) p.c += kl_coef * dkl;  // kl_coef = 0: no term, also where it is infinite
  }
  return p;
}

// counted tokens of each sequence into weights[seqs] (cu), and in every thread the
// number of sequences that have some, or (no cu) of all counted tokens.  1024 threads.
AXON_DEV double policy_counts(const int32_t* targets, int tokens, int V, const int32_t* cu, int seqs, double* weights,
                              double (*red)[16]) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  // of the tokens t, t + step, .. below t1, 8 loads at a time
  auto counted = [&](int t, int step, int t1) {
    int own = 0;
    for (; t < t1; t += 8 * step) {
      int tg[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) tg[u] = targets[min((int64_t)t + (int64_t)u * step, (int64_t)t1 - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u) own += (int64_t)t + (int64_t)u * step < t1 && tg[u] >= 0 && tg[u] < V;
      if (t > t1 - 8 * step) break;  // (t + 8 step may pass 2^31)
    }
    return (double)own;
  };
  double n[1] = {};
  if (cu) {
    for (int j = wave; j < seqs; j += 16) {
      const double c = wave_sum_f64(counted(max(0, cu[j]) + lane, 64, min(tokens, cu[j + 1])));
      if (lane == 0) weights[j] = c;
      n[0] += lane == 0 && c > 0.0 ? 1.0 : 0.0;
    }
  } else {
    n[0] = counted(tid, 1024, tokens);
  }
  block_sums_f64(n, red);  // (its barriers make the sequences' counts visible)
  return n[0];
}

// Tokens with ratio q = exp(lp - old) and advantage A: -min(q A, clip(q, 1 - lo, 1 +
// hi) A) + k (exp(g) - g - 1), g = ref - lp, weighted by w: 1 / counted tokens or
// (per sequence) 1 / (sequences with counted tokens x the sequence's counted tokens).
// dloss / dlp = w (-(not clipped) q A + k (1 - exp(g))).  stats: the weighted means of
// the clipped term, of exp(g) - g - 1 and of the clipped tokens.
AXON_DEV void policy_results(double (&sum)[4], double (*red)[16], float* loss, float* stats) {
  block_sums_f64(sum, red);
  if (threadIdx.x > 0) return;
  loss[0] = (float)sum[0];
  stats[0] = (float)sum[1];
  stats[1] = (float)sum[2];
  stats[2] = (float)sum[3];
}

template <typename T>
__global__ void __launch_bounds__(1024) policy_finish_kernel(
    const T* __restrict__ z, int64_t ld, int V, const int32_t* __restrict__ targets, int tokens,
    const float2* part /* may be stat */, int slices, const int32_t* __restrict__ cu, int seqs,
    const float* __restrict__ old, const float* __restrict__ ref, const float* __restrict__ adv, float lo, float hi,
    float kl_coef, float* __restrict__ loss, float* __restrict__ stats, float* __restrict__ logps,
    double* __restrict__ weights, float2* stat, float* __restrict__ coef) {
  __shared__ double red[4][16];
  __shared__ int32_t held[CU_HELD];
  const SeqLookup seq{cu, seqs};
  const int tid = threadIdx.x;
  seq.hold(held);
  const double n = policy_counts(targets, tokens, V, cu, seqs, weights, red);
  double sum[4] = {};
  constexpr int U = 4;  // tokens of a thread whose loads are under way together
  for (int t0 = tid; t0 < tokens; t0 += 1024 * U) {
    int tg[U];
    float zt[U], o[U], a[U], rf[U];
    float2 st[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * 1024;
      tg[u] = -1;
      if (t < tokens) tg[u] = targets[t];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * 1024;
      st[u] = float2{0.f, 1.f};
      zt[u] = o[u] = a[u] = rf[u] = 0.f;
      if (tg[u] < 0 || tg[u] >= V) continue;
      zt[u] = to_f32(z[t * ld + tg[u]]);
      if (slices == 1) st[u] = part[t];
      o[u] = old[t];
      a[u] = adv[t];
      if (ref) rf[u] = ref[t];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * 1024;
      if (t >= tokens) continue;
      PolicyTerms p{};
      double w = 0.0;
      if (tg[u] >= 0 && tg[u] < V) {
        if (slices > 1) st[u] = join_slices(part, t, slices);
        w = 1.0 / (cu ? n * weights[seq.of(held, t)] : n);
        p = policy_token(zt[u], st[u].x, st[u].y, o[u], a[u], ref != nullptr, rf[u], lo, hi, kl_coef);
        sum[0] += w * ((double)p.surrogate + (kl_coef > 0.f ? (double)kl_coef * p.kl : 0.0));
        sum[1] += w * (double)p.surrogate;
        sum[2] += w * (double)p.kl;
        sum[3] += p.clipped ? w : 0.0;
      }
      logps[t] = p.lp;
      if (coef) {
        stat[t] = st[u];
        coef[t] = (float)(w * p.c);
      }
    }
  }
  policy_results(sum, red, loss, stats);
}

// the same sums from the terms that the rows' own pass left (see RowCoef)
__global__ void __launch_bounds__(1024) policy_sum_kernel(int tokens, const float2* __restrict__ terms,
                                                          const float* __restrict__ clipped,
                                                          const double* __restrict__ w, float kl_coef,
                                                          float* __restrict__ loss, float* __restrict__ stats) {
  __shared__ double red[4][16];
  double sum[4] = {};
#pragma unroll 4
  for (int t = threadIdx.x; t < tokens; t += 1024) {
    const float2 p = terms[t];
    const double v = w[t];
    sum[0] += v * ((double)p.x + (kl_coef > 0.f ? (double)kl_coef * p.y : 0.0));
    sum[1] += v * (double)p.x;
    sum[2] += v * (double)p.y;
    sum[3] += v * (double)clipped[t];
  }
  policy_results(sum, red, loss, stats);
}

// joins (op) over the lanes that differ in lane % NW; every lane the same result (see
// wave_sum)
template <int NW, typename F>
AXON_DEV float over_waves(float v, F&& op) {
  if constexpr (NW > 1) v = op(v, dpp_move<0xB1>(v));
  if constexpr (NW > 2) v = op(v, dpp_move<0x4E>(v));
  if constexpr (NW > 4) v = op(v, dpp_move<0x141>(v));
  if constexpr (NW > 8) v = op(v, dpp_move<0x140>(v));
  return v;
}

// 8 logits to their gradients f exp(v - m), f = -c / S, and c more at the target, the
// ``at``-th of them if it is one
AXON_DEV void grad_run(float (&v)[8], const ExpFrom& e, float f, float c, int at) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = e(v[j]) * f;
  if ((unsigned)at < 8u)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += j == at ? c : 0.f;
}

// dz of one slice of a row, by a workgroup of 256.  z and dz may be one buffer: a thread
// writes what it has read, and what it reads beyond that (groups at the row's end)
// counts nothing.
constexpr int GRAD_COLS = 256 * 8 * GRAD_RUNS;
template <typename T, typename TO>
AXON_DEV void grad_slice(const T* row, int V, int tg, int first, float w, float2 st, TO* out) {
  constexpr int STRIDE = 256 * 8;
  const int c0 = first + threadIdx.x * 8;
  const ExpFrom e(st.x);
  const float f = -w / st.y;
  const int h = odd_head(row), n = V - h;
  tg -= h;
  row += h;
  out += h;
  if (h && c0 == 0) out[-1] = from_f32<TO>(w == 0.f ? 0.f : e(to_f32(row[-1])) * f + (tg == -1 ? w : 0.f));
  if (first + GRAD_COLS <= n) {
    float v[GRAD_RUNS][8] = {};
    if (w != 0.f) {
      Run8<T> r[GRAD_RUNS];
#pragma unroll
      for (int k = 0; k < GRAD_RUNS; ++k) r[k].load(row + c0 + k * STRIDE);
#pragma unroll
      for (int k = 0; k < GRAD_RUNS; ++k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[k][j] = r[k][j];
        grad_run(v[k], e, f, w, tg - (c0 + k * STRIDE));
      }
    }
#pragma unroll
    for (int k = 0; k < GRAD_RUNS; ++k) Run8<TO>::store(out + c0 + k * STRIDE, v[k]);
  } else {  // the row's last slice
    for (int c = c0; c < n; c += STRIDE) {
      float v[8] = {};
      if (w != 0.f) {
        load_run8(row, c, n, v, 0.f);
        grad_run(v, e, f, w, tg - c);
      }
      store_run8(out, c, n, v);
    }
  }
}

template <typename T, typename TO>
__global__ void __launch_bounds__(256) logit_grad_kernel(const T* z, int64_t ld, int V,
                                                         const int32_t* __restrict__ targets, int64_t items, int slices,
                                                         const float2* __restrict__ stat,
                                                         const float* __restrict__ coef, TO* dz, int64_t lddz) {
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t t = it / slices;
    grad_slice(z + t * ld, V, targets[t], (int)(it % slices) * GRAD_COLS, coef[t], stat[t], dz + t * lddz);
  }
}

// The preference loss and its gradient from the slices of at most FEW tokens in at most
// FEW sequences: every workgroup works the coefficients out for itself, the first
// writes the results, and a launch less is made.  chosen: the targets' logits, which dz
// may be about to replace.
template <typename T, typename TO>
__global__ void __launch_bounds__(256) preference_few_kernel(
    const T* z, int64_t ld, int V, const int32_t* __restrict__ targets, int tokens, const float2* __restrict__ part,
    int slices, const float* __restrict__ chosen, const double* __restrict__ lps, const int32_t* __restrict__ cu,
    int seqs, const float* __restrict__ ref, float beta, float smoothing, PairOut out, int grad_slices, TO* dz,
    int64_t lddz) {
  __shared__ double red[1][16], lp[FEW], sums[FEW];
  __shared__ float2 own;
  const int i = threadIdx.x, t = blockIdx.x / grad_slices;
  if (i < tokens) {
    const int tg = targets[i];
    const bool counts = tg >= 0 && tg < V;
    const float2 st = counts ? join_slices(part, i, slices) : float2{0.f, 1.f};
    if (slices > 1) put_logp(counts, chosen + i, st.x, st.y, nullptr, lp + i);
    else lp[i] = lps[i];
    if (i == t) own = st;
  }
  __syncthreads();
  pair_coefs<256>(lp, tokens, cu, seqs, ref, beta, smoothing, sums, red, blockIdx.x == 0, out);
  const int tg = targets[t];
  const float w = tg >= 0 && tg < V ? (float)sums[seq_of_token(cu, seqs, t)] : 0.f;
  grad_slice(z + (int64_t)t * ld, V, tg, (int)(blockIdx.x % grad_slices) * GRAD_COLS, w, own, dz + t * lddz);
}

// ---------------------------------------------------------------- whole rows, read once
//
// Where a row's coefficient depends on that row alone (a caller's own dlogps, the
// policy loss), a workgroup keeps its row in registers from the statistics to the
// gradient: the logits are read once.  RUNS groups of 8 logits a thread, THREADS x RUNS x
// 8 columns; what a row has beyond them is read a second time (soon enough to come from
// the L2).  HBM bound: 2 V values a row against 3.  4096 x 128256: bf16 390 us (5.4 TB/s
// of the 2 V; in two passes with a kernel for the coefficients between them 592), float32
// 811 (1153); 64 rows 17 us (34), one row 15 (14).

// the weights of more than FEW tokens, one launch before the rows: w[0] = 1 / counted
// tokens, or w[j] = 1 / (sequences with counted tokens x those of sequence j)
__global__ void __launch_bounds__(1024) policy_weights_kernel(const int32_t* __restrict__ targets, int tokens, int V,
                                                              const int32_t* __restrict__ cu, int seqs,
                                                              double* __restrict__ w) {
  __shared__ double red[1][16];
  const double n = policy_counts(targets, tokens, V, cu, seqs, w, red);
  if (!cu) {
    if (threadIdx.x == 0) w[0] = 1.0 / n;
    return;
  }
  for (int j = threadIdx.x; j < seqs; j += 1024) w[j] = 1.0 / (w[j] * n);
}

struct RowCoef {
  const float* dlogps;  // a caller's own, or the policy loss:
  const int32_t* cu;
  int seqs;
  const float *old, *ref, *adv;
  float lo, hi, kl_coef;
  const double* weights;  // null: each workgroup counts for itself (at most FEW tokens)
  int tokens;
  // out (policy), for the loss: of each token its log-probability, (clipped term, KL
  // term), whether it is clipped, and its weight; zeros where it does not count
  float* logps;
  float2* terms;
  float* clipped;
  double* w;
};

// bits [a, b) of mask, 64 a word
AXON_DEV int bits_in(const uint64_t* mask, int a, int b) {
  int n = 0;
#pragma unroll
  for (int k = 0; k < FEW / 64; ++k) {
    const int lo = min(max(a - k * 64, 0), 64), hi = min(max(b - k * 64, 0), 64);
    const uint64_t below_hi = hi == 64 ? ~0ull : (1ull << hi) - 1, below_lo = lo == 64 ? ~0ull : (1ull << lo) - 1;
    n += __popcll(mask[k] & below_hi & ~below_lo);
  }
  return n;
}

// token t's weight where there are at most FEW tokens (policy_weights_kernel's values):
// the counted ones as a bit mask; with cu, a token counts its sequence if it is
// the first of it that counts.  A launch less: 47 rows of 50257 float32 logits 20.7 ->
// 17.1 us a call; of 4096 rows of 128256 that launch is 5 us of 338.
template <int THREADS>
AXON_DEV double few_tokens_weight(const int32_t* targets, int V, const RowCoef& rc, int t) {
  static_assert(THREADS >= FEW, "a thread for every token");
  __shared__ uint64_t mask[FEW / 64];
  __shared__ int firsts[FEW / 64];
  const int i = threadIdx.x, wave = i >> 6;
  const int tg = i < rc.tokens && i < FEW ? targets[i] : -1;
  const bool counts = tg >= 0 && tg < V;
  const uint64_t mine = __ballot(counts);
  if (wave < FEW / 64 && (i & 63) == 0) mask[wave] = mine;
  __syncthreads();
  if (!rc.cu) return 1.0 / (double)bits_in(mask, 0, FEW);
  const bool first = counts && bits_in(mask, rc.cu[seq_of_token(rc.cu, rc.seqs, i)], i) == 0;
  const uint64_t heads = __ballot(first);
  if (wave < FEW / 64 && (i & 63) == 0) firsts[wave] = __popcll(heads);
  __syncthreads();
  int n = 0;
#pragma unroll
  for (int k = 0; k < FEW / 64; ++k) n += firsts[k];
  const int j = seq_of_token(rc.cu, rc.seqs, t);
  return 1.0 / ((double)bits_in(mask, rc.cu[j], rc.cu[j + 1]) * (double)n);
}

AXON_DEV void put_terms(const RowCoef& rc, int64_t t, const PolicyTerms& p, double weight) {
  rc.logps[t] = p.lp;
  rc.terms[t] = float2{p.surrogate, p.kl};
  rc.clipped[t] = p.clipped ? 1.f : 0.f;
  rc.w[t] = weight;
}

// the same from the (m, S) of whole rows, a thread a token: the loss alone of more than
// 2048 tokens, 131072 x 32000 bf16 1.41 ms a call, 4096 x 128256 192 us (1.76 and 202 with
// policy_finish_kernel, which is two launches less).
template <typename T>
__global__ void __launch_bounds__(256) policy_terms_kernel(const T* __restrict__ z, int64_t ld, int V,
                                                           const int32_t* __restrict__ targets,
                                                           const float2* __restrict__ stat, RowCoef rc) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= rc.tokens) return;
  const int tg = targets[t];
  PolicyTerms p{};
  double weight = 0.0;
  if (tg >= 0 && tg < V) {
    const float2 st = stat[t];
    weight = rc.weights[rc.cu ? seq_of_token(rc.cu, rc.seqs, (int)t) : 0];
    p = policy_token(to_f32(z[t * ld + tg]), st.x, st.y, rc.old[t], rc.adv[t], rc.ref != nullptr,
                     rc.ref ? rc.ref[t] : 0.f, rc.lo, rc.hi, rc.kl_coef);
  }
  put_terms(rc, t, p, weight);
}

// p + b bytes, b unsigned 32-bit: one register of address beside a uniform p
template <typename T>
AXON_DEV const T* at_byte(const T* p, unsigned b) {
  return (const T*)((const char*)p + b);
}
template <typename T>
AXON_DEV T* at_byte(T* p, unsigned b) {
  return (T*)((char*)p + b);
}

template <typename T, typename TO, int THREADS, int RUNS>
__global__ void __launch_bounds__(THREADS) logit_row_kernel(const T* z, int64_t ld, int V,
                                                            const int32_t* __restrict__ targets, int64_t first,
                                                            RowCoef rc, TO* dz, int64_t lddz) {
  constexpr int NW = THREADS / 64, STRIDE = THREADS * 8, HELD = STRIDE * RUNS;
  __shared__ float2 parts[16];
  __shared__ float coef;
  const int i = threadIdx.x;
  const int64_t t = first + blockIdx.x;
  const T* row = z + t * ld;
  const int h = odd_head(row), whole = V - h & ~7;
  row += h;
  TO* out = dz + t * lddz + h;
  const int tg = targets[t] - h;
  const bool counts = tg + h >= 0 && tg + h < V;
  // groups that every thread has, and whether this one has another after them
  const int full = min(whole / STRIDE, RUNS), groups = min((whole + STRIDE - 1) / STRIDE, RUNS);
  const bool more = full < groups && full * STRIDE + i * 8 < whole;
  // the columns beside the groups of 8, one a thread: the last few, and the head
  const bool single = i < V - h - whole || (i == 7 && h);
  const int at = i < V - h - whole ? whole + i : -1;
  auto zeros = [&] {
    const float zero[8] = {};
    for (int c = i * 8; c < whole; c += STRIDE) Run8<TO>::store(out + c, zero);
    if (single) out[at] = from_f32<TO>(0.f);
  };
  const bool policy = rc.dlogps == nullptr;
  if (!counts) {  // uniform over the workgroup
    zeros();
    if (policy && i == 0) put_terms(rc, t, PolicyTerms{}, 0.0);
    return;
  }
  const float zt = to_f32(row[tg]), given = policy ? rc.old[t] : rc.dlogps[t];
  const float adv = policy ? rc.adv[t] : 0.f, ref = policy && rc.ref ? rc.ref[t] : 0.f;
  double weight = 1.0;
  if (policy)
    weight = rc.weights ? rc.weights[rc.cu ? seq_of_token(rc.cu, rc.seqs, (int)t) : 0]
                        : few_tokens_weight<THREADS>(targets, V, rc, (int)t);
  // every load unconditional (past the row's groups its last one again), so that
  // each is waited for by itself and the sums run under the loads behind them
  Run8<T> r[RUNS];
  if (whole > 0)
#pragma unroll
    for (int k = 0; k < RUNS; ++k) r[k].load(at_byte(row, min(k * STRIDE + i * 8, whole - 8) * (unsigned)sizeof(T)));
  const float alone = single ? to_f32(row[at]) : -INFINITY;
  float m = -INFINITY, s = 0.f;
#pragma unroll
  for (int k = 0; k < RUNS; ++k) {
    if (k < groups) {  // (uniform)
      float v[1][8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[0][j] = k < full || more ? r[k][j] : -INFINITY;
      take_runs(m, s, v);
    }
    r[k].reread();  // (kept in float32 until the gradient, bf16 logits would take twice the registers)
  }
  for (int c = HELD + i * 8; c < whole; c += STRIDE) {  // not held
    Run8<T> q;
    q.load(row + c);
    float v[1][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[0][j] = q[j];
    take_runs(m, s, v);
  }
  join_part(m, s, alone, one_exp(alone));
  // over the wavefronts: lane l joins what wavefront l % NW left
  const float wm = wave_max(m);
  s = wave_sum(s * exp_join(m - (wm == -INFINITY ? 0.f : wm)));
  if ((i & 63) == 0) parts[i >> 6] = float2{wm, s};
  __syncthreads();
  const float2 p = parts[i % NW];
  m = over_waves<NW>(p.x, [](float a, float b) { return fmaxf(a, b); });
  s = over_waves<NW>(p.y * exp_join(p.x - (m == -INFINITY ? 0.f : m)), [](float a, float b) { return a + b; });
  float w = given;
  if (policy) {
    PolicyTerms p{};
    if (i == 0) {
      p = policy_token(zt, m, s, given, adv, rc.ref != nullptr, ref, rc.lo, rc.hi, rc.kl_coef);
      coef = (float)(weight * p.c);
    }
    __syncthreads();
    w = coef;
    if (i == 0) put_terms(rc, t, p, weight);
  }
  // a coefficient of 0 (clipped): zeros, whatever the row holds
  if (w == 0.f) {
    zeros();
    return;
  }
  const ExpFrom e(m);
  const float f = -w / s;
  auto grad = [&](const Run8<T>& q, TO* to) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = e(q[j]) * f;
    Run8<TO>::store(to, v);
  };
#pragma unroll
  for (int k = 0; k < RUNS; ++k)
    if (k < full || (k == full && more)) grad(r[k], at_byte(out, (k * STRIDE + i * 8) * (unsigned)sizeof(TO)));
  for (int c = HELD + i * 8; c < whole; c += STRIDE) {
    Run8<T> q;
    q.load(row + c);
    grad(q, out + c);
  }
  if (single) out[at] = from_f32<TO>(e(alone) * f);
  // the target's own column, by the thread that has just written it
  const int owner = tg < 0 ? 7 : tg < whole ? (tg >> 3) % THREADS : tg - whole;
  if (i == owner) out[tg] = from_f32<TO>(e(zt) * f + w);
}

// ---------------------------------------------------------------- within a training step

// (m, S) of a row from the np (largest, sum) partials of its 64-column pieces, and
// (lps) its target's log-probability, a workgroup a row; rows that do not count are skipped
__global__ void __launch_bounds__(PART_THREADS) piece_merge_kernel(const float2* __restrict__ pieces, int np, int V,
                                                                   const int32_t* __restrict__ targets,
                                                                   float2* __restrict__ stat,
                                                                   const float* __restrict__ z, int ldl,
                                                                   double* __restrict__ lps) {
  __shared__ float red[2][PART_THREADS / 64];
  const int t = blockIdx.x, tg = targets[t];
  const bool counts = tg >= 0 && tg < V;
  float m = -INFINITY, s = 0.f;
  if (counts) {
    for (int i = threadIdx.x; i < np; i += PART_THREADS) {
      const float2 p = pieces[(int64_t)t * np + i];
      join_part(m, s, p.x, p.y);
    }
    join_block(m, s, red);
  }
  if (threadIdx.x > 0) return;
  if (counts) stat[t] = float2{m, s};
  put_logp(counts, z + (int64_t)t * ldl + tg, m, s, nullptr, lps ? lps + t : nullptr);
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
// them for two rounds of 8 workgroups on each of the 256 CUs, else as many slices as
// give that, of at least one group of 8 per thread, and at most 16 (they are joined by
// one thread)
void part_shape(int64_t tokens, int V, int& slices, int& cols) {
  const int most = (V + PART_THREADS * 8 - 1) / (PART_THREADS * 8);
  const int64_t fill = std::max<int64_t>(1, 4096 / std::max<int64_t>(tokens, 1));
  const int want = (int)std::min<int64_t>({most, 16, fill});
  const int runs = (most + want - 1) / want;
  cols = runs * PART_THREADS * 8;
  slices = (V + cols - 1) / cols;
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

// the workspace of a call
struct LossWs {
  float2* part;
  float2* stat;  // (policy: RowCoef's terms)
  float* coef;   // (policy: its clipped)
  double* lps;   // preference: log-probabilities; policy: weights
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
int run_parts(const LogitRows& r, float2* part, float* logps, double* lps, float* chosen, hipStream_t s) {
  int slices, cols;
  part_shape(r.tokens, r.V, slices, cols);
  const int64_t items = r.tokens * slices;
  logit_part_kernel<T><<<(unsigned)std::min(items, MAX_WGS), PART_THREADS, 0, s>>>(
      (const T*)r.z, r.ld, r.V, r.targets, items, slices, cols, part, slices == 1 ? logps : nullptr,
      slices == 1 ? lps : nullptr, chosen);
  return slices;
}

template <typename T>
void run_grad(const LogitRows& r, const LossWs& w, hipStream_t s) {
  const int slices = (r.V + GRAD_COLS - 1) / GRAD_COLS;
  const int64_t items = r.tokens * slices;
  const unsigned wgs = (unsigned)std::min(items, MAX_WGS);
  if (r.dz_bf16)
    logit_grad_kernel<T, bf16><<<wgs, 256, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets, items, slices, w.stat, w.coef,
                                                   (bf16*)r.dz, r.lddz);
  else
    logit_grad_kernel<T, float><<<wgs, 256, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets, items, slices, w.stat, w.coef,
                                                    (float*)r.dz, r.lddz);
}

template <typename T, typename TO>
void run_rows(const LogitRows& r, const RowCoef& rc, hipStream_t s) {
  auto go = [&](auto kern, int threads) {
    for (int64_t first = 0; first < r.tokens; first += MAX_WGS)  // a launch holds at most 2^32 threads
      kern<<<(unsigned)std::min(r.tokens - first, MAX_WGS), threads, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets, first,
                                                                            rc, (TO*)r.dz, r.lddz);
  };
  constexpr int R = sizeof(T) == 2 ? 16 : 8;  // 64 registers of logits a thread
  if (r.V <= 256 * 8 * 4) go(logit_row_kernel<T, TO, 256, 4>, 256);
  else if (r.V <= 256 * 8 * R) go(logit_row_kernel<T, TO, 256, R>, 256);
  else if (r.V <= 512 * 8 * R) go(logit_row_kernel<T, TO, 512, R>, 512);
  else if (r.V <= 1024 * 8 * R) go(logit_row_kernel<T, TO, 1024, R>, 1024);
  else go(logit_row_kernel<T, TO, 1024, sizeof(T) == 2 ? 20 : 12>, 1024);
}
template <typename T>
void run_rows(const LogitRows& r, const RowCoef& rc, hipStream_t s) {
  r.dz_bf16 ? run_rows<T, bf16>(r, rc, s) : run_rows<T, float>(r, rc, s);
}

template <typename T>
void logprobs(const LogitRows& r, float* logps, void* wsp, hipStream_t s) {
  LossWs w;
  carve(r.tokens, r.V, 0, (char*)wsp, &w);
  const int slices = run_parts<T>(r, w.part, logps, nullptr, nullptr, s);
  if (slices > 1)
    logps_finish_kernel<T><<<(unsigned)((r.tokens + 255) / 256), 256, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets,
                                                                             r.tokens, w.part, slices, logps);
}

template <typename T>
void logprobs_bwd(const LogitRows& r, const float* dlogps, hipStream_t s) {
  RowCoef rc{};
  rc.dlogps = dlogps;
  run_rows<T>(r, rc, s);
}

// Every workgroup its own coefficients while there are few of both: us a call that way
// and with a launch between, 61 x 32000 bf16 15.0 and 16.4, 61 x 128256 float32 (976
// workgroups) 21.6 and 23.7, 128 x 128256 (2048) 42.9 and 41.7, 250 x 32000 bf16 (1000)
// 23.7 and 21.7, 250 x 128256 (4000) 55 and 41.
bool few_pairs(const LogitRows& r, int seqs) {
  return r.dz && r.tokens > 0 && r.tokens <= FEW / 2 && seqs <= FEW &&
         r.tokens * ((r.V + GRAD_COLS - 1) / GRAD_COLS) <= 1024;
}

template <typename T>
void preference(const LogitRows& r, const PreferenceArgs& a, void* wsp, hipStream_t s) {
  LossWs w;
  carve(r.tokens, r.V, a.seqs, (char*)wsp, &w);
  const bool few = few_pairs(r, a.seqs);
  const int slices = r.tokens > 0 ? run_parts<T>(r, w.part, nullptr, w.lps, few ? w.coef : nullptr, s) : 1;
  const PairOut out{a.loss, a.seq_logps, a.margins};
  if (few) {
    const int g = (r.V + GRAD_COLS - 1) / GRAD_COLS;
    auto go = [&](auto kern, auto* dz) {
      kern<<<(unsigned)r.tokens * g, 256, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets, (int)r.tokens, w.part, slices,
                                                  w.coef, w.lps, a.cu, a.seqs, a.ref, a.beta, a.smoothing, out, g, dz,
                                                  r.lddz);
    };
    r.dz_bf16 ? go(preference_few_kernel<T, bf16>, (bf16*)r.dz) : go(preference_few_kernel<T, float>, (float*)r.dz);
    return;
  }
  if (slices == 1) w.stat = w.part;
  preference_finish_kernel<T><<<1, 1024, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets, (int)r.tokens, w.part, slices,
                                                 a.cu, a.seqs, a.ref, a.beta, a.smoothing, out, w.lps, w.seq, w.stat,
                                                 r.dz ? w.coef : nullptr);
  if (r.dz && r.tokens > 0) run_grad<T>(r, w, s);
}

template <typename T>
void policy(const LogitRows& r, const PolicyArgs& a, void* wsp, hipStream_t s) {
  LossWs w;
  carve(r.tokens, r.V, a.seqs, (char*)wsp, &w);
  const bool grad = r.dz && r.tokens > 0, few = grad && r.tokens <= FEW;
  const int tokens = (int)r.tokens;
  int slices = 1;  // (of more than 2048 tokens always 1, see part_shape)
  if (!grad && tokens > 0) slices = run_parts<T>(r, w.part, nullptr, nullptr, nullptr, s);
  if (!grad && (tokens <= 2048 || slices > 1)) {
    policy_finish_kernel<T><<<1, 1024, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets, tokens, w.part, slices, a.cu,
                                               a.seqs, a.old, a.ref, a.adv, a.lo, a.hi, a.kl_coef, a.loss, a.stats,
                                               a.logps, w.seq, nullptr, nullptr);
    return;
  }
  const RowCoef rc{nullptr, a.cu, a.seqs, a.old, a.ref, a.adv, a.lo, a.hi, a.kl_coef, few ? nullptr : w.seq,
                   tokens, a.logps, w.stat, w.coef, w.lps};
  if (!few) policy_weights_kernel<<<1, 1024, 0, s>>>(r.targets, tokens, r.V, a.cu, a.seqs, w.seq);
  if (grad) run_rows<T>(r, rc, s);
  else
    policy_terms_kernel<T><<<(tokens + 255) / 256, 256, 0, s>>>((const T*)r.z, r.ld, r.V, r.targets, w.part, rc);
  policy_sum_kernel<<<1, 1024, 0, s>>>(tokens, w.stat, w.coef, w.lps, a.kl_coef, a.loss, a.stats);
}

}  // namespace

size_t loss_workspace_bytes(int64_t tokens, int V, int64_t seqs) { return carve(tokens, V, seqs, nullptr, nullptr); }

void launch_token_logps(const LogitRows& r, float* logps, void* ws, hipStream_t s) {
  if (r.z_bf16) logprobs<bf16>(r, logps, ws, s);
  else logprobs<float>(r, logps, ws, s);
}
void launch_token_logps_bwd(const LogitRows& r, const float* dlogps, hipStream_t s) {
  if (r.z_bf16) logprobs_bwd<bf16>(r, dlogps, s);
  else logprobs_bwd<float>(r, dlogps, s);
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

void train_stat(const TrainLogits& r, double* lps, hipStream_t s) {
  piece_merge_kernel<<<r.T, PART_THREADS, 0, s>>>(r.lse_part, (r.V + LSE_COLS - 1) / LSE_COLS, r.V, r.targets, r.stat,
                                                  r.z, r.ldl, lps);
}

void train_grad(const TrainLogits& r, hipStream_t s) {
  logit_grad_pair_kernel<<<dim3((r.ldl / 32 + 31) / 32, (r.T + 1) / 2), 256, 0, s>>>(r.z, r.ldl, r.V, r.T, r.targets,
                                                                                     r.stat, r.coef, r.dlog);
}

}  // namespace

void launch_preference_train(const TrainLogits& r, const PreferenceArgs& a, hipStream_t s) {
  train_stat(r, r.lps, s);
  preference_finish_kernel<float><<<1, 1024, 0, s>>>(r.z, r.ldl, r.V, r.targets, r.T, r.stat, 1, a.cu, a.seqs, a.ref,
                                                     a.beta, a.smoothing, PairOut{a.loss, a.seq_logps, a.margins},
                                                     r.lps, r.seq, r.stat, r.coef);
  train_grad(r, s);
}

void launch_policy_train(const TrainLogits& r, const PolicyArgs& a, hipStream_t s) {
  train_stat(r, nullptr, s);
  policy_finish_kernel<float><<<1, 1024, 0, s>>>(r.z, r.ldl, r.V, r.targets, r.T, r.stat, 1, a.cu, a.seqs, a.old, a.ref,
                                                 a.adv, a.lo, a.hi, a.kl_coef, a.loss, a.stats, a.logps, r.seq, r.stat,
                                                 r.coef);
  train_grad(r, s);
}

}  // namespace axon
