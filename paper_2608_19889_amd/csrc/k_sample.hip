// The next token of every row of logits, from a given uniform number.
//
// With x_i = (z_i - max) / T the weights are w_i = exp(x_i).  Top-k, top-p and min-p
// each keep a beginning of the tokens in descending order of z (the lowest index first
// among equals), so together they keep the tokens above a border value and some of
// those on it.  The token is the first, in the order of the vocabulary, at which the
// running sum of the kept weights passes ``uniform`` of their sum.
//
// Which token that is must not hang on a rounding: the weights are float64 (2^-51 of
// themselves) and summed as integers, W_i = w_i 2^(62 - log2 V) rounded, whose sums are
// exact and have no order, so that they can be added up by atomics.
//
// A border is found without sorting: a histogram (number and weight) over 2048 ranges of
// the values' bits, the range that the border is in, and again inside it.
//
// The logits are read once, by sample_scan_kernel: the maximum of every block of 32 and,
// where a row needs it, the weights' sum of every chunk of 2048.  What a filter keeps is
// above a value that the maxima alone give: k of them reach the k-th largest, or their
// weights the share p of the sum.  So sample_row_kernel, a workgroup per row, reads only
// the blocks whose maximum is above it (those of some hundred tokens where a row is sure
// of itself) and keeps their values in registers through its passes; without a filter
// the sums lead it to the token's chunk.
#include "common.h"
#include "kernels.h"

namespace axon {

typedef unsigned long long u64;
constexpr int S_THREADS = 1024;
constexpr int BINS = 2 * S_THREADS;

// 2^x for x <= 0 (0 below -1100): 2^f on [-1/2, 1/2] as the polynomial of degree 10
// through 2^f at Chebyshev's nodes, 4e-16 of itself off and exactly 1 at 0
AXON_DEV double exp2_neg(double x) {
  x = fmax(x, -1100.);  // (NaN, from infinities: no weight either)
  const double n = rint(x), f = x - n;
  double v = 7.072585949269224e-09;
  v = fma(v, f, 1.0208690299958306e-07);
  v = fma(v, f, 1.321544258792169e-06);
  v = fma(v, f, 1.5252657260200837e-05);
  v = fma(v, f, 0.0001540353044173605);
  v = fma(v, f, 0.0013333558230164974);
  v = fma(v, f, 0.009618129107606888);
  v = fma(v, f, 0.05550410866444772);
  v = fma(v, f, 0.24022650695910097);
  v = fma(v, f, 0.69314718055995);
  v = fma(v, f, 1.0);
  return ldexp(v, (int)n);
}

// a logit as it is compared: NaN cannot be chosen, zeros have one sign
AXON_DEV float sane(float z) { return z == 0.f ? 0.f : z == z ? z : -INFINITY; }
// its bits in ascending order
AXON_DEV uint32_t order_key(float z) {
  const uint32_t u = __float_as_uint(z);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
AXON_DEV float key_value(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }

struct Shared {
  u64 mass[BINS];
  uint32_t cnt[BINS];
  u64 wave_mass[16];
  uint32_t wave_cnt[16];
  u64 mass_before, mass_in;
  uint32_t cnt_before, cnt_in;
  int found;
  float red[16];
};

// number and weight in front of a place, and the place
struct Found {
  int at;
  u64 mass_before, mass_in;
  uint32_t cnt_before, cnt_in;
};

AXON_DEV void clear_bins(Shared& sh) {
  __syncthreads();
  for (int i = threadIdx.x; i < BINS; i += S_THREADS) {
    sh.mass[i] = 0;
    sh.cnt[i] = 0;
  }
  if (threadIdx.x == 0) sh.found = -1;
  __syncthreads();
}

// Over each thread's two entries, in the threads' order: the entry at which the running
// sum (of numbers or of weights) reaches target(total) >= 1.
template <bool COUNT, typename F>
AXON_DEV Found find_entry(Shared& sh, const u64 (&m)[2], const uint32_t (&c)[2], u64 m0, uint32_t c0, F&& target,
                          u64* total = nullptr) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 ms = m[0] + m[1];
  uint32_t csum = c[0] + c[1];
  const u64 own_m = ms;
  const uint32_t own_c = csum;
  for (int d = 1; d < 64; d <<= 1) {
    const u64 mu = __shfl_up(ms, d);
    const uint32_t cu = __shfl_up(csum, d);
    if (lane >= d) {
      ms += mu;
      csum += cu;
    }
  }
  if (lane == 63) {
    sh.wave_mass[wave] = ms;
    sh.wave_cnt[wave] = csum;
  }
  __syncthreads();
  u64 mb = m0 + ms - own_m, mt = m0;
  uint32_t cb = c0 + csum - own_c, ct = c0;
  for (int w = 0; w < 16; ++w) {
    if (w < wave) {
      mb += sh.wave_mass[w];
      cb += sh.wave_cnt[w];
    }
    mt += sh.wave_mass[w];
    ct += sh.wave_cnt[w];
  }
  const u64 want = target(COUNT ? (u64)ct : mt);
  if (total) *total = COUNT ? (u64)ct : mt;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const u64 before = COUNT ? (u64)cb : mb, after = before + (COUNT ? (u64)c[j] : m[j]);
    if (before < want && want <= after) {
      sh.found = 2 * threadIdx.x + j;
      sh.mass_before = mb;
      sh.mass_in = m[j];
      sh.cnt_before = cb;
      sh.cnt_in = c[j];
    }
    mb += m[j];
    cb += c[j];
  }
  __syncthreads();
  return Found{sh.found, sh.mass_before, sh.mass_in, sh.cnt_before, sh.cnt_in};
}

// ---------------------------------------------------------------- one reading of the logits

constexpr int BLOCK = 32;    // logits of a maximum
constexpr int CHUNK = 2048;  // logits of a wavefront, and of a sum
constexpr int SCAN_THREADS = 256;
constexpr int CHUNK_BLOCKS = CHUNK / BLOCK;

struct Settings {
  float t, p, low;
  int k;
  bool greedy, by_rank;  // the largest alone; a top-k that leaves some out
};
AXON_DEV Settings settings_of(const SampleArgs& a, int r) {
  Settings s;
  s.t = a.temperature ? a.temperature[r] : a.temperature_all;
  s.k = a.top_k ? a.top_k[r] : a.top_k_all;
  s.p = a.top_p ? a.top_p[r] : a.top_p_all;
  s.low = a.min_p ? a.min_p[r] : a.min_p_all;
  s.greedy = !(s.t > 0.f);
  s.by_rank = s.k > 0 && s.k < a.vocab;
  return s;
}
// whether the row's sum of weights is needed: for the share p of it, or to draw from all
AXON_DEV bool needs_sum(const Settings& s) { return !s.greedy && !s.by_rank && (s.p < 1.f || !(s.low > 0.f)); }
AXON_DEV double per_unit(const Settings& s) { return s.greedy ? 0. : 1.4426950408889634 / (double)s.t; }
// a weight relative to ``top``
AXON_DEV double weight_to(float z, float top, double c) { return z == top ? 1. : exp2_neg(((double)z - top) * c); }

template <typename T>
constexpr int RUN = 16 / sizeof(T);  // values of a 16-byte load
template <typename T>
struct Load;
template <>
struct Load<float> {
  typedef f32x4_any t;
};
template <>
struct Load<bf16> {
  typedef bf16x8_any t;
};
// values i .. i + RUN - 1 of a row as they are compared, -inf past its end
template <typename T>
AXON_DEV void load_run(const T* z, int i, int V, float (&v)[RUN<T>]) {
  if (i + RUN<T> <= V) {
    const typename Load<T>::t w = *(const typename Load<T>::t*)(z + i);
#pragma unroll
    for (int j = 0; j < RUN<T>; ++j) v[j] = sane(to_f32((T)w[j]));
  } else {
#pragma unroll
    for (int j = 0; j < RUN<T>; ++j) v[j] = i + j < V ? sane(to_f32(z[i + j])) : -INFINITY;
  }
}

struct RowSums {  // of a row, in the workspace
  float* block_max;   // [chunks 64]
  float* chunk_max;   // [chunks]
  double* chunk_sum;  // [chunks], relative to chunk_max
};
inline __host__ __device__ int chunks_of(int V) { return (V + CHUNK - 1) / CHUNK; }
inline __host__ __device__ int64_t row_bytes(int V) { return (int64_t)chunks_of(V) * (CHUNK_BLOCKS * 4 + 4 + 8) + 4 * (chunks_of(V) & 1); }
AXON_DEV RowSums row_sums(void* ws, int r, int V) {
  const int n = chunks_of(V);
  char* p = (char*)ws + r * row_bytes(V);
  return RowSums{(float*)(p + 8 * n), (float*)(p + 8 * n) + n * CHUNK_BLOCKS, (double*)p};
}

// a wavefront per chunk; a lane's load is RUN values, 32 / RUN lanes a block
template <typename T>
__global__ void __launch_bounds__(SCAN_THREADS) sample_scan_kernel(SampleArgs a, void* ws) {
  constexpr int N = RUN<T>, ROUNDS = CHUNK / (64 * N), LANES = BLOCK / N;
  const int r = blockIdx.y, chunk = blockIdx.x * (SCAN_THREADS / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (chunk >= chunks_of(a.vocab)) return;
  const T* z = (const T*)a.logits + r * a.ld;
  float v[ROUNDS][N], top[ROUNDS];
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) load_run(z, chunk * CHUNK + (j * 64 + lane) * N, a.vocab, v[j]);
  const Settings s = settings_of(a, r);
  const RowSums out = row_sums(ws, r, a.vocab);
  float mine = -INFINITY, all = -INFINITY;
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    top[j] = v[j][0];
#pragma unroll
    for (int i = 1; i < N; ++i) top[j] = fmaxf(top[j], v[j][i]);
    top[j] = fmaxf(top[j], dpp_move<0xB1>(top[j]));
    top[j] = fmaxf(top[j], dpp_move<0x4E>(top[j]));
    if (LANES == 8) top[j] = fmaxf(top[j], dpp_move<0x141>(top[j]));
    if (lane % LANES == j) mine = top[j];
    all = fmaxf(all, top[j]);
  }
  static_assert(LANES == ROUNDS, "each lane of a block's writes one block's maximum");
  out.block_max[chunk * CHUNK_BLOCKS + lane % LANES * (64 / LANES) + lane / LANES] = mine;
  all = wave_max(all);
  if (lane == 0) out.chunk_max[chunk] = all;
  if (!needs_sum(s)) return;
  const double c = per_unit(s);
  double sum = 0.;
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j)
#pragma unroll
    for (int i = 0; i < N; ++i) sum += all == -INFINITY ? 0. : weight_to(v[j][i], all, c);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) out.chunk_sum[chunk] = sum;
}

// ---------------------------------------------------------------- the rest of a row

constexpr int LIST = 4096;        // blocks that are listed; more: all of the row
constexpr int MAX_BLOCKS = 8192;  // maxima that fit into LDS (262144 logits)

// The values of a row that can matter: those of the listed blocks, or (n < 0) of all.
// What is below ``cut`` is passed over.  A thread's first 16 bytes stay in registers
// from pass to pass, the others are read again.
template <typename T>
struct Row {
  static constexpr int N = RUN<T>, LANES = BLOCK / N;
  const T* z;
  int V;
  float cut;
  int n;
  const int32_t* list;
  float v0[N];
  AXON_DEV int items() const { return n < 0 ? (V + N - 1) / N : n * LANES; }
  AXON_DEV int first(int e) const { return n < 0 ? e * N : list[e / LANES] * BLOCK + e % LANES * N; }
  AXON_DEV void fill() {
    if ((int)threadIdx.x < items()) load_run(z, first(threadIdx.x), V, v0);
  }
  template <typename F>
  AXON_DEV void each(F&& f) const {
    float v[N], next[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = v0[i];
    const int end = items();
#pragma unroll 1
    for (int e = threadIdx.x; e < end; e += S_THREADS) {
      const int at = first(e);
      if (e + S_THREADS < end) load_run(z, first(e + S_THREADS), V, next);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (v[i] >= cut) f(v[i], at + i);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = next[i];
    }
  }
};

// the value on the border in descending order, and what is above it
struct Border {
  uint32_t key;
  u64 mass_above;
  uint32_t cnt_above, cnt_on;
  u64 want;  // the target
};
// over the values from key ``lo`` to key ``hi``, which hold all that count
template <bool COUNT, typename R, typename W, typename F>
AXON_DEV Border find_border(Shared& sh, const R& row, uint32_t lo, uint32_t hi, W&& weight, F&& target) {
  Border b{};
  for (;;) {
    int shift = 0;
    while ((hi - lo) >> shift >= BINS) ++shift;
    clear_bins(sh);
    row.each([&](float z, int) {
      const uint32_t k = order_key(z);
      if (k < lo || k > hi) return;
      const uint32_t bin = (k - lo) >> shift;
      atomicAdd(&sh.cnt[bin], 1u);
      const u64 w = weight(z);
      if (w) atomicAdd(&sh.mass[bin], w);
    });
    __syncthreads();
    const int e = BINS - 1 - 2 * threadIdx.x;
    const u64 m[2] = {sh.mass[e], sh.mass[e - 1]};
    const uint32_t c[2] = {sh.cnt[e], sh.cnt[e - 1]};
    const Found f = find_entry<COUNT>(sh, m, c, b.mass_above, b.cnt_above, [&](u64 total) {
      if (!b.want) b.want = min(target(total), total);
      return b.want;
    });
    const uint32_t bin = BINS - 1 - f.at;
    lo += bin << shift;
    hi = min(hi, lo + ((1u << shift) - 1));
    b = Border{lo, f.mass_before, f.cnt_before, f.cnt_in, b.want};
    if (lo == hi) return b;
    if (f.cnt_in == 1) {  // one value is left: which
      __syncthreads();
      row.each([&](float z, int) {
        const uint32_t k = order_key(z);
        if (lo <= k && k <= hi) sh.found = (int)k;
      });
      __syncthreads();
      b.key = (uint32_t)sh.found;
      return b;
    }
  }
}

// the index at which the running sum of weight(z, i) reaches target(total); weight is 0
// below the row's cut
template <typename R, typename W, typename F>
AXON_DEV int find_index(Shared& sh, const R& row, W&& weight, F&& target, u64* total) {
  const int width = (row.V + BINS - 1) / BINS;  // <= BINS
  clear_bins(sh);
  row.each([&](float z, int i) {
    const u64 w = weight(z, i);
    if (w) atomicAdd(&sh.mass[i / width], w);
  });
  __syncthreads();
  u64 want = 0;
  const int e = 2 * threadIdx.x;
  const u64 m[2] = {sh.mass[e], sh.mass[e + 1]};
  const uint32_t c[2] = {};
  const Found f = find_entry<false>(sh, m, c, 0, 0, [&](u64 t) { return want = target(t); }, total);
  const int first = f.at * width;
  u64 w[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = first + e + j;
    w[j] = e + j < width && i < row.V ? weight(sane(to_f32(row.z[i])), i) : 0;
  }
  __syncthreads();
  return first + find_entry<false>(sh, w, c, f.mass_before, 0, [&](u64) { return want; }).at;
}

// the workgroup's maximum (of negated values: minimum)
AXON_DEV float block_top(Shared& sh, float v) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.red[threadIdx.x >> 6] = v;
  __syncthreads();
  for (int w = 0; w < S_THREADS / 64; ++w) v = fmaxf(v, sh.red[w]);
  return v;
}

template <typename T>
__global__ void __launch_bounds__(S_THREADS) sample_row_kernel(SampleArgs a, void* ws) {
  __shared__ Shared sh;
  __shared__ float maxima[MAX_BLOCKS];
  __shared__ int32_t list[LIST];
  const int r = blockIdx.x, V = a.vocab, chunks = chunks_of(V), blocks = chunks * CHUNK_BLOCKS, tid = threadIdx.x;
  const T* z = (const T*)a.logits + r * a.ld;
  const RowSums in = row_sums(ws, r, V);
  const Settings s = settings_of(a, r);
  float top = -INFINITY;
  for (int i = tid; i < chunks; i += S_THREADS) top = fmaxf(top, in.chunk_max[i]);
  const bool filtered = !s.greedy && (s.by_rank || s.p < 1.f || s.low > 0.f), fits = blocks <= MAX_BLOCKS;
  float lowest = INFINITY;  // of the maxima that are numbers
  if (filtered && fits)
    for (int i = tid; i < blocks; i += S_THREADS) {
      const float m = in.block_max[i];
      maxima[i] = m;
      if (m > -INFINITY) lowest = fminf(lowest, m);
    }
  top = block_top(sh, top);
  if (top == -INFINITY) {
    if (tid == 0) {
      a.tokens[r] = -1;
      a.logps[r] = 0.f;
    }
    return;
  }
  if (s.greedy) {  // the first block with the maximum, the first there
    if (tid == 0) sh.found = blocks;
    __syncthreads();
    for (int i = tid; i < blocks; i += S_THREADS)
      if (in.block_max[i] == top) {
        atomicMin(&sh.found, i);
        break;
      }
    __syncthreads();
    if (tid >= 64) return;
    const int i = sh.found * BLOCK + tid;
    const uint64_t has = __ballot(tid < BLOCK && i < V && sane(to_f32(z[min(i, V - 1)])) == top);
    if (tid == 0) {
      a.tokens[r] = sh.found * BLOCK + __ffsll((long long)has) - 1;
      a.logps[r] = 0.f;
    }
    return;
  }
  const int scale = 62 - (V > 1 ? 32 - __clz(V - 1) : 0);
  const double c = per_unit(s);
  auto weight_of = [&](float v) { return weight_to(v, top, c); };
  auto fixed = [&](double w) { return (u64)rint(ldexp(w, scale)); };
  auto weight = [&](float v) { return fixed(weight_of(v)); };
  // the place in the kept weights' running sum, 1 .. sum
  auto drawn = [&](u64 sum) {
    return min((u64)((double)fminf(fmaxf(a.uniform[r], 0.f), 1.f) * (double)sum), sum - 1) + 1;
  };
  u64 total;
  int token;
  if (!filtered) {
    u64 w[2], want = 0;
    const uint32_t none[2] = {};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = 2 * tid + j;
      const double f = i < chunks ? weight_of(in.chunk_max[i]) : 0.;
      w[j] = fixed(f) ? fixed(f * in.chunk_sum[i]) : 0;  // (a chunk whose weights are all 0 is not one to look in)
    }
    const Found f = find_entry<false>(sh, w, none, 0, 0, [&](u64 sum) { return want = drawn(sum); }, &total);
    const int first = f.at * CHUNK + 2 * tid;
#pragma unroll
    for (int j = 0; j < 2; ++j) w[j] = first + j < V ? weight(sane(to_f32(z[first + j]))) : 0;
    __syncthreads();
    token = f.at * CHUNK +
            find_entry<false>(sh, w, none, 0, 0, [&](u64 sum) { return min(want - f.mass_before, sum); }).at;
  } else {
    double sum = 0.;  // of all weights
    if (needs_sum(s)) {
      for (int i = tid; i < chunks; i += S_THREADS) sum += weight_of(in.chunk_max[i]) * in.chunk_sum[i];
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
      __syncthreads();
      if ((tid & 63) == 0) sh.wave_mass[tid >> 6] = __double_as_longlong(sum);
      __syncthreads();
      sum = 0.;
      for (int w = 0; w < S_THREADS / 64; ++w) sum += __longlong_as_double(sh.wave_mass[w]);
    }
    const double share = (double)fmaxf(s.p, 0.f);
    // nothing below ``cut`` is kept
    float cut = -3.402823466e38f;
    if (s.by_rank || s.p < 1.f) {
      lowest = -block_top(sh, -lowest);
      const float per_bin = (BINS - 1) / (top - lowest);
      if (fits && per_bin > 0.f && per_bin < INFINITY) {
        clear_bins(sh);
        for (int i = tid; i < blocks; i += S_THREADS)
          if (maxima[i] > -INFINITY) {
            const int bin = min((int)((top - maxima[i]) * per_bin), BINS - 1);
            if (s.by_rank) atomicAdd(&sh.cnt[bin], 1u);
            else atomicAdd(&sh.mass[bin], weight(maxima[i]));
          }
        __syncthreads();
        const int e = 2 * tid;
        const u64 m[2] = {sh.mass[e], sh.mass[e + 1]};
        const uint32_t n[2] = {sh.cnt[e], sh.cnt[e + 1]};
        // (a little more than the share, whose sum was rounded otherwise)
        const u64 want = s.by_rank ? (u64)s.k : (u64)(ldexp(share * sum, scale) * (1. + 1e-9)) + 1;
        const Found f = s.by_rank ? find_entry<true>(sh, m, n, 0, 0, [&](u64) { return want; })
                                  : find_entry<false>(sh, m, n, 0, 0, [&](u64) { return want; });
        // every value of bins 0 .. f.at, with the roundings of a bin's number
        if (f.at >= 0) cut = top - (f.at + 1) / per_bin * 1.000001f;
      }
    } else {
      cut = (float)(top + log2((double)fminf(s.low, 1.f)) / c);
    }
    cut = fmaxf(cut - fabsf(cut) * 1e-6f, -3.402823466e38f);
    Row<T> row{z, V, cut, -1, list};
    if (fits) {
      __syncthreads();
      if (tid == 0) sh.found = 0;
      __syncthreads();
      for (int i = tid; i < blocks; i += S_THREADS)
        if (maxima[i] >= cut) {
          const int n = atomicAdd(&sh.found, 1);
          if (n < LIST) list[n] = i;
        }
      __syncthreads();
      if (sh.found <= LIST) row.n = sh.found;
    }
    row.fill();
    const uint32_t lo = order_key(cut), hi = order_key(top);
    // the lowest value that is kept, how many have it and how many of them are kept
    uint32_t border = 0, on = 0, kept_on = 0;
    u64 mass = 0;  // of what top-k keeps
    if (s.by_rank) {
      const Border b = find_border<true>(sh, row, lo, hi, weight, [&](u64) { return (u64)s.k; });
      border = b.key;
      on = b.cnt_on;
      kept_on = (uint32_t)(b.want - b.cnt_above);
      mass = b.mass_above + kept_on * weight(key_value(border));
    }
    if (s.p < 1.f) {
      const double of = s.by_rank ? (double)mass : ldexp(sum, scale);
      const Border b = find_border<false>(sh, row, max(lo, border), hi, weight,
                                          [&](u64) { return max((u64)ceil(share * of), (u64)1); });
      const u64 w = weight(key_value(b.key));
      border = b.key;
      on = b.cnt_on;
      kept_on = (uint32_t)((b.want - b.mass_above + w - 1) / w);
    }
    int last_on = V;  // the last index on the border that is kept
    if (kept_on < on)
      last_on = find_index(sh, row, [&](float v, int) { return (u64)(order_key(v) == border); },
                           [&](u64) { return (u64)kept_on; }, &total);
    const double least = s.low > 0.f ? (double)fminf(s.low, 1.f) : -1.;
    token = find_index(
        sh, row,
        [&](float v, int i) {
          const uint32_t key = order_key(v);
          if (v == -INFINITY || key < border || (key == border && i > last_on)) return (u64)0;
          const double w = weight_of(v);
          return w >= least ? fixed(w) : (u64)0;
        },
        drawn, &total);
  }
  if (tid == 0) {
    a.tokens[r] = token;
    const float v = sane(to_f32(z[token]));
    const double x = v == top ? 0. : ((double)v - top) / s.t;
    a.logps[r] = (float)(x - log(ldexp((double)total, -scale)));
  }
}

int64_t sample_workspace(int64_t rows, int vocab) { return rows * row_bytes(vocab); }

template <typename T>
static void launch(const SampleArgs& a, void* ws, hipStream_t s) {
  constexpr int PER = SCAN_THREADS / 64;
  sample_scan_kernel<T><<<dim3((chunks_of(a.vocab) + PER - 1) / PER, a.rows), SCAN_THREADS, 0, s>>>(a, ws);
  sample_row_kernel<T><<<a.rows, S_THREADS, 0, s>>>(a, ws);
}

void launch_sample(const SampleArgs& a, void* ws, hipStream_t s) {
  if (a.bf16_logits) launch<bf16>(a, ws, s);
  else launch<float>(a, ws, s);
}

}  // namespace axon
