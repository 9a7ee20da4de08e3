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
// A workgroup per row, which reads the row in every pass.
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
  float top;
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

template <typename T>
struct Row {
  const T* z;
  int V;
  template <typename F>
  AXON_DEV void each(F&& f) const {
    for (int i = threadIdx.x; i < V; i += S_THREADS) f(sane(to_f32(z[i])), i);
  }
};

// the value on the border in descending order, and what is above it
struct Border {
  uint32_t key;
  u64 mass_above;
  uint32_t cnt_above, cnt_on;
  u64 want;  // the target
};
template <bool COUNT, typename R, typename W, typename F>
AXON_DEV Border find_border(Shared& sh, const R& row, W&& weight, F&& target) {
  Border b{};
  uint32_t lo = 0, hi = 0xffffffffu;
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
      if (!b.want) b.want = target(total);
      return b.want;
    });
    const uint32_t bin = BINS - 1 - f.at;
    lo += bin << shift;
    hi = min(hi, lo + ((1u << shift) - 1));
    b = Border{lo, f.mass_before, f.cnt_before, f.cnt_in, b.want};
    if (lo == hi) return b;
  }
}

// the index at which the running sum of weight(z, i) reaches target(total)
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

template <typename T>
__global__ void __launch_bounds__(S_THREADS) sample_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int r = blockIdx.x, V = a.vocab;
  const Row<T> row{(const T*)a.logits + r * a.ld, V};
  const float t = a.temperature ? a.temperature[r] : a.temperature_all;
  const int k = a.top_k ? a.top_k[r] : a.top_k_all;
  const float p = a.top_p ? a.top_p[r] : a.top_p_all, low = a.min_p ? a.min_p[r] : a.min_p_all;
  float top = -INFINITY;
  row.each([&](float z, int) { top = fmaxf(top, z); });
  top = wave_max(top);
  if ((threadIdx.x & 63) == 0) ((float*)sh.mass)[threadIdx.x >> 6] = top;
  __syncthreads();
  for (int w = 0; w < 16; ++w) top = fmaxf(top, ((float*)sh.mass)[w]);
  if (top == -INFINITY) {
    if (threadIdx.x == 0) {
      a.tokens[r] = -1;
      a.logps[r] = 0.f;
    }
    return;
  }
  const bool greedy = !(t > 0.f);
  const int scale = 62 - (V > 1 ? 32 - __clz(V - 1) : 0);
  const double c = greedy ? 0. : 1.4426950408889634 / (double)t;
  auto weight_of = [&](float z) { return z == top ? 1. : exp2_neg(((double)z - top) * c); };
  auto weight = [&](float z) { return (u64)rint(ldexp(weight_of(z), scale)); };
  u64 total;
  if (greedy) {
    const int i = find_index(sh, row, [&](float z, int) { return (u64)(z == top); }, [](u64) { return (u64)1; }, &total);
    if (threadIdx.x == 0) {
      a.tokens[r] = i;
      a.logps[r] = 0.f;
    }
    return;
  }
  // the lowest value that is kept, how many have it and how many of them are kept
  uint32_t border = 0, on = 0, kept_on = 0;
  u64 mass = 0;  // of what top-k keeps
  if (k > 0 && k < V) {
    const Border b = find_border<true>(sh, row, weight, [&](u64) { return (u64)k; });
    border = b.key;
    on = b.cnt_on;
    kept_on = (uint32_t)(b.want - b.cnt_above);
    mass = b.mass_above + kept_on * weight(key_value(border));
  }
  if (p < 1.f) {
    const Border b = find_border<false>(sh, row, weight, [&](u64 sum) {
      const u64 of = mass ? mass : sum;
      return min(max((u64)ceil((double)fmaxf(p, 0.f) * (double)of), (u64)1), of);
    });
    const u64 w = weight(key_value(b.key));
    border = b.key;
    on = b.cnt_on;
    kept_on = (uint32_t)((b.want - b.mass_above + w - 1) / w);
  }
  int last_on = V;  // the last index on the border that is kept
  if (kept_on < on)
    last_on = find_index(sh, row, [&](float z, int) { return (u64)(order_key(z) == border); },
                         [&](u64) { return (u64)kept_on; }, &total);
  const double least = low > 0.f ? (double)fminf(low, 1.f) : -1.;
  const int i = find_index(
      sh, row,
      [&](float z, int i) {
        const uint32_t key = order_key(z);
        if (key < border || (key == border && i > last_on)) return (u64)0;
        const double w = weight_of(z);
        return w >= least ? (u64)rint(ldexp(w, scale)) : (u64)0;
      },
      [&](u64 sum) { return min((u64)((double)fminf(fmaxf(a.uniform[r], 0.f), 1.f) * (double)sum), sum - 1) + 1; },
      &total);
  if (threadIdx.x == 0) {
    a.tokens[r] = i;
    const float z = sane(to_f32(row.z[i]));
    const double x = z == top ? 0. : ((double)z - top) / t;
    a.logps[r] = (float)(x - log(ldexp((double)total, -scale)));
  }
}

void launch_sample(const SampleArgs& a, hipStream_t s) {
  if (a.rows <= 0) return;
  if (a.bf16_logits) sample_kernel<bf16><<<a.rows, S_THREADS, 0, s>>>(a);
  else sample_kernel<float><<<a.rows, S_THREADS, 0, s>>>(a);
}

}  // namespace axon
