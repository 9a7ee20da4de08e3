// The next token of every row of logits, from a given uniform number.
//
// With x_i = (z_i - max) / T the weights are w_i = exp(x_i).  Top-k, top-p and min-p
// each keep a beginning of the tokens in descending order of z (the lowest index first
// among equals), so together they keep the tokens above a border value and some of
// those on it.  The token is the first, in the order of the vocabulary, at which the
// running sum of the kept weights passes ``uniform`` of their sum.
//
// Which token that is must hang on no rounding of 32 bits and no order of additions: the
// weights are float64 (2^-51 of themselves) and summed as integers, W_i = w_i 2^(62 - log2 V)
// rounded (half of one a value), whose sums are exact and have no order, so that they can be
// added up by atomics.  The scan's sums of chunks, by which a draw without a filter finds its
// chunk and of whose total a top-p without a top-k takes its share, are float64 sums in a
// fixed order, off by 2^-46 of themselves; where such a sum and that of the chunk's integers
// differ at the end, the draw is the chunk's last token that has a weight.
//
// A border is found without sorting: a histogram (number and weight) over 2048 ranges of
// the values' bits, the range that the border is in, and again inside it.
//
// The logits are read once, by sample_scan_kernel: the maximum of every block of 32 and,
// where a row needs it, the weights' sum of every chunk of 2048.  What a filter keeps is
// above a value that the maxima alone give: k of them reach the k-th largest, or their
// weights the share p of the sum.  So sample_row_kernel, a workgroup per row, reads only
// the blocks whose maximum is above it (those of some hundred tokens where a row is sure
// of itself), which its few passes find in the L2; without a filter the sums lead it to
// the token's chunk.
//
// Measured: 384 rows of 128256 float32, each with its own settings, 62 us (scan 44, 4.5
// TB/s; the rest 17); 64 of 152064 with a nucleus 35 (scan 16: the float64 weights, some
// 100 cycles each to a wavefront, stand beside 8 of reading; the rest 19: a chain of some
// ten exchanges through LDS, 11 for most rows, 19 where 200 candidates are compared); 8 of
// 32000 with top-k and top-p 17 (4 + 12, latency).  A scan of fewer wavefronts that load a
// chunk ahead is slower: 20 and 56 us with 4096.  Where a top-p keeps more than 2048 blocks or
// values, its workgroup goes through the whole row for each histogram: 64 flat rows of 152064
// 330 us (bf16 295), without a filter or with a top-k 21.
#include "common.h"
#include "kernels.h"
#include "search_range.h"

namespace axon {

typedef unsigned long long u64;

// 2^x for x <= 0 as v 2^n, v in [0.7, 1.42]: 2^f on [-1/2, 1/2] as the polynomial of
// degree 10 through 2^f at Chebyshev's nodes, 4e-16 of itself off and exactly 1 at 0.
// Rounding to whole numbers by an addition, whose low bits are n, and no other conversion:
// those take four times as long as sums and products.
struct Exp2 {
  double v;
  int n;
};
AXON_DEV Exp2 exp2_neg(double x) {
  x = fmax(x, -1000.);  // (NaN, from infinities: no weight either)
  constexpr double WHOLE = 6755399441055744.;  // 1.5 2^52
  const double t = x + WHOLE, f = x - (t - WHOLE);
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
  return Exp2{fma(v, f, 1.), __double2loint(t)};
}
AXON_DEV double as_double(Exp2 e) {
  return __hiloint2double(__double2hiint(e.v) + (e.n << 20), __double2loint(e.v));
}
// round(v 2^(n + scale)) for scale <= 62: v + 2 has v's first 51 bits behind the point
AXON_DEV u64 as_fixed(Exp2 e, int scale) {
  const u64 m = ((u64)__double_as_longlong(e.v + 2.) & ((1ull << 52) - 1)) << 11;
  const int r = 62 - scale - e.n;
  return r > 63 ? 0 : (m + (r ? 1ull << (r - 1) : 0)) >> r;
}

// a logit as it is compared: NaN cannot be chosen, zeros have one sign
AXON_DEV float sane(float z) { return z == 0.f ? 0.f : z == z ? z : -INFINITY; }
// its bits in ascending order, as many as the type has
template <typename T>
AXON_DEV uint32_t order_key(float z) {
  const uint32_t u = __float_as_uint(z), k = u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
  return sizeof(T) == 2 ? k >> 16 : k;
}
template <typename T>
AXON_DEV float key_value(uint32_t k) {
  if (sizeof(T) == 2) k = k << 16 | (k >> 15 ? 0 : 0xffff);
  return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu));
}

// A value that a filter can keep.  Descending order is that of ``key``, one comparison: the
// value's bits in ascending order above those of -1 - index.
struct Candidate {
  u64 key, w;
  AXON_DEV float z() const { return key_value<float>((uint32_t)(key >> 32)); }
  AXON_DEV int i() const { return (int)~(uint32_t)key; }
};
AXON_DEV Candidate candidate(float z, int i, u64 w) { return Candidate{(u64)order_key<float>(z) << 32 | ~(uint32_t)i, w}; }
constexpr int FEW = 256;  // candidates that are compared each with each

AXON_DEV u64 wave_total(u64 v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
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
  double* chunk_sum;  // [chunks], relative to chunk_max
  float* chunk_max;   // [chunks]
};
inline __host__ __device__ int chunks_of(int V) { return (V + CHUNK - 1) / CHUNK; }
inline __host__ __device__ int64_t row_bytes(int V) { return ((int64_t)chunks_of(V) * (CHUNK_BLOCKS * 4 + 8 + 4) + 15) / 16 * 16; }
AXON_DEV RowSums row_sums(void* ws, int r, int V) {
  const int n = chunks_of(V);
  float* p = (float*)((char*)ws + r * row_bytes(V));
  return RowSums{p, (double*)(p + n * CHUNK_BLOCKS), p + n * (CHUNK_BLOCKS + 2)};
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
  if (fabsf(all) < INFINITY) {
#pragma unroll
    for (int j = 0; j < ROUNDS; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) sum += as_double(exp2_neg(((double)v[j][i] - all) * c));
  } else if (all > 0.f) {  // infinities share all
#pragma unroll
    for (int j = 0; j < ROUNDS; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) sum += v[j][i] == all ? 1. : 0.;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) out.chunk_sum[chunk] = sum;
}

// ---------------------------------------------------------------- the rest of a row

constexpr int LIST = 2048;        // blocks that are listed; more: all of the row
constexpr int MAX_BLOCKS = 8192;  // maxima that fit into LDS (262144 logits)
constexpr int KEPT = MAX_BLOCKS * 4 / sizeof(Candidate);  // candidates that fit into their place

// What a workgroup of S_THREADS does for its row
template <int S_THREADS>
struct RowOf {
  static constexpr int EACH = BINS / S_THREADS;  // of BINS entries, a thread's
  static constexpr int SHARE = S_THREADS / FEW;  // threads of a candidate

  struct Shared {
    u64 bins[BINS];
    Candidate few[FEW];
    u64 wave_sum[S_THREADS / 64];
    u64 before, in;
    int found, count;
    u64 sum[2];
    float red[S_THREADS / 64];
  };

  static AXON_DEV void clear_bins(Shared& sh) {
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += S_THREADS) sh.bins[i] = 0;
    if (threadIdx.x == 0) sh.found = -1;
    __syncthreads();
  }

  // Over each thread's EACH entries, in the threads' order: the entry at which the running
  // sum (from ``from`` on) reaches target(total) >= 1; what is before it and in it.  -1:
  // none does, which is so only where a caller asks for more than there is.
  struct Found {
    int at;
    u64 before, in;
  };
  template <typename F>
  static AXON_DEV Found find_entry(Shared& sh, const u64 (&v)[EACH], u64 from, F&& target, u64* total = nullptr) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 mine = 0;
  #pragma unroll
    for (int j = 0; j < EACH; ++j) mine += v[j];
    u64 upto = mine;
  #pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const u64 u = __shfl_up(upto, d);
      if (lane >= d) upto += u;
    }
    if (lane == 63) sh.wave_sum[wave] = upto;
    if (threadIdx.x == 0) sh.found = -1;
    __syncthreads();
    u64 before = from + upto - mine, sum = from;
  #pragma unroll
    for (int w = 0; w < S_THREADS / 64; ++w) {
      before += w < wave ? sh.wave_sum[w] : 0;
      sum += sh.wave_sum[w];
    }
    const u64 want = target(sum);
    if (total) *total = sum;
  #pragma unroll
    for (int j = 0; j < EACH; ++j) {
      if (before < want && want <= before + v[j]) {
        sh.found = EACH * threadIdx.x + j;
        sh.before = before;
        sh.in = v[j];
      }
      before += v[j];
    }
    __syncthreads();
    return Found{sh.found, sh.before, sh.in};
  }

  // The values of a row that can matter: those of the listed blocks, or (n < 0) of all.
  // What is below ``cut`` is passed over.
  template <typename T>
  struct Row {
    static constexpr int N = RUN<T>, LANES = BLOCK / N;
    const T* z;
    int V;
    float cut;
    int n;
    const int32_t* list;
    const Candidate* kept;  // the values not below ``cut``, if they are here already (n_kept >= 0)
    int n_kept;
    AXON_DEV int items() const { return n < 0 ? (V + N - 1) / N : n * LANES; }
    AXON_DEV int first(int e) const { return n < 0 ? e * N : list[e / LANES] * BLOCK + e % LANES * N; }
    template <typename F>
    AXON_DEV void each(F&& f) const {
      if (n_kept >= 0) {
        for (int e = threadIdx.x; e < n_kept; e += S_THREADS) f(kept[e].z(), kept[e].i());
        return;
      }
      float v[N], next[N];
      const int end = items();
      if ((int)threadIdx.x < end) load_run(z, first(threadIdx.x), V, v);
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

  // up to ``most`` values of the row that ``take`` takes, in ``to`` in any order; their number
  // (more than ``most``: not all of them are there)
  template <typename R, typename P, typename W>
  static AXON_DEV int gather(Shared& sh, Candidate* to, int most, const R& row, P&& take, W&& weight) {
    __syncthreads();
    if (threadIdx.x == 0) {
      sh.count = 0;
      sh.found = -1;
    }
    __syncthreads();
    row.each([&](float z, int i) {
      if (!take(z)) return;
      const int n = atomicAdd(&sh.count, 1);
      if (n < most) to[n] = candidate(z, i, weight(z));
    });
    __syncthreads();
    const int n = sh.count;
    // (whole rounds of others())
    if ((int)threadIdx.x < 32 && n + (int)threadIdx.x < most) to[n + threadIdx.x] = Candidate{0, 0};
    __syncthreads();
    return n;
  }
  // SHARE threads to a candidate (thread / SHARE): f(candidate) over a part each, eight at a
  // time so that their reads are in flight together
  template <typename F>
  static AXON_DEV void others(const Candidate* all, int n, F&& f) {
    static_assert(FEW % 32 == 0 && 32 % (8 * SHARE) == 0, "rounds end inside few");
    for (int j = threadIdx.x % SHARE; j < n; j += 8 * SHARE) {
      Candidate c[8];
  #pragma unroll
      for (int k = 0; k < 8; ++k) c[k] = all[j + SHARE * k];
  #pragma unroll
      for (int k = 0; k < 8; ++k) f(c[k]);
    }
  }
  template <typename V>
  static AXON_DEV V share_sum(V v) {
  #pragma unroll
    for (int d = 1; d < SHARE; d <<= 1) v += __shfl_xor(v, d);
    return v;
  }

  // The border in descending order: values above key are kept, of those on it the indices
  // up to last.  COUNT: ``want`` values are kept, else as many as it takes for their weights
  // to reach ``want``; all there are if that is not reached.  A search that finds nothing
  // (none does) ends it with all of the range.
  struct Border {
    uint32_t key;
    int last;
  };
  template <bool COUNT, typename T, typename W>
  static AXON_DEV Border find_border(Shared& sh, const Row<T>& row, uint32_t lo, uint32_t hi, W&& weight, u64 want) {
    u64 above = 0;  // (number or weight) of what is above hi
    KeyRange range{lo, hi};
    for (;;) {
      lo = range.lo;
      hi = range.hi;
      const int shift = range.shift();
      clear_bins(sh);
      row.each([&](float z, int) {
        const uint32_t k = order_key<T>(z);
        if (k < lo || k > hi) return;
        const u64 w = COUNT ? 1 : weight(z);
        if (w) atomicAdd(&sh.bins[(k - lo) >> shift], w);
      });
      __syncthreads();
      u64 v[EACH];
  #pragma unroll
      for (int j = 0; j < EACH; ++j) v[j] = sh.bins[BINS - 1 - EACH * threadIdx.x - j];
      const Found f = find_entry(sh, v, above, [&](u64 total) { return want = min(want, total); });
      if (!range.narrow(f.at)) return Border{lo, row.V};
      lo = range.lo;
      hi = range.hi;
      above = f.before;
      if (lo == hi) {
        // all have one value: as many of them as are wanted, the lowest indices
        const u64 each = COUNT ? 1 : weight(key_value<T>(lo)), most = f.in / each, take = (want - above + each - 1) / each;
        int last = row.V;
        if (take < most) {
          const int width = (row.V + BINS - 1) / BINS;  // <= BINS
          clear_bins(sh);
          row.each([&](float z, int i) {
            if (order_key<T>(z) == lo) atomicAdd(&sh.bins[i / width], (u64)1);
          });
          __syncthreads();
          u64 b[EACH];
  #pragma unroll
          for (int j = 0; j < EACH; ++j) b[j] = sh.bins[EACH * threadIdx.x + j];
          const Found g = find_entry(sh, b, 0, [&](u64) { return take; });
          u64 w[EACH];
  #pragma unroll
          for (int j = 0; j < EACH; ++j) {
            const int in = EACH * threadIdx.x + j, i = max(g.at, 0) * width + in;
            w[j] = in < width && i < row.V && order_key<T>(sane(to_f32(row.z[i]))) == lo;
          }
          __syncthreads();
          last = g.at * width + find_entry(sh, w, g.before, [&](u64) { return take; }).at;
        }
        return Border{lo, last};
      }
      const int n = gather(sh, sh.few, FEW, row, [&](float z) { const uint32_t k = order_key<T>(z); return lo <= k && k <= hi; },
                           [&](float z) { return COUNT ? (u64)1 : weight(z); });
      if (n <= FEW) {  // few enough to compare
        const int i = threadIdx.x / SHARE;
        if (i < n) {
          const Candidate me = sh.few[i];
          u64 before = 0;
          others(sh.few, n, [&](const Candidate& c) { before += c.key > me.key ? c.w : 0; });
          before = above + share_sum(before);
          if (threadIdx.x % SHARE == 0 && before < want && want <= before + me.w) sh.found = i;
        }
        __syncthreads();
        if (sh.found < 0) return Border{lo, row.V};
        const Candidate me = sh.few[sh.found];
        return Border{order_key<T>(me.z()), me.i()};
      }
    }
  }

  // the workgroup's sum of f over the row's values
  template <typename R, typename F>
  static AXON_DEV u64 row_sum(Shared& sh, const R& row, F&& f) {
    u64 sum = 0;
    row.each([&](float z, int i) { sum += f(z, i); });
    sum = wave_total(sum);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.wave_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = 0;
  #pragma unroll
    for (int w = 0; w < S_THREADS / 64; ++w) sum += sh.wave_sum[w];
    return sum;
  }

  // The index at which the running sum of weight(z, i) reaches target(total), which is set.
  // weight is 0 below the row's cut.
  template <typename T, typename W, typename F>
  static AXON_DEV int find_index(Shared& sh, const Row<T>& row, W&& weight, F&& target, u64* total) {
    int width = (row.V + BINS - 1) / BINS;  // of a bin, <= BINS
    clear_bins(sh);
    if (row.n >= 0) {
      row.each([&](float z, int i) {
        const u64 w = weight(z, i);
        if (w) atomicAdd(&sh.bins[i / width], w);
      });
    } else {
      // all of the row: a wavefront adds up a chunk
      width = CHUNK;
      for (int c = threadIdx.x >> 6; c < chunks_of(row.V); c += S_THREADS / 64) {
        u64 sum = 0;
  #pragma unroll 2
        for (int j = 0; j < CHUNK / (64 * RUN<T>); ++j) {
          float v[RUN<T>];
          const int first = c * CHUNK + (j * 64 + (threadIdx.x & 63)) * RUN<T>;
          load_run(row.z, first, row.V, v);
  #pragma unroll
          for (int i = 0; i < RUN<T>; ++i)
            if (v[i] >= row.cut) sum += weight(v[i], first + i);
        }
        sum = wave_total(sum);
        if ((threadIdx.x & 63) == 0) sh.bins[c] = sum;
      }
    }
    __syncthreads();
    u64 want = 0;
    const int e = EACH * threadIdx.x;
    u64 v[EACH];
  #pragma unroll
    for (int j = 0; j < EACH; ++j) v[j] = sh.bins[e + j];
    const Found f = find_entry(sh, v, 0, [&](u64 t) { return want = target(t); }, total);
    u64 w[EACH];
  #pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const int i = max(f.at, 0) * width + e + j;
      const float z = i < row.V ? sane(to_f32(row.z[i])) : -INFINITY;
      w[j] = e + j < width && z >= row.cut ? weight(z, i) : 0;
    }
    __syncthreads();
    return f.at * width + find_entry(sh, w, f.before, [&](u64) { return want; }).at;
  }

  // the workgroup's maximum
  static AXON_DEV float block_top(Shared& sh, float v) {
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.red[threadIdx.x >> 6] = v;
    __syncthreads();
  #pragma unroll
    for (int w = 0; w < S_THREADS / 64; ++w) v = fmaxf(v, sh.red[w]);
    return v;
  }

  template <typename T>
  static AXON_DEV void run(const SampleArgs& a, void* ws, Shared& sh, float* maxima, int32_t* list) {
    constexpr float LOWEST = -3.402823466e38f;
    const int r = blockIdx.x, V = a.vocab, chunks = chunks_of(V), blocks = chunks * CHUNK_BLOCKS, tid = threadIdx.x;
    const T* z = (const T*)a.logits + r * a.ld;
    const RowSums in = row_sums(ws, r, V);
    const Settings s = settings_of(a, r);
    const float uniform = a.uniform[r];
    const bool filtered = !s.greedy && (s.by_rank || s.p < 1.f || s.low > 0.f), fits = blocks <= MAX_BLOCKS;
    // (loads of everything that is needed, in flight together)
    const float chunk_max = tid < chunks ? in.chunk_max[tid] : -INFINITY;
    const bool summed = needs_sum(s);
    const double chunk_sum = summed && tid < chunks ? in.chunk_sum[tid] : 0.;
    float top = chunk_max, lowest = INFINITY;  // of the maxima that are numbers
    for (int i = tid + S_THREADS; i < chunks; i += S_THREADS) top = fmaxf(top, in.chunk_max[i]);
    if (filtered && fits) {
      f32x4 m[MAX_BLOCKS / (4 * S_THREADS)];
  #pragma unroll
      for (int j = 0; j < MAX_BLOCKS / (4 * S_THREADS); ++j) {
        const int i = 4 * (j * S_THREADS + tid);
        m[j] = i < blocks ? *(const f32x4*)(in.block_max + i) : f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      }
  #pragma unroll
      for (int j = 0; j < MAX_BLOCKS / (4 * S_THREADS); ++j) {
        const int i = 4 * (j * S_THREADS + tid);
        if (i < blocks) *(f32x4*)(maxima + i) = m[j];
  #pragma unroll
        for (int k = 0; k < 4; ++k)
          if (m[j][k] > -INFINITY) lowest = fminf(lowest, m[j][k]);
      }
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
    const double c = per_unit(s), unit = ldexp(1., scale);
    auto parts = [&](float v) { return exp2_neg(v == top ? 0. : ((double)v - top) * c); };
    auto weight = [&](float v) { return as_fixed(parts(v), scale); };
    // the place in the kept weights' running sum, 1 .. sum
    auto drawn = [&](u64 sum) {
      return min((u64)((double)fminf(fmaxf(uniform, 0.f), 1.f) * (double)sum), sum - 1) + 1;
    };
    u64 total = 0;
    int token;
    if (!filtered) {
      u64 w[EACH], want = 0;
  #pragma unroll
      for (int j = 0; j < EACH; ++j) {
        const int i = EACH * tid + j;
        const float m = i < chunks ? in.chunk_max[i] : -INFINITY;
        // (a chunk whose weights are all 0 is not one to look in)
        w[j] = m > -INFINITY && weight(m) ? (u64)rint(as_double(parts(m)) * in.chunk_sum[i] * unit) : 0;
      }
      const Found f = find_entry(sh, w, 0, [&](u64 sum) { return want = drawn(sum); }, &total);
      const int first = max(f.at, 0) * CHUNK + EACH * tid;
  #pragma unroll
      for (int j = 0; j < EACH; ++j) {
        const float v = first + j < V ? sane(to_f32(z[first + j])) : -INFINITY;
        w[j] = v > -INFINITY ? weight(v) : 0;
      }
      __syncthreads();
      token = f.at * CHUNK + find_entry(sh, w, 0, [&](u64 sum) { return min(want - f.before, sum); }).at;
    } else {
      const double share = (double)fmaxf(s.p, 0.f), least = s.low > 0.f ? (double)fminf(s.low, 1.f) : -1.;
      double sum = 0.;  // of all weights
      if (summed) {
        if (chunk_max > -INFINITY) sum = as_double(parts(chunk_max)) * chunk_sum;
        for (int i = tid + S_THREADS; i < chunks; i += S_THREADS) {
          const float m = in.chunk_max[i];
          if (m > -INFINITY) sum += as_double(parts(m)) * in.chunk_sum[i];
        }
  #pragma unroll
        for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
        if ((tid & 63) == 0) sh.wave_sum[tid >> 6] = __double_as_longlong(sum);
        __syncthreads();
        sum = 0.;
  #pragma unroll
        for (int w = 0; w < S_THREADS / 64; ++w) sum += __longlong_as_double(sh.wave_sum[w]);
      }
      // Nothing below ``cut`` is kept (a top-k's weight, of which top-p takes its share,
      // has to be there in full).
      float cut = LOWEST;
      if (s.low > 0.f && !(s.by_rank && s.p < 1.f)) cut = (float)(top + log2(least) / c);
      if (s.by_rank || s.p < 1.f) {
        lowest = -block_top(sh, -lowest);
        const float per_bin = (BINS - 1) / (top - lowest);
        if (fits && per_bin > 0.f && per_bin < INFINITY) {
          clear_bins(sh);
          // (the share, a little more: these weights are rounded differently)
          const u64 want = s.by_rank ? (u64)s.k : (u64)(share * sum * (1ll << 32) * 1.0001) + 1;
          const float c32 = (float)c;
          for (int i = tid; i < blocks; i += S_THREADS) {
            const float m = maxima[i];
            if (m > -INFINITY)
              atomicAdd(&sh.bins[min((int)((top - m) * per_bin), BINS - 1)],
                        s.by_rank ? (u64)1 : (u64)(__builtin_amdgcn_exp2f((m - top) * c32) * 4294967296.f));
          }
          __syncthreads();
          u64 v[EACH];
  #pragma unroll
          for (int j = 0; j < EACH; ++j) v[j] = sh.bins[EACH * tid + j];
          const Found f = find_entry(sh, v, 0, [&](u64) { return want; });
          // every value of bins 0 .. f.at, with the roundings of a bin's number
          if (f.at >= 0) cut = fmaxf(cut, top - (f.at + 1) / per_bin * 1.000001f);
        }
      }
      cut = fmaxf(cut - fabsf(cut) * 1e-6f, LOWEST);
      Row<T> row{z, V, cut, -1, list, nullptr, -1};
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
      // (the maxima are not needed any more)
      Candidate* kept = (Candidate*)maxima;
      const int n = row.n < 0 ? KEPT + 1 : gather(sh, kept, KEPT, row, [](float) { return true; }, weight);
      if (n <= FEW) {
        // few: each compared with each, by rank and weight, then by index
        if (tid == 0) sh.sum[0] = sh.sum[1] = 0;
        if (tid == 0) sh.found = 0;
        __syncthreads();
        const int me = tid / SHARE;
        const bool leads = me < n && tid % SHARE == 0;
        const Candidate x = kept[min(me, n - 1)];
        u64 before = 0;
        uint32_t rank = 0;
        others(kept, n, [&](const Candidate& o) {
          const bool is = o.key > x.key;
          rank += is;
          before += is ? o.w : 0;
        });
        rank = share_sum(rank);
        before = share_sum(before);
        const bool first = !s.by_rank || rank < (uint32_t)s.k;
        if (s.by_rank && s.p < 1.f) {
          if (leads && first) atomicAdd(&sh.sum[0], x.w);
          __syncthreads();
        }
        const double of = s.by_rank ? (double)sh.sum[0] : sum * unit;
        bool stays = first && x.w > 0 && (double)x.w >= least * unit;
        if (s.p < 1.f) stays = stays && before < max((u64)ceil(share * of), (u64)1);
        if (leads && stays) atomicAdd(&sh.sum[1], x.w);
        __syncthreads();
        if (leads && !stays) kept[me].w = 0;
        __syncthreads();
        total = sh.sum[1];
        const u64 want = drawn(total);
        before = 0;
        others(kept, n, [&](const Candidate& o) { before += (uint32_t)o.key > (uint32_t)x.key ? o.w : 0; });
        before = share_sum(before);
        if (leads && stays && before < want && want <= before + x.w) sh.found = x.i();
        __syncthreads();
        token = sh.found;
      } else {
        if (n <= KEPT) {
          row.kept = kept;
          row.n_kept = n;
        }
        const uint32_t lo = order_key<T>(cut), hi = order_key<T>(top);
        Border b{0, V};
        if (s.by_rank) b = find_border<true>(sh, row, lo, hi, weight, (u64)s.k);
        if (s.p < 1.f) {
          const double of = s.by_rank ? (double)row_sum(sh, row, [&](float v, int i) {
            const uint32_t k = order_key<T>(v);
            return k > b.key || (k == b.key && i <= b.last) ? weight(v) : 0;
          }) : sum * unit;
          b = find_border<false>(sh, row, max(lo, b.key), hi, weight, max((u64)ceil(share * of), (u64)1));
        }
        token = find_index(
            sh, row,
            [&](float v, int i) {
              const uint32_t k = order_key<T>(v);
              if (v == -INFINITY || k < b.key || (k == b.key && i > b.last)) return (u64)0;
              const u64 w = weight(v);
              return (double)w >= least * unit ? w : (u64)0;
            },
            drawn, &total);
      }
    }
    if (tid == 0) {
      token = min(max(token, 0), V - 1);  // (it is there; no address hangs on it)
      a.tokens[r] = token;
      const float v = sane(to_f32(z[token]));
      const double x = v == top ? 0. : ((double)v - top) / s.t;
      a.logps[r] = (float)(x - log((double)total / unit));
    }
  }
};

template <typename T, int S_THREADS>
__global__ void __launch_bounds__(S_THREADS, 4) sample_row_kernel(SampleArgs a, void* ws) {
  using R = RowOf<S_THREADS>;
  __shared__ typename R::Shared sh;
  __shared__ alignas(16) float maxima[MAX_BLOCKS];
  __shared__ int32_t list[LIST];
  R::template run<T>(a, ws, sh, maxima, list);
}

int64_t sample_workspace(int64_t rows, int vocab) { return rows * row_bytes(vocab); }

template <typename T>
static void launch(const SampleArgs& a, void* ws, hipStream_t s) {
  constexpr int PER = SCAN_THREADS / 64;
  sample_scan_kernel<T><<<dim3((chunks_of(a.vocab) + PER - 1) / PER, a.rows), SCAN_THREADS, 0, s>>>(a, ws);
  // One large workgroup's registers fill a CU; two small ones have room, which counts
  // where rows are more than CUs (384 rows with their own settings 26 and 20 us, 64 with
  // a nucleus 21 and 26, measured before candidates had one key to compare).
  if (a.rows <= 256) sample_row_kernel<T, 1024><<<a.rows, 1024, 0, s>>>(a, ws);
  else sample_row_kernel<T, 512><<<a.rows, 512, 0, s>>>(a, ws);
}

void launch_sample(const SampleArgs& a, void* ws, hipStream_t s) {
  if (a.bf16_logits) launch<bf16>(a, ws, s);
  else launch<float>(a, ws, s);
}

}  // namespace axon
