// Row kernels of the GPT-2 family (the complete GPT-2 definition of the
// Technical Supplement): token + learned-position embedding with the first
// LayerNorm, and LayerNorm with gain and bias.  One workgroup of 256 threads
// per row; a thread keeps its (up to 8) groups of 4 features in registers, so
// the mean, the variance around it and the output come from one read of the
// row.  HBM/latency bound.
//
// Below them, layer norm over a caller's rows and its backward pass.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace axon {

constexpr int LN_MAXV = 8;  // rows of up to 8 * 1024 features

// h[row] = (v - mean) / sqrt(var + eps) * g + beta for the thread's feature
// groups; mean and the (biased) variance over the D features of the row.  pair:
// h in the row-pair layout (D % 32 == 0)
AXON_DEV void ln_store(const f32x4 (&v)[LN_MAXV], int D, float eps, const bf16* __restrict__ g,
                       const bf16* __restrict__ beta, bf16* __restrict__ h, int64_t row, bool pair, float* red) {
  const int t4 = threadIdx.x * 4;
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < LN_MAXV; ++j)
    if (t4 + j * 1024 < D) sum += (v[j][0] + v[j][1]) + (v[j][2] + v[j][3]);
  const float mean = block_sum(sum, red) / (float)D;
  float sq = 0.f;
#pragma unroll
  for (int j = 0; j < LN_MAXV; ++j)
    if (t4 + j * 1024 < D) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float d = v[j][c] - mean;
        sq += d * d;
      }
    }
  const float rstd = rsqrtf(block_sum(sq, red) / (float)D + eps);
#pragma unroll
  for (int j = 0; j < LN_MAXV; ++j) {
    const int i = t4 + j * 1024;
    if (i < D) {
      const bf16x4 gv = *(const bf16x4*)(g + i), bv = *(const bf16x4*)(beta + i);
      bf16x4 o;
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = (bf16)((v[j][c] - mean) * rstd * (float)gv[c] + (float)bv[c]);
      *(bf16x4*)(h + (pair ? xp_off(row, i, D) : row * D + i)) = o;
    }
  }
}

__global__ void __launch_bounds__(256) embed_pos_ln_kernel(const int32_t* __restrict__ tok,
                                                           const bf16* __restrict__ wte,
                                                           const bf16* __restrict__ wpe,
                                                           const bf16* __restrict__ g, const bf16* __restrict__ beta,
                                                           float* __restrict__ x, bf16* __restrict__ h, int D, int V,
                                                           int P, float eps, const int32_t* __restrict__ cu, int nseq,
                                                           const int32_t* __restrict__ ent_base,
                                                           const int32_t* __restrict__ len, bool pair) {
  __shared__ float red[16];
  const int t = blockIdx.x;
  int pos;
  if (len) {
    pos = len[t];
  } else {
    const int e = seq_of_token(cu, nseq, t);
    pos = (ent_base ? ent_base[e] : 0) + t - cu[e];
  }
  pos = min(max(pos, 0), P - 1);           // validated on the host; never read out of the table
  const int id = min(max(tok[t], 0), V - 1);  // ids outside [0, V) are clamped, never dereferenced
  f32x4 v[LN_MAXV];
#pragma unroll
  for (int j = 0; j < LN_MAXV; ++j) {
    const int i = threadIdx.x * 4 + j * 1024;
    if (i < D) {
      const bf16x4 a = *(const bf16x4*)(wte + wt_chunk(id, i >> 3, D) + (i & 7));  // fragment-tiled table
      const bf16x4 b = *(const bf16x4*)(wpe + (int64_t)pos * D + i);
#pragma unroll
      for (int c = 0; c < 4; ++c) v[j][c] = (float)a[c] + (float)b[c];
      *(f32x4*)(x + (int64_t)t * D + i) = v[j];
    }
  }
  ln_store(v, D, eps, g, beta, h, t, pair, red);
}

__global__ void __launch_bounds__(256) layernorm_kernel(const float* __restrict__ x, const bf16* __restrict__ g,
                                                        const bf16* __restrict__ beta, bf16* __restrict__ h, int D,
                                                        float eps, const int32_t* __restrict__ cu_last) {
  __shared__ float red[16];
  const int i_out = blockIdx.x;
  const int r = cu_last ? cu_last[i_out + 1] - 1 : i_out;
  f32x4 v[LN_MAXV];
#pragma unroll
  for (int j = 0; j < LN_MAXV; ++j) {
    const int i = threadIdx.x * 4 + j * 1024;
    if (i < D) v[j] = *(const f32x4*)(x + (int64_t)r * D + i);
  }
  ln_store(v, D, eps, g, beta, h, i_out, false, red);
}

void launch_embed_pos_ln(const int32_t* tok, const bf16* wte, const bf16* wpe, const bf16* g, const bf16* beta,
                         float* x, bf16* h, int T, int D, int V, int P, float eps, const int32_t* cu, int nseq,
                         const int32_t* ent_base, const int32_t* len, hipStream_t s, bool h_pair) {
  if (T <= 0) return;
  embed_pos_ln_kernel<<<T, 256, 0, s>>>(tok, wte, wpe, g, beta, x, h, D, V, P, eps, cu, nseq, ent_base, len, h_pair);
}

void launch_layernorm(const float* x, const bf16* g, const bf16* beta, bf16* h, int rows, int D, float eps,
                      const int32_t* cu_last, hipStream_t s) {
  if (rows <= 0) return;
  layernorm_kernel<<<rows, 256, 0, s>>>(x, g, beta, h, D, eps, cu_last);
}

// ---------------------------------------------------------------- rows of any width, forward and backward
//
// TPR threads share a row (a wavefront's 64, or a workgroup's 256 to 1024) and keep
// it in registers as NV groups of 8 consecutive columns each: group v of thread i
// starts at column (v * TPR + i) * 8, so a row is read once, 16 bytes a lane and
// load.  Rows may start at any element (their stride and width are free); of a width
// that is no multiple of 8 (ODD) the last few columns go to one thread each.  Every
// load is unconditional: threads past the row's end read its last columns again, which
// then count nothing.  (A load under a branch whose other arm fills the same registers
// is waited for there: nothing stays in flight.  Backward of 16384 x 8184 took 225 us
// that way, of 8192 columns 158.)
//
// A row's sums cost one exchange between its wavefronts: each takes the mean of its
// own columns first and its sums around that, and the joined ones follow from the
// wavefronts' (n_w columns, mean m_w, sum of squares Q_w around m_w; Chan, Golub and
// LeVeque's updating formula):
//   mean = sum n_w m_w / n,  Q = sum Q_w + n_w (m_w - mean)^2,
// so nothing is lost to a common offset of the row, as a sum of x^2 would lose it.

// what a thread holds of a row, and which of it counts
template <typename T, int NV, bool ODD>
struct RowRegs {
  Run8<T> g[NV];
  T t;  // ODD: one of the last cols % 8 columns
};
template <int TPR, int NV, bool ODD>
struct RowCols {
  int i, cols, whole;  // thread of the row; columns; those in groups of 8
  AXON_DEV explicit RowCols(int cols) : i(threadIdx.x % TPR), cols(cols), whole(ODD ? cols & ~7 : cols) {}
  AXON_DEV int at(int n) const { return (n * TPR + i) * 8; }
  AXON_DEV bool on(int n) const { return at(n) < whole; }
  AXON_DEV int tail() const { return whole + i; }
  AXON_DEV bool tail_on() const { return tail() < cols; }
  template <typename T>
  AXON_DEV void load(RowRegs<T, NV, ODD>& r, const T* row) const {
#pragma unroll
    for (int n = 0; n < NV; ++n)
      if (!ODD || whole > 0) r.g[n].load(row + min(at(n), whole - 8));
      else r.g[n].fill(0.f);  // (a row of fewer than 8 columns)
    if constexpr (ODD) r.t = row[min(tail(), cols - 1)];
  }
  // zero in what does not count, for factors that are kept
  template <typename T>
  AXON_DEV void mask(RowRegs<T, NV, ODD>& r) const {
#pragma unroll
    for (int n = 0; n < NV; ++n)
      if (!on(n)) r.g[n].fill(0.f);
    if constexpr (ODD)
      if (!tail_on()) r.t = from_f32<T>(0.f);
  }
  template <typename T>
  AXON_DEV void store(T* row, const float (&v)[NV][8], float t) const {
#pragma unroll
    for (int n = 0; n < NV; ++n)
      if (on(n)) Run8<T>::store(row + at(n), v[n]);
    if constexpr (ODD)
      if (tail_on()) row[tail()] = from_f32<T>(t);
  }
};

// a wavefront's sums over its columns of a row, h and hd for the backward pass only:
// mean, sum (x - mean)^2, sum h, sum h (x - mean)
struct __align__(16) RowSums {
  float mean, q, h, hd;
};
// what depends on the row's width alone, and the exchange.  Lane l joins what
// wavefront l % NW left: one 16-byte LDS read and log2 NW register moves a sum.
template <int TPR, int NV, bool ODD>
struct RowShape {
  static constexpr int NW = TPR / 64;
  float own;    // columns of this wavefront, at least 1
  float other;  // columns of wavefront lane % NW
  float all;    // columns of the row
  AXON_DEV explicit RowShape(int cols) {
    const int whole = ODD ? cols & ~7 : cols;
    auto count = [&](int wave) {
      int c = wave == 0 ? cols - whole : 0;
#pragma unroll
      for (int v = 0; v < NV; ++v) c += min(512, max(0, whole - (v * TPR + wave * 64) * 8));
      return (float)c;
    };
    own = fmaxf(count((threadIdx.x >> 6) % NW), 1.f);
    other = count(threadIdx.x % NW);
    all = (float)cols;
  }
  // over the lanes that differ in lane % NW; every lane the same result (see wave_sum)
  static AXON_DEV float over_waves(float v) {
    if constexpr (NW > 1) v += dpp_move<0xB1>(v);
    if constexpr (NW > 2) v += dpp_move<0x4E>(v);
    if constexpr (NW > 4) v += dpp_move<0x141>(v);
    if constexpr (NW > 8) v += dpp_move<0x140>(v);
    return v;
  }
  // the whole row's sums, around its mean, in every thread.  red: a slot per wavefront
  // that no wavefront may still read from an earlier call
  template <bool BWD>
  AXON_DEV RowSums join(RowSums w, RowSums* red) const {
    if constexpr (NW == 1) return w;
    if ((threadIdx.x & 63) == 0) red[(threadIdx.x >> 6) % NW] = w;
    __syncthreads();
    const RowSums p = red[threadIdx.x % NW];
    RowSums r{};
    r.mean = over_waves(other * p.mean) / all;
    const float d = p.mean - r.mean;
    r.q = over_waves(p.q + other * d * d);
    if (BWD) {
      r.h = over_waves(p.h);
      r.hd = over_waves(p.hd + d * p.h);
    }
    return r;
  }
};

// sums of a thread's columns: x, and around a mean (x - mean)^2
template <int TPR, int NV, bool ODD>
AXON_DEV float sum_cols(const RowCols<TPR, NV, ODD>& rc, const float (&v)[NV][8], float t) {
  float s = ODD && rc.tail_on() ? t : 0.f;
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    float g = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) g += v[n][j];
    s += rc.on(n) ? g : 0.f;
  }
  return s;
}
template <int TPR, int NV, bool ODD>
AXON_DEV float square_cols(const RowCols<TPR, NV, ODD>& rc, const float (&v)[NV][8], float t, float mean) {
  float s = ODD && rc.tail_on() ? (t - mean) * (t - mean) : 0.f;
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    float g = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) g += (v[n][j] - mean) * (v[n][j] - mean);
    s += rc.on(n) ? g : 0.f;
  }
  return s;
}

// y = (x - mean) rstd g + b, one row per TPR threads.  HBM bound.  The workgroups
// stay for several rows: g and b are loaded once, and the next row's loads are under
// way while this one is reduced.  PAIR: y in the row-pair layout (cols % 32 == 0).
template <typename TX, typename TY, typename TP, int TPR, int NV, bool ODD, bool PAIR = false>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR)
    ln_fwd_kernel(const TX* x, int64_t ldx, const TP* __restrict__ g, const TP* __restrict__ b, float eps, TY* y,
                  int64_t ldy, int64_t rows, int cols) {
  constexpr int RPW = TPR < 256 ? 256 / TPR : 1;  // rows of a workgroup
  __shared__ RowSums red[2][16];
  const RowCols<TPR, NV, ODD> rc(cols);
  const RowShape<TPR, NV, ODD> shape(cols);
  RowRegs<TP, NV, ODD> gv, bv;
  RowRegs<TX, NV, ODD> next;
  rc.load(gv, g);
  rc.load(bv, b ? b : g);
  // wave-uniform trip count: with TPR > 64 the whole workgroup shares the row
  const int64_t step = (int64_t)gridDim.x * RPW;
  int64_t r = (int64_t)blockIdx.x * RPW + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  if (r < rows) rc.load(next, x + r * ldx);
  for (int par = 0; r < rows; r += step, par ^= 1) {
    float v[NV][8], t = 0.f;
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[n][j] = next.g[n][j];
    if constexpr (ODD) t = to_f32(next.t);
    if (r + step < rows) rc.load(next, x + (r + step) * ldx);
    RowSums w{};
    w.mean = wave_sum(sum_cols(rc, v, t)) / shape.own;
    w.q = wave_sum(square_cols(rc, v, t, w.mean));
    w = shape.template join<false>(w, red[par]);
    const float rstd = rsqrtf(w.q / shape.all + eps);
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[n][j] = (v[n][j] - w.mean) * rstd * gv.g[n][j] + (b ? bv.g[n][j] : 0.f);
    if constexpr (ODD) t = (t - w.mean) * rstd * to_f32(gv.t) + (b ? to_f32(bv.t) : 0.f);
    if constexpr (PAIR) {
#pragma unroll
      for (int n = 0; n < NV; ++n)
        if (rc.on(n)) Run8<TY>::store(y + xp_off(r, rc.at(n), cols), v[n]);
    } else {
      rc.store(y + r * ldy, v, t);
    }
  }
}

// Backward of y = (x - mean) rstd g + b.  With h = dy g and d = x - mean:
//   dx = rstd h - rstd mean(h) - d rstd^3 mean(h d),  dg = sum dy d rstd,  db = sum dy
// (sums over the rows).  The statistics are taken from x again, which is read
// anyway.  HBM bound.  A workgroup takes every n-th row, TPR threads a row,
// every thread the same columns of each, so dg and db stay in registers until the
// workgroup leaves one partial row [2 cols] for the column sum.  The next row's
// operands are loaded before this row's reductions where registers allow it.
//
// TRAIN, the training step's form (float rows): dy is the sum of tr.np split-K
// partials in order; tr.accumulate: dx += instead of =; the new dx goes to tr.dxb in
// bf16 too (row-pair layout, the next projections' operand), and its column sums,
// the gradient of the bias that was added to the residual there, are a third
// part of the partial row [3 cols].
constexpr bool ln_ahead(int tpr, int nv) { return nv == 1 || (tpr > 64 && tpr < 1024); }

template <typename TX, typename TD, typename TP, int TPR, int NV, bool ODD, bool TRAIN>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR)
    ln_bwd_kernel(const TX* x, int64_t ldx, const TD* dy, int64_t lddy, const TP* __restrict__ g, float eps, TX* dx,
                  int64_t lddx, float* __restrict__ part, int64_t rows, int cols, LnTrain tr) {
  constexpr int RPW = TPR < 256 ? 256 / TPR : 1, SUMS = TRAIN ? 3 : 2;
  constexpr bool AHEAD = ln_ahead(TPR, NV);
  __shared__ RowSums red[2][16];
  const RowCols<TPR, NV, ODD> rc(cols);
  const RowShape<TPR, NV, ODD> shape(cols);
  RowRegs<TP, NV, ODD> gv;
  RowRegs<TX, NV, ODD> xn, an;
  RowRegs<TD, NV, ODD> dn;
  float dg[NV][8] = {}, db[NV][8] = {}, dr[NV][8] = {}, more[NV][8], dgt = 0.f, dbt = 0.f;
  rc.load(gv, g);
  rc.mask(gv);
  const int64_t step = (int64_t)gridDim.x * RPW;  // neighbouring rows at one time, over the chip
  auto load = [&](int64_t r) {
    rc.load(xn, x + r * ldx);
    rc.load(dn, dy + r * lddy);
    if constexpr (TRAIN) {
      if (tr.accumulate) rc.load(an, (const TX*)dx + r * lddx);
#pragma unroll
      for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int j = 0; j < 8; ++j) more[n][j] = 0.f;
      for (int p = 1; p < tr.np; ++p) {
        RowRegs<TD, NV, ODD> q;
        rc.load(q, dy + p * tr.stride + r * lddy);
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
          for (int j = 0; j < 8; ++j) more[n][j] += q.g[n][j];
      }
    }
  };
  int64_t r = (int64_t)blockIdx.x * RPW + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  if (AHEAD && r < rows) load(r);
  for (int par = 0; r < rows; r += step, par ^= 1) {
    float d[NV][8], e[NV][8], a[NV][8], dt = 0.f, et = 0.f;
    if (!AHEAD) load(r);
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        d[n][j] = xn.g[n][j];
        e[n][j] = dn.g[n][j] + (TRAIN ? more[n][j] : 0.f);
        a[n][j] = TRAIN && tr.accumulate ? an.g[n][j] : 0.f;
      }
    if constexpr (ODD) {
      dt = to_f32(xn.t);
      et = to_f32(dn.t);
    }
    if (AHEAD && r + step < rows) load(r + step);
    RowSums w{};
    w.mean = wave_sum(sum_cols(rc, d, dt)) / shape.own;
    w.q = wave_sum(square_cols(rc, d, dt, w.mean));
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) {  // past the row: g = 0
        const float h = e[n][j] * gv.g[n][j];
        w.h += h;
        w.hd += h * (d[n][j] - w.mean);
      }
    if constexpr (ODD) {
      const float h = et * to_f32(gv.t);
      w.h += h;
      w.hd += h * (dt - w.mean);
    }
    w.h = wave_sum(w.h);
    w.hd = wave_sum(w.hd);
    w = shape.template join<true>(w, red[par]);
    const float per_col = 1.f / shape.all;
    const float rstd = rsqrtf(w.q * per_col + eps);
    const float mh = w.h * per_col, k = rstd * rstd * (w.hd * per_col);
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float c = d[n][j] - w.mean;
        d[n][j] = rstd * (e[n][j] * gv.g[n][j] - mh - c * k);
        if (TRAIN) d[n][j] += a[n][j];
        dg[n][j] += e[n][j] * (c * rstd);
        db[n][j] += e[n][j];
        if (TRAIN) dr[n][j] += d[n][j];
      }
    if constexpr (ODD) {
      const float c = dt - w.mean;
      dt = rstd * (et * to_f32(gv.t) - mh - c * k);
      dgt += et * (c * rstd);
      dbt += et;
    }
    rc.store(dx + r * lddx, d, dt);
    if constexpr (TRAIN)
#pragma unroll
      for (int n = 0; n < NV; ++n)
        if (rc.on(n)) Run8<bf16>::store(tr.dxb + xp_off(r, rc.at(n), cols), d[n]);
  }
  float* out = part + (int64_t)blockIdx.x * SUMS * cols;
  if constexpr (RPW > 1) {  // the wavefronts' shares in order, a group of columns at a time
    __shared__ float sums[RPW - 1][64][SUMS * 8 + 3];
    const int w = threadIdx.x / TPR, i = rc.i;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      if (n > 0) __syncthreads();
      if (w > 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          sums[w - 1][i][j] = dg[n][j];
          sums[w - 1][i][8 + j] = db[n][j];
          if (TRAIN) sums[w - 1][i][SUMS * 8 - 8 + j] = dr[n][j];
        }
        sums[w - 1][i][SUMS * 8] = dgt;
        sums[w - 1][i][SUMS * 8 + 1] = dbt;
      }
      __syncthreads();
      if (w == 0)
        for (int k = 0; k < RPW - 1; ++k) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            dg[n][j] += sums[k][i][j];
            db[n][j] += sums[k][i][8 + j];
            if (TRAIN) dr[n][j] += sums[k][i][SUMS * 8 - 8 + j];
          }
          if (n == 0) {
            dgt += sums[k][i][SUMS * 8];
            dbt += sums[k][i][SUMS * 8 + 1];
          }
        }
    }
    if (w > 0) return;
  }
  rc.store(out, dg, dgt);
  rc.store(out + cols, db, dbt);
  if (TRAIN) rc.store(out + 2 * cols, dr, 0.f);
}

// Column c of part [n][C] summed in a fixed order: 64 interleaved groups of rows, then
// the groups in order, 16 columns a workgroup, so that a narrow layer norm's few
// columns still make a hundred workgroups.  Columns below c1 go to d0, below c2 to d1,
// the rest to d2; a null one is not written.
__global__ void __launch_bounds__(1024) ln_colsum_kernel(const float* __restrict__ part, int n, int C,
                                                         float* __restrict__ d0, int c1, float* __restrict__ d1, int c2,
                                                         float* __restrict__ d2) {
  __shared__ float sums[64][17];
  const int lane = threadIdx.x & 15, grp = threadIdx.x >> 4, c = blockIdx.x * 16 + lane;
  float s = 0.f;
  if (c < C)
    for (int i0 = grp; i0 < n; i0 += 64 * 8) {
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = i0 + q * 64 < n ? part[(int64_t)(i0 + q * 64) * C + c] : 0.f;
#pragma unroll
      for (int q = 0; q < 8; ++q) s += v[q];
    }
  sums[grp][lane] = s;
  __syncthreads();
  if (grp > 0 || c >= C) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 64; ++i) s += sums[i][lane];
  if (c < c1) d0[c] = s;
  else if (c < c2) d1[c - c1] = s;
  else if (d2) d2[c - c2] = s;
}

namespace {

void ln_colsum(const float* part, int n, int C, float* d0, int c1, float* d1, int c2, float* d2, hipStream_t s) {
  ln_colsum_kernel<<<(C + 15) / 16, 1024, 0, s>>>(part, n, C, d0, c1, d1, c2, d2);
}

// f(threads of a row, groups of 8 columns a thread, most workgroups) for rows of
// ``cols``, each a compile-time constant
template <int V>
struct Int {
  static constexpr int value = V;
};

// Threads by what a wavefront can hold without spilling; workgroups by what still
// fills the chip (each holds g and b, and in the backward pass leaves a partial row, so
// not more).  bf16, TB/s: forward 65536 x 384 5.3, 32768 x 768 5.7 (TPR 256: 3.9), 16384 x
// 4096 5.9, 16384 x 8192 6.0; backward 4.8, 4.8 (TPR 256: 1.7), 5.4, 5.5.  float32
// rows with bf16 outputs of 8192 x 1600: 6.2 and 4.8.
template <typename F>
void ln_fwd_shape(int cols, F&& f) {
  if (cols <= 512) f(Int<64>{}, Int<1>{}, 2048);
  else if (cols <= 1024) f(Int<64>{}, Int<2>{}, 4096);
  else if (cols <= 2048) f(Int<64>{}, Int<4>{}, 512);
  else if (cols <= 4096) f(Int<256>{}, Int<2>{}, 16384);
  else if (cols <= 8192) f(Int<512>{}, Int<2>{}, 16384);
  else f(Int<1024>{}, Int<2>{}, 16384);
}

template <typename F>
void ln_bwd_shape(int cols, F&& f) {
  if (cols <= 512) f(Int<64>{}, Int<1>{}, 1024);
  else if (cols <= 1024) f(Int<64>{}, Int<2>{}, 1024);
  else if (cols <= 2048) f(Int<64>{}, Int<4>{}, 256);
  else if (cols <= 4096) f(Int<256>{}, Int<2>{}, 256);
  else if (cols <= 8192) f(Int<512>{}, Int<2>{}, 256);
  else f(Int<1024>{}, Int<2>{}, 256);
}
// the training step's form keeps a third sum of the columns: one group a thread
template <typename F>
void ln_train_shape(int cols, F&& f) {
  if (cols <= 512) f(Int<64>{}, Int<1>{}, ROW_PARTS);
  else if (cols <= 2048) f(Int<256>{}, Int<1>{}, ROW_PARTS);
  else if (cols <= 4096) f(Int<512>{}, Int<1>{}, ROW_PARTS);
  else f(Int<1024>{}, Int<1>{}, ROW_PARTS);
}

// workgroups for ``rows`` at ``tpr`` threads each, at most ``most``: as many rows for each
unsigned ln_wgs(int64_t rows, int tpr, int most) {
  const int at_once = tpr < 256 ? 256 / tpr : 1;
  const int64_t turns = (rows + at_once - 1) / at_once, each = (turns + most - 1) / most;
  return (unsigned)((turns + each - 1) / each);
}

}  // namespace

int64_t ln_bwd_part_floats(int64_t rows, int cols) {
  int64_t n = 0;
  ln_bwd_shape(cols, [&](auto tpr, auto, int most) { n = ln_wgs(rows, decltype(tpr)::value, most); });
  return n * 2 * cols;
}

template <typename TX, typename TY, typename TP>
void launch_ln_fwd(const TX* x, int64_t ldx, const TP* g, const TP* b, float eps, TY* y, int64_t ldy, int64_t rows,
                   int cols, hipStream_t s) {
  if (rows <= 0) return;
  ln_fwd_shape(cols, [&](auto tpr, auto nv, int most) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    auto go = [&](auto kern) {
      kern<<<ln_wgs(rows, TPR, most), TPR < 256 ? 256 : TPR, 0, s>>>(x, ldx, g, b, eps, y, ldy, rows, cols);
    };
    cols % 8 ? go(ln_fwd_kernel<TX, TY, TP, TPR, NV, true>) : go(ln_fwd_kernel<TX, TY, TP, TPR, NV, false>);
  });
}

void launch_ln_fwd_pair(const float* x, const bf16* g, const bf16* b, float eps, bf16* y, int T, int D, hipStream_t s) {
  if (T <= 0) return;
  ln_fwd_shape(D, [&](auto tpr, auto nv, int most) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    ln_fwd_kernel<float, bf16, bf16, TPR, NV, false, true>
        <<<ln_wgs(T, TPR, most), TPR < 256 ? 256 : TPR, 0, s>>>(x, D, g, b, eps, y, D, T, D);
  });
}

template <typename TX, typename TD, typename TP>
void launch_ln_bwd(const TX* x, int64_t ldx, const TD* dy, int64_t lddy, const TP* g, float eps, TX* dx, int64_t lddx,
                   float* dg, float* db, float* part, int64_t rows, int cols, hipStream_t s) {
  if (rows <= 0) {  // sums over no rows
    launch_zero_i32((int32_t*)dg, cols, s);
    if (db) launch_zero_i32((int32_t*)db, cols, s);
    return;
  }
  ln_bwd_shape(cols, [&](auto tpr, auto nv, int most) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    const unsigned n = ln_wgs(rows, TPR, most);
    auto go = [&](auto kern) {
      kern<<<n, TPR < 256 ? 256 : TPR, 0, s>>>(x, ldx, dy, lddy, g, eps, dx, lddx, part, rows, cols, LnTrain{});
    };
    cols % 8 ? go(ln_bwd_kernel<TX, TD, TP, TPR, NV, true, false>) : go(ln_bwd_kernel<TX, TD, TP, TPR, NV, false, false>);
    ln_colsum(part, (int)n, 2 * cols, dg, cols, db, db ? 2 * cols : cols, nullptr, s);
  });
}

void launch_ln_bwd_train(const float* x, const bf16* g, const float* dy, const LnTrain& tr, int T, int D, float eps,
                         float* dx, float* dg, float* db, float* dres, float* part, hipStream_t s) {
  if (T <= 0) return;
  ln_train_shape(D, [&](auto tpr, auto nv, int most) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    const unsigned n = ln_wgs(T, TPR, most);
    ln_bwd_kernel<float, float, bf16, TPR, NV, false, true><<<n, TPR < 256 ? 256 : TPR, 0, s>>>(x, D, dy, D, g, eps, dx, D,
                                                                                        part, T, D, tr);
    ln_colsum(part, (int)n, 3 * D, dg, D, db, 2 * D, dres, s);
  });
}

#define LN_INSTANCE(TX, TY, TP)                                                                                  \
  template void launch_ln_fwd<TX, TY, TP>(const TX*, int64_t, const TP*, const TP*, float, TY*, int64_t, int64_t, \
                                          int, hipStream_t);                                                     \
  template void launch_ln_bwd<TX, TY, TP>(const TX*, int64_t, const TY*, int64_t, const TP*, float, TX*, int64_t, \
                                          float*, float*, float*, int64_t, int, hipStream_t);
LN_INSTANCE(float, float, float)
LN_INSTANCE(float, float, bf16)
LN_INSTANCE(float, bf16, float)
LN_INSTANCE(float, bf16, bf16)
LN_INSTANCE(bf16, float, float)
LN_INSTANCE(bf16, float, bf16)
LN_INSTANCE(bf16, bf16, float)
LN_INSTANCE(bf16, bf16, bf16)
#undef LN_INSTANCE

}  // namespace axon
