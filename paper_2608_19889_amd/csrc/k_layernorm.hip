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
                                                        float eps, const int32_t* __restrict__ cu_last, bool pair) {
  __shared__ float red[16];
  const int i_out = blockIdx.x;
  const int r = cu_last ? cu_last[i_out + 1] - 1 : i_out;
  f32x4 v[LN_MAXV];
#pragma unroll
  for (int j = 0; j < LN_MAXV; ++j) {
    const int i = threadIdx.x * 4 + j * 1024;
    if (i < D) v[j] = *(const f32x4*)(x + (int64_t)r * D + i);
  }
  ln_store(v, D, eps, g, beta, h, i_out, pair, red);
}

void launch_embed_pos_ln(const int32_t* tok, const bf16* wte, const bf16* wpe, const bf16* g, const bf16* beta,
                         float* x, bf16* h, int T, int D, int V, int P, float eps, const int32_t* cu, int nseq,
                         const int32_t* ent_base, const int32_t* len, hipStream_t s, bool h_pair) {
  if (T <= 0) return;
  embed_pos_ln_kernel<<<T, 256, 0, s>>>(tok, wte, wpe, g, beta, x, h, D, V, P, eps, cu, nseq, ent_base, len, h_pair);
}

void launch_layernorm(const float* x, const bf16* g, const bf16* beta, bf16* h, int rows, int D, float eps,
                      const int32_t* cu_last, hipStream_t s, bool h_pair) {
  if (rows <= 0) return;
  layernorm_kernel<<<rows, 256, 0, s>>>(x, g, beta, h, D, eps, cu_last, h_pair);
}

// ---------------------------------------------------------------- rows of any width, forward and backward
//
// TPR threads share a row (a wavefront's 64, or a workgroup's 256 to 1024) and keep
// it in registers as NV groups of 8 consecutive columns each: group v of thread i
// starts at column (v * TPR + i) * 8, so a row is read once, 16 bytes a lane and
// load.  Rows may start at any element (their stride and width are free): the wide
// loads ask for the element's alignment only, and the group that runs past the
// row's end is read and written one element at a time.

// sum over the TPR threads of a row, in every one of them; red: 16 floats per use
// that no earlier use still reads
template <int TPR>
AXON_DEV float row_sum(float v, float* red) {
  v = wave_sum(v);
  if constexpr (TPR == 64) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < TPR / 64; ++i) s += red[i];
  return s;
}

// y = (x - mean) rstd g + b, one row per TPR threads.  The mean first, then the
// variance around it, both from registers: no cancellation, one read of x.
template <typename TX, typename TY, typename TP, int TPR, int NV>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR)
    ln_fwd_kernel(const TX* x, int64_t ldx, const TP* __restrict__ g, const TP* __restrict__ b, float eps, TY* y,
                  int64_t ldy, int64_t rows, int cols) {
  constexpr int RPW = TPR < 256 ? 256 / TPR : 1;  // rows of a workgroup
  __shared__ float red[2][16];
  const int i = threadIdx.x % TPR;
  // wave-uniform trip count: with TPR > 64 the whole workgroup shares the row
  for (int64_t r = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR; r < rows; r += (int64_t)gridDim.x * RPW) {
    float v[NV][8];
    float s = 0.f;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      load_run8(x + r * ldx, (n * TPR + i) * 8, cols, v[n], 0.f);
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[n][j];
    }
    const float mean = row_sum<TPR>(s, red[0]) / (float)cols;
    float q = 0.f;
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = v[n][j] - mean;
        v[n][j] = d;
        q += (n * TPR + i) * 8 + j < cols ? d * d : 0.f;
      }
    const float rstd = 1.f / sqrtf(row_sum<TPR>(q, red[1]) / (float)cols + eps);
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * TPR + i) * 8;
      if (c >= cols) continue;
      float gv[8], bv[8] = {};
      load_run8(g, c, cols, gv, 0.f);
      if (b) load_run8(b, c, cols, bv, 0.f);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[n][j] = v[n][j] * rstd * gv[j] + bv[j];
      store_run8(y + r * ldy, c, cols, v[n]);
    }
  }
}

// Backward of y = (x - mean) rstd g + b.  With h = dy g and d = x - mean:
//   dx = rstd h - rstd mean(h) - d rstd^3 mean(h d),  dg = sum dy d rstd,  db = sum dy
// (sums over the rows).  The statistics are taken from x again, which is read
// anyway.  HBM bound.  A workgroup takes ``per`` rows in turn, TPR threads a row,
// every thread the same columns of each, so dg and db stay in registers until the
// workgroup leaves one partial row [2 cols] for the column sum; up to 8192 columns
// the next row's operands are loaded before this row's reductions.
//
// TRAIN, the training step's form (float rows): dy is the sum of tr.np split-K
// partials in order; tr.accumulate: dx += instead of =; the new dx goes to tr.dxb in
// bf16 too (row-pair layout, the next projections' operand), and its column sums,
// the gradient of the bias that was added to the residual there, are a third
// part of the partial row [3 cols].
template <typename TX, typename TD, typename TP, int TPR, int NV, bool TRAIN>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR)
    ln_bwd_kernel(const TX* x, int64_t ldx, const TD* dy, int64_t lddy, const TP* __restrict__ g, float eps, TX* dx,
                  int64_t lddx, float* __restrict__ part, int64_t rows, int cols, int64_t per, LnTrain tr) {
  constexpr int RPW = TPR < 256 ? 256 / TPR : 1, SUMS = TRAIN ? 3 : 2;
  __shared__ float red[2][4][16];
  const int i = threadIdx.x % TPR;
  const int64_t r1 = min(rows, ((int64_t)blockIdx.x + 1) * per);
  float gv[NV][8], dg[NV][8] = {}, db[NV][8] = {}, dr[NV][8] = {}, xn[NV][8], dn[NV][8], an[NV][8];
#pragma unroll
  for (int n = 0; n < NV; ++n) load_run8(g, (n * TPR + i) * 8, cols, gv[n], 0.f);
  auto load = [&](int64_t r) {
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      load_run8(x + r * ldx, (n * TPR + i) * 8, cols, xn[n], 0.f);
      load_run8(dy + r * lddy, (n * TPR + i) * 8, cols, dn[n], 0.f);
      if constexpr (TRAIN) {
#pragma unroll
        for (int j = 0; j < 8; ++j) an[n][j] = 0.f;
        if (tr.accumulate) load_run8(dx + r * lddx, (n * TPR + i) * 8, cols, an[n], 0.f);
      }
    }
    if constexpr (TRAIN)
      for (int p = 1; p < tr.np; ++p)
#pragma unroll
        for (int n = 0; n < NV; ++n) {
          float more[8];
          load_run8(dy + p * tr.stride + r * lddy, (n * TPR + i) * 8, cols, more, 0.f);
#pragma unroll
          for (int j = 0; j < 8; ++j) dn[n][j] += more[j];
        }
  };
  int64_t r = (int64_t)blockIdx.x * per + threadIdx.x / TPR;
  constexpr bool AHEAD = NV == 1;  // the registers of two rows at once, 128 a thread at most
  if (AHEAD && r < r1) load(r);
  for (int par = 0; r < r1; r += RPW, par ^= 1) {
    float d[NV][8], e[NV][8], a[NV][8];
    float s = 0.f;
    if (!AHEAD) load(r);
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        d[n][j] = xn[n][j];
        e[n][j] = dn[n][j];
        a[n][j] = TRAIN ? an[n][j] : 0.f;
        s += d[n][j];
      }
    if (AHEAD && r + RPW < r1) load(r + RPW);
    const float mean = row_sum<TPR>(s, red[par][0]) / (float)cols;
    float q = 0.f, sh = 0.f, shd = 0.f;
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) {  // past the row: g = dy = 0
        d[n][j] -= mean;
        const float h = e[n][j] * gv[n][j];
        q += (n * TPR + i) * 8 + j < cols ? d[n][j] * d[n][j] : 0.f;
        sh += h;
        shd += h * d[n][j];
      }
    q = wave_sum(q);
    sh = wave_sum(sh);
    shd = wave_sum(shd);
    if constexpr (TPR > 64) {
      if ((threadIdx.x & 63) == 0) {
        red[par][1][threadIdx.x >> 6] = q;
        red[par][2][threadIdx.x >> 6] = sh;
        red[par][3][threadIdx.x >> 6] = shd;
      }
      __syncthreads();
      q = sh = shd = 0.f;
#pragma unroll
      for (int w = 0; w < TPR / 64; ++w) {
        q += red[par][1][w];
        sh += red[par][2][w];
        shd += red[par][3][w];
      }
    }
    const float rstd = 1.f / sqrtf(q / (float)cols + eps);
    const float mh = sh / (float)cols, k = rstd * rstd * (shd / (float)cols);
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = rstd * (e[n][j] * gv[n][j] - mh - d[n][j] * k);
        if (TRAIN) o[j] += a[n][j];
        dg[n][j] += e[n][j] * (d[n][j] * rstd);
        db[n][j] += e[n][j];
        dr[n][j] += TRAIN && (n * TPR + i) * 8 < cols ? o[j] : 0.f;  // (TRAIN: cols a multiple of 32)
      }
      store_run8(dx + r * lddx, (n * TPR + i) * 8, cols, o);
      if constexpr (TRAIN)
        if ((n * TPR + i) * 8 < cols) store_run8(tr.dxb, xp_off(r, (n * TPR + i) * 8, cols), o);
    }
  }
  float* out = part + (int64_t)blockIdx.x * SUMS * cols;
  if constexpr (RPW > 1) {  // the wavefronts' shares in order
    static_assert(RPW == 4 && NV == 1, "one group of columns a lane");
    __shared__ float sums[3][64][SUMS * 8 + 1];
    const int w = threadIdx.x / TPR;
    if (w > 0)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sums[w - 1][i][j] = dg[0][j];
        sums[w - 1][i][8 + j] = db[0][j];
        if (TRAIN) sums[w - 1][i][SUMS * 8 - 8 + j] = dr[0][j];
      }
    __syncthreads();
    if (w > 0) return;
    for (int k = 0; k < 3; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dg[0][j] += sums[k][i][j];
        db[0][j] += sums[k][i][8 + j];
        if (TRAIN) dr[0][j] += sums[k][i][SUMS * 8 - 8 + j];
      }
  }
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    store_run8(out, (n * TPR + i) * 8, cols, dg[n]);
    store_run8(out + cols, (n * TPR + i) * 8, cols, db[n]);
    if (TRAIN) store_run8(out + 2 * cols, (n * TPR + i) * 8, cols, dr[n]);
  }
}

namespace {

// calls f(integral_constant TPR, integral_constant NV) for rows of ``cols``
template <int V>
struct Int {
  static constexpr int value = V;
};

template <typename F>
void ln_fwd_shape(int cols, F&& f) {
  if (cols <= 512) f(Int<64>{}, Int<1>{});
  else if (cols <= 1024) f(Int<64>{}, Int<2>{});
  else if (cols <= 2048) f(Int<256>{}, Int<1>{});
  else if (cols <= 4096) f(Int<256>{}, Int<2>{});
  else if (cols <= 8192) f(Int<512>{}, Int<2>{});
  else f(Int<1024>{}, Int<2>{});
}

template <typename F>
void ln_bwd_shape(int cols, F&& f) {
  if (cols <= 512) f(Int<64>{}, Int<1>{});
  else if (cols <= 2048) f(Int<256>{}, Int<1>{});
  else if (cols <= 4096) f(Int<512>{}, Int<1>{});
  else if (cols <= 8192) f(Int<1024>{}, Int<1>{});
  else f(Int<1024>{}, Int<2>{});
}

// rows of a workgroup of the backward kernel and the workgroups that leaves
int64_t ln_bwd_per(int64_t rows, int cols) {
  const int64_t step = cols <= 512 ? 4 : 1;  // rows a workgroup takes at once
  const int64_t per = (rows + ROW_PARTS - 1) / ROW_PARTS;
  return std::max(step, (per + step - 1) / step * step);
}

}  // namespace

int64_t ln_bwd_part_floats(int64_t rows, int cols) {
  const int64_t per = ln_bwd_per(rows, cols);
  return (rows + per - 1) / per * 2 * cols;
}

template <typename TX, typename TY, typename TP>
void launch_ln_fwd(const TX* x, int64_t ldx, const TP* g, const TP* b, float eps, TY* y, int64_t ldy, int64_t rows,
                   int cols, hipStream_t s) {
  if (rows <= 0) return;
  ln_fwd_shape(cols, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, RPW = TPR < 256 ? 256 / TPR : 1;
    const int64_t wgs = std::min<int64_t>((rows + RPW - 1) / RPW, 1 << 20);
    ln_fwd_kernel<TX, TY, TP, TPR, NV>
        <<<(unsigned)wgs, TPR < 256 ? 256 : TPR, 0, s>>>(x, ldx, g, b, eps, y, ldy, rows, cols);
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
  const int64_t per = ln_bwd_per(rows, cols), n = (rows + per - 1) / per;
  ln_bwd_shape(cols, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    ln_bwd_kernel<TX, TD, TP, TPR, NV, false><<<(unsigned)n, TPR < 256 ? 256 : TPR, 0, s>>>(
        x, ldx, dy, lddy, g, eps, dx, lddx, part, rows, cols, per, LnTrain{});
  });
  launch_colsum_final(part, (int)n, 2 * cols, dg, cols, db, db ? 2 * cols : cols, nullptr, s);
}

void launch_ln_bwd_train(const float* x, const bf16* g, const float* dy, const LnTrain& tr, int T, int D, float eps,
                         float* dx, float* dg, float* db, float* dres, float* part, hipStream_t s) {
  if (T <= 0) return;
  const int64_t per = ln_bwd_per(T, D), n = (T + per - 1) / per;
  ln_bwd_shape(D, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    if constexpr (NV == 1)  // D <= 8192
      ln_bwd_kernel<float, float, bf16, TPR, NV, true><<<(unsigned)n, TPR < 256 ? 256 : TPR, 0, s>>>(
          x, D, dy, D, g, eps, dx, D, part, T, D, per, tr);
  });
  launch_colsum_final(part, (int)n, 3 * D, dg, D, db, 2 * D, dres, s);
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
