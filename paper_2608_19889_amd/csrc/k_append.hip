// New tokens into a paged cache: queries and keys rotated by their position, keys and
// values stored in their pages.
//
// The pair (a, b) of dimension j of a head at position t turns by the angle
// t inv_freq[j]:  (a cos - b sin, b cos + a sin), times ``scale``; the pairs are
// dimensions (j, rot/2 + j) or (2j, 2j + 1) of the first ``rot`` ones.  The angle is a
// float64 product: at position 10^6 a float32 one is off by 0.03 of a radian.  It is
// reduced to half a turn either way with 1 / (2 pi) in two parts and the product's low
// digits kept: with one part a position of 4 10^8 is off by 4 10^-8 of a radian, however
// small the angle that is left.  Cosine and sine are float32 from there, and a value is
// rounded once, when it is stored.
//
// Each element is read once and written once, nothing else is moved: 17000 prompt tokens
// of 28 query and 2 x 4 key and value heads of 128 (bf16, 307 MB) take 56 us, 5.5 TB/s;
// one token of each of 8 sequences 3.6 us, a launch and the loads length, page, row.
#include "common.h"
#include "kernels.h"

namespace axon {

constexpr int APPEND_THREADS = 256;
constexpr int MAX_HALF = 64;  // pairs of a head

// the sequence of token t among cu[0 .. n] (n: behind the last one), all lanes of a
// wavefront together
AXON_DEV int find_sequence(const int32_t* cu, int n, int t) {
  int b = 0;
  for (int i = threadIdx.x & 63; i - (int)(threadIdx.x & 63) < n; i += 64)
    b += __popcll(__ballot(i < n && cu[i + 1] <= t));
  return b;
}

// 16 bytes of a head, of any element alignment in the caller's rows
template <typename T>
constexpr int RUN = 16 / sizeof(T);
template <typename T>
struct Run {
  typedef typename std::conditional<sizeof(T) == 2, bf16x8_any, f32x4_any>::type V;
  V v;
  AXON_DEV void load(const T* p) { v = *(const V*)p; }
  AXON_DEV void store(T* p) const { *(V*)p = v; }
};

// Where a token's head lies in its row and where it goes
template <typename T>
struct Place {
  const T* src;
  T* dst;
};

// A workgroup per token.  RUNS: a thread takes the pairs of 16 bytes of first dimensions
// with the 16 bytes of second ones (halves) or of 16 bytes (interleaved), or copies 16
// bytes; it has them in flight while the angles are worked out.  Otherwise (a rotated
// part that is no whole number of 16-byte runs) a pair or a value at a time.
template <typename T, bool RUNS>
__global__ void __launch_bounds__(APPEND_THREADS) rope_append_kernel(AppendArgs<T> a) {
  __shared__ float cs[MAX_HALF], sn[MAX_HALF];
  constexpr int E = RUN<T>;
  const int t = blockIdx.y * GRID_TOKENS + blockIdx.x, tid = threadIdx.x;
  if (t >= a.tokens) return;
  const int b = a.seqs.cu ? find_sequence(a.seqs.cu, a.seqs.seqs, t) : t;
  if (b >= a.seqs.seqs) return;  // behind the last sequence
  const int len = a.seqs.lens[b];
  if (len < 0) return;
  const int64_t slot = (int64_t)len + (a.seqs.cu ? t - a.seqs.cu[b] : 0);
  const int64_t pg = slot / a.kv.ps;
  const int page = pg < a.seqs.stride ? a.seqs.table[(int64_t)b * a.seqs.stride + pg] : -1;
  const bool stored = page >= 0 && page < a.kv.num_pages;
  const int half = a.rot >> 1, hd = a.kv.hd, kv = a.kv.kv_heads;
  // element (head 0, dimension 0) of this token's place in a cache, and a head's distance
  const int64_t at = ((int64_t)page * kv * a.kv.ps + slot % a.kv.ps) * hd, head_stride = (int64_t)a.kv.ps * hd;
  auto place = [&](int h) {  // query heads, key heads, value heads
    if (h < a.heads) return Place<T>{a.q + t * a.ldq + h * hd, a.q_out + t * a.ldqo + h * hd};
    h -= a.heads;
    if (h < kv) return Place<T>{a.k + t * a.ldk + h * hd, (T*)a.kv.k + at + h * head_stride};
    h -= kv;
    return Place<T>{a.v + t * a.ldv + h * hd, (T*)a.kv.v + at + h * head_stride};
  };
  // a head's items: the rotated ones, then the copied ones; value heads are copied
  const int step = RUNS ? E : 1;
  const int turned = a.interleaved && RUNS ? a.rot / E : half / step, per_head = turned + (hd - a.rot) / step;
  const int rotated = (a.heads + (stored ? kv : 0)) * per_head, all = rotated + (stored ? kv * (hd / step) : 0);
  struct Item {
    Place<T> p;
    int d, d2;  // the dimensions read; d2 < 0: copied
  };
  auto item = [&](int i) {
    Item x;
    if (i < rotated) {
      const int h = i / per_head, c = i - h * per_head;
      x.p = place(h);
      if (c < turned) {
        x.d = a.interleaved ? c * (RUNS ? E : 2) : c * step;
        x.d2 = a.interleaved ? x.d + (RUNS ? 0 : 1) : x.d + half;
      } else {
        x.d = a.rot + (c - turned) * step;
        x.d2 = -1;
      }
    } else {
      i -= rotated;
      const int h = i / (hd / step);
      x.p = place(a.heads + kv + h);
      x.d = (i - h * (hd / step)) * step;
      x.d2 = -1;
    }
    return x;
  };
  Item x;
  Run<T> u, w;
  auto load = [&](int i) {
    x = item(i);
    u.load(x.p.src + x.d);
    if (x.d2 > x.d) w.load(x.p.src + x.d2);
  };
  if constexpr (RUNS)
    if (tid < all) load(tid);
  if (tid < half) {
    constexpr double TURN = 0.15915494309189535, TURN_LOW = -9.839338337591243e-18;  // 1 / (2 pi)
    const double angle = (double)(slot + (a.offsets ? a.offsets[b] : 0)) * a.inv_freq[tid];
    const double part = fma(angle, TURN_LOW, fma(angle, TURN, -rint(angle * TURN)));
    float s, c;
    sincospif((float)(2. * part), &s, &c);
    cs[tid] = c * a.scale;
    sn[tid] = s * a.scale;
  }
  __syncthreads();
  for (int i = tid; i < all; i += APPEND_THREADS) {
    if constexpr (!RUNS) {
      x = item(i);
      if (x.d2 < 0) {
        x.p.dst[x.d] = x.p.src[x.d];
        continue;
      }
      const int j = a.interleaved ? x.d >> 1 : x.d;
      const float p = to_f32(x.p.src[x.d]), q = to_f32(x.p.src[x.d2]);
      x.p.dst[x.d] = from_f32<T>(p * cs[j] - q * sn[j]);
      x.p.dst[x.d2] = from_f32<T>(q * cs[j] + p * sn[j]);
    } else {
      if (i != tid) load(i);
      if (x.d2 > x.d) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float p = to_f32((T)u.v[e]), q = to_f32((T)w.v[e]), c = cs[x.d + e], s = sn[x.d + e];
          u.v[e] = from_f32<T>(p * c - q * s);
          w.v[e] = from_f32<T>(q * c + p * s);
        }
        w.store(x.p.dst + x.d2);
      } else if (x.d2 == x.d) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float p = to_f32((T)u.v[e]), q = to_f32((T)u.v[e + 1]), c = cs[(x.d + e) >> 1], s = sn[(x.d + e) >> 1];
          u.v[e] = from_f32<T>(p * c - q * s);
          u.v[e + 1] = from_f32<T>(q * c + p * s);
        }
      }
      u.store(x.p.dst + x.d);
    }
  }
}

template <typename T>
void launch_rope_append(const AppendArgs<T>& a, hipStream_t s) {
  if (a.tokens <= 0) return;
  if (a.rot % (a.interleaved ? RUN<T> : 2 * RUN<T>) == 0)
    rope_append_kernel<T, true><<<token_grid(a.tokens), APPEND_THREADS, 0, s>>>(a);
  else
    rope_append_kernel<T, false><<<token_grid(a.tokens), APPEND_THREADS, 0, s>>>(a);
}
template void launch_rope_append<float>(const AppendArgs<float>&, hipStream_t);
template void launch_rope_append<bf16>(const AppendArgs<bf16>&, hipStream_t);

}  // namespace axon
