// New tokens into a paged cache: queries and keys rotated by their position, keys and
// values stored in their pages.
//
// The pair (a, b) of dimension j of a head at position t turns by the angle
// t inv_freq[j]:  (a cos - b sin, b cos + a sin), times ``scale``; the pairs are
// dimensions (j, rot/2 + j) or (2j, 2j + 1) of the first ``rot`` ones.  The angle is a
// float64 product: at position 10^6 a float32 one is off by 0.03 of a radian.  It is
// reduced to (-1/2, 1/2] of a turn in float64 as well; cosine and sine are float32 from
// there, and a value is rounded once, when it is stored.
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

template <typename T>
__global__ void __launch_bounds__(APPEND_THREADS) rope_append_kernel(AppendArgs<T> a) {
  __shared__ float cs[MAX_HALF], sn[MAX_HALF];
  const int t = blockIdx.x;
  const int b = a.seqs.cu ? find_sequence(a.seqs.cu, a.seqs.seqs, t) : t;
  if (b >= a.seqs.seqs) return;  // behind the last sequence
  const int len = a.seqs.lens[b];
  if (len < 0) return;
  const int64_t slot = (int64_t)len + (a.seqs.cu ? t - a.seqs.cu[b] : 0);
  const int half = a.rot >> 1, hd = a.kv.hd;
  if ((int)threadIdx.x < half) {
    const double turns = (double)(slot + (a.offsets ? a.offsets[b] : 0)) * a.inv_freq[threadIdx.x] * 0.15915494309189535;
    float s, c;
    sincospif((float)(2. * (turns - rint(turns))), &s, &c);
    cs[threadIdx.x] = c * a.scale;
    sn[threadIdx.x] = s * a.scale;
  }
  __syncthreads();
  const int64_t pg = slot / a.kv.ps;
  const int page = pg < a.seqs.stride ? a.seqs.table[(int64_t)b * a.seqs.stride + pg] : -1;
  const bool stored = page >= 0 && page < a.kv.num_pages;
  // element (head h, dimension 0) of this token's place in a cache
  const int64_t at = ((int64_t)page * a.kv.kv_heads * a.kv.ps + slot % a.kv.ps) * hd;
  const int64_t head_stride = (int64_t)a.kv.ps * hd;
  for (int i = threadIdx.x; i < (a.heads + a.kv.kv_heads) * hd; i += APPEND_THREADS) {
    const int h = i / hd, d = i % hd;
    const bool is_q = h < a.heads;
    if (!is_q && !stored) continue;
    const T* src = is_q ? a.q + t * a.ldq + h * hd : a.k + t * a.ldk + (h - a.heads) * hd;
    T* dst = is_q ? a.q_out + t * a.ldqo + h * hd : (T*)a.kv.k + at + (h - a.heads) * head_stride;
    if (d >= a.rot) {
      dst[d] = src[d];
      continue;
    }
    if (a.interleaved ? d & 1 : d >= half) continue;  // its pair's first dimension does both
    const int j = a.interleaved ? d >> 1 : d, d2 = a.interleaved ? d + 1 : d + half;
    const float x = to_f32(src[d]), y = to_f32(src[d2]);
    dst[d] = from_f32<T>(x * cs[j] - y * sn[j]);
    dst[d2] = from_f32<T>(y * cs[j] + x * sn[j]);
  }
  if (!stored) return;
  for (int i = threadIdx.x; i < a.kv.kv_heads * hd; i += APPEND_THREADS)
    ((T*)a.kv.v)[at + i / hd * head_stride + i % hd] = a.v[t * a.ldv + i];
}

template <typename T>
void launch_rope_append(const AppendArgs<T>& a, hipStream_t s) {
  if (a.tokens > 0) rope_append_kernel<T><<<a.tokens, APPEND_THREADS, 0, s>>>(a);
}
template void launch_rope_append<float>(const AppendArgs<float>&, hipStream_t);
template void launch_rope_append<bf16>(const AppendArgs<bf16>&, hipStream_t);

}  // namespace axon
