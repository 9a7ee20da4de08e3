// Attention of new tokens over a shared prefix and their own keys in a paged cache:
//   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q k_j - max),
// j over the group's prefix and the sequence's own keys up to the token itself.
//
// A wavefront per (token, query head): a lane scores one key of 64, the running maximum
// and sum are float32, lane d accumulates dimensions d and d + 64.
#include "common.h"
#include "kernels.h"

namespace axon {

constexpr float LOG2E_F = 1.4426950408889634f;

template <typename T, int HD>
__global__ void __launch_bounds__(64) prefix_attn_kernel(PrefixAttnArgs<T> a) {
  constexpr int DL = HD / 64;
  __shared__ float qs[HD];
  const int t = blockIdx.x, head = blockIdx.y, lane = threadIdx.x;
  const int kvh = head / (a.heads / a.kv.kv_heads);
  T* out = a.out + t * a.ldo + head * HD;
  int b = t;
  if (a.seqs.cu) {
    b = 0;
    while (b < a.seqs.seqs && a.seqs.cu[b + 1] <= t) ++b;
  }
  if (b >= a.seqs.seqs) return;
  const int len = a.seqs.lens[b];
  float m = -INFINITY, l = 0.f, acc[DL] = {};
  if (len >= 0) {
    for (int d = lane; d < HD; d += 64) qs[d] = to_f32(a.q[t * a.ldq + head * HD + d]);
    __syncthreads();
    int g = 0;
    while (g < a.shared.groups && !(a.shared.cu[g] <= b && b < a.shared.cu[g + 1])) ++g;
    for (int part = 0; part < 2; ++part) {
      if (part == 0 && g >= a.shared.groups) continue;
      const int32_t* table = part ? a.seqs.table + (int64_t)b * a.seqs.stride : a.shared.table + (int64_t)g * a.shared.stride;
      const int64_t room = (int64_t)(part ? a.seqs.stride : a.shared.stride) * a.kv.ps;
      int64_t n = part ? (int64_t)len + (a.seqs.cu ? t - a.seqs.cu[b] : 0) + 1 : a.shared.lens[g];
      if (n > room) n = room;
      for (int64_t j0 = 0; j0 < n; j0 += 64) {
        const int64_t j = j0 + lane;
        int64_t row = -1;
        if (j < n) {
          const int page = table[j / a.kv.ps];
          if (page >= 0 && page < a.kv.num_pages)
            row = (((int64_t)page * a.kv.kv_heads + kvh) * a.kv.ps + j % a.kv.ps) * HD;
        }
        float s = -INFINITY;
        if (row >= 0) {
          const T* k = (const T*)a.kv.k + row;
          s = 0.f;
          for (int d = 0; d < HD; ++d) s += qs[d] * to_f32(k[d]);
          s *= a.scale * LOG2E_F;
        }
        const float top = fmaxf(m, wave_max(s));
        const float base = top == -INFINITY ? 0.f : top;
        const float fall = exp2f(m - base), p = row >= 0 ? exp2f(s - base) : 0.f;
        m = top;
        l = l * fall + wave_sum(p);
        for (int d = 0; d < DL; ++d) acc[d] *= fall;
        for (int i = 0; i < 64; ++i) {
          const int64_t r = __shfl(row, i);
          if (r < 0) continue;
          const float pi = __shfl(p, i);
          for (int d = 0; d < DL; ++d) acc[d] += pi * to_f32(((const T*)a.kv.v)[r + d * 64 + lane]);
        }
      }
    }
  }
  for (int d = 0; d < DL; ++d) out[d * 64 + lane] = from_f32<T>(m == -INFINITY ? 0.f : acc[d] / l);
  if (a.lse && lane == 0) a.lse[(int64_t)t * a.heads + head] = m == -INFINITY ? -INFINITY : (m + log2f(l)) / LOG2E_F;
}

template <typename T>
void launch_prefix_attn(const PrefixAttnArgs<T>& a, hipStream_t s) {
  if (!a.tokens) return;
  const dim3 grid(a.tokens, a.heads);
  if (a.kv.hd == 64) prefix_attn_kernel<T, 64><<<grid, 64, 0, s>>>(a);
  else prefix_attn_kernel<T, 128><<<grid, 64, 0, s>>>(a);
}
template void launch_prefix_attn<float>(const PrefixAttnArgs<float>&, hipStream_t);
template void launch_prefix_attn<bf16>(const PrefixAttnArgs<bf16>&, hipStream_t);

}  // namespace axon
