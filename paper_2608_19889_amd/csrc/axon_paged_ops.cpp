// C ABI of the operators that sample answers: rotating and appending to a caller's paged
// cache, attention over it with a shared prefix, and drawing tokens from logits.
// Argument checks only; the kernels are in k_append.hip, k_prefix.hip and k_sample.hip.
#include <hip/hip_runtime.h>

#include <cmath>

#include "kernels.h"
#include "op_checks.h"

using namespace axon;

namespace {

int check_pages(const axon_kv_pages* c) {
  if (!c) return fail(AXON_E_INVALID, "pages is NULL");
  if (int r = check_type("the cache", c->dtype)) return r;
  if (c->kv_heads < 1 || c->kv_heads > 1024)
    return fail(AXON_E_INVALID, "kv_heads must be in [1, 1024], got " + num(c->kv_heads));
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(AXON_E_INVALID, "head_dim must be 64 or 128, got " + num(c->head_dim));
  if (c->page_size < 16 || c->page_size % 16)
    return fail(AXON_E_INVALID, "page_size must be a multiple of 16, got " + num(c->page_size));
  if (c->num_pages < 1) return fail(AXON_E_INVALID, "num_pages must be >= 1, got " + num(c->num_pages));
  if (int r = check_array("the key cache", c->k, 16)) return r;
  return check_array("the value cache", c->v, 16);
}

int check_table(const char* name, const int32_t* table, int32_t stride, int32_t page_size) {
  if (stride < 1 || (int64_t)stride * page_size > MAX_TOKENS)
    return fail(AXON_E_CAPACITY, std::string("rows of ") + name + " must hold 1 to 2^30 keys, got " + num(stride) +
                                     " pages of " + num(page_size));
  return check_array(name, table, 4);
}

// prefix sums on both sides, from 0, never falling; the last one is at most ``most``
int check_sums(const char* name, const int32_t* d, const int32_t* h, int32_t n, int64_t most) {
  if (int r = check_array((std::string("d_") + name).c_str(), d, 4)) return r;
  if (int r = check_array((std::string("h_") + name).c_str(), h, 4)) return r;
  if (h[0] != 0) return fail(AXON_E_INVALID, std::string(name) + "[0] must be 0");
  for (int i = 0; i < n; ++i)
    if (h[i + 1] < h[i]) return fail(AXON_E_INVALID, std::string(name) + " falls at entry " + num(i + 1));
  if (h[n] > most) return fail(AXON_E_INVALID, std::string(name) + " end at " + num(h[n]) + ", past " + num(most));
  return AXON_OK;
}

int check_batch(const axon_kv_batch* b, int64_t tokens, int32_t page_size) {
  if (!b) return fail(AXON_E_INVALID, "batch is NULL");
  if (tokens < 0 || tokens > MAX_TOKENS) return fail(AXON_E_INVALID, "tokens must be in [0, 2^30], got " + num(tokens));
  if (b->seqs < 1 || b->seqs > KV_MAX_SEQS)
    return fail(AXON_E_INVALID, "seqs must be in [1, " + num(KV_MAX_SEQS) + "], got " + num(b->seqs));
  if (b->d_cu_seqlens || b->h_cu_seqlens) {
    if (int r = check_sums("cu_seqlens", b->d_cu_seqlens, b->h_cu_seqlens, b->seqs, tokens)) return r;
  } else if (tokens != b->seqs) {
    return fail(AXON_E_INVALID, num(tokens) + " tokens for " + num(b->seqs) + " sequences need cu_seqlens");
  }
  if (int r = check_array("d_lens", b->d_lens, 4)) return r;
  return check_table("d_block_table", b->d_block_table, b->table_stride, page_size);
}

int check_prefix(const axon_kv_prefix* p, int32_t seqs, int32_t page_size) {
  if (!p || p->groups == 0) return AXON_OK;
  if (p->groups < 0 || p->groups > KV_MAX_SEQS)
    return fail(AXON_E_INVALID, "groups must be in [0, " + num(KV_MAX_SEQS) + "], got " + num(p->groups));
  if (int r = check_sums("cu_groups", p->d_cu_groups, p->h_cu_groups, p->groups, seqs)) return r;
  if (int r = check_array("d_prefix_lens", p->d_prefix_lens, 4)) return r;
  return check_table("d_prefix_table", p->d_prefix_table, p->table_stride, page_size);
}

int check_heads(int32_t heads, int32_t kv_heads) {
  if (heads < 1 || heads > 4096 || heads % kv_heads)
    return fail(AXON_E_INVALID, "heads must be a multiple of kv_heads up to 4096, got " + num(heads) + " over " +
                                    num(kv_heads));
  return AXON_OK;
}

PagedKV pages_of(const axon_kv_pages& c) {
  return PagedKV{c.k, c.v, c.kv_heads, c.head_dim, c.page_size, c.num_pages};
}
PagedSeqs seqs_of(const axon_kv_batch& b) {
  return PagedSeqs{b.seqs, b.d_cu_seqlens, b.d_lens, b.d_block_table, b.table_stride};
}

PrefixAttnShape shape_of(const axon_kv_pages& pages, const axon_kv_batch& batch, const axon_kv_prefix* prefix,
                         int64_t tokens, int32_t heads) {
  const int groups = prefix ? prefix->groups : 0;
  return PrefixAttnShape{tokens, batch.seqs, groups, heads, pages.kv_heads, pages.head_dim, batch.h_cu_seqlens,
                         groups ? prefix->h_cu_groups : nullptr};
}

int check_attention(const axon_kv_pages* pages, const axon_kv_batch* batch, const axon_kv_prefix* prefix,
                    int64_t tokens, int32_t heads) {
  if (int r = check_pages(pages)) return r;
  if (int r = check_batch(batch, tokens, pages->page_size)) return r;
  if (int r = check_prefix(prefix, batch->seqs, pages->page_size)) return r;
  if (int r = check_heads(heads, pages->kv_heads)) return r;
  const PrefixAttnShape shape = shape_of(*pages, *batch, prefix, tokens, heads);
  const int64_t ps = pages->page_size, own = batch->table_stride, shared = shape.groups ? prefix->table_stride : 0;
  if (!prefix_attn_fits(shape, own * ps, shared * ps))
    return fail(AXON_E_CAPACITY, num(tokens) + " tokens of " + num(heads) + " heads over tables of " + num(own) + " and " +
                                     num(shared) + " pages are too many for one call");
  return AXON_OK;
}

}  // namespace

extern "C" int axon_rope_append(const axon_kv_pages* pages, const axon_kv_batch* batch, int64_t tokens, int32_t heads,
                                const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                void* q_out, int64_t ldqo, const double* d_inv_freq, int32_t rot, int32_t interleaved,
                                float scale, const int32_t* d_offsets, void* stream) {
  return entry([&]() -> int {
    if (int r = check_pages(pages)) return r;
    if (int r = check_batch(batch, tokens, pages->page_size)) return r;
    const int32_t dtype = pages->dtype, hd = pages->head_dim;
    if (heads != 0) {
      if (int r = check_heads(heads, pages->kv_heads)) return r;
      if (int r = check_rows("q", q, dtype, ldq, tokens, (int64_t)heads * hd)) return r;
      if (int r = check_rows("q_out", q_out, dtype, ldqo, tokens, (int64_t)heads * hd)) return r;
      if (q == q_out && ldq != ldqo) return fail(AXON_E_INVALID, "q_out in q's buffer needs its row stride");
    }
    if (int r = check_rows("k", k, dtype, ldk, tokens, (int64_t)pages->kv_heads * hd)) return r;
    if (int r = check_rows("v", v, dtype, ldv, tokens, (int64_t)pages->kv_heads * hd)) return r;
    if (rot < 0 || rot > hd || rot % 2)
      return fail(AXON_E_INVALID, "rot must be even and in [0, " + num(hd) + "], got " + num(rot));
    if (rot > 0)
      if (int r = check_array("d_inv_freq", d_inv_freq, 8)) return r;
    if (interleaved != 0 && interleaved != 1) return fail(AXON_E_INVALID, "interleaved must be 0 or 1");
    if (!std::isfinite(scale)) return fail(AXON_E_INVALID, "scale must be finite");
    if (d_offsets)
      if (int r = check_array("d_offsets", d_offsets, 4)) return r;
    auto launch = [&](auto* t) {
      using T = std::remove_pointer_t<decltype(t)>;
      launch_rope_append(AppendArgs<T>{pages_of(*pages), seqs_of(*batch), (int)tokens, heads, (const T*)q, (const T*)k,
                                       (const T*)v, (T*)q_out, ldq, ldk, ldv, ldqo, d_inv_freq, rot, interleaved == 1,
                                       scale, d_offsets},
                         (hipStream_t)stream);
    };
    if (dtype == AXON_BF16) launch((bf16*)nullptr);
    else launch((float*)nullptr);
    return check_launch("rope append");
  });
}

extern "C" int64_t axon_prefix_attention_workspace(const axon_kv_pages* pages, const axon_kv_batch* batch,
                                                   const axon_kv_prefix* prefix, int64_t tokens, int32_t heads) {
  int64_t bytes = 0;
  entry([&]() -> int {
    if (!check_attention(pages, batch, prefix, tokens, heads))
      bytes = prefix_attn_workspace(shape_of(*pages, *batch, prefix, tokens, heads));
    return AXON_OK;
  });
  return bytes;
}

extern "C" int axon_prefix_attention(const axon_kv_pages* pages, const axon_kv_batch* batch,
                                     const axon_kv_prefix* prefix, int64_t tokens, int32_t heads, const void* q,
                                     int64_t ldq, float scale, void* out, int64_t ldo, float* d_lse, void* workspace,
                                     int64_t workspace_bytes, void* stream) {
  return entry([&]() -> int {
    if (int r = check_attention(pages, batch, prefix, tokens, heads)) return r;
    const int64_t cols = (int64_t)heads * pages->head_dim;
    if (int r = check_rows("q", q, pages->dtype, ldq, tokens, cols)) return r;
    if (int r = check_rows("out", out, pages->dtype, ldo, tokens, cols)) return r;
    if (q == out && ldq != ldo) return fail(AXON_E_INVALID, "out in q's buffer needs its row stride");
    if (!std::isfinite(scale)) return fail(AXON_E_INVALID, "scale must be finite");
    if (d_lse)
      if (int r = check_array("d_lse", d_lse, 4)) return r;
    const PrefixAttnShape shape = shape_of(*pages, *batch, prefix, tokens, heads);
    if (int r = check_workspace(workspace, workspace_bytes, prefix_attn_workspace(shape))) return r;
    const SharedPrefix shared = prefix ? SharedPrefix{prefix->groups, prefix->d_cu_groups, prefix->d_prefix_lens,
                                                      prefix->d_prefix_table, prefix->table_stride}
                                       : SharedPrefix{};
    auto launch = [&](auto* t) {
      using T = std::remove_pointer_t<decltype(t)>;
      launch_prefix_attn(PrefixAttnArgs<T>{pages_of(*pages), seqs_of(*batch), shared, (int)tokens, heads, (const T*)q,
                                           (T*)out, ldq, ldo, scale, d_lse},
                         shape, workspace, (hipStream_t)stream);
    };
    if (pages->dtype == AXON_BF16) launch((bf16*)nullptr);
    else launch((float*)nullptr);
    return check_launch("prefix attention");
  });
}

extern "C" int64_t axon_sample_tokens_workspace(int64_t rows, int32_t vocab) {
  if (rows < 0 || rows > SAMPLE_MAX_ROWS || vocab < 1 || vocab > SAMPLE_MAX_VOCAB) return 0;
  return sample_workspace(rows, vocab);
}

extern "C" int axon_sample_tokens(int64_t rows, int32_t vocab, const void* logits, int32_t dtype, int64_t ld,
                                  const float* d_uniform, const float* d_temperature, float temperature,
                                  const int32_t* d_top_k, int32_t top_k, const float* d_top_p, float top_p,
                                  const float* d_min_p, float min_p, int32_t* d_tokens, float* d_logps, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
  return entry([&]() -> int {
    if (rows < 0 || rows > SAMPLE_MAX_ROWS)
      return fail(AXON_E_INVALID, "rows must be in [0, " + num(SAMPLE_MAX_ROWS) + "], got " + num(rows));
    if (vocab < 1 || vocab > SAMPLE_MAX_VOCAB)
      return fail(AXON_E_INVALID, "vocab must be in [1, " + num(SAMPLE_MAX_VOCAB) + "], got " + num(vocab));
    if (int r = check_rows("logits", logits, dtype, ld, rows, vocab)) return r;
    if (d_temperature) {
      if (int r = check_array("d_temperature", d_temperature, 4)) return r;
    } else if (!(temperature >= 0.f)) {
      return fail(AXON_E_INVALID, "temperature must be >= 0");
    }
    if (d_top_k) {
      if (int r = check_array("d_top_k", d_top_k, 4)) return r;
    } else if (top_k < 0) {
      return fail(AXON_E_INVALID, "top_k must be >= 0, got " + num(top_k));
    }
    if (d_top_p) {
      if (int r = check_array("d_top_p", d_top_p, 4)) return r;
    } else if (!(top_p > 0.f && top_p <= 1.f)) {
      return fail(AXON_E_INVALID, "top_p must be in (0, 1]");
    }
    if (d_min_p) {
      if (int r = check_array("d_min_p", d_min_p, 4)) return r;
    } else if (!(min_p >= 0.f && min_p <= 1.f)) {
      return fail(AXON_E_INVALID, "min_p must be in [0, 1]");
    }
    if (rows == 0) return AXON_OK;
    if (int r = check_array("d_uniform", d_uniform, 4)) return r;
    if (int r = check_array("d_tokens", d_tokens, 4)) return r;
    if (int r = check_array("d_logps", d_logps, 4)) return r;
    if (int r = check_workspace(workspace, workspace_bytes, axon_sample_tokens_workspace(rows, vocab))) return r;
    launch_sample(SampleArgs{logits, dtype == AXON_BF16, ld, (int)rows, vocab, d_uniform, d_temperature, d_top_k,
                             d_top_p, d_min_p, temperature, top_p, min_p, top_k, d_tokens, d_logps},
                  workspace, (hipStream_t)stream);
    return check_launch("sampling");
  });
}
