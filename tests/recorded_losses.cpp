// The recording HIP stand-in with scenarios of the row operators and of the training
// step's losses: besides what it writes down itself, a "parts" line for every buffer
// that these kernels keep partial results in.
// Usage: recorded_losses <operators | steps>.
#include <hip/hip_runtime.h>

#define hipLaunchKernel plain_launch
#define main plain_main
#include "recorded_hip.cpp"
#undef hipLaunchKernel
#undef main

namespace {

void row_partials(const std::string& k, dim3 grid, void** args) {
  auto is = [&](const char* part) { return k.find(part) != std::string::npos; };
  auto n = [&](int i) { return (int64_t) * (const int*)args[i]; };
  auto say = [&](int i, int64_t words) {
    const void* p = *(void**)args[i];
    if (p) printf("parts %llu %lld\n", (unsigned long long)p, (long long)words * 4);
  };
  if (is("ln_bwd_kernel")) say(8, grid.x * (is("Lb1EEEvPKT_") ? 3 : 2) * n(10));
  else if (is("gelu_bwd_kernel")) say(7, grid.y * n(5));
  else if (is("logit_part_kernel")) say(7, *(const int64_t*)args[4] * 2), say(9, *(const int64_t*)args[4] * 2), say(10, *(const int64_t*)args[4] / n(5));
  else if (is("logit_grad_kernel")) say(6, *(const int64_t*)args[4] / n(5) * 2), say(7, *(const int64_t*)args[4] / n(5));
  else if (is("piece_merge_kernel")) say(4, (int64_t)grid.x * 2), say(7, (int64_t)grid.x * 2);
  else if (is("policy_weights_kernel")) say(5, (*(void**)args[3] ? n(4) : 1) * 2);
  else if (is("preference_finish_kernel"))
    say(5, n(4) * n(6) * 2), say(13, n(4) * 2), say(14, n(8) * 2), say(15, n(4) * 2), say(16, n(4));
  else if (is("preference_few_kernel")) say(5, n(4) * n(6) * 2), say(7, n(4)), say(8, n(4) * 2);
  else if (is("policy_finish_kernel"))
    say(5, n(4) * n(6) * 2), say(18, (*(void**)args[7] ? n(8) : 1) * 2), say(19, n(4) * 2), say(20, n(4));
  else if (is("policy_sum_kernel")) say(1, n(0) * 2), say(2, n(0)), say(3, n(0) * 2);
}

float* const F = (float*)(uintptr_t)0x40000;

// every operator over many sizes, in a workspace of exactly the bytes it asks for
void operators() {
  for (int64_t rows : {1, 2, 3, 5, 63, 64, 257, 1000, 1025, 4097, 70001})
    for (int cols : {1, 7, 64, 509, 512, 513, 1024, 1025, 1600, 2048, 2049, 4096, 4104, 8192, 8193, 16384}) {
      mark("layer norm " + std::to_string(rows) + " x " + std::to_string(cols));
      const int64_t bytes = axon_layernorm_backward_workspace(rows, cols);
      void* ws = reserve(bytes);
      for (int t : {AXON_F32, AXON_BF16}) {
        check(axon_layernorm(rows, cols, F, t, cols, F, F, t, 1e-5f, F, t, cols, nullptr), "axon_layernorm");
        check(axon_layernorm_backward(rows, cols, F, t, cols, F, t, cols, F, t, 1e-5f, F, cols, F, F, ws, bytes, nullptr),
              "axon_layernorm_backward");
      }
    }
  for (int64_t tokens : {1, 2, 15, 16, 63, 300, 1024, 4097, 70001})
    for (int vocab : {1, 8, 2048, 2049, 8193, 32000, 50257, 128256, 300001})
      for (int seqs : {2, 4, 200}) {
        mark("losses " + std::to_string(tokens) + " x " + std::to_string(vocab) + ", " + std::to_string(seqs));
        std::vector<int32_t> cu;
        for (int i = 0; i <= seqs; ++i) cu.push_back((int32_t)(tokens * i / seqs));
        const int64_t bytes = axon_token_loss_workspace(tokens, vocab, seqs), few = axon_token_loss_workspace(tokens, vocab, 0);
        for (int t : {AXON_F32, AXON_BF16})
          for (void* dz : {(void*)nullptr, (void*)F}) {
            check(axon_token_logprobs(tokens, vocab, F, t, vocab, TOK, F, reserve(few), few, nullptr), "axon_token_logprobs");
            void* ws = reserve(bytes);
            check(axon_preference_loss(tokens, vocab, F, t, vocab, TOK, seqs / 2, TOK, cu.data(), F, 0.1f, 0.f, F, F, F,
                                       dz, t, vocab, ws, bytes, nullptr), "axon_preference_loss");
            for (int per : {0, 1})
              check(axon_policy_loss(tokens, vocab, F, t, vocab, TOK, seqs, TOK, cu.data(), F, F, F, 0.2f, 0.2f, 0.1f,
                                     per, F, F, F, dz, t, vocab, ws, bytes, nullptr), "axon_policy_loss");
          }
      }
}

// training steps with each loss, both families, each twice
void steps() {
  for (int gpt2 : {0, 1})
    for (int len : {1, 60, 700}) {
      axon_config c = llama(1024, 16, 16, 64, 1600, 1003);
      if (gpt2) {
        c.arch = AXON_ARCH_GPT2;
        c.rope_theta = 0;
        c.qkv_bias = 1;
        c.max_positions = 700;
      }
      c.max_batch = 4;
      c.max_seq = 700;
      mark("model");
      axon_model* m = make(c);
      Map g(c, AXON_F32);
      std::vector<int32_t> cu;
      for (int b = 0; b <= 4; ++b) cu.push_back(b * len);
      const int n = (int)g.w.size();
      for (int again = 0; again < 2; ++again) {
        mark(again ? "second" : "first");
        check(axon_preference_loss_and_grads(m, 2, TOK, TOK, cu.data(), TOK, F, 0.1f, 0.f, F, F, F, g.w.data(), n, nullptr),
              "axon_preference_loss_and_grads");
        for (int per : {0, 1})
          check(axon_policy_loss_and_grads(m, 4, TOK, TOK, cu.data(), TOK, F, F, F, 0.2f, 0.2f, 0.1f, per, F, F, F,
                                           g.w.data(), n, nullptr), "axon_policy_loss_and_grads");
        check(axon_loss_and_grads(m, 4, TOK, TOK, cu.data(), TOK, F, g.w.data(), n, nullptr), "axon_loss_and_grads");
      }
    }
}

}  // namespace

extern "C" hipError_t hipLaunchKernel(const void* f, dim3 g, dim3 b, void** args, size_t lds, hipStream_t s) {
  row_partials(name_of(f), g, args);
  return plain_launch(f, g, b, args, lds, s);
}

int main(int, char** argv) {
  setvbuf(stdout, nullptr, _IOFBF, 1 << 20);
  const std::string s = argv[1] ? argv[1] : "";
  if (s == "operators") operators();
  else if (s == "steps") steps();
  else return 2;
  printf("done\n");
  return 0;
}
