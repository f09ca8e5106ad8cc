// Host program of tests/test_mx_plans.py: for lines of "tokens k experts hidden ffn", the places to a
// block of wc_experts_mx's kernels, 0 where it runs the two kernels of few tokens.
#include <cstdio>

#include "wc_mx_experts.hip"

int main() {
  uint32_t tokens, k, n, hidden, ffn;
  while (std::scanf("%u %u %u %u %u", &tokens, &k, &n, &hidden, &ffn) == 5) {
    if (!sizes_ok(tokens, k, n, hidden, ffn)) return 1;
    const wc_mx_experts none{};
    const ExpertArgs a = args_of(nullptr, WC_BF16, tokens, hidden, k, n, hidden, ffn, &none, &none, &none, nullptr,
                                 hidden, layout(tokens, k, n, hidden, ffn), 0);
    std::printf("%u\n", is_few(tokens, k, hidden) ? 0 : places(a));
  }
}
