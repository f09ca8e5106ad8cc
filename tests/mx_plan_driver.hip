// Host program of tests/test_mx_plans.py: for lines of "m k n ldw lds", the kernel of a product with one
// matrix (the rows of W to a tile of a stream, those of a square tile, 0 for the kernel without
// tiles), the parts of k, and whether the matrix's scales are copied.
#include <cstdio>

#include "wc_mx.hip"

int main() {
  uint32_t m, k, n;
  unsigned long long ldw, lds;
  while (std::scanf("%u %u %u %llu %llu", &m, &k, &n, &ldw, &lds) == 5) {
    const wc_mx_job job = {reinterpret_cast<void*>(4096), reinterpret_cast<void*>(4096), nullptr,
                           reinterpret_cast<void*>(4096), ldw, lds, n, n, 0, WC_BF16, 0};
    if (!jobs_ok(m, k, 1, &job)) return 1;
    const Plan p = plan_of(m, k, 1, &job);
    const char* const names[] = {"stream16", "stream32", "stream64", "slim", "tile64", "tile128", "tile128deep", "tile256"};
    std::printf("%s %u %d\n", names[int(p.kernel)], p.splits, int(p.copies(job.scale, lds, k)));
  }
}
