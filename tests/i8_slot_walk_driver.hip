// Host program of tests/test_i8_slot_walk.py: the walk of wc_experts_i8's slot-by-slot down
// product over the blocks of a token's slots, for every pattern of empty slots.
#include <cstdio>

#include "wc_i8_ring.h"

int main() {
  uint64_t wrong = 0, walks = 0;
  for (uint32_t waves : {1u, 3u, 8u})
    for (uint32_t blocks = 1; blocks <= 17; blocks++)
      for (uint32_t slots = 1; slots <= 9; slots++)
        for (uint32_t used = 0; used < 1u << slots; used++) {
          uint32_t taken[9][17] = {};
          for (uint32_t wave = 0; wave < waves; wave++) {
            wc_i8::SlotBlock at = {used, wave};
            uint32_t steps = 0;
            for (wc_i8::settle_block(at, blocks); at.left && steps < 9 * 17; steps++) {
              wrong += at.block >= blocks;
              taken[at.slot()][at.block % 17]++;
              at.block += waves;
              wc_i8::settle_block(at, blocks);
            }
          }
          for (uint32_t s = 0; s < slots; s++)
            for (uint32_t b = 0; b < blocks; b++) wrong += taken[s][b] != (used >> s & 1);
          walks++;
        }
  std::printf("%llu walks, %llu wrong\n", (unsigned long long)walks, (unsigned long long)wrong);
  return wrong != 0;
}
