// The rotation's turn per position, on the host: reads frequencies, one per line, and prints the two parts of each.
#include <cinttypes>
#include <cstdio>

#include "kb_rope.cuh"

int main() {
  double f;
  while (std::scanf("%la", &f) == 1) {
    std::printf("%" PRIu64 " %a\n", kb::rope_turn(f), (double)kb::rope_rest(f));
  }
  return 0;
}
