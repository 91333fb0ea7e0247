// Prints the integer turns of each frequency (in hexadecimal floating point) on standard input. Built and run by
// tests/test_rotate_turns.py.
#include "../paper_2608_25332_gb300/csrc/turns.h"

#include <cstdio>

int main() {
  double f;
  while (std::scanf("%la", &f) == 1) std::printf("%llu\n", provip::turns_of(f));
  return 0;
}
