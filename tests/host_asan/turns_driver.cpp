// The turns of frequencies (turns.h): reads frequencies as hexadecimal floats, one a line, and
// prints theta / 2 pi mod 1 in units of 2^-64.
#include <cinttypes>
#include <cstdio>

#include "turns.h"

int main() {
  long double theta;
  while (std::scanf("%La", &theta) == 1) std::printf("%" PRIu64 "\n", libra::rotary_turns(theta));
  return 0;
}
