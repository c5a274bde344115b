// Prints what int8_route, int8_streams and int8_quantises_itself (csrc/int8_route.cpp, no HIP) decide.
//
// stdin:   T N K cus                                      (one line per call)
// stdout:  streams quantises_itself blocks tile           (the last two: of int8_route, also where the call streams)
#include <stdio.h>

#include "int8_route.h"

int main() {
  int T, N, K, cus;
  while (scanf("%d %d %d %d", &T, &N, &K, &cus) == 4) {
    const mm::Int8Route r = mm::int8_route(T, N, K, cus);
    printf("%d %d %d %d\n", (int)mm::int8_streams(T, K), (int)mm::int8_quantises_itself(T, K), r.blocks, (int)r.tile);
  }
}
