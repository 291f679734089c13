// Prints the route of a gated product for each line "M N K bits" on stdin, at 256
// compute units: decode, tile, wide, ksplit, tall or small, and the same for the
// product alone.
#include "gemm_rules.h"

#include <cstdio>

using namespace dptq;

int main() {
  static const char* const names[] = {"", "decode", "tile", "wide", "ksplit", "tall", "small"};
  long M, N;
  int K, bits;
  while (std::scanf("%ld %ld %d %d", &M, &N, &K, &bits) == 4)
    std::printf("%s %s\n", names[rules::gated_route(M, N, K, bits, 256).kernel],
                names[rules::gemm_route(M, N, K, bits, 256).kernel]);
  return 0;
}
