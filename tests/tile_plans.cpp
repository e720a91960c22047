// Prints what the matrix kernels' host code plans for given sizes: a line a case, "kind whole workgroups parts" a product.  The library's own sources are
// compiled in, for the host alone (nothing is launched, so the device's part of the program is empty).
#ifndef __HIP_DEVICE_COMPILE__
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#ifdef HEAD
#include "simple_head.hip"
#else
#include "simple_xent.hip"
#endif

using namespace simple::tiles;

static void print(int64_t rows, const Plan& r) { printf(" %d %d %d %d", (int)rows, r.whole, r.wgs, r.grid - r.wgs); }

int main(int argc, char** argv) {
  for (int i = 1; i + 2 < argc; i += 3) {
    const int64_t T = atoll(argv[i]), V = atoll(argv[i + 1]), D = atoll(argv[i + 2]);
#ifdef HEAD
    // D: whether rows are aligned, or copied to rows that are
    shaped<Int8>(tiles_for(T, V), [&](auto shape) {
      using S = decltype(shape);
      print(S::BP, D ? plan<S, many<S, true>>(T, V) : plan<S, many<S, false>>(T, V));
    });
#else
    if (D == 0) {
      shaped<Bf16>(tiles_for(T, V), [&](auto shape) { using S = decltype(shape); print(S::BP, plan<S, false>(T, V)); });
    } else {
      const int64_t rows = piece_rows(T, V), n = rows < V ? rows : V, k = ceil_div(n, 8) * 16, t16 = ceil_div(T, 16) * 32;
      const int splits = hidden_splits(T, V, D);
      printf("%lld %d", (long long)rows, splits);
      shaped<Bf16>(tiles_for(T, n) == TILE_256 ? TILE_256 : TILE_128, [&](auto shape) { using S = decltype(shape); print(S::BP, plan<S, false>(T, n)); });
      shaped<F16>(multiply_tiles(T, D, k, splits), [&](auto shape) { using S = decltype(shape); print(S::BP, plan<S, Cut<S>::CAN>(T, D, splits == 1)); });
      shaped<F16>(multiply_tiles(n, D, t16, 1), [&](auto shape) { using S = decltype(shape); print(S::BP, plan<S, Cut<S>::CAN>(n, D, true)); });
    }
#endif
    printf("\n");
  }
  return 0;
}
#endif
