// Prints how a product is computed and the lanes of its largest launch, for every line "M N K" of the input.
#include <cstdio>

#include "mxfp4_choice.hpp"

int main()
{
    size_t M, N, K;
    while (std::scanf("%zu %zu %zu", &M, &N, &K) == 3) {
        const Product p = product_of(M, N, K);
        std::printf("%d %d %d %u %d %d %d %llu\n", p.ring_rows, p.ring_waves, (int)p.tile, p.splits, (int)p.rest_tile, p.rest_m != 0, p.rest_n != 0,
                    lanes_of(p, M, N));
    }
    return 0;
}
