// Every kernel whose limit of dynamic LDS is raised has a bit of its own (test_lds_bits.py).
//
//   lds_bits RULE       "own": csrc/lds_bits.h; "shared": small_kernel and wide_kernel counted from the same bit
#include <stdio.h>
#include <string.h>
#include "lds_bits.h"

int main(int argc, char **argv)
{
    if (argc != 2) return 2;
    const bool shared = !strcmp(argv[1], "shared");
    if (!shared && strcmp(argv[1], "own")) return 2;
    unsigned long long all = 0;
    int twice = 0, kernels = 0;
    const auto take = [&](unsigned long long bit) {
        if (!bit || (bit & (bit - 1)) || (all & bit)) ++twice;
        all |= bit;
        ++kernels;
    };
    for (int h = 0; h < 2; ++h) {
        const int H = h ? 128 : 64;
        for (int k = 0; k < 8; ++k) take(lds_bit_pair(H, k & 4, k & 2, k & 1));
        for (int grad = 0; grad < 2; ++grad) {
            take(shared ? lds_bit_small(1 << (2 * h + grad)) : lds_bit_wide(H, grad));
            for (int extra = 0; extra < 2; ++extra)
                for (int tiles = 1; tiles <= 4; ++tiles) take(lds_bit_fit(H, tiles, grad, extra));
        }
    }
    for (int columns = 1; columns <= 8; columns *= 2) take(lds_bit_small(columns));
    printf("%d kernels, %d bits taken twice\n", kernels, twice);
    return twice ? 1 : 0;
}
