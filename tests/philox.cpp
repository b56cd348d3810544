// Blocks of philox.h against the answers published with the generator, and limits of dropouts against rint.
#include "philox.h"
#include <math.h>
#include <stdio.h>

int main()
{
    const struct { uint32_t c[4], k[2], w[4]; } known[] = {
        {{0, 0, 0, 0}, {0, 0}, {0x6627e8d5u, 0xe169c58du, 0xbc57ac4cu, 0x9b00dbd8u}},
        {{0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu}, {0xffffffffu, 0xffffffffu}, {0x408f276du, 0x41c83b0eu, 0xa20bc7c6u, 0x6d5451fdu}},
        {{0x243f6a88u, 0x85a308d3u, 0x13198a2eu, 0x03707344u}, {0xa4093822u, 0x299f31d0u}, {0xd16cfe09u, 0x94fdccebu, 0x5001e420u, 0x24126ea1u}},
    };
    for (const auto &t : known) {
        const Words4 r = philox(t.c[0], t.c[1], t.c[2], t.c[3], t.k[0], t.k[1]);
        for (int i = 0; i < 4; ++i)
            if (r.w[i] != t.w[i]) { printf("word %d is %08x, not %08x\n", i, r.w[i], t.w[i]); return 1; }
    }
    for (int t = 0; t <= 4 * 65536; ++t) {
        const double p = t / (4.0 * 65536.0);
        if ((double)drop_limit(p) != rint(p * 65536.0)) { printf("limit of %g\n", p); return 1; }
    }
    const DropRule d{1, 2, 3, 4, 0x8000u, 2.0f};
    const Words4 bits{{0x80007fffu, 0x7fff8000u, 0u, 0xffffffffu}};
    const bool keep[8] = {false, true, true, false, false, false, true, true};
    for (int i = 0; i < 8; ++i)
        if (drop_keeps(d, bits, i) != keep[i]) { printf("element %d\n", i); return 1; }
    const Words4 a = drop_bits(d, (7ull << 32) | 5u, 6), b = philox(5u, 7u | 6u << 16, 3, 4, 1, 2);
    for (int i = 0; i < 4; ++i)
        if (a.w[i] != b.w[i]) { printf("counter\n"); return 1; }
    printf("ok\n");
    return 0;
}
