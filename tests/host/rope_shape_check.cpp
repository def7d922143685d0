// Host-side check of the rotation's launch (csrc/hexi_rope.h).  A line "rows pieces" a launch; prints "tokens grid".
#include <cstdio>
#include "hexi_rope.h"

int main()
{
    long long rows, pieces;
    while (std::scanf("%lld %lld", &rows, &pieces) == 2) {
        const RopeShape s = hexi_rope_shape((int)rows, (unsigned)pieces);
        std::printf("%d %u\n", s.tokens, s.grid);
    }
    return 0;
}
