// Reads lines "R Mo No ctas", prints the split that the weight gradient takes and every worker's parts.
#include <stdio.h>

#include "act8_split.cuh"

int main()
{
    int R, Mo, No, ctas;
    while (scanf("%d %d %d %d", &R, &Mo, &No, &ctas) == 4) {
        const im::Split s = im::split_for(R, Mo, No, ctas);
        printf("split %d %d %d %d %d %d %d %d\n", s.block_n, (int)s.pair, s.tiles, s.kb, s.workers, s.slices, s.slice_kb, s.helpers);
        const int busy = s.helpers || s.tiles * s.slices >= s.workers ? s.workers : s.tiles * s.slices;
        im::Part p;
        for (int w = 0; w < busy; ++w)
            for (int i = 0; im::part_at(s, w, i, p); ++i) printf("part %d %d %d %d %d\n", w, p.tile, p.k0, p.n, p.slot);
        printf("end\n");
    }
    return 0;
}
