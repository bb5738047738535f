// Which kernels' variants calls take, by the rules of paper_1810_09868_amd/csrc/plans.h: reads lines "muon batch m n", "few planes rows
// cols" and "w4 dtype N In Out", and prints the tile, whether a launch takes a whole step, or "row", "tile" or the tiles of rows and outputs.
#include <cstdio>
#include <cstring>

#include "../../paper_1810_09868_amd/csrc/plans.h"

int main()
{
    char kind[8];
    while (scanf("%7s", kind) == 1) {
        int a, b, c, d;
        if (!strcmp(kind, "muon")) {
            if (scanf("%d %d %d", &a, &b, &c) != 3) return 1;
            printf("%d\n", vgg::muon_tile(a, b, c));
        } else if (!strcmp(kind, "few")) {
            if (scanf("%d %d %d", &a, &b, &c) != 3) return 1;
            printf("%d\n", vgg::small_blocks(a, b, c) || vgg::is_wide(a, b, c));
        } else {
            if (scanf("%d %d %d %d", &a, &b, &c, &d) != 4) return 1;
            const vgg::W4Plan t = vgg::w4_tiles_plan(a, b, c, d);
            if (b <= vgg::kW4FewRows) printf("row\n");
            else if (vgg::w4_one_tile(a, b, c)) printf("tile\n");
            else printf("%d %d\n", t.nt, t.rt);
        }
    }
    return 0;
}
