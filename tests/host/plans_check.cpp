// Which kernels' variants calls take, by the rules of paper_1810_09868_amd/csrc/plans.h: reads lines "muon batch m n", "few planes rows
// cols", "w4 dtype N In Out" and "xent dtype N In K", and prints the tile, whether a launch takes a whole step, "row", "tile" or the tiles of rows
// and outputs, or "small" or the pieces, the scores' ranges and the columns of the four products' tiles, once the plan holds together.
#include <cstdio>
#include <cstring>
#include <initializer_list>

#include "../../paper_1810_09868_amd/csrc/plans.h"

// What the kernels take for granted of a plan.
static const char *fault(const vgg::XentPlan &p, int dtype, int N, int In, int K)
{
    using namespace vgg;
    const long steps = p.InP / kStep, most = p.classes < K ? p.classes : K, row = 2l * p.PL;
    if (p.classes % kTA || (long)p.pieces * p.classes < K || (long)(p.pieces - 1) * p.classes >= K) return "pieces";
    if (p.z_splits && (p.pieces != 1 || p.z_splits < 2 || p.z_splits > steps)) return "scores' ranges";
    if (p.da_splits < 1 || p.da_splits > div_up(most, kStep) || p.dw_splits < 1 || p.dw_splits > (p.NP + p.rest_rows) / kStep) return "ranges";
    if (p.ld_dz % kStep || p.ld_dz < most || p.InP % kStep || p.InP < In || p.NP % kStep || p.NP < N || (p.rest_rows && p.rest_rows != p.NP)) return "strides";
    // a tile's offsets from its base, 32 bits of them
    if (p.ld_dz * row * 256 >= 1l << 31 || p.InP * row * 256 >= 1l << 31) return "offsets";
    for (int tn : {p.tn, p.grad_tn, p.da_tn, p.dw_tn})
        if (tn != 64 && tn != 128 && tn != 256) return "tiles";
    const long grids[] = {div_up(most, kTA) * div_up(N, p.tn) * (p.z_splits ? p.z_splits : 1), div_up(In, kTA) * div_up(N, p.da_tn) * p.da_splits,
                          div_up(In, kTA) * div_up(most, p.dw_tn) * p.dw_splits};
    for (long g : grids)
        if (g < 1 || g >= 1l << 31) return "workgroups";
    if (!p.z_splits && p.db_parts != div_up(N, p.grad_tn)) return "db";
    if (p.direct_w && (dtype != VGG_BF16 || In % kStep)) return "weights";
    const size_t order[] = {p.a_at, p.w_at, p.ea_at, p.most_at, p.z_at, p.a2_at, p.eg_at, p.tail_at, p.rest_at, p.dz_at, p.da_at, p.dw_at, p.db_at, p.backward_bytes};
    for (size_t k = 1; k < sizeof order / sizeof *order; ++k)
        if (order[k] < order[k - 1] || order[k] % 256) return "places";
    return nullptr;
}

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
        } else if (!strcmp(kind, "xent")) {
            if (scanf("%d %d %d %d", &a, &b, &c, &d) != 4) return 1;
            const vgg::XentPlan p = vgg::xent_plan(a, b, c, d);
            if (const char *what = fault(p, a, b, c, d)) printf("%s\n", what);
            else if (vgg::xent_is_small(a, b, c, d)) printf("small\n");
            else printf("%d %d %d %d %d %d\n", p.pieces, p.z_splits, p.tn, p.grad_tn, p.da_tn, p.dw_tn);
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
