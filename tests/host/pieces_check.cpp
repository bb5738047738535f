// What a piece of the classes takes of the workspace, by the rules of paper_1810_09868_amd/csrc/plans.h: reads lines "dtype N In K" and prints the
// bytes of a piece's dz and laid out weights, what they may be, whether the places of the forward call's workspace follow each other, and the number of pieces.
#include <cstdio>

#include "../../paper_1810_09868_amd/csrc/plans.h"

int main()
{
    int dtype, N, In, K;
    while (scanf("%d %d %d %d", &dtype, &N, &In, &K) == 4) {
        using namespace vgg;
        const XentPlan p = xent_plan(dtype, N, In, K);
        const size_t most = p.classes < K ? p.classes : K, dz = (size_t)p.PL * 2 * (p.NP + p.rest_rows) * p.ld_dz, w = p.direct_w ? 0 : (size_t)p.PL * 2 * up(most, kStep) * p.InP;
        // (256 classes are the least; where the scores' contraction is split all classes are one piece)
        const bool least = p.classes == kTA || p.z_splits;
        const size_t order[] = {p.a_at, p.w_at, p.ea_at, p.most_at, p.z_at, p.sums_at, p.label_at, p.forward_bytes};
        bool follow = p.dz_at + dz <= p.da_at && p.w_at + w <= p.ea_at;
        for (size_t k = 1; k < sizeof order / sizeof *order; ++k) follow = follow && order[k] >= order[k - 1] && order[k] % 256 == 0;
        if (!p.z_splits) follow = follow && p.sums_at + (size_t)div_up(K, kTA) * N * 8 <= p.label_at && p.label_at + (size_t)N * 4 <= p.forward_bytes;
        printf("%zu %zu %d %d\n", dz + w, least ? dz + w : kPieceBytes, follow, p.pieces);
    }
    return 0;
}
