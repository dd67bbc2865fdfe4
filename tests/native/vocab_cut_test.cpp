// The tiles that the loss over a vocabulary takes (gemm_cut.h), on the host.  "T D V": the
// tile of the statistics, of each piece's dz, and the tile and runs of both products with
// it ("dx" for one piece, "dx_sum" for several, whose first and later ones differ).
#include <cstdio>
#include <cstdlib>

#include "gemm_cut.h"

using namespace ar::dev;

int main(int argc, char **argv)
{
    if (argc != 4) return 2;
    const size_t t = (size_t)atoll(argv[1]), d = (size_t)atoll(argv[2]), v = (size_t)atoll(argv[3]);
    const VocabCut c = vocab_cut(t, d, v);
    printf("stats %d 1\n", logits_tile(t, d, v));
    for (size_t k = 0; k < c.pieces; ++k) {
        const size_t rows = v - k * c.piece < c.piece ? v - k * c.piece : c.piece, steps = (rows + kStepK - 1) / kStepK;
        printf("dz %d 1\n", logits_tile(t, d, rows));
        printf("%s %d %u\n", c.pieces == 1 ? "dx" : k ? "dx_more" : "dx_first", c.dx.tile, c.pieces > 1 && c.dx.splits > steps ? (uint32_t)steps : c.dx.splits);
        printf("dw %d %u\n", c.dw.tile, c.dw.splits);
    }
    return 0;
}
