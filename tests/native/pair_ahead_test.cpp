// Which 256 x 256 tile the gated feed-forward block's forward takes (gemm_cut.h), on the
// host.  "T D F SAVED": the tile, and whether it has a third buffer for A.
#include <cstdio>
#include <cstdlib>

#include "gemm_cut.h"

int main(int argc, char **argv)
{
    if (argc != 5) return 2;
    const size_t t = (size_t)atoll(argv[1]), d = (size_t)atoll(argv[2]), f = (size_t)atoll(argv[3]);
    printf("%d %d\n", ar::dev::ffn_cut(t, d, f).tile, (int)ar::dev::pair_ahead(t, d, f, atoi(argv[4]) != 0));
    return 0;
}
