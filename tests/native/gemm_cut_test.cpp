// The tiles that products take (gemm_cut.h), on the host.  Without arguments: every
// forward of the gated feed-forward block over a range of sizes takes the cheapest of
// the shapes that exist, by the rule's own prices.  "ffn T D F", "ortho PLANES M N
// BATCH": the tile and runs of each product of such a call.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>

#include "gemm_cut.h"

using namespace ar::dev;

static int failures = 0;
static void expect(bool ok, const char *what, size_t t, size_t d, size_t f, Cut c)
{
    if (!ok && ++failures < 20) printf("%s: %zu x %zu x %zu: tile %d, %u runs\n", what, t, d, f, c.tile, c.splits);
}

static void forward(size_t t, size_t d, size_t f)
{
    const Cut c = ffn_cut(t, d, f);
    const size_t steps = (d + kStepK - 1) / kStepK;
    expect(c.splits >= 1 && c.splits <= kMaxSplits && c.splits <= steps, "runs", t, d, f, c);
    if (t <= 64) {
        expect(c.tile == kFlat, "flat", t, d, f, c);
        return;
    }
    // the shapes that ffn.hip has for more than 64 tokens
    expect(c.tile == kPairSmall || c.tile == kPairLarge || c.tile == kPairDeep, "exists", t, d, f, c);
    expect(c.tile != kPairLarge || c.splits == 1, "256 in one piece", t, d, f, c);
    const double us = pair_us(c.tile, t, d, f, c.splits);
    expect(us <= pair_us(kPairLarge, t, d, f, 1), "256 is cheaper", t, d, f, c);
    const size_t tiles = pair_tiles(kPairSmall, t, f);
    for (uint32_t s = 1; s <= kMaxSplits && may_split(tiles, steps, s); ++s)
        expect(us <= pair_us(tiles * s <= 256 ? kPairDeep : kPairSmall, t, d, f, s), "128 is cheaper", t, d, f, c);
}

static void show(const char *name, Cut c) { printf("%s %d %u\n", name, c.tile, c.splits); }
static int shapes(int argc, char **argv)
{
    auto number = [&](int k) { return k < argc ? (size_t)atoll(argv[k]) : (size_t)0; };
    auto up = [](size_t v) { return (v + kStepK - 1) / kStepK * kStepK; };
    if (!strcmp(argv[1], "ffn") && argc == 5) {
        const size_t t = number(2), d = number(3), f = number(4);
        show("forward", ffn_cut(t, d, f)), show("dx", dx_cut(t, d, up(f))), show("dw", dw_cut(t, d, up(f)));
        return 0;
    }
    if (!strcmp(argv[1], "ortho") && argc == 6) {
        const int planes = (int)number(2);
        const size_t m = number(3), n = number(4), batch = number(5);
        show("a", a_cut(planes, m, up(n), batch)), show("b", b_cut(planes, m, up(m), batch)), show("x", x_cut(planes, m, n, up(m), batch));
        return 0;
    }
    return 2;
}

int main(int argc, char **argv)
{
    if (argc > 1) return shapes(argc, argv);
    for (size_t t : {1, 2, 33, 64, 65, 100, 128, 129, 200, 256, 300, 512, 777, 1000, 1024, 1536, 2048, 2100, 2500, 4096, 6144, 8192, 16384, 65536})
        for (size_t d : {1, 64, 100, 128, 512, 1000, 1024, 1999, 2048, 4096, 6000, 16384})
            for (size_t f : {1, 8, 64, 130, 512, 768, 1024, 1408, 1536, 2048, 2700, 2816, 4100, 4352, 5632, 11264, 16384}) forward(t, d, f);
    // measured: 54 us and less in tiles of 128, 65 of 256; and 92 of 256, 112 of 128
    const struct { size_t t, d, f; int tile; } measured[] = {
        {2048, 1024, 4352, kPairSmall}, {1536, 1024, 5632, kPairSmall}, {6144, 1024, 1408, kPairSmall},
        {1536, 4096, 2816, kPairLarge}, {3200, 4096, 1408, kPairLarge}, {8192, 4096, 11264, kPairLarge}};
    for (const auto &m : measured) {
        const Cut c = ffn_cut(m.t, m.d, m.f);
        expect(c.tile == m.tile, "as measured", m.t, m.d, m.f, c);
    }
    printf("gemm cut: %s\n", failures ? "FAILED" : "ok");
    return failures != 0;
}
