// Products of 4-bit matrices: the room for the parts of a contraction serves every smaller product.  With arguments, m n k of any number of products,
// prints which kernel serves each: its tile, the parts of the contraction, whether there are few rows, and the waves to a tile for those.
#include <cstdio>
#include <cstdlib>

#include "sl_mx4_rules.h"

static int failures = 0;
static void fail(const char *what, long long m, long long n, long long k)
{
    std::printf("%s: %lld x %lld x %lld\n", what, m, n, k);
    ++failures;
}

static int64_t needed(int64_t m, int64_t n, int64_t k)
{
    const int64_t parts = sl_mx4_choose(m, n, k).parts;
    return parts > 1 ? parts * m * sl_mx4_part_pitch(n) : 0;
}

static void room()
{
    // what a product takes, against its own room and that of a larger one: every number of row tiles that can be cut, sizes beside tiles'
    // ends, contractions on both sides of every line of the rule
    const int64_t widths[] = {1, 63, 64, 65, 512, 1000, 2048, 6400, 6401, 8192, 50257};
    const int64_t lengths[] = {1, 4480, 4481, 4608, 6252, 8192, 11212, 12288, 12289, 16384, 50257, 200000};
    for (const int64_t n : widths)
        for (const int64_t k : lengths) {
            int64_t before = 0;
            for (int64_t m = 1; m <= 6500; m += m < 130 ? 1 : 9) {
                const int64_t r = sl_mx4_parts_room(m, n, k);
                if (r < needed(m, n, k)) fail("its own parts", m, n, k);
                if (r < before) fail("fewer rows", m, n, k);
                if (r > sl_mx4_parts_room(m, n + 1, k) || r > sl_mx4_parts_room(m, n, k + 128)) fail("a smaller n or k", m, n, k);
                before = r;
            }
        }
    for (int64_t tiles = 1; tiles <= MX_PARTED_TILES; ++tiles)
        for (int64_t steps = 1; steps <= 2000; ++steps)
            if (needed(64 * tiles, 64, 128 * steps) > sl_mx4_parts_room(64 * tiles, 64, 128 * steps)) fail("its own parts", 64 * tiles, 64, 128 * steps);
}

int main(int argc, char **argv)
{
    for (int i = 1; i + 2 < argc; i += 3) {
        const long long m = std::atoll(argv[i]), n = std::atoll(argv[i + 1]), k = std::atoll(argv[i + 2]);
        const SlMx4Choice c = sl_mx4_choose(m, n, k);
        std::printf("%d %d %d %d\n", c.tile, c.parts, (int)sl_mx4_few_rows(m, k), 1 << sl_mx4_few_waves_log2(n));
    }
    if (argc > 1) return 0;
    room();
    if (!failures) std::printf("ok\n");
    return failures ? 1 : 0;
}
