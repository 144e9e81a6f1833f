// Attention's workspaces: what a call places in them begins where the kernels' accesses may, and lies within what the caller was asked for.
#include <cstdio>

#include "sl_attention_rules.h"

static int failures = 0;
static void fail(const char *what, long long a, long long b, long long c, long long d)
{
    if (++failures < 20) std::printf("%s: %lld %lld %lld %lld\n", what, a, b, c, d);
}

static void tokens()
{
    const int heads[][2] = {{1, 1}, {5, 1}, {5, 5}, {3, 3}, {9, 3}, {16, 16}, {20, 5}, {40, 1}, {66, 2}, {200, 2}, {65536, 1}, {2000, 2000}};
    for (const auto &h : heads)
        for (const int64_t n : {1, 2, 3, 64, 1000})
            for (int64_t tokens = 0; tokens < 3000000; tokens += tokens < 5000 ? 1 : tokens / 37)
                for (const int64_t dim : {8, 40, 128}) {
                    const int64_t units = sl_token_units(h[0], h[1]);
                    const int64_t parts = tokens / sl_token_part(tokens, units) + n, most = sl_token_most_parts(n, tokens, units);
                    const SlTokenRoom r = sl_token_room(parts, h[0], dim);
                    if (r.values % 4 != 0) fail("values at less than 16 bytes", n, tokens, h[0], dim);
                    if (r.stats < r.values + parts * h[0] * dim && r.values < r.stats + 2 * parts * h[0]) fail("overlap", n, tokens, h[0], dim);
                    if (r.floats > sl_token_room(most, h[0], dim).floats) fail("room", n, tokens, h[0], dim);
                    if (std::max(r.values + parts * h[0] * dim, r.stats + 2 * parts * h[0]) > r.floats) fail("end", n, tokens, h[0], dim);
                }
}

int main()
{
    tokens();
    if (failures == 0) std::puts("ok");
    return failures != 0;
}
