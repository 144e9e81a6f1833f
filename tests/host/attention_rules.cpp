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

static void backward()
{
    const int heads[][2] = {{1, 1}, {16, 16}, {2, 1}, {8, 1}, {20, 5}, {64, 16}, {16, 2}, {9, 3}, {4096, 1}, {65536, 4}};
    for (const auto &h : heads)
        for (const int64_t n : {1, 2, 7, 100, 5000}) {
            int64_t before[3] = {0, 0, 0};
            for (int64_t q = 1; q < 2000000; q += q < 300 ? 1 : q / 13) {
                const int64_t dims[3] = {8, 72, 128};
                for (int d = 0; d < 3; ++d) {
                    const int64_t room = sl_back_room(q, h[0], h[1], dims[d]);
                    if (sl_back_stats(q, h[0]) % 4 != 0 || sl_back_stats(q, h[0]) < 2 * q * h[0] + 2) fail("statistics", q, n, h[0], h[1]);
                    if (room < before[d] || room > sl_back_room(q, h[0], 1, 128)) fail("fewer queries, or any heads", q, n, h[0], h[1]);
                    if (h[0] == h[1] && room != sl_back_stats(q, h[0])) fail("room for parts that there are none of", q, n, h[0], h[1]);
                    before[d] = room;
                    for (const int64_t k : {q / 50, q / 2, q, 2 * q, 9 * q, (int64_t)1 << 20}) {
                        const int64_t slices = sl_back_slices(q, k, n, h[0], h[1]);
                        if (slices < 1 || slices > h[0] / h[1]) fail("slices", q, k, h[0], h[1]);
                        if (slices > 1 && sl_back_stats(q, h[0]) + slices * 2 * k * h[1] * dims[d] > room) fail("parts", q, k, h[0], h[1]);
                    }
                }
            }
        }
}

int main()
{
    tokens();
    backward();
    if (failures == 0) std::puts("ok");
    return failures != 0;
}
