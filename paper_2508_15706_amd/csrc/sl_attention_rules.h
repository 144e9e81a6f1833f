// Into how many parts attention cuts its work, by sizes alone, and the room that goes with it: plain C++.
#pragma once
#include <algorithm>
#include <stddef.h>
#include <stdint.h>

// Rows of a workgroup, 32 to each of its waves.
enum { AT_ROWS = 128 };

// ---- backward ----

// Parts of a group's heads that the passes over keys take apart, joined in fp32: workgroups that walk past all of a group's queries are few and long
// where key heads are few, and the longest walk is the pass.  From 512 workgroups of 128 keys on (two to a compute unit), and where no walk is long,
// the join costs what it gives.  Backward, us, one slice / sliced: 8192 tokens, 20 heads of 128 on 5 1775 / 1182, 4096, 8 on 1 543 / 257, 512, 8 on 1
// 72 / 47, 4 x 2048, 20 on 5 486 / 400; 2 x 512, 20 on 5 58 / 63, 8 x 1024, 16 heads of 64 on 4 99 / 121, 4 x 256, 16 on 2 34 / 41.
enum { AT_SLICED_BELOW = 512, AT_SLICED_TO = 1024, AT_LONG_WALK = 8192, AT_HARDLY_ANY = 64, AT_MOST_PART_ROWS = (AT_SLICED_BELOW + AT_SLICED_TO) * AT_ROWS };
// Rows of dk and of dv that the parts of any call with so many queries have; none where no heads share a key head.
inline int64_t sl_back_part_rows(int64_t tokens_q, int64_t heads, int64_t kv_heads)
{
    return heads == kv_heads ? 0 : std::min<int64_t>(tokens_q * heads, AT_MOST_PART_ROWS);
}
inline int sl_back_slices(int64_t tokens_q, int64_t tokens_k, int64_t sequences, int64_t heads, int64_t kv_heads)
{
    const int64_t w = (tokens_k / AT_ROWS + sequences) * kv_heads, group = heads / kv_heads;
    if (w >= AT_SLICED_BELOW || tokens_q == 0 || tokens_q / sequences * group < (w <= AT_HARDLY_ANY ? AT_LONG_WALK / 2 : AT_LONG_WALK)) return 1;
    int64_t slices = std::min<int64_t>(group, (AT_SLICED_TO + w - 1) / w);
    while (slices > 1 && slices * tokens_k * kv_heads > sl_back_part_rows(tokens_q, heads, kv_heads)) --slices;      // (more keys than queries: what the room holds)
    return (int)slices;
}
// A workspace, in floats: the queries' statistics and what stands for no query, then the parts.
inline int64_t sl_back_stats(int64_t tokens_q, int64_t heads) { return (2 * tokens_q * heads + 2 + 3) / 4 * 4; }
inline int64_t sl_back_room(int64_t tokens_q, int64_t heads, int64_t kv_heads, int64_t dim)
{
    return sl_back_stats(tokens_q, heads) + 2 * dim * sl_back_part_rows(tokens_q, heads, kv_heads);
}

// ---- single tokens ----

// Keys of a part: one wave's work.
enum { AT_LEAST_PART = 32, AT_LONGEST_PART = 512, AT_MOST_WAVES = 1280 };

// Parts are as short as leaves about AT_MOST_WAVES of them: for one sequence their number counts, for many their evenness.
inline unsigned sl_token_part(int64_t tokens, int64_t units)
{
    unsigned part = AT_LEAST_PART;
    while (part < AT_LONGEST_PART && tokens / part * units > AT_MOST_WAVES) part *= 2;
    return part;
}
inline int64_t sl_token_most_parts(int64_t sequences, int64_t tokens, int64_t units)
{
    return std::min(tokens / AT_LEAST_PART, std::max<int64_t>(AT_MOST_WAVES / units, tokens / AT_LONGEST_PART)) + sequences;
}
// Groups of up to 32 heads that share a key head.
inline int64_t sl_token_units(int64_t heads, int64_t kv_heads) { return kv_heads * ((heads / kv_heads + 31) / 32); }

// A workspace, in floats: per part and head dim values, which are written 16 bytes at a time, and then two statistics (in front of the values
// these would leave them at 8 bytes wherever parts x heads is odd).
struct SlTokenRoom {
    int64_t values, stats, floats;
};
inline SlTokenRoom sl_token_room(int64_t parts, int64_t heads, int64_t dim)
{
    return SlTokenRoom{0, parts * heads * dim, parts * heads * (dim + 2)};
}
