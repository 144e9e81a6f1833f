// Into how many parts attention cuts its work, by sizes alone, and the room that goes with it: plain C++.
#pragma once
#include <algorithm>
#include <stddef.h>
#include <stdint.h>

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
