// What the attention kernels share: where a workgroup's tile lies in the packed sequences, tiles of rows in LDS, and the
// operands that the matrix unit takes from them.
//
// Two shapes carry all of it (lane l, h = l / 32; the 32 x 32 x 16 product of bf16):
//   a score tile is computed with the other side's rows as its rows, so that column l % 32 - one query, or one key in the backward pass over
//   keys - belongs to lanes l and l ^ 32, and of it the rows 8 g + 4 h + e, g, e = 0 .. 3, at 4 g + e;
//   as the operand of the next product a lane needs eight of the contraction's sixteen: it takes the eight that it has, 4 h + {0..3} and
//   8 + 4 h + {0..3}, and the other operand is read in the same order - transposed, four rows at a time, out of LDS.  So no
//   probability ever moves between lanes.
#pragma once
#include "sl_attention_rules.h"
#include "sl_dma.h"
#include "sl_mx4.h"

#include <climits>
#include <cmath>

#include "sl_internal.h"

typedef float sl_f16 __attribute__((ext_vector_type(16)));
typedef __bf16 sl_b8 __attribute__((ext_vector_type(8)));

// Rows of the other side in a stage of LDS, and in a short one.
enum { AT_TILE = 64, AT_STAGE = 32 };

struct SlRows {                  // a tensor of tokens x heads x dim; strides in bytes
    unsigned char *p;
    long long token, head;
};

struct SlSequences {
    const int *q_start, *k_start, *k_count;
    int n, tokens_q, tokens_k;
    int heads, group;            // query heads, and how many of them share a key head
    int octets;                  // dim / 8
    int causal;
    unsigned tiles;              // in the grid; some are empty
    float scale, scale2;         // scale2 = scale * log2(e)
};

// Workgroup i of `tiles` x `heads`.  Workgroups reach the eight XCDs in turn; an XCD is given heads / 8 heads of its own, whose keys and
// values its L2 then holds for all tiles, and of each head that is left over every eighth tile.  Tiles come in order, all of an XCD's heads
// with one tile before the next.
struct SlItem { unsigned tile, head; };
SL_DEV SlItem sl_item(unsigned i, unsigned heads)
{
    const unsigned xcd = i & 7u, own = heads >> 3, block = (i >> 3) / heads, w = (i >> 3) % heads;
    if (w < 8u * own) return SlItem{block * 8u + w / own, xcd * own + w % own};
    const unsigned r = w - 8u * own;
    return SlItem{block * 8u + ((xcd + r) & 7u), 8u * own + r};
}
inline unsigned sl_item_groups(long long tiles, long long heads) { return (unsigned)((tiles + 7) / 8 * 8 * heads); }

// Tile t of the tokens: sequence s has ceil(length / rows) tiles from start / rows + s on, which no other one reaches, since
// ceil(b) <= floor(a + b) - floor(a) + 1; tokens / rows + n is no less than all of them.  Whatever the starts hold, the
// rows found lie within the tokens.
struct SlSpan { int s, first, count, row0; };        // the sequence's first row and its number of rows; this tile's first one in it
SL_DEV bool sl_find_tile(const int *start, int n, int tokens, unsigned rows, unsigned t, SlSpan &out)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        const unsigned first = (unsigned)min(max(start[mid], 0), tokens) / rows + (unsigned)mid;
        if (first <= t) lo = mid;
        else hi = mid - 1;
    }
    const int a = min(max(start[lo], 0), tokens), b = min(max(start[lo + 1], a), tokens);
    const long long row0 = ((long long)t - (long long)((unsigned)a / rows + (unsigned)lo)) * rows;
    out.s = lo, out.first = a, out.count = b - a, out.row0 = (int)row0;
    return row0 >= 0 && row0 < b - a;
}
// Rows of a sequence on one side; `count`: how many of them are used, or null.
SL_DEV void sl_rows_of(const int *start, const int *count, int s, int tokens, int &first, int &n)
{
    const int a = min(max(start[s], 0), tokens), b = min(max(start[s + 1], a), tokens);
    first = a;
    n = count ? min(max(count[s], 0), b - a) : b - a;
}

// The sum over the wave's lanes, in all of them (and known to be the same).
SL_DEV int sl_wave_sum(int v)
{
#pragma unroll
    for (int l = 0; l < 4; ++l) v += sl_partner(v, l);
    return (__builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16)) + (__builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48));
}

// The same by work: where queries see only keys before them, a sequence's tile `level` from its light end is `level` tiles' work more than the
// lightest, and a workgroup that begins with a heavy tile late keeps the others waiting.  Item t is the t-th of all sequences' tiles in
// descending order of their levels.  Each lane holds PER sequences' numbers of tiles; the sum of max(tiles - level, 0) over them is
// the number of tiles of that level or more.  Lists of more sequences than that have enough tiles for the order not to count.
// (eight sequences of 2048 tokens, forward: 209 us in the sequences' order, so 177)
// What belongs to a sequence is requested by its lane at the start, all of it at once, and then read from the lane.
template <int PER>
SL_DEV bool sl_find_level(const int *start, int tokens, const int *other_start, const int *other_count, int other_tokens, int n, unsigned rows, unsigned t,
                          bool light_first, SlSpan &out, int &other_first, int &other_n)
{
    const int lane = threadIdx.x & 63;
    int first[PER], count[PER], of[PER], on[PER], tiles[PER], most = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int s = min(i * 64 + lane, n - 1);
        const int a = start[s], b = start[s + 1], c = other_start[s], d = other_start[s + 1], e = other_count ? other_count[s] : INT_MAX;
        first[i] = min(max(a, 0), tokens), count[i] = min(max(b, first[i]), tokens) - first[i];
        of[i] = min(max(c, 0), other_tokens), on[i] = min(max(e, 0), min(max(d, of[i]), other_tokens) - of[i]);
        tiles[i] = i * 64 + lane < n ? (int)(((unsigned)count[i] + rows - 1) / rows) : 0;
        most = max(most, tiles[i]);
    }
    most = sl_wave_max(most);
    auto reach = [&](int level) __attribute__((always_inline)) {        // tiles of that level or more
        int c = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) c += max(tiles[i] - level, 0);
        return (unsigned)sl_wave_sum(c);
    };
    int lo = 0, hi = most;                       // reach(lo) > t >= reach(hi)
    if (reach(0) <= t) return false;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (reach(mid) > t) lo = mid;
        else hi = mid;
    }
    unsigned left = t - reach(lo + 1);           // which of the sequences that have this level
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const unsigned long long has = sl_ballot(tiles[i] > lo);
        const unsigned c = (unsigned)sl_popc(has);
        if (left < c) {
            const int l = sl_uniform(__builtin_ctzll(sl_ballot(tiles[i] > lo && (unsigned)sl_mbcnt(has) == left)));
            out.s = i * 64 + l, out.first = __builtin_amdgcn_readlane(first[i], l), out.count = __builtin_amdgcn_readlane(count[i], l);
            out.row0 = (light_first ? lo : __builtin_amdgcn_readlane(tiles[i], l) - 1 - lo) * (int)rows;
            other_first = __builtin_amdgcn_readlane(of[i], l), other_n = __builtin_amdgcn_readlane(on[i], l);
            return true;
        }
        left -= c;
    }
    return false;
}
// Item t of the list's tiles of `rows` rows, and the rows of its sequence on the other side, of which `other_count` (or null) says how many are used.
SL_DEV bool sl_find(const int *start, int tokens, const int *other_start, const int *other_count, int other_tokens, const SlSequences &s, unsigned rows, unsigned t,
                    bool light_first, SlSpan &out, int &other_first, int &other_n)
{
    if (s.n <= 64) return sl_find_level<1>(start, tokens, other_start, other_count, other_tokens, s.n, rows, t, light_first, out, other_first, other_n);
    if (s.n <= 256) return sl_find_level<4>(start, tokens, other_start, other_count, other_tokens, s.n, rows, t, light_first, out, other_first, other_n);
    if (!sl_find_tile(start, s.n, tokens, rows, light_first ? s.tiles - 1 - t : t, out)) return false;
    sl_rows_of(other_start, other_count, out.s, other_tokens, other_first, other_n);
    return true;
}

// ---- tiles in LDS ----

// Rows of D bf16 in pieces of 16 bytes; piece c of row r is at c ^ turn(r) of its row: eight consecutive rows' same piece, and four rows'
// four neighbouring ones (what half a wave reads transposed), are in banks of their own.
template <int D>
SL_DEV int sl_turn(int r) { return D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 3 & 1) << 1 | (r >> 2 & 1); }

// One wave's share of ROWS rows: 1 KB an instruction, every fourth from its own on.
template <int D, int ROWS = AT_TILE>
struct SlTileLoad {
    enum { PIECES = D / 8, PER = 64 / PIECES, LOADS = ROWS / PER / 4 };
    int row;                     // this lane's in the first load
    unsigned at;                 // its piece's offset in a row
    unsigned off;                // its byte offset from the tile's first row
    long long token;

    SL_DEV void setup(int wave, int lane, int octets, long long stride)
    {
        row = wave * PER + lane / PIECES;
        at = (unsigned)min((lane % PIECES) ^ sl_turn<D>(row), octets - 1) * 16u;       // (columns past the last: that piece again, never used)
        token = stride;
        off = (unsigned)row * (unsigned)token + at;
    }
    // rows tile .. + ROWS - 1 of `count`; what lies past the last one is read there
    SL_DEV void load(const unsigned char *base, int tile, int count, unsigned lds, int wave) const
    {
        const unsigned char *from = base + tile * token;
        const int last = count - 1 - tile;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const unsigned to = lds + (unsigned)(wave + 4 * i) * 1024u;
            if (last >= ROWS - 1) dma16(from + i * (4 * PER) * token, off, to);
            else dma16(from, (unsigned)min(row + i * 4 * PER, last) * (unsigned)token + at, to);
        }
    }
};

// 32 rows to a wave's own LDS.
template <int D>
struct SlWaveLoad {
    enum { PIECES = D / 8, PER = 64 / PIECES, LOADS = AT_STAGE / PER };
    unsigned at[LOADS], off[LOADS];
    int row;
    long long token;

    SL_DEV void setup(int lane, int octets, long long stride)
    {
        row = lane / PIECES, token = stride;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            at[i] = (unsigned)min((lane % PIECES) ^ sl_turn<D>(row + i * PER), octets - 1) * 16u;
            off[i] = (unsigned)(row + i * PER) * (unsigned)token + at[i];
        }
    }
    // rows first .. + 31, of which `count` exist (at least one)
    SL_DEV void load(const unsigned char *base, int first, int count, unsigned lds) const
    {
        const unsigned char *from = base + first * token;
        if (count >= AT_STAGE) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) dma16(from, off[i], lds + i * 1024u);
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) dma16(from, (unsigned)min(row + i * PER, count - 1) * (unsigned)token + at[i], lds + i * 1024u);
        }
    }
};

// Operand with rows of the tile as its rows (or columns): step s, 16 of D, of rows 32 t + l % 32.
template <int D>
SL_DEV int sl_plain_base(int lane) { return (lane & 31) * (2 * D) + (((lane >> 5) ^ sl_turn<D>(lane & 31)) << 4); }
template <int D>
SL_DEV sl_b8 sl_plain(const unsigned char *tile, int base, int t, int s)
{
    return *reinterpret_cast<const sl_b8 *>(tile + (base ^ (s << 5)) + t * 32 * (2 * D));
}
// Transposed operand: columns 32 m + l % 32 of the tile as rows, rows 16 g .. + 15 of it as the contraction, in the order above.
template <int D>
SL_DEV int sl_turned_base(int lane)
{
    const int r = 4 * (lane >> 5) + (lane >> 2 & 3), piece = (lane >> 4 & 1) * 2 + (lane >> 1 & 1);
    return r * (2 * D) + ((piece ^ sl_turn<D>(r)) << 4) + (lane & 1) * 8;
}
template <int D>
SL_DEV sl_b8 sl_turned(const unsigned char *tile, int base, int m, int g)
{
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s4 *lds_s4;
    const unsigned char *a = tile + (base ^ (m << 6)) + g * 16 * (2 * D), *b = tile + (base ^ (m << 6) ^ 32) + (g * 16 + 8) * (2 * D);
    union { s4 h[2]; sl_b8 v; } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(a));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(b));
    return u.v;
}

SL_DEV sl_f16 sl_mfma(sl_b8 a, sl_b8 b, sl_f16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
SL_DEV sl_f16 sl_zero16()
{
    sl_f16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}

// The order of N products, each with one read of LDS: AHEAD reads first, then one for each product.  (Left to itself the compiler waits for
// every pair of reads in front of its products: forward pass over 8192 tokens, 20 heads of 128, 389 us, so 357.)
template <int N, int AHEAD>
SL_DEV void sl_reads_ahead()
{
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < N - AHEAD; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
}

// Eight values of a score tile as the operand of the next product: rounded to bf16, which the matrix unit takes (off by half a step at most,
// 2^-8 of a probability, random from one key to the next).
SL_DEV sl_b8 sl_operand(const sl_f16 &s, int g)
{
    const sl_u4 w = g == 0 ? sl_u4{sl_bf16_pair(s[0], s[1]), sl_bf16_pair(s[2], s[3]), sl_bf16_pair(s[4], s[5]), sl_bf16_pair(s[6], s[7])}
                           : sl_u4{sl_bf16_pair(s[8], s[9]), sl_bf16_pair(s[10], s[11]), sl_bf16_pair(s[12], s[13]), sl_bf16_pair(s[14], s[15])};
    return __builtin_bit_cast(sl_b8, w);
}

// Of the other half of the wave.
SL_DEV float sl_both_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
SL_DEV float sl_both_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// One wave's softmax over 32 keys at a time.  The maximum that the exponents refer to moves only where a row's new one is more than 2^8 above
// it: the sum and the output then stay below 2^8 times their values, and the output's registers are scaled a few times in all.
struct SlRunning {
    float top = -INFINITY, ref = 0.0f, sum = 0.0f;       // the maximum, it or 0, this half's part of the sum

    // keys 8 g + e >= left of this half are not seen
    template <int D>
    SL_DEV void tile(const unsigned char *kt, const unsigned char *vt, int plain, int turned, const sl_b8 (&q)[D / 16], int left, float scale2, sl_f16 (&o)[D / 32])
    {
        sl_f16 s = sl_zero16();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) s = sl_mfma(sl_plain<D>(kt, plain, 0, i), q[i], s);
        sl_reads_ahead<D / 16, 4>();
        __builtin_amdgcn_sched_barrier(0);
        if (sl_ballot(left < AT_STAGE - 4)) {                // (the last key of either half is its 27th)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (8 * (e >> 2) + (e & 3) >= left) s[e] = -INFINITY;
        }
        float now = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) now = __builtin_elementwise_maximum(now, s[e]);
        now = sl_both_max(now) * scale2;
        if (sl_ballot(now > top + 8.0f)) {
            const float next = fmaxf(top, now), to = next == -INFINITY ? 0.0f : next, by = __builtin_amdgcn_exp2f(top - to);
            top = next, ref = to, sum = sum * by;
#pragma unroll
            for (int m = 0; m < D / 32; ++m)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[m][e] = o[m][e] * by;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], scale2, -ref));
            sum = sum + s[e];
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const sl_b8 p = sl_operand(s, g);
#pragma unroll
            for (int m = 0; m < D / 32; ++m) o[m] = sl_mfma(sl_turned<D>(vt, turned, m, g), p, o[m]);
        }
    }
};

// Row of a wave's own side: 16 bytes at every other piece, this half's.
template <int D>
SL_DEV void sl_own_row(const unsigned char *row, int half, int octets, sl_b8 (&v)[D / 16])
{
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        sl_u4 w = {0u, 0u, 0u, 0u};
        if (2 * s + half < octets) w = *reinterpret_cast<const sl_u4 *>(row + (2 * s + half) * 16);
        v[s] = __builtin_bit_cast(sl_b8, w);
    }
}

// 32 columns of a transposed result (this lane's column a row of memory) times `by`, in bf16: the halves exchange every second four so that
// each writes 16 bytes.
SL_DEV void sl_put_block(unsigned char *row, bool there, int half, int octets, const sl_f16 &v, int m, float by)
{
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
        const unsigned a0 = sl_bf16_pair(v[4 * g] * by, v[4 * g + 1] * by), a1 = sl_bf16_pair(v[4 * g + 2] * by, v[4 * g + 3] * by);
        const unsigned b0 = sl_bf16_pair(v[4 * g + 4] * by, v[4 * g + 5] * by), b1 = sl_bf16_pair(v[4 * g + 6] * by, v[4 * g + 7] * by);
        const auto r0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), r1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
        const int piece = m * 4 + g + half;
        if (there && piece < octets) *reinterpret_cast<sl_u4 *>(row + piece * 16) = sl_u4{r0[0], r1[0], r0[1], r1[1]};
    }
}
template <int D>
SL_DEV void sl_put_row(unsigned char *row, bool there, int half, int octets, const sl_f16 (&v)[D / 32], float by)
{
#pragma unroll
    for (int m = 0; m < D / 32; ++m) sl_put_block(row, there, half, octets, v[m], m, by);
}

// The same in fp32, as it is.
SL_DEV void sl_put_floats(float *row, bool there, int half, int octets, const sl_f16 &v, int m)
{
#pragma unroll
    for (int g = 0; g < 4; ++g)
        if (there && m * 4 + g < octets) *reinterpret_cast<sl_f4 *>(row + 32 * m + 8 * g + 4 * half) = sl_f4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
}

// A wave's block of a result to LDS and the sum of four waves' from there, in their order; 16 floats a lane, 4 KB a block.
SL_DEV void sl_leave_block(float *room, int lane, const sl_f16 &v)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<sl_f4 *>(room + j * 256 + lane * 4) = sl_f4{v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
}
SL_DEV sl_f16 sl_four_blocks(const float *room, int stride, int lane, sl_f4 by)
{
    sl_f16 v = sl_zero16();
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const sl_f4 x = *reinterpret_cast<const sl_f4 *>(room + w * stride + j * 256 + lane * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * j + e] = fmaf(x[e], by[w], v[4 * j + e]);
        }
    return v;
}

// ---- arguments ----

const int64_t AT_MOST_TOKENS = (int64_t)1 << 30, AT_MOST_HEADS = 1 << 16, AT_MOST_SEQUENCES = (int64_t)1 << 22, AT_MOST_STRIDE = (int64_t)1 << 24;

// False where the shape is none.  (A grid has less than 2^32 threads: 2^24 workgroups of 256.  The queries that a key is walked past, 32 at a time in all
// heads of its group, are then less than 2^27.)
inline bool sl_attention_sequences(const sl_attention_shape *p, SlSequences &s)
{
    if (!p || p->sequences < 0 || p->sequences > AT_MOST_SEQUENCES || p->tokens_q < 0 || p->tokens_q > AT_MOST_TOKENS || p->tokens_k < 0 || p->tokens_k > AT_MOST_TOKENS)
        return false;
    if (p->heads < 1 || p->heads > AT_MOST_HEADS || p->kv_heads < 1 || p->heads % p->kv_heads != 0) return false;
    if (p->head_dim < 8 || p->head_dim > 128 || p->head_dim % 8 != 0) return false;
    const double scale2 = p->scale * 1.4426950408889634;
    if (!(scale2 >= 1e-30 && scale2 <= 1e30)) return false;
    if (p->sequences > 0 && (!p->k_start || ((uintptr_t)p->q_start & 3) || ((uintptr_t)p->k_start & 3) || ((uintptr_t)p->k_count & 3))) return false;
    const int64_t most = p->tokens_q > p->tokens_k ? p->tokens_q : p->tokens_k;
    if (((most / AT_ROWS + p->sequences + 7) / 8 * 8) > ((int64_t)1 << 24) / p->heads - 1) return false;
    s.q_start = p->q_start, s.k_start = p->k_start, s.k_count = p->k_count;
    s.n = (int)p->sequences, s.tokens_q = (int)p->tokens_q, s.tokens_k = (int)p->tokens_k;
    s.heads = p->heads, s.group = p->heads / p->kv_heads, s.octets = p->head_dim / 8, s.causal = p->causal != 0;
    s.scale = (float)p->scale, s.scale2 = (float)scale2;
    return true;
}

// False where the tensor is not one that the kernels read; `needed`: it has rows.
inline bool sl_attention_in(const sl_heads *t, bool needed, SlRows &r)
{
    if (!needed) return true;
    if (!t || !t->data || ((uintptr_t)t->data & 15)) return false;
    if (t->token_stride < 0 || t->token_stride > AT_MOST_STRIDE || t->head_stride < 0 || t->head_stride > ((int64_t)1 << 40) ||
        t->token_stride % 8 != 0 || t->head_stride % 8 != 0)
        return false;
    r.p = static_cast<unsigned char *>(t->data), r.token = t->token_stride * 2, r.head = t->head_stride * 2;
    return true;
}
// ... or not one that they write: no two of its rows share memory.
inline bool sl_attention_out(const sl_heads *t, bool needed, int64_t tokens, int64_t heads, int64_t dim, SlRows &r)
{
    if (!sl_attention_in(t, needed, r)) return false;
    if (!needed) return true;
    if ((heads > 1 && t->head_stride < dim) || (tokens > 1 && t->token_stride < dim)) return false;
    return heads == 1 || tokens == 1 || t->token_stride >= t->head_stride * (heads - 1) + dim || t->head_stride >= t->token_stride * (tokens - 1) + dim;
}
