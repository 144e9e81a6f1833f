// Layout of the microscaled 4-bit matrices (include/sparseloco.h) and the conversions to and from them.
//
// The layout is that of the matrix unit's operands: in the 32 x 32 x 64 product of 4-bit operands lane l holds block
// l / 32 of row l % 32 - 16 bytes - and one byte of a register gives the block's scale.  A tile of 32 rows x 128
// columns is therefore two operands of 1 KB that a wave loads in lane order, and the scale tile of 64 rows is one
// word per lane whose four bytes serve the four operands of 64 rows x 128 columns.
#pragma once
#include "sl_device.h"
#include "sl_mx4_rules.h"

struct SlMx4Shape {
    long long rows, cols;
    long long row_tiles;        // tiles of 32 rows
    long long col_tiles;        // tiles of 128 columns
    long long scales;           // byte offset of the scales
    long long bytes;
};

// Offsets of block b of row r in its tile of codes and of its byte in its tile of scales.
__host__ __device__ inline int sl_mx4_code_at(int r, int b) { return 512 * b + 16 * (r & 31); }
__host__ __device__ inline int sl_mx4_scale_at(int r, int b) { return 128 * (b & 1) + 4 * (r & 31) + 2 * (r >> 5 & 1) + (b >> 1); }

// False where sl_mx4_bytes is 0.
inline bool sl_mx4_shape(long long rows, long long cols, SlMx4Shape &s)
{
    const long long most = 1ll << 40;
    if (rows < 1 || cols < 1 || rows > most || cols > most) return false;
    s.rows = rows, s.cols = cols;
    s.row_tiles = (rows + MX_ROWS - 1) / MX_ROWS;
    s.col_tiles = (cols + MX_COLS - 1) / MX_COLS;
    if (s.row_tiles > MX_MOST_TILES / s.col_tiles) return false;
    s.scales = s.row_tiles * s.col_tiles * MX_TILE_BYTES;
    s.bytes = s.scales + (rows + MX_SCALE_ROWS - 1) / MX_SCALE_ROWS * s.col_tiles * MX_SCALE_TILE_BYTES;
    return true;
}

typedef unsigned sl_u4 __attribute__((ext_vector_type(4)));
typedef unsigned sl_u2 __attribute__((ext_vector_type(2)));

// Scale byte of a block whose largest magnitude has these fp32 bits: the smallest X with it <= 6 * 2^(X - 127).
SL_DEV unsigned sl_mx4_scale(unsigned top)
{
    if (top >= 0x7F800000u) return 255u;
    return (unsigned)max((int)((top + 0x3FFFFFu) >> 23) - 2, 0);
}

// The factor as a number: 2^-127 is a subnormal, 255 a NaN.
SL_DEV float sl_mx4_factor(unsigned x)
{
    return __uint_as_float(x == 0u ? 0x400000u : x == 255u ? 0x7FC00000u : x << 23);
}

// Two elements to the byte SEL of a word (divided by the factor, to nearest even, cut off above 6).
template <int SEL>
SL_DEV unsigned sl_mx4_pair(unsigned old, float a, float b, float factor)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, factor, SEL);
}
typedef __bf16 sl_bf2 __attribute__((ext_vector_type(2)));
template <int SEL>
SL_DEV unsigned sl_mx4_pair(unsigned old, unsigned bf16_pair, float factor)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(sl_bf2, bf16_pair), factor, SEL);
}

// The same of a pair of bf16: each half's magnitude.
SL_DEV unsigned sl_pair_max(unsigned a, unsigned b)
{
    typedef unsigned short us2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
}

// Eight consecutive elements of a dense matrix as they lie in memory, of which the first n exist (n <= 0: none); the
// others are zero.  The address is aligned to the element only, which a 16-byte access of this target may be.
template <bool B16>
struct SlOctet {
    unsigned w[B16 ? 4 : 8];

    SL_DEV void load(const void *src, long long at, int n)
    {
        typedef unsigned u4a __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
        for (int i = 0; i < (B16 ? 4 : 8); ++i) w[i] = 0;
        if constexpr (B16) {
            const unsigned short *p = static_cast<const unsigned short *>(src) + at;
            if (n >= 8) {
                const sl_u4 v = __builtin_nontemporal_load(reinterpret_cast<const u4a *>(p));
                w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
            } else {
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (i < n) w[i >> 1] |= (unsigned)p[i] << (16 * (i & 1));
            }
        } else {
            const unsigned *p = static_cast<const unsigned *>(src) + at;
            if (n >= 8) {
                // (without the streaming hint: a line's second half is asked for by the second load; 50,257 x 2048 103 us with it, 91 so)
                const sl_u4 u = *reinterpret_cast<const u4a *>(p);
                const sl_u4 v = *reinterpret_cast<const u4a *>(p + 4);
                w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w, w[4] = v.x, w[5] = v.y, w[6] = v.z, w[7] = v.w;
            } else {
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (i < n) w[i] = p[i];
            }
        }
    }
    SL_DEV float value(int i) const
    {
        if constexpr (B16) return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
        else return __uint_as_float(w[i]);
    }
    // fp32 bits of the largest magnitude
    SL_DEV unsigned top() const
    {
        if constexpr (B16) {
            unsigned t = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) t = sl_pair_max(t, w[i] & 0x7FFF7FFFu);
            return max(t << 16, t & 0xFFFF0000u);
        } else {
            unsigned t = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) t = max(t, w[i] & 0x7FFFFFFFu);
            return t;
        }
    }
    SL_DEV unsigned pack(unsigned x) const
    {
        const float f = sl_mx4_factor(x);
        unsigned o = 0;
        if constexpr (B16) {
            o = sl_mx4_pair<0>(o, w[0], f), o = sl_mx4_pair<1>(o, w[1], f);
            o = sl_mx4_pair<2>(o, w[2], f), o = sl_mx4_pair<3>(o, w[3], f);
        } else {
            o = sl_mx4_pair<0>(o, __uint_as_float(w[0]), __uint_as_float(w[1]), f);
            o = sl_mx4_pair<1>(o, __uint_as_float(w[2]), __uint_as_float(w[3]), f);
            o = sl_mx4_pair<2>(o, __uint_as_float(w[4]), __uint_as_float(w[5]), f);
            o = sl_mx4_pair<3>(o, __uint_as_float(w[6]), __uint_as_float(w[7]), f);
        }
        return x == 255u ? 0u : o;
    }
};

// Maximum over the four lanes of a quad.
SL_DEV unsigned sl_quad_max(unsigned v)
{
    v = max(v, (unsigned)sl_dpp<SL_DPP_XOR1>((int)v));
    return max(v, (unsigned)sl_dpp<SL_DPP_XOR2>((int)v));
}

// Blocks of two columns: e[i] holds row i's elements of both in bf16; w their codes, x their scale bytes.
SL_DEV void sl_mx4_columns(const unsigned (&e)[32], sl_u4 (&w)[2], unsigned (&x)[2])
{
    unsigned t = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) t = sl_pair_max(t, e[i] & 0x7FFF7FFFu);
    x[0] = sl_mx4_scale(t << 16), x[1] = sl_mx4_scale(t & 0xFFFF0000u);
    const float f0 = sl_mx4_factor(x[0]), f1 = sl_mx4_factor(x[1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned o0 = 0, o1 = 0;
#define SL_PAIR(J)                                                                       \
    o0 = sl_mx4_pair<J>(o0, __builtin_amdgcn_perm(e[8 * i + 2 * J + 1], e[8 * i + 2 * J], 0x05040100u), f0); \
    o1 = sl_mx4_pair<J>(o1, __builtin_amdgcn_perm(e[8 * i + 2 * J + 1], e[8 * i + 2 * J], 0x07060302u), f1);
        SL_PAIR(0) SL_PAIR(1) SL_PAIR(2) SL_PAIR(3)
#undef SL_PAIR
        w[0][i] = x[0] == 255u ? 0u : o0, w[1][i] = x[1] == 255u ? 0u : o1;
    }
}

// fp32 to bf16, to nearest, ties to even (the conversion instruction of this target).
SL_DEV unsigned sl_bf16_bits(float x) { return (unsigned)__builtin_bit_cast(unsigned short, (__bf16)x); }
SL_DEV unsigned sl_bf16_pair(float a, float b)
{
    const sl_bf2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(unsigned, v);
}
