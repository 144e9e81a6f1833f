// Layout of the microscaled 4-bit matrices (include/sparseloco.h) and the conversions to and from them.
//
// The layout is that of the matrix unit's operands: in the 16 x 16 x 128 product of 4-bit operands lane l holds block
// l / 16 of row l % 16 - 16 bytes - and one byte of a register gives the block's scale.  A tile of 16 rows x 128
// columns is therefore 1 KB that a wave loads in lane order, and the scale tile of 64 rows is one word per lane
// whose four bytes serve four such tiles.
#pragma once
#include "sl_device.h"

enum { MX_ROWS = 16, MX_COLS = 128, MX_BLOCK = 32, MX_TILE_BYTES = 1024, MX_SCALE_ROWS = 64, MX_SCALE_TILE_BYTES = 256,
       MX_MOST_TILES = 1 << 25 };      // (a grid has less than 2^32 threads)

struct SlMx4Shape {
    long long rows, cols;
    long long row_tiles;        // tiles of 16 rows
    long long col_tiles;        // tiles of 128 columns
    long long scales;           // byte offset of the scales
    long long bytes;
};

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

// 32 elements to 16 bytes (the conversion divides by the factor, rounds to nearest even and cuts off above 6).
SL_DEV sl_u4 sl_mx4_pack(const float (&v)[32], unsigned x)
{
    sl_u4 w = {0, 0, 0, 0};
    if (x == 255u) return w;
    const float f = sl_mx4_factor(x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned o = 0;
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * i + 0], v[8 * i + 1], f, 0);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * i + 2], v[8 * i + 3], f, 1);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * i + 4], v[8 * i + 5], f, 2);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * i + 6], v[8 * i + 7], f, 3);
        w[i] = o;
    }
    return w;
}

SL_DEV unsigned sl_mx4_top(const float (&v)[32])
{
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return top;
}

template <bool B16>
SL_DEV float sl_dense_at(const void *p, long long i)
{
    if constexpr (B16) return __uint_as_float((unsigned)static_cast<const unsigned short *>(p)[i] << 16);
    else return static_cast<const float *>(p)[i];
}

// fp32 to bf16, to nearest, ties to even; NaN stays NaN.
SL_DEV unsigned sl_bf16_bits(float x)
{
    const unsigned b = __float_as_uint(x);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return (b >> 16) | 0x40u;
    return (b + 0x7FFFu + ((b >> 16) & 1u)) >> 16;
}
