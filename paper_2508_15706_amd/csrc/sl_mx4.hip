// Dense matrices to microscaled 4 bits and back.
#include "sl_internal.h"
#include "sl_mx4.h"

namespace {

struct QuantArgs {
    const void *src;
    long long rows, cols, ld;
    unsigned char *q, *qt;
    SlMx4Shape s, t;                 // of q and of qt
    long long col_groups;            // workgroups in a row of them
};

// A workgroup takes 128 columns of 128 (bf16) or 64 (fp32) rows, eight consecutive elements of a row in a lane at a
// time, 16 rows per access.
//
// Along the rows (Q) a block is a quad of lanes: its largest magnitude comes by two lane moves, its codes are one word
// a lane, and the 256 threads' words of two accesses are one tile of codes, 2 KB.  The scale bytes of blocks 0 and 2 (1 and
// 3) of a row and of the row 32 on are the word that the first lane of the quad writes.
// Along the columns (QT) the elements pass through LDS as they are; a lane then has 32 rows of two columns (bf16, one
// wave for each block of 32 rows) or of one (fp32, two waves), read row by row without bank conflicts.
template <bool B16, bool Q, bool QT>
__global__ void __launch_bounds__(256) k_quantize(QuantArgs A)
{
    constexpr int ROWS = B16 ? 128 : 64, WORDS = B16 ? 4 : 8;
    __shared__ sl_u4 tile[QT ? ROWS * 16 * WORDS / 4 : 1];
    const int tid = threadIdx.x, octet = tid & 15, sub = tid >> 4;
    const long long rg = blockIdx.x / A.col_groups, kt = blockIdx.x % A.col_groups;
    const long long row0 = rg * ROWS, col = kt * MX_COLS + octet * 8;
    const int n = (int)max(min(A.cols - col, 8ll), 0ll);
    SlOctet<B16> v[ROWS / 16];
#pragma unroll
    for (int i = 0; i < ROWS / 16; ++i) {
        const long long row = row0 + i * 16 + sub;
        v[i].load(A.src, row * A.ld + col, row < A.rows ? n : 0);
    }
    if constexpr (QT) {
#pragma unroll
        for (int i = 0; i < ROWS / 16; ++i)
#pragma unroll
            for (int j = 0; j < WORDS / 4; ++j)
                tile[((i * 16 + sub) * 16 + octet) * (WORDS / 4) + j] = sl_u4{v[i].w[4 * j], v[i].w[4 * j + 1], v[i].w[4 * j + 2], v[i].w[4 * j + 3]};
    }
    if constexpr (Q) {
        const int b = octet >> 2;
#pragma unroll
        for (int i = 0; i < ROWS / 16; i += 4) {
            const long long rt = row0 / MX_ROWS + i / 2;               // row tile of access i; i + 2 begins the next
            unsigned x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = sl_mx4_scale(sl_quad_max(v[i + j].top()));
                const unsigned w = v[i + j].pack(x[j]);
                if (rt + j / 2 < A.s.row_tiles)
                    *reinterpret_cast<unsigned *>(A.q + ((rt + j / 2) * A.s.col_tiles + kt) * MX_TILE_BYTES +
                                                  sl_mx4_code_at((j & 1) * 16 + sub, b) + (octet & 3) * 4) = w;
                x[j] |= (unsigned)sl_dpp<SL_DPP_ROW_ROR8>((int)x[j]) << 8;       // lanes of blocks 0 and 1: those of 2 and 3
            }
            if ((octet & 3) == 0 && octet < 8 && rt < A.s.row_tiles) {
                unsigned *to = reinterpret_cast<unsigned *>(A.q + A.s.scales + (rt / 2 * A.s.col_tiles + kt) * MX_SCALE_TILE_BYTES);
                to[sl_mx4_scale_at(sub, b) / 4] = x[0] | x[2] << 16;
                to[sl_mx4_scale_at(16 + sub, b) / 4] = x[1] | x[3] << 16;
            }
        }
    }
    if constexpr (QT) {
        __syncthreads();
        const unsigned *words = reinterpret_cast<const unsigned *>(tile);
        const int lane = tid & 63, wave = sl_uniform(tid >> 6);
        const long long ct0 = kt * 4, kt2 = row0 / MX_COLS;            // row tiles of qt from here, its column tile
        const int b = B16 ? wave : (int)(row0 / 32 & 3) + (wave >> 1);
        // one column's codes and scale byte
        auto put = [&](int c, sl_u4 w, unsigned x) __attribute__((always_inline)) {
            const long long ct = ct0 + (c >> 5);
            if (ct < A.t.row_tiles)
                *reinterpret_cast<sl_u4 *>(A.qt + (ct * A.t.col_tiles + kt2) * MX_TILE_BYTES + sl_mx4_code_at(c, b)) = w;
            if (ct < (A.t.row_tiles + 1) / 2 * 2)
                A.qt[A.t.scales + (ct / 2 * A.t.col_tiles + kt2) * MX_SCALE_TILE_BYTES + sl_mx4_scale_at(c, b)] = (unsigned char)x;
        };
        if constexpr (B16) {
            unsigned e[32], x[2];
            sl_u4 w[2];
#pragma unroll
            for (int i = 0; i < 32; ++i) e[i] = words[(wave * 32 + i) * 64 + lane];
            sl_mx4_columns(e, w, x);
            put(lane * 2, w[0], x[0]);
            put(lane * 2 + 1, w[1], x[1]);
        } else {
            const int c = (wave & 1) * 64 + lane;
            SlOctet<false> e[4];
            unsigned t = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) e[i >> 3].w[i & 7] = words[((wave >> 1) * 32 + i) * 128 + c];
#pragma unroll
            for (int i = 0; i < 4; ++i) t = max(t, e[i].top());
            const unsigned x = sl_mx4_scale(t);
            put(c, sl_u4{e[0].pack(x), e[1].pack(x), e[2].pack(x), e[3].pack(x)}, x);
        }
    }
}

// Eight elements - a word of codes - in a lane, 512 columns of a row in a wave, 16 rows in a workgroup: rows are written in pieces
// of 1 KB (in pieces of 256 bytes, neighbours meet in the lines at the ends of unaligned ones: 2048 x 50,257 bf16 89 us, so 45).
// HINT: streaming stores, for rows that begin on 16 bytes (50,257 x 2048 53 us without, 38 with).
template <bool B16, bool HINT>
__global__ void __launch_bounds__(256) k_dequantize(const unsigned char *q, SlMx4Shape s, void *out, long long ld, long long col_groups)
{
    typedef unsigned u4a __attribute__((ext_vector_type(4), aligned(2)));
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), b = lane >> 2 & 3;
    const long long row0 = blockIdx.x / col_groups * 16 + wave * 4, col = blockIdx.x % col_groups * 512 + lane * 8;
    const int n = (int)max(min(s.cols - col, 8ll), 0ll);
    const long long kt = min(col / MX_COLS, s.col_tiles - 1);
    unsigned code[4], byte[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long long row = min(row0 + i, s.rows - 1);
        code[i] = *reinterpret_cast<const unsigned *>(q + (row / MX_ROWS * s.col_tiles + kt) * MX_TILE_BYTES + sl_mx4_code_at((int)(row & 31), b) + (lane & 3) * 4);
        byte[i] = q[s.scales + (row / MX_SCALE_ROWS * s.col_tiles + kt) * MX_SCALE_TILE_BYTES + sl_mx4_scale_at((int)(row & 63), b)];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long long row = row0 + i;
        if (row >= s.rows) return;
        const unsigned x = byte[i];
        const float f = sl_mx4_factor(x);
        typedef float f2 __attribute__((ext_vector_type(2)));
        const f2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i], f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i], f, 1);
        const f2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i], f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i], f, 3);
        float e[8] = {p0.x, p0.y, p1.x, p1.y, p2.x, p2.y, p3.x, p3.y};
        if (x == 255u) {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = f;
        }
        const long long at = row * ld + col;
        auto put = [&](void *to, sl_u4 w) __attribute__((always_inline)) {
            if constexpr (HINT) __builtin_nontemporal_store(w, static_cast<sl_u4 *>(to));
            else *static_cast<u4a *>(to) = w;
        };
        if constexpr (B16) {
            unsigned short *o = static_cast<unsigned short *>(out) + at;
            const sl_u4 w = {sl_bf16_pair(e[0], e[1]), sl_bf16_pair(e[2], e[3]), sl_bf16_pair(e[4], e[5]), sl_bf16_pair(e[6], e[7])};
            if (n >= 8) {
                put(o, w);
            } else {
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (j < n) o[j] = (unsigned short)(w[j >> 1] >> (16 * (j & 1)));
            }
        } else {
            float *o = static_cast<float *>(out) + at;
            if (n >= 8) {
                put(o, sl_u4{__float_as_uint(e[0]), __float_as_uint(e[1]), __float_as_uint(e[2]), __float_as_uint(e[3])});
                put(o + 4, sl_u4{__float_as_uint(e[4]), __float_as_uint(e[5]), __float_as_uint(e[6]), __float_as_uint(e[7])});
            } else {
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (j < n) o[j] = e[j];
            }
        }
    }
}

int check_launch()
{
    const hipError_t err = hipGetLastError();
    if (err == hipSuccess) return SL_OK;
    sl_note_hip_error(err);
    return SL_ERR_HIP;
}

bool misaligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

template <bool B16>
void launch(const QuantArgs &A, unsigned groups, hipStream_t st)
{
    if (A.q && A.qt) hipLaunchKernelGGL((k_quantize<B16, true, true>), dim3(groups), dim3(256), 0, st, A);
    else if (A.q) hipLaunchKernelGGL((k_quantize<B16, true, false>), dim3(groups), dim3(256), 0, st, A);
    else hipLaunchKernelGGL((k_quantize<B16, false, true>), dim3(groups), dim3(256), 0, st, A);
}

}  // namespace

int slk_mx4_quantize(const void *src, int type, long long rows, long long cols, long long ld, unsigned char *q, unsigned char *qt,
                     hipStream_t st)
{
    QuantArgs A;
    A.s = A.t = SlMx4Shape{};
    if ((q && !sl_mx4_shape(rows, cols, A.s)) || (qt && !sl_mx4_shape(cols, rows, A.t))) return SL_ERR_INVALID_ARG;
    A.src = src, A.rows = rows, A.cols = cols, A.ld = ld, A.q = q, A.qt = qt;
    A.col_groups = (cols + MX_COLS - 1) / MX_COLS;
    // qt's tiles are 128 of these rows deep and are filled up, also past the last row
    const long long row_groups = type == SL_TYPE_BF16 ? (rows + 127) / 128 : qt ? (rows + 127) / 128 * 2 : (rows + 63) / 64;
    const unsigned groups = (unsigned)(row_groups * A.col_groups);
    if (type == SL_TYPE_BF16) launch<true>(A, groups, st);
    else launch<false>(A, groups, st);
    return check_launch();
}

extern "C" {

size_t sl_mx4_bytes(int64_t rows, int64_t cols)
{
    SlMx4Shape s;
    return sl_mx4_shape(rows, cols, s) ? (size_t)s.bytes : 0;
}

int sl_mx4_quantize(const void *src, int src_type, int64_t rows, int64_t cols, int64_t ld, void *q, void *qt, void *stream)
{
    SlMx4Shape s;
    if (rows < 0 || cols < 0) return SL_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return SL_OK;
    if (!src || (!q && !qt) || q == qt || q == src || qt == src) return SL_ERR_INVALID_ARG;
    if ((q && !sl_mx4_shape(rows, cols, s)) || (qt && !sl_mx4_shape(cols, rows, s))) return SL_ERR_INVALID_ARG;
    if (src_type != SL_TYPE_F32 && src_type != SL_TYPE_BF16) return SL_ERR_INVALID_ARG;
    if (ld < cols || ld > ((int64_t)1 << 40) || misaligned(q, 16) || misaligned(qt, 16) || misaligned(src, src_type == SL_TYPE_BF16 ? 2 : 4))
        return SL_ERR_INVALID_ARG;
    return slk_mx4_quantize(src, src_type, rows, cols, ld, static_cast<unsigned char *>(q), static_cast<unsigned char *>(qt),
                            static_cast<hipStream_t>(stream));
}

int sl_mx4_dequantize(const void *q, int64_t rows, int64_t cols, void *out, int out_type, int64_t ld, void *stream)
{
    SlMx4Shape s;
    if (rows < 0 || cols < 0) return SL_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return SL_OK;
    if (!q || !out || q == out || !sl_mx4_shape(rows, cols, s)) return SL_ERR_INVALID_ARG;
    if (out_type != SL_TYPE_F32 && out_type != SL_TYPE_BF16) return SL_ERR_INVALID_ARG;
    if (ld < cols || ld > ((int64_t)1 << 40) || misaligned(q, 16) || misaligned(out, out_type == SL_TYPE_BF16 ? 2 : 4)) return SL_ERR_INVALID_ARG;
    // (fp32: a lane's two pieces of 16 bytes would go to memory one by one)
    const bool b16 = out_type == SL_TYPE_BF16, hint = b16 && !misaligned(out, 16) && (ld & 7) == 0;
    const long long col_groups = (cols + 511) / 512;
    const dim3 grid((unsigned)((rows + 15) / 16 * col_groups));
    hipLaunchKernelGGL((b16 ? (hint ? k_dequantize<true, true> : k_dequantize<true, false>) : k_dequantize<false, false>), grid, dim3(256), 0,
                       static_cast<hipStream_t>(stream), static_cast<const unsigned char *>(q), s, out, (long long)ld, col_groups);
    return check_launch();
}

}  // extern "C"
