// Dense matrices to microscaled 4 bits and back.
#include "sl_internal.h"
#include "sl_mx4.h"

namespace {

struct QuantArgs {
    const void *src;
    long long rows, cols, ld;        // of src
    unsigned char *q;
    long long row_tiles, col_tiles, scales;   // of q
    long long groups;                // row tiles and what fills up the last scale tile
};

// A wave per tile of 16 rows x 128 columns of q: lane l has block l / 16 of row l % 16 to itself.  T: q is the
// transposed matrix, its rows are src's columns.
template <bool B16, bool T>
__global__ void __launch_bounds__(256) k_quantize(QuantArgs A)
{
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6));
    const long long tile = (long long)blockIdx.x * 4 + wave;
    if (tile >= A.groups * A.col_tiles) return;
    const long long rt = tile / A.col_tiles, kt = tile % A.col_tiles;
    const long long row = rt * MX_ROWS + (lane & 15), col = kt * MX_COLS + (lane >> 4) * MX_BLOCK;
    const long long n_rows = T ? A.cols : A.rows, n_cols = T ? A.rows : A.cols;
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        v[i] = 0.0f;
        if (row < n_rows && col + i < n_cols) v[i] = sl_dense_at<B16>(A.src, T ? (col + i) * A.ld + row : row * A.ld + col + i);
    }
    const unsigned x = sl_mx4_scale(sl_mx4_top(v));
    if (rt < A.row_tiles)
        *reinterpret_cast<sl_u4 *>(A.q + tile * MX_TILE_BYTES + lane * 16) = sl_mx4_pack(v, x);
    A.q[A.scales + ((rt >> 2) * A.col_tiles + kt) * MX_SCALE_TILE_BYTES + lane * 4 + (rt & 3)] = (unsigned char)x;
}

// A lane per block again.
template <bool B16>
__global__ void __launch_bounds__(256) k_dequantize(const unsigned char *q, SlMx4Shape s, void *out, long long ld)
{
    const float grid[8] = {0.0f, 0.5f, 1.0f, 1.5f, 2.0f, 3.0f, 4.0f, 6.0f};
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6));
    const long long tile = (long long)blockIdx.x * 4 + wave;
    if (tile >= s.row_tiles * s.col_tiles) return;
    const long long rt = tile / s.col_tiles, kt = tile % s.col_tiles;
    const long long row = rt * MX_ROWS + (lane & 15), col = kt * MX_COLS + (lane >> 4) * MX_BLOCK;
    if (row >= s.rows) return;
    const sl_u4 w = *reinterpret_cast<const sl_u4 *>(q + tile * MX_TILE_BYTES + lane * 16);
    const float f = sl_mx4_factor(q[s.scales + ((rt >> 2) * s.col_tiles + kt) * MX_SCALE_TILE_BYTES + lane * 4 + (rt & 3)]);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        if (col + i >= s.cols) return;
        const unsigned c = w[i >> 3] >> (4 * (i & 7)) & 15u;
        float x = grid[c & 7u] * f;
        if (c & 8u) x = -x;
        const long long at = row * ld + col + i;
        if constexpr (B16) static_cast<unsigned short *>(out)[at] = (unsigned short)sl_bf16_bits(x);
        else static_cast<float *>(out)[at] = x;
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

template <bool T>
int quantize(const void *src, int type, long long rows, long long cols, long long ld, unsigned char *q, hipStream_t st)
{
    SlMx4Shape s;
    if (!sl_mx4_shape(T ? cols : rows, T ? rows : cols, s)) return SL_ERR_INVALID_ARG;
    QuantArgs A;
    A.src = src, A.rows = rows, A.cols = cols, A.ld = ld, A.q = q;
    A.row_tiles = s.row_tiles, A.col_tiles = s.col_tiles, A.scales = s.scales;
    A.groups = (s.row_tiles + 3) / 4 * 4;
    const dim3 grid((unsigned)((A.groups * A.col_tiles + 3) / 4));
    hipLaunchKernelGGL((type == SL_TYPE_BF16 ? k_quantize<true, T> : k_quantize<false, T>), grid, dim3(256), 0, st, A);
    return check_launch();
}

}  // namespace

int slk_mx4_quantize(const void *src, int type, long long rows, long long cols, long long ld, unsigned char *q, unsigned char *qt,
                     hipStream_t st)
{
    if (q)
        if (const int rc = quantize<false>(src, type, rows, cols, ld, q, st)) return rc;
    if (qt)
        if (const int rc = quantize<true>(src, type, rows, cols, ld, qt, st)) return rc;
    return SL_OK;
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
    if (!src || (!q && !qt) || q == qt || q == src || qt == src || !sl_mx4_shape(rows, cols, s)) return SL_ERR_INVALID_ARG;
    if (src_type != SL_TYPE_F32 && src_type != SL_TYPE_BF16) return SL_ERR_INVALID_ARG;
    if (ld < cols || ld > ((int64_t)1 << 40) || misaligned(q, 16) || misaligned(qt, 16) || misaligned(src, src_type == SL_TYPE_BF16 ? 2 : 4))
        return SL_ERR_INVALID_ARG;
    return slk_mx4_quantize(src, src_type, rows, cols, ld, static_cast<unsigned char *>(q), static_cast<unsigned char *>(qt),
                            static_cast<hipStream_t>(stream));
}

int sl_mx4_dequantize(const void *q, int64_t rows, int64_t cols, void *out, int out_type, int64_t ld, void *stream)
{
    SlMx4Shape s;
    if (!q || !out || q == out || !sl_mx4_shape(rows, cols, s)) return SL_ERR_INVALID_ARG;
    if (out_type != SL_TYPE_F32 && out_type != SL_TYPE_BF16) return SL_ERR_INVALID_ARG;
    if (ld < cols || ld > ((int64_t)1 << 40) || misaligned(q, 16) || misaligned(out, out_type == SL_TYPE_BF16 ? 2 : 4)) return SL_ERR_INVALID_ARG;
    const dim3 grid((unsigned)((s.row_tiles * s.col_tiles + 3) / 4));
    hipLaunchKernelGGL(out_type == SL_TYPE_BF16 ? k_dequantize<true> : k_dequantize<false>, grid, dim3(256), 0,
                       static_cast<hipStream_t>(stream), static_cast<const unsigned char *>(q), s, out, (long long)ld);
    return check_launch();
}

}  // extern "C"
