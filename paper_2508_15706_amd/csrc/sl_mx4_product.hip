// Products of microscaled 4-bit matrices, c = a b^T.
#include "sl_internal.h"
#include "sl_mx4.h"

int slk_mx4_quantize(const void *src, int type, long long rows, long long cols, long long ld, unsigned char *q, unsigned char *qt,
                     hipStream_t st);

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

struct ProductArgs {
    const unsigned char *a, *b;
    long long a_tiles, b_tiles;          // row tiles of 16
    long long k_tiles;                   // column tiles of 128
    long long a_scales, b_scales;        // byte offsets
    long long m, n;
    long long n_tiles;                   // tiles of c in a row of them
    void *c;
    long long ldc;
    int accumulate;
};

// One step of 128 of the contraction for a tile of 16 x 16: row i of the result is b's row i, column j a's row j.
template <int OB, int OA>
SL_DEV sl_f4 mx4_step(sl_u4 b, sl_u4 a, sl_f4 c, unsigned sb, unsigned sa)
{
    const v8i x = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0}, y = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, OB, (int)sb, OA, (int)sa);
}

template <bool B16>
SL_DEV void store_c(const ProductArgs &A, long long i, long long j, float v)
{
    if (i >= A.m || j >= A.n) return;
    const long long at = i * A.ldc + j;
    if constexpr (B16) {
        static_cast<unsigned short *>(A.c)[at] = (unsigned short)sl_bf16_bits(v);
    } else {
        float *c = static_cast<float *>(A.c) + at;
        *c = A.accumulate ? *c + v : v;
    }
}

// 128 x 128 of c in a workgroup, 64 x 64 in a wave, operands straight from memory.  Tiles past the end are read
// at the last one and not stored.
template <bool B16>
__global__ void __launch_bounds__(256) k_product(ProductArgs A)
{
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6));
    const long long i0 = blockIdx.x / A.n_tiles * 8 + (wave >> 1) * 4, j0 = blockIdx.x % A.n_tiles * 8 + (wave & 1) * 4;
    const unsigned char *pa[4], *pb[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        pa[t] = A.a + min(i0 + t, A.a_tiles - 1) * A.k_tiles * MX_TILE_BYTES + lane * 16;
        pb[t] = A.b + min(j0 + t, A.b_tiles - 1) * A.k_tiles * MX_TILE_BYTES + lane * 16;
    }
    const unsigned char *qa = A.a + A.a_scales + min(i0, A.a_tiles - 1) / 4 * A.k_tiles * MX_SCALE_TILE_BYTES + lane * 4;
    const unsigned char *qb = A.b + A.b_scales + min(j0, A.b_tiles - 1) / 4 * A.k_tiles * MX_SCALE_TILE_BYTES + lane * 4;
    sl_f4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = sl_f4{0.f, 0.f, 0.f, 0.f};
    for (long long k = 0; k < A.k_tiles; ++k) {
        sl_u4 a[4], b[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            a[t] = *reinterpret_cast<const sl_u4 *>(pa[t] + k * MX_TILE_BYTES);
            b[t] = *reinterpret_cast<const sl_u4 *>(pb[t] + k * MX_TILE_BYTES);
        }
        const unsigned sa = *reinterpret_cast<const unsigned *>(qa + k * MX_SCALE_TILE_BYTES);
        const unsigned sb = *reinterpret_cast<const unsigned *>(qb + k * MX_SCALE_TILE_BYTES);
#define MX4_ROW(I)                                              \
    acc[I][0] = mx4_step<0, I>(b[0], a[I], acc[I][0], sb, sa);  \
    acc[I][1] = mx4_step<1, I>(b[1], a[I], acc[I][1], sb, sa);  \
    acc[I][2] = mx4_step<2, I>(b[2], a[I], acc[I][2], sb, sa);  \
    acc[I][3] = mx4_step<3, I>(b[3], a[I], acc[I][3], sb, sa);
        MX4_ROW(0) MX4_ROW(1) MX4_ROW(2) MX4_ROW(3)
#undef MX4_ROW
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                store_c<B16>(A, (i0 + i) * 16 + (lane & 15), (j0 + j) * 16 + (lane >> 4) * 4 + e, acc[i][j][e]);
}

int check_launch()
{
    const hipError_t err = hipGetLastError();
    if (err == hipSuccess) return SL_OK;
    sl_note_hip_error(err);
    return SL_ERR_HIP;
}

bool misaligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

const int64_t LONGEST = (int64_t)1 << 40;

// (with m n <= 2^36 and at most 2^29 rows each, tiles of 128 x 128 are less than 2^24)
bool bad_sizes(int64_t m, int64_t n, int64_t k)
{
    if (m < 0 || n < 0 || k < 0) return true;
    if (m == 0 || n == 0) return false;
    SlMx4Shape s;
    return m > ((int64_t)1 << 36) / n || !sl_mx4_shape(m, k > 0 ? k : 1, s) || !sl_mx4_shape(n, k > 0 ? k : 1, s);
}

int product(const unsigned char *a, const unsigned char *b, int64_t m, int64_t n, int64_t k, void *c, int type, int64_t ldc,
            int accumulate, hipStream_t st)
{
    ProductArgs A;
    SlMx4Shape sa = {}, sb = {};
    if (k > 0) {
        (void)sl_mx4_shape(m, k, sa);
        (void)sl_mx4_shape(n, k, sb);
    }
    A.a = a, A.b = b;
    A.a_tiles = sa.row_tiles, A.b_tiles = sb.row_tiles, A.k_tiles = k > 0 ? sa.col_tiles : 0;
    A.a_scales = sa.scales, A.b_scales = sb.scales;
    A.m = m, A.n = n, A.c = c, A.ldc = ldc, A.accumulate = accumulate;
    A.n_tiles = (n + 127) / 128;
    const dim3 grid((unsigned)(A.n_tiles * ((m + 127) / 128)));
    hipLaunchKernelGGL(type == SL_TYPE_BF16 ? k_product<true> : k_product<false>, grid, dim3(256), 0, st, A);
    return check_launch();
}

}  // namespace

extern "C" {

size_t sl_mx4_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (bad_sizes(m, n, k) || m == 0 || n == 0 || k == 0) return 0;
    return sl_mx4_bytes(m, k);
}

int sl_mx4_product(const void *a, const void *b, int64_t m, int64_t n, int64_t k, void *c, int c_type, int64_t ldc,
                   int accumulate, void *workspace, void *stream)
{
    if (bad_sizes(m, n, k) || (c_type != SL_TYPE_F32 && c_type != SL_TYPE_BF16) || (accumulate && c_type != SL_TYPE_F32))
        return SL_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return SL_OK;
    if (!c || (k > 0 && (!a || !b)) || c == a || c == b || ldc < n || ldc > LONGEST) return SL_ERR_INVALID_ARG;
    if (misaligned(a, 16) || misaligned(b, 16) || misaligned(c, c_type == SL_TYPE_BF16 ? 2 : 4) || misaligned(workspace, 16))
        return SL_ERR_INVALID_ARG;
    if (!workspace && sl_mx4_workspace_bytes(m, n, k)) return SL_ERR_INVALID_ARG;
    return product(static_cast<const unsigned char *>(a), static_cast<const unsigned char *>(b), m, n, k, c, c_type, ldc,
                   accumulate, static_cast<hipStream_t>(stream));
}

int sl_mx4_linear(const void *x, int x_type, int64_t ldx, const void *w, int64_t m, int64_t n, int64_t k, void *y,
                  int y_type, int64_t ldy, void *workspace, void *stream)
{
    if (bad_sizes(m, n, k) || (x_type != SL_TYPE_F32 && x_type != SL_TYPE_BF16) || (y_type != SL_TYPE_F32 && y_type != SL_TYPE_BF16))
        return SL_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return SL_OK;
    if (!y || (k > 0 && (!x || !w)) || y == x || y == w || ldy < n || ldy > LONGEST || ldx < k || ldx > LONGEST) return SL_ERR_INVALID_ARG;
    if (misaligned(x, x_type == SL_TYPE_BF16 ? 2 : 4) || misaligned(w, 16) || misaligned(y, y_type == SL_TYPE_BF16 ? 2 : 4) ||
        misaligned(workspace, 16))
        return SL_ERR_INVALID_ARG;
    if (!workspace && sl_mx4_workspace_bytes(m, n, k)) return SL_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char *q = static_cast<unsigned char *>(workspace);
    if (k > 0)
        if (const int rc = slk_mx4_quantize(x, x_type, m, k, ldx, q, nullptr, st)) return rc;
    return product(q, static_cast<const unsigned char *>(w), m, n, k, y, y_type, ldy, 0, st);
}

}  // extern "C"
