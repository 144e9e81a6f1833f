// Products of microscaled 4-bit matrices, c = a b^T.
#include <type_traits>

#include "sl_internal.h"
#include "sl_mx4.h"

int slk_mx4_quantize(const void *src, int type, long long rows, long long cols, long long ld, unsigned char *q, unsigned char *qt,
                     hipStream_t st);

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

struct ProductArgs {
    const unsigned char *a, *b;
    long long a_tiles, b_tiles;          // row tiles of 32
    long long k_tiles;                   // column tiles of 128
    long long a_scales, b_scales;        // byte offsets
    long long m, n;
    long long m_tiles, n_tiles;          // tiles of c
    void *c;
    long long ldc;
    int accumulate;
};

typedef float sl_f16 __attribute__((ext_vector_type(16)));

// One step of 64 of the contraction for a tile of 32 x 32: row i of the result is b's row i, column j a's row j; lane l
// has column l % 32 and of it the rows 8 g + 4 (l / 32) + e, g, e = 0 .. 3, at 4 g + e.
// (Of the two shapes of the instruction this one is fed with half the instructions: nothing but products on random
// operands in registers, one / two / four waves per SIMD, PFLOP/s: 32 x 32 x 64 5.9 / 6.6 / 6.7, 16 x 16 x 128 4.3 / 5.2 / 6.1.)
template <int OB, int OA>
SL_DEV sl_f16 mx4_step(sl_u4 b, sl_u4 a, sl_f16 c, unsigned sb, unsigned sa)
{
    const v8i x = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0}, y = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, OB, (int)sb, OA, (int)sa);
}

// Eight consecutive columns of a row of c.
template <bool B16>
SL_DEV void store_octet(const ProductArgs &A, long long row, long long col, sl_f4 lo, sl_f4 hi)
{
    const int n = (int)max(min(A.n - col, 8ll), 0ll);
    const long long at = row * A.ldc + col;
    const float e[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    if constexpr (B16) {
        typedef unsigned u4a __attribute__((ext_vector_type(4), aligned(2)));
        unsigned short *c = static_cast<unsigned short *>(A.c) + at;
        const sl_u4 w = {sl_bf16_pair(e[0], e[1]), sl_bf16_pair(e[2], e[3]), sl_bf16_pair(e[4], e[5]), sl_bf16_pair(e[6], e[7])};
        if (n >= 8) {
            *reinterpret_cast<u4a *>(c) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < n) c[i] = (unsigned short)(w[i >> 1] >> (16 * (i & 1)));
        }
    } else {
        typedef float f4a __attribute__((ext_vector_type(4), aligned(4)));
        float *c = static_cast<float *>(A.c) + at;
        if (n >= 8) {
            f4a *p = reinterpret_cast<f4a *>(c);
            p[0] = A.accumulate ? (sl_f4)(p[0] + lo) : lo;
            p[1] = A.accumulate ? (sl_f4)(p[1] + hi) : hi;
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < n) c[i] = A.accumulate ? c[i] + e[i] : e[i];
        }
    }
}

// ---- large products ----

// Which tile of c workgroup i of `tiles` takes: workgroups reach the eight XCDs in turn, and each XCD is given a run of
// consecutive places of an order that walks bands of eight tile rows column by column, so that the 32 tiles an XCD works on
// together share eight tiles' rows of a and four of b in its L2.
struct TilePlace { long long m, n; };
SL_DEV TilePlace tile_place(unsigned i, unsigned tiles, long long m_tiles, long long n_tiles)
{
    const unsigned xcd = i & 7u, per = tiles >> 3, rest = tiles & 7u;
    const unsigned at = xcd * per + min(xcd, rest) + (i >> 3);
    const unsigned band_size = 8u * (unsigned)n_tiles, band = at / band_size, in = at % band_size;
    const unsigned rows = min(8u, (unsigned)m_tiles - band * 8u);
    return TilePlace{(long long)(band * 8u + in % rows), (long long)(in / rows)};
}

// 16 (scales: the same) bytes per lane from memory to LDS at `lds` + 16 * lane, past the registers.  The instruction is
// written out because the compiler, which cannot tell the stages apart, would wait for all of them before every read
// of LDS; it has no result in a register, the waits for it are
// written out too, and nothing else in these kernels uses m0.
SL_DEV void dma16(const unsigned char *base, unsigned lane_off, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(lane_off), "s"(base) : "memory");
}
template <int N>
SL_DEV void wait_dma() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// All waves' reads of LDS are done and have arrived.
SL_DEV void stage_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Four waves, 2 x 2, TM x TN tiles of 32 x 32 each: 64 TM x 64 TN of c in a workgroup.  Per step of 128 of the
// contraction a stage of LDS holds the workgroup's operands as they lie in memory - an operand is what a wave reads in lane
// order - and four stages are filled ahead; a wave's operands of the next step are read into registers while the matrix unit works
// on this one's.
// Row i of a result's tile is not b's row i: i = 8 g + 4 q + e takes 16 (g / 2) + 8 q + 4 (g % 2) + e, so that a lane has
// eight consecutive columns of c twice and writes them 16 bytes (bf16) at a time.
template <bool B16, int TM, int TN>
__global__ void __launch_bounds__(256, 2) k_product(ProductArgs A)
{
    constexpr int CODES = (2 * TM + 2 * TN) * MX_TILE_BYTES, STAGE = CODES + 2048, STAGES = 4;
    constexpr int PER_WAVE = TM + TN, D = PER_WAVE + 1;             // loads of a wave per stage, 1 KB each
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), wm = wave >> 1, wn = wave & 1;
    const TilePlace at = tile_place(blockIdx.x, gridDim.x, A.m_tiles, A.n_tiles);
    const long long i0 = at.m * (2 * TM), j0 = at.n * (2 * TN);     // row tiles of a and b
    const int steps = (int)A.k_tiles;
    const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char *)lds;

    const unsigned char *src[PER_WAVE];
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
        const int half = wave + 4 * i, t = half >> 1;
        src[i] = (t < 2 * TM ? A.a + min(i0 + t, A.a_tiles - 1) * A.k_tiles * MX_TILE_BYTES
                             : A.b + min(j0 + t - 2 * TM, A.b_tiles - 1) * A.k_tiles * MX_TILE_BYTES) + (half & 1) * 1024;
    }
    // even waves bring a's scales, odd ones b's: up to four tiles of 64 rows, 16 lanes each
    const unsigned char *scales = wave & 1 ? A.b + A.b_scales : A.a + A.a_scales;
    const long long group0 = (wave & 1 ? j0 : i0) >> 1, groups = ((wave & 1 ? A.b_tiles : A.a_tiles) + 1) >> 1;
    scales += min(group0, groups - 1) * A.k_tiles * MX_SCALE_TILE_BYTES;
    const unsigned scale_off = (unsigned)((min(group0 + (lane >> 4), groups - 1) - min(group0, groups - 1)) * A.k_tiles * MX_SCALE_TILE_BYTES) + (lane & 15) * 16;

    // (past the last step it brings that one again, so that every step waits for the same number of loads)
    auto fill = [&](int at) __attribute__((always_inline)) {
        const unsigned to = lds0 + (unsigned)(at & (STAGES - 1)) * STAGE;
        const long long s = min(at, steps - 1);
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) dma16(src[i] + s * MX_TILE_BYTES, lane * 16, to + (wave + 4 * i) * 1024);
        dma16(scales + s * MX_SCALE_TILE_BYTES, scale_off, to + CODES + (wave & 1) * 1024);
    };

    // b's row that this lane has in a tile
    const int i = lane & 31, r = 16 * (i >> 4) + 8 * (i >> 2 & 1) + 4 * (i >> 3 & 1) + (i & 3);
    const int b_off = (lane >> 5) * 512 + r * 16, b_scale = (lane >> 5) * 128 + r * 4;

    sl_u4 a[2][TM][2], b[2][TN][2];
    unsigned sa[2][TM / 2], sb[2][TN / 2];
    constexpr int READS = TM / 2 + TN / 2 + 2 * (TM + TN);
    auto read = [&](int s, auto set) __attribute__((always_inline)) {
        constexpr int S = decltype(set)::value;
        const unsigned char *st = lds + (s & (STAGES - 1)) * STAGE;
#pragma unroll
        for (int t = 0; t < TM / 2; ++t) sa[S][t] = *reinterpret_cast<const unsigned *>(st + CODES + (wm * (TM / 2) + t) * 256 + lane * 4);
#pragma unroll
        for (int t = 0; t < TN / 2; ++t) sb[S][t] = *reinterpret_cast<const unsigned *>(st + CODES + 1024 + (wn * (TN / 2) + t) * 256 + b_scale);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int t = 0; t < TN; ++t) b[S][t][h] = *reinterpret_cast<const sl_u4 *>(st + (2 * TM + wn * TN + t) * MX_TILE_BYTES + h * 1024 + b_off);
#pragma unroll
            for (int t = 0; t < TM; ++t) a[S][t][h] = *reinterpret_cast<const sl_u4 *>(st + (wm * TM + t) * MX_TILE_BYTES + h * 1024 + lane * 16);
        }
    };
    sl_f16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    auto multiply = [&](auto set) __attribute__((always_inline)) {
        constexpr int S = decltype(set)::value;
        // (the byte of a scale word that an operand takes is part of the instruction)
#define MX4_AT(H, I, J) \
    if constexpr (I < TM && J < TN) \
        acc[I][J] = mx4_step<2 * (J & 1) + H, 2 * (I & 1) + H>(b[S][J][H], a[S][I][H], acc[I][J], sb[S][J >> 1], sa[S][I >> 1]);
#define MX4_ROW(H, I) MX4_AT(H, I, 0) MX4_AT(H, I, 1) MX4_AT(H, I, 2) MX4_AT(H, I, 3)
#define MX4_HALF(H) MX4_ROW(H, 0) MX4_ROW(H, 1) MX4_ROW(H, 2) MX4_ROW(H, 3)
        MX4_HALF(0) MX4_HALF(1)
#undef MX4_HALF
#undef MX4_ROW
#undef MX4_AT
    };
    // The next step's operands into registers, this one's into the matrix unit.  Between the two barriers of the scheduler
    // reads of LDS and products alternate; without them the compiler moves the products behind the next step's reads.
    auto step = [&](int s, auto set) __attribute__((always_inline)) {
        constexpr int S = decltype(set)::value;
        wait_dma<2 * D>();
        stage_barrier();
        fill(s + 4);
        __builtin_amdgcn_sched_barrier(0);
        read(s + 1, std::integral_constant<int, 1 - S>{});
        multiply(set);
        constexpr int PRODUCTS = 2 * TM * TN, EACH = (READS + PRODUCTS - 1) / PRODUCTS;
#pragma unroll
        for (int i = 0; i < PRODUCTS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);   // reads of LDS
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);      // products
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    if (steps > 0) {
#pragma unroll
        for (int s = 0; s < STAGES; ++s) fill(s);
        wait_dma<3 * D>();
        stage_barrier();
        read(0, std::integral_constant<int, 0>{});
        __builtin_amdgcn_sched_barrier(0);
        int s = 0;
#pragma unroll 1
        for (; s + 1 < steps; s += 2) {
            step(s, std::integral_constant<int, 0>{});
            step(s + 1, std::integral_constant<int, 1>{});
        }
        if (s < steps) multiply(std::integral_constant<int, 0>{});
        wait_dma<0>();               // (nothing may arrive in LDS that another workgroup has been given)
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const long long row = (i0 + wm * TM + i) * MX_ROWS + (lane & 31);
        if (row >= A.m) continue;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const sl_f16 v = acc[i][j];
                store_octet<B16>(A, row, (j0 + wn * TN + j) * MX_ROWS + 16 * p + (lane >> 5) * 8,
                                 sl_f4{v[8 * p], v[8 * p + 1], v[8 * p + 2], v[8 * p + 3]},
                                 sl_f4{v[8 * p + 4], v[8 * p + 5], v[8 * p + 6], v[8 * p + 7]});
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

const int64_t LONGEST = (int64_t)1 << 40;

// (with m n <= 2^36 and at most 2^29 rows each, tiles of 128 x 128 are less than 2^24)
bool bad_sizes(int64_t m, int64_t n, int64_t k)
{
    if (m < 0 || n < 0 || k < 0) return true;
    if (m == 0 || n == 0) return false;
    SlMx4Shape s;
    return m > ((int64_t)1 << 36) / n || !sl_mx4_shape(m, k > 0 ? k : 1, s) || !sl_mx4_shape(n, k > 0 ? k : 1, s);
}

template <bool B16, int TM, int TN>
void launch_tiles(ProductArgs A, hipStream_t st)
{
    A.m_tiles = (A.m + 64 * TM - 1) / (64 * TM);
    A.n_tiles = (A.n + 64 * TN - 1) / (64 * TN);
    constexpr unsigned bytes = 4 * ((2 * TM + 2 * TN) * MX_TILE_BYTES + 2048);
    static const hipError_t allowed = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_product<B16, TM, TN>),
                                                          hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    (void)allowed;
    hipLaunchKernelGGL((k_product<B16, TM, TN>), dim3((unsigned)(A.m_tiles * A.n_tiles)), dim3(256), bytes, st, A);
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
    if (type == SL_TYPE_BF16) launch_tiles<true, 2, 2>(A, st);
    else launch_tiles<false, 2, 2>(A, st);
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
