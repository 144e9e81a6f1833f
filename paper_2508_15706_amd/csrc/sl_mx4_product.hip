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
    long long a_tiles, b_tiles;          // row tiles of 16
    long long k_tiles;                   // column tiles of 128
    long long a_scales, b_scales;        // byte offsets
    long long m, n;
    long long m_tiles, n_tiles;          // tiles of c
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

// Four waves, 2 x 2, TM x TN tiles of 16 x 16 each: 32 TM x 32 TN of c in a workgroup.  Per step of 128 of the
// contraction a stage of LDS holds the workgroup's operands as they lie in memory - a tile is what a wave reads in lane order -
// and four stages are filled ahead; a wave's operands of the next step are read into registers while the matrix unit works on this one's.
// Row i of the result's tile j is not b's row 16 j + i: of each 32 rows of b, a pair of tiles takes 8 (i / 4) + i % 4 and those 4 on,
// so that a lane has eight consecutive columns of c and writes 16 bytes of bf16 (32 of fp32).
template <bool B16, int TM, int TN>
__global__ void __launch_bounds__(256, TM * TN > 32 ? 1 : 2) k_product(ProductArgs A)
{
    constexpr int CODES = (2 * TM + 2 * TN) * MX_TILE_BYTES, STAGE = CODES + 2048, STAGES = 4;
    constexpr int PER_WAVE = (TM + TN) / 2, D = PER_WAVE + 1;       // loads of a wave per stage
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), wm = wave >> 1, wn = wave & 1;
    const TilePlace at = tile_place(blockIdx.x, gridDim.x, A.m_tiles, A.n_tiles);
    const long long i0 = at.m * (2 * TM), j0 = at.n * (2 * TN);     // row tiles of a and b
    const int steps = (int)A.k_tiles;
    const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char *)lds;

    const unsigned char *src[PER_WAVE];
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
        const int t = wave + 4 * i;
        src[i] = t < 2 * TM ? A.a + min(i0 + t, A.a_tiles - 1) * A.k_tiles * MX_TILE_BYTES
                            : A.b + min(j0 + t - 2 * TM, A.b_tiles - 1) * A.k_tiles * MX_TILE_BYTES;
    }
    // even waves bring a's scales, odd ones b's: up to four tiles of 64 rows, 16 lanes each
    const unsigned char *scales = wave & 1 ? A.b + A.b_scales : A.a + A.a_scales;
    const long long group0 = (wave & 1 ? j0 : i0) >> 2, groups = ((wave & 1 ? A.b_tiles : A.a_tiles) + 3) >> 2;
    scales += min(group0, groups - 1) * A.k_tiles * MX_SCALE_TILE_BYTES;
    const unsigned scale_off = (unsigned)((min(group0 + (lane >> 4), groups - 1) - min(group0, groups - 1)) * A.k_tiles * MX_SCALE_TILE_BYTES) + (lane & 15) * 16;

    // (past the last step it brings that one again, so that every step waits for the same number of loads)
    auto fill = [&](int at) __attribute__((always_inline)) {
        const unsigned to = lds0 + (unsigned)(at & (STAGES - 1)) * STAGE;
        const int s = min(at, steps - 1);
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) dma16(src[i] + (long long)s * MX_TILE_BYTES, lane * 16, to + (wave + 4 * i) * MX_TILE_BYTES);
        dma16(scales + (long long)s * MX_SCALE_TILE_BYTES, scale_off, to + CODES + (wave & 1) * 1024);
    };

    // where in b's 32 rows this lane's row of a tile lies, even and odd tiles
    const int r0 = 8 * ((lane & 15) >> 2) + (lane & 3);
    const int b_off = (r0 >> 4) * MX_TILE_BYTES + (lane >> 4) * 256 + (r0 & 15) * 16;
    const int b_scale = (lane >> 4) * 64 + (r0 & 15) * 4, b_shift = 8 * (r0 >> 4);

    sl_u4 a[2][TM], b[2][TN];
    unsigned sa[2][TM / 4], sb[2][TN / 2];
    auto read = [&](int s, auto set) __attribute__((always_inline)) {
        constexpr int S = decltype(set)::value;
        const unsigned char *st = lds + (s & (STAGES - 1)) * STAGE;
#pragma unroll
        for (int t = 0; t < TM / 4; ++t) sa[S][t] = *reinterpret_cast<const unsigned *>(st + CODES + (wm * (TM / 4) + t) * 256 + lane * 4);
#pragma unroll
        for (int t = 0; t < TN / 2; ++t)
            sb[S][t] = *reinterpret_cast<const unsigned *>(st + CODES + 1024 + (wn * (TN / 4) + t / 2) * 256 + b_scale + (t & 1) * 16);
#pragma unroll
        for (int t = 0; t < TN; ++t)
            b[S][t] = *reinterpret_cast<const sl_u4 *>(st + (2 * TM + wn * TN + (t & ~1)) * MX_TILE_BYTES + b_off + (t & 1) * 64);
#pragma unroll
        for (int t = 0; t < TM; ++t) a[S][t] = *reinterpret_cast<const sl_u4 *>(st + (wm * TM + t) * MX_TILE_BYTES + lane * 16);
    };
    sl_f4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = sl_f4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](auto set) __attribute__((always_inline)) {
        constexpr int S = decltype(set)::value;
        unsigned sbs[TN / 2];
#pragma unroll
        for (int t = 0; t < TN / 2; ++t) sbs[t] = sb[S][t] >> b_shift;
        // (the byte of a scale word that a tile takes is part of the instruction)
        auto row = [&](auto ic) __attribute__((always_inline)) {
            constexpr int I = decltype(ic)::value;
#define MX4_AT(J) \
    if constexpr (J < TN) acc[I][J] = mx4_step<(J & 2), I & 3>(b[S][J], a[S][I], acc[I][J], sbs[(J >> 2) * 2 + (J & 1)], sa[S][I >> 2]);
            MX4_AT(0) MX4_AT(1) MX4_AT(2) MX4_AT(3) MX4_AT(4) MX4_AT(5) MX4_AT(6) MX4_AT(7)
#undef MX4_AT
        };
#define MX4_ROW(I) if constexpr (I < TM) row(std::integral_constant<int, I>{});
        MX4_ROW(0) MX4_ROW(1) MX4_ROW(2) MX4_ROW(3) MX4_ROW(4) MX4_ROW(5) MX4_ROW(6) MX4_ROW(7)
#undef MX4_ROW
    };
    // The next step's operands into registers, this one's into the matrix unit.  Between the two barriers of the scheduler
    // reads of LDS and products alternate; without them the compiler moves the products behind the next step's reads.
    auto body = [&](int s, auto set) __attribute__((always_inline)) {
        constexpr int S = decltype(set)::value;
        read(s + 1, std::integral_constant<int, 1 - S>{});
        multiply(set);
        constexpr int READS = TM / 4 + TN / 2 + TM + TN, EACH = TM * TN / READS;
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);      // LDS
            __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);   // products
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto step = [&](int s, auto set) __attribute__((always_inline)) {
        wait_dma<2 * D>();
        stage_barrier();
        fill(s + 4);
        __builtin_amdgcn_sched_barrier(0);
        body(s, set);
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
        const long long row = (i0 + wm * TM + i) * 16 + (lane & 15);
        if (row >= A.m) continue;
#pragma unroll
        for (int j = 0; j < TN; j += 2) {
            const long long col = (j0 + wn * TN + j) * 16 + (lane >> 4) * 8;
            store_octet<B16>(A, row, col, acc[i][j], acc[i][j + 1]);
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
    A.m_tiles = (A.m + 32 * TM - 1) / (32 * TM);
    A.n_tiles = (A.n + 32 * TN - 1) / (32 * TN);
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
    if (type == SL_TYPE_BF16) launch_tiles<true, 4, 4>(A, st);
    else launch_tiles<false, 4, 4>(A, st);
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
