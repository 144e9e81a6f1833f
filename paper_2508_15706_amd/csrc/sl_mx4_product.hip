// Products of microscaled 4-bit matrices, c = a b^T.
#include <algorithm>
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
    long long part_steps, part_size;     // steps of 128 in a part of the contraction, elements between the parts' results
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

// Four columns of a row of an fp32 c; those that do not exist are zero.
SL_DEV sl_f4 load_piece(const ProductArgs &A, long long row, long long col)
{
    typedef float f4a __attribute__((ext_vector_type(4), aligned(4)));
    const long long n = row < A.m ? A.n - col : 0;
    const float *c = static_cast<const float *>(A.c) + row * A.ldc + col;
    sl_f4 v = {0.f, 0.f, 0.f, 0.f};
    if (n >= 4) {
        v = *reinterpret_cast<const f4a *>(c);
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) v[i] = c[i];
    }
    return v;
}

// 16 bytes of a row of c: eight columns of bf16, four of fp32.
template <bool B16>
SL_DEV void store_piece(const ProductArgs &A, unsigned part, long long row, long long col, sl_u4 w)
{
    if (row >= A.m) return;
    const long long at = part * A.part_size + row * A.ldc + col, n = A.n - col;
    if constexpr (B16) {
        typedef unsigned u4a __attribute__((ext_vector_type(4), aligned(2)));
        unsigned short *c = static_cast<unsigned short *>(A.c) + at;
        if (n >= 8) {
            *reinterpret_cast<u4a *>(c) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < n) c[i] = (unsigned short)(w[i >> 1] >> (16 * (i & 1)));
        }
    } else {
        typedef unsigned u4a __attribute__((ext_vector_type(4), aligned(4)));
        unsigned *c = static_cast<unsigned *>(A.c) + at;
        if (n >= 4) {
            *reinterpret_cast<u4a *>(c) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < n) c[i] = w[i];
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
// of LDS; it has no result in a register, and the waits for it are written out too.  (m0 is the compiler's own, which warns that it will not
// be kept: that is what the list of clobbers is to say.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
SL_DEV void dma16(const unsigned char *base, unsigned lane_off, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(lane_off), "s"(base) : "m0", "memory");
}
#pragma clang diagnostic pop
template <int N>
SL_DEV void wait_dma() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// All waves' reads of LDS are done and have arrived.
SL_DEV void stage_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Four waves, 2 x 2, TM x TN tiles of 32 x 32 each: 64 TM x 64 TN of c in a workgroup.  Per step of 128 of the
// contraction a stage of LDS holds the workgroup's operands as they lie in memory - an operand is what a wave reads in lane
// order - and STAGES are filled ahead; a wave's operands of the next step are read into registers while the matrix unit works on
// this one's.
// Row i of a result's tile is not b's row i: i = 8 g + 4 q + e takes 16 (g / 2) + 8 q + 4 (g % 2) + e, so that a lane has
// eight consecutive columns of c twice.
// Workgroup `tiles` and on: the next part of the contraction, with a c of its own.
template <bool B16, int TM, int TN, int STAGES, int WGS>
__global__ void __launch_bounds__(256, WGS) k_product(ProductArgs A)
{
    constexpr int CODES = (2 * TM + 2 * TN) * MX_TILE_BYTES, STAGE = CODES + 2048;
    constexpr int PER_WAVE = TM + TN, D = PER_WAVE + 1;             // loads of a wave per stage, 1 KB each
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), wm = wave >> 1, wn = wave & 1;
    const unsigned tiles = (unsigned)(A.m_tiles * A.n_tiles), part = blockIdx.x / tiles;
    const TilePlace at = tile_place(blockIdx.x % tiles, tiles, A.m_tiles, A.n_tiles);
    const long long i0 = at.m * (2 * TM), j0 = at.n * (2 * TN);     // row tiles of a and b
    const long long k0 = part * A.part_steps;
    const int steps = (int)min(A.part_steps, A.k_tiles - k0);
    const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char *)lds;

    // what lies past the last row tile is read at that one and not stored
    const unsigned char *src[PER_WAVE];
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
        const int half = wave + 4 * i, t = half >> 1;
        src[i] = (t < 2 * TM ? A.a + (min(i0 + t, A.a_tiles - 1) * A.k_tiles + k0) * MX_TILE_BYTES
                             : A.b + (min(j0 + t - 2 * TM, A.b_tiles - 1) * A.k_tiles + k0) * MX_TILE_BYTES) + (half & 1) * 1024;
    }
    // even waves bring a's scales, odd ones b's: up to four tiles of 64 rows, 16 lanes each
    const unsigned char *scales = wave & 1 ? A.b + A.b_scales : A.a + A.a_scales;
    const long long group0 = (wave & 1 ? j0 : i0) >> 1, groups = ((wave & 1 ? A.b_tiles : A.a_tiles) + 1) >> 1;
    scales += (min(group0, groups - 1) * A.k_tiles + k0) * MX_SCALE_TILE_BYTES;
    const unsigned scale_off = (unsigned)((min(group0 + (lane >> 4), groups - 1) - min(group0, groups - 1)) * A.k_tiles * MX_SCALE_TILE_BYTES) + (lane & 15) * 16;

    // (past the last step it brings that one again, so that every step waits for the same number of loads)
    auto fill = [&](int at) __attribute__((always_inline)) {
        const unsigned to = lds0 + (unsigned)at % STAGES * STAGE;
        const long long s = min(at, steps - 1);
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) dma16(src[i] + s * MX_TILE_BYTES, lane * 16, to + (wave + 4 * i) * 1024);
        dma16(scales + s * MX_SCALE_TILE_BYTES, scale_off, to + CODES + (wave & 1) * 1024);
    };

    // b's row that this lane has in a tile
    const int i = lane & 31, r = 16 * (i >> 4) + 8 * (i >> 2 & 1) + 4 * (i >> 3 & 1) + (i & 3);
    const int b_off = (lane >> 5) * 512 + r * 16, b_scale = (lane >> 5) * 128 + r * 4;

    sl_u4 a[2][TM][2], b[2][TN][2];
    constexpr int WA = (TM + 1) / 2, WB = (TN + 1) / 2;             // scale words: 64 rows each
    unsigned sa[2][WA], sb[2][WB];
    constexpr int READS = WA + WB + 2 * (TM + TN);
    auto read = [&](int s, auto set) __attribute__((always_inline)) {
        constexpr int S = decltype(set)::value;
        const unsigned char *st = lds + (unsigned)s % STAGES * STAGE;
#pragma unroll
        for (int t = 0; t < WA; ++t) sa[S][t] = *reinterpret_cast<const unsigned *>(st + CODES + ((wm * TM >> 1) + t) * 256 + lane * 4);
#pragma unroll
        for (int t = 0; t < WB; ++t) sb[S][t] = *reinterpret_cast<const unsigned *>(st + CODES + 1024 + ((wn * TN >> 1) + t) * 256 + b_scale);
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
        // (the byte of a scale word that an operand takes is part of the instruction; a wave with one tile of the word's two has
        // it moved to the first)
        unsigned ta[WA], tb[WB];
#pragma unroll
        for (int t = 0; t < WA; ++t) ta[t] = TM == 1 ? sa[S][t] >> (16 * wm) : sa[S][t];
#pragma unroll
        for (int t = 0; t < WB; ++t) tb[t] = TN == 1 ? sb[S][t] >> (16 * wn) : sb[S][t];
#define MX4_AT(H, I, J) \
    if constexpr (I < TM && J < TN) \
        acc[I][J] = mx4_step<2 * (J & 1) + H, 2 * (I & 1) + H>(b[S][J][H], a[S][I][H], acc[I][J], tb[J >> 1], ta[I >> 1]);
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
        wait_dma<(STAGES - 2) * D>();
        stage_barrier();
        fill(s + STAGES);
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
        wait_dma<(STAGES - 1) * D>();
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
    // c through LDS, 32 rows of a wave at a time, so that a row's columns are written in one piece
    __syncthreads();
    constexpr int PITCH = TN * 32 * (B16 ? 2 : 4) + 16, PIECES = TN * 32 * (B16 ? 2 : 4) / 16, TOGETHER = PIECES < 8 ? PIECES / 2 : 4;
    static_assert(PIECES / 2 % TOGETHER == 0, "whole groups of pieces");
    unsigned char *mine = lds + wave * (32 * PITCH);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const sl_f16 v = acc[i][j];
                unsigned char *to = mine + (lane & 31) * PITCH + (32 * j + 16 * p + (lane >> 5) * 8) * (B16 ? 2 : 4);
                if constexpr (B16) {
                    *reinterpret_cast<sl_u4 *>(to) = sl_u4{sl_bf16_pair(v[8 * p], v[8 * p + 1]), sl_bf16_pair(v[8 * p + 2], v[8 * p + 3]),
                                                           sl_bf16_pair(v[8 * p + 4], v[8 * p + 5]), sl_bf16_pair(v[8 * p + 6], v[8 * p + 7])};
                } else {
                    *reinterpret_cast<sl_f4 *>(to) = sl_f4{v[8 * p], v[8 * p + 1], v[8 * p + 2], v[8 * p + 3]};
                    *reinterpret_cast<sl_f4 *>(to + 16) = sl_f4{v[8 * p + 4], v[8 * p + 5], v[8 * p + 6], v[8 * p + 7]};
                }
            }
        sl_wave_sync();
        const long long row0 = (i0 + wm * TM + i) * MX_ROWS, col0 = (j0 + wn * TN) * MX_ROWS;
        // (four pieces at a time: what c already holds, where it is added to, is requested together)
#pragma unroll
        for (int t = 0; t < PIECES / 2; t += TOGETHER) {
            sl_f4 there[TOGETHER];
            if (!B16 && A.accumulate) {
#pragma unroll
                for (int u = 0; u < TOGETHER; ++u) {
                    const int piece = (t + u) * 64 + lane, row = piece / PIECES, at = piece % PIECES;
                    there[u] = load_piece(A, row0 + row, col0 + at * 4);
                }
            }
#pragma unroll
            for (int u = 0; u < TOGETHER; ++u) {
                const int piece = (t + u) * 64 + lane, row = piece / PIECES, at = piece % PIECES;
                sl_u4 w = *reinterpret_cast<const sl_u4 *>(mine + row * PITCH + at * 16);
                if (!B16 && A.accumulate) w = __builtin_bit_cast(sl_u4, there[u] + __builtin_bit_cast(sl_f4, w));
                store_piece<B16>(A, part, row0 + row, col0 + at * (B16 ? 8 : 4), w);
            }
        }
        sl_wave_sync();
    }
}

// c from the parts' results, added in their order.
template <bool B16>
__global__ void __launch_bounds__(256) k_join(ProductArgs A, const float *parts, long long ldp, int n_parts)
{
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, row = at / (ldp / 4), col = at % (ldp / 4) * 4;
    if (row >= A.m) return;
    const float *p = parts + row * ldp + col;
    sl_f4 v = *reinterpret_cast<const sl_f4 *>(p);
    for (int i = 1; i < n_parts; ++i) v = v + *reinterpret_cast<const sl_f4 *>(p + i * A.part_size);
    const int n = (int)min(A.n - col, 4ll);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= n) break;
        if constexpr (B16) {
            static_cast<unsigned short *>(A.c)[row * A.ldc + col + i] = (unsigned short)sl_bf16_bits(v[i]);
        } else {
            float *c = static_cast<float *>(A.c) + row * A.ldc + col + i;
            *c = A.accumulate ? *c + v[i] : v[i];
        }
    }
}

// ---- few rows ----

// y = Q(x) w^T for up to 16 rows of x, in the 16 x 16 x 128 shape of the matrix unit: lane l has block l / 16 of row
// l % 16.  Every workgroup quantises x for itself, into LDS; w's first bytes are requested before x's, and loads complete in
// the order of their requests, so that x is waited for together with them.  Its eight waves then take 8 / KW tiles of 16 rows of w, KW waves for a tile, each every KW-th step of 128 of the contraction,
// and the sums of a tile's waves are added in their order.  Bound by the way of w's bytes to the registers, each of which is
// used once, and for small layers by the launch.
struct FewArgs {
    const void *x;
    long long ldx;
    const unsigned char *w;
    SlMx4Shape s;                    // of w
    int m;
    void *y;
    long long ldy;
};

enum { FEW_AHEAD = 4 };              // steps of w that a wave has under way

template <bool X16, bool Y16, int KW>
__global__ void __launch_bounds__(512) k_few_rows(FewArgs A)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), slice = wave % KW;
    const int steps = (int)A.s.col_tiles, m = A.m;
    sl_f4 *sums = reinterpret_cast<sl_f4 *>(lds);
    unsigned char *xc = lds + (KW > 1 ? 8 * 1024 : 0), *xs = xc + steps * m * 64;         // block by block, row by row
    const long long tile = (long long)blockIdx.x * (8 / KW) + wave / KW, tiles = (A.s.rows + 15) / 16, at = min(tile, tiles - 1);
    const int row = (int)(at & 1) * 16 + (lane & 15), b = lane >> 4;                      // of w, in its row tile
    const unsigned char *codes = A.w + (at >> 1) * A.s.col_tiles * MX_TILE_BYTES + sl_mx4_code_at(row, b);
    const unsigned char *scales = A.w + A.s.scales + (at >> 2) * A.s.col_tiles * MX_SCALE_TILE_BYTES + sl_mx4_scale_at((int)(at >> 1 & 1) * 32 + row, b);
    sl_u4 c[FEW_AHEAD];
    unsigned q[FEW_AHEAD];
    auto request = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < FEW_AHEAD; ++u) {
            const int k = min(k0 + u * KW, steps - 1);                        // (past the end: that one again, not used)
            c[u] = *reinterpret_cast<const sl_u4 *>(codes + (long long)k * MX_TILE_BYTES);
            q[u] = scales[(long long)k * MX_SCALE_TILE_BYTES];
        }
    };
    request(slice);
    // x: a quad of lanes to a block
    for (int i = threadIdx.x; i < m * steps * 16; i += 512) {
        const int r = i / (steps * 16), o = i % (steps * 16), at = (o >> 2) * m + r;
        SlOctet<X16> v;
        v.load(A.x, r * A.ldx + (long long)o * 8, (int)max(min(A.s.cols - (long long)o * 8, 8ll), 0ll));
        const unsigned sx = sl_mx4_scale(sl_quad_max(v.top()));
        *reinterpret_cast<unsigned *>(xc + at * 16 + (o & 3) * 4) = v.pack(sx);
        if ((o & 3) == 0) xs[at] = (unsigned char)sx;
    }
    __syncthreads();
    const int xr = min(lane & 15, m - 1);                                     // (rows past the last: that one again, not stored)
    sl_f4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = slice; k0 < steps; k0 += KW * FEW_AHEAD) {
        sl_u4 d[FEW_AHEAD];
        unsigned p[FEW_AHEAD];
#pragma unroll
        for (int u = 0; u < FEW_AHEAD; ++u) d[u] = c[u], p[u] = q[u];
        request(k0 + KW * FEW_AHEAD);
#pragma unroll
        for (int u = 0; u < FEW_AHEAD; ++u) {
            const int k = k0 + u * KW;
            if (k >= steps) break;
            const int at = (k * 4 + b) * m + xr;
            const sl_u4 e = *reinterpret_cast<const sl_u4 *>(xc + at * 16);
            const v8i ws = {(int)d[u].x, (int)d[u].y, (int)d[u].z, (int)d[u].w, 0, 0, 0, 0}, xv = {(int)e.x, (int)e.y, (int)e.z, (int)e.w, 0, 0, 0, 0};
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ws, xv, acc, 4, 4, 0, (int)p[u], 0, (int)xs[at]);
        }
    }
    if constexpr (KW > 1) {
        sums[wave * 64 + lane] = acc;
        __syncthreads();
        if (slice != 0) return;
#pragma unroll
        for (int i = 1; i < KW; ++i) acc = acc + sums[(wave + i) * 64 + lane];
    }
    // lane l: row l % 16 of x, columns 4 (l / 16) .. + 3 of the tile
    const long long r = lane & 15, col = tile * 16 + b * 4;
    if (tile >= tiles || r >= m) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (col + e >= A.s.rows) break;
        if constexpr (Y16) static_cast<unsigned short *>(A.y)[r * A.ldy + col + e] = (unsigned short)sl_bf16_bits(acc[e]);
        else static_cast<float *>(A.y)[r * A.ldy + col + e] = acc[e];
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

// (with m n <= 2^36 and at most 2^27 rows each, tiles of 128 x 128 are less than 2^24: a grid has less than 2^32 threads)
bool bad_sizes(int64_t m, int64_t n, int64_t k)
{
    if (m < 0 || n < 0 || k < 0) return true;
    if (m == 0 || n == 0) return false;
    SlMx4Shape s;
    return m > ((int64_t)1 << 36) / n || !sl_mx4_shape(m, k > 0 ? k : 1, s) || !sl_mx4_shape(n, k > 0 ? k : 1, s);
}

template <bool B16, int TM, int TN, int STAGES, int WGS>
int launch_tiles(ProductArgs A, int parts, hipStream_t st)
{
    A.m_tiles = (A.m + 64 * TM - 1) / (64 * TM);
    A.n_tiles = (A.n + 64 * TN - 1) / (64 * TN);
    constexpr unsigned bytes = STAGES * ((2 * TM + 2 * TN) * MX_TILE_BYTES + 2048);
    if (bytes > 65536) {
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_product<B16, TM, TN, STAGES, WGS>),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (err != hipSuccess) {
            sl_note_hip_error(err);
            return SL_ERR_HIP;
        }
    }
    hipLaunchKernelGGL((k_product<B16, TM, TN, STAGES, WGS>), dim3((unsigned)(A.m_tiles * A.n_tiles * parts)), dim3(256), bytes, st, A);
    return check_launch();
}

template <bool B16>
int launch(const ProductArgs &A, SlMx4Choice c, hipStream_t st)
{
    return c.tile == 0 ? launch_tiles<B16, 1, 1, 4, 4>(A, c.parts, st)
         : c.tile == 1 ? launch_tiles<B16, 2, 2, 4, 2>(A, c.parts, st)
                       : launch_tiles<B16, 2, 4, 3, 2>(A, c.parts, st);
}

// parts: room for the results of the parts of the contraction
int product(const unsigned char *a, const unsigned char *b, int64_t m, int64_t n, int64_t k, void *c, int type, int64_t ldc,
            int accumulate, float *parts, hipStream_t st)
{
    ProductArgs A;
    SlMx4Shape sa = {}, sb = {};
    if (k > 0) {
        (void)sl_mx4_shape(m, k, sa);
        (void)sl_mx4_shape(n, k, sb);
    }
    const SlMx4Choice how = sl_mx4_choose(m, n, k);
    A.a = a, A.b = b;
    A.a_tiles = sa.row_tiles, A.b_tiles = sb.row_tiles, A.k_tiles = k > 0 ? sa.col_tiles : 0;
    A.a_scales = sa.scales, A.b_scales = sb.scales;
    A.m = m, A.n = n, A.c = c, A.ldc = ldc, A.accumulate = accumulate;
    A.part_steps = (A.k_tiles + how.parts - 1) / how.parts, A.part_size = 0;
    if (how.parts == 1)
        return type == SL_TYPE_BF16 ? launch<true>(A, how, st) : launch<false>(A, how, st);
    ProductArgs P = A;
    const long long ldp = sl_mx4_part_pitch(n);
    P.c = parts, P.ldc = ldp, P.part_size = A.part_size = m * ldp, P.accumulate = 0;
    if (const int rc = launch<false>(P, how, st)) return rc;
    const dim3 grid((unsigned)((m * (ldp / 4) + 255) / 256));
    hipLaunchKernelGGL(type == SL_TYPE_BF16 ? k_join<true> : k_join<false>, grid, dim3(256), 0, st, A, parts, ldp, how.parts);
    return check_launch();
}

// Bytes of LDS for the few rows' kernel: the sums of the waves and x in 4 bits.
int64_t few_rows_lds(int64_t m, int64_t k) { return 8 * 1024 + (k + MX_COLS - 1) / MX_COLS * m * 68; }

template <bool X16, bool Y16>
int launch_few_rows(const FewArgs &A, int64_t lds, hipStream_t st)
{
    typedef void (*kernel_t)(FewArgs);
    static const kernel_t table[4] = {k_few_rows<X16, Y16, 1>, k_few_rows<X16, Y16, 2>, k_few_rows<X16, Y16, 4>, k_few_rows<X16, Y16, 8>};
    const int64_t tiles = (A.s.rows + 15) / 16;
    const int log2 = sl_mx4_few_waves_log2(A.s.rows);
    const int64_t per = 8 >> log2;
    hipLaunchKernelGGL(table[log2], dim3((unsigned)((tiles + per - 1) / per)), dim3(512), (unsigned)lds, st, A);
    return check_launch();
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

extern "C" {

size_t sl_mx4_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (bad_sizes(m, n, k) || m == 0 || n == 0 || k == 0) return 0;
    return (sl_mx4_few_rows(m, k) ? 0 : align256(sl_mx4_bytes(m, k))) + sizeof(float) * (size_t)sl_mx4_parts_room(m, n, k);
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
    if (!workspace && k > 0 && (!sl_mx4_few_rows(m, k) || sl_mx4_choose(m, n, k).parts > 1)) return SL_ERR_INVALID_ARG;
    return product(static_cast<const unsigned char *>(a), static_cast<const unsigned char *>(b), m, n, k, c, c_type, ldc,
                   accumulate, static_cast<float *>(workspace), static_cast<hipStream_t>(stream));
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
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (k > 0 && sl_mx4_few_rows(m, k)) {
        FewArgs A;
        A.x = x, A.ldx = ldx, A.w = static_cast<const unsigned char *>(w), A.m = (int)m, A.y = y, A.ldy = ldy;
        (void)sl_mx4_shape(n, k, A.s);
        const int64_t lds = few_rows_lds(m, k);
        if (x_type == SL_TYPE_BF16) return y_type == SL_TYPE_BF16 ? launch_few_rows<true, true>(A, lds, st) : launch_few_rows<true, false>(A, lds, st);
        return y_type == SL_TYPE_BF16 ? launch_few_rows<false, true>(A, lds, st) : launch_few_rows<false, false>(A, lds, st);
    }
    if (!workspace && k > 0) return SL_ERR_INVALID_ARG;
    unsigned char *q = static_cast<unsigned char *>(workspace);
    if (k > 0)
        if (const int rc = slk_mx4_quantize(x, x_type, m, k, ldx, q, nullptr, st)) return rc;
    float *parts = k > 0 ? reinterpret_cast<float *>(q + align256(sl_mx4_bytes(m, k))) : nullptr;
    return product(q, static_cast<const unsigned char *>(w), m, n, k, y, y_type, ldy, 0, parts, st);
}

}  // extern "C"
