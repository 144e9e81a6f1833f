// Root-mean-square norm of rows, with the residual's addition in front of it and the 4-bit matrices of its result behind it,
// and its backward pass.
//   h = x + residual ;  s = 1 / sqrt(mean(h^2) + eps) ;  y = (h s) w
//   dx = dh + s (g - u mean(g u)),  g = dy w, u = h s ;  dw = sum over the rows of dy u
// All of it is bound by memory: a row is read once and kept in registers until its sums are known.  mean(h^2) is summed in 64 bits, so
// that s, and with it the 4-bit codes of values next to a border, do not depend on the order of the sum.
#include <algorithm>
#include <cmath>

#include "sl_internal.h"
#include "sl_mx4.h"

namespace {

struct NormArgs {
    const void *x, *residual, *w;
    void *h, *y;
    float *rstd;
    unsigned char *q, *qt;
    SlMx4Shape s, t;                 // of q and of qt
    long long rows, cols, ldx, ldr, ldh, ldy;
    double eps;
    int w16, y16;
};

struct BackArgs {
    const void *h, *w, *dy, *dh;
    const float *rstd;
    void *dx;
    float *parts;                    // sums over the rows of a group, one row of cols per group
    long long rows, cols, ldh, lddy, lddh, lddx;
    int w16;
};

enum { NONE = 0, F32 = 1, B16 = 2 };            // residual
enum { WIDE = 32768, PANEL = 2048, GROUPS = 512 };

// Eight values to a dense row, of which the first n exist.
SL_DEV void put_octet(void *to, bool b16, long long at, int n, const float (&v)[8])
{
    if (n <= 0) return;
    if (b16) {
        typedef unsigned u4a __attribute__((ext_vector_type(4), aligned(2)));
        unsigned short *o = static_cast<unsigned short *>(to) + at;
        if (n >= 8) {
            *reinterpret_cast<u4a *>(o) = sl_u4{sl_bf16_pair(v[0], v[1]), sl_bf16_pair(v[2], v[3]), sl_bf16_pair(v[4], v[5]), sl_bf16_pair(v[6], v[7])};
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < n) o[i] = (unsigned short)sl_bf16_bits(v[i]);
        }
    } else {
        typedef float f4a __attribute__((ext_vector_type(4), aligned(4)));
        float *o = static_cast<float *>(to) + at;
        if (n >= 8) {
            *reinterpret_cast<f4a *>(o) = sl_f4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f4a *>(o + 4) = sl_f4{v[4], v[5], v[6], v[7]};
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < n) o[i] = v[i];
        }
    }
}

SL_DEV void get_octet(const void *from, bool b16, long long at, int n, float (&v)[8])
{
    if (b16) {
        SlOctet<true> o;
        o.load(from, at, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = o.value(i);
    } else {
        SlOctet<false> o;
        o.load(from, at, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = o.value(i);
    }
}

SL_DEV int octet_left(long long cols, long long col) { return (int)max(min(cols - col, 8ll), 0ll); }

// h of eight elements of a row, in the values that its type has.
template <bool X16, int R>
SL_DEV void form_h(const NormArgs &A, long long row, long long col, int n, float (&h)[8])
{
    get_octet(A.x, X16, row * A.ldx + col, n, h);
    if constexpr (R != NONE) {
        float r[8];
        get_octet(A.residual, R == B16, row * A.ldr + col, n, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[i] = h[i] + r[i];
            if constexpr (R == B16) h[i] = __uint_as_float(sl_bf16_bits(h[i]) << 16);
        }
    }
}

SL_DEV double square_sum(const float (&h)[8])
{
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = fma((double)h[i], (double)h[i], t);
    return t;
}

SL_DEV float reciprocal_rms(double sum, const NormArgs &A) { return (float)(1.0 / sqrt(sum / (double)A.cols + A.eps)); }

SL_DEV void scale_octet(const NormArgs &A, long long col, int n, float s, const float (&h)[8], float (&y)[8])
{
    float w[8];
    get_octet(A.w, A.w16, col, n, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = h[i] * s * w[i];
}

// The sum of a value over WAVES waves, in their order, in all of them.
template <int WAVES, class T>
SL_DEV T team_sum(T v, T *room, int wave, int lane)
{
    if constexpr (WAVES == 1) return v;
    if (lane == 0) room[wave] = v;
    __syncthreads();
    T t = room[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) t = t + room[i];
    __syncthreads();
    return t;
}

// ---- y alone: WAVES waves to a row, OCT times eight elements in a lane ----

// One wave to a row as long as its registers hold it: no barrier.  16,384 x 2048, all bf16: 44 us, 6.2 TB/s.

// (LONG: rows that do not fit the registers are read twice)
template <bool X16, int R, int WAVES, int OCT, bool LONG>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) k_norm(NormArgs A)
{
    __shared__ double room[WAVES];
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6));
    const long long row = WAVES == 1 ? blockIdx.x * 4ll + wave : blockIdx.x;
    if (row >= A.rows) return;                    // (one wave to a row: no barrier follows)
    const int part = WAVES == 1 ? 0 : wave;
    constexpr long long STEP = WAVES * OCT * 512;
    float h[OCT][8];
    double sum = 0.0;
    for (long long base = 0; base < (LONG ? A.cols : 1); base += STEP)
#pragma unroll
        for (int j = 0; j < OCT; ++j) {
            const long long col = base + ((j * WAVES + part) * 64 + lane) * 8;
            form_h<X16, R>(A, row, col, octet_left(A.cols, col), h[j]);
            if constexpr (LONG) {
                if constexpr (R != NONE) put_octet(A.h, R == B16, row * A.ldh + col, octet_left(A.cols, col), h[j]);
                sum = sum + square_sum(h[j]);
            }
        }
    if constexpr (!LONG) {
#pragma unroll
        for (int j = 0; j < OCT; ++j) {
            if constexpr (R != NONE) {
                const long long col = ((j * WAVES + part) * 64 + lane) * 8;
                put_octet(A.h, R == B16, row * A.ldh + col, octet_left(A.cols, col), h[j]);
            }
            sum = sum + square_sum(h[j]);
        }
    }
    sum = team_sum<WAVES>(sl_wave_tree(sum, 6), room, wave, lane);
    const float s = reciprocal_rms(sum, A);
    if (A.rstd && part == 0 && lane == 0) A.rstd[row] = s;
    if (!A.y) return;
    for (long long base = 0; base < (LONG ? A.cols : 1); base += STEP)
#pragma unroll
        for (int j = 0; j < OCT; ++j) {
            const long long col = base + ((j * WAVES + part) * 64 + lane) * 8;
            const int n = octet_left(A.cols, col);
            if constexpr (LONG) {
                if constexpr (R != NONE) get_octet(A.h, R == B16, row * A.ldh + col, n, h[j]);
                else get_octet(A.x, X16, row * A.ldx + col, n, h[j]);
            }
            float y[8];
            scale_octet(A, col, n, s, h[j], y);
            put_octet(A.y, A.y16, row * A.ldy + col, n, y);
        }
}

// ---- 4-bit matrices: 32 rows to a workgroup ----

// 16 waves with two rows each, OCT times eight elements of either in a lane; y in bf16 goes to LDS, 2048 columns at a time, from which a thread then takes blocks of 32 along a row
// (q) and of 32 rows of two columns (qt): neither needs another lane, and what a wave writes lies together.  16,384 x 2048 bf16 on an fp32
// residual: 76 to 82 us, 4.5 to 4.9 TB/s - one workgroup to a compute unit, whose start and end nothing hides; y in bf16 and its
// quantisation apart 70 + 21.
// (LONG: more than 2048 columns, which are read twice)
template <bool X16, int R, int OCT, bool LONG>
__global__ void __launch_bounds__(1024) k_norm_mx4(NormArgs A, int pitch)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = sl_uniform(tid >> 6);
    const long long row0 = blockIdx.x * 32ll;
    float h[2][OCT][8], s[2];
    double sum[2] = {0.0, 0.0};
    for (long long base = 0; base < (LONG ? A.cols : 1); base += PANEL) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const long long row = row0 + wave * 2 + i;
#pragma unroll
            for (int j = 0; j < OCT; ++j) {
                const long long col = base + (j * 64 + lane) * 8;
                form_h<X16, R>(A, row, col, row < A.rows ? octet_left(A.cols, col) : 0, h[i][j]);
            }
#pragma unroll
            for (int j = 0; j < OCT; ++j) {
                const long long col = base + (j * 64 + lane) * 8;
                if constexpr (R != NONE) put_octet(A.h, R == B16, row * A.ldh + col, row < A.rows ? octet_left(A.cols, col) : 0, h[i][j]);
                sum[i] = sum[i] + square_sum(h[i][j]);
            }
            __builtin_amdgcn_sched_barrier(0);            // (with the second row's loads up here the registers do not suffice)
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const long long row = row0 + wave * 2 + i;
        s[i] = reciprocal_rms(sl_wave_tree(sum[i], 6), A);
        if (A.rstd && lane == 0 && row < A.rows) A.rstd[row] = s[i];
    }
    const long long rt = row0 / MX_ROWS;
    for (long long base = 0; base < (LONG ? A.cols : 1); base += PANEL) {
        if constexpr (LONG) __syncthreads();              // h has been written; LDS has been read
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < OCT; ++j) {
                const long long row = row0 + wave * 2 + i, col = base + (j * 64 + lane) * 8;
                const int n = row < A.rows ? octet_left(A.cols, col) : 0;
                if constexpr (LONG) {
                    if constexpr (R != NONE) get_octet(A.h, R == B16, row * A.ldh + col, n, h[i][j]);
                    else get_octet(A.x, X16, row * A.ldx + col, n, h[i][j]);
                }
                float y[8];
                scale_octet(A, col, n, s[i], h[i][j], y);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e >= n) y[e] = 0.0f;              // (not NaN, where the row is: blocks past the last column are zero)
                if ((j * 64 + lane) * 16 < pitch - 16)
                    *reinterpret_cast<sl_u4 *>(lds + (wave * 2 + i) * pitch + (j * 64 + lane) * 16) =
                        sl_u4{sl_bf16_pair(y[0], y[1]), sl_bf16_pair(y[2], y[3]), sl_bf16_pair(y[4], y[5]), sl_bf16_pair(y[6], y[7])};
                if (A.y) put_octet(A.y, A.y16, row * A.ldy + col, n, y);
            }
        __syncthreads();
        const long long tile0 = base / MX_COLS;
        if (A.q && rt < (A.s.row_tiles + 1) / 2 * 2) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = tid & 31, block = i * 32 + (tid >> 5);
                const long long tile = tile0 + (block >> 2);
                if (tile >= A.s.col_tiles) break;
                SlOctet<true> v[4];
                unsigned top = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const sl_u4 w = *reinterpret_cast<const sl_u4 *>(lds + r * pitch + block * 64 + j * 16);
                    v[j].w[0] = w.x, v[j].w[1] = w.y, v[j].w[2] = w.z, v[j].w[3] = w.w;
                    top = max(top, v[j].top());
                }
                const unsigned x = sl_mx4_scale(top);
                if (rt < A.s.row_tiles)
                    *reinterpret_cast<sl_u4 *>(A.q + (rt * A.s.col_tiles + tile) * MX_TILE_BYTES + sl_mx4_code_at(r, block & 3)) =
                        sl_u4{v[0].pack(x), v[1].pack(x), v[2].pack(x), v[3].pack(x)};
                A.q[A.s.scales + (rt / 2 * A.s.col_tiles + tile) * MX_SCALE_TILE_BYTES + sl_mx4_scale_at((int)(rt & 1) * 32 + r, block & 3)] = (unsigned char)x;
            }
        }
        if (A.qt && tid * 4 < pitch - 16) {
            unsigned e[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) e[i] = *reinterpret_cast<const unsigned *>(lds + i * pitch + tid * 4);
            sl_u4 w[2];
            unsigned x[2];
            sl_mx4_columns(e, w, x);
            const long long kt = row0 / MX_COLS;
            const int b = (int)(rt & 3);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const long long c = base + tid * 2 + i, ct = c / MX_ROWS;
                if (ct < A.t.row_tiles)
                    *reinterpret_cast<sl_u4 *>(A.qt + (ct * A.t.col_tiles + kt) * MX_TILE_BYTES + sl_mx4_code_at((int)(c & 31), b)) = w[i];
                if (ct < (A.t.row_tiles + 1) / 2 * 2)
                    A.qt[A.t.scales + (ct / 2 * A.t.col_tiles + kt) * MX_SCALE_TILE_BYTES + sl_mx4_scale_at((int)(c & 63), b)] = (unsigned char)x[i];
            }
        }
    }
}

// ---- backward ----

// A group of rows to a workgroup, one after the other (WAVES == 1: its four waves take one each at a time); dw's sums over them stay in
// registers.  16,384 x 2048, fp32 h and dx, bf16 dy: 94 us, 5.0 TB/s, and 4 for the join.  Tried and not kept: the next row requested ahead (99), four waves
// to a row (94 to 98), 768 and 1024 groups (95, 98).
// (LONG: rows that do not fit the registers are read twice, and dw is k_column_sums's)
template <bool H16, bool DY16, bool DX16, int WAVES, int OCT, bool LONG>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) k_back(BackArgs A, long long per_group)
{
    __shared__ double room[WAVES];
    __shared__ float team[WAVES == 1 ? 3 : 1][WAVES == 1 ? OCT * 512 : 1];
    constexpr long long STEP = WAVES * OCT * 512;
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), part = WAVES == 1 ? 0 : wave;
    const long long first = blockIdx.x * per_group, end = min(first + per_group, A.rows);
    float dw[OCT][8];
#pragma unroll
    for (int j = 0; j < OCT; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[j][e] = 0.0f;
    for (long long row = first + (WAVES == 1 ? wave : 0); row < end; row += WAVES == 1 ? 4 : 1) {
        const float s = A.rstd[row];
        float u[OCT][8], g[OCT][8];
        double sum = 0.0;
        auto load = [&](long long base, bool sums) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < OCT; ++j) {
                const long long col = base + ((j * WAVES + part) * 64 + lane) * 8;
                const int n = octet_left(A.cols, col);
                get_octet(A.h, H16, row * A.ldh + col, n, u[j]);
                get_octet(A.dy, DY16, row * A.lddy + col, n, g[j]);
            }
#pragma unroll
            for (int j = 0; j < OCT; ++j) {
                const long long col = base + ((j * WAVES + part) * 64 + lane) * 8;
                float w[8];
                get_octet(A.w, A.w16, col, octet_left(A.cols, col), w);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    u[j][e] = u[j][e] * s;
                    if constexpr (!LONG) dw[j][e] = dw[j][e] + g[j][e] * u[j][e];
                    g[j][e] = g[j][e] * w[e];
                    if (sums) sum = fma((double)g[j][e], (double)u[j][e], sum);
                }
            }
        };
        for (long long base = 0; base < (LONG ? A.cols : 1); base += STEP) load(base, true);
        sum = team_sum<WAVES>(sl_wave_tree(sum, 6), room, wave, lane);
        const float c = (float)(sum / (double)A.cols);
        for (long long base = 0; base < (LONG ? A.cols : 1); base += STEP) {
            if constexpr (LONG) load(base, false);
#pragma unroll
            for (int j = 0; j < OCT; ++j) {
                const long long col = base + ((j * WAVES + part) * 64 + lane) * 8;
                const int n = octet_left(A.cols, col);
                float d[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = s * (g[j][e] - u[j][e] * c);
                if (A.dh) {
                    float o[8];
                    get_octet(A.dh, DX16, row * A.lddh + col, n, o);
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[e] = o[e] + d[e];
                }
                put_octet(A.dx, DX16, row * A.lddx + col, n, d);
            }
        }
    }
    if constexpr (!LONG) {
        if (!A.parts) return;
        if constexpr (WAVES == 1) {
            if (wave > 0) {
#pragma unroll
                for (int j = 0; j < OCT; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) team[wave - 1][(j * 8 + e) * 64 + lane] = dw[j][e];
            }
            __syncthreads();
            if (wave > 0) return;
#pragma unroll
            for (int i = 0; i < 3; ++i)
#pragma unroll
                for (int j = 0; j < OCT; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) dw[j][e] = dw[j][e] + team[i][(j * 8 + e) * 64 + lane];
        }
#pragma unroll
        for (int j = 0; j < OCT; ++j) {
            const long long col = ((j * WAVES + part) * 64 + lane) * 8;
            put_octet(A.parts, false, blockIdx.x * A.cols + col, octet_left(A.cols, col), dw[j]);
        }
    }
}

template <bool H16, bool DY16>
__global__ void __launch_bounds__(256) k_column_sums(BackArgs A, long long per_group)
{
    const long long col = blockIdx.x * 256ll + threadIdx.x, first = blockIdx.y * per_group, end = min(first + per_group, A.rows);
    if (col >= A.cols) return;
    float t = 0.0f;
    for (long long row = first; row < end; ++row) {
        const float h = H16 ? __uint_as_float((unsigned)static_cast<const unsigned short *>(A.h)[row * A.ldh + col] << 16)
                            : static_cast<const float *>(A.h)[row * A.ldh + col];
        const float dy = DY16 ? __uint_as_float((unsigned)static_cast<const unsigned short *>(A.dy)[row * A.lddy + col] << 16)
                              : static_cast<const float *>(A.dy)[row * A.lddy + col];
        t = t + dy * (h * A.rstd[row]);
    }
    A.parts[blockIdx.y * A.cols + col] = t;
}

// dw from the groups' sums: 64 columns to a workgroup, its 16 waves take every 16th group; in 64 bits, in a fixed order.
__global__ void __launch_bounds__(1024) k_join_dw(const float *parts, int groups, long long cols, float *dw, int accumulate)
{
    __shared__ double room[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long col = blockIdx.x * 64ll + lane;
    double t = 0.0;
    if (col < cols) {
#pragma unroll 8
        for (int g = wave; g < groups; g += 16) t = t + (double)parts[g * cols + col];
    }
    room[wave][lane] = t;
    __syncthreads();
    if (wave > 0 || col >= cols) return;
    for (int i = 1; i < 16; ++i) t = t + room[i][lane];
    dw[col] = (float)(accumulate ? (double)dw[col] + t : t);
}

int check_launch()
{
    const hipError_t err = hipGetLastError();
    if (err == hipSuccess) return SL_OK;
    sl_note_hip_error(err);
    return SL_ERR_HIP;
}

bool bad_type(int type) { return type != SL_TYPE_F32 && type != SL_TYPE_BF16; }
// Address and row stride of a matrix that is there.
bool bad_matrix(const void *p, int type, int64_t cols, int64_t ld)
{
    return ((uintptr_t)p & (type == SL_TYPE_BF16 ? 1 : 3)) != 0 || ld < cols || ld > ((int64_t)1 << 40);
}

template <bool X16, int R>
int launch_norm(const NormArgs &A, hipStream_t st)
{
    if (A.q || A.qt) {
        const bool wide = A.cols > PANEL;
        const int pitch = 2 * (int)std::min<long long>((A.cols + MX_COLS - 1) / MX_COLS * MX_COLS, PANEL) + 16;
        const unsigned groups = (unsigned)(A.qt ? (A.rows + 127) / 128 * 4 : (A.rows + 63) / 64 * 2), bytes = 32u * pitch;
        typedef void (*kernel_t)(NormArgs, int);
        const kernel_t k = wide ? k_norm_mx4<X16, R, 4, true> : A.cols > 512 ? k_norm_mx4<X16, R, 4, false> : k_norm_mx4<X16, R, 1, false>;
        if (bytes > 65536) {
            const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
            if (err != hipSuccess) {
                sl_note_hip_error(err);
                return SL_ERR_HIP;
            }
        }
        hipLaunchKernelGGL(k, dim3(groups), dim3(1024), bytes, st, A, pitch);
        return check_launch();
    }
    const unsigned four = (unsigned)((A.rows + 3) / 4), one = (unsigned)A.rows;
    if (A.cols <= 512) hipLaunchKernelGGL((k_norm<X16, R, 1, 1, false>), dim3(four), dim3(256), 0, st, A);
    else if (A.cols <= 2048) hipLaunchKernelGGL((k_norm<X16, R, 1, 4, false>), dim3(four), dim3(256), 0, st, A);
    else if (A.cols <= 8192) hipLaunchKernelGGL((k_norm<X16, R, 4, 4, false>), dim3(one), dim3(256), 0, st, A);
    else if (A.cols <= WIDE) hipLaunchKernelGGL((k_norm<X16, R, 16, 4, false>), dim3(one), dim3(1024), 0, st, A);
    else hipLaunchKernelGGL((k_norm<X16, R, 16, 4, true>), dim3(one), dim3(1024), 0, st, A);
    return check_launch();
}

long long group_count(long long rows, long long &per)
{
    per = std::max<long long>((rows + GROUPS - 1) / GROUPS, std::min<long long>(rows, 4));
    return (rows + per - 1) / per;
}

template <bool H16, bool DY16, bool DX16>
int launch_back(const BackArgs &A, hipStream_t st)
{
    long long per;
    const unsigned groups = (unsigned)group_count(A.rows, per);
    if (A.cols <= 512) hipLaunchKernelGGL((k_back<H16, DY16, DX16, 1, 1, false>), dim3(groups), dim3(256), 0, st, A, per);
    else if (A.cols <= 2048) hipLaunchKernelGGL((k_back<H16, DY16, DX16, 1, 4, false>), dim3(groups), dim3(256), 0, st, A, per);
    else if (A.cols <= 8192) hipLaunchKernelGGL((k_back<H16, DY16, DX16, 4, 4, false>), dim3(groups), dim3(256), 0, st, A, per);
    else if (A.cols <= WIDE / 2) hipLaunchKernelGGL((k_back<H16, DY16, DX16, 16, 2, false>), dim3(groups), dim3(1024), 0, st, A, per);
    else {
        hipLaunchKernelGGL((k_back<H16, DY16, DX16, 16, 2, true>), dim3(groups), dim3(1024), 0, st, A, per);
        if (A.parts) {
            if (const int rc = check_launch()) return rc;
            hipLaunchKernelGGL((k_column_sums<H16, DY16>), dim3((unsigned)((A.cols + 255) / 256), groups), dim3(256), 0, st, A, per);
        }
    }
    return check_launch();
}

const int64_t MOST_ROWS = (int64_t)1 << 21, MOST_COLS = (int64_t)1 << 20;

}  // namespace

extern "C" {

int sl_rms_norm(const void *x, int x_type, int64_t ldx, const void *residual, int64_t ldr, void *h, int h_type, int64_t ldh,
                const void *weight, int w_type, int64_t rows, int64_t cols, double eps, void *y, int y_type, int64_t ldy, float *rstd,
                void *q, void *qt, void *stream)
{
    if (rows < 0 || cols < 0 || rows > MOST_ROWS || cols > MOST_COLS) return SL_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return SL_OK;
    if (!x || !weight || (!h) != (!residual) || (!y && !rstd && !q && !qt && !h) || !(eps >= 1e-30) || !std::isfinite(eps)) return SL_ERR_INVALID_ARG;
    if (bad_type(x_type) || bad_type(w_type) || (h && bad_type(h_type)) || (y && bad_type(y_type))) return SL_ERR_INVALID_ARG;
    if (bad_matrix(x, x_type, cols, ldx) || bad_matrix(weight, w_type, cols, cols) || (h && (bad_matrix(h, h_type, cols, ldh) || bad_matrix(residual, h_type, cols, ldr))) ||
        (y && bad_matrix(y, y_type, cols, ldy)) || ((uintptr_t)rstd & 3) || ((uintptr_t)q & 15) || ((uintptr_t)qt & 15))
        return SL_ERR_INVALID_ARG;
    const void *out[5] = {h, y, rstd, q, qt};
    for (int i = 0; i < 5; ++i) {
        if (!out[i]) continue;
        if (out[i] == x || out[i] == weight || (out[i] == residual && (i != 0 || ldh != ldr))) return SL_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (out[i] == out[j]) return SL_ERR_INVALID_ARG;
    }
    NormArgs A = {};
    if ((q && !sl_mx4_shape(rows, cols, A.s)) || (qt && !sl_mx4_shape(cols, rows, A.t))) return SL_ERR_INVALID_ARG;
    A.x = x, A.residual = residual, A.w = weight, A.h = h, A.y = y, A.rstd = rstd;
    A.q = static_cast<unsigned char *>(q), A.qt = static_cast<unsigned char *>(qt);
    A.rows = rows, A.cols = cols, A.ldx = ldx, A.ldr = ldr, A.ldh = ldh, A.ldy = ldy, A.eps = eps;
    A.w16 = w_type == SL_TYPE_BF16, A.y16 = y_type == SL_TYPE_BF16;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int r = !h ? NONE : h_type == SL_TYPE_F32 ? F32 : B16;
    if (x_type == SL_TYPE_BF16) return r == NONE ? launch_norm<true, NONE>(A, st) : r == F32 ? launch_norm<true, F32>(A, st) : launch_norm<true, B16>(A, st);
    return r == NONE ? launch_norm<false, NONE>(A, st) : r == F32 ? launch_norm<false, F32>(A, st) : launch_norm<false, B16>(A, st);
}

size_t sl_rms_norm_workspace_bytes(int64_t rows, int64_t cols)
{
    if (rows < 1 || cols < 1 || rows > MOST_ROWS || cols > MOST_COLS) return 0;
    return sizeof(float) * (size_t)(std::min<int64_t>(rows, GROUPS) * cols);
}

int sl_rms_norm_backward(const void *h, int h_type, int64_t ldh, const void *weight, int w_type, const float *rstd, const void *dy,
                         int dy_type, int64_t lddy, const void *dh, int64_t lddh, void *dx, int dx_type, int64_t lddx, float *dw,
                         int accumulate, int64_t rows, int64_t cols, void *workspace, void *stream)
{
    if (rows < 0 || cols < 0 || rows > MOST_ROWS || cols > MOST_COLS) return SL_ERR_INVALID_ARG;
    if (cols == 0) return SL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows == 0) {                                          // sums of nothing
        if (!dw || accumulate) return SL_OK;
        if ((uintptr_t)dw & 3) return SL_ERR_INVALID_ARG;
        hipLaunchKernelGGL(k_join_dw, dim3((unsigned)((cols + 63) / 64)), dim3(1024), 0, st, (const float *)nullptr, 0, cols, dw, 0);
        return check_launch();
    }
    if (!h || !weight || !rstd || !dy || !dx || (dw && !workspace)) return SL_ERR_INVALID_ARG;
    if (bad_type(h_type) || bad_type(w_type) || bad_type(dy_type) || bad_type(dx_type)) return SL_ERR_INVALID_ARG;
    if (bad_matrix(h, h_type, cols, ldh) || bad_matrix(weight, w_type, cols, cols) || bad_matrix(dy, dy_type, cols, lddy) ||
        bad_matrix(dx, dx_type, cols, lddx) || (dh && bad_matrix(dh, dx_type, cols, lddh)) || ((uintptr_t)rstd & 3) || ((uintptr_t)dw & 3) ||
        (dw && ((uintptr_t)workspace & 15)))
        return SL_ERR_INVALID_ARG;
    if (dx == h || dx == dy || dx == weight || dx == rstd || (dx == dh && lddx != lddh)) return SL_ERR_INVALID_ARG;
    if (dw && (dw == dx || dw == weight || dw == workspace || workspace == dx)) return SL_ERR_INVALID_ARG;
    BackArgs A = {};
    A.h = h, A.w = weight, A.dy = dy, A.dh = dh, A.rstd = rstd, A.dx = dx, A.parts = dw ? static_cast<float *>(workspace) : nullptr;
    A.rows = rows, A.cols = cols, A.ldh = ldh, A.lddy = lddy, A.lddh = lddh, A.lddx = lddx, A.w16 = w_type == SL_TYPE_BF16;
    typedef int (*launch_t)(const BackArgs &, hipStream_t);
    static const launch_t table[8] = {launch_back<false, false, false>, launch_back<false, false, true>, launch_back<false, true, false>,
                                      launch_back<false, true, true>, launch_back<true, false, false>, launch_back<true, false, true>,
                                      launch_back<true, true, false>, launch_back<true, true, true>};
    if (const int rc = table[(h_type == SL_TYPE_BF16) * 4 + (dy_type == SL_TYPE_BF16) * 2 + (dx_type == SL_TYPE_BF16)](A, st)) return rc;
    if (!dw) return SL_OK;
    long long per;
    const int groups = (int)group_count(rows, per);
    hipLaunchKernelGGL(k_join_dw, dim3((unsigned)((cols + 63) / 64)), dim3(1024), 0, st, A.parts, groups, cols, dw, accumulate);
    return check_launch();
}

}  // extern "C"
