// The inner step's optimiser: AdamW over a list of tensors with its moments in 32 or in 8 bits, and the global norm of
// the gradients.  All of it is streams over flat arenas, bound by memory: a unit is up to 4096 consecutive elements
// of one tensor and belongs to one workgroup of four waves, wave w of which takes elements 1024 i + 256 w .. + 255 in
// access i - one block of the 8-bit states, whose largest value is then a maximum over the wave's registers.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <type_traits>
#include <vector>

#include "sl_device.h"
#include "sl_internal.h"
#include "sl_mx4.h"

namespace {

enum { UNIT = 4096, BLOCK = 256, NORM_GROUPS = 2048, NORM_UNITS = 4, MAX_UNITS = (1 << 24) - 1 };   // (a grid has less than 2^32 threads)

struct Unit {               // one 32-byte scalar load
    long long base;         // first element in the arenas
    int block0;             // its first block in the list
    int count;              // elements, 1 .. UNIT
    float decay;            // the tensor's factor on the weight decay
    int reserved[3];
};
static_assert(sizeof(Unit) == 32, "descriptor is one 32-byte load");

}  // namespace

struct sl_adamw {
    int device;
    int64_t n_units, n_blocks;
    Unit *d_units;
};

namespace {

// Four elements at element p of a gradient arena, of which `n` exist; what does not comes as +0.0f.
template <bool B16>
SL_DEV sl_f4 load_grad(const void *arena, long long p, int n)
{
    if constexpr (B16) {
        const unsigned short *g = static_cast<const unsigned short *>(arena) + p;
        unsigned lo = 0, hi = 0;
        if (n >= 4) {
            typedef unsigned u2 __attribute__((ext_vector_type(2)));
            const u2 w = __builtin_nontemporal_load(reinterpret_cast<const u2 *>(g));
            lo = w.x, hi = w.y;
        } else {
            if (n > 0) lo = g[0];
            if (n > 1) lo |= (unsigned)g[1] << 16;
            if (n > 2) hi = g[2];
        }
        return sl_f4{__uint_as_float(lo << 16), __uint_as_float(lo & 0xFFFF0000u), __uint_as_float(hi << 16),
                     __uint_as_float(hi & 0xFFFF0000u)};
    } else {
        return sl_load_edge(static_cast<const float *>(arena) + p, n);
    }
}

SL_DEV void store_bf16(unsigned short *p, int n, sl_f4 v)
{
    if (n >= 4) {
        typedef unsigned u2 __attribute__((ext_vector_type(2)));
        u2 w;
        w.x = sl_bf16_pair(v.x, v.y);
        w.y = sl_bf16_pair(v.z, v.w);
        __builtin_nontemporal_store(w, reinterpret_cast<u2 *>(p));
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c < n) p[c] = (unsigned short)sl_bf16_bits(v[c]);
    }
}

struct StepArgs {
    const Unit *units;
    float *theta;
    const void *grad;
    float *m, *v;                    // 32-bit states
    unsigned char *m8, *v8;          // 8-bit states
    unsigned char *ms, *vs;
    const float *grad_scale;
    unsigned short *theta16;
    float b1, c1, b2, c2;            // beta1, 1 - beta1, beta2, 1 - beta2
    float rate, r, eps, shrink;      // lr/(1 - beta1^t), 1/sqrt(1 - beta2^t), eps, lr * weight_decay
    unsigned seed_hash;
    unsigned order;                  // sl_work_group
};

// LDS that a workgroup of a long list asks for and does not use: two fit a compute unit then (see sl_outer.hip).
enum { STREAM_LDS = 54272, STREAM8_LDS = 40960, SHORT_UNITS = 4096 };

// One element: moments and parameter brought up to date.
SL_DEV void adamw_update(const StepArgs &A, float keep, float scale, float grad, float &theta, float &m, float &v)
{
    const float g = grad * scale;
    m = m * A.b1 + g * A.c1;
    v = v * A.b2 + (g * g) * A.c2;
    const float den = __fsqrt_rn(v) * A.r + A.eps;
    theta = theta * keep - __fdiv_rn(m * A.rate, den);
}

// Long lists take one access of a unit after the other, with two workgroups to a compute unit (STREAM_LDS) and the
// units in the order of sl_work_group: with more under way the memory has more rows open than it keeps.  Short ones, which give
// a compute unit a few workgroups only, request a whole unit at once (SHORT).  us, so / SHORT: 1M elements 6.4 / 6.2, 4M
// 23.6 / 20.0, 16M 80.9 / 80.3, 64M 315 / 322, 1.8B 8700 / 9260 (5.8 and 5.5 TB/s; 9250 without the order, 9180 with four
// workgroups); two or four accesses at once on the 1.8B list 9070 and 9180.
template <bool B16, bool SHORT>
__global__ void __launch_bounds__(256) k_adamw(StepArgs A)
{
    const Unit u = A.units[SHORT ? blockIdx.x : sl_work_group(blockIdx.x, A.order)];
    const float scale = A.grad_scale ? *A.grad_scale : 1.0f;
    if (scale != scale) return;
    const float keep = 1.0f - u.decay * A.shrink;
    constexpr int STEP = SHORT ? 4 : 1;
    auto part = [&](int q, auto is_full) __attribute__((always_inline)) {
        constexpr bool full = decltype(is_full)::value;
        auto place = [&](int i) -> long long { return u.base + ((q * STEP + i) * 1024 + (int)threadIdx.x * 4); };
        auto exist = [&](int i) -> int { return full ? 4 : u.count - ((q * STEP + i) * 1024 + (int)threadIdx.x * 4); };
        sl_f4 g[STEP], th[STEP], m[STEP], v[STEP];
#pragma unroll
        for (int i = 0; i < STEP; ++i) g[i] = load_grad<B16>(A.grad, place(i), exist(i));
#pragma unroll
        for (int i = 0; i < STEP; ++i) th[i] = sl_load_edge(A.theta + place(i), exist(i));
#pragma unroll
        for (int i = 0; i < STEP; ++i) m[i] = sl_load_edge(A.m + place(i), exist(i));
#pragma unroll
        for (int i = 0; i < STEP; ++i) v[i] = sl_load_edge(A.v + place(i), exist(i));
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float t = th[i][c], mm = m[i][c], vv = v[i][c];
                adamw_update(A, keep, scale, g[i][c], t, mm, vv);
                th[i][c] = t, m[i][c] = mm, v[i][c] = vv;
            }
            sl_store_edge(A.theta + place(i), exist(i), th[i]);
            sl_store_edge(A.m + place(i), exist(i), m[i]);
            sl_store_edge(A.v + place(i), exist(i), v[i]);
            if (A.theta16) store_bf16(A.theta16 + place(i), exist(i), th[i]);
        }
    };
    if (u.count == UNIT) {
#pragma unroll 1
        for (int q = 0; q < UNIT / 1024 / STEP; ++q) part(q, std::true_type{});
    } else {
#pragma unroll 1
        for (int q = 0; q < UNIT / 1024 / STEP; ++q) part(q, std::false_type{});
    }
}

// ---- 8-bit states ----

SL_DEV unsigned fmix(unsigned h)
{
    h ^= h >> 16;
    h *= 0x85EBCA6Bu;
    h ^= h >> 13;
    h *= 0xC2B2AE35u;
    return h ^ (h >> 16);
}

SL_DEV unsigned load_codes(const unsigned char *p, int n)
{
    if (n >= 4) return *reinterpret_cast<const unsigned *>(p);
    unsigned w = 0;
    if (n > 0) w = p[0];
    if (n > 1) w |= (unsigned)p[1] << 8;
    if (n > 2) w |= (unsigned)p[2] << 16;
    return w;
}

SL_DEV void store_codes(unsigned char *p, int n, unsigned w)
{
    if (n >= 4) {
        *reinterpret_cast<unsigned *>(p) = w;
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c < n) p[c] = (unsigned char)(w >> (8 * c));
    }
}

SL_DEV float block_scale(unsigned x) { return x == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(x << 23); }

// The codes are the upper bits of an fp32 number: exponent and three mantissa bits, shifted so that the format's
// subnormals are fp32's.  Both factors are exact (2^112: four exponent bits, 2^96: five).
SL_DEV float decode_m(unsigned c, float scale)
{
    const float x = __uint_as_float((c & 127u) << 20) * 0x1p112f;
    return (c & 128u ? -x : x) * scale;
}
SL_DEV float decode_v(unsigned c, float scale) { return __uint_as_float(c << 20) * 0x1p96f * scale; }

// Scale byte for a block whose largest magnitude has these bits.
SL_DEV unsigned scale_byte(int top)
{
    if (top >= 0x7F800000) return 255u;
    const int x = (top + 0xFFFFF) >> 23;
    return (unsigned)min(max(x, 1), 253);
}
SL_DEV unsigned encode_m(float x, float inv, unsigned rnd)
{
    const unsigned b = __float_as_uint(fabsf(x) * inv * 0x1p-112f);
    return min((b + rnd) >> 20, 127u) | (x < 0.0f ? 128u : 0u);
}
SL_DEV unsigned encode_v(float x, float inv, unsigned rnd)
{
    const unsigned b = __float_as_uint(x * inv * 0x1p-96f);
    return max(min((b + rnd) >> 20, 255u), x > 0.0f ? 1u : 0u);
}

// A wave has a block per access; a unit's four accesses are requested together.  Long lists: four workgroups to a compute
// unit (STREAM8_LDS) in the order of sl_work_group, as in k_adamw.  us, so / as many workgroups as the registers allow, in list order: 64M
// elements 176 / 174, 256M 740 / 802, 1.8B 5008 / 5396 (5.8 and 5.4 TB/s); two accesses at a time 5084, with two workgroups 7174; a lane with eight
// elements in place of four writes its theta in pieces of 16 bytes that the streaming hint sends to memory by themselves: 6672 at best.
template <bool B16, bool SHORT>
__global__ void __launch_bounds__(256) k_adamw8(StepArgs A)
{
    const Unit u = A.units[SHORT ? blockIdx.x : sl_work_group(blockIdx.x, A.order)];
    const float scale = A.grad_scale ? *A.grad_scale : 1.0f;
    if (scale != scale) return;
    const float keep = 1.0f - u.decay * A.shrink;
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6));
    constexpr int STEP = UNIT / 1024;
    auto all = [&](auto is_full) __attribute__((always_inline)) {
        constexpr bool full = decltype(is_full)::value;
        sl_f4 g[STEP], th[STEP];
        unsigned cm[STEP], cv[STEP];
        float sm[STEP], sv[STEP];
        // access i: a block of the wave; one that does not exist is read as the unit's first, and not written
        auto first = [&](int i) -> int { return i * 1024 + wave * BLOCK; };
        auto exist = [&](int i) -> int { return full ? 4 : u.count - first(i) - lane * 4; };
        auto has = [&](int i) -> bool { return full || first(i) < u.count; };
        auto place = [&](int i) -> long long { return u.base + (first(i) + lane * 4); };
        auto block = [&](int i) -> int { return u.block0 + (has(i) ? first(i) / BLOCK : 0); };
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
            g[i] = load_grad<B16>(A.grad, place(i), exist(i));
            th[i] = sl_load_edge(A.theta + place(i), exist(i));
            cm[i] = load_codes(A.m8 + place(i), exist(i)), cv[i] = load_codes(A.v8 + place(i), exist(i));
            sm[i] = block_scale(A.ms[block(i)]), sv[i] = block_scale(A.vs[block(i)]);
        }
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
            const int n = exist(i);
            float m[4], v[4];
            int top_m = 0, top_v = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                m[c] = decode_m(cm[i] >> (8 * c) & 255u, sm[i]);
                v[c] = decode_v(cv[i] >> (8 * c) & 255u, sv[i]);
                float t = th[i][c];
                adamw_update(A, keep, scale, g[i][c], t, m[c], v[c]);
                th[i][c] = t;
                if (c >= n) m[c] = v[c] = 0.0f;           // places that do not exist count for nothing
                top_m = max(top_m, __float_as_int(m[c]) & 0x7FFFFFFF);
                top_v = max(top_v, __float_as_int(v[c]) & 0x7FFFFFFF);
            }
            const unsigned xm = scale_byte(sl_wave_max(top_m)), xv = scale_byte(sl_wave_max(top_v));
            const float im = __uint_as_float((254u - min(xm, 253u)) << 23), iv = __uint_as_float((254u - min(xv, 253u)) << 23);
            const unsigned key = fmix(A.seed_hash ^ (unsigned)block(i));
            unsigned om = 0, ov = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const unsigned h = fmix(key ^ (unsigned)(lane * 4 + c));
                om |= encode_m(m[c], im, (h & 0xFFFFu) << 4 | 8u) << (8 * c);
                ov |= encode_v(v[c], iv, (h >> 16) << 4 | 8u) << (8 * c);
            }
            if (xm == 255u) om = 0;
            if (xv == 255u) ov = 0;
            sl_store_edge(A.theta + place(i), n, th[i]);
            store_codes(A.m8 + place(i), n, om);
            store_codes(A.v8 + place(i), n, ov);
            if (A.theta16) store_bf16(A.theta16 + place(i), n, th[i]);
            if (lane == 0 && has(i)) A.ms[block(i)] = (unsigned char)xm, A.vs[block(i)] = (unsigned char)xv;
        }
    };
    if (u.count == UNIT) all(std::true_type{});
    else all(std::false_type{});
}

template <bool V>
__global__ void __launch_bounds__(256) k_state_values(const Unit *units, const unsigned char *codes,
                                                      const unsigned char *scales, float *values)
{
    const Unit u = units[blockIdx.x];
#pragma unroll
    for (int i = 0; i < UNIT / 1024; ++i) {
        const int at = i * 1024 + (int)threadIdx.x * 4, n = u.count - at;
        if (n <= 0) return;
        const long long p = u.base + at;
        const unsigned w = load_codes(codes + p, n);
        const float s = block_scale(scales[u.block0 + at / BLOCK]);
        sl_f4 x;
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = V ? decode_v(w >> (8 * c) & 255u, s) : decode_m(w >> (8 * c) & 255u, s);
        sl_store_edge(values + p, n, x);
    }
}

// ---- norm of the gradients ----

// Sum over the workgroup in a fixed order, in thread 0.
SL_DEV double group_sum(double x)
{
    __shared__ double part[4];
    const double w = sl_wave_tree0(x, 6);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = w;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// fp64: the square of an fp32 number and its sums neither overflow nor vanish there.  A workgroup takes NORM_UNITS consecutive
// units at a time, all of them requested before the first is added: 8 accesses of 16 bytes per lane in flight (bf16), where one unit
// at a time reads 64M bf16 in 35 us and the 1.8B list in 677, this 24.6 and 530 to 553 (6.6 to 6.9 TB/s).
template <bool B16>
__global__ void __launch_bounds__(256) k_norm_parts(const Unit *units, long long n_units, const void *grad, double *parts)
{
    double sum = 0.0;
    for (long long t0 = (long long)blockIdx.x * NORM_UNITS; t0 < n_units; t0 += (long long)gridDim.x * NORM_UNITS) {
        SlOctet<B16> g[NORM_UNITS][UNIT / 2048];
#pragma unroll
        for (int k = 0; k < NORM_UNITS; ++k) {
            const Unit u = units[min(t0 + k, n_units - 1)];
            const int count = t0 + k < n_units ? u.count : 0;
#pragma unroll
            for (int i = 0; i < UNIT / 2048; ++i) {
                const int at = i * 2048 + (int)threadIdx.x * 8;
                g[k][i].load(grad, u.base + at, count - at);
            }
        }
#pragma unroll
        for (int k = 0; k < NORM_UNITS; ++k)
#pragma unroll
            for (int i = 0; i < UNIT / 2048; ++i) {
                double s[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const double x = g[k][i].value(c);
                    s[c] = x * x;
                }
                sum += ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
            }
    }
    sum = group_sum(sum);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(256) k_norm_result(const double *parts, int n, float max_norm, float *result)
{
    double part[NORM_GROUPS / 256], sum = 0.0;
#pragma unroll
    for (int k = 0; k < NORM_GROUPS / 256; ++k) {              // (all requested at once)
        const int i = k * 256 + (int)threadIdx.x;
        part[k] = i < n ? parts[i] : 0.0;
    }
#pragma unroll
    for (int k = 0; k < NORM_GROUPS / 256; ++k) sum += part[k];
    sum = group_sum(sum);
    if (threadIdx.x == 0) {
        const double norm = sqrt(sum);
        result[0] = (float)norm;
        result[1] = !(norm < (double)INFINITY) ? __uint_as_float(0x7FC00000u) : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f;
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

int check_device(const sl_adamw *o)
{
    int dev = -1;
    const hipError_t err = hipGetDevice(&dev);
    if (err != hipSuccess) {
        sl_note_hip_error(err);
        return SL_ERR_HIP;
    }
    return dev == o->device ? SL_OK : SL_ERR_DEVICE;
}

bool bad_type(int t) { return t != SL_TYPE_F32 && t != SL_TYPE_BF16; }

// The constants of a step; false where a parameter is out of range, or a constant in fp32: an eps that is 0 there divides 0 by 0
// wherever a gradient has always been zero, an infinite factor makes NaN of the zeros it meets.
bool step_constants(const sl_adamw_params *P, StepArgs &A)
{
    if (!P || P->step < 1) return false;
    if (!(P->beta1 >= 0.0 && P->beta1 < 1.0) || !(P->beta2 >= 0.0 && P->beta2 < 1.0)) return false;
    if (!(P->eps > 0.0) || !std::isfinite(P->eps) || !std::isfinite(P->lr) || !std::isfinite(P->weight_decay)) return false;
    A.b1 = (float)P->beta1, A.c1 = (float)(1.0 - P->beta1);
    A.b2 = (float)P->beta2, A.c2 = (float)(1.0 - P->beta2);
    A.rate = (float)(P->lr / (1.0 - std::pow(P->beta1, (double)P->step)));
    A.r = (float)(1.0 / std::sqrt(1.0 - std::pow(P->beta2, (double)P->step)));
    A.eps = (float)P->eps;
    A.shrink = (float)(P->lr * P->weight_decay);
    return A.eps > 0.0f && std::isfinite(A.eps) && std::isfinite(A.rate) && std::isfinite(A.r) && std::isfinite(A.shrink);
}

unsigned host_fmix(unsigned h)
{
    h ^= h >> 16;
    h *= 0x85EBCA6Bu;
    h ^= h >> 13;
    h *= 0xC2B2AE35u;
    return h ^ (h >> 16);
}

}  // namespace

extern "C" {

int sl_adamw_create(const sl_tensor *tensors, int n_tensors, const float *decay, sl_adamw **out)
{
    if (!out) return SL_ERR_INVALID_ARG;
    *out = nullptr;
    if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return SL_ERR_INVALID_ARG;
    std::vector<Unit> units;
    int64_t blocks = 0, n_units = 0;
    try {
        std::vector<std::pair<int64_t, int64_t>> span;
        span.reserve((size_t)n_tensors);
        for (int t = 0; t < n_tensors; ++t) {
            const sl_tensor &T = tensors[t];
            if (T.rows < 1 || T.cols < 1 || T.offset < 0 || (T.offset & 3) || T.reserved != 0) return SL_ERR_INVALID_ARG;
            if (T.layout != SL_LAYOUT_FLAT && T.layout != SL_LAYOUT_TILE64) return SL_ERR_INVALID_ARG;
            if (T.rows > ((int64_t)1 << 40) / T.cols || T.offset > ((int64_t)1 << 60)) return SL_ERR_INVALID_ARG;
            if (decay && !std::isfinite(decay[t])) return SL_ERR_INVALID_ARG;
            span.emplace_back(T.offset, T.offset + T.rows * T.cols);
            n_units += (T.rows * T.cols + UNIT - 1) / UNIT;
            if (n_units > MAX_UNITS) return SL_ERR_INVALID_ARG;
        }
        std::sort(span.begin(), span.end());
        for (size_t i = 1; i < span.size(); ++i)
            if (span[i].first < span[i - 1].second) return SL_ERR_INVALID_ARG;
        units.reserve((size_t)n_units);
        for (int t = 0; t < n_tensors; ++t) {
            const sl_tensor &T = tensors[t];
            const int64_t n = T.rows * T.cols;
            for (int64_t a = 0; a < n; a += UNIT) {
                Unit u;
                std::memset(&u, 0, sizeof(u));
                u.base = T.offset + a;
                u.block0 = (int)(blocks + a / BLOCK);
                u.count = (int)std::min<int64_t>(UNIT, n - a);
                u.decay = decay ? decay[t] : 1.0f;
                units.push_back(u);
            }
            blocks += (n + BLOCK - 1) / BLOCK;
        }
    } catch (const std::bad_alloc &) {
        return SL_ERR_NOMEM;
    }
    sl_adamw *o = new (std::nothrow) sl_adamw();
    if (!o) return SL_ERR_NOMEM;
    o->n_units = (int64_t)units.size();
    o->n_blocks = blocks;
    o->d_units = nullptr;
    hipError_t err = hipGetDevice(&o->device);
    if (err == hipSuccess && !units.empty()) {
        const size_t bytes = units.size() * sizeof(Unit);
        if ((err = hipMalloc((void **)&o->d_units, bytes)) == hipSuccess)
            err = hipMemcpy(o->d_units, units.data(), bytes, hipMemcpyHostToDevice);
    }
    if (err != hipSuccess) {
        sl_note_hip_error(err);
        sl_adamw_destroy(o);
        return err == hipErrorOutOfMemory ? SL_ERR_NOMEM : SL_ERR_HIP;
    }
    *out = o;
    return SL_OK;
}

int sl_adamw_destroy(sl_adamw *o)
{
    if (!o) return SL_OK;
    if (o->d_units) (void)hipFree(o->d_units);
    delete o;
    return SL_OK;
}

int64_t sl_adamw_num_blocks(const sl_adamw *o) { return o ? o->n_blocks : -1; }
size_t sl_grad_norm_workspace_bytes(const sl_adamw *o) { return o ? NORM_GROUPS * sizeof(double) : 0; }

int sl_grad_norm(sl_adamw *o, const void *grad, int grad_type, float max_norm, float *result, void *workspace,
                 void *stream)
{
    if (!o || !grad || !result || !workspace || bad_type(grad_type) || !(max_norm > 0.0f)) return SL_ERR_INVALID_ARG;
    if (misaligned(grad, 16) || misaligned(result, 4) || misaligned(workspace, 256)) return SL_ERR_INVALID_ARG;
    if (const int rc = check_device(o)) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    double *parts = static_cast<double *>(workspace);
    const int groups = (int)std::min<int64_t>((o->n_units + NORM_UNITS - 1) / NORM_UNITS, NORM_GROUPS);
    if (groups > 0)
        hipLaunchKernelGGL(grad_type == SL_TYPE_BF16 ? k_norm_parts<true> : k_norm_parts<false>, dim3(groups), dim3(256), 0, st,
                           o->d_units, (long long)o->n_units, grad, parts);
    hipLaunchKernelGGL(k_norm_result, dim3(1), dim3(256), 0, st, parts, groups, max_norm, result);
    return check_launch();
}

int sl_adamw_step(sl_adamw *o, float *theta, const void *grad, int grad_type, float *m, float *v,
                  const sl_adamw_params *params, const float *grad_scale, void *theta16, void *stream)
{
    StepArgs A;
    std::memset(&A, 0, sizeof(A));
    if (!o || !theta || !grad || !m || !v || bad_type(grad_type) || !step_constants(params, A)) return SL_ERR_INVALID_ARG;
    if (theta == m || theta == v || m == v || grad == theta || grad == m || grad == v || theta16 == theta || theta16 == m ||
        theta16 == v || theta16 == grad)
        return SL_ERR_INVALID_ARG;
    if (misaligned(theta, 16) || misaligned(grad, 16) || misaligned(m, 16) || misaligned(v, 16) || misaligned(theta16, 16) ||
        misaligned(grad_scale, 4))
        return SL_ERR_INVALID_ARG;
    if (const int rc = check_device(o)) return rc;
    if (o->n_units == 0) return SL_OK;
    A.units = o->d_units, A.theta = theta, A.grad = grad, A.m = m, A.v = v, A.grad_scale = grad_scale;
    A.theta16 = static_cast<unsigned short *>(theta16);
    A.order = (unsigned)o->n_units / SL_ORDER_WINDOW * SL_ORDER_WINDOW;
    const bool b16 = grad_type == SL_TYPE_BF16, is_short = o->n_units < SHORT_UNITS;
    hipLaunchKernelGGL(is_short ? (b16 ? k_adamw<true, true> : k_adamw<false, true>) : (b16 ? k_adamw<true, false> : k_adamw<false, false>),
                       dim3((unsigned)o->n_units), dim3(256), is_short ? 0 : STREAM_LDS, static_cast<hipStream_t>(stream), A);
    return check_launch();
}

int sl_adamw_step8(sl_adamw *o, float *theta, const void *grad, int grad_type, uint8_t *m_codes, uint8_t *v_codes,
                   uint8_t *m_scales, uint8_t *v_scales, uint32_t seed, const sl_adamw_params *params,
                   const float *grad_scale, void *theta16, void *stream)
{
    StepArgs A;
    std::memset(&A, 0, sizeof(A));
    if (!o || !theta || !grad || !m_codes || !v_codes || !m_scales || !v_scales || bad_type(grad_type) || !step_constants(params, A))
        return SL_ERR_INVALID_ARG;
    const void *all[7] = {theta, grad, m_codes, v_codes, m_scales, v_scales, theta16};
    for (int i = 0; i < 7; ++i)
        for (int j = 0; j < i; ++j)
            if (all[i] == all[j]) return SL_ERR_INVALID_ARG;
    if (misaligned(theta, 16) || misaligned(grad, 16) || misaligned(m_codes, 16) || misaligned(v_codes, 16) ||
        misaligned(theta16, 16) || misaligned(grad_scale, 4))
        return SL_ERR_INVALID_ARG;
    if (const int rc = check_device(o)) return rc;
    if (o->n_units == 0) return SL_OK;
    A.units = o->d_units, A.theta = theta, A.grad = grad, A.grad_scale = grad_scale;
    A.order = (unsigned)o->n_units / SL_ORDER_WINDOW * SL_ORDER_WINDOW;
    A.m8 = m_codes, A.v8 = v_codes, A.ms = m_scales, A.vs = v_scales;
    A.seed_hash = host_fmix(seed);
    A.theta16 = static_cast<unsigned short *>(theta16);
    const bool b16 = grad_type == SL_TYPE_BF16, is_short = o->n_units < SHORT_UNITS;
    hipLaunchKernelGGL(is_short ? (b16 ? k_adamw8<true, true> : k_adamw8<false, true>) : (b16 ? k_adamw8<true, false> : k_adamw8<false, false>),
                       dim3((unsigned)o->n_units), dim3(256), is_short ? 0 : STREAM8_LDS, static_cast<hipStream_t>(stream), A);
    return check_launch();
}

int sl_adamw_state_values(sl_adamw *o, int moment, const uint8_t *codes, const uint8_t *scales, float *values,
                          void *stream)
{
    if (!o || !codes || !scales || !values || (moment != 1 && moment != 2)) return SL_ERR_INVALID_ARG;
    if (misaligned(codes, 16) || misaligned(values, 16) || (const void *)codes == values || (const void *)scales == values)
        return SL_ERR_INVALID_ARG;
    if (const int rc = check_device(o)) return rc;
    if (o->n_units == 0) return SL_OK;
    hipLaunchKernelGGL(moment == 2 ? k_state_values<true> : k_state_values<false>, dim3((unsigned)o->n_units), dim3(256), 0,
                       static_cast<hipStream_t>(stream), o->d_units, codes, scales, values);
    return check_launch();
}

}  // extern "C"
