// Loss of tokens from their logits and its gradient: negative log-likelihood, or the clipped ratio of a policy step with a KL term.
//   logp = z_t - log sum exp z ;  dz = w l'(logp) (onehot(t) - softmax(z))
// l' needs no other token, so that one launch does both ways: a workgroup reads a row into registers, knows its largest value and its sum of
// exponentials after two barriers, and writes the gradient from the registers - bound by memory, one read and one write of the logits.
// The exponentials are fp32, what a row has one of (the sums across lanes, logp, the ratio, the loss) is 64 bits: log ratios are
// differences of numbers near each other, and on the border of the clipped range one rounding decides between a gradient and none.
#include <algorithm>
#include <cmath>

#include "sl_internal.h"
#include "sl_mx4.h"

namespace {

const float LOG2E = 1.44269504088896340736f;

struct LossArgs {
    const void *logits;
    void *dlogits;
    const long long *targets;
    const float *weights, *old_logp, *advantage, *ref_logp;
    float *logp;
    double *each;                    // the rows' losses
    long long ld, ldd, rows, vocab;
    double low, high, kl;            // 1 - clip_low, 1 + clip_high
    int policy;
};

SL_DEV float wave_max(float v)
{
#pragma unroll
    for (int l = 0; l < 6; ++l) v = __builtin_elementwise_maximum(v, __int_as_float(sl_partner(__float_as_int(v), l)));
    return v;
}

template <int WAVES>
SL_DEV float all_max(float v, float *room, int wave, int lane)
{
    v = wave_max(v);
    if constexpr (WAVES > 1) {
        if (lane == 0) room[wave] = v;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v = __builtin_elementwise_maximum(v, room[i]);
    }
    return v;
}

// Loss of a token and its derivative by logp.
SL_DEV void token_loss(const LossArgs &A, long long row, double logp, double &loss, double &slope)
{
    if (!A.policy) {
        loss = -logp, slope = -1.0;
        return;
    }
    const double a = (double)A.advantage[row], r = exp(logp - (double)A.old_logp[row]);
    // (min(r a, clip(r) a) without the product of an infinite ratio and a zero)
    const bool up = a >= 0.0, kept = up ? r <= A.high : r >= A.low;
    const double c = kept || r != r ? r : up ? A.high : A.low;
    loss = -(a * c), slope = kept || r != r ? -(a * r) : 0.0;
    if (a == 0.0) loss = r != r ? r : 0.0, slope = loss;
    if (A.kl != 0.0) {
        const double d = (double)A.ref_logp[row] - logp, e = expm1(d);
        loss = loss + A.kl * (e - d), slope = slope - A.kl * e;
    }
}

// Eight elements of a row from `col` on, of which `from` .. n - 1 exist (the row does not reach further, or begins inside them).
template <bool B16>
SL_DEV void put_octet(const LossArgs &A, long long at, int from, int n, const float (&v)[8])
{
    if constexpr (B16) {
        typedef unsigned u4a __attribute__((ext_vector_type(4), aligned(2)));
        unsigned short *o = static_cast<unsigned short *>(A.dlogits) + at;
        if (from <= 0 && n >= 8) {
            __builtin_nontemporal_store(u4a{sl_bf16_pair(v[0], v[1]), sl_bf16_pair(v[2], v[3]), sl_bf16_pair(v[4], v[5]), sl_bf16_pair(v[6], v[7])},
                                        reinterpret_cast<u4a *>(o));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= from && i < n) o[i] = (unsigned short)sl_bf16_bits(v[i]);
        }
    } else {
        typedef float f4a __attribute__((ext_vector_type(4), aligned(4)));
        float *o = static_cast<float *>(A.dlogits) + at;
        if (n >= 8) {
            *reinterpret_cast<f4a *>(o) = f4a{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f4a *>(o + 4) = f4a{v[4], v[5], v[6], v[7]};
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < n) o[i] = v[i];
        }
    }
}

// Elements that do not exist are -infinity: the largest and the sum do not see them.
template <bool B16>
SL_DEV void load_octet(const LossArgs &A, long long row, long long col, SlOctet<B16> &v)
{
    const int n = (int)max(min(A.vocab - col, 8ll), 0ll);
    if constexpr (B16) {
        if (col >= 0 && n >= 8) {
            v.load(A.logits, row * A.ld + col, 8);
        } else {
            const unsigned short *p = static_cast<const unsigned short *>(A.logits) + (row * A.ld + col);
#pragma unroll
            for (int i = 0; i < 4; ++i) v.w[i] = 0xFF80FF80u;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i >= 0 && i < n) v.w[i >> 1] = (v.w[i >> 1] & (i & 1 ? 0xFFFFu : 0xFFFF0000u)) | (unsigned)p[i] << (16 * (i & 1));
        }
    } else {
        v.load(A.logits, row * A.ld + col, n);
        if (n < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= n) v.w[i] = 0xFF800000u;
        }
    }
}

// (a NaN makes the largest one, and with it everything of the row)
template <bool B16>
SL_DEV float octet_max(const SlOctet<B16> &v, float m)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) m = __builtin_elementwise_maximum(m, v.value(i));
    return m;
}

SL_DEV float exp_at(float z, float m) { return __builtin_amdgcn_exp2f((z - m) * LOG2E); }

// One row to a team of WAVES waves, OCT times eight logits in a lane.  The exponentials take the logits' place in the registers: the
// gradient is them times the row's share, and half of the arithmetic is exponentials.  Teams are as small as the registers allow, several to
// a compute unit: one reads while another writes.  8192 x 50,257 bf16: 306 us, 5.4 TB/s (exponentials made twice, 16 waves, one team: 436).
// Rows of bf16 that begin inside 16 bytes are taken from the 16 bytes' begin on (rows of 50,257: 428 us without, 353 with aligned ones).
// (LONG: a vocabulary that does not fit the registers is read twice)
template <bool B16, int WAVES, int OCT, bool LONG>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES, OCT == 13 ? 4 : 1) k_token_loss(LossArgs A)
{
    __shared__ float tops[WAVES];
    __shared__ double sums[WAVES];
    __shared__ float told[2];
    constexpr long long STEP = WAVES * OCT * 512;
    const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : sl_uniform((int)(threadIdx.x >> 6));
    const long long row = WAVES == 1 ? blockIdx.x * 4ll + sl_uniform((int)(threadIdx.x >> 6)) : blockIdx.x;
    if (row >= A.rows) return;                    // (one wave to a row: no barrier follows)
    const bool leader = wave == 0 && lane == 0;
    const long long target = A.targets[row];
    const float weight = A.weights ? A.weights[row] : 1.0f;
    const bool there = target >= 0 && target < A.vocab, counts = there && weight != 0.0f;
    if (!counts && leader) {
        if (A.each) A.each[row] = 0.0;
        if (!there && A.logp) A.logp[row] = 0.0f;
    }
    const int pre = B16 ? (int)(((unsigned long long)A.logits >> 1) + (unsigned long long)(row * A.ld)) & 7 : 0;     // elements in front of the row
    float slope = 0.0f, share = 0.0f, m = 0.0f;
    float e[OCT][8];
    if (counts || (there && A.logp)) {
        m = -INFINITY;
        double sum = 0.0;
        const float zt = B16 ? __uint_as_float((unsigned)static_cast<const unsigned short *>(A.logits)[row * A.ld + target] << 16)
                             : static_cast<const float *>(A.logits)[row * A.ld + target];
        if constexpr (LONG) {
            float mine = -INFINITY, part = 0.0f;
            for (long long base = 0; base < A.vocab + pre; base += STEP) {
                SlOctet<B16> v[OCT];
#pragma unroll
                for (int j = 0; j < OCT; ++j) load_octet(A, row, base + ((j * WAVES + wave) * 64 + lane) * 8 - pre, v[j]);
                float now = mine;
#pragma unroll
                for (int j = 0; j < OCT; ++j) now = octet_max(v[j], now);
                if (now != mine) part = part * exp_at(mine, now), mine = now;
                const float from = mine == -INFINITY ? 0.0f : mine;
#pragma unroll
                for (int j = 0; j < OCT; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) part = part + exp_at(v[j].value(i), from);
            }
            m = all_max<WAVES>(mine, tops, wave, lane);
            sum = mine == -INFINITY ? (double)part : (double)part * (double)exp_at(mine, m);
        } else {
            SlOctet<B16> v[OCT];
#pragma unroll
            for (int j = 0; j < OCT; ++j) load_octet(A, row, ((j * WAVES + wave) * 64 + lane) * 8 - pre, v[j]);
#pragma unroll
            for (int j = 0; j < OCT; ++j) m = octet_max(v[j], m);
            m = all_max<WAVES>(m, tops, wave, lane);
            float part = 0.0f;
#pragma unroll
            for (int j = 0; j < OCT; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    e[j][i] = exp_at(v[j].value(i), m);
                    part = part + e[j][i];
                }
            sum = (double)part;
        }
        sum = sl_wave_tree(sum, 6);
        if constexpr (WAVES > 1) {
            if (lane == 0) sums[wave] = sum;
            __syncthreads();
        }
        if (leader) {
            if constexpr (WAVES > 1) {
#pragma unroll
                for (int i = 1; i < WAVES; ++i) sum = sum + sums[i];
            }
            const double logp = ((double)zt - (double)m) - log(sum);
            if (counts) {
                double loss, d;
                token_loss(A, row, logp, loss, d);
                if (A.each) A.each[row] = (double)weight * loss;
                slope = (float)((double)weight * d), share = (float)(-((double)weight * d) / sum);
                if constexpr (WAVES > 1) told[0] = slope, told[1] = share;
            }
            if (A.logp) A.logp[row] = (float)logp;        // (it may lie where the row's policy inputs did)
        }
        if (A.dlogits && counts) {
            if constexpr (WAVES > 1) {
                __syncthreads();
                slope = told[0], share = told[1];
            } else {
                slope = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(slope)));
                share = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(share)));
            }
        }
    }
    if (!A.dlogits) return;
    for (long long base = 0; base < (LONG ? A.vocab + pre : 1); base += STEP)
#pragma unroll
        for (int j = 0; j < OCT; ++j) {
            const long long col = base + ((j * WAVES + wave) * 64 + lane) * 8 - pre;
            const int n = (int)max(min(A.vocab - col, 8ll), 0ll);
            float d[8];
            if (counts) {
                if constexpr (LONG) {
                    SlOctet<B16> v;
                    load_octet(A, row, col, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] = exp_at(v.value(i), m) * share;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] = e[j][i] * share;
                }
                const long long at = target - col;
                if (at >= 0 && at < 8) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i == at) d[i] = d[i] + slope;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = 0.0f;
            }
            if (n > 0) put_octet<B16>(A, row * A.ldd + col, (int)max(-col, 0ll), n, d);
        }
}

// The rows' losses in a fixed order.
__global__ void __launch_bounds__(1024) k_join_loss(const double *each, long long rows, float *loss)
{
    __shared__ double sums[16];
    double t = 0.0;
    for (long long i = threadIdx.x; i < rows; i += 1024) t = t + each[i];
    t = sl_wave_tree(t, 6);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = t;
    __syncthreads();
    if (threadIdx.x > 0) return;
    for (int i = 1; i < 16; ++i) t = t + sums[i];
    *loss = (float)t;
}

int check_launch()
{
    const hipError_t err = hipGetLastError();
    if (err == hipSuccess) return SL_OK;
    sl_note_hip_error(err);
    return SL_ERR_HIP;
}

template <bool B16>
void launch(const LossArgs &A, hipStream_t st)
{
    // (as few waves as hold the row: 64 exponentials in a lane, and 104 where that leaves two teams of eight waves 128 registers each)
    const dim3 grid((unsigned)A.rows), four((unsigned)((A.rows + 3) / 4));
    const bool aligned = !B16 || (((uintptr_t)A.logits & 15) == 0 && A.ld % 8 == 0);
    const long long octets = (A.vocab + (aligned ? 7 : 14)) / 8;
    if (octets <= 64) hipLaunchKernelGGL((k_token_loss<B16, 1, 1, false>), four, dim3(256), 0, st, A);
    else if (octets <= 128) hipLaunchKernelGGL((k_token_loss<B16, 1, 2, false>), four, dim3(256), 0, st, A);
    else if (octets <= 256) hipLaunchKernelGGL((k_token_loss<B16, 1, 4, false>), four, dim3(256), 0, st, A);
    else if (octets <= 1024) hipLaunchKernelGGL((k_token_loss<B16, 4, 4, false>), grid, dim3(256), 0, st, A);
    else if (octets <= 2048) hipLaunchKernelGGL((k_token_loss<B16, 4, 8, false>), grid, dim3(256), 0, st, A);
    else if (octets <= 4096) hipLaunchKernelGGL((k_token_loss<B16, 8, 8, false>), grid, dim3(512), 0, st, A);
    else if (octets <= 6656) hipLaunchKernelGGL((k_token_loss<B16, 8, 13, false>), grid, dim3(512), 0, st, A);
    else if (octets <= 8192) hipLaunchKernelGGL((k_token_loss<B16, 16, 8, false>), grid, dim3(1024), 0, st, A);
    else hipLaunchKernelGGL((k_token_loss<B16, 16, 4, true>), grid, dim3(1024), 0, st, A);
}

const int64_t MOST_ROWS = (int64_t)1 << 21, MOST_VOCAB = (int64_t)1 << 24;

}  // namespace

extern "C" {

size_t sl_token_loss_workspace_bytes(int64_t rows)
{
    return rows < 1 || rows > MOST_ROWS ? 0 : sizeof(double) * (size_t)rows;
}

int sl_token_loss(const void *logits, int type, int64_t ld, int64_t rows, int64_t vocab, const int64_t *targets, const float *weights,
                  const sl_policy *policy, float *loss, float *logp, void *dlogits, int64_t ldd, void *workspace, void *stream)
{
    if (rows < 0 || rows > MOST_ROWS || vocab < 1 || vocab > MOST_VOCAB || (type != SL_TYPE_F32 && type != SL_TYPE_BF16)) return SL_ERR_INVALID_ARG;
    if (!loss && !logp && !dlogits) return SL_ERR_INVALID_ARG;
    const uintptr_t word = type == SL_TYPE_BF16 ? 1 : 3;
    if (((uintptr_t)loss & 3) || ((uintptr_t)logp & 3) || ((uintptr_t)dlogits & word) || ((uintptr_t)workspace & 15)) return SL_ERR_INVALID_ARG;
    LossArgs A = {};
    if (policy) {
        if (!(policy->clip_low >= 0.0 && policy->clip_low <= 1.0 && policy->clip_high >= 0.0 && policy->kl >= 0.0) || !std::isfinite(policy->clip_high) ||
            !std::isfinite(policy->kl))
            return SL_ERR_INVALID_ARG;
        if (rows > 0 && (!policy->old_logp || !policy->advantage || (policy->kl > 0.0 && !policy->ref_logp))) return SL_ERR_INVALID_ARG;
        if (((uintptr_t)policy->old_logp & 3) || ((uintptr_t)policy->advantage & 3) || ((uintptr_t)policy->ref_logp & 3)) return SL_ERR_INVALID_ARG;
        A.policy = 1, A.old_logp = policy->old_logp, A.advantage = policy->advantage, A.ref_logp = policy->ref_logp;
        A.low = 1.0 - policy->clip_low, A.high = 1.0 + policy->clip_high, A.kl = policy->kl;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows > 0) {
        if (!logits || !targets || (loss && !workspace) || ld < vocab || ld > ((int64_t)1 << 40) || (dlogits && (ldd < vocab || ldd > ((int64_t)1 << 40))))
            return SL_ERR_INVALID_ARG;
        if (((uintptr_t)logits & word) || ((uintptr_t)targets & 7) || ((uintptr_t)weights & 3)) return SL_ERR_INVALID_ARG;
        if (dlogits == logits && ldd != ld) return SL_ERR_INVALID_ARG;
        if (loss && (workspace == logits || workspace == dlogits || (const void *)workspace == (const void *)targets)) return SL_ERR_INVALID_ARG;
        A.logits = logits, A.dlogits = dlogits, A.targets = reinterpret_cast<const long long *>(targets), A.weights = weights;
        A.logp = logp, A.each = loss ? static_cast<double *>(workspace) : nullptr;
        A.ld = ld, A.ldd = ldd, A.rows = rows, A.vocab = vocab;
        if (type == SL_TYPE_BF16) launch<true>(A, st);
        else launch<false>(A, st);
        if (const int rc = check_launch()) return rc;
    }
    if (!loss) return SL_OK;
    hipLaunchKernelGGL(k_join_loss, dim3(1), dim3(1024), 0, st, A.each, rows, loss);
    return check_launch();
}

}  // extern "C"
