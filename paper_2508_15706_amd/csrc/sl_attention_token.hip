// Attention of one new token per sequence over its cache.
#include <algorithm>

#include "sl_attention.h"

namespace {

// Keys of a workgroup, and how many a wave takes at a time.
enum { LEAST_PART = 128, KEYS = AT_STAGE, MOST_GROUPS = 1280, LONGEST_PART = 2048 };

struct TokenArgs {
    SlSequences s;
    SlRows q, k, v, out;
    float *stats;                // per part and head: the maximum (in base 2) and the sum
    float *parts;                // per part and head: dim values
    unsigned part;               // keys in a part
};

// A part of a sequence's keys for up to 32 heads that share a key head: the heads are the columns of the score tile.  Every wave takes every
// fourth 32 keys of the part, in two stages of LDS of its own, and waits for nobody; the waves' results meet at the end.  Bound by the cache's
// bytes: each is read once, and the matrix unit idles.
template <int D>
__global__ void __launch_bounds__(256, 1) k_token(TokenArgs A, unsigned blocks)
{
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int TILE = KEYS * 2 * D, STEPS = D / 16, BLOCKS = D / 32, LOADS = 2 * SlWaveLoad<D>::LOADS;
    const unsigned kv_heads = (unsigned)(A.s.heads / A.s.group);
    const SlItem item = sl_item(blockIdx.x, kv_heads * blocks);
    if (item.tile >= A.s.tiles) return;
    SlSpan at;
    if (!sl_find_tile(A.s.k_start, A.s.n, A.s.tokens_k, A.part, item.tile, at)) return;
    const int kn = A.s.k_count ? min(max(A.s.k_count[at.s], 0), at.count) : at.count, n = min((int)A.part, kn - at.row0);
    if (n <= 0) return;
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), half = lane >> 5;
    const int kv = (int)(item.head / blocks), first_head = (int)(item.head % blocks) * 32, in_group = first_head + (lane & 31);
    const int head = kv * A.s.group + min(in_group, A.s.group - 1);
    sl_b8 q[STEPS];
    sl_own_row<D>(A.q.p + at.s * A.q.token + head * A.q.head, half, A.s.octets, q);
    const long long k0 = (long long)at.first + at.row0;
    const unsigned char *k = A.k.p + k0 * A.k.token + kv * A.k.head, *v = A.v.p + k0 * A.v.token + kv * A.v.head;
    SlWaveLoad<D> lk, lv;
    lk.setup(lane, A.s.octets, A.k.token);
    lv.setup(lane, A.s.octets, A.v.token);
    unsigned char *mine = lds + wave * (4 * TILE);
    const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char *)mine;
    const int plain = sl_plain_base<D>(lane), turned = sl_turned_base<D>(lane);
    sl_f16 o[BLOCKS];
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) o[m] = sl_zero16();
    SlRunning run;
    const int tiles = (n + KEYS - 1) / KEYS, steps = tiles > wave ? (tiles - wave + 3) / 4 : 0;
    // (past the last step it brings that one again, so that every step waits for the same number of loads)
    auto fill = [&](int i) __attribute__((always_inline)) {
        const int from = (wave + 4 * min(i, steps - 1)) * KEYS;
        const unsigned to = lds0 + (unsigned)(i & 1) * (2 * TILE);
        lk.load(k, from, n - from, to);
        lv.load(v, from, n - from, to + TILE);
    };
    if (steps > 0) fill(0), fill(1);
#pragma unroll 1
    for (int t = 0; t < steps; ++t) {
        wait_dma<LOADS>();
        const unsigned char *kt = mine + (t & 1) * (2 * TILE);
        run.tile<D>(kt, kt + TILE, plain, turned, q, min(n - (wave + 4 * t) * KEYS, (int)KEYS) - 4 * half, A.s.scale2, o);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // (the stage has been read)
        fill(t + 2);
    }
    wait_dma<0>();
    run.sum = sl_both_sum(run.sum);
    __syncthreads();
    // the waves' sums through LDS: column after column, a pad of one between them
    float *all = reinterpret_cast<float *>(lds);
    constexpr int PITCH = D + 1;
    float *stats = all + 4 * 32 * PITCH;
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) all[(wave * 32 + (lane & 31)) * PITCH + 32 * m + 8 * (e >> 2) + 4 * half + (e & 3)] = o[m][e];
    if (half == 0) stats[(wave * 32 + lane) * 2] = run.top, stats[(wave * 32 + lane) * 2 + 1] = run.sum;
    __syncthreads();
    const int heads_here = min(A.s.group - first_head, 32), dim = A.s.octets * 8;
    for (int i = threadIdx.x; i < heads_here * dim; i += 256) {
        const int c = i / dim, d = i % dim;
        float m = stats[c * 2];
#pragma unroll
        for (int w = 1; w < 4; ++w) m = fmaxf(m, stats[(w * 32 + c) * 2]);
        const float to = m == -INFINITY ? 0.0f : m;
        float value = 0.0f, total = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float by = __builtin_amdgcn_exp2f(stats[(w * 32 + c) * 2] - to);
            value = fmaf(all[(w * 32 + c) * PITCH + d], by, value);
            total = fmaf(stats[(w * 32 + c) * 2 + 1], by, total);
        }
        const long long place = (long long)item.tile * A.s.heads + kv * A.s.group + first_head + c;
        A.parts[place * dim + d] = value;
        if (d == 0) A.stats[place * 2] = m, A.stats[place * 2 + 1] = total;
    }
}

// One head of one sequence to a workgroup: its parts, in their order.
__global__ void __launch_bounds__(128) k_token_join(TokenArgs A)
{
    const int s = (int)(blockIdx.x / (unsigned)A.s.heads), head = (int)(blockIdx.x % (unsigned)A.s.heads), dim = A.s.octets * 8;
    int first, n;
    sl_rows_of(A.s.k_start, A.s.k_count, s, A.s.tokens_k, first, n);
    const unsigned part0 = (unsigned)first / A.part + (unsigned)s, parts = ((unsigned)n + A.part - 1) / A.part;
    if ((int)threadIdx.x >= dim) return;
    float m = -INFINITY;
    for (unsigned i = 0; i < parts; ++i) m = fmaxf(m, A.stats[((long long)(part0 + i) * A.s.heads + head) * 2]);
    const float to = m == -INFINITY ? 0.0f : m;
    float value = 0.0f, total = 0.0f;
#pragma unroll 4
    for (unsigned i = 0; i < parts; ++i) {
        const long long place = (long long)(part0 + i) * A.s.heads + head;
        const float by = __builtin_amdgcn_exp2f(A.stats[place * 2] - to);
        value = fmaf(A.parts[place * dim + threadIdx.x], by, value);
        total = fmaf(A.stats[place * 2 + 1], by, total);
    }
    reinterpret_cast<unsigned short *>(A.out.p + s * A.out.token + head * A.out.head)[threadIdx.x] =
        (unsigned short)sl_bf16_bits(total == 0.0f ? 0.0f : value / total);
}

int check_launch()
{
    const hipError_t err = hipGetLastError();
    if (err == hipSuccess) return SL_OK;
    sl_note_hip_error(err);
    return SL_ERR_HIP;
}

// Parts are as short as leaves about MOST_GROUPS workgroups: the number of them counts for one sequence, their evenness for many.
unsigned part_size(int64_t tokens, int64_t units)
{
    unsigned part = LEAST_PART;
    while (part < LONGEST_PART && tokens / part * units > MOST_GROUPS) part *= 2;
    return part;
}
int64_t most_parts(int64_t sequences, int64_t tokens, int64_t units)
{
    return std::min(tokens / LEAST_PART, std::max<int64_t>(MOST_GROUPS / units, tokens / LONGEST_PART)) + sequences;
}
int64_t unit_count(int64_t heads, int64_t kv_heads) { return kv_heads * ((heads / kv_heads + 31) / 32); }

}  // namespace

extern "C" {

size_t sl_attention_token_workspace_bytes(int64_t sequences, int64_t tokens_k, int heads, int kv_heads, int head_dim)
{
    if (sequences < 1 || sequences > AT_MOST_SEQUENCES || tokens_k < 0 || tokens_k > AT_MOST_TOKENS || heads < 1 || heads > AT_MOST_HEADS ||
        kv_heads < 1 || heads % kv_heads != 0 || head_dim < 8 || head_dim > 128 || head_dim % 8 != 0)
        return 0;
    return sizeof(float) * (size_t)(most_parts(sequences, tokens_k, unit_count(heads, kv_heads)) * heads * (head_dim + 2));
}

int sl_attention_token(const sl_attention_shape *shape, const sl_heads *q, const sl_heads *k, const sl_heads *v, const sl_heads *out, void *workspace,
                       void *stream)
{
    TokenArgs A = {};
    if (!sl_attention_sequences(shape, A.s) || shape->tokens_q != shape->sequences) return SL_ERR_INVALID_ARG;
    if (A.s.n == 0) return SL_OK;
    const bool keys = A.s.tokens_k > 0;
    if (!sl_attention_in(q, true, A.q) || !sl_attention_in(k, keys, A.k) || !sl_attention_in(v, keys, A.v) ||
        !sl_attention_out(out, true, A.s.n, A.s.heads, shape->head_dim, A.out) || !workspace || ((uintptr_t)workspace & 15))
        return SL_ERR_INVALID_ARG;
    const void *in[4] = {q->data, keys ? k->data : nullptr, keys ? v->data : nullptr, workspace};
    for (const void *p : in)
        if (p == out->data) return SL_ERR_INVALID_ARG;
    const int64_t units = unit_count(shape->heads, shape->kv_heads);
    A.part = part_size(A.s.tokens_k, units);
    A.s.tiles = (unsigned)A.s.tokens_k / A.part + (unsigned)A.s.n;
    if ((int64_t)(A.s.tiles + 7) / 8 * 8 * units >= (int64_t)1 << 24 || (int64_t)A.s.n * A.s.heads >= (int64_t)1 << 25) return SL_ERR_INVALID_ARG;
    A.stats = static_cast<float *>(workspace);
    A.parts = A.stats + 2 * (int64_t)A.s.tiles * A.s.heads;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (keys) {
        const bool narrow = A.s.octets <= 8;
        const unsigned lds = 4u * 4 * KEYS * 2 * (narrow ? 64 : 128);
        const auto kernel = narrow ? k_token<64> : k_token<128>;
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (err != hipSuccess) {
            sl_note_hip_error(err);
            return SL_ERR_HIP;
        }
        hipLaunchKernelGGL(kernel, dim3(sl_item_groups(A.s.tiles, units)), dim3(256), lds, st, A, (unsigned)(units / shape->kv_heads));
        if (const int rc = check_launch()) return rc;
    }
    hipLaunchKernelGGL(k_token_join, dim3((unsigned)(A.s.n * A.s.heads)), dim3(128), 0, st, A);
    return check_launch();
}

}  // extern "C"
