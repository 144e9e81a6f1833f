// Attention of one new token per sequence over its cache.
#include "sl_attention.h"

namespace {

struct TokenArgs {
    SlSequences s;
    SlRows q, k, v, out;
    float *stats;                // per part and head: the maximum (in base 2) and the sum
    float *parts;                // per part and head: dim values
    unsigned part;               // keys in a part
};

// A part of a sequence's keys for up to 32 heads that share a key head: the heads are the columns of the score tile.  One wave does it, 32
// keys at a time, in two stages of LDS, and waits for nobody: five of them fit a compute unit, so that one's start and end lie beside
// the others' loads.  Bound by the cache's bytes; the matrix unit idles.  64 sequences, up to 16,384 keys, 5 heads of 128 - 596 MB: 114 us, 5.2
// TB/s (parts of 256 and 1024 keys 123 and 124; four waves to a part of 2048 122, of 512 183).
template <int D>
__global__ void __launch_bounds__(64, 2) k_token(TokenArgs A, unsigned blocks)
{
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int TILE = AT_STAGE * 2 * D, STEPS = D / 16, BLOCKS = D / 32, LOADS = 2 * SlWaveLoad<D>::LOADS;
    const unsigned kv_heads = (unsigned)(A.s.heads / A.s.group);
    const SlItem item = sl_item(blockIdx.x, kv_heads * blocks);
    if (item.tile >= A.s.tiles) return;
    SlSpan at;
    if (!sl_find_tile(A.s.k_start, A.s.n, A.s.tokens_k, A.part, item.tile, at)) return;
    const int kn = A.s.k_count ? min(max(A.s.k_count[at.s], 0), at.count) : at.count, n = min((int)A.part, kn - at.row0);
    if (n <= 0) return;
    const int lane = threadIdx.x, half = lane >> 5;
    const int kv = (int)(item.head / blocks), first_head = (int)(item.head % blocks) * 32, in_group = first_head + (lane & 31);
    const int head = kv * A.s.group + min(in_group, A.s.group - 1);
    const long long k0 = (long long)at.first + at.row0;
    const unsigned char *k = A.k.p + k0 * A.k.token + kv * A.k.head, *v = A.v.p + k0 * A.v.token + kv * A.v.head;
    SlWaveLoad<D> lk, lv;
    lk.setup(lane, A.s.octets, A.k.token);
    lv.setup(lane, A.s.octets, A.v.token);
    const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char *)lds;
    const int steps = (n + AT_STAGE - 1) / AT_STAGE;
    // (past the last step it brings that one again, so that every step waits for the same number of loads)
    auto fill = [&](int i) __attribute__((always_inline)) {
        const int from = min(i, steps - 1) * AT_STAGE;
        const unsigned to = lds0 + (unsigned)(i & 1) * (2 * TILE);
        lk.load(k, from, n - from, to);
        lv.load(v, from, n - from, to + TILE);
    };
    fill(0), fill(1);
    sl_b8 q[STEPS];
    sl_own_row<D>(A.q.p + at.s * A.q.token + head * A.q.head, half, A.s.octets, q);
    const int plain = sl_plain_base<D>(lane), turned = sl_turned_base<D>(lane);
    sl_f16 o[BLOCKS];
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) o[m] = sl_zero16();
    SlRunning run;
#pragma unroll 1
    for (int t = 0; t < steps; ++t) {
        wait_dma<LOADS>();
        const unsigned char *kt = lds + (t & 1) * (2 * TILE);
        run.tile<D>(kt, kt + TILE, plain, turned, q, min(n - t * AT_STAGE, (int)AT_STAGE) - 4 * half, A.s.scale2, o);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // (the stage has been read)
        fill(t + 2);
    }
    wait_dma<0>();
    run.sum = sl_both_sum(run.sum);
    if (in_group >= A.s.group) return;
    const long long place = (long long)item.tile * A.s.heads + head;
    float *to = A.parts + place * (A.s.octets * 8) + 4 * half;
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            if (m * 4 + g < A.s.octets)
                *reinterpret_cast<sl_f4 *>(to + 32 * m + 8 * g) = sl_f4{o[m][4 * g], o[m][4 * g + 1], o[m][4 * g + 2], o[m][4 * g + 3]};
    if (half == 0) A.stats[place * 2] = run.top, A.stats[place * 2 + 1] = run.sum;
}

// One head of one sequence to a workgroup: its parts, in their order; their weights first, 128 at a time, each in a thread of its own.
__global__ void __launch_bounds__(128) k_token_join(TokenArgs A)
{
    __shared__ float weight[128], totals[2], tops[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int s = (int)(blockIdx.x / (unsigned)A.s.heads), head = (int)(blockIdx.x % (unsigned)A.s.heads), dim = A.s.octets * 8;
    int first, n;
    sl_rows_of(A.s.k_start, A.s.k_count, s, A.s.tokens_k, first, n);
    const long long place0 = ((long long)((unsigned)first / A.part + (unsigned)s)) * A.s.heads + head;
    const int parts = (int)(((unsigned)n + A.part - 1) / A.part);
    float top = -INFINITY, total = 0.0f, value = 0.0f;
    for (int base = 0; base < parts; base += 128) {
        const int here = min(parts - base, 128);
        float m = -INFINITY, sum = 0.0f;
        if (tid < here) m = A.stats[(place0 + (long long)(base + tid) * A.s.heads) * 2], sum = A.stats[(place0 + (long long)(base + tid) * A.s.heads) * 2 + 1];
        float most = m;
#pragma unroll
        for (int l = 0; l < 6; ++l) most = __builtin_elementwise_maximum(most, __int_as_float(sl_partner(__float_as_int(most), l)));
        if (lane == 0) tops[wave] = most;
        __syncthreads();
        most = __builtin_elementwise_maximum(__builtin_elementwise_maximum(tops[0], tops[1]), top);
        const float ref = most == -INFINITY ? 0.0f : most, by = __builtin_amdgcn_exp2f(m - ref), before = __builtin_amdgcn_exp2f(top - ref);
        weight[tid] = by;
        double t = (double)(sum * by);
        t = sl_wave_tree(t, 6);
        if (lane == 0) totals[wave] = (float)t;
        __syncthreads();
        total = total * before + (totals[0] + totals[1]), value = value * before, top = most;
        if (tid < dim) {
            const float *p = A.parts + (place0 + (long long)base * A.s.heads) * dim + tid;
            const long long step = (long long)A.s.heads * dim;
            int i = 0;
            for (; i + 8 <= here; i += 8) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = p[(i + j) * step];
#pragma unroll
                for (int j = 0; j < 8; ++j) value = fmaf(x[j], weight[i + j], value);
            }
            for (; i < here; ++i) value = fmaf(p[i * step], weight[i], value);
        }
        __syncthreads();
    }
    if (tid < dim)
        reinterpret_cast<unsigned short *>(A.out.p + s * A.out.token + head * A.out.head)[tid] = (unsigned short)sl_bf16_bits(total == 0.0f ? 0.0f : value / total);
}

int check_launch()
{
    const hipError_t err = hipGetLastError();
    if (err == hipSuccess) return SL_OK;
    sl_note_hip_error(err);
    return SL_ERR_HIP;
}

}  // namespace

extern "C" {

size_t sl_attention_token_workspace_bytes(int64_t sequences, int64_t tokens_k, int heads, int kv_heads, int head_dim)
{
    if (sequences < 1 || sequences > AT_MOST_SEQUENCES || tokens_k < 0 || tokens_k > AT_MOST_TOKENS || heads < 1 || heads > AT_MOST_HEADS ||
        kv_heads < 1 || heads % kv_heads != 0 || head_dim < 8 || head_dim > 128 || head_dim % 8 != 0)
        return 0;
    return sizeof(float) * (size_t)(sl_token_room(sl_token_most_parts(sequences, tokens_k, sl_token_units(heads, kv_heads)), heads, head_dim).floats);
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
    const int64_t units = sl_token_units(shape->heads, shape->kv_heads);
    A.part = sl_token_part(A.s.tokens_k, units);
    A.s.tiles = (unsigned)A.s.tokens_k / A.part + (unsigned)A.s.n;
    if ((int64_t)(A.s.tiles + 7) / 8 * 8 * units >= (int64_t)1 << 24 || (int64_t)A.s.n * A.s.heads >= (int64_t)1 << 25) return SL_ERR_INVALID_ARG;
    const SlTokenRoom room = sl_token_room(A.s.tiles, A.s.heads, shape->head_dim);
    A.parts = static_cast<float *>(workspace) + room.values;
    A.stats = static_cast<float *>(workspace) + room.stats;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (keys) {
        const bool narrow = A.s.octets <= 8;
        const unsigned lds = 4u * AT_STAGE * 2 * (narrow ? 64 : 128);
        const auto kernel = narrow ? k_token<64> : k_token<128>;
        hipLaunchKernelGGL(kernel, dim3(sl_item_groups(A.s.tiles, units)), dim3(64), lds, st, A, (unsigned)(units / shape->kv_heads));
        if (const int rc = check_launch()) return rc;
    }
    hipLaunchKernelGGL(k_token_join, dim3((unsigned)(A.s.n * A.s.heads)), dim3(128), 0, st, A);
    return check_launch();
}

}  // extern "C"
