// Attention over packed sequences, forward and backward.
//   S = scale q k^T ;  P = softmax over the keys that a query sees ;  out = P v ;  lse = log sum exp S
//   dP = dout v^T ;  dS = P (dP - sum dout out) ;  dq = scale dS k ;  dk = scale dS^T q ;  dv = P^T dout
#include <algorithm>
#include <cmath>

#include "sl_attention.h"
#include "sl_internal.h"

namespace {

const float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

struct AttendArgs {
    SlSequences s;
    SlRows q, k, v, out;
    float *lse;
};

struct BackArgs {
    SlSequences s;
    SlRows q, k, v, out, dout, dq, dk, dv;
    const float *lse;
    float *stats;                // per query: lse in base 2, sum dout out; heads x tokens each.  Behind them what stands for no query: infinity, whose
                                 // probabilities are 0, and 0
    long long none;              // where
    // keys' and values' gradients of `slices` parts of a group's heads, fp32: [slice][dk, dv][token][key head][dim]; one slice: none
    float *parts;
    int slices;
};

// ---- forward ----

// 128 queries of one head, 32 to a wave, over 64 keys at a time, two stages of LDS; the softmax in one pass, as in SlRunning (whose 32 keys
// would leave the matrix unit one chain of products; here are two).  Two workgroups to a compute unit: 32 products of 32 cycles a wave and
// 64 keys stand against about 900 cycles of exponentials, sums and maxima, of which less than half runs beside the other's products, since
// nothing keeps the two out of phase.  The same loop on constant operands, without masks, starts and ends, at 2.4 GHz, 64 keys of two waves:
// products alone 1005 ns, all but the reads of LDS 1440, all of it 1630; here 2170 at 2.0 GHz.
// 8192 tokens, 20 heads of 128 on 5: 349 us, 0.98 PFLOP/s, the matrix unit busy 45 % of the time, the vector unit 42, LDS 23; 8 x 2048 tokens,
// 16 heads: 175 us, 0.79.  Tried and not kept: the next tile's scores beside this one's exponentials in the same wave (111 registers spilled,
// 704 us), priorities of waves around products or exponentials (the same time).
template <int D>
__global__ void __launch_bounds__(256, 2) k_attend(AttendArgs A)
{
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int TILE = AT_TILE * 2 * D, STEPS = D / 16, BLOCKS = D / 32;
    const SlItem item = sl_item(blockIdx.x, (unsigned)A.s.heads);
    if (item.tile >= A.s.tiles) return;
    SlSpan at;
    int k0, kn;
    if (!sl_find(A.s.q_start, A.s.tokens_q, A.s.k_start, A.s.k_count, A.s.tokens_k, A.s, AT_ROWS, item.tile, true, at, k0, kn)) return;
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), half = lane >> 5;
    const int head = (int)item.head, kv = head / A.s.group, shift = kn - at.count;
    const int row = at.row0 + wave * 32 + (lane & 31), mine = min(row, at.count - 1);
    sl_b8 q[STEPS];
    sl_own_row<D>(A.q.p + (long long)(at.first + mine) * A.q.token + head * A.q.head, half, A.s.octets, q);

    // keys that this row sees, the first and the last row of the wave, the last of the workgroup
    const int sees = A.s.causal ? min(kn, mine + shift + 1) : kn;
    const int fewest = A.s.causal ? min(kn, min(at.row0 + wave * 32, at.count - 1) + shift + 1) : kn;
    const int most = A.s.causal ? min(kn, min(at.row0 + wave * 32 + 31, at.count - 1) + shift + 1) : kn;
    const int all = A.s.causal ? min(kn, min(at.row0 + AT_ROWS - 1, at.count - 1) + shift + 1) : kn;
    const unsigned char *k = A.k.p + (long long)k0 * A.k.token + kv * A.k.head, *v = A.v.p + (long long)k0 * A.v.token + kv * A.v.head;
    SlTileLoad<D> lk, lv;
    lk.setup(wave, lane, A.s.octets, A.k.token);
    lv.setup(wave, lane, A.s.octets, A.v.token);
    const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char *)lds;
    const int plain = sl_plain_base<D>(lane), turned = sl_turned_base<D>(lane);

    sl_f16 o[BLOCKS];
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) o[m] = sl_zero16();
    float top = -INFINITY, ref = 0.0f, sum = 0.0f;      // the maximum that the exponents refer to, and it or 0
    const int tiles = (max(all, 0) + AT_TILE - 1) / AT_TILE;
    if (tiles > 0) {
        lk.load(k, 0, kn, lds0, wave);
        lv.load(v, 0, kn, lds0 + 2 * TILE, wave);
    }
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) {
        wait_dma<0>();
        stage_barrier();
        if (t + 1 < tiles) {
            const unsigned to = lds0 + (unsigned)((t + 1) & 1) * TILE;
            lk.load(k, (t + 1) * AT_TILE, kn, to, wave);
            lv.load(v, (t + 1) * AT_TILE, kn, to + 2 * TILE, wave);
        }
        if (t * AT_TILE >= most) continue;
        const unsigned char *kt = lds + (t & 1) * TILE, *vt = kt + 2 * TILE;
        sl_f16 s[2];
        s[0] = s[1] = sl_zero16();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            s[0] = sl_mfma(sl_plain<D>(kt, plain, 0, i), q[i], s[0]);
            s[1] = sl_mfma(sl_plain<D>(kt, plain, 1, i), q[i], s[1]);
        }
        sl_reads_ahead<2 * STEPS, 8>();
        __builtin_amdgcn_sched_barrier(0);
        if ((t + 1) * AT_TILE > fewest) {
            const int left = sees - t * AT_TILE - 4 * half;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (32 * i + 8 * (e >> 2) + (e & 3) >= left) s[i][e] = -INFINITY;
        }
        float now = s[0][0];
#pragma unroll
        for (int e = 0; e < 16; ++e) now = __builtin_elementwise_maximum(now, __builtin_elementwise_maximum(s[0][e], s[1][e]));
        now = sl_both_max(now) * A.s.scale2;
        if (sl_ballot(now > top + 8.0f)) {
            const float next = fmaxf(top, now), to = next == -INFINITY ? 0.0f : next, by = __builtin_amdgcn_exp2f(top - to);
            top = next, ref = to, sum = sum * by;
#pragma unroll
            for (int m = 0; m < BLOCKS; ++m)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[m][e] = o[m][e] * by;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[i][e] = __builtin_amdgcn_exp2f(fmaf(s[i][e], A.s.scale2, -ref));
                sum = sum + s[i][e];
            }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const sl_b8 p = sl_operand(s[g >> 1], g & 1);
#pragma unroll
            for (int m = 0; m < BLOCKS; ++m) o[m] = sl_mfma(sl_turned<D>(vt, turned, m, g), p, o[m]);
        }
    }
    sum = sl_both_sum(sum);
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
    const bool there = row < at.count;
    sl_put_row<D>(A.out.p + (long long)(at.first + mine) * A.out.token + head * A.out.head, there, half, A.s.octets, o, by);
    if (A.lse && there && half == 0)
        A.lse[(long long)head * A.s.tokens_q + at.first + mine] = sum == 0.0f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * LN2;
}

// Few tiles: 32 queries to a workgroup, whose four waves take every fourth 32 keys, in LDS of their own, and wait for nobody; their sums meet
// at the end.
template <int D>
__global__ void __launch_bounds__(256, 1) k_attend_few(AttendArgs A)
{
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int TILE = AT_STAGE * 2 * D, STEPS = D / 16, BLOCKS = D / 32, LOADS = 2 * SlWaveLoad<D>::LOADS;
    const SlItem item = sl_item(blockIdx.x, (unsigned)A.s.heads);
    if (item.tile >= A.s.tiles) return;
    SlSpan at;
    int k0, kn;
    if (!sl_find(A.s.q_start, A.s.tokens_q, A.s.k_start, A.s.k_count, A.s.tokens_k, A.s, 32, item.tile, true, at, k0, kn)) return;
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), half = lane >> 5;
    const int head = (int)item.head, kv = head / A.s.group, shift = kn - at.count;
    const int row = at.row0 + (lane & 31), mine = min(row, at.count - 1);
    const unsigned char *k = A.k.p + (long long)k0 * A.k.token + kv * A.k.head, *v = A.v.p + (long long)k0 * A.v.token + kv * A.v.head;
    SlWaveLoad<D> lk, lv;
    lk.setup(lane, A.s.octets, A.k.token);
    lv.setup(lane, A.s.octets, A.v.token);
    unsigned char *own = lds + wave * (4 * TILE);
    const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char *)own;
    // keys that this row sees, the first row of the workgroup, its last
    const int sees = A.s.causal ? min(kn, mine + shift + 1) : kn, fewest = A.s.causal ? min(kn, at.row0 + shift + 1) : kn;
    const int all = A.s.causal ? min(kn, min(at.row0 + 31, at.count - 1) + shift + 1) : kn;
    const int tiles = (max(all, 0) + AT_STAGE - 1) / AT_STAGE, steps = tiles > wave ? (tiles - wave + 3) / 4 : 0;
    // (past the last step it brings that one again, so that every step waits for the same number of loads)
    auto fill = [&](int i) __attribute__((always_inline)) {
        const int from = (wave + 4 * min(i, steps - 1)) * AT_STAGE;
        const unsigned to = lds0 + (unsigned)(i & 1) * (2 * TILE);
        lk.load(k, from, kn - from, to);
        lv.load(v, from, kn - from, to + TILE);
    };
    if (steps > 0) fill(0), fill(1);
    sl_b8 q[STEPS];
    sl_own_row<D>(A.q.p + (long long)(at.first + mine) * A.q.token + head * A.q.head, half, A.s.octets, q);
    const int plain = sl_plain_base<D>(lane), turned = sl_turned_base<D>(lane);
    sl_f16 o[BLOCKS];
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) o[m] = sl_zero16();
    SlRunning run;
#pragma unroll 1
    for (int t = 0; t < steps; ++t) {
        wait_dma<LOADS>();
        const unsigned char *kt = own + (t & 1) * (2 * TILE);
        const int first = (wave + 4 * t) * AT_STAGE;
        run.tile<D>(kt, kt + TILE, plain, turned, q, first + AT_STAGE > fewest ? sees - first - 4 * half : AT_STAGE, A.s.scale2, o);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // (the stage has been read)
        fill(t + 2);
    }
    wait_dma<0>();
    run.sum = sl_both_sum(run.sum);
    __syncthreads();
    float *room = reinterpret_cast<float *>(lds), *stats = room + 4 * BLOCKS * 1024;
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) sl_leave_block(room + (wave * BLOCKS + m) * 1024, lane, o[m]);
    if (half == 0) stats[wave * 64 + lane] = run.top, stats[wave * 64 + 32 + lane] = run.sum;
    __syncthreads();
    float top[4], sum = 0.0f, most = -INFINITY;
    sl_f4 by;
#pragma unroll
    for (int w = 0; w < 4; ++w) top[w] = stats[w * 64 + (lane & 31)], most = fmaxf(most, top[w]);
    const float ref = most == -INFINITY ? 0.0f : most;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        by[w] = __builtin_amdgcn_exp2f(top[w] - ref);
        sum = fmaf(stats[w * 64 + 32 + (lane & 31)], by[w], sum);
    }
    const bool there = row < at.count;
    const float whole = sum == 0.0f ? 0.0f : 1.0f / sum;
    unsigned char *out = A.out.p + (long long)(at.first + mine) * A.out.token + head * A.out.head;
    for (int m = wave; m < BLOCKS; m += 4) sl_put_block(out, there, half, A.s.octets, sl_four_blocks(room + m * 1024, BLOCKS * 1024, lane, by), m, whole);
    if (A.lse && there && wave == 0 && half == 0)
        A.lse[(long long)head * A.s.tokens_q + at.first + mine] = sum == 0.0f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * LN2;
}

// ---- backward ----

// dq: queries to lanes as in the forward pass; S and dP of 32 keys at a time.  It also leaves what the pass over keys needs of a query.
// Three products where the pass over keys has four; 8 x 2048 tokens, 16 heads of 128: 230 us, 0.90 PFLOP/s.  (dq from that pass would need
// sums over workgroups, in memory or in an order that changes.)
// sum dout out is that of P dP, too: for queries that see few keys, whose dP - sum dout out is small beside its terms, it is taken from there,
// in a pass over the keys in front.  From out, which is rounded, it moves the dS of all of a query's keys the same way, by its own
// rounding's share of |dout| |out|, which does not average out over few keys (1024 tokens, N(0, 1.5) queries: dq's error 0.28 % of its norm
// with it, 0.24 % with the sum, of which the roundings of dS and dq themselves are 0.24).
enum { FEW_KEYS = 256 };

template <int D>
__global__ void __launch_bounds__(256, 2) k_back_q(BackArgs A)
{
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int TILE = AT_TILE * 2 * D, STEPS = D / 16, BLOCKS = D / 32;
    const SlItem item = sl_item(blockIdx.x, (unsigned)A.s.heads);
    if (blockIdx.x == 0 && threadIdx.x < 2) A.stats[A.none + threadIdx.x] = threadIdx.x == 0 ? INFINITY : 0.0f;
    if (item.tile >= A.s.tiles) return;
    SlSpan at;
    int k0, kn;
    if (!sl_find(A.s.q_start, A.s.tokens_q, A.s.k_start, A.s.k_count, A.s.tokens_k, A.s, AT_ROWS, item.tile, true, at, k0, kn)) return;
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), half = lane >> 5;
    const int head = (int)item.head, kv = head / A.s.group, shift = kn - at.count;
    const int row = at.row0 + wave * 32 + (lane & 31), mine = min(row, at.count - 1);
    const long long token = at.first + mine;
    sl_b8 q[STEPS], g[STEPS];
    sl_own_row<D>(A.dout.p + token * A.dout.token + head * A.dout.head, half, A.s.octets, g);
    float delta = 0.0f;
    {
        sl_own_row<D>(A.out.p + token * A.out.token + head * A.out.head, half, A.s.octets, q);
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf((float)q[i][e], (float)g[i][e], delta);
        delta = sl_both_sum(delta);
    }
    sl_own_row<D>(A.q.p + token * A.q.token + head * A.q.head, half, A.s.octets, q);
    const float lse = A.lse[(long long)head * A.s.tokens_q + token], lse2 = lse == -INFINITY ? 0.0f : lse * LOG2E;
    const int sees = A.s.causal ? min(kn, mine + shift + 1) : kn;
    const int all = A.s.causal ? min(kn, min(at.row0 + AT_ROWS - 1, at.count - 1) + shift + 1) : kn;
    const unsigned char *k = A.k.p + (long long)k0 * A.k.token + kv * A.k.head, *v = A.v.p + (long long)k0 * A.v.token + kv * A.v.head;
    SlTileLoad<D> lk, lv;
    lk.setup(wave, lane, A.s.octets, A.k.token);
    lv.setup(wave, lane, A.s.octets, A.v.token);
    const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char *)lds;
    const int plain = sl_plain_base<D>(lane), turned = sl_turned_base<D>(lane);
    sl_f16 dq[BLOCKS];
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) dq[m] = sl_zero16();
    const int tiles = (max(all, 0) + AT_TILE - 1) / AT_TILE;
    const bool few = (A.s.causal ? min(kn, at.row0 + shift + 1) : kn) <= FEW_KEYS;
    auto load = [&](int step, int t) __attribute__((always_inline)) {
        const unsigned to = lds0 + (unsigned)(step & 1) * TILE;
        lk.load(k, t * AT_TILE, kn, to, wave);
        lv.load(v, t * AT_TILE, kn, to + 2 * TILE, wave);
    };
    // P (dP - less) of half i of tile t
    auto half_tile = [&](int step, int t, int i, float less) __attribute__((always_inline)) {
        const unsigned char *kt = lds + (step & 1) * TILE, *vt = kt + 2 * TILE;
        sl_f16 s = sl_zero16(), dp = sl_zero16();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            s = sl_mfma(sl_plain<D>(kt, plain, i, j), q[j], s);
            dp = sl_mfma(sl_plain<D>(vt, plain, i, j), g[j], dp);
        }
        sl_reads_ahead<2 * STEPS, 6>();
        __builtin_amdgcn_sched_barrier(0);
        const int left = sees - t * AT_TILE - 4 * half - 32 * i;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float x = fmaf(s[e], A.s.scale2, -lse2);
            s[e] = __builtin_amdgcn_exp2f(8 * (e >> 2) + (e & 3) < left ? x : -INFINITY) * (dp[e] - less);
        }
        return s;
    };
    int step = 0;
    if (tiles > 0) load(0, 0);
    if (few) {
        float sum = 0.0f;
#pragma unroll 1
        for (int t = 0; t < tiles; ++t, ++step) {
            wait_dma<0>();
            stage_barrier();
            load(step + 1, t + 1 < tiles ? t + 1 : 0);
#pragma unroll 1
            for (int i = 0; i < 2; ++i) {
                const sl_f16 s = half_tile(step, t, i, 0.0f);
#pragma unroll
                for (int e = 0; e < 16; ++e) sum = sum + s[e];
            }
        }
        delta = sl_both_sum(sum);
    }
#pragma unroll 1
    for (int t = 0; t < tiles; ++t, ++step) {
        wait_dma<0>();
        stage_barrier();
        if (t + 1 < tiles) load(step + 1, t + 1);
        const unsigned char *kt = lds + (step & 1) * TILE;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const sl_f16 s = half_tile(step, t, i, delta);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const sl_b8 ds = sl_operand(s, j);
#pragma unroll
                for (int m = 0; m < BLOCKS; ++m) dq[m] = sl_mfma(sl_turned<D>(kt, turned, m, 2 * i + j), ds, dq[m]);
            }
        }
    }
    if (row < at.count && half == 0) {
        float *to = A.stats + (long long)head * A.s.tokens_q + token;
        to[0] = lse2;
        to[(long long)A.s.heads * A.s.tokens_q] = delta;
    }
    sl_put_row<D>(A.dq.p + token * A.dq.token + head * A.dq.head, row < at.count, half, A.s.octets, dq, A.s.scale);
}

// Few tiles: 32 queries to a workgroup, whose four waves take every fourth 32 keys; see k_attend_few.
template <int D>
__global__ void __launch_bounds__(256, 1) k_back_q_few(BackArgs A)
{
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ float sums[4][32];
    constexpr int TILE = AT_STAGE * 2 * D, STEPS = D / 16, BLOCKS = D / 32, LOADS = 2 * SlWaveLoad<D>::LOADS;
    const SlItem item = sl_item(blockIdx.x, (unsigned)A.s.heads);
    if (blockIdx.x == 0 && threadIdx.x < 2) A.stats[A.none + threadIdx.x] = threadIdx.x == 0 ? INFINITY : 0.0f;
    if (item.tile >= A.s.tiles) return;
    SlSpan at;
    int k0, kn;
    if (!sl_find(A.s.q_start, A.s.tokens_q, A.s.k_start, A.s.k_count, A.s.tokens_k, A.s, 32, item.tile, true, at, k0, kn)) return;
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), half = lane >> 5;
    const int head = (int)item.head, kv = head / A.s.group, shift = kn - at.count;
    const int row = at.row0 + (lane & 31), mine = min(row, at.count - 1);
    const long long token = at.first + mine;
    const unsigned char *k = A.k.p + (long long)k0 * A.k.token + kv * A.k.head, *v = A.v.p + (long long)k0 * A.v.token + kv * A.v.head;
    SlWaveLoad<D> lk, lv;
    lk.setup(lane, A.s.octets, A.k.token);
    lv.setup(lane, A.s.octets, A.v.token);
    unsigned char *own = lds + wave * (4 * TILE);
    const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char *)own;
    const int sees = A.s.causal ? min(kn, mine + shift + 1) : kn;
    const int all = A.s.causal ? min(kn, min(at.row0 + 31, at.count - 1) + shift + 1) : kn;
    const int tiles = (max(all, 0) + AT_STAGE - 1) / AT_STAGE, steps = tiles > wave ? (tiles - wave + 3) / 4 : 0;
    const bool few = (A.s.causal ? min(kn, at.row0 + shift + 1) : kn) <= FEW_KEYS;
    const int total = few ? 2 * steps : steps;
    auto fill = [&](int i) __attribute__((always_inline)) {
        const int from = (wave + 4 * (min(i, total - 1) % steps)) * AT_STAGE;
        const unsigned to = lds0 + (unsigned)(i & 1) * (2 * TILE);
        lk.load(k, from, kn - from, to);
        lv.load(v, from, kn - from, to + TILE);
    };
    if (steps > 0) fill(0), fill(1);
    sl_b8 q[STEPS], g[STEPS];
    sl_own_row<D>(A.dout.p + token * A.dout.token + head * A.dout.head, half, A.s.octets, g);
    float delta = 0.0f;
    {
        sl_own_row<D>(A.out.p + token * A.out.token + head * A.out.head, half, A.s.octets, q);
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf((float)q[i][e], (float)g[i][e], delta);
        delta = sl_both_sum(delta);
    }
    sl_own_row<D>(A.q.p + token * A.q.token + head * A.q.head, half, A.s.octets, q);
    const float lse = A.lse[(long long)head * A.s.tokens_q + token], lse2 = lse == -INFINITY ? 0.0f : lse * LOG2E;
    const int plain = sl_plain_base<D>(lane), turned = sl_turned_base<D>(lane);
    // P (dP - less) of step n
    auto scores = [&](int n, float less) __attribute__((always_inline)) {
        wait_dma<LOADS>();
        const unsigned char *kt = own + (n & 1) * (2 * TILE), *vt = kt + TILE;
        sl_f16 s = sl_zero16(), dp = sl_zero16();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            s = sl_mfma(sl_plain<D>(kt, plain, 0, j), q[j], s);
            dp = sl_mfma(sl_plain<D>(vt, plain, 0, j), g[j], dp);
        }
        sl_reads_ahead<2 * STEPS, 8>();
        __builtin_amdgcn_sched_barrier(0);
        const int left = sees - (wave + 4 * (n % steps)) * AT_STAGE - 4 * half;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float x = fmaf(s[e], A.s.scale2, -lse2);
            s[e] = __builtin_amdgcn_exp2f(8 * (e >> 2) + (e & 3) < left ? x : -INFINITY) * (dp[e] - less);
        }
        return s;
    };
    auto again = [&](int n) __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // (the stage has been read)
        fill(n + 2);
    };
    int n = 0;
    if (few) {
        float sum = 0.0f;
#pragma unroll 1
        for (; n < steps; ++n) {
            const sl_f16 s = scores(n, 0.0f);
#pragma unroll
            for (int e = 0; e < 16; ++e) sum = sum + s[e];
            again(n);
        }
        sum = sl_both_sum(sum);
        if (half == 0) sums[wave][lane] = sum;
        __syncthreads();
        delta = ((sums[0][lane & 31] + sums[1][lane & 31]) + sums[2][lane & 31]) + sums[3][lane & 31];
    }
    sl_f16 dq[BLOCKS];
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) dq[m] = sl_zero16();
#pragma unroll 1
    for (; n < total; ++n) {
        const sl_f16 s = scores(n, delta);
        const unsigned char *kt = own + (n & 1) * (2 * TILE);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const sl_b8 ds = sl_operand(s, j);
#pragma unroll
            for (int m = 0; m < BLOCKS; ++m) dq[m] = sl_mfma(sl_turned<D>(kt, turned, m, j), ds, dq[m]);
        }
        again(n);
    }
    wait_dma<0>();
    __syncthreads();
    float *room = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) sl_leave_block(room + (wave * BLOCKS + m) * 1024, lane, dq[m]);
    __syncthreads();
    for (int m = wave; m < BLOCKS; m += 4)
        sl_put_block(A.dq.p + token * A.dq.token + head * A.dq.head, row < at.count, half, A.s.octets,
                     sl_four_blocks(room + m * 1024, BLOCKS * 1024, lane, sl_f4{1.0f, 1.0f, 1.0f, 1.0f}), m, A.s.scale);
    if (row < at.count && wave == 0 && half == 0) {
        float *to = A.stats + (long long)head * A.s.tokens_q + token;
        to[0] = lse2;
        to[(long long)A.s.heads * A.s.tokens_q] = delta;
    }
}

// Which heads of its group workgroup `item` of the passes over keys walks past, and where it leaves what it finds.
struct Slice { int kv, slice, first, heads; };
SL_DEV Slice slice_of(const BackArgs &A, unsigned item)
{
    const int kv = (int)item / A.slices, slice = (int)item % A.slices, first = slice * A.s.group / A.slices;
    return Slice{kv, slice, kv * A.s.group + first, (slice + 1) * A.s.group / A.slices - first};
}
SL_DEV float *part_row(const BackArgs &A, const Slice &w, int which, long long token)
{
    return A.parts + ((((long long)w.slice * 2 + which) * A.s.tokens_k + token) * (A.s.heads / A.s.group) + w.kv) * (A.s.octets * 8);
}

// Scores and dP of 32 queries (rows 8 j + e of a lane) into P and dS; queries before row `from` do not see the lane's key.
SL_DEV void back_scores(sl_f16 &s, sl_f16 &dp, const float *stats, int from, float scale2)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const sl_f4 lse = *reinterpret_cast<const sl_f4 *>(stats + 8 * j), delta = *reinterpret_cast<const sl_f4 *>(stats + 32 + 8 * j);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = fmaf(s[4 * j + e], scale2, -lse[e]);
            s[4 * j + e] = __builtin_amdgcn_exp2f(8 * j + e < from ? -INFINITY : x);
            dp[4 * j + e] = s[4 * j + e] * (dp[4 * j + e] - delta[e]);
        }
    }
}

// dk and dv: 128 keys of one key head, 32 to a wave, over all queries of the heads that share it, 32 at a time; the sums over the heads are
// made in registers, in their order.  A wave holds its keys in registers and its values in LDS, so that two workgroups fit a compute unit
// and some of one's exponentials run beside the other's products: 8 x 2048 tokens, 16 heads of 128, 300 to 320 us, 0.86 to 0.92 PFLOP/s, the
// matrix unit busy 45 % of the time, the vector unit 38, LDS 34 (keys and values in registers, one workgroup to a compute unit, 412 us).
template <int D>
__global__ void __launch_bounds__(256, 2) k_back_kv(BackArgs A)
{
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int VALUES = AT_ROWS * 2 * D, TILE = AT_STAGE * 2 * D, STAGE = 2 * TILE + 256, STEPS = D / 16, BLOCKS = D / 32;
    const SlItem item = sl_item(blockIdx.x, (unsigned)(A.s.heads / A.s.group * A.slices));
    if (item.tile >= A.s.tiles) return;
    SlSpan at;
    int q0, qn;
    if (!sl_find(A.s.k_start, A.s.tokens_k, A.s.q_start, nullptr, A.s.tokens_q, A.s, AT_ROWS, item.tile, false, at, q0, qn)) return;
    const int k0 = at.first, kn = A.s.k_count ? min(max(A.s.k_count[at.s], 0), at.count) : at.count;
    if (at.row0 >= kn) return;
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), half = lane >> 5;
    const Slice work = slice_of(A, item.head);
    const int kv = work.kv, shift = kn - qn;
    const int key = at.row0 + wave * 32 + (lane & 31), mine = min(key, kn - 1);
    const long long token = k0 + mine;
    const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char *)lds;
    {
        SlTileLoad<D, AT_ROWS> lv;
        lv.setup(wave, lane, A.s.octets, A.v.token);
        lv.load(A.v.p + (long long)k0 * A.v.token + kv * A.v.head, at.row0, kn, lds0, wave);
    }
    sl_b8 k[STEPS];
    sl_own_row<D>(A.k.p + token * A.k.token + kv * A.k.head, half, A.s.octets, k);
    SlTileLoad<D, AT_STAGE> lq, lg;
    lq.setup(wave, lane, A.s.octets, A.q.token);
    lg.setup(wave, lane, A.s.octets, A.dout.token);
    const int plain = sl_plain_base<D>(lane), turned = sl_turned_base<D>(lane);
    sl_f16 dk[BLOCKS], dv[BLOCKS];
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) dk[m] = dv[m] = sl_zero16();
    // the first query that sees a key of the workgroup, of the wave, this lane's key
    const int first = A.s.causal ? max(at.row0 - shift, 0) / AT_STAGE : 0, tiles = (qn + AT_STAGE - 1) / AT_STAGE;
    const int wave_first = A.s.causal ? at.row0 + wave * 32 - shift : 0, key_first = A.s.causal ? key - shift : 0;
    const int per_head = max(tiles - first, 0), stages = per_head * work.heads;
    auto load = [&](int i) __attribute__((always_inline)) {
        const int head = work.first + i / per_head, tile = (first + i % per_head) * AT_STAGE;
        const unsigned to = lds0 + VALUES + (unsigned)(i & 1) * STAGE;
        lq.load(A.q.p + (long long)q0 * A.q.token + head * A.q.head, tile, qn, to, wave);
        lg.load(A.dout.p + (long long)q0 * A.dout.token + head * A.dout.head, tile, qn, to + TILE, wave);
        if (wave == 0) {
            const int row = tile + (lane & 31);
            const float *stats = A.stats + ((long long)half * A.s.heads + head) * A.s.tokens_q + q0 + row;
            dma4(row < qn ? stats : A.stats + A.none + half, to + 2 * TILE);
        }
    };
    if (stages > 0) load(0);
    if (A.s.octets < D / 8) {
        // (both operands of dP come out of LDS: one of them has to be zero past the last column)
        wait_dma<0>();
        __syncthreads();
        const int pieces = D / 8 - A.s.octets;
        for (int i = threadIdx.x; i < AT_ROWS * pieces; i += 256) {
            const int r = i / pieces, c = A.s.octets + i % pieces;
            *reinterpret_cast<sl_u4 *>(lds + r * (2 * D) + ((c ^ sl_turn<D>(r)) << 4)) = sl_u4{0u, 0u, 0u, 0u};
        }
    }
#pragma unroll 1
    for (int n = 0; n < stages; ++n) {
        wait_dma<0>();
        stage_barrier();
        if (n + 1 < stages) load(n + 1);
        const int tile = (first + n % per_head) * AT_STAGE;
        if (tile + AT_STAGE <= wave_first) continue;
        const unsigned char *qt = lds + VALUES + (n & 1) * STAGE, *gt = qt + TILE;
        const float *stats = reinterpret_cast<const float *>(qt + 2 * TILE) + 4 * half;
        sl_f16 s = sl_zero16(), dp = sl_zero16();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < STEPS; ++j) s = sl_mfma(sl_plain<D>(qt, plain, 0, j), k[j], s);
#pragma unroll
        for (int j = 0; j < STEPS; ++j) dp = sl_mfma(sl_plain<D>(gt, plain, 0, j), sl_plain<D>(lds, plain, wave, j), dp);
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        back_scores(s, dp, stats, key_first - tile - 4 * half, A.s.scale2);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const sl_b8 p = sl_operand(s, j), ds = sl_operand(dp, j);
#pragma unroll
            for (int m = 0; m < BLOCKS; ++m) {
                dv[m] = sl_mfma(sl_turned<D>(gt, turned, m, j), p, dv[m]);
                dk[m] = sl_mfma(sl_turned<D>(qt, turned, m, j), ds, dk[m]);
            }
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
        for (int j = 0; j < 4 * BLOCKS; ++j) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
    }
    wait_dma<0>();               // (the values, where there was no stage)
    if (A.slices > 1) {
        float *to_k = part_row(A, work, 0, token), *to_v = part_row(A, work, 1, token);
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m) {
            sl_put_floats(to_k, key < kn, half, A.s.octets, dk[m], m);
            sl_put_floats(to_v, key < kn, half, A.s.octets, dv[m], m);
        }
        return;
    }
    sl_put_row<D>(A.dk.p + token * A.dk.token + kv * A.dk.head, key < kn, half, A.s.octets, dk, A.s.scale);
    sl_put_row<D>(A.dv.p + token * A.dv.token + kv * A.dv.head, key < kn, half, A.s.octets, dv, 1.0f);
}

// Few tiles: 32 keys to a workgroup, whose four waves take every fourth 32 queries (of the heads that share the keys, one head after the
// other), in LDS of their own, and wait for nobody; their sums meet at the end.
template <int D>
__global__ void __launch_bounds__(256, 1) k_back_kv_few(BackArgs A)
{
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int TILE = AT_STAGE * 2 * D, STAGE = 2 * TILE + 256, STEPS = D / 16, BLOCKS = D / 32, LOADS = 2 * SlWaveLoad<D>::LOADS + 1;
    const SlItem item = sl_item(blockIdx.x, (unsigned)(A.s.heads / A.s.group * A.slices));
    if (item.tile >= A.s.tiles) return;
    SlSpan at;
    int q0, qn;
    if (!sl_find(A.s.k_start, A.s.tokens_k, A.s.q_start, nullptr, A.s.tokens_q, A.s, 32, item.tile, false, at, q0, qn)) return;
    const int k0 = at.first, kn = A.s.k_count ? min(max(A.s.k_count[at.s], 0), at.count) : at.count;
    if (at.row0 >= kn) return;
    const int lane = threadIdx.x & 63, wave = sl_uniform((int)(threadIdx.x >> 6)), half = lane >> 5;
    const Slice work = slice_of(A, item.head);
    const int kv = work.kv, shift = kn - qn;
    const int key = at.row0 + (lane & 31), mine = min(key, kn - 1);
    const long long token = k0 + mine;
    unsigned char *own = lds + wave * (2 * STAGE);
    const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char *)own;
    SlWaveLoad<D> lq, lg;
    lq.setup(lane, A.s.octets, A.q.token);
    lg.setup(lane, A.s.octets, A.dout.token);
    const int first = A.s.causal ? max(at.row0 - shift, 0) / AT_STAGE : 0, tiles = (qn + AT_STAGE - 1) / AT_STAGE;
    const int key_first = A.s.causal ? key - shift : 0;
    const int per_head = max(tiles - first, 0), stages = per_head * work.heads, steps = stages > wave ? (stages - wave + 3) / 4 : 0;
    auto fill = [&](int n) __attribute__((always_inline)) {
        const int i = wave + 4 * min(n, steps - 1), head = work.first + i / per_head, tile = (first + i % per_head) * AT_STAGE;
        const unsigned to = lds0 + (unsigned)(n & 1) * STAGE;
        lq.load(A.q.p + (long long)q0 * A.q.token + head * A.q.head, tile, qn - tile, to);
        lg.load(A.dout.p + (long long)q0 * A.dout.token + head * A.dout.head, tile, qn - tile, to + TILE);
        const int row = tile + (lane & 31);
        const float *stats = A.stats + ((long long)half * A.s.heads + head) * A.s.tokens_q + q0 + row;
        dma4(row < qn ? stats : A.stats + A.none + half, to + 2 * TILE);
    };
    if (steps > 0) fill(0), fill(1);
    sl_b8 k[STEPS], v[STEPS];
    sl_own_row<D>(A.k.p + token * A.k.token + kv * A.k.head, half, A.s.octets, k);
    sl_own_row<D>(A.v.p + token * A.v.token + kv * A.v.head, half, A.s.octets, v);
    const int plain = sl_plain_base<D>(lane), turned = sl_turned_base<D>(lane);
    sl_f16 dk[BLOCKS], dv[BLOCKS];
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) dk[m] = dv[m] = sl_zero16();
#pragma unroll 1
    for (int n = 0; n < steps; ++n) {
        wait_dma<LOADS>();
        const int tile = (first + (wave + 4 * n) % per_head) * AT_STAGE;
        const unsigned char *qt = own + (n & 1) * STAGE, *gt = qt + TILE;
        const float *stats = reinterpret_cast<const float *>(qt + 2 * TILE) + 4 * half;
        sl_f16 s = sl_zero16(), dp = sl_zero16();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            s = sl_mfma(sl_plain<D>(qt, plain, 0, j), k[j], s);
            dp = sl_mfma(sl_plain<D>(gt, plain, 0, j), v[j], dp);
        }
        sl_reads_ahead<2 * STEPS, 8>();
        __builtin_amdgcn_sched_barrier(0);
        back_scores(s, dp, stats, key_first - tile - 4 * half, A.s.scale2);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const sl_b8 p = sl_operand(s, j), ds = sl_operand(dp, j);
#pragma unroll
            for (int m = 0; m < BLOCKS; ++m) {
                dv[m] = sl_mfma(sl_turned<D>(gt, turned, m, j), p, dv[m]);
                dk[m] = sl_mfma(sl_turned<D>(qt, turned, m, j), ds, dk[m]);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // (the stage has been read)
        fill(n + 2);
    }
    wait_dma<0>();
    __syncthreads();
    float *room = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) {
        sl_leave_block(room + (wave * 2 * BLOCKS + m) * 1024, lane, dk[m]);
        sl_leave_block(room + (wave * 2 * BLOCKS + BLOCKS + m) * 1024, lane, dv[m]);
    }
    __syncthreads();
    for (int i = wave; i < 2 * BLOCKS; i += 4) {
        const sl_f16 x = sl_four_blocks(room + i * 1024, 2 * BLOCKS * 1024, lane, sl_f4{1.0f, 1.0f, 1.0f, 1.0f});
        if (A.slices > 1) sl_put_floats(part_row(A, work, i < BLOCKS ? 0 : 1, token), key < kn, half, A.s.octets, x, i < BLOCKS ? i : i - BLOCKS);
        else if (i < BLOCKS) sl_put_block(A.dk.p + token * A.dk.token + kv * A.dk.head, key < kn, half, A.s.octets, x, i, A.s.scale);
        else sl_put_block(A.dv.p + token * A.dv.token + kv * A.dv.head, key < kn, half, A.s.octets, x, i - BLOCKS, 1.0f);
    }
}

// dk and dv from the slices' sums, in their order: 128 keys of one key head to a workgroup, eight elements to a thread.
__global__ void __launch_bounds__(256) k_join_kv(BackArgs A)
{
    const int kv_heads = A.s.heads / A.s.group;
    const SlItem item = sl_item(blockIdx.x, (unsigned)kv_heads);
    if (item.tile >= A.s.tiles) return;
    SlSpan at;
    if (!sl_find_tile(A.s.k_start, A.s.n, A.s.tokens_k, AT_ROWS, item.tile, at)) return;
    const int kn = A.s.k_count ? min(max(A.s.k_count[at.s], 0), at.count) : at.count, rows = min(AT_ROWS, kn - at.row0), kv = (int)item.head;
    for (int i = threadIdx.x; i < rows * A.s.octets; i += 256) {
        const long long token = at.first + at.row0 + i / A.s.octets;
        const int octet = i % A.s.octets;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.0f;
#pragma unroll 4
            for (int slice = 0; slice < A.slices; ++slice) {
                const float *p = part_row(A, Slice{kv, slice, 0, 0}, which, token) + octet * 8;
                const sl_f4 a = *reinterpret_cast<const sl_f4 *>(p), b = *reinterpret_cast<const sl_f4 *>(p + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = v[e] + a[e], v[4 + e] = v[4 + e] + b[e];
            }
            const float by = which == 0 ? A.s.scale : 1.0f;
            const SlRows &to = which == 0 ? A.dk : A.dv;
            *reinterpret_cast<sl_u4 *>(to.p + token * to.token + kv * to.head + octet * 16) =
                sl_u4{sl_bf16_pair(v[0] * by, v[1] * by), sl_bf16_pair(v[2] * by, v[3] * by), sl_bf16_pair(v[4] * by, v[5] * by), sl_bf16_pair(v[6] * by, v[7] * by)};
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

// 32 rows to a workgroup, which splits the other side among its waves, or 128.  With W workgroups of 128 rows that each walk a mean of `walk`
// rows, these all run at once below two to a compute unit, and take as long as the longest walk; the others take a quarter of the walk each,
// four times as many of them, one (heads up to 64: two) to a compute unit, and a start of about 4 us every time.  So the limit
// rises with the walk to 400 (900), and is 64 (128) where four times as many still run at once.  Forward, us, 32 rows / 128, 16 heads of 128: 2 x 1024 tokens (W = 288) 37 / 26, 2048 (272) 48 / 44, 4 heads, 8192 (260)
// 125 / 178; 16 heads of 64: 4 x 1024 (576) 32 / 22, 2048 (272) 25 / 36, 4096 (528) 67 / 69; keys and values, 4 heads of 64 for 16, 9 sequences up to 1021 (160) 46 / 151.
bool few_tiles(int64_t rows, int64_t n, int64_t heads, int64_t other, int64_t times, bool narrow)
{
    const int64_t w = (rows / AT_ROWS + n) * heads, walk = other / n * times;
    return w <= (narrow ? 128 : 64) || w * (walk + 1400) < (narrow ? 900 : 400) * walk;
}
unsigned tile_count(int64_t tokens, int64_t n, bool few) { return (unsigned)(tokens / (few ? 32 : AT_ROWS) + n); }

template <class Args>
int launch(void (*k)(Args), const Args &A, long long heads, unsigned lds, hipStream_t st)
{
    if (lds > 65536) {
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (err != hipSuccess) {
            sl_note_hip_error(err);
            return SL_ERR_HIP;
        }
    }
    hipLaunchKernelGGL(k, dim3(sl_item_groups(A.s.tiles, heads)), dim3(256), lds, st, A);
    return check_launch();
}

}  // namespace

extern "C" {

int sl_attention(const sl_attention_shape *shape, const sl_heads *q, const sl_heads *k, const sl_heads *v, const sl_heads *out, float *lse,
                 void *stream)
{
    AttendArgs A = {};
    if (!sl_attention_sequences(shape, A.s) || ((uintptr_t)lse & 3)) return SL_ERR_INVALID_ARG;
    if (A.s.tokens_q == 0 || A.s.n == 0) return SL_OK;
    const bool keys = A.s.tokens_k > 0;
    const int64_t dim = shape->head_dim;
    if (!shape->q_start || !sl_attention_in(q, true, A.q) || !sl_attention_in(k, keys, A.k) || !sl_attention_in(v, keys, A.v) ||
        !sl_attention_out(out, true, A.s.tokens_q, A.s.heads, dim, A.out))
        return SL_ERR_INVALID_ARG;
    if (out->data == q->data || (keys && (out->data == k->data || out->data == v->data)) || out->data == (void *)lse) return SL_ERR_INVALID_ARG;
    A.lse = lse;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool narrow = A.s.octets <= 8, few = few_tiles(A.s.tokens_q, A.s.n, A.s.heads, A.s.tokens_k, 1, narrow);
    const unsigned tile = AT_TILE * 2 * (narrow ? 64 : 128);
    A.s.tiles = tile_count(A.s.tokens_q, A.s.n, few);
    if (few) return launch(narrow ? k_attend_few<64> : k_attend_few<128>, A, A.s.heads, 8 * tile, st);
    return launch(narrow ? k_attend<64> : k_attend<128>, A, A.s.heads, 4 * tile, st);
}

size_t sl_attention_group_workspace_bytes(int64_t tokens_q, int heads, int kv_heads, int head_dim)
{
    if (tokens_q < 1 || tokens_q > AT_MOST_TOKENS || heads < 1 || heads > AT_MOST_HEADS || kv_heads < 1 || heads % kv_heads != 0 || head_dim < 8 ||
        head_dim > 128 || head_dim % 8 != 0)
        return 0;
    return sizeof(float) * (size_t)sl_back_room(tokens_q, heads, kv_heads, head_dim);
}

size_t sl_attention_workspace_bytes(int64_t tokens_q, int64_t heads)
{
    if (tokens_q < 1 || heads < 1 || tokens_q > AT_MOST_TOKENS || heads > AT_MOST_HEADS) return 0;
    return sizeof(float) * (size_t)sl_back_room(tokens_q, heads, 1, 128);
}

int sl_attention_backward(const sl_attention_shape *shape, const sl_heads *q, const sl_heads *k, const sl_heads *v, const sl_heads *out,
                          const float *lse, const sl_heads *dout, const sl_heads *dq, const sl_heads *dk, const sl_heads *dv, void *workspace,
                          void *stream)
{
    BackArgs A = {};
    if (!sl_attention_sequences(shape, A.s)) return SL_ERR_INVALID_ARG;
    const bool queries = A.s.tokens_q > 0, keys = A.s.tokens_k > 0;
    if (A.s.n == 0 || (!queries && !keys)) return SL_OK;
    const int64_t dim = shape->head_dim, kv_heads = shape->kv_heads;
    if (!shape->q_start || !sl_attention_in(q, queries, A.q) || !sl_attention_in(out, queries, A.out) || !sl_attention_in(dout, queries, A.dout) ||
        !sl_attention_in(k, keys, A.k) || !sl_attention_in(v, keys, A.v) || !sl_attention_out(dq, queries, A.s.tokens_q, A.s.heads, dim, A.dq) ||
        !sl_attention_out(dk, keys, A.s.tokens_k, kv_heads, dim, A.dk) || !sl_attention_out(dv, keys, A.s.tokens_k, kv_heads, dim, A.dv))
        return SL_ERR_INVALID_ARG;
    if (queries && (!lse || !workspace || ((uintptr_t)lse & 3) || ((uintptr_t)workspace & 15) || (const void *)lse == workspace)) return SL_ERR_INVALID_ARG;
    const void *in[6] = {queries ? q->data : nullptr, queries ? out->data : nullptr, queries ? dout->data : nullptr, keys ? k->data : nullptr, keys ? v->data : nullptr, workspace};
    const void *res[3] = {queries ? dq->data : nullptr, keys ? dk->data : nullptr, keys ? dv->data : nullptr};
    for (int i = 0; i < 3; ++i)
        for (int j = 0; res[i] && j < 6 + i; ++j)
            if (res[i] == (j < 6 ? in[j] : res[j - 6])) return SL_ERR_INVALID_ARG;
    A.lse = lse, A.stats = static_cast<float *>(workspace), A.none = 2ll * A.s.heads * A.s.tokens_q;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool narrow = A.s.octets <= 8;
    const unsigned tile = AT_TILE * 2 * (narrow ? 64 : 128);
    if (queries) {
        const bool few = few_tiles(A.s.tokens_q, A.s.n, A.s.heads, A.s.tokens_k, 1, narrow);
        A.s.tiles = tile_count(A.s.tokens_q, A.s.n, few);
        if (const int rc = few ? launch(narrow ? k_back_q_few<64> : k_back_q_few<128>, A, A.s.heads, 8 * tile, st)
                               : launch(narrow ? k_back_q<64> : k_back_q<128>, A, A.s.heads, 4 * tile, st))
            return rc;
    }
    if (!keys) return SL_OK;
    A.slices = sl_back_slices(A.s.tokens_q, A.s.tokens_k, A.s.n, A.s.heads, kv_heads);
    A.parts = A.stats + sl_back_stats(A.s.tokens_q, A.s.heads);
    const bool few = few_tiles(A.s.tokens_k, A.s.n, kv_heads * A.slices, A.s.tokens_q, (A.s.group + A.slices - 1) / A.slices, narrow);
    A.s.tiles = tile_count(A.s.tokens_k, A.s.n, few);
    if (const int rc = few ? launch(narrow ? k_back_kv_few<64> : k_back_kv_few<128>, A, kv_heads * A.slices, 8 * tile + 2048, st)
                           : launch(narrow ? k_back_kv<64> : k_back_kv<128>, A, kv_heads * A.slices, 4 * tile + 512, st))
        return rc;
    if (A.slices == 1) return SL_OK;
    A.s.tiles = tile_count(A.s.tokens_k, A.s.n, false);
    return launch(k_join_kv, A, kv_heads, 0, st);
}

}  // extern "C"
