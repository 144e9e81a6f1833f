"""Attention over packed sequences, its backward pass and its form for single tokens against their definitions in 64 bits."""
import math

import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


def tensors(tokens_q, tokens_k, heads, kv_heads, dim, seed=0, std=1.0):
    """q, k, v, dout as views of wider tensors: rows of q and of k and v lie between those of others."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*s):
        return torch.empty(*s, device="cuda").normal_(0, std, generator=g).bfloat16()
    q = normal(tokens_q, heads + 1, dim + 8)[:, :heads, 8:]
    kv = normal(tokens_k, 2 * kv_heads, dim)
    return q, kv[:, :kv_heads], kv[:, kv_heads:], normal(heads, tokens_q, dim).transpose(0, 1)


def starts(lengths, first=0):
    import torch
    s = [first]
    for n in lengths:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32, device="cuda")


def worst(got, want, off):
    got = got.double()
    bound = off + HALF * (want.abs() + off) + 1e-30
    return float(((got - want).abs() / bound).max()) if got.numel() else 0.0


def check(q, k, v, dout, q_lengths, k_lengths, causal, scale, k_count=None, first=0, tail=0):
    """Runs both passes and compares every sequence and head; everything outside the sequences stays as it was."""
    import torch
    from paper_2508_15706_amd import binding as sl
    heads, kv_heads, dim = q.shape[1], k.shape[1], q.shape[2]
    qs, ks = starts(q_lengths, first), starts(k_lengths, first)
    count = None if k_count is None else torch.tensor(k_count, dtype=torch.int32, device="cuda")
    out = torch.full((heads, q.shape[0], dim), 9.0, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    lse = torch.full((heads, q.shape[0]), 9.0, device="cuda")
    sl.sl_attention(q, k, v, out, qs, ks, count, scale=scale, causal=causal, lse=lse)
    dq = torch.full((q.shape[0], heads, dim), 9.0, device="cuda", dtype=torch.bfloat16)
    dkv = torch.full((k.shape[0], kv_heads, 2, dim), 9.0, device="cuda", dtype=torch.bfloat16)
    dk, dv = dkv[:, :, 0], dkv[:, :, 1]
    ws = sl.alloc_attention_workspace(q.shape[0], heads)
    sl.sl_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, qs, ks, count, scale=scale, causal=causal, workspace=ws)
    used_q, used_k = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda"), torch.zeros(k.shape[0], dtype=torch.bool, device="cuda")
    group, s = heads // kv_heads, dim ** -0.5 if scale is None else scale
    for i, (n, m) in enumerate(zip(q_lengths, k_lengths)):
        a, b = int(qs[i]), int(ks[i])
        m = m if k_count is None else k_count[i]
        rows, keys = slice(a, a + n), slice(b, b + m)
        used_q[rows], used_k[keys] = True, True
        for g in range(kv_heads):
            sums = {"dk": 0.0, "dv": 0.0, "dk_off": 0.0, "dv_off": 0.0}
            for h in range(g * group, (g + 1) * group):
                r = ref.attention(q[rows, h], k[keys, g], v[keys, g], causal, s, dout[rows, h])
                where = (i, h, n, m)
                assert worst(out[rows, h], r["out"], r["out_off"]) <= 1.0, ("out", where)
                assert worst(dq[rows, h], r["dq"], r["dq_off"]) <= 1.0, ("dq", where)
                seen = r["lse"] > -math.inf
                assert bool((lse[h, rows][~seen] == -math.inf).all()) and bool((out[rows, h][~seen] == 0).all()), where
                assert bool((dq[rows, h][~seen] == 0).all())
                assert bool(((lse[h, rows].double() - r["lse"])[seen].abs() <= r["lse_off"][seen]).all()), ("lse", where)
                for name in sums:
                    sums[name] = sums[name] + r[name]
            assert worst(dk[keys, g], sums["dk"], sums["dk_off"]) <= 1.0, ("dk", where)
            assert worst(dv[keys, g], sums["dv"], sums["dv_off"]) <= 1.0, ("dv", where)
    assert bool((out[~used_q] == 9).all()) and bool((lse[:, ~used_q] == 9).all()) and bool((dq[~used_q] == 9).all())
    assert bool((dk[~used_k] == 9).all()) and bool((dv[~used_k] == 9).all())
    return out, lse, dq, dk, dv


@pytest.mark.parametrize("dim", [8, 40, 64, 72, 128])
@pytest.mark.parametrize("length", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257, 385])
def test_one_sequence(length, dim):
    q, k, v, dout = tensors(length, length, 2, 1, dim, seed=length)
    check(q, k, v, dout, [length], [length], True, None)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (4, 2), (5, 1), (8, 8), (9, 3), (16, 2), (20, 5)])
@pytest.mark.parametrize("causal", [True, False])
def test_packed(heads, kv_heads, causal):
    lengths = [70, 1, 0, 129, 5, 64, 0, 33]
    q, k, v, dout = tensors(sum(lengths), sum(lengths), heads, kv_heads, 64, seed=heads)
    check(q, k, v, dout, lengths, lengths, causal, 0.2)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_different_lengths_on_both_sides(dim, causal):
    """Fewer queries than keys (a prompt behind a cache), more (queries that see nothing), none on either side."""
    qn, kn = [3, 130, 200, 0, 17, 65, 1], [200, 300, 70, 40, 0, 64, 193]
    q, k, v, dout = tensors(sum(qn), sum(kn), 4, 2, dim, seed=3)
    check(q, k, v, dout, qn, kn, causal, None)


def test_parts_of_a_cache_are_used():
    """k_count: rows past it, before the first sequence and behind the last hold NaN, which reaches nothing."""
    import torch
    qn, room, count = [5, 70, 1, 9], [40, 200, 64, 32], [33, 130, 0, 32]
    first, tail = 11, 13
    q, k, v, dout = tensors(first + sum(qn) + tail, first + sum(room) + tail, 4, 2, 64, seed=4)
    ks = starts(room, first)
    unused = torch.ones(k.shape[0], dtype=torch.bool, device="cuda")
    for i, n in enumerate(count):
        unused[int(ks[i]):int(ks[i]) + n] = False
    k[unused], v[unused] = math.nan, math.nan
    for t in (q, dout):
        t[:first], t[first + sum(qn):] = math.nan, math.nan
    check(q, k, v, dout, qn, room, True, None, k_count=count, first=first, tail=tail)


def test_sequences_are_apart():
    """NaN and infinities in one sequence leave the others' bits as they were."""
    import torch
    lengths = [100, 64, 90]
    q, k, v, dout = tensors(sum(lengths), sum(lengths), 2, 2, 64, seed=5)
    clean = check(q, k, v, dout, lengths, lengths, True, None)
    from paper_2508_15706_amd import binding as sl
    q[110], k[120], v[130], dout[140] = math.nan, math.inf, math.nan, -math.inf
    qs = starts(lengths)
    out, lse = torch.empty_like(q), torch.empty(2, q.shape[0], device="cuda")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    sl.sl_attention(q, k, v, out, qs, lse=lse)
    sl.sl_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, qs, workspace=sl.alloc_attention_workspace(q.shape[0], 2))
    keep = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
    keep[100:164] = False
    for got, want in zip((out, dq, dk, dv), (clean[0], *clean[2:])):
        assert torch.equal(got[keep], want[keep])
    assert torch.equal(lse[:, keep], clean[1][:, keep])


@pytest.mark.parametrize("std", [0.01, 4.0, 30.0])
def test_flat_and_peaked_scores(std):
    """Scores of almost nothing and of thousands: one key takes all of a query."""
    q, k, v, dout = tensors(150, 150, 2, 1, 128, seed=6, std=std)
    check(q, k, v, dout, [150], [150], True, None)


def test_rising_scores():
    """The running maximum moves in every tile, by less and by more than what a row is scaled for at once."""
    import torch
    for slope in (0.02, 0.4):
        q, k, v, dout = tensors(300, 300, 1, 1, 64, seed=7, std=0.1)
        q[:, 0, 0] = 1.0
        k[:, 0, 0] = (torch.arange(300, device="cuda") * slope).bfloat16()
        check(q, k, v, dout, [300], [300], True, 1.0)


def test_the_same_bits_again():
    import torch
    from paper_2508_15706_amd import binding as sl
    lengths = [300, 17, 211]
    q, k, v, dout = tensors(sum(lengths), sum(lengths), 8, 2, 128, seed=8)
    qs = starts(lengths)
    results = []
    for _ in range(2):
        out, lse = torch.empty_like(q), torch.empty(8, q.shape[0], device="cuda")
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        sl.sl_attention(q, k, v, out, qs, lse=lse)
        sl.sl_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, qs, workspace=sl.alloc_attention_workspace(q.shape[0], 8))
        results.append((out, lse, dq, dk, dv))
    for a, b in zip(*results):
        assert torch.equal(a, b)


# ---- single tokens ----

@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 8), (4, 4, 64), (5, 1, 40), (16, 16, 128), (20, 5, 128), (40, 1, 64), (66, 2, 72)])
@pytest.mark.parametrize("room,count", [([1], None), ([40], [33]), ([128], None), ([129, 1, 0, 64], None), ([300, 300, 300], [0, 1, 299]), ([2500, 700], [2500, 3]),
                                        ([9000], None)])
def test_token(heads, kv_heads, dim, room, count):
    import torch
    from paper_2508_15706_amd import binding as sl
    n = len(room)
    q, k, v, _ = tensors(n, sum(room) + 7, heads, kv_heads, dim, seed=dim)
    ks = starts(room)
    used = room if count is None else count
    free = torch.ones(k.shape[0], dtype=torch.bool, device="cuda")
    for i, m in enumerate(used):
        free[int(ks[i]):int(ks[i]) + m] = False
    k[free], v[free] = math.nan, math.nan
    out = torch.full((n, heads, dim + 8), 9.0, device="cuda", dtype=torch.bfloat16)
    c = None if count is None else torch.tensor(count, dtype=torch.int32, device="cuda")
    ws = sl.alloc_attention_token_workspace(n, k.shape[0], heads, kv_heads, dim).fill_(255)
    sl.sl_attention_token(q, k, v, out[:, :, :dim], ks, c, scale=0.3, workspace=ws)
    for i, m in enumerate(used):
        for h in range(heads):
            g = h // (heads // kv_heads)
            keys = slice(int(ks[i]), int(ks[i]) + m)
            r = ref.attention(q[i:i + 1, h], k[keys, g], v[keys, g], False, 0.3)
            assert worst(out[i:i + 1, h, :dim], r["out"], r["out_off"]) <= 1.0, (i, h, m)
    assert bool((out[:, :, dim:] == 9).all())


def test_token_is_the_last_row_of_a_prompt():
    import torch
    from paper_2508_15706_amd import binding as sl
    lengths = [300, 1, 77]
    q, k, v, _ = tensors(sum(lengths), sum(lengths), 8, 2, 128, seed=9)
    qs = starts(lengths)
    out = torch.empty_like(q)
    sl.sl_attention(q, k, v, out, qs)
    last = (qs[1:] - 1).long()
    one = torch.empty(3, 8, 128, device="cuda", dtype=torch.bfloat16)
    sl.sl_attention_token(q[last], k, v, one, qs, workspace=sl.alloc_attention_token_workspace(3, k.shape[0], 8, 2, 128))
    assert float((one.float() - out[last].float()).abs().max()) <= 3 * HALF * float(v.float().abs().max())


# ---- starts that are none ----

def test_starts_outside_the_tokens_are_cut_off():
    """Nothing outside the tensors is read or written (their ends are checked by the guards around them), and sequences that are well formed
    have their results."""
    import torch
    from paper_2508_15706_amd import binding as sl
    q, k, v, dout = tensors(200, 200, 2, 1, 64, seed=10)
    want = torch.empty_like(q)
    sl.sl_attention(q, k, v, want, torch.tensor([0, 120, 200], dtype=torch.int32, device="cuda"))
    for bad in ([0, 120, 100000], [-50, 120, 200], [0, 120, 2**31 - 1]):
        s = torch.tensor(bad, dtype=torch.int32, device="cuda")
        room = torch.full((202, 2, 64), 9.0, device="cuda", dtype=torch.bfloat16)
        sl.sl_attention(q, k, v, room[1:201], s)
        assert torch.equal(room[1:201], want) and bool((room[0] == 9).all()) and bool((room[201] == 9).all())
    lse = torch.zeros(2, 200, device="cuda")
    count = torch.tensor([2**31 - 1, -5, 2**31 - 1], dtype=torch.int32, device="cuda")
    for bad in ([150, 20, 90, 10], [2**31 - 1] * 4, [-2**31] * 4, [0, 0, 200, 0]):
        s = torch.tensor(bad, dtype=torch.int32, device="cuda")
        for c in (None, count):
            room, back = torch.full((202, 2, 64), 9.0, device="cuda", dtype=torch.bfloat16), torch.full((3, 202, 2, 64), 9.0, device="cuda", dtype=torch.bfloat16)
            sl.sl_attention(q, k, v, room[1:201], s, s, c, lse=lse)
            sl.sl_attention_backward(q, k, v, room[1:201], lse, dout, back[0, 1:201], back[1, 1:201, :1], back[2, 1:201, :1], s, s, c,
                                     workspace=sl.alloc_attention_workspace(200, 2))
            assert bool((room[[0, 201]] == 9).all()) and bool((back[:, [0, 201]] == 9).all())
            one = torch.full((5, 2, 64), 9.0, device="cuda", dtype=torch.bfloat16)
            sl.sl_attention_token(q[:3], k, v, one[1:4], s, c, workspace=sl.alloc_attention_token_workspace(3, 200, 2, 1, 64))
            assert bool((one[[0, 4]] == 9).all())


# ---- long lists: workgroups of 128 rows ----

@pytest.mark.parametrize("dim", [40, 64, 104, 128])
@pytest.mark.parametrize("length", [1, 63, 64, 65, 127, 128, 129, 200, 257, 385])
def test_many_heads(length, dim):
    """Enough heads for workgroups of 128 rows; a few of the heads are compared, all of them are finite."""
    import torch
    from paper_2508_15706_amd import binding as sl
    heads = 200
    q, k, v, dout = tensors(length, length, heads, heads, dim, seed=length)
    s = starts([length])
    out, lse = torch.empty(length, heads, dim, device="cuda", dtype=torch.bfloat16), torch.empty(heads, length, device="cuda")
    dq, dk, dv = (torch.empty_like(out) for _ in range(3))
    sl.sl_attention(q, k, v, out, s, lse=lse)
    sl.sl_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, s, workspace=sl.alloc_attention_workspace(length, heads))
    for h in (0, 1, 24, 25, 100, 191, 192, 199):
        r = ref.attention(q[:, h], k[:, h], v[:, h], True, dim ** -0.5, dout[:, h])
        for name, t in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
            assert worst(t[:, h], r[name], r[name + "_off"]) <= 1.0, (name, h)
        assert bool(((lse[h].double() - r["lse"]).abs() <= r["lse_off"]).all())
    assert all(bool(t.isfinite().all()) for t in (out, lse, dq, dk, dv))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_many_sequences_of_both_lengths(dim, causal):
    """Workgroups of 128 rows with fewer queries than keys, more, none, and grouped heads."""
    qn, kn = [3, 130, 200, 0, 17, 65, 1, 260], [200, 300, 70, 40, 0, 64, 193, 260]
    q, k, v, dout = tensors(sum(qn), sum(kn), 48, 24, dim, seed=3)
    check(q, k, v, dout, qn, kn, causal, None)


@pytest.mark.parametrize("qn,kn,count,heads,kv_heads,dim", [
    ([700], [700], None, 8, 1, 128), ([1500, 20], [1500, 40], [1400, 33], 8, 1, 64), ([600], [1000], None, 8, 1, 72), ([520], [4000], None, 8, 1, 40),
    ([1400], [1400], None, 9, 3, 128), ([2048], [2048], None, 64, 16, 128), ([0, 1100], [300, 1100], None, 16, 2, 64)])
def test_few_key_heads_on_long_sequences(qn, kn, count, heads, kv_heads, dim):
    """Gradients of keys and values whose group is walked past in parts, by workgroups of 32 keys and of 128; more keys than the parts have room for."""
    first = 11
    q, k, v, dout = tensors(first + sum(qn) + 3, first + sum(kn) + 3, heads, kv_heads, dim, seed=12)
    check(q, k, v, dout, qn, kn, True, None, k_count=count, first=first, tail=3)


@pytest.mark.parametrize("n", [63, 64, 65, 256, 257, 400])
def test_numbers_of_sequences(n):
    """Lists that are ordered by work and lists that are too many for it."""
    lengths = [(7 * i) % 41 for i in range(n)]
    q, k, v, dout = tensors(sum(lengths), sum(lengths), 1, 1, 64, seed=n)
    check(q, k, v, dout, lengths, lengths, True, None)


def test_offsets_beyond_32_bits():
    """Keys, values and queries whose elements lie more than 2^31 elements into their tensors; a cache of which the last rows are used."""
    import torch
    from paper_2508_15706_amd import binding as sl
    heads, dim, tokens = 40, 128, 440_000                      # 2.25e9 elements, 4.5 GB
    k = torch.zeros(tokens, heads, dim, device="cuda", dtype=torch.bfloat16)
    q, v, dout = torch.zeros_like(k), torch.zeros_like(k), torch.zeros_like(k)
    lengths = [tokens - 300, 200, 100]
    s = starts(lengths)
    for t, seed in ((q, 1), (k, 2), (v, 3), (dout, 4)):
        t[-300:].normal_(0, 1, generator=torch.Generator(device="cuda").manual_seed(seed))
    few = starts([0, 200, 100], tokens - 300)                  # (the long sequence itself is left out of the attention)
    out, lse = torch.empty(tokens, heads, dim, device="cuda", dtype=torch.bfloat16), torch.empty(heads, tokens, device="cuda")
    sl.sl_attention(q, k, v, out, few, lse=lse)
    dq, dk, dv = (torch.empty_like(k) for _ in range(3))
    sl.sl_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, few, workspace=sl.alloc_attention_workspace(tokens, heads))
    one = torch.empty(3, heads, dim, device="cuda", dtype=torch.bfloat16)
    count = torch.tensor([1, 200, 100], dtype=torch.int32, device="cuda")
    sl.sl_attention_token(q[-3:], k, v, one, s, count, workspace=sl.alloc_attention_token_workspace(3, tokens, heads, heads, dim))
    for i, (a, n) in enumerate(((tokens - 300, 200), (tokens - 100, 100))):
        rows = slice(a, a + n)
        for h in (0, 17, 39):
            r = ref.attention(q[rows, h], k[rows, h], v[rows, h], True, dim ** -0.5, dout[rows, h])
            for name, t in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
                assert worst(t[rows, h], r[name], r[name + "_off"]) <= 1.0, (name, i, h)
            r = ref.attention(q[tokens - 2 + i: tokens - 1 + i, h] if i == 0 else q[tokens - 1:, h], k[rows, h], v[rows, h], False, dim ** -0.5)
            assert worst(one[i + 1: i + 2, h], r["out"], r["out_off"]) <= 1.0, ("token", i, h)
