"""Attention over lists long enough for the order of work to matter, with NaN in all that a call does not use, and with starts that are none,
in workgroups of 128 rows as well."""
import math
import random

import pytest

from test_gpu_attention import check, starts, tensors

pytestmark = pytest.mark.gpu


def spoil(q, k, v, dout, q_lengths, room, count, first):
    """NaN in the tokens before the first sequence, behind the last one and behind a sequence's used keys."""
    import torch
    used = torch.zeros(k.shape[0], dtype=torch.bool, device="cuda")
    at = first
    for r, n in zip(room, count):
        used[at:at + n] = True
        at += r
    k[~used], v[~used] = math.nan, math.nan
    for t in (q, dout):
        t[:first], t[first + sum(q_lengths):] = math.nan, math.nan


def mixture(n, lengths, seed):
    """Every length of the list, and n in all, out of order; the longest last as well as somewhere."""
    rng = random.Random(seed)
    m = [lengths[i % len(lengths)] for i in range(n - 1)]
    rng.shuffle(m)
    return m + [max(lengths)]


# (65 to 256 sequences are ordered four to a lane, more are looked up by their starts; one head of 64 and lengths below 300 make workgroups of 32 rows, the others
# of 128)
@pytest.mark.parametrize("n,lengths,heads,kv_heads,dim", [
    (65, [0, 1, 31, 127, 129, 300], 1, 1, 64), (100, [0, 1, 5, 33, 65], 1, 1, 40), (65, [0, 1, 127, 129, 300, 700], 4, 2, 64), (200, [0, 1, 127, 129, 300], 2, 1, 128),
    (256, [0, 1, 127, 129, 257], 2, 1, 64), (257, [0, 1, 127, 129, 300, 700], 2, 1, 64), (300, [0, 1, 127, 128, 129, 385], 2, 2, 128)])
def test_lists_of_several_tiles_each(n, lengths, heads, kv_heads, dim):
    first, tail = 9, 5
    q_lengths = mixture(n, lengths, n)
    q, k, v, dout = tensors(first + sum(q_lengths) + tail, first + sum(q_lengths) + tail, heads, kv_heads, dim, seed=n)
    spoil(q, k, v, dout, q_lengths, q_lengths, q_lengths, first)
    check(q, k, v, dout, q_lengths, q_lengths, True, None, first=first, tail=tail)


@pytest.mark.parametrize("n", [65, 200, 257, 300])
@pytest.mark.parametrize("causal", [True, False])
def test_lists_with_other_lengths_on_the_key_side(n, causal):
    first, tail = 9, 5
    q_lengths, room = mixture(n, [0, 1, 127, 129, 300], n), mixture(n, [0, 1, 127, 129, 200, 300], n + 1)
    rng = random.Random(n)
    count = [rng.choice([r, r, r // 2, 0]) for r in room]
    q, k, v, dout = tensors(first + sum(q_lengths) + tail, first + sum(room) + tail, 2, 1, 64, seed=n)
    spoil(q, k, v, dout, q_lengths, room, count, first)
    check(q, k, v, dout, q_lengths, room, causal, None, k_count=count, first=first, tail=tail)


@pytest.mark.parametrize("dim", [40, 64, 104, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_nan_beside_what_is_used_in_workgroups_of_128_rows(dim, causal):
    qn, room, count = [3, 130, 200, 0, 17, 65, 1, 260], [200, 300, 70, 40, 0, 64, 193, 260], [129, 300, 1, 0, 0, 33, 128, 257]
    first, tail = 11, 13
    q, k, v, dout = tensors(first + sum(qn) + tail, first + sum(room) + tail, 48, 24, dim, seed=4)
    spoil(q, k, v, dout, qn, room, count, first)
    check(q, k, v, dout, qn, room, causal, None, k_count=count, first=first, tail=tail)


@pytest.mark.parametrize("qn,room,count,heads,kv_heads,dim", [
    ([700], [900], [650], 8, 1, 128), ([1500, 20], [1500, 90], [1400, 33], 8, 1, 64), ([2048], [2100], [2048], 64, 16, 128)])
def test_nan_beside_what_is_used_in_parts_of_a_group(qn, room, count, heads, kv_heads, dim):
    first, tail = 11, 13
    q, k, v, dout = tensors(first + sum(qn) + tail, first + sum(room) + tail, heads, kv_heads, dim, seed=5)
    spoil(q, k, v, dout, qn, room, count, first)
    check(q, k, v, dout, qn, room, True, None, k_count=count, first=first, tail=tail)


def test_nan_and_infinities_stay_in_their_sequence():
    import torch
    from paper_2508_15706_amd import binding as sl
    lengths, heads = [200, 150, 300], 100
    q, k, v, dout = tensors(sum(lengths), sum(lengths), heads, 50, 64, seed=6)
    qs, ws = starts(lengths), sl.alloc_attention_workspace(sum(lengths), heads)

    def run():
        out, lse = torch.empty_like(q), torch.empty(heads, q.shape[0], device="cuda")
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        sl.sl_attention(q, k, v, out, qs, lse=lse)
        sl.sl_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, qs, workspace=ws)
        return out, lse.transpose(0, 1), dq, dk, dv
    clean = run()
    q[210], k[220], v[230], dout[240] = math.nan, math.inf, math.nan, -math.inf
    keep = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
    keep[200:350] = False
    for got, want in zip(run(), clean):
        assert torch.equal(got[keep], want[keep])


# ---- starts that are none ----

def everything(q, k, v, dout, s, count):
    """All passes between rows that have to stay; lse as the forward pass leaves it."""
    import torch
    from paper_2508_15706_amd import binding as sl
    tokens, heads, dim = q.shape
    kv_heads = k.shape[1]
    room = torch.full((tokens + 2, heads, dim), 9.0, device="cuda", dtype=torch.bfloat16)
    back = torch.full((tokens + 2, heads, dim), 9.0, device="cuda", dtype=torch.bfloat16)
    keys = torch.full((2, tokens + 2, kv_heads, dim), 9.0, device="cuda", dtype=torch.bfloat16)
    lse = torch.zeros(heads, tokens, device="cuda")
    size = sl.sl_attention_group_workspace_bytes(tokens, heads, kv_heads, dim)
    ws = torch.zeros(size + 512, dtype=torch.uint8, device="cuda")
    ws[:256], ws[256 + size:] = 171, 171
    sl.sl_attention(q, k, v, room[1:-1], s, s, count, lse=lse)
    sl.sl_attention_backward(q, k, v, room[1:-1], lse, dout, back[1:-1], keys[0, 1:-1], keys[1, 1:-1], s, s, count, workspace=ws[256:256 + size])
    ends = [0, -1]
    assert bool((room[ends] == 9).all()) and bool((back[ends] == 9).all()) and bool((keys[:, ends] == 9).all())
    assert bool((ws[:256] == 171).all()) and bool((ws[256 + size:] == 171).all())


@pytest.mark.parametrize("heads,kv_heads", [(200, 200), (200, 100)])
def test_starts_outside_the_tokens_in_workgroups_of_128_rows(heads, kv_heads):
    import torch
    q, k, v, dout = tensors(300, 300, heads, kv_heads, 64, seed=10)
    count = torch.tensor([2**31 - 1, -5, 2**31 - 1], dtype=torch.int32, device="cuda")
    for bad in ([0, 120, 300, 100000], [-50, 120, 200, 300], [150, 20, 290, 10], [2**31 - 1] * 4, [-2**31] * 4, [0, 0, 300, 0]):
        for c in (None, count):
            everything(q, k, v, dout, torch.tensor(bad, dtype=torch.int32, device="cuda"), c)


@pytest.mark.parametrize("n,heads,kv_heads", [(100, 1, 1), (100, 6, 3), (300, 6, 3)])
def test_starts_outside_the_tokens_in_long_lists(n, heads, kv_heads):
    import torch
    q, k, v, dout = tensors(700, 700, heads, kv_heads, 64, seed=11)
    rng = random.Random(n)
    for edge in (700, 5000, 2**31 - 1):
        s = torch.tensor([rng.choice([0, rng.randint(-edge, edge), rng.randint(0, 700)]) for _ in range(n + 1)], dtype=torch.int32, device="cuda")
        count = torch.tensor([rng.randint(-3, edge) for _ in range(n)], dtype=torch.int32, device="cuda")
        for c in (None, count):
            everything(q, k, v, dout, s, c)
