"""What the layers between the linear ones refuse, through the C ABI and through the binding: every check is made on the host before
anything is launched, so this runs without a GPU (the addresses are never looked at)."""
import ctypes as C

import pytest
import torch

INVALID = -1
P = [0x10000 * (i + 1) for i in range(16)]          # addresses on 16 bytes


def call(fn, given, **change):
    from paper_2508_15706_amd import binding
    a = dict(given)
    assert set(change) <= set(a), change
    a.update(change)
    return getattr(binding.lib(), fn)(*a.values())


NORM = dict(x=P[0], x_type=1, ldx=64, residual=P[1], ldr=64, h=P[2], h_type=0, ldh=64, weight=P[3], w_type=0, rows=4, cols=64, eps=1e-5,
            y=P[4], y_type=1, ldy=64, rstd=P[5], q=P[6], qt=P[7], stream=None)


@pytest.mark.parametrize("change", [
    dict(x=None), dict(weight=None), dict(h=None), dict(residual=None), dict(x_type=2), dict(h_type=-1), dict(w_type=5), dict(y_type=3),
    dict(ldx=63), dict(ldr=63), dict(ldh=63), dict(ldy=63), dict(ldx=2**41), dict(rows=-1), dict(cols=-1), dict(rows=2**21 + 1), dict(cols=2**20 + 1),
    dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=P[0] + 1), dict(h=P[2] + 2), dict(residual=P[1] + 2),
    dict(y=P[4] + 1), dict(weight=P[3] + 2), dict(rstd=P[5] + 2), dict(q=P[6] + 8), dict(qt=P[7] + 8), dict(y=P[0]), dict(h=P[0]), dict(y=P[2]),
    dict(y=P[1]), dict(rstd=P[4]), dict(q=P[7]), dict(q=P[4]), dict(h=P[1], ldh=65), dict(y=P[3]),
    dict(h=None, residual=None, y=None, rstd=None, q=None, qt=None)])
def test_norm(change):
    assert call("sl_rms_norm", NORM, **change) == INVALID


def test_nothing_to_do():
    assert call("sl_rms_norm", NORM, rows=0) == 0 and call("sl_rms_norm", NORM, cols=0) == 0
    assert call("sl_rms_norm_backward", BACK, cols=0) == 0 and call("sl_rms_norm_backward", BACK, rows=0, accumulate=1) == 0
    assert call("sl_rms_norm_backward", BACK, rows=0, dweight=None) == 0


BACK = dict(h=P[0], h_type=0, ldh=64, weight=P[1], w_type=0, rstd=P[2], dy=P[3], dy_type=1, lddy=64, dh=P[4], lddh=64, dx=P[5], dx_type=0, lddx=64,
            dweight=P[6], accumulate=0, rows=4, cols=64, workspace=P[7], stream=None)


@pytest.mark.parametrize("change", [
    dict(h=None), dict(weight=None), dict(rstd=None), dict(dy=None), dict(dx=None), dict(workspace=None), dict(h_type=2), dict(w_type=2),
    dict(dy_type=2), dict(dx_type=2), dict(ldh=63), dict(lddy=63), dict(lddh=63), dict(lddx=63), dict(rows=-1), dict(cols=2**20 + 1), dict(rows=2**21 + 1),
    dict(dx=P[0]), dict(dx=P[3]), dict(dx=P[1]), dict(dx=P[2]), dict(dx=P[4], lddx=65), dict(dweight=P[5]), dict(dweight=P[1]), dict(dweight=P[7]),
    dict(workspace=P[5]), dict(workspace=P[7] + 8), dict(h=P[0] + 2), dict(dy=P[3] + 1), dict(dx=P[5] + 2), dict(dh=P[4] + 2), dict(dweight=P[6] + 2), dict(rstd=P[2] + 1)])
def test_norm_backward(change):
    assert call("sl_rms_norm_backward", BACK, **change) == INVALID


def policy(**change):
    from paper_2508_15706_amd import binding
    a = dict(old_logp=P[8], advantage=P[9], ref_logp=P[10], clip_low=0.2, clip_high=0.2, kl=0.1)
    a.update(change)
    return C.pointer(binding.SlPolicy(*a.values()))


LOSS = dict(logits=P[0], type=1, ld=100, rows=4, vocab=100, targets=P[1], weights=P[2], policy=None, loss=P[3], logp=P[4], dlogits=P[5], ldd=100, workspace=P[6],
            stream=None)


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(targets=None), dict(workspace=None), dict(type=2), dict(ld=99), dict(ldd=99), dict(rows=-1), dict(rows=2**21 + 1), dict(vocab=0),
    dict(vocab=2**24 + 1), dict(logits=P[0] + 1), dict(targets=P[1] + 4), dict(weights=P[2] + 2), dict(loss=P[3] + 2), dict(logp=P[4] + 2), dict(dlogits=P[5] + 1),
    dict(workspace=P[6] + 8), dict(dlogits=P[0], ldd=101), dict(workspace=P[0]), dict(workspace=P[5]), dict(workspace=P[1]),
    dict(loss=None, logp=None, dlogits=None)])
def test_token_loss(change):
    assert call("sl_token_loss", LOSS, **change) == INVALID


@pytest.mark.parametrize("change", [
    dict(old_logp=None), dict(advantage=None), dict(ref_logp=None), dict(old_logp=P[8] + 2), dict(advantage=P[9] + 1), dict(ref_logp=P[10] + 3), dict(clip_low=-0.1),
    dict(clip_low=1.1), dict(clip_high=-0.1), dict(clip_high=float("inf")), dict(kl=-1.0), dict(kl=float("nan")), dict(clip_low=float("nan")), dict(kl=float("inf"))])
def test_policy(change):
    assert call("sl_token_loss", LOSS, policy=policy(**change)) == INVALID


def shape(**change):
    from paper_2508_15706_amd import binding
    a = dict(sequences=3, tokens_q=300, tokens_k=300, heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.125, q_start=P[0], k_start=P[1], k_count=P[2])
    a.update(change)
    return C.pointer(binding.SlAttentionShape(*a.values()))


def heads(i, token=256, head=64):
    from paper_2508_15706_amd import binding
    return C.pointer(binding.SlHeads(None if i is None else P[i] if isinstance(i, int) and i < 16 else i, token, head))


def attend():
    return dict(shape=shape(), q=heads(3), k=heads(4), v=heads(5), out=heads(6), lse=P[7], stream=None)


def attend_back():
    return dict(shape=shape(), q=heads(3), k=heads(4), v=heads(5), out=heads(6), lse=P[7], dout=heads(8), dq=heads(9), dk=heads(10), dv=heads(11),
                workspace=P[12], stream=None)


def attend_token():
    return dict(shape=shape(tokens_q=3, q_start=None), q=heads(3), k=heads(4), v=heads(5), out=heads(6), workspace=P[12], stream=None)


SHAPES = [dict(sequences=-1), dict(sequences=2**22 + 1), dict(tokens_q=-1), dict(tokens_q=2**30 + 1), dict(tokens_k=-1), dict(tokens_k=2**30 + 1), dict(heads=0),
          dict(heads=5), dict(kv_heads=0), dict(kv_heads=-2), dict(heads=2**16 + 2), dict(head_dim=0), dict(head_dim=12), dict(head_dim=136), dict(scale=0.0), dict(scale=-1.0),
          dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=1e-35), dict(k_start=None), dict(q_start=P[0] + 2), dict(k_start=P[1] + 1),
          dict(k_count=P[2] + 2), dict(heads=2**15, kv_heads=2**15, tokens_q=2**20)]
TENSORS = [None, (P[3] + 8, 256, 64), (None, 256, 64), (P[3], 260, 64), (P[3], 256, 68), (P[3], -256, 64), (P[3], 256, -64), (P[3], 2**24 + 8, 64)]
OVERLAPPING = [(P[3], 256, 56), (P[3], 56, 64), (P[3], 248, 64), (P[3], 0, 64), (P[3], 256, 0), (P[3], 64, 128)]


def tensor(t):
    return None if t is None else heads(t[0], t[1], t[2])


@pytest.mark.parametrize("fn,given", [("sl_attention", attend), ("sl_attention_backward", attend_back)])
def test_attention(fn, given):
    assert call(fn, given(), shape=None) == INVALID
    for change in SHAPES + [dict(q_start=None)]:
        assert call(fn, given(), shape=shape(**change)) == INVALID, change
    names = [n for n in given() if n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")]
    outputs = ["out"] if fn == "sl_attention" else ["dq", "dk", "dv"]
    for name in names:
        for t in TENSORS + (OVERLAPPING if name in outputs else []):
            if name in ("dk", "dv") and t in ((P[3], 64, 128), (P[3], 248, 64)):
                continue                                   # (two heads: these do not overlap)
            assert call(fn, given(), **{name: tensor(t)}) == INVALID, (name, t)
        for other in names:
            if name in outputs and other != name:
                assert call(fn, given(), **{name: given()[other]}) == INVALID, (name, other)
    for change in [dict(lse=P[7] + 2)] + ([dict(lse=P[6])] if fn == "sl_attention" else [dict(lse=None), dict(workspace=None), dict(workspace=P[12] + 8), dict(workspace=P[9]),
                                                                                       dict(workspace=P[7])]):
        assert call(fn, given(), **change) == INVALID, change


def test_attention_token():
    given = attend_token
    for change in SHAPES:
        change = dict(change)
        change.setdefault("tokens_q", change.get("sequences", 3))
        assert call("sl_attention_token", given(), shape=shape(**change)) == INVALID, change
    assert call("sl_attention_token", given(), shape=shape(tokens_q=4)) == INVALID
    for name in ("q", "k", "v", "out"):
        for t in TENSORS + (OVERLAPPING if name == "out" else []):
            assert call("sl_attention_token", given(), **{name: tensor(t)}) == INVALID, (name, t)
    for change in (dict(workspace=None), dict(workspace=P[12] + 8), dict(workspace=P[6]), dict(out=heads(3)), dict(out=heads(4)), dict(out=heads(5))):
        assert call("sl_attention_token", given(), **change) == INVALID, change


def test_attention_without_tokens():
    assert call("sl_attention", attend(), shape=shape(tokens_q=0)) == 0
    assert call("sl_attention", attend(), shape=shape(sequences=0)) == 0
    assert call("sl_attention_backward", attend_back(), shape=shape(tokens_q=0, tokens_k=0)) == 0
    assert call("sl_attention_backward", attend_back(), shape=shape(sequences=0)) == 0
    assert call("sl_attention_token", attend_token(), shape=shape(sequences=0, tokens_q=0)) == 0


def test_workspaces():
    from paper_2508_15706_amd import binding as sl
    assert sl.sl_rms_norm_workspace_bytes(0, 5) == 0 and sl.sl_rms_norm_workspace_bytes(5, 2**21) == 0
    assert sl.sl_token_loss_workspace_bytes(-1) == 0 and sl.sl_attention_workspace_bytes(0, 4) == 0
    assert sl.sl_attention_token_workspace_bytes(1, 100, 5, 2, 64) == 0 and sl.sl_attention_token_workspace_bytes(1, 100, 4, 2, 65) == 0
    # that of the largest call serves every smaller one
    for heads_, kv in ((16, 16), (20, 5), (1, 1), (64, 1), (200, 2)):
        last = [0] * 5
        for tokens in sorted({0, 1, 127, 128, 129, 1000, 2047, 2048, 4096, 10**5, 10**6, 2**24, 163840, 327680, 327679}):
            now = [sl.sl_attention_token_workspace_bytes(n, tokens, heads_, kv, 128) for n in (1, 2, 7, 64, 1000)]
            assert all(a <= b for a, b in zip(last, now)) and now == sorted(now)
            last = now
    for fn in (lambda r: sl.sl_rms_norm_workspace_bytes(r, 64), sl.sl_token_loss_workspace_bytes, lambda r: sl.sl_attention_workspace_bytes(r, 4)):
        sizes = [fn(r) for r in (1, 2, 511, 512, 513, 100000)]
        assert sizes == sorted(sizes)


# ---- the binding ----

def test_binding_shapes():
    from paper_2508_15706_amd import binding as sl
    x, w = torch.zeros(4, 64), torch.zeros(64)
    q = torch.zeros(10, 4, 64, dtype=torch.bfloat16)
    k = torch.zeros(10, 2, 64, dtype=torch.bfloat16)
    s = torch.tensor([0, 10], dtype=torch.int32)
    for bad in (lambda: sl.sl_rms_norm(x, w, None),                                      # not on a device
                lambda: sl.sl_attention(q, k, k, q, s), lambda: sl.sl_attention_token(q[:1], k, k, q[:1], s),
                lambda: sl.sl_token_loss(x, torch.zeros(4, dtype=torch.int64), None, w[:1])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ValueError, match="lse"):
        sl._same("lse", torch.zeros(3, 4), (4, 3), torch.float32)
    with pytest.raises(ValueError, match="k_start"):
        sl._starts("k_start", s.long())
    with pytest.raises(ValueError, match="k_count"):
        sl._starts("k_count", s, 1)


def test_binding_devices(monkeypatch):
    """A tensor of another device than the current one is refused: the library's calls are of the current device."""
    import types

    from paper_2508_15706_amd import binding as sl
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    there = types.SimpleNamespace(get_device=lambda: 1, device="cuda:1")
    here = types.SimpleNamespace(get_device=lambda: 0, device="cuda:0")
    sl._on_current_device(here, None, here)
    with pytest.raises(ValueError, match="current device"):
        sl._on_current_device(here, there)
