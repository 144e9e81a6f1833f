"""The token loss - negative log-likelihood and policy - against its definition in 64 bits."""
import math

import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu


def inputs(rows, vocab, kind, seed=0, pad=0, std=3.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[kind]
    z = torch.empty(rows, vocab + pad, device="cuda").normal_(0, std, generator=g).to(t)[:, :vocab]
    targets = torch.randint(vocab, (rows,), device="cuda", generator=g)
    weights = torch.rand(rows, device="cuda", generator=g) + 0.1
    return z, targets, weights


def check(z, targets, weights, policy, loss, logp, dz):
    """Exponentials (z - top) log2(e) are off by a step of an exponent of size `reach`, their sum by its additions; the gradient has the
    products with the share and, at the target, one addition on top, then its own rounding."""
    import torch
    vocab = z.shape[1]
    el, ep, ez = ref.token_loss(z, targets, weights, policy)
    reach = float((z.double().amax(1) - z.double().clamp(min=-1e4).amin(1)).max()) * 1.5 + 4
    exp_rel = 3 * ref.F32 * (reach + 2)
    sum_rel = exp_rel + ref.F32 * (vocab ** 0.5 + 64)
    assert float((logp.double() - ep).abs().max()) <= sum_rel + ref.F32 * float(ep.abs().max())
    slope = (ez.abs().sum(1, keepdim=True))                  # >= |w l'| (1 - p_t), at most twice |w l'|
    p = (z.double() - torch.logsumexp(z.double(), 1, keepdim=True)).exp()
    w = torch.ones_like(ep) if weights is None else weights.double()
    step = torch.ones_like(ep)
    if policy is not None:
        old, a, low, high, r, kl = policy
        ratio = (ep - old.double()).exp()
        step = a.double().abs() * ratio + (kl * ((r.double() - ep).exp() + 1) if kl else 0.0)
    size = (w * step)[:, None]
    ok = ((targets >= 0) & (targets < vocab) & (w != 0))[:, None]
    hot = torch.zeros_like(p).scatter_(1, targets.clamp(0, vocab - 1)[:, None], 1.0)
    off = torch.where(ok, size * ((exp_rel + 4 * sum_rel + 8 * ref.F32) * p + hot * (4 * sum_rel + 8 * ref.F32)), torch.zeros_like(p))
    bound = off + ref.HALF[dz.dtype] * (ez.abs() + off) + 1e-37
    worst = ((dz.double() - ez).abs() / bound).max()
    assert float(worst) <= 1.0, float(worst)
    each = (w * step * (1 + ep.abs())).sum()
    assert abs(float(loss) - float(el)) <= 4 * sum_rel * float(each) + 2 * ref.F32 * abs(float(el))
    assert slope.shape == (z.shape[0], 1)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (5, 7), (9, 64), (9, 511), (7, 513), (4, 2047), (3, 2049), (4, 8192), (3, 8193), (3, 16385), (2, 32000), (3, 32769),
                                        (2, 50257), (2, 53248), (2, 53249), (2, 57345), (2, 65536), (2, 65537), (1, 200003)])
@pytest.mark.parametrize("policy", [None, "clip", "kl"])
def test_against_the_definition(rows, vocab, kind, policy):
    import torch
    from paper_2508_15706_amd import binding as sl
    z, targets, weights = inputs(rows, vocab, kind, seed=rows, pad=3)
    if rows > 3:
        targets[1], targets[2], weights[3] = -100, vocab, 0.0
    given = pol = None
    if policy:
        now = ref.token_loss(z, targets, weights)[1].float()
        g = torch.Generator(device="cuda").manual_seed(5)
        old = now + 0.4 * torch.randn(rows, device="cuda", generator=g)
        a = torch.randn(rows, device="cuda", generator=g)
        r = now + 0.5 * torch.randn(rows, device="cuda", generator=g) if policy == "kl" else None
        given = (old, a, 0.2, 0.28, r, 0.1 if policy == "kl" else 0.0)
        pol = sl.Policy(old, a, 0.2, 0.28, r, given[5])
    loss, logp = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda")
    dz = torch.full((rows, vocab + 5), 7.0, device="cuda", dtype=z.dtype)
    ws = sl.alloc_token_loss_workspace(rows)
    sl.sl_token_loss(z, targets, weights, loss, logp=logp, dlogits=dz[:, :vocab], policy=pol, workspace=ws)
    check(z, targets, weights, given, loss, logp, dz[:, :vocab])
    assert bool((dz[:, vocab:] == 7.0).all())
    # log probabilities alone, and the gradient in place: the same bits
    alone = torch.empty_like(logp)
    sl.sl_token_loss(z, targets, None, None, logp=alone)
    assert torch.equal(alone, logp)
    l2 = torch.empty(1, device="cuda")
    sl.sl_token_loss(z, targets, weights, l2, dlogits=z, policy=pol, workspace=ws)
    assert torch.equal(z, dz[:, :vocab]) and torch.equal(l2, loss)


@pytest.mark.parametrize("vocab", [100, 5000, 20000, 70000])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_masked_logits_and_tokens_that_do_not_count(vocab, kind):
    """Logits of -infinity have no probability; a token that does not count may hold anything."""
    import torch
    from paper_2508_15706_amd import binding as sl
    z, targets, weights = inputs(6, vocab, kind)
    z[:, ::3] = -math.inf
    z[0, : vocab - 2] = -math.inf
    targets[:] = vocab - 1 - (vocab - 1) % 3 + 1 if (vocab - 1) % 3 else vocab - 2
    targets[1], weights[2] = -1, 0.0
    z[1, 0], z[2, 1] = math.nan, math.inf
    old, a = torch.zeros(6, device="cuda"), torch.ones(6, device="cuda")
    old[1], a[2] = math.nan, math.inf
    for policy in (None, sl.Policy(old, a, 0.2, 0.2)):
        loss, logp, dz = torch.empty(1, device="cuda"), torch.empty(6, device="cuda"), torch.full_like(z, 7.0)
        sl.sl_token_loss(z, targets, weights, loss, logp=logp, dlogits=dz, policy=policy, workspace=sl.alloc_token_loss_workspace(6))
        assert bool(dz.isfinite().all()) and bool(loss.isfinite().all())
        assert bool((dz[1:3] == 0).all()) and float(logp[1]) == 0.0
        assert bool((dz[3:, ::3] == 0).all())
        if policy is None:
            keep = [0, 3, 4, 5]
            want = ref.token_loss(z[keep], targets[keep], weights[keep])[0]
            assert abs(float(loss) - float(want)) < 1e-4 * abs(float(want))


def test_borders_of_the_range():
    """Ratios on both sides of the clipped range for either sign, an advantage of zero, an infinite ratio."""
    import torch
    from paper_2508_15706_amd import binding as sl
    rows, vocab = 8, 50
    z, targets, weights = inputs(rows, vocab, "f32")
    now = ref.token_loss(z, targets, weights)[1].float()
    shift = torch.tensor([0.5, 0.5, -0.5, -0.5, 0.1, -0.1, 2000.0, 2000.0], device="cuda")
    a = torch.tensor([1.0, -1.0, 1.0, -1.0, 1.0, -1.0, 0.0, 1.0], device="cuda")
    loss, dz = torch.empty(1, device="cuda"), torch.empty_like(z)
    sl.sl_token_loss(z, targets, weights, loss, dlogits=dz, policy=sl.Policy(now - shift, a, 0.2, 0.2), workspace=sl.alloc_token_loss_workspace(rows))
    zero = (dz == 0).all(1).tolist()
    assert zero == [True, False, False, True, False, False, True, True]
    ratio = shift.double().clamp(max=700).exp()
    each = torch.minimum(ratio * a, ratio.clamp(0.8, 1.2) * a)
    each[6] = 0.0
    want = -(weights.double() * each).sum()
    assert abs(float(loss) - float(want)) < 1e-5 * float((weights.double() * each.abs()).sum())


def test_offsets_beyond_32_bits():
    import torch
    from paper_2508_15706_amd import binding as sl
    rows, vocab = 45_000, 50_257                               # 2.26e9 elements
    z = torch.zeros(rows, vocab, device="cuda", dtype=torch.bfloat16)
    z[-3:], targets, weights = inputs(3, vocab, "bf16")[0], torch.full((rows,), -1, device="cuda"), torch.ones(rows, device="cuda")
    targets[-3:] = torch.tensor([0, vocab - 1, 777], device="cuda")
    loss, logp = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda")
    tail, last = z[-3:].clone(), targets[-3:]
    sl.sl_token_loss(z, targets, weights, loss, logp=logp, dlogits=z, workspace=sl.alloc_token_loss_workspace(rows))
    check(tail, last, weights[-3:], None, loss, logp[-3:], z[-3:])
    assert bool((z[0] == 0).all()) and bool((logp[:-3] == 0).all())
