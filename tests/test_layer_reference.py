"""The definitions that the layers' kernels are held to, against differences of their own forward passes (64 bits, no GPU)."""
import pytest
import torch

from layer_reference import attention, norm, norm_backward, token_loss

STEP = 1e-5          # central differences: off by about STEP^2 of a third derivative, 1e-10, and 1e-16 / STEP = 1e-11 of rounding
TOL = 1e-7


def differences(f, x):
    g = torch.zeros_like(x)
    flat, out = x.view(-1), g.view(-1)
    for i in range(flat.numel()):
        was = float(flat[i])
        flat[i] = was + STEP
        up = float(f())
        flat[i] = was - STEP
        down = float(f())
        flat[i] = was
        out[i] = (up - down) / (2 * STEP)
    return g


def test_norm():
    g = torch.Generator().manual_seed(0)
    x, w, dy, dh = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((3, 7), (7,), (3, 7), (3, 7)))

    def value():
        h, _, y = norm(x, None, w, 1e-5, torch.float64)
        return (y * dy).sum() + (h * dh).sum()
    h, s, _ = norm(x, None, w, 1e-5, torch.float64)
    dx, _, dw, _ = norm_backward(h, w, s, dy, dh)
    assert (dx - differences(value, x)).abs().max() < TOL
    assert (dw - differences(value, w)).abs().max() < TOL


@pytest.mark.parametrize("n,m,causal", [(4, 4, True), (3, 6, True), (6, 3, True), (4, 5, False), (1, 1, True), (2, 0, False)])
def test_attention(n, m, causal):
    g = torch.Generator().manual_seed(1)
    q, k, v, dout = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((n, 4), (m, 4), (m, 4), (n, 4)))

    def value():
        return (attention(q, k, v, causal, 0.6)["out"] * dout).sum()
    r = attention(q, k, v, causal, 0.6, dout)
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        if x.numel():
            assert (r[name] - differences(value, x)).abs().max() < TOL
    if causal and n > m:
        assert bool((r["out"][: n - m] == 0).all()) and bool((r["lse"][: n - m] == -torch.inf).all())


@pytest.mark.parametrize("kind", ["nll", "clip", "kl"])
def test_token_loss(kind):
    g = torch.Generator().manual_seed(2)
    z = torch.randn(8, 5, generator=g, dtype=torch.float64)
    targets = torch.tensor([0, 4, -1, 2, 5, 1, 3, 0])
    weights = torch.tensor([0.5, 1.0, 1.0, 0.0, 1.0, 2.0, 0.25, 1.0])
    policy = None
    if kind != "nll":
        now = token_loss(z, targets, weights)[1]
        old = now + torch.tensor([0.0, 0.5, 0.0, 0.0, 0.0, -0.5, 0.05, -0.4])
        a = torch.tensor([1.0, -1.0, 1.0, 1.0, 1.0, 1.0, -2.0, -0.5])
        policy = (old, a, 0.2, 0.28, now + 0.3 if kind == "kl" else None, 0.1 if kind == "kl" else 0.0)
    loss, logp, dz = token_loss(z, targets, weights, policy)
    assert bool((logp[[2, 4]] == 0).all()) and bool((dz[[2, 3, 4]] == 0).all())
    assert (dz - differences(lambda: token_loss(z, targets, weights, policy)[0], z)).abs().max() < TOL
    assert (dz.sum(1).abs() < 1e-12).all()
