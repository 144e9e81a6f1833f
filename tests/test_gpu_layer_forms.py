"""Forms of operands that a caller may have: weights in bf16, rows and heads that share memory, logits inside a wider matrix."""
import pytest

import layer_reference as ref
from test_gpu_attention import starts, worst

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(1, 1), (33, 200), (131, 513), (9, 8192), (6, 9000), (5, 20001)])
def test_norm_backward_with_weights_in_bf16(shape):
    import torch
    from paper_2508_15706_amd import binding as sl
    rows, cols = shape
    g = torch.Generator(device="cuda").manual_seed(cols)
    h, dy = torch.randn(rows, cols, device="cuda", generator=g), torch.randn(rows, cols, device="cuda", generator=g).bfloat16()
    w = (1.0 + 0.3 * torch.randn(cols, device="cuda", generator=g)).bfloat16()
    s = (1.0 / torch.sqrt(h.double().square().mean(1) + 1e-5)).float()
    dx, dw = torch.empty_like(h), torch.empty(cols, device="cuda")
    sl.sl_rms_norm_backward(h, w, s, dy, dx, dw=dw, workspace=sl.alloc_rms_norm_workspace(rows, cols))
    ex, ox, ew, ow = ref.norm_backward(h, w, s, dy, None)
    for got, want, off in ((dx, ex, ox), (dw, ew, ow)):
        assert float(((got.double() - want).abs() / (off + ref.F32 * (want.abs() + off) + 1e-300)).max()) <= 1.0


@pytest.mark.parametrize("heads,n", [(4, 150), (200, 150)])
def test_attention_on_operands_whose_rows_share_memory(heads, n):
    """One key head expanded to many, one query expanded to all tokens, one gradient for all heads."""
    import torch
    from paper_2508_15706_amd import binding as sl
    dim = 64
    g = torch.Generator(device="cuda").manual_seed(n + heads)

    def normal(*s):
        return torch.randn(*s, device="cuda", generator=g).bfloat16()
    q, k, v = normal(1, heads, dim).expand(n, heads, dim), normal(n, 1, dim).expand(n, heads, dim), normal(n, 1, dim).expand(n, heads, dim)
    dout, s = normal(n, 1, dim).expand(n, heads, dim), starts([100, n - 100])
    out, lse = torch.empty(n, heads, dim, device="cuda", dtype=torch.bfloat16), torch.empty(heads, n, device="cuda")
    dq, dk, dv = (torch.empty_like(out) for _ in range(3))
    sl.sl_attention(q, k, v, out, s, lse=lse)
    sl.sl_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, s, workspace=sl.alloc_attention_workspace(n, heads, kv_heads=heads, dim=dim))
    one = torch.empty(2, heads, dim, device="cuda", dtype=torch.bfloat16)
    sl.sl_attention_token(q[:2], k, v, one, s, workspace=sl.alloc_attention_token_workspace(2, n, heads, heads, dim))
    for i, (a, b) in enumerate(((0, 100), (100, n))):
        for h in {0, 1, heads - 1}:
            r = ref.attention(q[a:b, h], k[a:b, h], v[a:b, h], True, dim ** -0.5, dout[a:b, h])
            for name, t in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
                assert worst(t[a:b, h], r[name], r[name + "_off"]) <= 1.0, (name, i, h)
            r = ref.attention(q[i:i + 1, h], k[a:b, h], v[a:b, h], False, dim ** -0.5)
            assert worst(one[i:i + 1, h], r["out"], r["out_off"]) <= 1.0, ("token", i, h)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [7, 513, 8191, 50257, 65537])
def test_loss_of_logits_inside_a_wider_matrix(kind, vocab):
    """Rows that begin at any element, in place: what lies beside them stays, and the results are those of a matrix of their own."""
    import torch
    from paper_2508_15706_amd import binding as sl
    rows, t = 5, {"f32": torch.float32, "bf16": torch.bfloat16}[kind]
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = (2.0 * torch.randn(rows, vocab, device="cuda", generator=g)).to(t)
    targets = torch.randint(vocab, (rows,), device="cuda", generator=g)
    targets[1], targets[3] = 0, vocab - 1
    ws = sl.alloc_token_loss_workspace(rows)
    want, dz = torch.empty(1, device="cuda"), torch.empty_like(z)
    sl.sl_token_loss(z, targets, None, want, dlogits=dz, workspace=ws)
    el, _, ez = ref.token_loss(z, targets, None)
    assert abs(float(want) - float(el)) <= 1e-5 * float(el)
    for left in (1, 3, 8, 13):
        wide = torch.full((rows, left + vocab + 2), 7.0, device="cuda", dtype=t)
        inside = wide[:, left:left + vocab]
        inside.copy_(z)
        loss = torch.empty(1, device="cuda")
        sl.sl_token_loss(inside, targets, None, loss, dlogits=inside, workspace=ws)
        assert bool((wide[:, :left] == 7).all()) and bool((wide[:, left + vocab:] == 7).all())
        # (an exponential is off by three roundings of an exponent up to 24, 5e-6 of it; the sum is made in another order; the gradient has its own rounding)
        assert abs(float(loss) - float(want)) <= 1e-5 * abs(float(want))
        assert float((inside.double() - ez).abs().max()) <= (ref.HALF[t] + 1e-5) * float(ez.abs().max())
