"""Norm, linear layers, attention and loss as a step runs them: each against its definition on what the one before it left, captured into graphs
beside eager work, on other streams, and in the example that trains with them."""
import math

import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


def model():
    import torch
    from paper_2508_15706_amd.block_example import BlockModel, text
    m = BlockModel(vocab=301, d=96, heads=4, kv_heads=2, dim=40, lengths=(70, 1, 130, 33), seed=3)
    tokens, targets = text(m, torch.Generator(device="cuda").manual_seed(4))
    weights = torch.full((m.tokens,), 1.0 / m.tokens, device="cuda")
    return m, tokens, targets, weights


def dense(q, rows, cols):
    import torch
    from paper_2508_15706_amd import binding as sl
    out = torch.empty(rows, cols, device="cuda")
    sl.sl_mx4_dequantize(q, out)
    return out


def linear(x, w, rows, n, k):
    """A product of 4-bit matrices: exact products, sums in fp32."""
    a, b = dense(x, rows, k).double(), dense(w, n, k).double()
    return a @ b.T, (k + 4) * ref.F32 * (a.abs() @ b.abs().T)


def near(got, want, off, half=HALF):
    got = got.double()
    assert bool(got.isfinite().all())
    assert float(((got - want).abs() / (off + half * (want.abs() + off) + 1e-30)).max()) <= 1.0


def test_every_step_of_the_block():
    import torch
    from paper_2508_15706_amd import binding as sl
    m, tokens, targets, weights = model()
    m.forward(tokens, targets, weights)
    dlogits = m.logits.clone()
    n, d, L = m.tokens, m.d, m.layers
    # forward
    h, s, y = ref.norm(m.h0, None, m.view(m.theta, "norm1"), 1e-5, torch.float32)
    near(m.rstd1, s, 1e-15 * s, ref.F32)
    q16 = [sl.alloc_mx4(n, d), sl.alloc_mx4(d, n)]
    y16 = torch.empty(n, d, device="cuda", dtype=torch.bfloat16)
    sl.sl_rms_norm(m.h0, m.view(m.theta, "norm1"), y16)
    near(y16, y, 3 * ref.F32 * y.abs())
    sl.sl_mx4_quantize(y16, *q16)
    assert torch.equal(dense(q16[0], n, d), dense(L["qkv"].x, n, d)) and torch.equal(dense(q16[1], d, n), dense(L["qkv"].xt, d, n))
    near(m.qkv.view(n, -1), *linear(L["qkv"].x, L["qkv"].w, n, m.qkv.shape[1] * m.dim, d))
    near(m.added, *linear(L["out"].x, L["out"].w, n, d, m.heads * m.dim))
    h1, s, _ = ref.norm(m.added, m.h0, m.view(m.theta, "norm2"), 1e-5, torch.float32)
    assert torch.equal(m.h1.double(), h1)
    logits = linear(L["head"].x, L["head"].w, n, m.vocab, d)[0].bfloat16()
    loss, logp, dz = ref.token_loss(logits, targets, weights)
    # (a logit next to a border of bf16 may be rounded the other way: a step of it, and what that moves)
    assert abs(float(m.loss) - float(loss)) < 2 * HALF * float(logits.float().abs().max()) and float((m.logp - logp).abs().max()) < 4 * HALF * float(logits.float().abs().max())
    assert float((dlogits.double() - dz).abs().max()) <= 2 * HALF * 2 * float(dz.abs().max())
    # backward
    m.backward(tokens)
    q, k, v = m.parts(m.qkv)
    dq, dk, dv = m.parts(m.dqkv)
    ends = m.starts.tolist()
    for a, b in zip(ends, ends[1:]):
        rows = slice(a, b)
        for g in range(m.kv_heads):
            sums = {x: 0.0 for x in ("dk", "dv", "dk_off", "dv_off")}
            for head in range(g * 2, g * 2 + 2):
                r = ref.attention(q[rows, head], k[rows, g], v[rows, g], True, m.dim ** -0.5, m.dmixed[rows, head])
                near(m.mixed[rows, head], r["out"], r["out_off"])
                near(dq[rows, head], r["dq"], r["dq_off"])
                for x in sums:
                    sums[x] = sums[x] + r[x]
            near(dk[rows, g], sums["dk"], sums["dk_off"])
            near(dv[rows, g], sums["dv"], sums["dv_off"])
    g = {x: m.view(m.grad, x) for x in m.part}
    ex, ox, ew, ow = ref.norm_backward(m.h1, m.view(m.theta, "norm2"), m.rstd2, m.dy2, None)
    near(g["norm2"], ew, ow, ref.F32)
    fx, fo, fw, fwo = ref.norm_backward(m.h0, m.view(m.theta, "norm1"), m.rstd1, m.dy1, ex)
    near(g["norm1"], fw, fwo, ref.F32)
    near(m.dh, fx, fo + ox + 2 * ref.F32 * ex.abs(), ref.F32)
    want = torch.zeros(m.vocab, d, device="cuda", dtype=torch.float64).index_add_(0, tokens, m.dh.double())
    near(g["embed"], want, n * ref.F32 * torch.zeros_like(want).index_add_(0, tokens, m.dh.double().abs()), ref.F32)
    for name, rows, cols in (("qkv", m.qkv.shape[1] * m.dim, d), ("out", d, m.heads * m.dim), ("head", m.vocab, d)):
        near(g[name], *linear(L[name].gt, L[name].xt, rows, cols, n), ref.F32)


def test_a_captured_step_is_the_eager_one():
    """Replayed with eager work on the same buffers, and synchronizations, between the replays; two graphs share every workspace."""
    import torch
    m, tokens, targets, weights = model()

    def step():
        m.forward(tokens, targets, weights)
        m.backward(tokens)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (m.loss, m.logp, m.logits, m.mixed, m.lse, m.dqkv, m.dh, m.grad)]
    step()
    want = results()
    other = targets.roll(5)
    targets_was = targets.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(results(), want))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            # (the embedding's own gradient is torch's work, and sorts: it stays outside)
            m.forward(tokens, targets, weights)
        graphs.append(graph)
    for i in range(4):
        targets.copy_(other if i % 2 else targets_was)
        for t in (m.loss, m.logp, m.mixed, m.lse, m.dqkv, m.dh):
            t.fill_(math.nan)
        m.grad.zero_()
        graphs[i % 2].replay()
        m.backward(tokens)
        got = results()
        step()
        again = results()
        assert all(torch.equal(a, b) for a, b in zip(got, again)), i
        if i % 2 == 0:
            assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_captured_backward_beside_an_eager_graph():
    """Every entry point captured alone and replayed, while torch's own autograd graph of the same leaves is alive."""
    import torch
    from paper_2508_15706_amd import binding as sl
    n, heads, dim = 150, 4, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, dout = (torch.randn(n, heads, dim, device="cuda", generator=g).bfloat16() for _ in range(4))
    leaf = q.clone().requires_grad_()
    alive = (leaf.float() ** 2).sum()
    s = torch.tensor([0, 64, n], dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(heads, n, device="cuda")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = sl.alloc_attention_workspace(n, heads)
    one, tws = torch.empty(2, heads, dim, device="cuda", dtype=torch.bfloat16), sl.alloc_attention_token_workspace(2, n, heads, heads, dim)
    x, w, dy = torch.randn(n, 200, device="cuda", generator=g), torch.ones(200, device="cuda"), torch.randn(n, 200, device="cuda", generator=g)
    y, rstd, dx, dw, rws = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty_like(x), torch.empty(200, device="cuda"), sl.alloc_rms_norm_workspace(n, 200)

    def run():
        sl.sl_attention(leaf.detach(), k, v, out, s, lse=lse)
        sl.sl_attention_backward(leaf.detach(), k, v, out, lse, dout, dq, dk, dv, s, workspace=ws)
        sl.sl_attention_token(leaf.detach()[:2], k, v, one, s, workspace=tws)
        sl.sl_rms_norm(x, w, y, rstd=rstd)
        sl.sl_rms_norm_backward(x, w, rstd, dy, dx, dw=dw, workspace=rws)
    run()
    torch.cuda.synchronize()
    results = [out, lse, dq, dk, dv, one, y, dx, dw]
    want = [t.clone() for t in results]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for t in results:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want))
    alive.backward()
    assert torch.equal(leaf.grad, 2 * leaf.detach())


def test_two_streams_at_once():
    """Calls with workspaces of their own on two streams do not meet."""
    import torch
    from paper_2508_15706_amd import binding as sl
    streams, jobs = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(2):
        g = torch.Generator(device="cuda").manual_seed(i)
        z = torch.randn(300, 9000, device="cuda", generator=g).bfloat16()
        t = torch.randint(9000, (300,), device="cuda", generator=g)
        jobs.append((z, t, torch.empty(1, device="cuda"), torch.empty_like(z), sl.alloc_token_loss_workspace(300)))
    for z, t, loss, dz, ws in jobs:
        sl.sl_token_loss(z, t, None, loss, dlogits=dz, workspace=ws)
    torch.cuda.synchronize()
    want = [(loss.clone(), dz.clone()) for _, _, loss, dz, _ in jobs]
    for _ in range(5):
        for stream, (z, t, loss, dz, ws) in zip(streams, jobs):
            sl.sl_token_loss(z, t, None, loss, dlogits=dz, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    for (a, b), (_, _, loss, dz, _) in zip(want, jobs):
        assert torch.equal(a, loss) and torch.equal(b, dz)


def test_example_runs():
    import torch
    from paper_2508_15706_amd import block_example
    losses, m = block_example.train(workers=2, rounds=2, inner_steps=2, lengths=(40, 9))
    assert len(losses) == 2 and all(math.isfinite(x) for x in losses) and bool(m.theta.isfinite().all())
    again, m2 = block_example.train(workers=2, rounds=2, inner_steps=2, lengths=(40, 9))
    assert torch.equal(m.theta, m2.theta) and losses == again
