"""Calls that carry a workspace from launch to launch, on two streams at once and in graphs, against the same calls one after the other."""
import math

import pytest

pytestmark = pytest.mark.gpu


def attend(n, heads, kv_heads, dim, seed):
    """Attention both ways and its single-token form; -> (call, results)."""
    import torch
    from paper_2508_15706_amd import binding as sl
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, dout = (torch.randn(n, heads, dim, device="cuda", generator=g).bfloat16() for _ in range(2))
    k, v = (torch.randn(n, kv_heads, dim, device="cuda", generator=g).bfloat16() for _ in range(2))
    s = torch.tensor([0, n // 3, n], dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(heads, n, device="cuda")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    one, two = torch.empty_like(q[:2]), q[:2].clone()
    ws = sl.alloc_attention_workspace(n, heads, kv_heads=kv_heads, dim=dim)
    token_ws = sl.alloc_attention_token_workspace(2, n, heads, kv_heads, dim)

    def call(stream=None):
        sl.sl_attention(q, k, v, out, s, lse=lse, stream=stream)
        sl.sl_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, s, workspace=ws, stream=stream)
        sl.sl_attention_token(two, k, v, one, s, workspace=token_ws, stream=stream)
    return call, [out, lse, dq, dk, dv, one]


def norm(rows, cols, seed):
    """The norm into 4-bit matrices, and back."""
    import torch
    from paper_2508_15706_amd import binding as sl
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, r, dy = (torch.randn(rows, cols, device="cuda", generator=g) for _ in range(3))
    w, h, y, dx = torch.ones(cols, device="cuda"), torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    rstd, dw = torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
    q, qt = sl.alloc_mx4(rows, cols).zero_(), sl.alloc_mx4(cols, rows).zero_()
    ws = sl.alloc_rms_norm_workspace(rows, cols)

    def call(stream=None):
        sl.sl_rms_norm(x, w, y, residual=r, h=h, rstd=rstd, q=q, qt=qt, stream=stream)
        sl.sl_rms_norm_backward(h, w, rstd, dy, dx, dw=dw, workspace=ws, stream=stream)
    return call, [h, y, rstd, q, qt, dx, dw]


def loss(rows, vocab, seed):
    import torch
    from paper_2508_15706_amd import binding as sl
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(rows, vocab, device="cuda", generator=g).bfloat16()
    t = torch.randint(vocab, (rows,), device="cuda", generator=g)
    total, logp, dz, ws = torch.empty(1, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(z), sl.alloc_token_loss_workspace(rows)

    def call(stream=None):
        sl.sl_token_loss(z, t, None, total, logp=logp, dlogits=dz, workspace=ws, stream=stream)
    return call, [total, logp, dz]


def jobs():
    """Two of every kind, of different sizes (attention with parts of a group, in workgroups of 32 rows and of 128)."""
    return [[attend(1500, 8, 1, 64, 1), norm(700, 1000, 2), loss(300, 9000, 3)], [attend(2048, 64, 16, 128, 4), norm(3000, 200, 5), loss(90, 50257, 6)]]


def test_two_streams_at_once():
    import torch
    streams, both = [torch.cuda.Stream() for _ in range(2)], jobs()
    for side in both:
        for call, _ in side:
            call()
    torch.cuda.synchronize()
    want = [[t.clone() for t in results] for side in both for _, results in side]
    for _ in range(5):
        for side in both:
            for _, results in side:
                for t in results:
                    t.zero_()
        torch.cuda.synchronize()
        for parts in zip(*both):
            for (call, _), stream in zip(parts, streams):
                call(stream)
        torch.cuda.synchronize()
        got = [results for side in both for _, results in side]
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


def test_a_captured_training_step():
    """Forward and backward passes of the block in a graph each, replayed beside eager work on the same buffers."""
    import torch
    from paper_2508_15706_amd.block_example import BlockModel, text
    m = BlockModel(vocab=301, d=96, heads=4, kv_heads=2, dim=40, lengths=(70, 1, 130, 33), seed=3)
    tokens, targets = text(m, torch.Generator(device="cuda").manual_seed(4))
    weights = torch.full((m.tokens,), 1.0 / m.tokens, device="cuda")
    buffers = [m.loss, m.logp, m.logits, m.mixed, m.lse, m.dqkv, m.dh, m.grad]

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in buffers]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.forward(tokens, targets, weights)
        m.backward_to_embeddings()
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        m.forward(tokens, targets, weights)
    with torch.cuda.graph(graphs[1]):
        m.backward_to_embeddings()
    kept = targets.clone()
    for i in range(4):
        targets.copy_(kept.roll(5) if i % 2 else kept)
        for t in buffers[:-1]:
            t.fill_(math.nan)
        m.grad.zero_()
        for graph in graphs:
            graph.replay()
        m.embedding_gradient(tokens)
        got = results()
        m.grad.zero_()
        m.forward(tokens, targets, weights)
        m.backward(tokens)
        assert all(torch.equal(a, b) for a, b in zip(got, results())), i
