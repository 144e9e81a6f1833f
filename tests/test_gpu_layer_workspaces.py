"""Workspaces of exactly the size that a call names, between bytes that have to stay."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths,heads,kv_heads,dim", [([300, 5], 3, 3, 64), ([700], 8, 1, 40), ([1500, 20], 8, 1, 128), ([2048], 20, 5, 72), ([130] * 9, 16, 16, 128)])
def test_backward(lengths, heads, kv_heads, dim):
    import torch
    from paper_2508_15706_amd import binding as sl
    n = sum(lengths)
    g = torch.Generator(device="cuda").manual_seed(n)
    q, dout = (torch.randn(n, heads, dim, device="cuda", generator=g).bfloat16() for _ in range(2))
    k, v = (torch.randn(n, kv_heads, dim, device="cuda", generator=g).bfloat16() for _ in range(2))
    ends = [0]
    for length in lengths:
        ends.append(ends[-1] + length)
    s = torch.tensor(ends, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(heads, n, device="cuda")
    sl.sl_attention(q, k, v, out, s, lse=lse)
    size = sl.sl_attention_group_workspace_bytes(n, heads, kv_heads, dim)
    guarded = torch.full((size + 512,), 171, dtype=torch.uint8, device="cuda")
    results = []
    for ws in (guarded[256:256 + size], sl.alloc_attention_workspace(n, heads), sl.alloc_attention_workspace(n, heads, kv_heads=kv_heads, dim=dim)):
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        sl.sl_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, s, workspace=ws)
        results.append((dq, dk, dv))
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], r))
    assert bool((guarded[:256] == 171).all()) and bool((guarded[256 + size:] == 171).all())
    with pytest.raises(ValueError, match="workspace"):
        sl.sl_attention_backward(q, k, v, out, lse, dout, dq, dk, dv, s, workspace=guarded[256:255 + size])
