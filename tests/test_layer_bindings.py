"""What the binding of the layers between the linear ones compares before it hands addresses on; without a GPU."""
import pytest
import torch


def test_keys_as_wide_as_queries():
    """The kernels take a row's width from the queries: keys and values of another one would be read past their end."""
    from paper_2508_15706_amd import binding as sl
    s = torch.tensor([0, 10], dtype=torch.int32)
    q, lse = torch.zeros(10, 4, 64, dtype=torch.bfloat16), torch.zeros(4, 10)
    for dim in (8, 56, 72, 128):
        k = torch.zeros(10, 2, dim, dtype=torch.bfloat16)
        for call in (lambda: sl.sl_attention(q, k, k.clone(), q.clone(), s),
                     lambda: sl.sl_attention(q, k, k.clone(), q.clone(), s, s, s[1:]),
                     lambda: sl.sl_attention_backward(q, k, k.clone(), q.clone(), lse, q.clone(), q.clone(), k.clone(), k.clone(), s),
                     lambda: sl.sl_attention_token(q[:1], k, k.clone(), q[:1].clone(), s)):
            with pytest.raises(ValueError, match="k: expected"):
                call()


def test_workspaces_of_the_backward_pass():
    """Where every head has a key head of its own there are statistics alone; narrow heads have narrow parts; any heads' room is enough for all."""
    from paper_2508_15706_amd import binding as sl
    size = sl.sl_attention_group_workspace_bytes
    assert size(16384, 16, 16, 128) == 8 * 16384 * 16 + 16
    assert size(8192, 20, 5, 64) - (8 * 8192 * 20 + 16) == 2 * 64 * 4 * 8192 * 20
    for tokens, heads in ((1, 1), (33, 5), (8192, 20), (100000, 64)):
        every = sl.sl_attention_workspace_bytes(tokens, heads)
        for kv_heads in (1, heads):
            for dim in (8, 40, 128):
                assert 0 < size(tokens, heads, kv_heads, dim) <= every
    assert [size(*bad) for bad in ((0, 4, 2, 64), (2**30 + 1, 4, 2, 64), (9, 4, 3, 64), (9, 4, 0, 64), (9, 0, 1, 64), (9, 4, 2, 60), (9, 4, 2, 136), (9, 2**17, 1, 8))] == [0] * 8
