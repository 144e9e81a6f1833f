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
