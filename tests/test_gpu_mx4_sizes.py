"""Linear layers on 4-bit operands at the sizes that the other kernels of the products serve."""
import numpy as np
import pytest

from inner_reference import mx4_reference
from test_gpu_mx4 import host, matrix, product_bound

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 17, 64, 300, 512])
def test_a_layer_of_the_example_takes_any_number_of_rows(rows):
    """A contraction that is cut into parts for few rows and not for the most: the layer's own buffers serve both."""
    from paper_2508_15706_amd.inner_example import Mx4Linear
    m, n, k = 512, 1024, 8192
    layer = Mx4Linear(m, n, k)
    w, x = matrix(n, k, "bf16", 1, spread=False), matrix(rows, k, "bf16", 2, spread=False)
    layer.set_weight(w)
    a, b = mx4_reference(host(x))[2], mx4_reference(host(w))[2]
    assert (np.abs(host(layer.infer(x)) - a @ b.T) <= product_bound(a, b, k, "bf16")).all()


@pytest.mark.parametrize("rows", [1, 8])
def test_few_rows_need_no_workspace(rows):
    """A contraction that a product would cut into parts: the call for few rows is one launch and keeps nothing."""
    import torch
    from paper_2508_15706_amd import binding as sl
    n, k = 2048, 8192
    w, x = matrix(n, k, "bf16", 1, spread=False), matrix(rows, k, "bf16", 2, spread=False)
    q, y = sl.alloc_mx4(n, k), torch.empty(rows, n, device="cuda")
    sl.sl_mx4_quantize(w, q)
    sl.sl_mx4_linear(x, q, y)
    a, b = mx4_reference(host(x))[2], mx4_reference(host(w))[2]
    assert (np.abs(host(y) - a @ b.T) <= product_bound(a, b, k, "f32")).all()
    with pytest.raises(sl.SparseLoCoError):                    # more rows do
        sl.sl_mx4_linear(matrix(17, k, "bf16", 3, spread=False), q, torch.empty(17, n, device="cuda"))
    with pytest.raises(sl.SparseLoCoError):                    # and so does the product
        sl.sl_mx4_product(q, q, torch.empty(rows, n, device="cuda"), k)
