"""Linear layers on 4-bit operands at the sizes that the other kernels of the products serve."""
import numpy as np
import pytest

from inner_reference import mx4_reference
from test_gpu_mx4 import host, matrix, product_bound

pytestmark = pytest.mark.gpu

# Products by the tile that serves them (1: 128 x 128, 2: 128 x 256): whole and ragged tiles, bands of fewer than eight tile rows, one row or
# column of tiles, contractions of one step of 128 to nine, also beside a step's end.
TILES = {1: [(1601, 1500, 385), (1500, 1603, 600), (2048, 1152, 256), (33_001, 65, 40), (30, 50_257, 257), (1153, 3000, 1100)],
         2: [(3500, 3700, 300), (3457, 3841, 520), (3584, 3584, 256), (517, 50_257, 64), (3600, 3500, 1025)]}
# Widths of the layers for few rows by the waves that share a tile, and (rows, length of the contraction)
FEW = {8: [2040], 4: [8203], 2: [16_405], 1: [32_777, 50_257]}
FEW_ROWS = [(1, 200), (3, 33), (16, 513), (5, 2048)]


def on_grid(m, k, seed):
    """(4-bit matrix, its values in 64 bits) on the device: quantisation and the way back are held to their definitions bit by bit in
    test_gpu_mx4."""
    import torch
    from paper_2508_15706_amd import binding as sl
    x = torch.empty(m, k, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(seed))
    q = sl.alloc_mx4(m, k)
    sl.sl_mx4_quantize(x, q)
    sl.sl_mx4_dequantize(q, x)
    return q, x.double()


def bound(a, b, k, kind):
    """product_bound of test_gpu_mx4, on the device."""
    e = k * 2.0 ** -23 * (a.abs() @ b.abs().T)
    return e + (2.0 ** -8 * (a @ b.T).abs() if kind == "bf16" else 0)


@pytest.mark.parametrize("kind", ["f32", "bf16", "added"])
@pytest.mark.parametrize("sizes", [s for t in TILES.values() for s in t])
def test_larger_tiles(sizes, kind):
    import torch
    from paper_2508_15706_amd import binding as sl
    m, n, k = sizes
    (qa, a), (qb, b) = on_grid(m, k, 1), on_grid(n, k, 2)
    typ = torch.bfloat16 if kind == "bf16" else torch.float32
    c = torch.full((m + 2, n + 3), 7.0, dtype=typ, device="cuda")
    inner = c[1:m + 1, 2:n + 2]
    want, limit = a @ b.T, bound(a, b, k, kind)
    if kind == "added":
        inner.normal_(generator=torch.Generator(device="cuda").manual_seed(3))
        before = inner.double()
        want = want + before
        limit = limit + 2.0 ** -23 * (want.abs() + before.abs())
    again = c.clone()
    ws = sl.alloc_mx4_workspace(m, n, k)
    sl.sl_mx4_product(qa, qb, inner, k, ws, accumulate=kind == "added")
    assert bool(((inner.double() - want).abs() <= limit).all())
    sl.sl_mx4_product(qa, qb, again[1:m + 1, 2:n + 2], k, ws, accumulate=kind == "added")
    assert torch.equal(c, again)
    inner.fill_(7.0)
    assert bool((c == 7.0).all())                             # nothing was written beside it


@pytest.mark.parametrize("sizes", [t[0] for t in TILES.values()])
def test_blocks_of_nan_stay_in_their_row_of_larger_tiles(sizes):
    import torch
    from paper_2508_15706_amd import binding as sl
    m, n, k = sizes
    x, w = matrix(m, k, "bf16", 1, spread=False), matrix(n, k, "bf16", 2, spread=False)
    rows, cols = [1, 700, m - 1], [7, 129, n - 1]
    x[rows, 5] = float("inf")
    w[cols, k - 1] = float("nan")
    want = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    want[rows] = True
    want[:, cols] = True
    qx, qw = sl.alloc_mx4(m, k), sl.alloc_mx4(n, k)
    sl.sl_mx4_quantize(x, qx)
    sl.sl_mx4_quantize(w, qw)
    for typ in (torch.float32, torch.bfloat16):
        c = torch.empty(m, n, dtype=typ, device="cuda")
        sl.sl_mx4_product(qx, qw, c, k, sl.alloc_mx4_workspace(m, n, k))
        assert torch.equal(torch.isnan(c), want) and not bool(torch.isinf(c).any())


def test_larger_tiles_in_a_graph():
    """Recorded once and replayed, with the eager calls between the replays."""
    import torch
    from paper_2508_15706_amd import binding as sl
    calls = []
    for (m, n, k), typ in ((TILES[1][0], torch.float32), (TILES[1][1], torch.bfloat16), (TILES[2][0], torch.float32), (TILES[2][1], torch.bfloat16)):
        (qa, _), (qb, _) = on_grid(m, k, 1), on_grid(n, k, 2)
        calls.append((qa, qb, k, typ == torch.float32, sl.alloc_mx4_workspace(m, n, k),
                      [torch.zeros(m, n, dtype=typ, device="cuda") for _ in range(2)]))

    def products(i):
        for qa, qb, k, add, ws, c in calls:
            sl.sl_mx4_product(qa, qb, c[i], k, ws, accumulate=add)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        products(1)
    for _ in range(3):
        products(0)
        graph.replay()
        torch.cuda.synchronize()
        for *_, c in calls:
            assert torch.equal(c[0], c[1]) and bool(c[0].any())


@pytest.mark.parametrize("x_kind, y_kind", [("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("n", [n for w in FEW.values() for n in w])
def test_few_rows_of_wide_layers(n, x_kind, y_kind):
    import torch
    from paper_2508_15706_amd import binding as sl
    typ = torch.bfloat16 if y_kind == "bf16" else torch.float32
    for m, k in FEW_ROWS:
        qw, w = on_grid(n, k, 2)
        x = matrix(m, k + 3, x_kind, 1, spread=False)[:, 1:k + 1]
        a = torch.from_numpy(mx4_reference(host(x))[2]).cuda()
        y = torch.full((m, n + 1), 7.0, dtype=typ, device="cuda")
        sl.sl_mx4_linear(x, qw, y[:, :n])
        assert bool(((y[:, :n].double() - a @ w.T).abs() <= bound(a, w, k, y_kind)).all())
        assert bool((y[:, n] == 7.0).all())


def test_transposed_matrix_beyond_32_bits_of_bytes():
    """Codes and scale bytes of rows whose offsets pass 32 bits, and of the last ones, through the way back to dense."""
    import torch
    from paper_2508_15706_amd import binding as sl
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs more device memory")
    n, k = 2_200_003, 4096
    w = torch.empty(n, k, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(5))
    qt = sl.alloc_mx4(k, n)
    sl.sl_mx4_quantize(w, None, qt)
    out = torch.empty(k, n, dtype=torch.bfloat16, device="cuda")
    sl.sl_mx4_dequantize(qt, out)
    rows = torch.tensor([0, 1023, 3700, 3967, 4063, 4064, 4095], device="cuda")
    assert (4095 // 32 * -(-n // 128)) * 2048 > 1 << 32
    for at, size in ((0, 64), (1_099_968, 96), (n - 35, 35)):            # (whole blocks of 32: n = 32 * 68,750 + 3)
        want = mx4_reference(w[at:at + size][:, rows].double().cpu().numpy().T)[2]
        assert np.array_equal(out[rows, at:at + size].double().cpu().numpy(), want)


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
