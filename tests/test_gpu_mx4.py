"""Microscaled 4-bit matrices: quantisation, products and linear layers against their definitions in 64 bits."""
import numpy as np
import pytest

from inner_reference import mx4_layout, mx4_reference

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 32), (1, 2048), (3, 33), (16, 128), (17, 129), (63, 31), (64, 64), (65, 127), (100, 200), (130, 530),
          (256, 257), (1000, 96)]


def matrix(rows, cols, kind, seed=0, spread=True):
    """A device matrix of the kind; rows of very different sizes, so that blocks have scales of their own."""
    import torch
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 1, (rows, cols))
    if spread:
        x *= 2.0 ** rng.integers(-20, 20, (rows, 1))
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16 if kind == "bf16" else torch.float32).cuda()


def host(t):
    return t.double().cpu().numpy()


def check_layout(q, rows, cols, codes, scales):
    got_codes, got_scales = mx4_layout(q.cpu().numpy(), rows, cols)
    want = np.zeros_like(got_codes)
    want[:rows, :codes.shape[1]] = codes
    # (the padding of a row's last block is +0)
    assert np.array_equal(got_codes, want)
    want = np.zeros_like(got_scales)
    want[:rows, :scales.shape[1]] = scales
    assert np.array_equal(got_scales, want)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("way", ["rows", "columns", "both"])
def test_quantize(shape, kind, way):
    import torch
    from paper_2508_15706_amd import binding as sl
    rows, cols = shape
    x = matrix(rows, cols, kind)
    q = torch.full((sl.sl_mx4_bytes(rows, cols),), 171, dtype=torch.uint8, device="cuda")
    qt = torch.full((sl.sl_mx4_bytes(cols, rows),), 171, dtype=torch.uint8, device="cuda")
    sl.sl_mx4_quantize(x, q if way != "columns" else None, qt if way != "rows" else None)
    if way != "columns":
        check_layout(q, rows, cols, *mx4_reference(host(x))[:2])
    if way != "rows":
        check_layout(qt, cols, rows, *mx4_reference(host(x).T)[:2])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_quantize_edges_of_the_format(kind):
    """Ties, the largest values of a binade, subnormals, zeros, the ends of fp32's range, infinities and NaN."""
    import torch
    from paper_2508_15706_amd import binding as sl
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    rows = []
    for e in (-126, -30, 0, 30, 120):
        rows.append([6.0 * 2.0 ** e] + [t * 2.0 ** e for t in ties] + [-t * 2.0 ** e for t in ties])
        rows.append([6.5 * 2.0 ** e, 1.0 * 2.0 ** e])                    # just above 6: the next scale
        rows.append([-4.0 * 2.0 ** e, 0.125 * 2.0 ** e, 0.126 * 2.0 ** e])
    rows += [[], [2.0 ** -126, 2.0 ** -127], [2.0 ** -133], [1.0, -0.0], [3.3e38, -3.0e38]]
    rows += [[np.inf, 1.0], [1.0, -np.inf], [np.nan, 0.0]]
    x = np.zeros((len(rows), 64))
    for i, r in enumerate(rows):
        x[i, :len(r)] = r
        x[i, 32:32 + len(r)] = r[::-1]
    x[-1, 32:] = 1.0                                                      # the other block of the NaN row is sound
    t = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16 if kind == "bf16" else torch.float32).cuda()
    codes, scales, values = mx4_reference(host(t))
    q, qt = sl.alloc_mx4(*t.shape), sl.alloc_mx4(*t.shape)
    sl.sl_mx4_quantize(t, q)
    check_layout(q, *t.shape, codes, scales)
    sl.sl_mx4_quantize(t.t().contiguous(), None, qt)
    check_layout(qt, *t.shape, codes, scales)
    for out_kind in (torch.float32, torch.bfloat16):
        out = torch.empty(t.shape, dtype=out_kind, device="cuda")
        sl.sl_mx4_dequantize(q, out)
        want = torch.from_numpy(values).to(torch.float32).to(out_kind)
        assert torch.equal(torch.nan_to_num(out.cpu().float(), nan=777.0), torch.nan_to_num(want.float(), nan=777.0))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(5, 70), (33, 257), (64, 256)])
def test_strides_and_offsets(shape, kind):
    """A window of a larger matrix, at an address aligned to its element only, in and out."""
    import torch
    from paper_2508_15706_amd import binding as sl
    rows, cols = shape
    big = matrix(rows + 2, cols + 5, kind, 3)
    x = big[1:rows + 1, 3:cols + 3]
    q, qt = sl.alloc_mx4(rows, cols), sl.alloc_mx4(cols, rows)
    sl.sl_mx4_quantize(x, q, qt)
    codes, scales, values = mx4_reference(host(x))
    check_layout(q, rows, cols, codes, scales)
    check_layout(qt, cols, rows, *mx4_reference(host(x).T)[:2])
    out = torch.full_like(big, 9.0)
    sl.sl_mx4_dequantize(q, out[1:rows + 1, 3:cols + 3])
    got = host(out)
    assert np.array_equal(got[1:rows + 1, 3:cols + 3], values)
    got[1:rows + 1, 3:cols + 3] = 9.0
    assert (got == 9.0).all()


def quantized(x):
    from paper_2508_15706_amd import binding as sl
    q = sl.alloc_mx4(*x.shape)
    sl.sl_mx4_quantize(x, q)
    return q, mx4_reference(host(x))[2]


def product_bound(a, b, k, kind):
    """Exact products, k fp32 additions of one rounding each (of which the matrix unit may cut off instead of rounding: 2^-23 of
    the sum of magnitudes), then one rounding to bf16."""
    bound = k * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)
    return bound + (2.0 ** -8 * np.abs(a @ b.T) if kind == "bf16" else 0)


PRODUCTS = [(1, 1, 1), (1, 1, 32), (1, 64, 128), (1, 530, 200), (2, 16, 2048), (5, 1030, 96), (16, 257, 640), (17, 48, 129), (31, 33, 35), (33, 128, 1000),
            (64, 64, 256), (100, 300, 513), (128, 128, 128), (129, 127, 384), (200, 530, 1000), (257, 259, 1024), (512, 768, 320), (300, 50, 5000),
            (1000, 530, 200), (40, 2100, 512), (700, 1100, 2048)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", PRODUCTS)
def test_product(sizes, kind):
    import torch
    from paper_2508_15706_amd import binding as sl
    m, n, k = sizes
    qa, a = quantized(matrix(m, k, "bf16", 1, spread=False))
    qb, b = quantized(matrix(n, k, "f32", 2, spread=False))
    c = torch.full((m + 2, n + 3), 7.0, dtype=torch.bfloat16 if kind == "bf16" else torch.float32, device="cuda")
    ws = sl.alloc_mx4_workspace(m, n, k)
    sl.sl_mx4_product(qa, qb, c[1:m + 1, 2:n + 2], k, ws)
    got = host(c)
    assert (np.abs(got[1:m + 1, 2:n + 2] - a @ b.T) <= product_bound(a, b, k, kind)).all()
    got[1:m + 1, 2:n + 2] = 7.0
    assert (got == 7.0).all()
    again = torch.full_like(c, 7.0)
    sl.sl_mx4_product(qa, qb, again[1:m + 1, 2:n + 2], k, ws)
    assert torch.equal(c, again)


@pytest.mark.parametrize("sizes", [(1, 64, 256), (100, 300, 513), (257, 259, 1024), (300, 50, 5000), (128, 256, 4096)])
def test_product_adds_to_what_is_there(sizes):
    import torch
    from paper_2508_15706_amd import binding as sl
    m, n, k = sizes
    qa, a = quantized(matrix(m, k, "bf16", 1, spread=False))
    qb, b = quantized(matrix(n, k, "bf16", 2, spread=False))
    c = matrix(m, n, "f32", 5, spread=False)
    before = host(c)
    sl.sl_mx4_product(qa, qb, c, k, sl.alloc_mx4_workspace(m, n, k), accumulate=True)
    want = before + a @ b.T
    assert (np.abs(host(c) - want) <= product_bound(a, b, k, "f32") + 2.0 ** -23 * (np.abs(want) + np.abs(before))).all()


def test_product_of_nothing():
    import torch
    from paper_2508_15706_amd import binding as sl
    q = torch.zeros(16, dtype=torch.uint8, device="cuda")
    c = torch.full((3, 5), 7.0, device="cuda")
    sl.sl_mx4_product(q, q, c, 0, accumulate=True)
    assert bool((c == 7.0).all())
    sl.sl_mx4_product(q, q, c, 0)
    assert bool((c == 0.0).all())
    sl.sl_mx4_product(q, q, torch.empty(0, 5, device="cuda"), 64)
    sl.sl_mx4_product(q, q, torch.empty(5, 0, device="cuda"), 64)


def test_an_empty_batch():
    """No tokens: nothing to quantise, no rows of y and dx, and a dW of zeros."""
    import torch
    from paper_2508_15706_amd import binding as sl
    n, k = 70, 100
    x, dy = torch.empty(0, k, device="cuda", dtype=torch.bfloat16), torch.empty(0, n, device="cuda", dtype=torch.bfloat16)
    w, _ = quantized(matrix(n, k, "bf16", 1))
    q = [sl.alloc_mx4(*s) for s in ((0, k), (k, 0), (0, n), (n, 0))]
    sl.sl_mx4_quantize(x, q[0], q[1])
    sl.sl_mx4_quantize(dy, q[2], q[3])
    sl.sl_mx4_dequantize(q[0], torch.empty(0, k, device="cuda"))
    y = torch.empty(0, n, device="cuda", dtype=torch.bfloat16)
    sl.sl_mx4_linear(x, w, y, sl.alloc_mx4_workspace(0, n, k))
    sl.sl_mx4_product(q[0], w, y, k, sl.alloc_mx4_workspace(0, n, k))
    dw = torch.full((n, k), 7.0, device="cuda")
    sl.sl_mx4_product(q[3], q[1], dw, 0, sl.alloc_mx4_workspace(n, k, 0))
    assert float(dw.abs().sum()) == 0.0


@pytest.mark.parametrize("sizes", [(5, 40, 300), (40, 40, 300), (300, 200, 1100)])
def test_blocks_of_nan_stay_in_their_row(sizes):
    import torch
    from paper_2508_15706_amd import binding as sl
    m, n, k = sizes
    x, w = matrix(m, k, "bf16", 1, spread=False), matrix(n, k, "bf16", 2, spread=False)
    x[3, 5] = float("inf")
    x[1, k - 1] = float("nan")
    w[7, 200] = float("nan")
    ws = sl.alloc_mx4_workspace(m, n, k)
    want = np.zeros((m, n), bool)
    want[[3, 1]] = True
    want[:, 7] = True
    (qa, _), (qb, _) = quantized(x), quantized(w)
    c, y = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    sl.sl_mx4_product(qa, qb, c, k, ws)
    sl.sl_mx4_linear(x, qb, y, ws)
    for t in (c, y):
        assert np.array_equal(np.isnan(host(t)), want) and not np.isinf(host(t)).any()


@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** -60, 2.0 ** 60])
def test_products_far_from_one(scale):
    """Scales multiply outside the elements: sums below fp32's range vanish, others keep their precision."""
    import torch
    from paper_2508_15706_amd import binding as sl
    x, w = matrix(20, 256, "f32", 1, spread=False) * scale, matrix(24, 256, "f32", 2, spread=False) * scale
    (qa, a), (qb, b) = quantized(x), quantized(w)
    c = torch.empty(20, 24, device="cuda")
    sl.sl_mx4_product(qa, qb, c, 256, sl.alloc_mx4_workspace(20, 24, 256))
    assert (np.abs(host(c) - a @ b.T) <= product_bound(a, b, 256, "f32") + 2.0 ** -126).all()


@pytest.mark.parametrize("x_kind", ["f32", "bf16"])
@pytest.mark.parametrize("y_kind", ["f32", "bf16"])
@pytest.mark.parametrize("m", [1, 2, 7, 16, 17, 33, 64, 65, 150])
@pytest.mark.parametrize("n, k", [(64, 128), (530, 200), (1, 33), (2051, 1024), (48, 4099)])
def test_linear(m, n, k, x_kind, y_kind):
    import torch
    from paper_2508_15706_amd import binding as sl
    big = matrix(m, k + 3, x_kind, 1, spread=False)
    x = big[:, 1:k + 1]                                       # rows that are aligned to their element only
    qw, w = quantized(matrix(n, k, "f32", 2, spread=False))
    a = mx4_reference(host(x))[2]
    y = torch.full((m, n + 1), 7.0, dtype=torch.bfloat16 if y_kind == "bf16" else torch.float32, device="cuda")
    ws = sl.alloc_mx4_workspace(m, n, k)
    sl.sl_mx4_linear(x, qw, y[:, :n], ws)
    got = host(y)
    assert (np.abs(got[:, :n] - a @ w.T) <= product_bound(a, w, k, y_kind)).all()
    assert (got[:, n] == 7.0).all()
    aligned = torch.empty_like(y[:, :n].contiguous())
    sl.sl_mx4_linear(x.contiguous(), qw, aligned, ws)
    assert torch.equal(aligned, y[:, :n])


def test_gradients_of_a_linear_layer():
    """x, W and dy on the format's grid, so that quantisation loses nothing: the gradients of L = sum(y dy) are dy W and dy^T x
    (checked against the formula) and, L being linear in each element, equal differences of L, which is computed through the forward call."""
    import torch
    from paper_2508_15706_amd import binding as sl
    m, n, k = 48, 70, 100
    rng = np.random.default_rng(0)

    def grid(r, c):
        v = rng.choice([-2.0, -1.5, -1.0, -0.5, 0.0, 0.5, 1.0, 1.5, 2.0], (r, c))
        v[rng.integers(0, 1, r), :] = np.where(v[rng.integers(0, 1, r), :] == 0, 0.5, v[rng.integers(0, 1, r), :])
        return v

    def onto(v):
        return torch.from_numpy(v.astype(np.float32)).cuda()

    def pair(t):
        q, qt = sl.alloc_mx4(*t.shape), sl.alloc_mx4(t.shape[1], t.shape[0])
        sl.sl_mx4_quantize(t, q, qt)
        back = torch.empty_like(t)
        sl.sl_mx4_dequantize(q, back)
        assert torch.equal(back, t)                            # nothing lost
        return q, qt

    X, W, G = grid(m, k), grid(n, k), grid(m, n)

    def forward(x, w):
        y = torch.empty(m, n, device="cuda")
        sl.sl_mx4_product(pair(onto(x))[0], pair(onto(w))[0], y, k, sl.alloc_mx4_workspace(m, n, k))
        return y

    def loss(x, w):
        return float((host(forward(x, w)) * G).sum())

    (qx, qxt), (qw, qwt), (qg, qgt) = pair(onto(X)), pair(onto(W)), pair(onto(G))
    dx, dw = torch.empty(m, k, device="cuda"), torch.empty(n, k, device="cuda")
    sl.sl_mx4_product(qg, qwt, dx, n, sl.alloc_mx4_workspace(m, k, n))
    sl.sl_mx4_product(qgt, qxt, dw, m, sl.alloc_mx4_workspace(n, k, m))
    assert np.array_equal(host(dx), G @ W) and np.array_equal(host(dw), G.T @ X)     # multiples of 1/4, exact in fp32
    for _ in range(6):
        i, j, l = rng.integers(0, m), rng.integers(0, n), rng.integers(0, k)
        for base, grad, at in ((X, dx, (i, l)), (W, dw, (j, l))):
            up, down = base.copy(), base.copy()
            up[at], down[at] = 2.0, -2.0
            diff = (loss(up, W) - loss(down, W)) / 4 if base is X else (loss(X, up) - loss(X, down)) / 4
            assert diff == float(grad[at])


def test_other_stream_and_graph():
    import torch
    from paper_2508_15706_amd import binding as sl
    m, n, k = 150, 270, 400
    x, w, dy = matrix(m, k, "bf16", 1, False), matrix(n, k, "bf16", 2, False), matrix(m, n, "bf16", 3, False)
    ws = [sl.alloc_mx4_workspace(m, n, k) for _ in range(3)]
    sizes = {"x": (m, k), "xt": (k, m), "w": (n, k), "g": (m, n), "gt": (n, m)}

    def fresh():
        return {**{a: sl.alloc_mx4(*s) for a, s in sizes.items()}, "y": torch.empty(m, n, device="cuda"), "z": torch.empty(2, n, device="cuda"),
                "dw": torch.zeros(n, k, device="cuda")}

    def step(s, stream=None):
        sl.sl_mx4_quantize(x, s["x"], s["xt"], stream=stream)
        sl.sl_mx4_quantize(w, s["w"], stream=stream)
        sl.sl_mx4_quantize(dy, s["g"], s["gt"], stream=stream)
        sl.sl_mx4_product(s["x"], s["w"], s["y"], k, ws[0], stream=stream)
        sl.sl_mx4_linear(x[:2], s["w"], s["z"], ws[1], stream=stream)
        sl.sl_mx4_product(s["gt"], s["xt"], s["dw"], m, None if not sl.sl_mx4_workspace_bytes(n, k, m) else sl_ws, accumulate=True, stream=stream)

    sl_ws = sl.alloc_mx4_workspace(n, k, m)
    want, got, replayed = fresh(), fresh(), fresh()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    step(got, side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(replayed)
    for i in range(4):
        step(want)
        graph.replay()
        torch.cuda.synchronize()
        for key in ("y", "z", "dw"):
            assert torch.equal(want[key], replayed[key])
            if i == 0:
                assert torch.equal(want[key], got[key])


def test_refusals():
    import torch
    from paper_2508_15706_amd import binding as sl
    assert sl.sl_mx4_bytes(0, 5) == 0 and sl.sl_mx4_bytes(5, -1) == 0 and sl.sl_mx4_bytes(1 << 30, 1 << 30) == 0
    x = torch.zeros(8, 64, device="cuda")
    q, y = sl.alloc_mx4(8, 64), torch.zeros(8, 8, device="cuda")
    ws = sl.alloc_mx4_workspace(8, 8, 64)
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_mx4_quantize(x, None, None)
    with pytest.raises(ValueError):
        sl.sl_mx4_quantize(x.double(), q)
    with pytest.raises(ValueError):
        sl.sl_mx4_quantize(x, q[:64])                           # too small
    with pytest.raises(ValueError):
        sl.sl_mx4_quantize(x.t(), q)                            # rows that are not contiguous
    big = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_mx4_quantize(x, big[1:])                          # misaligned
    with pytest.raises(ValueError):
        sl.sl_mx4_product(q, q, torch.zeros(8, 8, device="cuda"), 65 * 1024, ws)
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_mx4_product(q, q, y.bfloat16(), 64, ws, accumulate=True)
    with pytest.raises(ValueError):
        sl.sl_mx4_linear(x[:4], q, y, ws)
    L = sl.lib()
    assert L.sl_mx4_product(q.data_ptr(), q.data_ptr(), 8, 8, 64, y.data_ptr(), 0, 7, 0, ws.data_ptr(), None) == -1     # ldc < n
    assert L.sl_mx4_product(q.data_ptr(), q.data_ptr(), 8, 8, -1, y.data_ptr(), 0, 8, 0, ws.data_ptr(), None) == -1
    assert L.sl_mx4_product(q.data_ptr(), q.data_ptr(), 8, 8, 64, y.data_ptr(), 2, 8, 0, ws.data_ptr(), None) == -1
    assert L.sl_mx4_linear(x.data_ptr(), 0, 63, q.data_ptr(), 8, 8, 64, y.data_ptr(), 0, 8, ws.data_ptr(), None) == -1  # ldx < k
    assert float(y.abs().sum()) == 0.0
