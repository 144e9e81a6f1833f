"""The root-mean-square norm and its backward pass against their definitions in 64 bits."""
import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu

EPS = 1e-5


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}


def rand(shape, kind, seed, std=1.0, pad=0):
    """A device matrix of the kind, as a view of one whose rows are `pad` elements longer."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.empty(shape[0], shape[1] + pad, device="cuda").normal_(0, std, generator=g).to(types()[kind])
    return t[:, :shape[1]]


def near(got, want, off, what):
    got = got.double()
    bound = off + ref.HALF[got_type(what)] * (want.abs() + off) + 1e-300
    worst = ((got - want).abs() / bound).max()
    assert float(worst) <= 1.0, (what, float(worst))


def got_type(what):
    return what[1]


SHAPES = [(1, 1), (1, 2048), (3, 7), (5, 8), (33, 200), (64, 512), (31, 513), (129, 1000), (4, 2049), (7, 8192), (2, 9000), (3, 16385), (2, 40001)]


@pytest.mark.parametrize("x_type,r_type,w_type,y_type", [("bf16", "f32", "f32", "bf16"), ("bf16", "bf16", "bf16", "bf16"), ("f32", "f32", "f32", "f32"),
                                                         ("f32", "bf16", "bf16", "f32"), ("bf16", None, "f32", "bf16"), ("f32", None, "bf16", "f32")])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, x_type, r_type, w_type, y_type):
    import torch
    from paper_2508_15706_amd import binding as sl
    x = rand(shape, x_type, 1, pad=3)
    r = None if r_type is None else rand(shape, r_type, 2, std=3.0, pad=1)
    w = rand((1, shape[1]), w_type, 3)[0].contiguous()
    y = torch.full((shape[0], shape[1] + 5), 7.0, device="cuda", dtype=types()[y_type])
    h = None if r is None else torch.full_like(r, 7.0)
    s = torch.empty(shape[0], device="cuda")
    sl.sl_rms_norm(x, w, y[:, :shape[1]], residual=r, h=h, rstd=s, eps=EPS)
    eh, es, ey = ref.norm(x, r, w, EPS, x.dtype if r is None else r.dtype)
    if h is not None:
        assert torch.equal(h.double(), eh)
    near(s, es, 1e-15 * es, ("rstd", torch.float32))
    # the rounding of s, of the product with it and of that with w, the last one y's own
    near(y[:, :shape[1]], ey, 2 * ref.F32 * ey.abs() * (1 + 2 ** -20) + (ref.F32 * ey.abs() if y_type == "bf16" else 0.0), ("y", types()[y_type]))
    assert bool((y[:, shape[1]:] == 7.0).all())


@pytest.mark.parametrize("x_type,r_type", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", None), ("bf16", None)])
@pytest.mark.parametrize("shape", [(1, 1), (1, 2048), (2, 33), (31, 130), (32, 64), (33, 200), (65, 1023), (130, 2048), (200, 2049), (40, 5000)])
@pytest.mark.parametrize("way", ["q", "qt", "both"])
def test_four_bits(shape, x_type, r_type, way):
    """The 4-bit matrices are those of the bf16 result, byte for byte, what fills up their tiles included."""
    import torch
    from paper_2508_15706_amd import binding as sl
    rows, cols = shape
    x = rand(shape, x_type, 1, std=2.0)
    r = None if r_type is None else rand(shape, r_type, 2)
    w = rand((1, cols), "f32", 3)[0].contiguous()
    y = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
    h = None if r is None else torch.empty_like(r)
    h2 = None if r is None else torch.empty_like(r)
    sl.sl_rms_norm(x, w, y, residual=r, h=h, eps=EPS)
    want = [torch.full((sl.sl_mx4_bytes(*s),), 171, dtype=torch.uint8, device="cuda") for s in ((rows, cols), (cols, rows))]
    sl.sl_mx4_quantize(y, *want)
    got = [torch.full_like(t, 171) for t in want]
    y2, s2, s1 = torch.empty_like(y), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    sl.sl_rms_norm(x, w, y2 if way == "both" else None, residual=r, h=h2, rstd=s2, q=got[0] if way != "qt" else None, qt=got[1] if way != "q" else None, eps=EPS)
    sl.sl_rms_norm(x, w, None, residual=r, h=h, rstd=s1, eps=EPS)
    assert torch.equal(s1, s2)
    if r is not None:
        assert torch.equal(h, h2)
    if way == "both":
        assert torch.equal(y, y2)
    if way != "qt":
        assert torch.equal(got[0], want[0])
    if way != "q":
        assert torch.equal(got[1], want[1])


@pytest.mark.parametrize("h_type,dy_type,dx_type", [("f32", "bf16", "f32"), ("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "f32"),
                                                    ("f32", "f32", "bf16"), ("bf16", "bf16", "f32"), ("f32", "bf16", "bf16"), ("bf16", "f32", "bf16")])
@pytest.mark.parametrize("shape", [(1, 1), (1, 2048), (3, 7), (33, 200), (64, 512), (131, 513), (5, 2049), (9, 8192), (6, 9000), (5, 20001), (3000, 40)])
@pytest.mark.parametrize("past", [True, False])
def test_backward(shape, h_type, dy_type, dx_type, past):
    import torch
    from paper_2508_15706_amd import binding as sl
    rows, cols = shape
    h, dy = rand(shape, h_type, 1, pad=2), rand(shape, dy_type, 2, pad=1)
    w = rand((1, cols), "f32", 3)[0].contiguous()
    dh = rand(shape, dx_type, 4, pad=3) if past else None
    s = (1.0 / torch.sqrt(h.double().square().mean(1) + EPS)).float()
    dx, dw = torch.empty(shape, device="cuda", dtype=types()[dx_type]), torch.full((cols,), 3.0, device="cuda")
    ws = sl.alloc_rms_norm_workspace(rows, cols)
    sl.sl_rms_norm_backward(h, w, s, dy, dx, dh=dh, dw=dw, workspace=ws)
    ex, ox, ew, ow = ref.norm_backward(h, w, s, dy, dh)
    near(dx, ex, ox, ("dx", dx.dtype))
    near(dw, ew, ow, ("dw", torch.float32))
    first = dw.clone()
    sl.sl_rms_norm_backward(h, w, s, dy, dx, dh=dh, dw=dw, workspace=ws, accumulate=True)
    assert float((dw.double() - 2 * first.double()).abs().max()) <= float(4 * ref.F32 * (first.abs().max()))
    dx2 = torch.empty_like(dx)
    sl.sl_rms_norm_backward(h, w, s, dy, dx2, dh=dh)
    assert torch.equal(dx, dx2)
    if dh is not None:                                        # in place, and the same bits again
        sl.sl_rms_norm_backward(h, w, s, dy, dh, dh=dh, dw=dw, workspace=ws)
        assert torch.equal(dh, dx) and torch.equal(dw, first)


def test_in_place_residual_and_empty():
    import torch
    from paper_2508_15706_amd import binding as sl
    for cols in (100, 2500, 40000):
        x, r = rand((6, cols), "bf16", 1), rand((6, cols), "f32", 2).contiguous()
        w = torch.ones(cols, device="cuda")
        y, y2, h = (torch.empty(6, cols, device="cuda") for _ in range(3))
        q = sl.alloc_mx4(6, cols)
        r2 = r.clone()
        sl.sl_rms_norm(x, w, y, residual=r, h=h)
        sl.sl_rms_norm(x, w, y2, residual=r2, h=r2)
        assert torch.equal(h, r2) and torch.equal(y, y2)
        sl.sl_rms_norm(x, w, y2, residual=r, h=r, q=q)
        assert torch.equal(h, r) and torch.equal(y, y2)
    empty = torch.empty(0, 64, device="cuda")
    sl.sl_rms_norm(empty, torch.ones(64, device="cuda"), empty.clone())
    dw = torch.full((64,), 5.0, device="cuda")
    sl.sl_rms_norm_backward(empty, torch.ones(64, device="cuda"), torch.empty(0, device="cuda"), empty.clone(), empty.clone(), dw=dw,
                            workspace=sl.alloc_rms_norm_workspace(0, 64), accumulate=True)
    assert bool((dw == 5.0).all())
    sl.sl_rms_norm_backward(empty, torch.ones(64, device="cuda"), torch.empty(0, device="cuda"), empty.clone(), empty.clone(), dw=dw,
                            workspace=sl.alloc_rms_norm_workspace(0, 64))
    assert bool((dw == 0.0).all())


def test_rows_are_apart():
    """Zeros, infinities, NaN and the ends of the range in one row change no other one, and no block of another row's 4-bit matrix."""
    import torch
    from paper_2508_15706_amd import binding as sl
    x = rand((40, 96), "f32", 1)
    w = torch.ones(96, device="cuda")
    y, clean = torch.empty_like(x), torch.empty_like(x)
    q, q2 = sl.alloc_mx4(40, 96), sl.alloc_mx4(40, 96)
    x[7] = 0.0
    sl.sl_rms_norm(x, w, clean, q=q2)
    assert bool((clean[7] == 0).all())
    x[3, 5], x[4, 0], x[9] = float("inf"), float("nan"), 1e37
    sl.sl_rms_norm(x, w, y, q=q)
    rest = [i for i in range(40) if i not in (3, 4, 9)]
    assert torch.equal(y[rest], clean[rest])
    assert bool(y[4].isnan().all()) and bool(y[3, 5].isnan()) and float((y[9] - 1).abs().max()) < 1e-5
    dense = torch.empty(40, 96, device="cuda")
    sl.sl_mx4_dequantize(q, dense)
    want = torch.empty(40, 96, device="cuda")
    sl.sl_mx4_dequantize(q2, want)
    assert torch.equal(dense[rest], want[rest]) and bool(dense[4].isnan().all())


def test_offsets_beyond_32_bits():
    import torch
    from paper_2508_15706_amd import binding as sl
    rows, cols = 1_100_000, 2000                               # 2.2e9 elements
    x = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    x[-40:] = rand((40, cols), "bf16", 1)
    w = rand((1, cols), "f32", 3)[0].contiguous()
    y, s = torch.empty_like(x), torch.empty(rows, device="cuda")
    sl.sl_rms_norm(x, w, y, rstd=s, eps=EPS)
    _, es, ey = ref.norm(x[-40:], None, w, EPS, torch.bfloat16)
    near(y[-40:], ey, 3 * ref.F32 * ey.abs(), ("y", torch.bfloat16))
    assert bool((y[:100] == 0).all())
    dx, dw = torch.empty_like(x), torch.empty(cols, device="cuda")
    sl.sl_rms_norm_backward(x, w, s, y, dx, dw=dw, workspace=sl.alloc_rms_norm_workspace(rows, cols))
    ex, ox, ew, ow = ref.norm_backward(x[-40:], w, s[-40:], y[-40:], None)
    near(dx[-40:], ex, ox, ("dx", torch.bfloat16))
    near(dw, ew, ow, ("dw", torch.float32))
