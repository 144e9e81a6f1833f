"""AdamW over tensor lists (32- and 8-bit moments) and the gradient norm, against their definitions in 64 bits."""
import numpy as np
import pytest

from inner_reference import adamw_reference, decode8, encode8_positions, random_bits

pytestmark = pytest.mark.gpu

LISTS = {
    "one": [(1, 1)],
    "tiny": [(1, 3), (1, 4), (1, 5), (2, 1)],
    "edges": [(1, 255), (1, 256), (1, 257), (1, 4095), (1, 4096), (1, 4097), (3, 1366)],
    "ragged": [(200, 530), (1, 200), (67, 31), (1, 1), (64, 64), (5003, 20)],
    "long": [(1024, 1024), (1, 1024)],
}
PARAMS = {"lr": 3e-3, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "weight_decay": 0.1, "step": 7}


def layout(name, gap=4):
    """descs with gaps between the tensors, the arena's length, a mask of its elements that belong to a tensor, and for
    those the tensor, the block in the list and the place in the block."""
    descs, off, blocks = [], 8, 0
    parts = []
    for t, (r, c) in enumerate(LISTS[name]):
        n = r * c
        descs.append((r, c, off, 1 if r > 1 else 0))
        i = np.arange(n)
        parts.append((off + i, np.full(n, t), blocks + i // 256, i % 256))
        blocks += -(-n // 256)
        off += (n + 3) // 4 * 4 + gap
    at, tensor, block, place = (np.concatenate(z) for z in zip(*parts))
    return descs, off, at, tensor, block, place, blocks


def inputs(n, at, seed, grad_std=1e-2):
    rng = np.random.default_rng(seed)
    a = {"theta": rng.normal(0, 0.05, n), "grad": rng.normal(0, grad_std, n), "m": rng.normal(0, 3e-3, n),
         "v": rng.uniform(0, 2e-4, n)}
    a["v"][at[::7]] = 0.0
    a["m"][at[::7]] = 0.0
    a["grad"][at[::21]] = 0.0
    return {k: z.astype(np.float32) for k, z in a.items()}


def device(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


@pytest.mark.parametrize("grad_type", ["f32", "bf16"])
@pytest.mark.parametrize("name", sorted(LISTS))
@pytest.mark.parametrize("scaled", [False, True])
def test_step_against_64_bits(name, grad_type, scaled):
    import torch
    from paper_2508_15706_amd import binding as sl
    descs, n, at, tensor, *_ = layout(name)
    a = inputs(n, at, 1)
    decay = [0.0 if i % 2 else 0.5 for i in range(len(descs))]
    grad = device(a["grad"], torch.bfloat16 if grad_type == "bf16" else None)
    g64 = grad.double().cpu().numpy()
    theta, m, v = (device(a[k]) for k in ("theta", "m", "v"))
    t16 = torch.full((n,), -7.0, dtype=torch.bfloat16, device="cuda")
    scale = torch.tensor([0.625], device="cuda") if scaled else None
    opt = sl.sl_adamw_create(descs, decay)
    sl.sl_adamw_step(opt, theta, grad, m, v, **PARAMS, grad_scale=scale, theta16=t16 if scaled else None)
    keep = 1 - np.array(decay)[tensor] * PARAMS["lr"] * PARAMS["weight_decay"]
    wt, wm, wv, et, em, ev = adamw_reference(*(a[k].astype(np.float64)[at] for k in ("theta",)), g64[at],
                                             a["m"].astype(np.float64)[at], a["v"].astype(np.float64)[at],
                                             0.625 if scaled else 1.0, keep, PARAMS)
    for got, want, bound, was in ((theta, wt, et, a["theta"]), (m, wm, em, a["m"]), (v, wv, ev, a["v"])):
        got = got.cpu().numpy()
        assert (np.abs(got[at].astype(np.float64) - want) <= bound).all()
        gaps = np.ones(n, bool)
        gaps[at] = False
        assert np.array_equal(got[gaps], was[gaps])          # what belongs to no tensor is not written
    if scaled:
        want16 = theta.to(torch.bfloat16)
        assert torch.equal(t16[torch.from_numpy(at).cuda()], want16[torch.from_numpy(at).cuda()])
        assert bool((t16[torch.from_numpy(gaps).cuda()] == -7.0).all())


def test_steps_carry_their_state():
    """Five steps in a row: every step from the state of the one before."""
    from paper_2508_15706_amd import binding as sl
    descs, n, at, tensor, *_ = layout("ragged")
    a = inputs(n, at, 3)
    theta, m, v = device(a["theta"]), device(np.zeros(n, np.float32)), device(np.zeros(n, np.float32))
    opt = sl.sl_adamw_create(descs)
    for step in range(1, 6):
        p = dict(PARAMS, step=step)
        grad = np.random.default_rng(step).normal(0, 1e-2, n).astype(np.float32)
        before = [z.cpu().numpy().astype(np.float64)[at] for z in (theta, m, v)]
        sl.sl_adamw_step(opt, theta, device(grad), m, v, **p)
        wt, wm, wv, et, em, ev = adamw_reference(before[0], grad.astype(np.float64)[at], before[1], before[2], 1.0,
                                                 1 - PARAMS["lr"] * PARAMS["weight_decay"], p)
        for got, want, bound in ((theta, wt, et), (m, wm, em), (v, wv, ev)):
            assert (np.abs(got.cpu().numpy().astype(np.float64)[at] - want) <= bound).all()


def state8(n, at, block, blocks, seed):
    """Random 8-bit moments: codes of every magnitude, blocks of zeros, scales over a wide range."""
    rng = np.random.default_rng(seed)
    m, v = rng.integers(0, 256, n).astype(np.uint8), rng.integers(0, 256, n).astype(np.uint8)
    ms, vs = rng.integers(112, 122, blocks).astype(np.uint8), rng.integers(100, 116, blocks).astype(np.uint8)
    m[np.isin(np.arange(n), at[block % 5 == 2])] = 0
    v[np.isin(np.arange(n), at[block % 5 == 2])] = 0
    return m, v, ms, vs


def check8(at, block, place, blocks, got, scales, want, spread, seed, signed):
    """Codes and scale bytes after a step against the 64-bit moments `want`, known to within `spread`."""
    bits = random_bits(seed, block, place).astype(np.int64)
    rnd = bits & 0xFFFF if signed else bits >> 16
    top = np.zeros(blocks)
    np.maximum.at(top, block, np.abs(want))
    X, _ = encode8_positions(want, rnd, top[block], signed)
    # the block's exponent may differ where its largest value lies on the edge of a binade, within the error of fp32
    lo, _ = encode8_positions(want, rnd, top[block] * (1 - 1e-6), signed)
    hi, _ = encode8_positions(want, rnd, top[block] * (1 + 1e-6), signed)
    gx = scales.astype(np.int64)[block]
    assert ((gx == X) | (gx == lo) | (gx == hi)).all()
    same = gx == X
    code = got[at].astype(np.int64)
    mag = code & 127 if signed else code
    _, low = encode8_positions(np.maximum(np.abs(want) - spread, 0), rnd, top[block], signed)
    _, high = encode8_positions(np.abs(want) + spread, rnd, top[block], signed)
    most = 127 if signed else 255
    low, high = np.minimum(np.floor(low - 1e-6), most), np.minimum(np.floor(high + 1e-6), most)
    if not signed:
        low, high = np.maximum(low, (want > 0) * 1), np.maximum(high, (want > 0) * 1)
    assert ((mag >= low) & (mag <= high))[same].all()
    if signed:
        assert ((code > 127) == (want < 0))[same & (np.abs(want) > spread)].all()


@pytest.mark.parametrize("grad_type", ["f32", "bf16"])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_step8_against_64_bits(name, grad_type):
    import torch
    from paper_2508_15706_amd import binding as sl
    descs, n, at, tensor, block, place, blocks = layout(name)
    a = inputs(n, at, 5)
    m8, v8, ms, vs = state8(n, at, block, blocks, 6)
    grad = device(a["grad"], torch.bfloat16 if grad_type == "bf16" else None)
    theta = device(a["theta"])
    dm, dv, dms, dvs = device(m8), device(v8), device(ms), device(vs)
    t16 = torch.full((n,), -7.0, dtype=torch.bfloat16, device="cuda")
    opt = sl.sl_adamw_create(descs)
    assert opt.num_blocks == blocks
    seed = 0x9E3779B9
    sl.sl_adamw_step8(opt, theta, grad, dm, dv, dms, dvs, seed, **PARAMS, theta16=t16)
    m = decode8(m8[at], ms, block, True)
    v = decode8(v8[at], vs, block, False)
    wt, wm, wv, et, em, ev = adamw_reference(a["theta"].astype(np.float64)[at], grad.double().cpu().numpy()[at], m, v, 1.0,
                                             1 - PARAMS["lr"] * PARAMS["weight_decay"], PARAMS)
    assert (np.abs(theta.cpu().numpy().astype(np.float64)[at] - wt) <= et).all()
    check8(at, block, place, blocks, dm.cpu().numpy(), dms.cpu().numpy(), wm, em, seed, True)
    check8(at, block, place, blocks, dv.cpu().numpy(), dvs.cpu().numpy(), wv, ev, seed, False)
    gaps = np.ones(n, bool)
    gaps[at] = False
    for got, was in ((theta, a["theta"]), (dm, m8), (dv, v8)):
        assert np.array_equal(got.cpu().numpy()[gaps], was[gaps])
    tat = torch.from_numpy(at).cuda()
    assert torch.equal(t16[tat], theta.to(torch.bfloat16)[tat])
    # the values they stand for
    for moment, codes, scales, signed in ((1, dm, dms, True), (2, dv, dvs, False)):
        out = torch.full((n,), 5.0, device="cuda")
        sl.sl_adamw_state_values(opt, moment, codes, scales, out)
        want = decode8(codes.cpu().numpy()[at], scales.cpu().numpy(), block, signed)
        assert np.array_equal(out.cpu().numpy()[at].astype(np.float64), want)
        assert (out.cpu().numpy()[gaps] == 5.0).all()


def test_every_code_and_scale_has_its_value():
    """All 256 codes in blocks of ordinary and of the lowest scales: what fp32 can hold is exact, below it rounded once."""
    import torch
    from paper_2508_15706_amd import binding as sl
    scales = np.array([0, 1, 2, 127, 252, 253, 254, 255], np.uint8)
    n = 256 * len(scales)
    opt = sl.sl_adamw_create([(1, n, 0, 0)])
    codes = np.tile(np.arange(256, dtype=np.uint8), len(scales))
    block = np.arange(n) // 256
    for moment, signed in ((1, True), (2, False)):
        out = torch.empty(n, device="cuda")
        sl.sl_adamw_state_values(opt, moment, device(codes), device(scales), out)
        want = decode8(codes, scales, block, signed)
        np.testing.assert_array_equal(out.cpu().numpy(), want.astype(np.float32))


def test_positive_second_moment_is_never_stored_as_zero():
    from paper_2508_15706_amd import binding as sl
    import torch
    n = 256
    grad = np.full(n, 1e-12, np.float32)
    grad[0] = 1.0
    grad[1] = 0.0
    opt = sl.sl_adamw_create([(1, n, 0, 0)])
    z = lambda k: torch.zeros(k, dtype=torch.uint8, device="cuda")  # noqa: E731
    m, v, ms, vs = z(n), z(n), z(1), z(1)
    sl.sl_adamw_step8(opt, torch.zeros(n, device="cuda"), device(grad), m, v, ms, vs, 1, **PARAMS)
    v = v.cpu().numpy()
    assert v[1] == 0 and (v[2:] == 1).all()


def test_random_rounding_follows_a_slow_second_moment():
    """v moves by (1 - beta2) = 0.1 % of its distance a step, far below half a code's step (6 %): rounded to nearest it would
    stand still.  The mean over 65,536 elements is within 5 standard errors of the recursion's value: one rounding
    changes v by less than 1/8 of itself, 500 of them, each damped by what follows, by 1/8 * sqrt(500) / 256 in the mean."""
    from paper_2508_15706_amd import binding as sl
    import torch
    n = 65536
    opt = sl.sl_adamw_create([(256, 256, 0, 1)])
    grad = torch.full((n,), 1e-3, device="cuda")
    z = lambda k: torch.zeros(k, dtype=torch.uint8, device="cuda")  # noqa: E731
    m, v, ms, vs = z(n), z(n), z(256), z(256)
    theta = torch.zeros(n, device="cuda")
    p = dict(PARAMS, beta2=0.999)
    for step in range(1, 501):
        sl.sl_adamw_step8(opt, theta, grad, m, v, ms, vs, step, **dict(p, step=step))
    out = torch.empty(n, device="cuda")
    sl.sl_adamw_state_values(opt, 2, v, vs, out)
    want = 1e-6 * (1 - 0.999 ** 500)
    got = float(out.double().mean())
    assert abs(got / want - 1) < 5 * 0.125 * 500 ** 0.5 / 256


def test_nothing_is_written_where_the_factor_is_nan():
    from paper_2508_15706_amd import binding as sl
    import torch
    descs, n, at, _, block, _, blocks = layout("ragged")
    a = inputs(n, at, 9)
    opt = sl.sl_adamw_create(descs)
    nan = torch.tensor([float("nan")], device="cuda")
    theta, m, v = (device(a[k]) for k in ("theta", "m", "v"))
    t16 = torch.full((n,), -7.0, dtype=torch.bfloat16, device="cuda")
    sl.sl_adamw_step(opt, theta, device(a["grad"]), m, v, **PARAMS, grad_scale=nan, theta16=t16)
    for got, k in ((theta, "theta"), (m, "m"), (v, "v")):
        assert np.array_equal(got.cpu().numpy(), a[k])
    m8, v8, ms, vs = state8(n, at, block, blocks, 10)
    dev = [device(z) for z in (m8, v8, ms, vs)]
    sl.sl_adamw_step8(opt, theta, device(a["grad"]), *dev, 3, **PARAMS, grad_scale=nan, theta16=t16)
    for got, was in zip([theta] + dev, [a["theta"], m8, v8, ms, vs]):
        assert np.array_equal(got.cpu().numpy(), was)
    assert bool((t16 == -7.0).all())


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_values_that_are_not_finite(bad):
    """Without a factor: 32 bits - the element alone; 8 bits - its block is NaN in the moments, theta the element alone."""
    from paper_2508_15706_amd import binding as sl
    import torch
    n = 4096 + 300
    rng = np.random.default_rng(4)
    grad = rng.normal(0, 1e-2, n).astype(np.float32)
    grad[1000] = bad
    opt = sl.sl_adamw_create([(1, n, 0, 0)])
    theta, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    sl.sl_adamw_step(opt, theta, device(grad), m, v, **PARAMS)
    for t in (theta, m, v):
        finite = torch.isfinite(t).cpu().numpy()
        assert not finite[1000] and finite.sum() == n - 1
    theta = torch.zeros(n, device="cuda")
    z = lambda k: torch.zeros(k, dtype=torch.uint8, device="cuda")  # noqa: E731
    m8, v8, ms, vs = z(n), z(n), z(18), z(18)
    sl.sl_adamw_step8(opt, theta, device(grad), m8, v8, ms, vs, 1, **PARAMS)
    for s in (ms, vs):
        s = s.cpu().numpy()
        assert s[1000 // 256] == 255 and (np.delete(s, 1000 // 256) < 255).all()
    finite = torch.isfinite(theta).cpu().numpy()
    assert not finite[1000] and finite.sum() == n - 1
    out = torch.empty(n, device="cuda")
    sl.sl_adamw_state_values(opt, 1, m8, ms, out)
    nan = torch.isnan(out).cpu().numpy()
    assert nan[768:1024].all() and nan.sum() == 256


@pytest.mark.parametrize("grad_type", ["f32", "bf16"])
@pytest.mark.parametrize("name", sorted(LISTS))
@pytest.mark.parametrize("std", [1e-25, 1e-3, 1e30])
def test_norm(name, grad_type, std):
    """Squares of 1e-25 and 1e30 leave the range of fp32; the norm does not.  fp64 sums of n squares: a relative error of
    n 2^-53, then one rounding to fp32."""
    import torch
    from paper_2508_15706_amd import binding as sl
    descs, n, at, *_ = layout(name)
    g = np.random.default_rng(2).normal(0, 1, n) * std
    grad = device(g.astype(np.float32), torch.bfloat16 if grad_type == "bf16" else None)
    gaps = np.ones(n, bool)
    gaps[at] = False
    grad[torch.from_numpy(gaps).cuda()] = float("nan")        # elements of no tensor are not read
    x = grad.double().cpu().numpy()[at]
    want = np.sqrt(np.sum(x * x))
    opt = sl.sl_adamw_create(descs)
    ws = sl.alloc_norm_workspace(opt)
    for limit in (want * 0.5, want * 2, np.inf):
        out = torch.full((2,), -1.0, device="cuda")
        sl.sl_grad_norm(opt, grad, limit, out, ws)
        norm, factor = out.cpu().tolist()
        assert abs(norm - want) <= 2.0 ** -23 * want
        limit32 = float(np.float32(limit))
        assert abs(factor - min(1.0, limit32 / want)) <= 2.0 ** -22 * factor
        again = torch.empty(2, device="cuda")
        sl.sl_grad_norm(opt, grad, limit, again, ws)
        assert torch.equal(out, again)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_norm_of_what_is_not_finite_stops_the_step(bad):
    import torch
    from paper_2508_15706_amd import binding as sl
    descs, n, at, *_ = layout("ragged")
    a = inputs(n, at, 1)
    a["grad"][at[777]] = bad
    opt = sl.sl_adamw_create(descs)
    out = torch.empty(2, device="cuda")
    sl.sl_grad_norm(opt, device(a["grad"]), 1.0, out, sl.alloc_norm_workspace(opt))
    assert not np.isfinite(out[0].item()) and np.isnan(out[1].item())
    theta, m, v = (device(a[k]) for k in ("theta", "m", "v"))
    sl.sl_adamw_step(opt, theta, device(a["grad"]), m, v, **PARAMS, grad_scale=out[1:])
    assert np.array_equal(theta.cpu().numpy(), a["theta"]) and np.array_equal(m.cpu().numpy(), a["m"])


def test_empty_list():
    import torch
    from paper_2508_15706_amd import binding as sl
    opt = sl.sl_adamw_create([])
    z = [torch.zeros(64, device="cuda") for _ in range(4)]
    out = torch.full((2,), -1.0, device="cuda")
    sl.sl_grad_norm(opt, z[0], 1.0, out, sl.alloc_norm_workspace(opt))
    assert out.tolist() == [0.0, 1.0]
    sl.sl_adamw_step(opt, z[0], z[1], z[2], z[3], **PARAMS)


def test_other_stream_and_graph():
    """The step on a stream of its own, then recorded once and replayed, against the eager calls."""
    import torch
    from paper_2508_15706_amd import binding as sl
    descs, n, at, _, block, _, blocks = layout("ragged")
    a = inputs(n, at, 11)
    m8, v8, ms, vs = state8(n, at, block, blocks, 12)
    opt = sl.sl_adamw_create(descs)
    grad, ws = device(a["grad"]), sl.alloc_norm_workspace(opt)

    def fresh():
        return [device(a[k]) for k in ("theta", "m", "v")] + [device(a["theta"])] + [device(z) for z in (m8, v8, ms, vs)] + [torch.empty(2, device="cuda")]

    def step(s, stream=None):
        sl.sl_grad_norm(opt, grad, 0.01, s[8], ws, stream=stream)
        sl.sl_adamw_step(opt, s[0], grad, s[1], s[2], **PARAMS, grad_scale=s[8][1:], stream=stream)
        sl.sl_adamw_step8(opt, s[3], grad, *s[4:8], 77, **PARAMS, grad_scale=s[8][1:], stream=stream)

    want = fresh()
    side, got = torch.cuda.Stream(), fresh()
    torch.cuda.synchronize()
    step(got, side)
    side.synchronize()
    replayed = fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(replayed)
    for i in range(4):
        step(want)
        graph.replay()
        torch.cuda.synchronize()
        for w, r in zip(want, replayed):
            assert torch.equal(w, r)
        if i == 0:
            for w, g in zip(want, got):
                assert torch.equal(w, g)


def test_refusals():
    import torch
    from paper_2508_15706_amd import binding as sl
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_create([(1, 8, 2, 0)])                     # offset not a multiple of 4
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_create([(1, 8, 0, 0), (1, 8, 4, 0)])       # overlap
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_create([(0, 8, 0, 0)])
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_create([(1, 8, 0, 0)], [float("inf")])
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_create([(1 << 20, 1 << 20, 0, 0)])         # more units than a grid holds
    opt = sl.sl_adamw_create([(1, 8, 0, 0)])
    t = [torch.zeros(16, device="cuda") for _ in range(4)]
    for change in ({"step": 0}, {"beta1": 1.0}, {"beta2": -0.1}, {"eps": 0.0}, {"lr": float("nan")}, {"weight_decay": float("inf")}):
        with pytest.raises(sl.SparseLoCoError):
            sl.sl_adamw_step(opt, *t, **dict(PARAMS, **change))
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_step(opt, t[0], t[1], t[2], t[2], **PARAMS)
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_step(opt, t[0][1:], t[1], t[2], t[3], **PARAMS)
    with pytest.raises(ValueError):
        sl.sl_adamw_step(opt, t[0], t[1].double(), t[2], t[3], **PARAMS)
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_grad_norm(opt, t[0], 0.0, t[1][:2], sl.alloc_norm_workspace(opt))
    c = [torch.zeros(16, dtype=torch.uint8, device="cuda") for _ in range(4)]
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_step8(opt, t[0], t[1], c[0], c[0], c[2], c[3], 1, **PARAMS)
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_state_values(opt, 3, c[0], c[1], t[0])
    assert all(float(z.abs().sum()) == 0 for z in t)
