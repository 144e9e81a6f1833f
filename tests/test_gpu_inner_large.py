"""The inner step's operators where offsets pass 32 bits: arenas of more than 2^32 elements, 4-bit matrices of more than 2^32 bytes."""
import numpy as np
import pytest

from inner_reference import adamw_reference, decode8, mx4_reference
from test_gpu_adamw import PARAMS, check8, inputs

pytestmark = pytest.mark.gpu

FAR = (1 << 32) + 4096


def need(gigabytes):
    import torch
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip("needs more device memory")


def test_adamw_far_into_an_arena():
    import torch
    from paper_2508_15706_amd import binding as sl
    need(100)
    shapes = [(1, 5000, 0, 0), (3, 1366, FAR, 1), (1, 257, FAR + 8192, 0)]
    n = FAR + 16384
    parts, blocks = [], 0
    for r, c, off, _ in shapes:
        i = np.arange(r * c)
        parts.append((off + i, blocks + i // 256, i % 256))
        blocks += -(-r * c // 256)
    at, block, place = (np.concatenate(z) for z in zip(*parts))
    tat = torch.from_numpy(at).cuda()
    k = at.size
    a = inputs(k, np.arange(k), 1)
    opt = sl.sl_adamw_create(shapes)

    def spread(values, dtype):
        t = torch.empty(n, dtype=dtype, device="cuda")
        t[tat] = torch.from_numpy(values).cuda().to(dtype)
        return t

    grad = spread(a["grad"], torch.bfloat16)
    g64 = grad[tat].double().cpu().numpy()
    out = torch.empty(2, device="cuda")
    sl.sl_grad_norm(opt, grad, 1e9, out, sl.alloc_norm_workspace(opt))
    want = np.sqrt((g64 * g64).sum())
    assert abs(float(out[0]) - want) <= 2.0 ** -23 * want
    theta, m, v = (spread(a[x], torch.float32) for x in ("theta", "m", "v"))
    t16 = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    sl.sl_adamw_step(opt, theta, grad, m, v, **PARAMS, theta16=t16)
    keep = 1 - PARAMS["lr"] * PARAMS["weight_decay"]
    wt, wm, wv, et, em, ev = adamw_reference(*(a[x].astype(np.float64) if x != "grad" else g64 for x in ("theta", "grad", "m", "v")), 1.0, keep, PARAMS)
    for got, ref, bound in ((theta, wt, et), (m, wm, em), (v, wv, ev)):
        assert (np.abs(got[tat].double().cpu().numpy() - ref) <= bound).all()
    assert torch.equal(t16[tat], theta[tat].to(torch.bfloat16))
    del m, v
    rng = np.random.default_rng(2)
    m8, v8 = rng.integers(0, 256, k).astype(np.uint8), rng.integers(0, 256, k).astype(np.uint8)
    ms, vs = rng.integers(112, 122, blocks).astype(np.uint8), rng.integers(100, 116, blocks).astype(np.uint8)
    theta[tat] = torch.from_numpy(a["theta"]).cuda()
    dm, dv = spread(m8, torch.uint8), spread(v8, torch.uint8)
    dms, dvs = torch.from_numpy(ms).cuda(), torch.from_numpy(vs).cuda()
    sl.sl_adamw_step8(opt, theta, grad, dm, dv, dms, dvs, 5, **PARAMS)
    wt, wm, wv, et, em, ev = adamw_reference(a["theta"].astype(np.float64), g64, decode8(m8, ms, block, True),
                                             decode8(v8, vs, block, False), 1.0, keep, PARAMS)
    assert (np.abs(theta[tat].double().cpu().numpy() - wt) <= et).all()
    here = np.arange(k)
    check8(here, block, place, blocks, dm[tat].cpu().numpy(), dms.cpu().numpy(), wm, em, 5, True)
    check8(here, block, place, blocks, dv[tat].cpu().numpy(), dvs.cpu().numpy(), wv, ev, 5, False)


def test_matrices_of_more_than_32_bits_of_bytes():
    import torch
    from paper_2508_15706_amd import binding as sl
    need(80)
    n, k, m = 2_200_003, 4096, 40
    w = torch.empty(n, k, dtype=torch.bfloat16, device="cuda").normal_()
    q, qt = sl.alloc_mx4(n, k), sl.alloc_mx4(k, n)
    assert q.numel() > 1 << 32
    sl.sl_mx4_quantize(w, q, qt)
    rows = np.array([0, 1, 1_048_575, 2_097_151, 2_097_152, 2_199_999, n - 1])
    picked = mx4_reference(w[torch.from_numpy(rows).cuda()].double().cpu().numpy())[2]
    back = torch.empty_like(w)
    sl.sl_mx4_dequantize(q, back)
    assert np.array_equal(back[torch.from_numpy(rows).cuda()].double().cpu().numpy(), picked)
    del back
    x = torch.empty(m, k, dtype=torch.bfloat16, device="cuda").normal_()
    qx = sl.alloc_mx4(m, k)
    sl.sl_mx4_quantize(x, qx)
    a = mx4_reference(x.double().cpu().numpy())[2]
    bound = k * 2.0 ** -23 * (np.abs(a) @ np.abs(picked).T) + 2.0 ** -8 * np.abs(a @ picked.T)
    y = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    ws = sl.alloc_mx4_workspace(m, n, k)
    at = torch.from_numpy(rows).cuda()
    sl.sl_mx4_product(qx, q, y, k, ws)
    assert (np.abs(y[:, at].double().cpu().numpy() - a @ picked.T) <= bound).all()
    sl.sl_mx4_linear(x[:2], q, y[:2].zero_(), ws)
    assert (np.abs(y[:2, at].double().cpu().numpy() - a[:2] @ picked.T) <= bound[:2]).all()
    # along the columns: the first 128 of the transposed matrix, whose blocks begin every 32 rows of w
    cols = mx4_reference(w[:64, :3].double().cpu().numpy().T)[2]
    last = mx4_reference(w[n - 35:, :3].double().cpu().numpy().T[:, -3 - 32:])[2]        # (n = 32 * 68,750 + 3)
    out = torch.empty(3, n, dtype=torch.bfloat16, device="cuda")
    first = sl.alloc_mx4(3, n)
    sl.sl_mx4_quantize(w[:, :3].t().contiguous(), first)
    sl.sl_mx4_dequantize(first, out)
    assert np.array_equal(out[:, :64].double().cpu().numpy(), cols)
    assert np.array_equal(out[:, n - 35:].double().cpu().numpy(), last)
    # the same blocks inside qt: codes of its first row tile, that tile's last column tile
    tiles = -(-n // 128)
    assert torch.equal(qt[:tiles * 2048].view(tiles, 4, 32, 16)[:, :, :3], first[:tiles * 2048].view(tiles, 4, 32, 16)[:, :, :3])
