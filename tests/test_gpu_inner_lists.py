"""AdamW and the gradient norm on lists that are long enough for the kernels of long ones, against their definitions in 64 bits on the
device: every element of theta and of the 32-bit moments, codes and scale bytes of blocks all over the list."""
import numpy as np
import pytest

from inner_reference import decode8
from test_gpu_adamw import PARAMS, check8

pytestmark = pytest.mark.gpu

# A unit is up to 4096 elements of one tensor; from 4096 units on a list is long, 1024 of them are a window of the order that it is taken in,
# and the norm's workgroups come round a second time above 8192.
LISTS = {
    "4095 units": [(4093, 4096), (1, 4097)],
    "4096 units": [(4093, 4096), (1, 4097), (1, 3)],
    "9818 units": [(3000, 5003), (1, 777), (1, 4095), (4099, 4099), (1, 1), (1234, 6791), (1, 257)],
}


def layout(name):
    """descs with gaps between the tensors, the arena's length, units, blocks."""
    descs, off, units, blocks = [], 8, 0, 0
    for r, c in LISTS[name]:
        n = r * c
        descs.append((r, c, off, 1 if r > 1 else 0))
        off += (n + 3) // 4 * 4 + 4
        units, blocks = units + -(-n // 4096), blocks + -(-n // 256)
    assert units == int(name.split()[0])
    return descs, off, units, blocks


def arenas(descs, n, grad_type):
    import torch
    g = torch.Generator(device="cuda").manual_seed(7)
    theta = torch.empty(n, device="cuda").normal_(0, 0.05, generator=g)
    grad = torch.empty(n, device="cuda").normal_(0, 1e-2, generator=g).to(torch.bfloat16 if grad_type == "bf16" else torch.float32)
    m = torch.empty(n, device="cuda").normal_(0, 3e-3, generator=g)
    v = torch.empty(n, device="cuda").uniform_(0, 2e-4, generator=g)
    v[::7] = 0.0
    m[::7] = 0.0
    grad[::21] = 0.0
    keep = torch.ones(n, dtype=torch.float64, device="cuda")       # 1 - decay * lr * weight_decay
    own = torch.zeros(n, dtype=torch.bool, device="cuda")          # elements of a tensor
    decay = [0.0 if i % 2 else 0.5 for i in range(len(descs))]
    for d, (r, c, off, _) in zip(decay, descs):
        keep[off:off + r * c] = 1 - d * PARAMS["lr"] * PARAMS["weight_decay"]
        own[off:off + r * c] = True
    return theta, grad, m, v, keep, own, decay


def reference(theta, grad, m, v, scale, keep):
    """adamw_reference of inner_reference, on the device."""
    import torch
    p, u = PARAMS, 2.0 ** -24
    g = grad * scale
    m1 = p["beta1"] * m + (1 - p["beta1"]) * g
    v1 = p["beta2"] * v + (1 - p["beta2"]) * g * g
    em = 5 * u * ((p["beta1"] * m).abs() + ((1 - p["beta1"]) * g).abs())
    ev = 7 * u * v1
    r, rate = 1 / (1 - p["beta2"] ** p["step"]) ** 0.5, p["lr"] / (1 - p["beta1"] ** p["step"])
    den = torch.sqrt(v1) * r + p["eps"]
    upd = rate * m1 / den
    new = theta * keep - upd
    et = em * rate / den + upd.abs() * ((3.5 + 5 + 4) * u) + 6 * u * theta.abs() + u * new.abs()
    return new, m1, v1, et + 2e-45, em + 2e-45, ev + 2e-45


def check(got, want, limit, was, own):
    import torch
    d = (got.double() - want).abs()
    assert bool((d <= limit)[own].all())
    assert torch.equal(got[~own], was[~own])                       # what belongs to no tensor is not written


@pytest.mark.parametrize("grad_type", ["f32", "bf16"])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_step(name, grad_type):
    import torch
    from paper_2508_15706_amd import binding as sl
    descs, n, *_ = layout(name)
    theta, grad, m, v, keep, own, decay = arenas(descs, n, grad_type)
    was = [t.clone() for t in (theta, m, v)]
    t16 = torch.full((n,), -7.0, dtype=torch.bfloat16, device="cuda")
    scale = torch.tensor([0.625], device="cuda")
    sl.sl_adamw_step(sl.sl_adamw_create(descs, decay), theta, grad, m, v, **PARAMS, grad_scale=scale, theta16=t16)
    new = reference(was[0].double(), grad.double(), was[1].double(), was[2].double(), 0.625, keep)
    for i, got in enumerate((theta, m, v)):
        check(got, new[i], new[3 + i], was[i], own)
    assert torch.equal(t16[own], theta.to(torch.bfloat16)[own]) and bool((t16[~own] == -7.0).all())


@pytest.mark.parametrize("grad_type", ["f32", "bf16"])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_step8(name, grad_type):
    import torch
    from paper_2508_15706_amd import binding as sl
    descs, n, units, blocks = layout(name)
    theta, grad, _, _, keep, own, decay = arenas(descs, n, grad_type)
    rng = np.random.default_rng(3)
    codes = [torch.from_numpy(rng.integers(0, 256, n).astype(np.uint8)).cuda() for _ in range(2)]
    scales = [torch.from_numpy(rng.integers(lo, lo + 10, blocks).astype(np.uint8)).cuda() for lo in (112, 106)]
    opt = sl.sl_adamw_create(descs, decay)
    assert opt.num_blocks == blocks
    before = [torch.zeros(n, device="cuda") for _ in range(2)]      # (exact: tests of the values have that)
    for i in range(2):
        sl.sl_adamw_state_values(opt, i + 1, codes[i], scales[i], before[i])
    was, codes_were = theta.clone(), [c.clone() for c in codes]
    t16 = torch.full((n,), -7.0, dtype=torch.bfloat16, device="cuda")
    seed = 0x9E3779B9
    sl.sl_adamw_step8(opt, theta, grad, *codes, *scales, seed, **PARAMS, theta16=t16)
    new = reference(was.double(), grad.double(), before[0].double(), before[1].double(), 1.0, keep)
    check(theta, new[0], new[3], was, own)
    assert torch.equal(t16[own], theta.to(torch.bfloat16)[own]) and bool((t16[~own] == -7.0).all())
    # the first and the last blocks of every tensor, and every 401st
    at, block, place, first = [], [], [], 0
    for r, c, off, _ in descs:
        of = -(-r * c // 256)
        picked = np.unique(np.concatenate([np.arange(min(of, 5)), np.arange(max(0, of - 5), of), np.arange(0, of, 401)]))
        i = (picked[:, None] * 256 + np.arange(256)).ravel()
        i = i[i < r * c]
        at.append(off + i), block.append(first + i // 256), place.append(i % 256)
        first += of
    at, block, place = (np.concatenate(z) for z in (at, block, place))
    tat = torch.from_numpy(at).cuda()
    here = np.arange(at.size)
    for i, signed in ((0, True), (1, False)):
        got, sc = codes[i][tat].cpu().numpy(), scales[i].cpu().numpy()
        assert torch.equal(codes[i][~own], codes_were[i][~own])
        # (the random bits go by the block's number in the list)
        check8(here, block, place, blocks, got, sc, new[1 + i][tat].cpu().numpy(), new[4 + i][tat].cpu().numpy(), seed, signed)
        out = torch.full((n,), 5.0, device="cuda")
        sl.sl_adamw_state_values(opt, i + 1, codes[i], scales[i], out)
        assert np.array_equal(out[tat].double().cpu().numpy(), decode8(got, sc, block, signed)) and bool((out[~own] == 5.0).all())


@pytest.mark.parametrize("grad_type", ["f32", "bf16"])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_norm(name, grad_type):
    """Bounds as for short lists; a unit left out or counted twice would change the norm by a part in 20,000 at least."""
    import torch
    from paper_2508_15706_amd import binding as sl
    descs, n, *_ = layout(name)
    _, grad, *_, own, _ = arenas(descs, n, grad_type)
    grad[~own] = float("nan")                                      # elements of no tensor are not read
    want = float(grad[own].double().square().sum().sqrt())
    opt = sl.sl_adamw_create(descs)
    out, ws = torch.empty(2, device="cuda"), sl.alloc_norm_workspace(opt)
    for limit in (want * 0.5, want * 2):
        sl.sl_grad_norm(opt, grad, limit, out, ws)
        norm, factor = out.cpu().tolist()
        assert abs(norm - want) <= 2.0 ** -23 * want
        assert abs(factor - min(1.0, float(np.float32(limit)) / want)) <= 2.0 ** -22 * factor
