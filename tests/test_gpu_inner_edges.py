"""The inner step's optimiser: parameters at the ends of fp32's range."""
import pytest

from test_gpu_adamw import PARAMS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("change", [{"eps": 1e-50}, {"eps": 1e40}, {"lr": 1e39}, {"lr": 1e38, "step": 1}, {"lr": 1e20, "weight_decay": 1e20}])
def test_constants_that_fp32_does_not_hold_are_refused(change):
    """An eps of 0 in fp32 would make NaN of every element whose gradient has always been zero; so would an infinite factor."""
    import torch
    from paper_2508_15706_amd import binding as sl
    opt = sl.sl_adamw_create([(1, 8, 0, 0)])
    theta, grad, m, v = (torch.zeros(8, device="cuda") for _ in range(4))
    theta[:] = 1.0
    p = dict(PARAMS, **change)
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_step(opt, theta, grad, m, v, **p)
    codes = [torch.zeros(16, dtype=torch.uint8, device="cuda") for _ in range(4)]
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_step8(opt, theta, grad, *codes, 1, **p)
    assert bool((theta == 1.0).all()) and not bool(m.any()) and not bool(v.any())


@pytest.mark.parametrize("change", [{"eps": 1e-40}, {"eps": 1e38}, {"lr": 0.0, "weight_decay": 1e300}, {"lr": 1e30}, {"beta1": 0.0, "beta2": 0.0}])
def test_a_gradient_that_has_always_been_zero_leaves_theta_finite(change):
    """What fp32 holds is accepted, a subnormal eps too, and 0 / eps is 0."""
    import torch
    from paper_2508_15706_amd import binding as sl
    opt = sl.sl_adamw_create([(1, 8, 0, 0)], [0.0])
    theta, grad, m, v = (torch.zeros(8, device="cuda") for _ in range(4))
    theta[:] = 1.0
    sl.sl_adamw_step(opt, theta, grad, m, v, **dict(PARAMS, **change))
    codes = [torch.zeros(16, dtype=torch.uint8, device="cuda") for _ in range(4)]
    sl.sl_adamw_step8(opt, theta, grad, *codes, 1, **dict(PARAMS, **change))
    assert bool((theta == 1.0).all())


def test_a_norm_beyond_fp32_still_clips():
    """Finite gradients whose norm only fp64 holds: 3e38 * sqrt(8) = 8.5e38.  The factor is a subnormal, to within half of 2^-149."""
    import torch
    from paper_2508_15706_amd import binding as sl
    opt = sl.sl_adamw_create([(1, 8, 0, 0)])
    grad, out = torch.full((8,), 3e38, device="cuda"), torch.empty(2, device="cuda")
    norm = float(grad[0]) * 8 ** 0.5
    sl.sl_grad_norm(opt, grad, 1.0, out, sl.alloc_norm_workspace(opt))
    assert out[0] == float("inf") and abs(float(out[1]) - 1 / norm) <= 2.0 ** -150 * (1 + 2.0 ** -20)
    sl.sl_grad_norm(opt, grad, float("inf"), out, sl.alloc_norm_workspace(opt))
    assert out.tolist() == [float("inf"), 1.0]
