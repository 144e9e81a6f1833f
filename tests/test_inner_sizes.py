"""The binding of the inner step's optimiser without a GPU: what is shorter than a call needs is refused for its size."""
import pytest
import torch

from test_gpu_adamw import PARAMS

N, BLOCKS, NORM = 5000, 20, 16384


def opt():
    from paper_2508_15706_amd import binding as sl
    return sl, sl.AdamW(None, 1, N, BLOCKS, NORM)


def on_device(t):
    """A stand-in for a device tensor: the checks read its size, type and place only, and no call is made."""
    class Fake:
        is_cuda = True
        dtype = t.dtype

        def numel(self):
            return t.numel()

        def is_contiguous(self):
            return True

        def data_ptr(self):
            return 4096
    return Fake()


@pytest.mark.parametrize("short", ["grad", "result", "workspace"])
def test_norm(short):
    sl, o = opt()
    sizes = {"grad": N, "result": 2, "workspace": NORM}
    sizes[short] -= 1
    t = {k: on_device(torch.zeros(n, dtype=torch.uint8 if k == "workspace" else torch.float32)) for k, n in sizes.items()}
    with pytest.raises(ValueError, match=f"^{short} has {sizes[short]} elements, {sizes[short] + 1} are needed"):
        sl.sl_grad_norm(o, t["grad"], 1.0, t["result"], t["workspace"])


@pytest.mark.parametrize("short", ["theta", "grad", "m", "v", "grad_scale", "theta16"])
def test_step(short):
    sl, o = opt()
    sizes = {"theta": N, "grad": N, "m": N, "v": N, "grad_scale": 1, "theta16": N}
    sizes[short] -= 1
    t = {k: on_device(torch.zeros(n, dtype=torch.bfloat16 if k == "theta16" else torch.float32)) for k, n in sizes.items()}
    with pytest.raises(ValueError, match=f"^{short} has {sizes[short]} elements, {sizes[short] + 1} are needed"):
        sl.sl_adamw_step(o, t["theta"], t["grad"], t["m"], t["v"], **PARAMS, grad_scale=t["grad_scale"], theta16=t["theta16"])


@pytest.mark.parametrize("short", ["theta", "grad", "m_codes", "v_codes", "m_scales", "v_scales", "grad_scale", "theta16"])
def test_step8(short):
    sl, o = opt()
    sizes = {"theta": N, "grad": N, "m_codes": N, "v_codes": N, "m_scales": BLOCKS, "v_scales": BLOCKS, "grad_scale": 1, "theta16": N}
    sizes[short] -= 1
    types = {"theta16": torch.bfloat16, "m_codes": torch.uint8, "v_codes": torch.uint8, "m_scales": torch.uint8, "v_scales": torch.uint8}
    t = {k: on_device(torch.zeros(n, dtype=types.get(k, torch.float32))) for k, n in sizes.items()}
    with pytest.raises(ValueError, match=f"^{short} has {sizes[short]} elements, {sizes[short] + 1} are needed"):
        sl.sl_adamw_step8(o, t["theta"], t["grad"], t["m_codes"], t["v_codes"], t["m_scales"], t["v_scales"], 1, **PARAMS,
                          grad_scale=t["grad_scale"], theta16=t["theta16"])


@pytest.mark.parametrize("short", ["codes", "scales", "values"])
def test_state_values(short):
    sl, o = opt()
    sizes = {"codes": N, "scales": BLOCKS, "values": N}
    sizes[short] -= 1
    t = {k: on_device(torch.zeros(n, dtype=torch.float32 if k == "values" else torch.uint8)) for k, n in sizes.items()}
    with pytest.raises(ValueError, match=f"^{short} has {sizes[short]} elements, {sizes[short] + 1} are needed"):
        sl.sl_adamw_state_values(o, 1, t["codes"], t["scales"], t["values"])
