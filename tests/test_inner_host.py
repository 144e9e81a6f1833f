"""The inner step without a GPU: sizes and refusals of the C ABI, and the 64-bit reference that the GPU tests use against brute force."""
import os

import numpy as np
import pytest

import inner_reference as ref

HERE = os.path.dirname(os.path.abspath(__file__))


def test_sizes():
    from paper_2508_15706_amd import binding as sl
    for rows in (1, 31, 32, 33, 63, 64, 65, 1000):
        for cols in (1, 32, 127, 128, 129, 530):
            tiles = -(-cols // 128)
            assert sl.sl_mx4_bytes(rows, cols) == -(-rows // 32) * tiles * 2048 + -(-rows // 64) * tiles * 256
    assert [sl.sl_mx4_bytes(*z) for z in ((0, 1), (1, 0), (-1, 5), (1 << 27, 129), (1 << 62, 1 << 62))] == [0] * 5
    assert sl.sl_mx4_bytes(1 << 27, 128) > 0
    assert sl.sl_mx4_workspace_bytes(0, 5, 5) == sl.sl_mx4_workspace_bytes(5, 5, 0) == 0
    assert sl.sl_mx4_workspace_bytes(1, 64, 128) == 0                   # one launch, nothing to keep
    assert sl.sl_mx4_workspace_bytes(100, 64, 128) >= sl.sl_mx4_bytes(100, 128)
    assert sl.sl_mx4_workspace_bytes(1 << 20, 1 << 20, 128) == 0        # more than 2^36 elements of c: no such product


def test_refusals_before_any_device_work():
    """Pointers here are never followed: every call is refused for its sizes, types, alignment or aliases."""
    from paper_2508_15706_amd import binding as sl
    L = sl.lib()
    a, b, c, w = 4096, 8192, 16384, 32768
    assert L.sl_mx4_quantize(a, 0, 4, 4, 3, b, None, None) == -1        # ld < cols
    assert L.sl_mx4_quantize(a, 2, 4, 4, 4, b, None, None) == -1
    assert L.sl_mx4_quantize(a, 0, 4, 4, 4, None, None, None) == -1
    assert L.sl_mx4_quantize(a, 0, 4, 4, 4, b + 8, None, None) == -1
    assert L.sl_mx4_quantize(a + 2, 0, 4, 4, 4, b, None, None) == -1
    assert L.sl_mx4_quantize(a, 0, 4, 4, 4, b, b, None) == -1
    assert L.sl_mx4_quantize(None, 0, 4, 4, 4, b, None, None) == -1
    assert L.sl_mx4_quantize(a, 0, -1, 4, 4, b, None, None) == -1 and L.sl_mx4_dequantize(a, 4, -1, b, 1, 4, None) == -1
    assert L.sl_mx4_quantize(None, 0, 0, 4, 4, b, None, None) == 0 and L.sl_mx4_dequantize(a, 4, 0, None, 1, 4, None) == 0   # nothing to do
    assert L.sl_mx4_quantize(a, 0, 1 << 40, 1 << 40, 1 << 40, b, None, None) == -1
    assert L.sl_mx4_dequantize(a, 4, 4, b, 1, 3, None) == -1
    assert L.sl_mx4_dequantize(a, 4, 4, a, 1, 4, None) == -1
    assert L.sl_mx4_product(a, b, 4, 4, 32, c, 1, 4, 1, w, None) == -1   # adding to bf16
    assert L.sl_mx4_product(a, b, 4, 4, 32, a, 0, 4, 0, w, None) == -1
    assert L.sl_mx4_product(a, b, 4, 4, 32, c, 0, 3, 0, w, None) == -1
    assert L.sl_mx4_product(a, b, 100, 100, 32, c, 0, 100, 0, None, None) == -1   # no workspace
    assert L.sl_mx4_product(a, b, 1 << 20, 1 << 20, 32, c, 0, 1 << 20, 0, w, None) == -1
    assert L.sl_mx4_product(a, b, 0, 4, 32, c, 0, 4, 0, None, None) == 0
    assert L.sl_mx4_linear(a, 0, 31, b, 4, 4, 32, c, 0, 4, w, None) == -1
    assert L.sl_mx4_linear(a, 3, 32, b, 4, 4, 32, c, 0, 4, w, None) == -1
    assert L.sl_mx4_linear(a, 0, 32, b, 4, 4, 32, a, 0, 4, w, None) == -1
    assert L.sl_adamw_step(None, a, b, 0, c, w, None, None, None, None) == -1
    assert L.sl_grad_norm(None, a, 0, 1.0, b, c, None) == -1
    assert L.sl_adamw_num_blocks(None) == -1 and L.sl_adamw_destroy(None) == 0


def test_bindings_check_shapes_on_the_host():
    import torch
    from paper_2508_15706_amd import binding as sl
    with pytest.raises(ValueError):
        sl.sl_mx4_quantize(torch.zeros(4, 4), None)                      # not on a device
    with pytest.raises(ValueError):
        sl.sl_adamw_create([(1, 4, 0, 0)], [1.0, 2.0])
    with pytest.raises(sl.SparseLoCoError):
        sl.sl_adamw_create([(1, 4, 1, 0)])


def test_reference_of_4_bits():
    """Values on a fine grid around one block: nearest in E2M1 under the smallest scale that cuts nothing off, by brute force."""
    rng = np.random.default_rng(0)
    x = rng.normal(0, 1, (50, 70)) * 2.0 ** rng.integers(-20, 20, (50, 1))
    x[0] = np.arange(70) * 0.125 - 4                                     # exact ties
    codes, X, values = ref.mx4_reference(x)
    for r in range(50):
        for b in range(3):
            blk = x[r, 32 * b:32 * b + 32]
            top = np.abs(blk).max()
            s = 2.0 ** (int(X[r, b]) - 127)
            assert top <= 6 * s and (top > 3 * s or X[r, b] == 0)
            for i, v in enumerate(blk):
                allowed = [abs(v / s) - g for g in ref.GRID]
                best = min(abs(d) for d in allowed)
                got = values[r, 32 * b + i]
                assert abs(abs(got) - abs(v)) == best * s
                near = [k for k, d in enumerate(allowed) if abs(d) == best]
                assert (codes[r, 32 * b + i] & 7) == (near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1])


def test_reference_of_8_bits():
    """Every code's value, encoded again with any random part, is that code; halfway between two it goes up for half of the parts."""
    for signed, most in ((True, 127), (False, 255)):
        codes = np.arange(most + 1)
        one = np.zeros(most + 1, np.int64)
        values = ref.decode8(codes, np.array([130]), one, signed)
        assert values[-1] == 1.875 * 8 and (np.diff(values) > 0).all() and values[1] == 8 * 2.0 ** (-17 if signed else -33)
        top = np.full(most + 1, values[-1])
        for rnd in (0, 1, 65535):
            X, at = ref.encode8_positions(values, np.full(most + 1, rnd), top, signed)
            assert (X == 130).all() and np.array_equal(np.floor(at), codes)
        mid = (values[:-1] + values[1:]) / 2
        up = [np.floor(ref.encode8_positions(mid, np.full(most, r), top[:-1], signed)[1]) - codes[:-1] for r in (0, 32767, 32768, 65535)]
        assert all((u == w).all() for u, w in zip(up, (0, 0, 1, 1)))


def test_finalizer_against_published_values():
    path = os.path.join(HERE, "golden", "murmur3_vectors.txt")
    text = [line.split("#")[0].split() for line in open(path)]
    pairs = [(int(a, 0), int(b, 0)) for a, b, *rest in (t for t in text if len(t) == 2)]
    for a, b in pairs:
        assert int(ref.fmix32(a)) == b
    assert int(ref.fmix32(0)) == 0 and int(ref.fmix32(1)) == 0x514E28B7
