"""Dropout from a counter: the generator's published vectors, masks and values against numpy, ragged rows, refusals."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2101_03961_b200 import build as sbuild
from paper_2101_03961_b200 import switch_moe as sm
from tests import operator_reference as ref

gpu = pytest.mark.gpu
KEY, OFFSET = 0x7FEDCBA987654321, 0x00000001FFFFFFFF


def test_reference_generator_gives_the_published_vectors():
    """Known answers of philox4x32-10 from the paper's own library."""
    ones = 0xFFFFFFFF
    for counter, key, want in [
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((ones,) * 4, (ones,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
             (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]:
        assert tuple(int(v) for v in ref.philox4x32_10(np.array([counter], np.uint64), key)[0]) == want


def run(rows, cols, rate, dtype, residual, pad=0, site=3, seed=0):
    sbuild.build()
    r = np.random.default_rng(seed)
    x, _ = ref.rows_tensor(r.standard_normal((rows, cols)), dtype, pad)
    res, _ = ref.rows_tensor(r.standard_normal((rows, cols)), dtype, pad)
    y, y_all = ref.rows_tensor(np.full((rows, cols), 7.0), dtype, pad, fill=5.0)
    rng = torch.tensor([KEY, OFFSET], dtype=torch.int64, device="cuda")
    cfg = sm.make_dropout_config(rows, cols, rate, dtype=dtype, site=site, ld=x.stride(0))
    sm.switch_moe_dropout_fwd(cfg, x, res if residual else None, rng, y)
    torch.cuda.synchronize()
    return cfg, x, res, rng, y, y_all


@gpu
@pytest.mark.parametrize("dtype", [sm.BF16, sm.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,rate,pad", [(1, 1, 0.5, 0), (1, 8, 0.1, 0), (3, 7, 0.9, 8), (33, 203, 0.1, 0), (64, 768, 0.1, 16),
                                                (1000, 264, 0.4, 0), (7, 4099, 0.05, 24), (5000, 9, 0.3, 0), (16, 64, 0.0, 0),
                                                (16, 64, 1e-6, 0), (16, 64, 0.99998, 0)])
@pytest.mark.parametrize("residual", [False, True])
def test_values_and_masks(rows, cols, rate, pad, residual, dtype):
    cfg, x, res, rng, y, y_all = run(rows, cols, rate, dtype, residual, pad)
    factor = ref.dropout_factors(rows, cols, rate, 3, KEY, OFFSET)
    u = ref.HALF_STEP[dtype]
    want = ref.to64(x) * factor
    slack = 2.0**-23 * np.abs(want)                                    # the scale and the product, one float32 rounding each
    if residual:
        want = want + ref.to64(res)
        slack = slack + 2.0**-24 * np.abs(want)
    assert np.all(np.abs(ref.to64(y) - want) <= u * np.abs(want) + (1 + u) * slack)
    assert bool((y_all[:, cols:] == 5.0).all())
    dx = torch.empty_strided((rows, cols), (x.stride(0), 1), dtype=x.dtype, device="cuda")
    sm.switch_moe_dropout_bwd(cfg, x, rng, dx)
    plain = torch.empty_strided((rows, cols), (x.stride(0), 1), dtype=x.dtype, device="cuda")
    sm.switch_moe_dropout_fwd(cfg, x, None, rng, plain)
    assert torch.equal(dx, plain)


@gpu
def test_dropped_values_do_not_matter_and_in_place():
    cfg, x, res, rng, y, _ = run(40, 72, 0.5, sm.BF16, True)
    drop = torch.from_numpy(ref.dropout_factors(40, 72, 0.5, 3, KEY, OFFSET) == 0).cuda()
    bad = x.clone()
    bad[drop] = float("nan")
    bad[drop & (torch.rand(40, 72, device="cuda") < 0.5)] = float("inf")
    out = torch.empty_like(y)
    sm.switch_moe_dropout_fwd(cfg, bad, res, rng, out)
    assert torch.equal(out, y)
    for at in (x.clone(), res.clone()):                                # y may be x or residual
        first = at if torch.equal(at, x) else x
        sm.switch_moe_dropout_fwd(cfg, first, at if first is x else res, rng, at)
        assert torch.equal(at, y)


@gpu
def test_sites_offsets_and_rates_differ():
    masks = []
    for site, key, offset in [(0, 1, 0), (1, 1, 0), (65535, 1, 0), (0, 2, 0), (0, 1, 1), (0, 1, 1 << 32), (0, 1 << 32, 0)]:
        x, y = torch.ones(256, 256, device="cuda"), torch.empty(256, 256, device="cuda")
        cfg = sm.make_dropout_config(256, 256, 0.25, dtype=sm.F32, site=site)
        sm.switch_moe_dropout_fwd(cfg, x, None, torch.tensor([key, offset], device="cuda"), y)
        assert np.array_equal(ref.to64(y) > 0, ref.dropout_factors(256, 256, 0.25, site, key, offset) > 0)
        masks.append(y > 0)
        # 65536 draws of rate 1/4: 16384 dropped with a standard deviation of 111
        assert abs(int((y == 0).sum()) - 16384) < 6 * 111
    for i in range(len(masks)):
        for j in range(i):
            # independent masks agree in 1 - 2 . 3/16 = 5/8 of the places, standard deviation 124
            assert abs(int((masks[i] == masks[j]).sum()) - 40960) < 6 * 124


@gpu
def test_rows_past_32_bit_offsets():
    rows, cols = 2**20 + 5, 4104                                       # 2^32 elements and more
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    rng = torch.tensor([KEY, OFFSET], dtype=torch.int64, device="cuda")
    cfg = sm.make_dropout_config(rows, cols, 0.5)
    sm.switch_moe_dropout_fwd(cfg, x, None, rng, x)
    for r0 in (0, rows - 7):
        want = ref.dropout_factors(7, cols, 0.5, 0, KEY, OFFSET, row0=r0)
        assert np.array_equal(ref.to64(x[r0:r0 + 7]), want)


@pytest.fixture(scope="module")
def lib():
    sbuild.build()
    return sm.load_library()


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), sm.INVALID_ARGUMENT), (dict(cols=0), sm.INVALID_ARGUMENT), (dict(ld=63), sm.INVALID_ARGUMENT),
    (dict(ld=-64), sm.INVALID_ARGUMENT), (dict(dtype=5), sm.INVALID_ARGUMENT), (dict(site=65536), sm.INVALID_ARGUMENT),
    (dict(rate=1.0), sm.INVALID_ARGUMENT), (dict(rate=float("nan")), sm.INVALID_ARGUMENT), (dict(rate=-0.5), sm.INVALID_ARGUMENT),
    (dict(cols=60), sm.UNSUPPORTED_SHAPE), (dict(ld=68), sm.UNSUPPORTED_SHAPE),
    (dict(rows=2**30 + 1), sm.UNSUPPORTED_SHAPE), (dict(cols=2**30 + 64), sm.UNSUPPORTED_SHAPE), (dict(rows=0), sm.OK),
])
def test_bad_configs_are_refused(lib, kw, status):
    cfg = sm.make_dropout_config(**{**dict(rows=32, cols=64, rate=0.1), **kw})
    if status == sm.OK:
        assert lib.switch_moe_dropout_fwd(ctypes.byref(cfg), None, None, None, None, None) == sm.OK
        return
    assert lib.switch_moe_dropout_fwd(ctypes.byref(cfg), 16, 16, 16, 16, None) == status
    assert lib.switch_moe_dropout_bwd(ctypes.byref(cfg), 16, 16, 16, None) == status


def test_bad_pointers_are_refused(lib):
    c = ctypes.byref(sm.make_dropout_config(32, 64, 0.1))
    assert lib.switch_moe_dropout_fwd(c, None, None, 16, 16, None) == sm.INVALID_ARGUMENT
    assert lib.switch_moe_dropout_fwd(c, 16, None, None, 16, None) == sm.INVALID_ARGUMENT
    assert lib.switch_moe_dropout_fwd(c, 16, None, 16, None, None) == sm.INVALID_ARGUMENT
    for at in range(4):
        args = [16, 16, 16, 16]
        args[at] = 20
        assert lib.switch_moe_dropout_fwd(c, *args, None) == sm.UNSUPPORTED_SHAPE
    assert lib.switch_moe_dropout_bwd(None, 16, 16, 16, None) == sm.INVALID_ARGUMENT
    with pytest.raises(sm.SwitchMoeError):
        sm.switch_moe_dropout_fwd(sm.make_dropout_config(4, 64, 0.1), torch.zeros(4, 64), None, None, None)
