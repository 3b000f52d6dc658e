"""The tensor-core products at every tile width, whole and with the contraction cut, and where a CTA pair takes one tile after
another; infinities and NaN in the gradients; tensors past 32-bit offsets in the backward pass."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2101_03961_b200 import build as sbuild
from paper_2101_03961_b200 import switch_moe as sm
from tests import operator_reference as ref
from tests.test_gpu_linear import KEY, OFFSET, Case, rng_state, within

gpu = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [sm.BF16, sm.F32], ids=["bf16", "f32"])
# M, K, N.  Together: each of the three products at each of the three widths, whole and cut, in both types (asserted below).
SHAPES = [(6212, 72, 412), (68, 3850, 2316), (80, 3566, 3336), (6404, 389, 19), (2017, 17, 1967), (1322, 18, 3472), (68, 1558, 3529),
          (4093, 17, 631), (2500, 1032, 776), (71, 1223, 17), (70, 17, 16)]


class Tiling(ctypes.Structure):
    _fields_ = [("splits", ctypes.c_int), ("width", ctypes.c_int)]


def tilings(M, K, N, dtype):
    """(splits, width) of the forward product, dx and dW, from the library's own rule (a host function)."""
    sbuild.build()
    rule = sm.load_library()._ZN5swmoe12dense_tilingENS_9DenseKindEbxxx
    rule.restype, rule.argtypes = Tiling, [ctypes.c_int, ctypes.c_bool] + [ctypes.c_longlong] * 3
    chosen = [rule(kind, dtype == sm.F32, *s) for kind, s in enumerate([(M, N, K), (M, K, N), (K, N, M)])]
    return [(t.splits, t.width) for t in chosen]


@TYPES
def test_shapes_take_every_width_whole_and_cut(dtype):
    seen = {(kind, width, splits > 1) for s in SHAPES for kind, (splits, width) in enumerate(tilings(*s, dtype))}
    assert seen == {(kind, width, cut) for kind in range(3) for width in (128, 192, 256) for cut in (False, True)}


@gpu
@TYPES
@pytest.mark.parametrize("act,residual,rate,save", [(sm.ACT_GELU, False, 0.0, True), (sm.ACT_RELU, True, 0.1, False),
                                                    (sm.ACT_GELU, True, 0.0, True)], ids=["gelu_z", "relu_drop_res", "gelu_z_res"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward_at_every_width(shape, act, residual, rate, save, dtype):
    c = Case(*shape, dtype=dtype, act=act, residual=residual, rate=rate, seed=1)
    c.forward(save=save)
    c.check_forward(saved=save)


@gpu
@TYPES
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gradients_at_every_width(shape, dtype):
    c = Case(*shape, dtype=dtype, act=sm.ACT_RELU, rate=0.1, seed=2)
    c.forward()
    c.backward()
    c.check_backward()


@gpu
@TYPES
@pytest.mark.parametrize("save,rate", [(False, 0.0), (False, 0.2), (True, 0.0)])
@pytest.mark.parametrize("shape", [(12003, 72, 763), (9003, 136, 1531), (9003, 72, 523)], ids=lambda s: "x".join(map(str, s)))
def test_residual_in_place_over_several_tiles_of_a_pair(shape, save, rate, dtype):
    """More tiles than CTA pairs, ragged on both sides: the residual of a pair's next tile is asked for while its last one's results
    leave, and both are y."""
    splits, width = tilings(*shape, dtype)[0]
    assert splits == 1 and -(-shape[0] // 256) * -(-shape[2] // width) > 74
    c = Case(*shape, dtype=dtype, act=sm.ACT_RELU, residual=True, rate=rate, seed=3)
    start = c.residual.clone()
    c.forward(save=save)
    c.check_forward(saved=save)
    y0 = c.y.clone()
    c.y.copy_(start)
    c.residual = c.y
    c.forward(save=save)
    assert torch.equal(c.y, y0)
    Case.check_outside(c.y, c.y_all)


# -------------------------------------------------------------------------------------------------- infinities and NaN
def same_kind(got, want):
    """NaN where NaN is due, and each infinity with its sign."""
    got, want = got.float().cpu(), want.float()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.isposinf(got), torch.isposinf(want)) and torch.equal(torch.isneginf(got), torch.isneginf(want))


@gpu
@TYPES
@pytest.mark.parametrize("shape", [(13, 80, 140), (60, 80, 140), (150, 80, 140), (700, 72, 2056), (2500, 1032, 776), (9000, 64, 96),
                                   (71, 1223, 17), (68, 1558, 3529)], ids=lambda s: "x".join(map(str, s)))
def test_infinities_and_nan_in_gradients_and_cut_contractions(shape, dtype):
    """An infinity or a NaN reaches the results that it is a term of and no others, in whichever part of a contraction it lies; an
    infinity of either sign in two parts is a NaN."""
    M, K, N = shape
    c = Case(M, K, N, dtype=dtype, bias=True)
    inf, nan = float("inf"), float("nan")
    c.x[3, 5], c.x[M - 1, K - 1], c.x[7, 0] = inf, -inf, nan
    c.W[K - 1, 9] = -inf
    c.W[2, N - 1] = nan
    c.dy[4, 1], c.dy[M - 2, N - 1], c.dy[M - 1, 3], c.dy[0, 3] = inf, nan, inf, -inf
    c.forward(save=False)
    c.backward()
    x, W, dy = (t.double().cpu() for t in (c.x, c.W, c.dy))
    same_kind(c.y, x @ W + c.bias.double().cpu())
    for got, a, b, depth, name in ((c.dx, dy, W.t(), N, "dx"), (c.dW, x.t(), dy, M, "dW")):
        want = a @ b
        same_kind(got, want)
        fine = torch.isfinite(want)
        a0, b0 = (torch.nan_to_num(t, 0.0, 0.0, 0.0).abs() for t in (a, b))
        bound = (2 * ref.HALF_STEP[dtype] * want.abs() + 1.01 * ref.product_error(dtype, depth) * (a0 @ b0) + 2.0**-148)[fine]
        assert bool(((got.double().cpu() - want).abs()[fine] <= bound).all()), name
    same_kind(c.db, dy.sum(0))


@gpu
@pytest.mark.parametrize("shape", [(150, 80, 140), (700, 72, 2056), (9000, 64, 96)], ids=lambda s: "x".join(map(str, s)))
def test_float32_gradients_of_very_large_values(shape):
    """Operands and sums beyond the range of the bfloat16 parts are formed again by fused multiply-adds."""
    M, K, N = shape
    c = Case(M, K, N, dtype=sm.F32, bias=False)
    c.dy[5] *= 2.0**100                                                # sums past 2^80
    c.x[:, 3] *= 2.0**106                                              # operands past 2^104
    c.W[1] *= 2.0**-60
    c.backward()
    x, W, dy = (t.double().cpu() for t in (c.x, c.W, c.dy))
    for got, a, b, depth in ((c.dx, dy, W.t(), N), (c.dW, x.t(), dy, M)):
        want = a @ b
        over = want.abs() > torch.finfo(torch.float32).max * (1 - 2.0**-12)
        # a sum of `depth` products by fused multiply-adds, or of the bfloat16 parts
        bound = (max(ref.product_error(sm.F32, depth), (depth + 32) * 2.0**-24)) * (a.abs() @ b.abs()) + 2.0**-148
        got = got.double().cpu()
        assert bool(((got - want).abs() <= bound)[~over].all())
        assert bool((torch.isinf(got) | ((got - want).abs() <= bound))[over].all())


# ------------------------------------------------------------------------------------------------------ long tensors
@gpu
@TYPES
def test_gradients_past_32_bit_offsets(dtype):
    """dy, dz and its parts of more than 2^31 elements: the last rows of dx and the last columns of dW and dbias."""
    M, K, N = 2**17 + 3, 32, 2**14 + 8
    g = torch.Generator(device="cuda").manual_seed(0)
    t, u = ref.TYPES[dtype], ref.HALF_STEP[dtype]
    x = torch.randn(M, K, device="cuda", generator=g).to(t)
    W = torch.randn(K, N, device="cuda", generator=g).to(t)
    dy = torch.randn(M, N, device="cuda", generator=g, dtype=torch.bfloat16).to(t)
    dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty(N, device="cuda")
    cfg = sm.make_linear_config(M, K, N, dtype=dtype, dropout=0.25, site=2)
    ws = sm.allocate_linear_workspace(cfg, backward=True)
    sm.switch_moe_linear_bwd(cfg, dy, x, W, None, rng_state(), ws, dx, dW, db)
    sm.switch_moe_linear_check_device_status(cfg, ws)
    scale = 2.0**-23 + (u if dtype == sm.BF16 else 2.0**-24)           # dropout's product, dz rounded
    for r0 in (0, M - 5):
        keep = ref.dropout_factors(5, N, 0.25, 2, KEY, OFFSET, row0=r0)
        dz, Ws = ref.to64(dy[r0:r0 + 5]) * keep, ref.to64(W)
        want, size = dz @ Ws.T, np.abs(dz) @ np.abs(Ws.T)
        within(dx[r0:r0 + 5], want, u * np.abs(want) + 1.01 * (ref.product_error(dtype, N) + scale) * size, "dx")
    # the last eight columns of every row: the last block of eight of each
    per_row = N // 8
    b = np.arange(1, M + 1, dtype=np.uint64) * np.uint64(per_row) - np.uint64(1)
    counter = np.stack([b & np.uint64(0xFFFFFFFF), (b >> np.uint64(32)) + np.uint64(2 << 16), np.full(M, OFFSET & 0xFFFFFFFF, np.uint64),
                        np.full(M, OFFSET >> 32, np.uint64)], axis=1)
    words = ref.philox4x32_10(counter, (KEY & 0xFFFFFFFF, KEY >> 32))
    halves = np.stack([words & 0xFFFF, words >> 16], axis=2).reshape(M, 8)
    dz = ref.to64(dy[:, N - 8:]) * np.where(halves >= 16384, 65536.0 / 49152, 0.0)
    xs = ref.to64(x)
    want, size = xs.T @ dz, np.abs(xs.T) @ np.abs(dz)
    within(dW[:, N - 8:], want, u * np.abs(want) + 1.01 * (ref.product_error(dtype, M) + scale) * size, "dW")
    within(db[N - 8:], dz.sum(0), (M * 2.0**-24 + 2.0**-23) * np.abs(dz).sum(0), "dbias")
