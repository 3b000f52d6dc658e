"""The balance loss, its counts and its gradient against float64: types, layouts, masks, choices, odd values, refusals."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2101_03961_b200 import build as sbuild
from paper_2101_03961_b200 import switch_moe as sm
from tests import operator_reference as ref

gpu = pytest.mark.gpu


def call(logits, index=None, mask=None, k=1, groups=1, alpha=0.01, d_loss=1.0, dtype=sm.F32, ld=0, in_place=False):
    sbuild.build()
    T, E = logits.shape
    cfg = sm.make_balance_config(T, E, k=k, groups=groups, alpha=alpha, dtype=dtype, ld=ld)
    ws = sm.allocate_balance_workspace(cfg)
    ws.fill_(0xFF)
    loss = torch.full((1,), 7.0, device="cuda")
    counts = torch.full((groups, E), -7, dtype=torch.int32, device="cuda")
    tokens = torch.full((groups,), -7, dtype=torch.int32, device="cuda")
    sm.switch_moe_balance_fwd(cfg, logits, index, mask, loss, counts, tokens, ws)
    dl = logits if in_place else torch.full((T, ld or E), 5.0, dtype=logits.dtype, device="cuda")[:, :E]
    sm.switch_moe_balance_bwd(cfg, logits, mask, counts, tokens, d_loss, dl)
    torch.cuda.synchronize()
    return loss, counts, tokens, dl


def check(logits, index=None, mask=None, k=1, groups=1, alpha=0.01, d_loss=1.0, dtype=sm.F32, **kw):
    want = ref.balance(ref.to64(logits), None if index is None else index.cpu().numpy(), None if mask is None else mask.cpu().numpy(),
                       k, groups, alpha, d_loss)
    loss, counts, tokens, dl = call(logits, index, mask, k, groups, alpha, d_loss, dtype, **kw)
    assert np.array_equal(counts.cpu().numpy(), want[1]) and np.array_equal(tokens.cpu().numpy(), want[2])
    # a probability: the exponent's argument (up to 2^-24 of 30), exp (2 ulp), sum and quotient: 2^-19 relative; float32 sums of
    # one lane's probabilities, up to T / 64 of them, and of 8 warps
    T, E = logits.shape
    tol = 2.0**-19 + (T / 64 + 16) * 2.0**-24
    assert abs(float(loss) - want[0]) <= tol * abs(want[0]) + 1e-30
    grad, got = want[3], ref.to64(dl)
    # p (g - <p, g>): both terms up to p max|g|, each probability off by 2^-19
    per = max(1, T // groups)
    n = np.maximum(want[2], 1)
    gmax = np.repeat(np.abs(d_loss) * alpha * E / groups / n * (want[1].max(1) / (k * n)), per)[:, None]
    lg = ref.to64(logits)
    with np.errstate(invalid="ignore", over="ignore"):
        p = np.exp(lg - lg.max(1, keepdims=True))
        p = np.nan_to_num(p / p.sum(1, keepdims=True))
    u = ref.HALF_STEP[dtype]
    bound = u * np.abs(grad) + 4 * 2.0**-19 * p * gmax + 2.0**-133
    assert np.all(np.abs(got - grad) <= bound), (np.abs(got - grad) - bound).max()
    return loss, counts, tokens, dl


def randn(*s, seed=0, dtype=sm.F32):
    return torch.randn(*s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(ref.TYPES[dtype])


@gpu
@pytest.mark.parametrize("dtype", [sm.F32, sm.BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,E,k,groups", [(1, 1, 1, 1), (1, 8, 1, 1), (3, 2, 2, 1), (64, 5, 3, 4), (513, 8, 1, 1), (200, 33, 2, 2),
                                          (300, 64, 2, 3), (1000, 128, 1, 1), (640, 200, 4, 32), (500, 256, 8, 1), (96, 511, 2, 1),
                                          (70, 512, 16, 1), (60, 1000, 1, 2), (33, 1024, 2, 1), (65, 1023, 16, 1)])
def test_loss_counts_and_gradient(T, E, k, groups, dtype):
    logits = randn(T, E, seed=T + E, dtype=dtype)
    check(logits, k=k, groups=groups, dtype=dtype)
    mask = (torch.arange(T, device="cuda") * 7 % 5 < 3)
    check(logits, mask=mask.to(torch.uint8), k=k, groups=groups, dtype=dtype, alpha=0.3, d_loss=-2.5)
    index = torch.randint(-2, E + 2, (T, k), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(1))
    check(logits, index=index, mask=mask, k=k, groups=groups, dtype=dtype)


@gpu
@pytest.mark.parametrize("dtype", [sm.F32, sm.BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("E", [8, 6, 129, 256])
def test_rows_at_a_distance_and_misaligned(E, dtype):
    for ld, off in ((E + 3, 0), (E + 8, 8), (E + 8, 1)):
        whole = torch.full((90 * ld + 16,), float("nan"), dtype=ref.TYPES[dtype], device="cuda")
        logits = whole[off:off + 90 * ld].view(90, ld)[:, :E]
        logits.copy_(randn(90, E, dtype=dtype))
        dl = check(logits, k=min(2, E), dtype=dtype, ld=ld)[3].clone()
        assert torch.equal(call(logits, k=min(2, E), dtype=dtype, ld=ld, in_place=True)[3], dl)
        assert bool(torch.isnan(whole[off:off + 90 * ld].view(90, ld)[:, E:]).all())


@gpu
@pytest.mark.parametrize("E", [7, 64, 300])
def test_ties_masked_experts_and_empty_rows(E):
    logits = torch.zeros(40, E, device="cuda")
    logits[1] = -torch.finfo(torch.float32).max                        # a mask of the type's lowest value, everywhere
    logits[2] = float("-inf")                                          # a row that leaves nothing
    logits[3, 1:] = float("-inf")                                      # fewer experts left than choices
    logits[4, E - 2:] = 3.0
    logits[5] = torch.arange(E, device="cuda") % 3                     # ties in the middle
    logits[6, :E // 2] = -torch.finfo(torch.float32).max
    loss, counts, tokens, dl = check(logits, k=2)
    assert int(tokens) == 39 and int(counts.sum()) == 2 * 39 - 1
    assert not dl[2].any()


@gpu
def test_values_in_padded_rows_do_not_matter():
    logits = randn(100, 24)
    mask = torch.ones(100, dtype=torch.uint8, device="cuda")
    mask[50:] = 0
    clean = call(logits, mask=mask, k=2)
    logits[60], logits[70], logits[80, 3], logits[99] = float("nan"), float("inf"), float("nan"), float("-inf")
    for a, b in zip(clean, call(logits, mask=mask, k=2)):
        assert torch.equal(a, b)
    logits[10, 3] = float("nan")                                       # .. and a NaN in a row that counts shows
    loss, counts, tokens, dl = call(logits, mask=mask, k=2)
    assert torch.isnan(loss).all() and torch.isnan(dl[10]).all() and not torch.isnan(dl[11]).any()
    assert int(counts.sum()) == 100 and int(tokens) == 50


@gpu
def test_groups_without_tokens_and_empty_calls():
    logits = randn(64, 16)
    mask = torch.ones(64, dtype=torch.bool, device="cuda")
    mask[16:32] = False
    check(logits, mask=mask, groups=4)
    loss, counts, tokens, dl = call(logits, mask=torch.zeros(64, dtype=torch.bool, device="cuda"), groups=4)
    assert float(loss) == 0.0 and not counts.any() and not tokens.any() and not dl.any()
    cfg = sm.make_balance_config(0, 16)
    ws = sm.allocate_balance_workspace(cfg)
    loss, counts, tokens = torch.full((1,), 7.0, device="cuda"), torch.full((1, 16), 7, dtype=torch.int32, device="cuda"), \
        torch.full((1,), 7, dtype=torch.int32, device="cuda")
    empty = torch.empty(0, 16, device="cuda")
    sm.switch_moe_balance_fwd(cfg, empty, None, None, loss, counts, tokens, ws)
    sm.switch_moe_balance_bwd(cfg, empty, None, counts, tokens, 1.0, empty)
    assert float(loss) == 0.0 and not counts.any() and not tokens.any()


@gpu
@pytest.mark.parametrize("groups", [1, 5])
def test_long_batches_repeat_bit_for_bit(groups):
    logits = randn(100000, 96)
    a, b = call(logits, k=2, groups=groups), call(logits, k=2, groups=groups)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    p = torch.softmax(logits.double().view(groups, -1, 96), -1)
    top = torch.topk(logits.view(groups, -1, 96), 2)[1].reshape(groups, -1)
    counts = torch.stack([torch.bincount(t, minlength=96) for t in top])
    assert torch.equal(a[1].long(), counts)
    n = 100000 // groups
    want = float((0.01 * 96 * (counts / (2 * n) * p.mean(1)).sum(-1)).mean())
    assert abs(float(a[0]) - want) <= (2.0**-19 + 16 * 2.0**-20) * want


@gpu
def test_gradient_against_differences():
    """f stands still (it carries no gradient): the loss in the probabilities alone."""
    logits = randn(40, 12, seed=3)
    loss, counts, tokens, dl = call(logits, k=2, groups=2, alpha=0.7)
    f = counts.cpu().double().numpy() / (2 * 20)
    def value(l):
        e = np.exp(l - l.max(1, keepdims=True))
        p = (e / e.sum(1, keepdims=True)).reshape(2, 20, 12)
        return float(np.mean(0.7 * 12 * (f * p.mean(1)).sum(1)))
    l0, r = ref.to64(logits), np.random.default_rng(0)
    for _ in range(5):
        v = r.standard_normal(l0.shape)
        want = (value(l0 + 1e-5 * v) - value(l0 - 1e-5 * v)) / 2e-5
        # rounding of the difference: 1e-16 / 1e-5; float32 gradients: 1e-5 of the terms
        assert abs(float((ref.to64(dl) * v).sum()) - want) <= 1e-10 + 1e-5 * float(np.abs(ref.to64(dl) * v).sum())


@gpu
@pytest.mark.parametrize("E,dtype", [(2, sm.F32), (4, sm.BF16), (9, sm.F32)])
def test_every_expert_chosen_leaves_no_gradient(E, dtype):
    """k = E: f is 1 / E for every expert, the loss alpha whatever the router does."""
    loss, counts, tokens, dl = call(randn(300, E, dtype=dtype), k=E, groups=3, dtype=dtype)
    assert bool((counts == 100).all()) and not dl.any()
    assert abs(float(loss) - 0.01) <= 0.01 * (2.0**-19 + 24 * 2.0**-24)


@gpu
def test_the_layer_and_this_loss_agree():
    """The layer's own auxiliary loss, from the probabilities' logits and its expert indices."""
    from paper_2101_03961_b200 import inputs as si
    from tests.gpu_helpers import GpuLayer
    scfg = si.SwitchConfig("agree", 1024, 128, 256, 16, 1.25, bias_std=0.3, dtype=si.DTYPE_F32)
    layer = GpuLayer(scfg, si.gen_layer(scfg, seed=1))
    y, aux = torch.empty_like(layer.x), torch.zeros(1, device="cuda")
    sm.switch_moe_fwd(layer.cfg, layer.x, layer.W_r, layer.bias, layer.W_in, layer.W_out, y, aux, layer.ws)
    probs = sm.switch_moe_workspace_view(layer.cfg, layer.ws, sm.WS_PROBS).view(1024, 16)
    index = sm.switch_moe_workspace_view(layer.cfg, layer.ws, sm.WS_EXPERT_INDEX)
    loss, counts, _, _ = call(torch.log(probs), index=index, alpha=scfg.alpha)
    assert torch.equal(counts[0], sm.switch_moe_workspace_view(layer.cfg, layer.ws, sm.WS_COUNT))
    assert abs(float(loss) - float(aux)) <= 1e-5 * float(aux)


@pytest.fixture(scope="module")
def lib():
    sbuild.build()
    return sm.load_library()


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), sm.INVALID_ARGUMENT), (dict(E=0), sm.INVALID_ARGUMENT), (dict(k=0), sm.INVALID_ARGUMENT), (dict(k=9), sm.INVALID_ARGUMENT),
    (dict(groups=3), sm.INVALID_ARGUMENT), (dict(groups=-1), sm.INVALID_ARGUMENT), (dict(dtype=2), sm.INVALID_ARGUMENT),
    (dict(ld=7), sm.INVALID_ARGUMENT), (dict(ld=-8), sm.INVALID_ARGUMENT), (dict(alpha=float("nan")), sm.INVALID_ARGUMENT),
    (dict(E=1025), sm.UNSUPPORTED_SHAPE), (dict(E=64, k=17), sm.UNSUPPORTED_SHAPE), (dict(T=2**30, groups=2**17), sm.UNSUPPORTED_SHAPE),
    (dict(T=2**30, k=2), sm.UNSUPPORTED_SHAPE), (dict(T=2**30 + 1), sm.UNSUPPORTED_SHAPE),
])
def test_bad_configs_are_refused(lib, kw, status):
    cfg = ctypes.byref(sm.make_balance_config(**{**dict(T=64, E=8), **kw}))
    out = ctypes.c_size_t(0)
    assert lib.switch_moe_balance_workspace_bytes(cfg, ctypes.byref(out)) == status
    assert lib.switch_moe_balance_fwd(cfg, 16, None, None, 16, 16, 16, 1024, 1 << 30, None) == status
    assert lib.switch_moe_balance_bwd(cfg, 16, None, 16, 16, 1.0, 16, None) == status


def test_bad_arguments_are_refused(lib):
    cfg = sm.make_balance_config(64, 8)
    n = sm.switch_moe_balance_workspace_bytes(cfg)
    for at in (0, 3, 4, 5, 6):
        args = [16, None, None, 16, 16, 16, 1024]
        args[at] = None
        assert lib.switch_moe_balance_fwd(ctypes.byref(cfg), *args, n, None) == sm.INVALID_ARGUMENT
    assert lib.switch_moe_balance_fwd(ctypes.byref(cfg), 16, None, None, 16, 16, 16, 1024, n - 1, None) == sm.WORKSPACE_TOO_SMALL
    assert lib.switch_moe_balance_fwd(ctypes.byref(cfg), 18, None, None, 16, 16, 16, 1024, n, None) == sm.UNSUPPORTED_SHAPE
    assert lib.switch_moe_balance_fwd(ctypes.byref(cfg), 16, None, None, 16, 16, 16, 1040, n, None) == sm.UNSUPPORTED_SHAPE
    for at in (0, 2, 3, 5):
        args = [16, None, 16, 16, 1.0, 16]
        args[at] = None
        assert lib.switch_moe_balance_bwd(ctypes.byref(cfg), *args, None) == sm.INVALID_ARGUMENT
    assert lib.switch_moe_balance_bwd(None, 16, None, 16, 16, 1.0, 16, None) == sm.INVALID_ARGUMENT
    with pytest.raises(sm.SwitchMoeError):
        sm.switch_moe_balance_fwd(cfg, torch.zeros(64, 9), None, None, None, None, None, None)
