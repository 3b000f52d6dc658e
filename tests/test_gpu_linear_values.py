"""GELU and its derivative value by value, the negative tail among them, in every kernel that applies them."""
import math

import pytest
import torch

from paper_2101_03961_b200 import build as sbuild
from paper_2101_03961_b200 import switch_moe as sm
from tests import operator_reference as ref

gpu = pytest.mark.gpu


def phi_error(a):
    """Relative error of Phi(-a), a = |z|: the fit and its float32 evaluation (7.3e-7 up to 2, 5.2e-6 up to 6, 7.5e-5 up to 10, by
    emulation at 2 million points on the CPU) and the exponential (2^-22)."""
    return torch.where(a <= 2, 1e-6, torch.where(a <= 6, 5.5e-6, 7.6e-5)).double() + 2.0**-22


def density_error(a):
    """Relative error of phi(a) = 2^(-a^2 / 2 log2 e - 1.33): two roundings of the exponent, the exponential, one product."""
    return math.log(2.0) * 2 * 2.0**-24 * (0.7214 * a * a + 1.33) + 2.0**-22 + 2.0**-24


def values(dtype):
    """Both signs from 2^-20 to 13, every tail among them, zero and infinity; exact in the type."""
    a = torch.cat([torch.linspace(0.0, 13.0, 1300), 2.0 ** torch.linspace(-20, 0, 81), torch.tensor([0.0, 50.0, 3e38, float("inf")])])
    return torch.cat([a, -a]).to(ref.TYPES[dtype])


@gpu
@pytest.mark.parametrize("dtype", [sm.BF16, sm.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,K", [(1, 8), (16, 8), (60, 8), (200, 8), (71, 4000)])
def test_gelu_and_its_derivative_keep_their_tails(M, K, dtype):
    """z = 1 . w + 0 + ..: exactly the weights' first row.  Few rows, the tile kernel, and a contraction cut into parts."""
    sbuild.build()
    z = values(dtype)
    N = z.numel()
    t = ref.TYPES[dtype]
    x, W = torch.zeros(M, K, dtype=t, device="cuda"), torch.zeros(K, (N + 7) // 8 * 8, dtype=t, device="cuda")
    x[:, 0] = 1
    W[0, :N] = z.cuda()
    N = W.shape[1]
    z = W[0].cpu()
    cfg = sm.make_linear_config(M, K, N, dtype=dtype, activation=sm.ACT_GELU)
    ws = sm.allocate_linear_workspace(cfg, backward=True)
    y, pre, dy = (torch.zeros(M, N, dtype=t, device="cuda") for _ in range(3))
    sm.switch_moe_linear_fwd(cfg, x, W, None, None, None, y, pre, ws)
    sm.switch_moe_linear_check_device_status(cfg, ws)
    assert torch.equal(pre, pre[:1].expand(M, N)) and bool(torch.isinf(pre.cpu()[0]).eq(torch.isinf(z)).all())
    z, asked = pre[0].cpu().double(), z.double()
    assert bool(((z - asked).abs() <= ref.product_error(dtype, K) * asked.abs())[torch.isfinite(asked)].all())
    a = z.abs()
    tail = 0.5 * torch.special.erfc(a / math.sqrt(2.0))                # Phi(-a)
    lost = 8e-23                                                       # from -10 on: what GELU is there, or nothing
    small = torch.where(torch.isinf(a), 0.0, a * tail)
    want = z.clamp(min=0.0) - small
    u = ref.HALF_STEP[dtype]
    bound = (1 + u) * (small * phi_error(a) + 2.0**-24 * want.abs() + lost) + u * want.abs()
    got = y.cpu().double()
    finite = torch.isfinite(want)
    bad = finite & ~((got - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), z[bad[0]][:4], got[0][bad[0]][:4], want[bad[0]][:4])
    assert bool((got[:, ~finite] == float("inf")).all())

    # the derivative, through the bias gradient of one row: float32, one term, the others 0
    dy[M // 2] = 1
    db = torch.full((N,), 7.0, device="cuda")
    sm.switch_moe_linear_bwd(cfg, dy, x, W, pre, None, ws, None, None, db)
    sm.switch_moe_linear_check_device_status(cfg, ws)
    slope = torch.where(torch.isinf(a), 0.0, a * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi))
    w = tail - slope                                                   # GELU'(-a)
    want = torch.where(z > 0, 1 - w, w)
    bound = tail * phi_error(a) + slope * density_error(a.clamp(max=100.0)) + 2.0**-23 * want.abs() + 2.0**-24 * w.abs() + 10 * lost
    bad = ~((db.cpu().double() - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), z[bad][:4], db.cpu()[bad][:4], want[bad][:4])


def test_saved_pre_activations_on_top_of_the_output_or_the_residual_are_refused():
    """Both are written, or read, in the same pass: z would take y's place or be added as the residual."""
    sbuild.build()
    lib = sm.load_library()
    cfg = sm.make_linear_config(32, 64, 72, activation=sm.ACT_GELU)
    n = sm.switch_moe_linear_workspace_bytes(cfg)
    call = lambda res, y, pre: lib.switch_moe_linear_fwd(cfg, 16, 32, None, res, None, y, pre, 1024, n, None)
    assert call(None, 48, 48) == sm.INVALID_ARGUMENT
    assert call(64, 48, 64) == sm.INVALID_ARGUMENT
    assert call(48, 48, 48) == sm.INVALID_ARGUMENT


@gpu
@pytest.mark.parametrize("act,rate", [(sm.ACT_GELU, 0.0), (sm.ACT_NONE, 0.3), (sm.ACT_GELU, 0.3)], ids=["gelu", "drop", "gelu_drop"])
@pytest.mark.parametrize("M", [1, 2, 9, 40, 64])
def test_weight_gradient_of_few_rows_takes_dz_unrounded(M, act, rate):
    """bfloat16, the kernel that forms dz itself and multiplies it in float32: one rounding of each result, none of dz."""
    sbuild.build()
    K, N, key = 72, 200, 1234567
    g = torch.Generator(device="cuda").manual_seed(M)
    x, W, dy, z = (torch.randn(*s, device="cuda", generator=g).bfloat16() for s in ((M, K), (K, N), (M, N), (M, N)))
    dW, db = torch.empty_like(W), torch.empty(N, device="cuda")
    rng = torch.tensor([key, 3], device="cuda")
    cfg = sm.make_linear_config(M, K, N, activation=act, dropout=rate, site=4)
    ws = sm.allocate_linear_workspace(cfg, backward=True)
    sm.switch_moe_linear_bwd(cfg, dy, x, W, z, rng, ws, None, dW, db)
    sm.switch_moe_linear_check_device_status(cfg, ws)
    dz = ref.to64(dy) * ref.dropout_factors(M, N, rate, 4, key, 3) * ref.d_act(ref.to64(z), act)
    xs = ref.to64(x)
    want, size = xs.T @ dz, abs(xs).T @ abs(dz)
    # dz: the mask's scale and product 2^-23, GELU' 1e-6 of its terms (up to 0.5 each) and one product; sums of M products
    slope = 1e-6 * (abs(xs).T @ abs(ref.to64(dy))) / (1 - rate) if act else 0.0
    bound = 2.0**-8 * abs(want) + 1.01 * ((M + 4) * 2.0**-23 * size + slope)
    bad = abs(ref.to64(dW) - want) > bound
    assert not bad.any(), (int(bad.sum()), bad.size)
