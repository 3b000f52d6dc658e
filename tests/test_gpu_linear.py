"""The dense product with its epilogue and its gradients against float64, over types, shapes, distances between rows, activations,
dropout, residual; rows and columns outside a call's tensors; refusals."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2101_03961_b200 import build as sbuild
from paper_2101_03961_b200 import switch_moe as sm
from tests import operator_reference as ref

gpu = pytest.mark.gpu
KEY, OFFSET = 0x1234567890ABCDEF, 0x0FEDCBA987654321


def rng_state(key=KEY, offset=OFFSET):
    return torch.tensor([key, offset], dtype=torch.int64, device="cuda")


class Case:
    def __init__(self, M, K, N, dtype=sm.BF16, act=sm.ACT_NONE, bias=True, residual=False, rate=0.0, pad=0, seed=0, site=9):
        sbuild.build()
        r = np.random.default_rng(seed)
        rnd = lambda *s: r.standard_normal(s)
        self.M, self.K, self.N, self.dtype, self.act, self.rate, self.site = M, K, N, dtype, act, rate, site
        self.x, _ = ref.rows_tensor(rnd(M, K), dtype, pad)
        self.W, _ = ref.rows_tensor(rnd(K, N) / np.sqrt(K), dtype, pad)
        self.dy, _ = ref.rows_tensor(rnd(M, N), dtype, pad)
        self.residual = ref.rows_tensor(rnd(M, N), dtype, pad)[0] if residual else None
        self.bias = torch.from_numpy(rnd(N)).float().cuda() if bias else None
        self.y, self.y_all = ref.rows_tensor(np.full((M, N), 7.0), dtype, pad, fill=5.0)
        self.pre, self.pre_all = ref.rows_tensor(np.full((M, N), 7.0), dtype, pad, fill=5.0)
        self.dx, self.dx_all = ref.rows_tensor(np.full((M, K), 7.0), dtype, pad, fill=5.0)
        self.dW, self.dW_all = ref.rows_tensor(np.full((K, N), 7.0), dtype, pad, fill=5.0)
        self.db = torch.full((N,), 7.0, device="cuda") if bias else None
        self.rng = rng_state() if rate else None
        ld = lambda t: t.stride(0)
        self.cfg = sm.make_linear_config(M, K, N, dtype=dtype, activation=act, dropout=rate, site=site, ldx=ld(self.x), ldw=ld(self.W),
                                         ldy=ld(self.y))
        self.ws = sm.allocate_linear_workspace(self.cfg, backward=True)
        self.ws.fill_(0xFF)

    def forward(self, save=True):
        sm.switch_moe_linear_fwd(self.cfg, self.x, self.W, self.bias, self.residual, self.rng, self.y, self.pre if save else None,
                                 self.ws)
        sm.switch_moe_linear_check_device_status(self.cfg, self.ws)

    def backward(self):
        sm.switch_moe_linear_bwd(self.cfg, self.dy, self.x, self.W, self.pre if self.act else None, self.rng, self.ws, self.dx,
                                 self.dW, self.db)
        sm.switch_moe_linear_check_device_status(self.cfg, self.ws)

    def check_forward(self, saved=True):
        u = ref.HALF_STEP[self.dtype]
        x, W = ref.to64(self.x), ref.to64(self.W)
        z = x @ W
        dz = ref.product_error(self.dtype, self.K) * (np.abs(x) @ np.abs(W)) + 2.0**-148
        if self.bias is not None:
            b = ref.to64(self.bias)
            z = z + b
            dz = dz + 2.0**-24 * np.abs(z)
        if saved:
            within(self.pre, z, u * np.abs(z) + (1 + u) * dz, "pre")
        h = ref.act(z, self.act)
        dh = (1.13 if self.act == sm.ACT_GELU else 1.0) * dz           # the largest slope of GELU is below 1.13
        if self.act == sm.ACT_GELU:
            dh = dh + ref.GELU_ERROR * np.abs(z) + 2.0**-23 * np.abs(h)
        keep = ref.dropout_factors(self.M, self.N, self.rate, self.site, KEY, OFFSET)
        h, dh = h * keep, dh * keep + 2.0**-23 * np.abs(h * keep)
        if self.residual is not None:
            h = h + ref.to64(self.residual)
            dh = dh + 2.0**-24 * np.abs(h)
        within(self.y, h, u * np.abs(h) + (1 + u) * dh, "y")
        if self.residual is None:
            assert not self.y[torch.from_numpy(keep == 0).cuda()].any()
        self.check_outside(self.y, self.y_all)
        self.check_outside(self.pre, self.pre_all)

    def check_backward(self):
        u = ref.HALF_STEP[self.dtype]
        keep = ref.dropout_factors(self.M, self.N, self.rate, self.site, KEY, OFFSET)
        g = ref.to64(self.dy) * keep
        dg = 2.0**-23 * np.abs(g) * (self.rate > 0)
        if self.act:
            d = ref.d_act(ref.to64(self.pre), self.act)
            dg = dg * np.abs(d) + np.abs(g) * (2 * ref.GELU_ERROR if self.act == sm.ACT_GELU else 0) + 2.0**-24 * np.abs(g * d)
            g = g * d
        if self.db is not None:                                        # sums of M terms: one rounding per addition
            within(self.db, g.sum(0), dg.sum(0) + (self.M + 8) * 2.0**-24 * np.abs(g).sum(0) + 2.0**-148, "dbias")
        if self.act or self.rate:                                      # the products take dz in the activation type
            dg = dg + u * np.abs(g)
        x, W = ref.to64(self.x), ref.to64(self.W)
        for got, a, b, da, db, K, name in ((self.dx, g, W.T, dg, 0 * W.T, self.N, "dx"), (self.dW, x.T, g, 0 * x.T, dg, self.M, "dW")):
            want = a @ b
            err = ref.product_error(self.dtype, K) * ((np.abs(a) + da) @ (np.abs(b) + db)) + da @ np.abs(b) + np.abs(a) @ db
            within(got, want, u * np.abs(want) + (1 + u) * err + 2.0**-148, name)
        self.check_outside(self.dx, self.dx_all)
        self.check_outside(self.dW, self.dW_all)

    @staticmethod
    def check_outside(t, whole):
        """What lies between rows is left as it was."""
        assert bool((whole[:, t.shape[1]:] == 5.0).all())


def within(got, want, bound, name):
    got = ref.to64(got)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (name, int(bad.sum()), [int(i) for i in np.argwhere(bad)[0]], got[bad][:3], want[bad][:3], bound[bad][:3])


SHAPES = [(1, 8, 8), (1, 768, 520), (2, 64, 136), (3, 100, 7), (17, 65, 33), (48, 512, 256), (127, 96, 260), (129, 64, 129),
          (255, 200, 512), (257, 320, 264), (300, 1000, 1), (512, 17, 1000), (1000, 640, 384), (5, 1, 300), (700, 72, 2056)]


@gpu
@pytest.mark.parametrize("dtype", [sm.BF16, sm.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_plain_product_and_gradients(shape, dtype):
    c = Case(*shape, dtype=dtype, bias=shape[0] % 2 == 0, pad=8 * (shape[0] % 3))
    c.forward(save=False)
    c.check_forward(saved=False)
    c.backward()
    c.check_backward()


@gpu
@pytest.mark.parametrize("dtype", [sm.BF16, sm.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 4, 5, 8, 9, 16, 17, 32, 33, 63, 64, 65])
@pytest.mark.parametrize("K,N", [(65, 200), (1000, 65), (2048, 24), (24, 2051)])
def test_few_rows(M, K, N, dtype):
    """Both sides of each limit of the kernel for few rows: odd depths and widths, one slice of the contraction and eight."""
    c = Case(M, K, N, dtype=dtype, act=sm.ACT_GELU, residual=M % 2 == 1, rate=0.2 * (M % 3 == 0), pad=8, seed=M)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@gpu
@pytest.mark.parametrize("dtype", [sm.BF16, sm.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("act", [sm.ACT_NONE, sm.ACT_RELU, sm.ACT_GELU], ids=["none", "relu", "gelu"])
@pytest.mark.parametrize("residual,rate", [(False, 0.0), (True, 0.0), (False, 0.4), (True, 0.1)])
@pytest.mark.parametrize("shape", [(1, 64, 72), (33, 40, 203), (300, 136, 392), (5, 256, 24)], ids=lambda s: "x".join(map(str, s)))
def test_epilogues_and_gradients(shape, dtype, act, residual, rate):
    c = Case(*shape, dtype=dtype, act=act, residual=residual, rate=rate, pad=16)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@gpu
@pytest.mark.parametrize("dtype", [sm.BF16, sm.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(4100, 256, 512), (2500, 1032, 776), (9000, 64, 96)], ids=lambda s: "x".join(map(str, s)))
def test_many_tiles_and_a_split_contraction(shape, dtype):
    c = Case(*shape, dtype=dtype, act=sm.ACT_GELU, residual=True, rate=0.1, seed=3)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@gpu
@pytest.mark.parametrize("dtype", [sm.BF16, sm.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(4100, 520, 1400), (300, 1400, 2000), (4100, 1000, 520), (1500, 1160, 2000)], ids=lambda s: "x".join(map(str, s)))
def test_tile_widths(shape, dtype):
    """Shapes for which each of the three products takes each of the three tile widths, split or not."""
    c = Case(*shape, dtype=dtype, act=sm.ACT_RELU, rate=0.05, seed=4)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@gpu
def test_float32_products_are_as_exact_as_fused_multiply_adds():
    """Against float64, in the root mean square: no worse than the library product that torch calls for float32."""
    for M, K, N in [(256, 64, 256), (256, 512, 256), (512, 4096, 256)]:
        c = Case(M, K, N, dtype=sm.F32, bias=False)
        c.forward(save=False)
        want = c.x.double() @ c.W.double()
        ours, fma = (float((t.double() - want).square().mean().sqrt()) for t in (c.y, c.x @ c.W))
        assert ours <= 1.1 * fma, (K, ours, fma)


@gpu
@pytest.mark.parametrize("scale", [2.0**-100, 2.0**-60, 2.0**60])
def test_float32_products_of_small_and_large_values(scale):
    c = Case(70, 130, 72, dtype=sm.F32, bias=False)
    c.x.mul_(scale)
    c.forward(save=False)
    c.check_forward(saved=False)


@gpu
@pytest.mark.parametrize("dtype", [sm.BF16, sm.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M", [13, 60, 150])
def test_infinities_and_nan_stay_in_their_rows_and_columns(M, dtype):
    c = Case(M, 80, 140, dtype=dtype, act=sm.ACT_RELU)
    c.x[3, 5], c.x[7, 0], c.W[9, 20], c.x[M - 1, 79] = float("inf"), float("nan"), float("-inf"), 3e38
    c.forward()
    x, W, b = c.x.float().cpu(), c.W.float().cpu(), c.bias.float().cpu()
    want = (x.double() @ W.double()).float() + b
    want[3] = torch.where(W[5] == 0, float("nan"), torch.sign(W[5]) * float("inf"))
    want[3, 20] = (x[3] * W[:, 20]).sum()
    got = c.pre.float().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.isinf(got), torch.isinf(want.to(got.dtype if dtype == sm.F32 else torch.bfloat16)))
    assert torch.isnan(c.y[7]).all()                                   # ReLU keeps a NaN


@gpu
@pytest.mark.parametrize("dtype", [sm.BF16, sm.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M", [7, 40, 200])
def test_residual_in_place_and_replayed_graph_draws_new_masks(M, dtype):
    """y may be the residual; a captured call reads the state when it runs."""
    c = Case(M, 96, 264, dtype=dtype, residual=True, rate=0.3, act=sm.ACT_GELU)
    start = c.residual.clone()
    c.forward()
    y0 = c.y.clone()
    c.y.copy_(start)
    res, c.residual = c.residual, c.y
    c.forward()
    assert torch.equal(c.y, y0)
    c.residual = res
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            sm.switch_moe_linear_fwd(c.cfg, c.x, c.W, c.bias, c.residual, c.rng, c.y, c.pre, c.ws)
            sm.switch_moe_linear_bwd(c.cfg, c.dy, c.x, c.W, c.pre, c.rng, c.ws, c.dx, c.dW, c.db)
            c.rng[1] += 1
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.y, y0)
    dx0 = c.dx.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(c.y, y0) and not torch.equal(c.dx, dx0)
    c.rng.copy_(rng_state())
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.y, y0) and torch.equal(c.dx, dx0)


@gpu
def test_gradients_against_differences():
    """Float32, a handful of directions: (L(w + h v) - L(w - h v)) / 2 h against <dL/dw, v>, L = <y, dy> in float64."""
    c = Case(24, 40, 56, dtype=sm.F32, act=sm.ACT_GELU, residual=True, rate=0.25)
    c.forward()
    c.backward()
    keep = ref.dropout_factors(c.M, c.N, c.rate, c.site, KEY, OFFSET)
    x, W, b, dy = (ref.to64(t) for t in (c.x, c.W, c.bias, c.dy))
    loss = lambda x, W, b: float((ref.act(x @ W + b, c.act) * keep * dy).sum())
    r = np.random.default_rng(1)
    for grad, at in ((c.dx, 0), (c.dW, 1), (c.db, 2)):
        v = r.standard_normal(ref.to64(grad).shape)
        args = [x, W, b]
        h = 1e-4
        sides = []
        for s in (h, -h):
            a = list(args)
            a[at] = a[at] + s * v
            sides.append(loss(*a))
        want = (sides[0] - sides[1]) / (2 * h)
        got = float((ref.to64(grad) * v).sum())
        # truncation of the difference: h^2 / 6 times a third derivative of order |v|^3 sums; float32 gradients: 1e-5
        assert abs(got - want) <= 2e-5 * float((np.abs(ref.to64(grad) * v)).sum()) + 1e-5, (at, got, want)


@gpu
@pytest.mark.parametrize("M", [40, 300])
def test_optional_outputs_and_empty_calls(M):
    c = Case(M, 64, 72, act=sm.ACT_RELU, rate=0.2)
    c.forward()
    c.backward()
    dx, dW, db = c.dx.clone(), c.dW.clone(), c.db.clone()
    for want in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (0, 1, 1), (0, 0, 0)):
        c.dx.fill_(7.0); c.dW.fill_(7.0); c.db.fill_(7.0)
        sm.switch_moe_linear_bwd(c.cfg, c.dy, c.x if want[1] else None, c.W if want[0] else None, c.pre, c.rng, c.ws,
                                 c.dx if want[0] else None, c.dW if want[1] else None, c.db if want[2] else None)
        sm.switch_moe_linear_check_device_status(c.cfg, c.ws)
        for got, full, asked in ((c.dx, dx, want[0]), (c.dW, dW, want[1]), (c.db, db, want[2])):
            assert torch.equal(got, full) if asked else bool((got == 7.0).all())
    c.ws.fill_(0xFF)                                                   # the status word is written whatever is asked for
    sm.switch_moe_linear_bwd(c.cfg, c.dy, None, None, c.pre, c.rng, c.ws, None, None, None)
    sm.switch_moe_linear_check_device_status(c.cfg, c.ws)
    e = Case(0, 64, 72, pad=8)
    e.forward()
    e.backward()
    assert not e.dW.any() and not e.db.any() and bool((e.dW_all[:, 72:] == 5.0).all())


@gpu
def test_calls_repeat_bit_for_bit_and_share_a_workspace():
    a, b = Case(3000, 256, 264, act=sm.ACT_GELU, rate=0.1), Case(77, 512, 136, act=sm.ACT_RELU, seed=5)
    n = max(a.ws.numel(), b.ws.numel())
    raw = torch.full((n + 1024,), 0xFF, dtype=torch.uint8, device="cuda")
    off = (-raw.data_ptr()) % 1024
    a.ws = b.ws = raw[off:off + n]
    outs = []
    for _ in range(2):
        for c in (a, b):
            c.forward()
            c.backward()
        outs.append([t.clone() for c in (a, b) for t in (c.y, c.pre, c.dx, c.dW, c.db)])
    assert all(torch.equal(p, q) for p, q in zip(*outs))
    a.check_backward()
    b.check_backward()


@gpu
def test_output_past_32_bit_offsets():
    """y of more than 2^32 bytes and 2^31 elements: the last rows, far from the base, against their own product."""
    M, K, N = 2**17 + 3, 64, 2**14 + 8
    cfg = sm.make_linear_config(M, K, N, dropout=0.1, site=1)
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(M, K, device="cuda", generator=g).bfloat16()
    W = torch.randn(K, N, device="cuda", generator=g).bfloat16()
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    ws = sm.allocate_linear_workspace(cfg)
    sm.switch_moe_linear_fwd(cfg, x, W, None, None, rng_state(), y, None, ws)
    sm.switch_moe_linear_check_device_status(cfg, ws)
    for r0 in (0, M - 5):
        keep = ref.dropout_factors(5, N, 0.1, 1, KEY, OFFSET, row0=r0)
        xs, Ws = ref.to64(x[r0:r0 + 5]), ref.to64(W)
        want, u = xs @ Ws * keep, 2.0**-8
        err = ref.product_error(sm.BF16, K) * (np.abs(xs) @ np.abs(Ws)) * keep + 2.0**-23 * np.abs(want)
        within(y[r0:r0 + 5], want, u * np.abs(want) + (1 + u) * err, r0)


# ---------------------------------------------------------------------------------------------------------- refusals
@pytest.fixture(scope="module")
def lib():
    sbuild.build()
    return sm.load_library()


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), sm.INVALID_ARGUMENT), (dict(K=0), sm.INVALID_ARGUMENT), (dict(N=0), sm.INVALID_ARGUMENT),
    (dict(dtype=2), sm.INVALID_ARGUMENT), (dict(activation=3), sm.INVALID_ARGUMENT), (dict(activation=-1), sm.INVALID_ARGUMENT),
    (dict(dropout=1.0), sm.INVALID_ARGUMENT), (dict(dropout=-0.1), sm.INVALID_ARGUMENT), (dict(dropout=float("nan")), sm.INVALID_ARGUMENT),
    (dict(dropout=0.9999999), sm.INVALID_ARGUMENT), (dict(site=-1), sm.INVALID_ARGUMENT), (dict(site=65536), sm.INVALID_ARGUMENT),
    (dict(ldx=56), sm.INVALID_ARGUMENT), (dict(ldw=64), sm.INVALID_ARGUMENT), (dict(ldy=8), sm.INVALID_ARGUMENT),
    (dict(ldx=-8), sm.INVALID_ARGUMENT), (dict(K=65), sm.UNSUPPORTED_SHAPE), (dict(N=73), sm.UNSUPPORTED_SHAPE),
    (dict(N=73, ldw=80, ldy=76), sm.UNSUPPORTED_SHAPE), (dict(N=74, dtype=sm.F32), sm.UNSUPPORTED_SHAPE),
    (dict(M=2**30 + 1), sm.UNSUPPORTED_SHAPE), (dict(K=2**30 + 64), sm.UNSUPPORTED_SHAPE), (dict(N=2**30 + 64), sm.UNSUPPORTED_SHAPE),
])
def test_bad_configs_are_refused(lib, kw, status):
    cfg = sm.make_linear_config(**{**dict(M=32, K=64, N=72), **kw})
    out = ctypes.c_size_t(0)
    assert lib.switch_moe_linear_workspace_bytes(ctypes.byref(cfg), 1, ctypes.byref(out)) == status
    args = [1024] * 8 + [1 << 40, None]
    assert lib.switch_moe_linear_fwd(ctypes.byref(cfg), *args) == status
    assert lib.switch_moe_linear_bwd(ctypes.byref(cfg), *([1024] * 6), 1 << 40, 1024, 1024, 1024, None) == status


def test_bad_arguments_are_refused_before_the_device(lib):
    cfg = sm.make_linear_config(32, 64, 72, activation=sm.ACT_GELU, dropout=0.1)
    need = sm.switch_moe_linear_workspace_bytes(cfg)
    c = ctypes.byref(cfg)
    fwd = lambda **kw: lib.switch_moe_linear_fwd(c, *[{**dict(x=16, W=16, bias=16, res=16, rng=16, y=16, pre=16, ws=1024, n=need,
                                                              st=None), **kw}[k] for k in "x W bias res rng y pre ws n st".split()])
    for k in ("x", "W", "rng", "y", "ws"):
        assert fwd(**{k: None}) == sm.INVALID_ARGUMENT, k
    for k in ("x", "W", "bias", "res", "y", "pre"):
        assert fwd(**{k: 24}) == sm.UNSUPPORTED_SHAPE, k
    assert fwd(ws=1024 + 512) == sm.UNSUPPORTED_SHAPE and fwd(rng=20) == sm.UNSUPPORTED_SHAPE
    assert fwd(n=need - 1) == sm.WORKSPACE_TOO_SMALL
    need = sm.switch_moe_linear_workspace_bytes(cfg, backward=True)
    bwd = lambda **kw: lib.switch_moe_linear_bwd(c, *[{**dict(dy=16, x=16, W=16, pre=16, rng=16, ws=1024, n=need, dx=16, dW=16, db=16,
                                                              st=None), **kw}[k] for k in "dy x W pre rng ws n dx dW db st".split()])
    for k in ("dy", "x", "W", "pre", "rng", "ws"):
        assert bwd(**{k: None}) == sm.INVALID_ARGUMENT, k
    for k in ("dy", "x", "W", "pre", "dx", "dW", "db"):
        assert bwd(**{k: 24}) == sm.UNSUPPORTED_SHAPE, k
    assert bwd(n=need - 1) == sm.WORKSPACE_TOO_SMALL
    assert lib.switch_moe_linear_fwd(None, *([1024] * 8), 1 << 40, None) == sm.INVALID_ARGUMENT
    assert lib.switch_moe_linear_workspace_bytes(c, 0, None) == sm.INVALID_ARGUMENT


def test_tensors_that_do_not_fit_the_config_are_refused():
    cfg = sm.make_linear_config(32, 64, 72)
    good = dict(x=torch.zeros(32, 64).bfloat16())
    for bad in (torch.zeros(32, 64), torch.zeros(31, 64).bfloat16(), torch.zeros(32, 128).bfloat16()[:, :64],
                torch.zeros(64, 32).bfloat16().t(), good["x"]):       # (the last one only is not on a GPU)
        with pytest.raises(sm.SwitchMoeError):
            sm.switch_moe_linear_fwd(cfg, bad, None, None, None, None, None, None, None)


def test_forward_needs_no_more_workspace_than_its_operands():
    a = sm.switch_moe_linear_workspace_bytes(sm.make_linear_config(32768, 768, 2048))
    b = sm.switch_moe_linear_workspace_bytes(sm.make_linear_config(32768, 768, 2048, activation=sm.ACT_GELU), backward=True)
    assert a == 1024 and b < 32768 * 2048 * 2 + 16 * 768 * 2048 * 4 + (1 << 22)
