"""The operators as a model strings them together: a dense feed-forward layer with dropout on the residual stream, a router whose
balance loss leaves padding out, and the Switch layer behind it, forward and backward."""
import numpy as np
import pytest
import torch

from oracle import switch_oracle as so
from paper_2101_03961_b200 import build as sbuild
from paper_2101_03961_b200 import inputs as si
from paper_2101_03961_b200 import switch_moe as sm
from tests import operator_reference as ref
from tests.gpu_helpers import TOL_BF16, GpuLayer, rel_err, to_np

gpu = pytest.mark.gpu
T, D, F, E, RATE = 700, 192, 264, 12, 0.1
KEY, OFFSET = 77, 5


class Block:
    """y = x + dropout(W2 dropout(gelu(W1 x + b1)) + b2); logits = y Wr; balance loss of two choices in two groups."""

    def __init__(self, dtype, seed=0):
        sbuild.build()
        g = torch.Generator(device="cuda").manual_seed(seed)
        t = ref.TYPES[dtype]
        rnd = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale)
        self.x, self.dy = rnd(T, D).to(t), rnd(T, D).to(t)
        self.W1, self.W2 = rnd(D, F, scale=D**-0.5).to(t), rnd(F, D, scale=F**-0.5).to(t)
        self.b1, self.b2 = rnd(F, scale=0.1), rnd(D, scale=0.1)
        self.Wr = rnd(D, E, scale=D**-0.5)
        self.mask = (torch.arange(T, device="cuda") % (T // 2) < 300).to(torch.uint8)
        self.rng = torch.tensor([KEY, OFFSET], device="cuda")
        self.up = sm.make_linear_config(T, D, F, dtype=dtype, activation=sm.ACT_GELU, dropout=RATE, site=1)
        self.down = sm.make_linear_config(T, F, D, dtype=dtype, dropout=RATE, site=2)
        self.router = sm.make_linear_config(T, D, E, dtype=sm.F32)
        self.balance = sm.make_balance_config(T, E, k=2, groups=2, alpha=0.5)
        self.ws = [sm.allocate_linear_workspace(c, backward=True) for c in (self.up, self.down, self.router)]
        self.bws = sm.allocate_balance_workspace(self.balance)
        self.h, self.pre, self.dh = (torch.empty(T, F, dtype=t, device="cuda") for _ in range(3))
        self.y, self.dx, self.dyr = (torch.empty_like(self.x) for _ in range(3))
        self.dW1, self.dW2 = torch.empty_like(self.W1), torch.empty_like(self.W2)
        self.db1, self.db2 = torch.empty_like(self.b1), torch.empty_like(self.b2)
        self.yf, self.dyf = (torch.empty(T, D, device="cuda") for _ in range(2))
        self.logits, self.dlogits = (torch.empty(T, E, device="cuda") for _ in range(2))
        self.dWr, self.loss = torch.empty_like(self.Wr), torch.empty(1, device="cuda")
        self.counts, self.tokens = torch.empty(2, E, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")

    def forward(self):
        sm.switch_moe_linear_fwd(self.up, self.x, self.W1, self.b1, None, self.rng, self.h, self.pre, self.ws[0])
        sm.switch_moe_linear_fwd(self.down, self.h, self.W2, self.b2, self.x, self.rng, self.y, None, self.ws[1])
        self.yf.copy_(self.y)
        sm.switch_moe_linear_fwd(self.router, self.yf, self.Wr, None, None, None, self.logits, None, self.ws[2])
        sm.switch_moe_balance_fwd(self.balance, self.logits, None, self.mask, self.loss, self.counts, self.tokens, self.bws)

    def backward(self):
        sm.switch_moe_balance_bwd(self.balance, self.logits, self.mask, self.counts, self.tokens, 1.0, self.dlogits)
        sm.switch_moe_linear_bwd(self.router, self.dlogits, self.yf, self.Wr, None, None, self.ws[2], self.dyf, self.dWr, None)
        self.dyr.copy_(self.dyf.add_(self.dy))
        sm.switch_moe_linear_bwd(self.down, self.dyr, self.h, self.W2, None, self.rng, self.ws[1], self.dh, self.dW2, self.db2)
        sm.switch_moe_linear_bwd(self.up, self.dh, self.x, self.W1, self.pre, self.rng, self.ws[0], self.dx, self.dW1, self.db1)
        self.dx.add_(self.dyr)

    def results(self):
        return [t.clone() for t in (self.y, self.loss, self.counts, self.tokens, self.dx, self.dW1, self.db1, self.dW2, self.db2,
                                    self.dWr)]


def _autograd(b):
    """The same in float64 with torch's autograd, the masks and choices as constants."""
    keep = [torch.from_numpy(ref.dropout_factors(T, n, RATE, site, KEY, OFFSET)).cuda() for n, site in ((F, 1), (D, 2))]
    leaves = [t.double().requires_grad_() for t in (b.x, b.W1, b.b1, b.W2, b.b2, b.Wr)]
    x, W1, b1, W2, b2, Wr = leaves
    h = torch.special.ndtr(x @ W1 + b1) * (x @ W1 + b1) * keep[0]
    y = x + (h @ W2 + b2) * keep[1]
    p = torch.softmax(y @ Wr, -1) * b.mask.double()[:, None]
    n = b.tokens.double()[:, None]
    f = b.counts.double() / (2 * n)
    loss = (0.5 * E * (f * p.view(2, -1, E).sum(1) / n).sum(-1)).mean()
    ((y * b.dy.double()).sum() + loss).backward()
    return [y, loss] + [t.grad for t in leaves]


@gpu
def test_float32_block_against_autograd():
    b = Block(sm.F32)
    b.forward()
    b.backward()
    y, loss, dx, dW1, db1, dW2, db2, dWr = (t.detach().cpu().numpy() for t in _autograd(b))
    # Float32 throughout: a product of K terms is off by a few 2^-24 of the root of the sum of its squared terms (random signs),
    # GELU by 5e-7 of its argument; four products and two activations in a row stay under 1e-5 of the tensor's norm.
    for got, want in ((b.y, y), (b.dx, dx), (b.dW1, dW1), (b.db1, db1), (b.dW2, dW2), (b.db2, db2), (b.dWr, dWr)):
        got = ref.to64(got)
        assert np.linalg.norm(got - want) <= 1e-5 * np.linalg.norm(want)
    assert abs(float(b.loss) - float(loss)) <= 1e-5 * abs(float(loss))
    valid = b.mask.bool().view(2, -1)
    assert torch.equal(b.tokens, valid.sum(1).int())
    top = torch.topk(b.logits, 2)[1].view(2, -1, 2)
    assert torch.equal(b.counts, torch.stack([torch.bincount(t[v].reshape(-1), minlength=E) for t, v in zip(top, valid)]).int())


@gpu
@pytest.mark.parametrize("dtype", [sm.BF16, sm.F32], ids=["bf16", "f32"])
def test_captured_step_on_a_side_stream_equals_the_eager_one(dtype):
    b = Block(dtype)
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    eager = b.results()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.forward()
        b.backward()
        b.rng[1] += 1
    for t in (b.y, b.loss, b.counts, b.tokens, b.dx, b.dW1, b.db1, b.dW2, b.db2, b.dWr):
        t.fill_(7)
    b.rng.copy_(torch.tensor([KEY, OFFSET]))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(eager, b.results()))
    graph.replay()                                                      # the state has moved on: other masks
    torch.cuda.synchronize()
    assert not torch.equal(eager[0], b.y)


@gpu
def test_dense_layer_in_front_of_a_switch_layer():
    """bf16: the dense layer's output is the Switch layer's input, the Switch layer's dx the dense layer's dy."""
    b = Block(sm.BF16)
    b.forward()
    scfg = si.SwitchConfig("behind", T, D, 128, 8, 1.25)
    data = si.gen_layer(scfg, seed=2)
    layer = GpuLayer(scfg, data)
    layer.x = b.y
    y, aux, dx = torch.empty_like(b.y), torch.zeros(1, device="cuda"), torch.empty_like(b.y)
    dW_r, dW_in, dW_out = torch.empty_like(layer.W_r), torch.empty_like(layer.W_in), torch.empty_like(layer.W_out)
    sm.switch_moe_fwd(layer.cfg, layer.x, layer.W_r, layer.bias, layer.W_in, layer.W_out, y, aux, layer.ws)
    sm.switch_moe_bwd(layer.cfg, b.dy, 1.0, layer.x, layer.W_r, layer.W_in, layer.W_out, y, layer.ws, dx, dW_r, dW_in, dW_out)
    sm.switch_moe_check_device_status(layer.cfg, layer.ws)
    index = sm.switch_moe_workspace_view(layer.cfg, layer.ws, sm.WS_EXPERT_INDEX).cpu().numpy().astype(np.int64)
    fwd = so.switch_forward(to_np(b.y), to_np(layer.W_r), to_np(layer.W_in), to_np(layer.W_out), 1.25, scfg.alpha, expert_index=index)
    assert rel_err(to_np(y), fwd["y"]) <= TOL_BF16
    # its gradient goes on through the dense layer: dropout, both products
    b.dyr.copy_(dx)
    sm.switch_moe_linear_bwd(b.down, b.dyr, b.h, b.W2, None, b.rng, b.ws[1], b.dh, b.dW2, b.db2)
    keep = ref.dropout_factors(T, D, RATE, 2, KEY, OFFSET)
    g = to_np(dx) * keep
    # dz is rounded to bfloat16 (2^-8 an element), so is the result
    assert rel_err(to_np(b.dh), g @ to_np(b.W2).T) <= TOL_BF16
    assert rel_err(to_np(b.dW2), to_np(b.h).T @ g) <= TOL_BF16
    assert rel_err(to_np(b.db2), g.sum(0)) <= 1e-5


@gpu
def test_fused_and_separate_dropout_draw_the_same_mask():
    """The product's dropout and switch_moe_dropout of its result, with one state and site."""
    for dtype in (sm.F32, sm.BF16):
        t = ref.TYPES[dtype]
        for M in (5, 300):
            x, W = torch.randn(M, 64, device="cuda").to(t), torch.randn(64, 136, device="cuda").to(t)
            rng = torch.tensor([KEY, OFFSET], device="cuda")
            y, z = torch.empty(M, 136, dtype=t, device="cuda"), torch.empty(M, 136, dtype=t, device="cuda")
            cfg = sm.make_linear_config(M, 64, 136, dtype=dtype, dropout=0.3, site=4)
            sm.switch_moe_linear_fwd(cfg, x, W, None, None, rng, y, None, sm.allocate_linear_workspace(cfg))
            ones = torch.ones_like(y)
            sm.switch_moe_dropout_fwd(sm.make_dropout_config(M, 136, 0.3, dtype=dtype, site=4), ones, None, rng, z)
            assert torch.equal(y == 0, z == 0)
