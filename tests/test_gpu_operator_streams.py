"""Calls of the operators at the same time on several streams, each with a workspace of its own, eager and replayed: every result is
bit for bit what the same call gives by itself."""
import pytest
import torch

from paper_2101_03961_b200 import switch_moe as sm
from tests.test_gpu_linear import Case

gpu = pytest.mark.gpu


class Balance:
    def __init__(self, T, E, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.logits = torch.randn(T, E, device="cuda", generator=g)
        self.cfg = sm.make_balance_config(T, E, k=2)
        self.ws = sm.allocate_balance_workspace(self.cfg)
        self.out = [torch.empty(1, device="cuda"), torch.empty(1, E, dtype=torch.int32, device="cuda"),
                    torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty_like(self.logits)]

    def run(self):
        loss, counts, tokens, dl = self.out
        sm.switch_moe_balance_fwd(self.cfg, self.logits, None, None, loss, counts, tokens, self.ws)
        sm.switch_moe_balance_bwd(self.cfg, self.logits, None, counts, tokens, 1.0, dl)


class Linear(Case):
    def run(self):
        sm.switch_moe_linear_fwd(self.cfg, self.x, self.W, self.bias, self.residual, self.rng, self.y, self.pre, self.ws)
        sm.switch_moe_linear_bwd(self.cfg, self.dy, self.x, self.W, self.pre, self.rng, self.ws, self.dx, self.dW, self.db)

    @property
    def out(self):
        return [self.y, self.pre, self.dx, self.dW, self.db]


@gpu
@pytest.mark.parametrize("captured", [False, True], ids=["eager", "captured"])
def test_calls_at_the_same_time(captured):
    gelu = dict(act=sm.ACT_GELU, rate=0.1, residual=True)
    calls = [Linear(5000, 256, 520, **gelu), Linear(40, 512, 1000, seed=1, **gelu), Linear(3000, 200, 264, dtype=sm.F32, seed=2, **gelu),
             Linear(7, 96, 203, dtype=sm.F32, seed=3, **gelu), Balance(200000, 64, 4), Balance(300, 40, 5)]
    alone = []
    for c in calls:
        c.run()
        torch.cuda.synchronize()
        alone.append([t.clone() for t in c.out])
        for t in c.out:
            t.fill_(3)
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    if captured:
        graphs = []
        for c, s in zip(calls, streams):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                c.run()
            graphs.append(graph)
        torch.cuda.synchronize()
    for _ in range(20):
        for i, (c, s) in enumerate(zip(calls, streams)):
            with torch.cuda.stream(s):
                graphs[i].replay() if captured else c.run()
    torch.cuda.synchronize()
    for c, want in zip(calls, alone):
        assert all(torch.equal(a, b) for a, b in zip(c.out, want))
        if isinstance(c, Linear):
            sm.switch_moe_linear_check_device_status(c.cfg, c.ws)
