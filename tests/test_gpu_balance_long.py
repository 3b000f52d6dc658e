"""The balance loss and its gradient of more than 2^31 logits."""
import numpy as np
import pytest
import torch

from paper_2101_03961_b200 import build as sbuild
from paper_2101_03961_b200 import switch_moe as sm
from tests import operator_reference as ref

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype,E", [(sm.F32, 72), (sm.BF16, 71)], ids=["f32", "bf16_odd"])
def test_logits_past_32_bit_offsets(dtype, E):
    """Two groups, the second one beyond 2^31 bytes and ending beyond 2^31 elements; a quarter of it padding; given choices."""
    sbuild.build()
    T, k, alpha = 2**25 + 8, 2, 0.01
    per = T // 2
    g = torch.Generator(device="cuda").manual_seed(0)
    logits = torch.randn(T, E, device="cuda", generator=g, dtype=torch.bfloat16).to(ref.TYPES[dtype])
    index = torch.randint(0, E, (T, k), device="cuda", dtype=torch.int32, generator=g)
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    mask[T - per // 4:T - 3] = 0                                       # the last three tokens count
    cfg = sm.make_balance_config(T, E, k=k, groups=2, alpha=alpha, dtype=dtype)
    ws = sm.allocate_balance_workspace(cfg)
    loss = torch.full((1,), 7.0, device="cuda")
    counts, tokens = torch.full((2, E), -7, dtype=torch.int32, device="cuda"), torch.full((2,), -7, dtype=torch.int32, device="cuda")
    sm.switch_moe_balance_fwd(cfg, logits, index, mask, loss, counts, tokens, ws)
    want_tokens = [per, per - per // 4 + 3]
    assert tokens.tolist() == want_tokens
    want_loss, p_last = 0.0, None
    for i in range(2):
        rows = slice(i * per, (i + 1) * per)
        used = index[rows][mask[rows] != 0].flatten().long()
        assert torch.equal(counts[i].long(), torch.bincount(used, minlength=E))
        total = torch.zeros(E, dtype=torch.float64, device="cuda")
        for r in range(i * per, (i + 1) * per, 2**20):
            s = slice(r, min(r + 2**20, (i + 1) * per))
            total += (torch.softmax(logits[s].double(), -1) * mask[s, None]).sum(0)
        f = counts[i].double() / (k * want_tokens[i])
        want_loss += float(alpha * E * (f * total).sum() / want_tokens[i] / 2)
    # a probability 2^-19; float32 sums of a lane's, at most T / 1184 rows where a block an SM works on a row a warp
    assert abs(float(loss) - want_loss) <= (2.0**-19 + (T / 1184 + 16) * 2.0**-24) * want_loss
    last = logits[T - 6:].clone()
    sm.switch_moe_balance_bwd(cfg, logits, mask, counts, tokens, 1e6, logits)          # in place
    got = ref.to64(logits[T - 6:])
    assert not got[:3].any()
    lg = ref.to64(last[3:])
    p = np.exp(lg - lg.max(1, keepdims=True))
    p = p / p.sum(1, keepdims=True)
    n = want_tokens[1]
    up = 1e6 * alpha * E / 2 / n * ref.to64(counts[1]) / (k * n)
    want = p * (up - (p * up).sum(1, keepdims=True))
    # counted from the first expert's choices: both terms up to p max|up - up_0|, each probability off by 2^-19; the factors of `up`
    # and its products five roundings
    spread = np.abs(up - up[0]).max()
    bound = ref.HALF_STEP[dtype] * np.abs(want) + (4 * 2.0**-19 + 8 * 2.0**-24) * p * spread + 2.0**-133
    assert np.all(np.abs(got[3:] - want) <= bound), (np.abs(got[3:] - want) - bound).max()
    del logits, index, mask
    torch.cuda.empty_cache()
