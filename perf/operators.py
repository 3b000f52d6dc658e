"""Calls of the operators around a Switch FFN layer whose time is followed: the dense product with its epilogue, dropout
from a counter, and the load-balancing loss of any router.  One `run` is what a user's program asks of the library.

linear   y = r + dropout(act(x W + b)) and its gradients.  "fwd": switch_moe_linear_fwd, which with
         "save" also writes the pre-activation for the backward pass; "bwd": switch_moe_linear_bwd, the saved
         pre-activation an input; "train": both calls.
dropout  y = r + x keep / (1 - rate), keep drawn from Philox4x32-10 by element; "train" adds the backward call.
balance  loss = mean over groups of alpha E sum_i f_i P_i, the counts behind f, and d loss / d logits.

With `own` false `run` computes the same in elementary torch operations in 32 bits, so that both can be timed and compared.
Inputs are drawn on the GPU from the seed with the distributions of `paper_2101_03961_b200/inputs.py`: activations and
upstream gradients ~ N(0, 1), weights truncated normal with sigma sqrt(0.1 / fan_in).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_LINEAR = {"op": "linear", "dtype": "bf16", "act": "none", "bias": True, "residual": False, "dropout": 0.0,
           "save": False}
_DROPOUT = {"op": "dropout", "dtype": "bf16", "residual": True}
_BALANCE = {"op": "balance", "dtype": "f32", "k": 1, "groups": 1, "padded": False, "given": False}


def _linear(M, K, N, **kw):
    return {**_LINEAR, "M": M, "K": K, "N": N, **kw}


def _dropout(rows, cols, rate, **kw):
    return {**_DROPOUT, "rows": rows, "cols": cols, "rate": rate, **kw}


def _balance(T, E, **kw):
    return {**_BALANCE, "T": T, "E": E, **kw}


def listed():
    return [
        # one token of one sequence through the first product of a dense feed-forward layer: all latency
        _linear(1, 768, 2048, act="gelu", **{"pass": "fwd"}, name="linear_token_fwd"),
        # one decoding step of a batch of sequences through the second product, added to the residual stream
        _linear(48, 2048, 768, residual=True, **{"pass": "fwd"}, name="linear_batch_fwd"),
        # scores of a last batch of tokens over a vocabulary of odd size (rows padded to 16 bytes)
        _linear(257, 768, 32101, bias=False, **{"pass": "fwd"}, name="linear_vocab_fwd"),
        # one training step of a dense feed-forward layer between two Switch layers: first product, forward and backward ..
        _linear(32768, 768, 2048, act="gelu", save=True, **{"pass": "fwd"}, name="linear_up_fwd"),
        _linear(32768, 768, 2048, act="gelu", **{"pass": "bwd"}, name="linear_up_bwd"),
        # .. and second product, with dropout, on the residual stream
        _linear(32768, 2048, 768, residual=True, dropout=0.1, **{"pass": "train"}, name="linear_down_train"),
        # a smaller such layer in a full-precision run, a ragged number of tokens
        _linear(4001, 512, 2048, act="gelu", dtype="f32", **{"pass": "train"}, name="linear_f32_train"),
        # the largest: backward pass of a wide layer
        _linear(16384, 4096, 10240, act="relu", **{"pass": "bwd"}, name="linear_wide_bwd"),
        # dropout of an attention block's output in a small batch, on the residual stream
        _dropout(512, 768, 0.1, **{"pass": "fwd"}, name="dropout_small_fwd"),
        # a training step's, forward and backward
        _dropout(32768, 2048, 0.1, **{"pass": "train"}, name="dropout_train"),
        # the loss of a unit-test-sized router
        _balance(512, 8, name="balance_small"),
        # a padded long batch in eight groups, two choices of 128 experts a token
        _balance(262144, 128, k=2, groups=8, padded=True, name="balance_long"),
    ]


def _log_int(rng, lo, hi, step=1):
    return max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step)


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "dropout", "balance"])
    if op == "linear":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        kind = rng.choice(["fwd", "train", "bwd"])
        step = rng.choice([1, 8, 64])
        while True:
            M = _log_int(rng, 1, 32768)
            K, N = _log_int(rng, 64, 4096, step), _log_int(rng, 64, 32768 if kind == "fwd" else 8192, step)
            if M * K * N <= (4e11 if dtype == "bf16" else 2e10):
                break
        # (a training pass through a bfloat16 activation is its forward and its backward call: the value saved between
        # them is bfloat16, and an input of the second)
        act = rng.choice({"train": ["none", "gelu"][:1 + (dtype == "f32")]}.get(kind, ["none", "relu", "gelu"]))
        return _linear(M, K, N, dtype=dtype, act=act, bias=rng.random() < 0.7, residual=rng.random() < 0.4,
                       save=kind == "fwd" and act != "none" and rng.random() < 0.5,
                       dropout=rng.choice([0.0, 0.0, 0.1, 0.4]), **{"pass": kind})
    if op == "dropout":
        return _dropout(_log_int(rng, 1, 32768), _log_int(rng, 8, 4096, rng.choice([1, 8])), rng.choice([0.05, 0.1, 0.4]),
                        dtype=rng.choice(["bf16", "f32"]), residual=rng.random() < 0.5,
                        **{"pass": rng.choice(["fwd", "train"])})
    groups = rng.choice([1, 1, 4, 32])
    E = _log_int(rng, 2, 512)
    return _balance(groups * _log_int(rng, max(1, 64 // groups), 131072 // groups), E, k=min(E, rng.choice([1, 1, 2, 4])),
                    groups=groups, dtype=rng.choice(["f32", "bf16"]), padded=rng.random() < 0.5, given=rng.random() < 0.3)


# ------------------------------------------------------------------------------------------------------------- inputs
def _rows(rows, cols, dtype, fill, gen):
    """[rows, cols] on rows padded to 16 bytes."""
    pad = 16 // torch.empty(0, dtype=dtype).element_size()
    t = torch.zeros(rows, (cols + pad - 1) // pad * pad, dtype=dtype, device="cuda")[:, :cols]
    if fill == "normal":
        t.copy_(torch.randn(rows, cols, generator=gen, device="cuda"))
    elif fill == "weight":
        w = torch.empty(rows, cols, device="cuda")
        torch.nn.init.trunc_normal_(w, 0.0, 1.0, -2.0, 2.0, generator=gen)
        t.copy_(w * math.sqrt(0.1 / rows))
    return t


def _rng_state(gen):
    return torch.randint(0, 2**62, (2,), generator=gen, device="cuda", dtype=torch.int64)


def _workspace(nbytes):
    raw = torch.empty(nbytes + 1024, dtype=torch.uint8, device="cuda")
    off = (-raw.data_ptr()) % 1024
    return raw[off:off + nbytes]


def _prepare_linear(c, gen):
    M, K, N, dt = c["M"], c["K"], c["N"], _TYPES[c["dtype"]]
    s = {"case": c, "x": _rows(M, K, dt, "normal", gen), "W": _rows(K, N, dt, "weight", gen), "bias": None,
         "residual": None, "rng": _rng_state(gen) if c["dropout"] else None, "pre": None, "dy": None}
    if c["bias"]:
        s["bias"] = 0.1 * torch.randn(N, generator=gen, device="cuda")
    if c["residual"] and c["pass"] != "bwd":
        s["residual"] = _rows(M, N, dt, "normal", gen)
    if c["pass"] != "fwd":
        s["dy"] = _rows(M, N, dt, "normal", gen)
    if c["act"] != "none" and (c["save"] or c["pass"] != "fwd"):
        s["pre"] = _rows(M, N, dt, "normal" if c["pass"] == "bwd" else "zero", gen)
        if c["pass"] == "bwd":
            s["pre"].mul_(math.sqrt(0.1))
    if own:
        from paper_2101_03961_b200 import switch_moe as sm
        s["cfg"] = sm.make_linear_config(M, K, N, dtype={"bf16": sm.BF16, "f32": sm.F32}[c["dtype"]],
                                         activation={"none": sm.ACT_NONE, "relu": sm.ACT_RELU, "gelu": sm.ACT_GELU}[c["act"]],
                                         dropout=c["dropout"], site=3, ldx=s["x"].stride(0), ldw=s["W"].stride(0),
                                         ldy=_rows(1, N, dt, "zero", gen).stride(0))
        s["ws"] = _workspace(sm.switch_moe_linear_workspace_bytes(s["cfg"], backward=c["pass"] != "fwd"))
        if c["pass"] != "bwd":
            s["y"] = _rows(M, N, dt, "zero", gen)
        if c["pass"] != "fwd":
            s["dx"], s["dW"] = _rows(M, K, dt, "zero", gen), _rows(K, N, dt, "zero", gen)
            s["db"] = torch.empty(N, device="cuda") if c["bias"] else None
    return s


def _prepare_dropout(c, gen):
    dt = _TYPES[c["dtype"]]
    new = lambda fill: _rows(c["rows"], c["cols"], dt, fill, gen)
    s = {"case": c, "x": new("normal"), "residual": new("normal") if c["residual"] else None, "rng": _rng_state(gen),
         "dy": new("normal") if c["pass"] == "train" else None}
    if own:
        from paper_2101_03961_b200 import switch_moe as sm
        s["cfg"] = sm.make_dropout_config(c["rows"], c["cols"], c["rate"], site=5, ld=s["x"].stride(0),
                                          dtype={"bf16": sm.BF16, "f32": sm.F32}[c["dtype"]])
        s["y"], s["dx"] = new("zero"), new("zero") if c["pass"] == "train" else None
    return s


def _prepare_balance(c, gen):
    T, E, G = c["T"], c["E"], c["groups"]
    dt = _TYPES[c["dtype"]]
    skew = torch.randn(E, generator=gen, device="cuda")
    s = {"case": c, "logits": (torch.randn(T, E, generator=gen, device="cuda") + 0.5 * skew).to(dt), "mask": None,
         "index": None}
    if c["padded"]:                                    # every sequence of a group ends somewhere
        length = torch.randint(0, T // G + 1, (G, 1), generator=gen, device="cuda")
        s["mask"] = (torch.arange(T // G, device="cuda")[None] < length).to(torch.uint8).reshape(T)
    if c["given"]:                                     # another router's choices; -1: none
        s["index"] = torch.randint(-1, E, (T, c["k"]), generator=gen, device="cuda", dtype=torch.int32)
    if own:
        from paper_2101_03961_b200 import switch_moe as sm
        s["cfg"] = sm.make_balance_config(T, E, k=c["k"], groups=G, alpha=0.01,
                                          dtype={"bf16": sm.BF16, "f32": sm.F32}[c["dtype"]])
        s["ws"] = _workspace(sm.switch_moe_balance_workspace_bytes(s["cfg"]))
        s["loss"] = torch.empty(1, device="cuda")
        s["counts"] = torch.empty(G, E, dtype=torch.int32, device="cuda")
        s["tokens"] = torch.empty(G, dtype=torch.int32, device="cuda")
        s["dlogits"] = torch.empty_like(s["logits"])
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"linear": _prepare_linear, "dropout": _prepare_dropout, "balance": _prepare_balance}[case["op"]](case, gen)


# --------------------------------------------------------------------------------------------------------- plain forms
_M32 = 0xFFFFFFFF


def _mulhilo(m, c):
    """High and low 32 bits of m c, c < 2^32 in int64."""
    p = m * (c & 0xFFFF)
    q = m * (c >> 16) + (p >> 16)
    return q >> 16, ((q & 0xFFFF) << 16) | (p & 0xFFFF)


def _keep(rows, cols, rate, site, rng):
    """keep / (1 - rate) of every element: Philox4x32-10 (Salmon et al., 2011) with the state's first word as key; a
    counter is the number of eight elements of a row (and the site), then the state's second word.  Element i of the
    eight is 16 bits of the result, and is dropped below the rate in 65536ths."""
    blocks = (cols + 7) // 8
    b = torch.arange(rows * blocks, device=rng.device)
    c0, c1 = b & _M32, (b >> 32) | (site << 16)
    c2, c3 = rng[1] & _M32, (rng[1] >> 32) & _M32
    k0, k1 = rng[0] & _M32, (rng[0] >> 32) & _M32
    for _ in range(10):
        h0, l0 = _mulhilo(0xD2511F53, c0)
        h1, l1 = _mulhilo(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    bits = torch.stack([h for w in (c0, c1, c2, c3) for h in (w & 0xFFFF, w >> 16)], -1)
    threshold = int(math.floor(rate * 65536 + 0.5))
    return (bits >= threshold).reshape(rows, blocks * 8)[:, :cols].float() * (65536 / (65536 - threshold))


def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    return 0.5 * z * torch.erfc(z * -math.sqrt(0.5)) if act == "gelu" else z


def _d_act(z, act):
    if act == "relu":
        return (z > 0).float()
    return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)


def _plain_linear(s):
    c, out = s["case"], {}
    dt, pre = s["x"].dtype, s["pre"]
    x, W = s["x"].float(), s["W"].float()
    keep = _keep(c["M"], c["N"], c["dropout"], 3, s["rng"]) if c["dropout"] else None
    if c["pass"] != "bwd":
        z = x @ W
        if c["bias"]:
            z = z + s["bias"]
        y = _act(z, c["act"])
        if keep is not None:
            y = y * keep
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out["y"] = y.to(dt)
        if pre is not None:
            out["pre"] = z.to(dt)
            pre = z
    if c["pass"] != "fwd":
        dz = s["dy"].float()
        if keep is not None:
            dz = dz * keep
        if c["act"] != "none":
            dz = dz * _d_act(pre.float(), c["act"])
        out["dx"], out["dW"] = (dz @ W.T).to(dt), (x.T @ dz).to(dt)
        if c["bias"]:
            out["db"] = dz.sum(0)
    return out


def _plain_dropout(s):
    c = s["case"]
    keep = _keep(c["rows"], c["cols"], c["rate"], 5, s["rng"])
    y = s["x"].float() * keep
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(s["x"].dtype)}
    if c["pass"] == "train":
        out["dx"] = (s["dy"].float() * keep).to(s["x"].dtype)
    return out


def _plain_balance(s):
    c = s["case"]
    G, E, k = c["groups"], c["E"], c["k"]
    logits = s["logits"].float().reshape(G, -1, E)
    Tg = logits.shape[1]
    e = torch.exp(logits - logits.amax(-1, keepdim=True))
    p = e / e.sum(-1, keepdim=True)
    if s["index"] is None:
        index = torch.sort(logits, dim=-1, descending=True, stable=True)[1][..., :k]
    else:
        index = s["index"].long().reshape(G, Tg, k)
    valid = torch.ones(G, Tg, dtype=torch.bool, device=p.device) if s["mask"] is None else s["mask"].reshape(G, Tg) != 0
    index = torch.where(valid[..., None] & (index >= 0), index, E)
    ones = torch.ones_like(index, dtype=torch.int32).reshape(G, -1)
    counts = torch.zeros(G, E + 1, dtype=torch.int32, device=p.device).scatter_add_(1, index.reshape(G, -1), ones)[:, :E]
    tokens = valid.sum(1)
    n = tokens.clamp_min(1).float()[:, None]
    f = counts.float() / (k * n)
    P = (p * valid[..., None]).double().sum(1).float() / n
    loss = (0.01 * E * (f * P).sum(-1)).mean().reshape(1)
    g = (0.01 * E / G) * f / n
    dl = p * (g[:, None] - (p * g[:, None]).sum(-1, keepdim=True)) * valid[..., None]
    return {"loss": loss, "counts": counts, "tokens": tokens.int(), "dlogits": dl.reshape(-1, E).to(s["logits"].dtype)}


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"linear": _plain_linear, "dropout": _plain_dropout, "balance": _plain_balance}[op](state)
    from paper_2101_03961_b200 import switch_moe as sm
    s, kind = state, state["case"].get("pass")
    if op == "linear":
        out = {}
        if kind != "bwd":
            sm.switch_moe_linear_fwd(s["cfg"], s["x"], s["W"], s["bias"], s["residual"], s["rng"], s["y"], s["pre"], s["ws"])
            out["y"] = s["y"]
            if s["pre"] is not None:
                out["pre"] = s["pre"]
        if kind != "fwd":
            sm.switch_moe_linear_bwd(s["cfg"], s["dy"], s["x"], s["W"], s["pre"], s["rng"], s["ws"], s["dx"], s["dW"], s["db"])
            out["dx"], out["dW"] = s["dx"], s["dW"]
            if s["db"] is not None:
                out["db"] = s["db"]
        return out
    if op == "dropout":
        sm.switch_moe_dropout_fwd(s["cfg"], s["x"], s["residual"], s["rng"], s["y"])
        if kind == "fwd":
            return {"y": s["y"]}
        sm.switch_moe_dropout_bwd(s["cfg"], s["dy"], s["rng"], s["dx"])
        return {"y": s["y"], "dx": s["dx"]}
    sm.switch_moe_balance_fwd(s["cfg"], s["logits"], s["index"], s["mask"], s["loss"], s["counts"], s["tokens"], s["ws"])
    sm.switch_moe_balance_bwd(s["cfg"], s["logits"], s["mask"], s["counts"], s["tokens"], 1.0, s["dlogits"])
    return {"loss": s["loss"], "counts": s["counts"], "tokens": s["tokens"], "dlogits": s["dlogits"]}


# ------------------------------------------------------------------------------------------------------- what it takes
def work(case):
    c = case
    elt = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "linear":
        M, K, N, kind = c["M"], c["K"], c["N"], c["pass"]
        saved = c["act"] != "none" and (c["save"] or kind != "fwd")
        n = M * K + K * N + (N * 4 // elt if c["bias"] else 0)                     # x, W, bias or its gradient
        n += M * N * ((kind != "bwd") * (1 + c["residual"]) + (kind != "fwd") + saved)   # y, residual; dy; pre
        n += (M * K + K * N) * (kind != "fwd")                                     # dx, dW
        return {"bytes": n * elt, "flops": 2 * M * K * N * {"fwd": 1, "bwd": 2, "train": 3}[kind]}
    if c["op"] == "dropout":
        n = c["rows"] * c["cols"]
        passes = 2 + c["residual"] + (2 if c["pass"] == "train" else 0)
        return {"bytes": n * elt * passes, "flops": n * (passes - 1)}
    T, E, G = c["T"], c["E"], c["groups"]
    nbytes = 2 * T * E * elt + T * c["padded"] + T * c["k"] * 4 * c["given"] + G * (E + 1) * 4 + 4
    return {"bytes": nbytes, "flops": 12 * T * E}


# -------------------------------------------------------------------------------------------- the definition in 64 bits
def _philox_bits(rows, cols, site, state):
    """uint16 [rows, 8 ceil(cols / 8)] on the host."""
    u32, u64 = np.uint32, np.uint64
    n = rows * ((cols + 7) // 8)
    number = np.arange(n, dtype=u64)
    ctr = [number.astype(u32), ((number >> u64(32)) + u64(site * 65536)).astype(u32),
           np.full(n, state[1] % 2**32, u32), np.full(n, state[1] // 2**32, u32)]
    key = [state[0] % 2**32, state[0] // 2**32]
    for _ in range(10):
        a, b = ctr[0].astype(u64) * u64(0xD2511F53), ctr[2].astype(u64) * u64(0xCD9E8D57)
        ctr = [(b >> u64(32)).astype(u32) ^ ctr[1] ^ u32(key[0]), b.astype(u32),
               (a >> u64(32)).astype(u32) ^ ctr[3] ^ u32(key[1]), a.astype(u32)]
        key = [(key[0] + 0x9E3779B9) % 2**32, (key[1] + 0xBB67AE85) % 2**32]
    words = np.stack(ctr, axis=1).astype("<u4")
    return np.ascontiguousarray(words).view("<u2").reshape(rows, -1)


def _exact_factor(rows, cols, rate, site, rng):
    limit = round(rate * 65536)
    bits = torch.from_numpy(_philox_bits(rows, cols, site, [int(v) for v in rng.cpu()])[:, :cols].astype(np.int32))
    return torch.where(bits.cuda() < limit, 0.0, 65536.0 / (65536 - limit)).double()


def _exact_linear(s):
    c, out = s["case"], {}
    x, W = s["x"].double(), s["W"].double()
    factor = _exact_factor(c["M"], c["N"], c["dropout"], 3, s["rng"]) if c["dropout"] else 1.0
    if c["pass"] == "bwd":
        z = None if s["pre"] is None else s["pre"].double()
    else:
        z = torch.mm(x, W)
        if s["bias"] is not None:
            z += s["bias"].double()
        h = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0.0),
             "gelu": lambda: z * torch.special.ndtr(z)}[c["act"]]()
        h = h * factor
        out["y"] = h if s["residual"] is None else h + s["residual"].double()
        if s["pre"] is not None:
            out["pre"] = z
    if c["pass"] != "fwd":
        dz = s["dy"].double() * factor
        if c["act"] == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        elif c["act"] == "gelu":
            dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        out["dx"], out["dW"] = torch.mm(dz, W.t()), torch.mm(x.t(), dz)
        if s["bias"] is not None:
            out["db"] = dz.sum(dim=0)
    return out


def _exact_dropout(s):
    c = s["case"]
    factor = _exact_factor(c["rows"], c["cols"], c["rate"], 5, s["rng"])
    y = s["x"].double() * factor
    out = {"y": y if s["residual"] is None else y + s["residual"].double()}
    if s["dy"] is not None:
        out["dx"] = s["dy"].double() * factor
    return out


def _exact_balance(s):
    c = s["case"]
    G, E, k, T = c["groups"], c["E"], c["k"], c["T"]
    per = T // G
    loss, counts, tokens, grads = 0.0, [], [], []
    for g in range(G):
        rows = slice(g * per, (g + 1) * per)
        l = s["logits"][rows].double()
        p = torch.exp(l - torch.logsumexp(l, dim=1, keepdim=True))
        use = torch.ones(per, dtype=torch.bool, device=l.device) if s["mask"] is None else s["mask"][rows].bool()
        if s["index"] is not None:
            chosen = s["index"][rows][use]
        else:                                          # the largest, ties to the lowest index, k times
            left, picks = l[use].clone(), []
            for _ in range(k):
                best = left == left.max(dim=1, keepdim=True)[0]
                first = best & (best.to(torch.int32).cumsum(dim=1) == 1)
                picks.append(first.nonzero()[:, 1])
                left.masked_fill_(first, -math.inf)
            chosen = torch.stack(picks, 1)
        chosen = chosen[chosen >= 0].long()
        count = torch.bincount(chosen, minlength=E)
        n = int(use.sum())
        counts.append(count.to(torch.int32))
        tokens.append(n)
        dl = torch.zeros_like(l)
        if n:
            f = count.double() / (k * n)
            loss += 0.01 * E * float((f * p[use].sum(dim=0)).sum()) / n / G
            up = (0.01 * E / G / n) * f
            q = p[use]
            dl[use] = q * up - q * (q @ up)[:, None]
        grads.append(dl)
    dev = s["logits"].device
    return {"loss": torch.tensor([loss], dtype=torch.float64, device=dev), "counts": torch.stack(counts),
            "tokens": torch.tensor(tokens, dtype=torch.int32, device=dev), "dlogits": torch.cat(grads)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "dropout": _exact_dropout, "balance": _exact_balance}[case["op"]](s)
