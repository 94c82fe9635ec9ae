"""The operators of a gated block and of its update whose time is measured:
norms of queries and keys with the rotation of their positions, the gated
feed-forward block, and updates made orthogonal by Newton-Schulz products,
each through a public call of ``paper_2510_14614_amd.fal`` and, with ``own``
false, in its plain form: products, sums, exponentials and indexing in 32 bits
(angles and sums over a whole matrix in 64), rounded once at the end.

A case is a dict of plain values.  ``kind`` names the operator:

* ``rotary``  ``qk_norm_rope_fwd`` on packed [Q | K | V] rows and, with
              ``train``, ``qk_norm_rope_bwd``: rows, their gradient and those
              of both norms' weights;
* ``ffn``     ``gated_ffn_fwd`` and, with ``train``, ``gated_ffn_bwd``: output
              and the gradients of the input and the three matrices;
* ``schulz``  ``newton_schulz``: every matrix of a batch made orthogonal;
* ``muon``    ``muon_step``: momentum, orthogonal update, weights.
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16 = 0, 1

EPS = 1e-6                                    # of the norms
COEFFICIENTS = (3.4444, -4.7750, 2.0315)      # of the Newton-Schulz polynomial
LR, BETA, DECAY = 0.02, 0.95, 0.01            # of the step


def _rotary(name, **kw):
    base = {"kind": "rotary", "B": 1, "T": 1, "H": 1, "kv": 0, "hd": 64, "rotary": 0, "interleaved": False,
            "theta": 10000.0, "weights": True, "first": -1, "ragged": False, "pad": 0, "dtype": BF16, "train": True}
    base.update(kw)
    return {"name": name, **base} if name else base


def _ffn(name, **kw):
    base = {"kind": "ffn", "M": 1, "d": 64, "f": 256, "act": "silu", "pad": 0, "dtype": BF16, "train": True}
    base.update(kw)
    return {"name": name, **base} if name else base


def _update(name, kind, **kw):
    base = {"kind": kind, "count": 1, "rows": 64, "cols": 64, "steps": 5, "dtype": BF16}
    if kind == "muon":
        base.update(nesterov=True)
    base.update(kw)
    return {"name": name, **base} if name else base


def listed():
    return [
        # One new token of each of 32 texts, far into a long context, shared
        # key and value heads: what a step of generation calls.
        _rotary("rope-one-token", B=32, T=1, H=16, kv=2, hd=128, theta=1e6, first=100000, train=False),
        # A layer's training batch on the GPT-2-small shape.
        _rotary("rope-gpt2-small", B=8, T=1024, H=12, hd=64),
        # Two long documents through wide heads, shared in eight groups.
        _rotary("rope-long-gqa", B=2, T=8192, H=32, kv=8, hd=128, theta=500000.0),
        # fp32, half of each head rotated in neighbouring pairs, a padded
        # batch of odd length in wider rows.
        _rotary("rope-partial-fp32", B=5, T=1021, H=6, kv=3, hd=32, rotary=16, interleaved=True, ragged=True, pad=32,
                dtype=F32),
        # The smallest training call: the tiny fp32 model's block.
        _ffn("ffn-tiny-fp32", M=64, d=64, f=256, act="gelu_tanh", dtype=F32),
        # Five texts' next tokens: bound by the weights.
        _ffn("ffn-few-tokens", M=5, d=2048, f=5504, train=False),
        # A training batch of the ~1.3B shape, two thirds of its ungated width.
        _ffn("ffn-gpt-1.3b", M=8192, d=2048, f=5504),
        # Odd numbers of rows and of tiles, rows in a wider buffer, erf GELU.
        _ffn("ffn-ragged", M=1501, d=1000, f=2744, act="gelu", pad=24),
        # The tiny model's matrices.
        _update("schulz-tiny-fp32", "schulz", count=4, rows=64, cols=192, dtype=F32),
        # Query, key and value projections of GPT-2 small's layers.
        _update("schulz-gpt2-small", "schulz", count=12, rows=768, cols=2304),
        # The step of two layers' up-projections of the ~1.3B shape.
        _update("muon-gpt-1.3b", "muon", count=2, rows=2048, cols=5504),
        # Tall matrices of odd sizes, fp32 weights.
        _update("muon-tall-fp32", "muon", count=3, rows=1001, cols=333, dtype=F32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _products(case):
    """Multiplications of one Newton-Schulz step of all matrices."""
    p, q = sorted((case["rows"], case["cols"]))
    return case["count"] * p * p * (2 * q + p)


def draw(rng):
    cap = {c["name"]: c for c in listed()}
    rows = 2 * 8192 * (32 + 16) * 128
    while True:
        dtype = F32 if rng.random() < 0.35 else BF16
        kind = rng.choice(("rotary", "ffn", "ffn", "schulz", "muon"))
        if kind == "rotary":
            heads, hd = rng.choice((1, 2, 3, 4, 6, 8, 12, 16, 32)), rng.choice((16, 32, 64, 64, 128, 128))
            groups = [k for k in range(1, heads) if heads % k == 0]
            c = _rotary(None, B=_log_int(rng, 1, 64), T=_log_int(rng, 1, 8192), H=heads, hd=hd,
                        kv=rng.choice(groups) if groups and rng.random() < 0.5 else 0,
                        rotary=rng.choice((0, 0, hd // 2)), interleaved=rng.random() < 0.3,
                        theta=rng.choice((10000.0, 500000.0, 1e6)), weights=rng.random() < 0.8,
                        first=rng.choice((-1, -1, _log_int(rng, 1, 1000000))), ragged=rng.random() < 0.4,
                        pad=rng.choice((0, 0, 64)), dtype=dtype, train=rng.random() < 0.7)
            if c["B"] * c["T"] * (heads + 2 * (c["kv"] or heads)) * hd * (2 if dtype == F32 else 1) <= rows:
                return c
        elif kind == "ffn":
            unit = 1 if dtype == F32 else 8
            c = _ffn(None, M=_log_int(rng, 1, 8192), d=unit * _log_int(rng, 64 // unit, 4096 // unit),
                     f=unit * _log_int(rng, 64 // unit, 11008 // unit), act=rng.choice(("silu", "silu", "gelu", "gelu_tanh")),
                     pad=rng.choice((0, 0, 8, 64)), dtype=dtype, train=rng.random() < 0.7)
            top = cap["ffn-gpt-1.3b"]
            if c["M"] * c["d"] * c["f"] * (8 if dtype == F32 else 1) <= top["M"] * top["d"] * top["f"]:
                return c
        else:
            c = _update(None, kind, count=_log_int(rng, 1, 24), rows=_log_int(rng, 8, 4096),
                        cols=_log_int(rng, 8, 8192), steps=rng.choice((5, 5, 5, 3, 6)), dtype=dtype)
            if kind == "muon":
                c["nesterov"] = rng.random() < 0.8
            if c["steps"] * _products(c) <= 5 * _products(cap["muon-gpt-1.3b"]):
                return c


# ------------------------------------------------------------------ inputs --
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == BF16 else torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale)


def _wide(x, pad):
    """x in rows that are pad elements longer."""
    buffer = torch.zeros(*x.shape[:-1], x.shape[-1] + pad, dtype=x.dtype, device=x.device)
    buffer[..., :x.shape[-1]] = x
    return buffer[..., :x.shape[-1]]


def _lengths(case):
    """Sequence lengths of a padded batch: spread over 1 .. T, the first
    sequence whole and, among four or more, the last one empty."""
    B, T = case["B"], case["T"]
    if not case["ragged"]:
        return [T] * B
    return [0 if B >= 4 and b == B - 1 else max(1, T - (b * T) // (B + 1)) for b in range(B)]


def _rotary_inputs(case, seed):
    g, dt = _gen(seed), _dtype(case)
    B, T, hd, kv = case["B"], case["T"], case["hd"], case["kv"] or case["H"]
    width = (case["H"] + 2 * kv) * hd
    # a projection's channels differ in size
    size = torch.exp(_normal(g, (width,), 0.5))
    got = {"qkv": _wide((_normal(g, (B, T, width)) * size).to(dt), case["pad"]), "lens": None, "positions": None,
           "wq": None, "wk": None}
    if case["weights"]:
        got["wq"], got["wk"] = ((1 + _normal(g, (hd,), 0.2)).to(dt) for _ in range(2))
    if case["first"] >= 0:
        start = case["first"] + torch.randint(0, 1000, (B, 1), generator=g, device="cuda")
        got["positions"] = (start + torch.arange(T, device="cuda")).to(torch.int32)
    if case["ragged"]:
        order = torch.randperm(B, generator=torch.Generator().manual_seed(seed))
        got["lens"] = torch.tensor(_lengths(case), dtype=torch.int32)[order].cuda()
    if case["train"]:
        # an output gradient of the size that a mean loss leaves
        got["dout"] = _wide(_normal(g, (B, T, width), 1.0 / math.sqrt(B * T)).to(dt), case["pad"])
    return got


def _ffn_inputs(case, seed):
    g, dt = _gen(seed), _dtype(case)
    M, d, f = case["M"], case["d"], case["f"]
    # normalised rows, weights of a model that has trained for a while
    got = {"x": _wide(_normal(g, (M, d)).to(dt), case["pad"]),
           "w_gate": _normal(g, (d, f), 1.2 / math.sqrt(d)).to(dt),
           "w_up": _normal(g, (d, f), 1.0 / math.sqrt(d)).to(dt),
           "w_down": _normal(g, (f, d), 1.0 / math.sqrt(f)).to(dt)}
    if case["train"]:
        got["dy"] = _wide(_normal(g, (M, d), 1.0 / math.sqrt(M)).to(dt), case["pad"])
    return got


def _update_inputs(case, seed):
    """Gradients as training leaves them: a few strong directions over noise."""
    g = _gen(seed)
    n, rows, cols = case["count"], case["rows"], case["cols"]
    few = min(16, rows, cols)
    strong = torch.arange(1, few + 1, device="cuda", dtype=torch.float32).pow_(-0.7)
    common = torch.matmul(_normal(g, (n, rows, few)) * strong, _normal(g, (n, few, cols))).mul_(1e-3)
    grads = common + _normal(g, (n, rows, cols), 1e-3)
    if case["kind"] == "schulz":
        return {"x": grads.to(_dtype(case))}
    got = {"grads": grads, "momentum": common.mul_(10.0).add_(_normal(g, (n, rows, cols), 3e-3)),
           "master": _normal(g, (n, rows, cols), 0.02), "params": None}
    if case["dtype"] == BF16:
        got["params"] = got["master"].to(torch.bfloat16)
    return got


INPUTS = {"rotary": _rotary_inputs, "ffn": _ffn_inputs, "schulz": _update_inputs, "muon": _update_inputs}


def prepare(case, seed):
    return {"case": case, **INPUTS[case["kind"]](case, seed)}


# ------------------------------------------------------------- plain forms --
def _angles(case, s):
    """cos and sin of every position and pair, [B or 1, T, 1, pairs], from
    angles in 64 bits."""
    r = case["rotary"] or case["hd"]
    if s["positions"] is None:
        at = torch.arange(case["T"], device="cuda", dtype=torch.float64)[None]
    else:
        at = s["positions"].double()
    step = torch.arange(0, r, 2, device="cuda", dtype=torch.float64).mul_(-math.log(case["theta"]) / r).exp_()
    angle = at[:, :, None, None] * step
    return angle.cos().float(), angle.sin().float()


def _turn(case, x, cos, sin):
    """The first `rotary` elements of each head, [..., hd], turned."""
    r = case["rotary"] or case["hd"]
    head, tail = x[..., :r], x[..., r:]
    if case["interleaved"]:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = head[..., :r // 2], head[..., r // 2:]
        head = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((head, tail), -1)


def _plain_rotary(s):
    case = s["case"]
    B, T, H, hd = case["B"], case["T"], case["H"], case["hd"]
    kv = case["kv"] or H
    x = s["qkv"].float().reshape(B, T, H + 2 * kv, hd)
    cos, sin = _angles(case, s)
    one = torch.ones(hd, device="cuda")
    wq, wk = (one if w is None else w.float() for w in (s["wq"], s["wk"]))
    w = torch.cat((wq.expand(H, hd), wk.expand(kv, hd)))
    qk, v = x[:, :, :H + kv], x[:, :, H + kv:]
    live = None
    if s["lens"] is not None:
        live = (torch.arange(T, device="cuda") < s["lens"][:, None])[:, :, None, None]
        qk = torch.where(live, qk, 0.0)
    rstd = (qk.square().mean(-1, keepdim=True) + EPS).rsqrt()
    hat = qk * rstd

    def rows(qk, v):
        got = torch.cat((qk, v), 2)
        if live is not None:
            got = torch.where(live, got, 0.0)
        return got.flatten(2).to(s["qkv"].dtype)

    got = {"out": rows(_turn(case, hat * w, cos, sin), v)}
    if case["train"]:
        dout = s["dout"].float().reshape(B, T, H + 2 * kv, hd)
        dn = _turn(case, dout[:, :, :H + kv], cos, -sin)
        if live is not None:
            dn = torch.where(live, dn, 0.0)
        dw = dn * hat
        dn = dn * w
        got["dqkv"] = rows(rstd * (dn - hat * (dn * hat).mean(-1, keepdim=True)), dout[:, :, H + kv:])
        if case["weights"]:
            got["dq_weight"] = dw[:, :, :H].sum((0, 1, 2), dtype=torch.float64).float()
            got["dk_weight"] = dw[:, :, H:].sum((0, 1, 2), dtype=torch.float64).float()
    return got


def _activation(kind, g):
    """The activation and its derivative."""
    if kind == "silu":
        p = 1 / (1 + (-g).exp())
        return g * p, p * (1 + g * (1 - p))
    if kind == "gelu":
        p = 0.5 * (1 + (g * math.sqrt(0.5)).erf())
        return g * p, p + g * (-0.5 * g * g).exp() * (1 / math.sqrt(2 * math.pi))
    c = math.sqrt(2 / math.pi)
    t = (c * (g + 0.044715 * g * g * g)).tanh()
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 0.134145 * g * g)


def _plain_ffn(s):
    case, dt = s["case"], s["x"].dtype
    x, wg, wu, wd = (s[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    g, u = x @ wg, x @ wu
    a, da = _activation(case["act"], g)
    h = a * u
    got = {"y": h @ wd}
    if case["train"]:
        dy = s["dy"].float()
        dh = dy @ wd.T.contiguous()
        dg, du = dh * u * da, dh * a
        got["dx"] = dg @ wg.T.contiguous() + du @ wu.T.contiguous()
        xt = x.T.contiguous()
        got.update(dw_gate=xt @ dg, dw_up=xt @ du, dw_down=h.T.contiguous() @ dy)
    return {k: v.to(dt) for k, v in got.items()}


def _orthogonal(x, steps):
    """Newton-Schulz steps on each matrix of x, float32 [n, rows, cols]."""
    a, b, c = COEFFICIENTS
    flip = x.shape[1] > x.shape[2]
    if flip:
        x = x.transpose(1, 2).contiguous()
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt()
    x = (x.double() / torch.where(norm == 0, 1.0, norm)).float()
    for _ in range(steps):
        m = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * m + c * torch.matmul(m, m), x)
    return x.transpose(1, 2) if flip else x


def _plain_schulz(s):
    return {"x": _orthogonal(s["x"].float(), s["case"]["steps"]).to(s["x"].dtype)}


def _scale(case):
    return math.sqrt(max(1.0, case["cols"] / case["rows"]))


def _plain_muon(s):
    case, g, m, w = s["case"], s["grads"], s["momentum"], s["master"]
    m.mul_(BETA).add_(g)
    update = _orthogonal(g + BETA * m if case["nesterov"] else m, case["steps"])
    w.mul_(1 - LR * DECAY).sub_(LR * _scale(case) * update)
    if s["params"] is not None:
        s["params"].copy_(w)
    return {k: s[k] for k in ("master", "momentum", "params") if s[k] is not None}


PLAIN = {"rotary": _plain_rotary, "ffn": _plain_ffn, "schulz": _plain_schulz, "muon": _plain_muon}


# ---------------------------------------------------------- the framework's --
def _own(s):
    from paper_2510_14614_amd import fal
    case = s["case"]
    if case["kind"] == "rotary":
        call = {"n_head": case["H"], "n_kv_head": case["kv"], "q_weight": s["wq"], "k_weight": s["wk"],
                "positions": s["positions"], "lens": s["lens"], "rotary_dim": case["rotary"] or case["hd"],
                "theta": case["theta"], "eps": EPS, "interleaved": case["interleaved"]}
        got = {"out": fal.qk_norm_rope_fwd(s["qkv"], **call)}
        if case["train"]:
            grads = fal.qk_norm_rope_bwd(s["qkv"], s["dout"], **call)
            got["dqkv"] = grads.dqkv
            if case["weights"]:
                got.update(dq_weight=grads.dq_weight, dk_weight=grads.dk_weight)
        return got
    if case["kind"] == "ffn":
        weights = (s["w_gate"], s["w_up"], s["w_down"])
        y, saved = fal.gated_ffn_fwd(s["x"], *weights, activation=case["act"], save=case["train"])
        got = {"y": y}
        if case["train"]:
            grads = fal.gated_ffn_bwd(s["x"], *weights, saved, s["dy"], activation=case["act"])
            got.update(dx=grads.dx, dw_gate=grads.dw_gate, dw_up=grads.dw_up, dw_down=grads.dw_down)
        return got
    if case["kind"] == "schulz":
        return {"x": fal.newton_schulz(s["x"], steps=case["steps"], coefficients=COEFFICIENTS)}
    fal.muon_step(s["master"], s["grads"], s["momentum"], params=s["params"], lr=LR, beta=BETA, weight_decay=DECAY,
                  nesterov=case["nesterov"], scale=_scale(case), steps=case["steps"], coefficients=COEFFICIENTS)
    return {k: s[k] for k in ("master", "momentum", "params") if s[k] is not None}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["kind"]](state)


# -------------------------------------------------------------------- work --
def work(case):
    """Rows, matrices and gradients once in and once out.  Products: three of
    M d f forward, six backward; of each Newton-Schulz step, the halves of both
    symmetric products and the whole of the third."""
    es = 2 if case["dtype"] == BF16 else 4
    if case["kind"] == "rotary":
        kv = case["kv"] or case["H"]
        live, N = sum(_lengths(case)), case["B"] * case["T"]
        elements = (case["H"] + kv) * case["hd"]
        row = (case["H"] + 2 * kv) * case["hd"] * es
        # the backward reads rows without V, gradients with it
        nbytes = (live + N) * row + (live * (row + elements * es) + N * row if case["train"] else 0)
        return {"bytes": nbytes, "flops": live * elements * (8.0 + (16.0 if case["train"] else 0.0))}
    if case["kind"] == "ffn":
        M, d, f = case["M"], case["d"], case["f"]
        matrices, rows = 3 * d * f * es, M * d * es
        if case["train"]:
            return {"bytes": 2 * matrices + 4 * rows, "flops": 18.0 * M * d * f}
        return {"bytes": matrices + 2 * rows, "flops": 6.0 * M * d * f}
    n, (p, q) = case["count"], sorted((case["rows"], case["cols"]))
    flops = case["steps"] * n * (p * (p + 1.0) * q + p * p * (p + 1.0) + 2.0 * p * p * q)
    # the step reads gradients, momentum and weights and writes the latter two
    each = 2 * es if case["kind"] == "schulz" else 20 + (2 if case["dtype"] == BF16 else 0)
    return {"bytes": n * p * q * each, "flops": flops}


# ------------------------------------------------------------------- exact --
def exact(case, seed):
    def rotary(s):
        """Rotations as products of complex numbers; gradients by autograd."""
        B, T, H, hd = case["B"], case["T"], case["H"], case["hd"]
        kv, r = case["kv"] or H, case["rotary"] or hd
        lens = torch.full((B,), T, device="cuda") if s["lens"] is None else s["lens"].long()
        live = torch.arange(T, device="cuda")[None] < lens[:, None]
        at = torch.arange(T, device="cuda").expand(B, T) if s["positions"] is None else s["positions"]
        rate = case["theta"] ** (torch.arange(r // 2, device="cuda", dtype=torch.float64) / (-r / 2))
        angle = at[live].double()[:, None] * rate
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        x = s["qkv"][live].double().requires_grad_()
        wq, wk = ((torch.ones(hd, device="cuda") if w is None else w).double().requires_grad_()
                  for w in (s["wq"], s["wk"]))
        parts = []
        for w, rows in ((wq, x[:, :H * hd]), (wk, x[:, H * hd:(H + kv) * hd])):
            z = rows.unflatten(-1, (-1, hd))
            z = z * w / torch.sqrt(z.pow(2).mean(-1, keepdim=True) + EPS)
            pairs = z[..., :r].unflatten(-1, (-1, 2) if case["interleaved"] else (2, -1))
            axis = -1 if case["interleaved"] else -2
            c = torch.complex(pairs.select(axis, 0), pairs.select(axis, 1)) * turn
            parts.append(torch.cat((torch.stack((c.real, c.imag), axis).flatten(-2), z[..., r:]), -1).flatten(1))
        out = torch.cat((*parts, x[:, (H + kv) * hd:]), -1)

        def whole(rows):
            full = torch.zeros(B, T, rows.shape[-1], dtype=torch.float64, device="cuda")
            full[live] = rows
            return full

        got = {"out": whole(out.detach())}
        if case["train"]:
            dx, dq, dk = torch.autograd.grad(out, (x, wq, wk), s["dout"][live].double())
            got["dqkv"] = whole(dx)
            if case["weights"]:
                got.update(dq_weight=dq, dk_weight=dk)
        return got

    def ffn(s):
        names = ("x", "w_gate", "w_up", "w_down")
        x, wg, wu, wd = leaves = [s[k].double().requires_grad_(case["train"]) for k in names]
        gate = x @ wg
        if case["act"] == "silu":
            gate = torch.nn.functional.silu(gate)
        else:
            gate = torch.nn.functional.gelu(gate, approximate="tanh" if case["act"] == "gelu_tanh" else "none")
        y = (gate * (x @ wu)) @ wd
        if not case["train"]:
            return {"y": y}
        grads = torch.autograd.grad(y, leaves, s["dy"].double())
        return {"y": y.detach(), **{"d" + k: v for k, v in zip(names, grads)}}

    def orthogonal(u):
        """The odd polynomial of each matrix, one matrix at a time, as
        products from the left of the smaller side."""
        a, b, c = COEFFICIENTS
        done = []
        for m in u:
            z = m if m.shape[0] <= m.shape[1] else m.T
            size = torch.linalg.matrix_norm(z)
            z = z / size if size > 0 else z
            for _ in range(case["steps"]):
                gram = z @ z.T
                first = gram @ z
                z = a * z + b * first + c * (gram @ first)
            done.append(z if m.shape[0] <= m.shape[1] else z.T)
        return torch.stack(done)

    s = INPUTS[case["kind"]](case, seed)
    if case["kind"] == "rotary":
        return rotary(s)
    if case["kind"] == "ffn":
        return ffn(s)
    if case["kind"] == "schulz":
        return {"x": orthogonal(s["x"].double())}
    g, m = s["grads"].double(), s["momentum"].double()
    m = BETA * m + g
    update = orthogonal(g + BETA * m if case["nesterov"] else m)
    w = s["master"].double() * (1 - LR * DECAY) - LR * max(1.0, case["cols"] / case["rows"]) ** 0.5 * update
    return {"master": w, "momentum": m, **({"params": w} if case["dtype"] == BF16 else {})}
