"""The operators whose time is measured: attention over a sliding window with
a few first tokens that stay visible, token log-probabilities, the clipped
policy loss with a KL term and the preference loss, each through a public
call of ``paper_2510_14614_amd.fal`` and, with ``own`` false, in its plain
form: products, sums, exponentials, comparisons and indexing in 32 bits (sums
over a sequence in 64), rounded once at the end.

A case is a dict of plain values.  ``kind`` names the operator:

* ``attention``   ``window_attention_fwd`` and, with ``train``,
                  ``window_attention_bwd``: output, log-sum-exp and the
                  gradient of the packed queries, keys and values;
* ``logprobs``    ``token_logprobs``, with or without the entropy;
* ``policy``      ``policy_loss``: loss, its parts, log-probabilities and the
                  gradient of the logits;
* ``preference``  ``preference_loss``: loss, sequence log-probabilities and
                  the gradient of the logits.
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16 = 0, 1


def _attention(name, **kw):
    base = {"kind": "attention", "B": 1, "T": 1, "H": 1, "kv": 0, "hd": 64, "window": 1, "sinks": 0, "dtype": BF16,
            "ragged": False, "pad": 0, "train": True}
    base.update(kw)
    return {"name": name, **base} if name else base


def _rows(name, kind, **kw):
    base = {"kind": kind, "B": 1, "T": 1, "V": 256, "pad": 0, "dtype": BF16, "answers": True, "temperature": 1.0}
    base.update({"logprobs": {"entropy": False},
                 "policy": {"ref": True, "sequences": False},
                 "preference": {"ipo": False, "mean": False}}[kind])
    base.update(kw)
    return {"name": name, **base} if name else base


def listed():
    return [
        # The smallest call: the tiny fp32 model that unit tests train.
        _attention("attn-tiny-fp32", B=2, T=32, H=4, hd=16, window=8, sinks=2, dtype=F32),
        # A GPT-2-small layer's training attention at the benchmark's batch,
        # a quarter of the context in the window.
        _attention("attn-gpt2-small", B=8, T=1024, H=12, hd=64, window=256, sinks=4),
        # A long document through the heads of the ~1.3B shape: what the
        # window is for.
        _attention("attn-long-hd128", B=1, T=8192, H=16, hd=128, window=1024, sinks=16),
        # The forward pass over a padded batch of prompts, key and value
        # heads shared in two groups, nothing a multiple of a tile, one
        # sequence empty; rows sit in a wider buffer.
        _attention("attn-ragged-gqa-prompts", B=6, T=1501, H=16, kv=2, hd=64, window=500, sinks=1, ragged=True,
                   pad=64, train=False),
        # fp32 training, as a run that checks bf16 against fp32 does.
        _attention("attn-odd-fp32", B=2, T=1999, H=8, kv=4, hd=128, window=300, sinks=5, dtype=F32),
        # Scores of one prompt's tokens.
        _rows("logprobs-one-prompt", "logprobs", B=1, T=128, V=50257, pad=47, answers=False),
        # Old and reference log-probabilities of a batch of answers, with
        # their entropy.
        _rows("logprobs-batch", "logprobs", B=8, T=1024, V=50257, pad=47, entropy=True),
        # The tiny model's policy step.
        _rows("policy-tiny-fp32", "policy", B=2, T=32, V=256, dtype=F32),
        # The policy step of a GPT-2-small batch: logits as the LM head
        # leaves them, rows padded to 64.
        _rows("policy-gpt2", "policy", B=8, T=1024, V=50257, pad=47),
        # A large odd vocabulary in fp32, dense rows of no alignment, the
        # loss averaged sequence by sequence, sampled at a temperature.
        _rows("policy-large-vocab-fp32", "policy", B=4, T=257, V=128001, dtype=F32, sequences=True, temperature=0.8),
        # Four preference pairs on the GPT-2-small shape.
        _rows("preference-gpt2", "preference", B=8, T=1024, V=50257, pad=47),
        # Three short pairs, odd sizes, fp32, squared loss of mean
        # log-probabilities.
        _rows("preference-short-fp32", "preference", B=6, T=45, V=8009, dtype=F32, ipo=True, mean=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    pairs, logits = 16 * 8192 ** 2, 8 * 1024 * 50304
    while True:
        dtype = F32 if rng.random() < 0.35 else BF16
        if rng.random() < 0.5:
            heads = rng.choice((1, 2, 3, 4, 6, 8, 12, 16))
            groups = [k for k in range(1, heads) if heads % k == 0]
            T = _log_int(rng, 1, 8192)
            c = _attention(None, B=_log_int(rng, 1, 16), T=T, H=heads,
                           kv=rng.choice(groups) if groups and rng.random() < 0.4 else 0,
                           hd=rng.choice((16, 32, 64, 64, 128, 128)), window=_log_int(rng, 1, T + 1),
                           sinks=rng.choice((0, 1, 2, 4, 5, 16, 37, 64)), dtype=dtype, ragged=rng.random() < 0.4,
                           pad=rng.choice((0, 0, 64)), train=rng.random() < 0.7)
            if c["B"] * c["H"] * c["T"] ** 2 * (2 if dtype == F32 else 1) <= pairs:
                return c
            continue
        kind = rng.choice(("logprobs", "policy", "policy", "preference"))
        V = _log_int(rng, 100, 150000)
        c = _rows(None, kind, B=2 * _log_int(rng, 1, 16) if kind == "preference" else _log_int(rng, 1, 32),
                  T=_log_int(rng, 1, 2048), V=V, pad=rng.choice((0, -V % 64, -V % 64)), dtype=dtype,
                  answers=rng.random() < 0.7, temperature=rng.choice((1.0, 1.0, 0.7, 1.3)))
        if kind == "logprobs":
            c["entropy"] = rng.random() < 0.5
        elif kind == "policy":
            c.update(ref=rng.random() < 0.7, sequences=rng.random() < 0.4)
        else:
            c.update(ipo=rng.random() < 0.3, mean=rng.random() < 0.3)
        if c["B"] * c["T"] * (V + c["pad"]) * (2 if dtype == F32 else 1) <= logits:
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


def _lengths(case):
    """Sequence lengths of a padded batch: spread over 1 .. T, the first
    sequence whole and, among four or more, the last one empty."""
    B, T = case["B"], case["T"]
    if not case["ragged"]:
        return [T] * B
    return [0 if B >= 4 and b == B - 1 else max(1, T - (b * T) // (B + 1)) for b in range(B)]


def _spans(case):
    """First and last-plus-one trained position of each sequence: the answer
    after a prompt, before the padding; in a policy batch of four or more
    one sequence has no answer."""
    B, T = case["B"], case["T"]
    if not case["answers"]:
        return [(0, T)] * B

    def span(b):
        u = (b + 1) * 0.6180339887 % 1.0
        lo, hi = int(0.4 * u * T), T - int(0.3 * (7 * u % 1.0) * T)
        return (lo, lo) if case["kind"] != "preference" and B >= 4 and b == B - 1 else (lo, max(lo + 1, hi))

    return [span(b) for b in range(B)]


def _pairs(case):
    """Visible (query, key) pairs of one head, all sequences: t + 1 keys
    while the window and the sinks cover all of them."""
    most = case["window"] + case["sinks"]
    full = [min(T, most) for T in _lengths(case)]
    return sum(n * (n + 1) // 2 + (T - n) * most for n, T in zip(full, _lengths(case)))


def _attention_inputs(case, seed):
    g = _gen(seed)
    B, T, hd = case["B"], case["T"], case["hd"]
    kv = case["kv"] or case["H"]
    width, dA = (case["H"] + 2 * kv) * hd, case["H"] * hd
    qkv = _normal(g, (B, T, width + case["pad"])).to(_dtype(case))[:, :, :width]
    got = {"qkv": qkv, "lens": None, "out": torch.empty(B, T, dA, dtype=qkv.dtype, device="cuda"),
           "lse": torch.empty(B, case["H"], T, dtype=torch.float32, device="cuda")}
    if case["ragged"]:
        order = torch.randperm(B, generator=torch.Generator().manual_seed(seed))
        got["lens"] = torch.tensor(_lengths(case), dtype=torch.int32)[order].cuda()
    if case["train"]:
        # an output gradient of the size that a mean loss leaves
        got["dout"] = _normal(g, (B, T, dA), 1.0 / math.sqrt(B * T)).to(qkv.dtype)
        got["dqkv"] = torch.empty(B, T, width, dtype=qkv.dtype, device="cuda")
    return got


def _off(x, edge):
    return torch.where((x - edge).abs() < 1e-3, torch.where(x < edge, edge - 2e-3, edge + 2e-3), x)


def _rows_inputs(case, seed):
    g = _gen(seed)
    B, T, V, inv = case["B"], case["T"], case["V"], 1.0 / case["temperature"]
    # a model's logits: a common falling part as word frequencies make it
    # and a part of each row's own
    base = torch.arange(1, V + 1, device="cuda", dtype=torch.float32).log_().mul_(-0.8)
    logits = torch.zeros(B, T, V + case["pad"], dtype=_dtype(case), device="cuda")
    logits[:, :, :V] = _normal(g, (B, T, V), 1.5).add_(base).to(logits.dtype)
    x = logits[:, :, :V].float().mul_(inv)
    lse = x.logsumexp(-1)
    # answers are sampled from the model: the largest of x - log(Exp(1))
    noise = torch.empty_like(x).exponential_(generator=g).log_()
    targets = x.sub(noise).argmax(-1)
    del noise
    logp = x.gather(-1, targets[:, :, None])[:, :, 0] - lse
    del x
    got = {"logits": logits, "targets": targets.to(torch.int32), "mask": None,
           "dlogits": torch.empty_like(logits) if case["kind"] != "logprobs" else None}
    if case["answers"]:
        order = torch.randperm(B, generator=torch.Generator().manual_seed(seed))
        span = torch.tensor(_spans(case))[order].cuda()
        t = torch.arange(T, device="cuda")
        got["mask"] = (t >= span[:, :1]) & (t < span[:, 1:])
    live = torch.ones(B, T, device="cuda") if got["mask"] is None else got["mask"].float()
    if case["kind"] == "policy":
        # the policy has moved a little since it sampled; log ratios within
        # 1e-3 of a clip border are moved off it, where every rounding of
        # the same ratio falls on the same side
        ratio = _normal(g, (B, T), 0.15)
        ratio = _off(_off(ratio, math.log(1 - CLIP_LOW)), math.log(1 + CLIP_HIGH))
        got["old_logp"] = logp - ratio
        got["ref_logp"] = logp + _normal(g, (B, T), 0.3) if case["ref"] else None
        # one reward for an answer, normalised over the batch
        got["advantages"] = _normal(g, (B, 1)).expand(B, T).contiguous()
    if case["kind"] == "preference":
        total = (logp.double() * live).sum(-1)
        if case["mean"]:
            total = total / live.sum(-1).clamp(min=1)
        got["ref_logp"] = (total + _normal(g, (B,), 0.1 if case["mean"] else 3.0)).float()
    return got


CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.04
BETA, SMOOTHING = 0.1, 0.05


def prepare(case, seed):
    got = _attention_inputs(case, seed) if case["kind"] == "attention" else _rows_inputs(case, seed)
    return {"case": case, **got}


# ------------------------------------------------------------- plain forms --
def _visible(case, lens, device):
    """[B or 1, T, T] truth values: query t sees key j."""
    t = torch.arange(case["T"], device=device)
    q, k = t[:, None], t[None, :]
    see = ((k <= q) & ((k > q - case["window"]) | (k < case["sinks"])))[None]
    if lens is not None:
        n = lens.to(device).long()[:, None, None]
        see = see & (q < n) & (k < n)
    return see


def _heads(case, x, n):
    """[B, T, n * hd] as [B, kv, n / kv, T, hd]."""
    kv = case["kv"] or case["H"]
    return x.view(x.shape[0], case["T"], kv, n // kv, case["hd"]).permute(0, 2, 3, 1, 4)


def _flat(x):
    """Inverse of _heads."""
    return x.permute(0, 3, 1, 2, 4).flatten(2)


def _product(a, b):
    return torch.matmul(a, b.contiguous())


def _plain_attention(s):
    case = s["case"]
    H, kv, hd = case["H"], case["kv"] or case["H"], case["hd"]
    q, k, v = s["qkv"].float().split((H * hd, kv * hd, kv * hd), -1)
    q, k, v = (_heads(case, x.contiguous(), n) for x, n in ((q, H), (k, kv), (v, kv)))
    see = _visible(case, s["lens"], q.device)[:, None, None]
    scale = 1.0 / math.sqrt(hd)
    p = _product(q * scale, k.transpose(-1, -2)).masked_fill_(~see, -math.inf)
    top = p.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)  # a row that sees nothing
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log())[..., 0]
    p = p.div_(torch.where(total > 0, total, 1.0))
    out = _product(p, v)
    got = {"out": _flat(out).to(s["qkv"].dtype), "lse": lse.flatten(1, 2)}
    if case["train"]:
        do = _heads(case, s["dout"].float(), H)
        ds = _product(do, v.transpose(-1, -2)).sub_((do * out).sum(-1, keepdim=True)).mul_(p)
        dq = _product(ds, k) * scale
        dk = _product(ds.transpose(-1, -2), q).sum(2, keepdim=True) * scale
        dv = _product(p.transpose(-1, -2), do).sum(2, keepdim=True)
        got["dqkv"] = torch.cat([_flat(x) for x in (dq, dk, dv)], -1).to(s["qkv"].dtype)
    return got


def _softmax_rows(s):
    """Log-probability of each target, and the softmax of each row."""
    case = s["case"]
    x = s["logits"][:, :, :case["V"]].float() * (1.0 / case["temperature"])
    top = x.amax(-1, keepdim=True)
    p = (x - top).exp_()
    total = p.sum(-1, keepdim=True)
    target = s["targets"].long()[:, :, None]
    logp = (x.gather(-1, target) - top - total.log())[:, :, 0]
    return x, top[:, :, 0] + total.log()[:, :, 0], logp, p.div_(total), target


def _live(s):
    return torch.ones_like(s["targets"], dtype=torch.bool) if s["mask"] is None else s["mask"]


def _gradient(s, p, target, c):
    """c (onehot - p) / temperature, rows of zeros where c is zero and zeros in
    the padding, in the logits' type."""
    case = s["case"]
    c = (c / case["temperature"])[:, :, None]
    d = (p * -c).scatter_add_(-1, target, c)
    d = torch.nn.functional.pad(d, (0, case["pad"]))
    return torch.where(_live(s)[:, :, None], d, 0.0).to(s["logits"].dtype)


def _plain_logprobs(s):
    x, lse, logp, p, _ = _softmax_rows(s)
    live = _live(s)
    got = {"logp": torch.where(live, logp, 0.0)}
    if s["case"]["entropy"]:
        got["entropy"] = torch.where(live, lse - (p * x).sum(-1), 0.0)
    return got


def _plain_policy(s):
    case = s["case"]
    _, _, logp, p, target = _softmax_rows(s)
    live, adv = _live(s), s["advantages"]
    n = live.double().sum(-1, keepdim=True)
    weight = live / (n.clamp(min=1) * case["B"] if case["sequences"] else n.sum().clamp(min=1))
    ratio = (logp - s["old_logp"]).exp()
    clipped = ((adv > 0) & (ratio > 1 + CLIP_HIGH)) | ((adv < 0) & (ratio < 1 - CLIP_LOW))
    surrogate = torch.minimum(ratio * adv, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv)
    c = torch.where(clipped, 0.0, -ratio * adv)
    kl = torch.zeros_like(logp)
    if s["ref_logp"] is not None:
        d = s["ref_logp"] - logp
        kl = d.exp() - d - 1
        c = c + KL * (1 - d.exp())
    mean = [torch.where(live, v.double() * weight, 0.0).sum() for v in (-surrogate, kl, clipped)]
    stats = torch.stack((mean[0] + KL * mean[1], *mean)).float()
    return {"stats": stats, "logp": torch.where(live, logp, 0.0),
            "dlogits": _gradient(s, p, target, (c * weight).float())}


def _plain_preference(s):
    case = s["case"]
    _, _, logp, p, target = _softmax_rows(s)
    live, half = _live(s), case["B"] // 2
    total = torch.where(live, logp.double(), 0.0).sum(-1)
    share = torch.ones_like(total)
    if case["mean"]:
        share = 1 / live.double().sum(-1).clamp(min=1)
    seq = total * share
    h = (seq - s["ref_logp"])[:half] - (seq - s["ref_logp"])[half:]
    if case["ipo"]:
        loss, dh = (h - 0.5 / BETA) ** 2, 2 * (h - 0.5 / BETA)
    else:
        z = BETA * h
        # log(1 + exp(-|z|)) + max(-z, 0) is -log sigmoid(z)
        tail = torch.log1p((-z.abs()).exp())
        loss = (1 - SMOOTHING) * (tail + (-z).clamp(min=0)) + SMOOTHING * (tail + z.clamp(min=0))
        dh = BETA * (1 / (1 + (-z).exp()) - (1 - SMOOTHING))
    c = torch.cat((dh, -dh)) / half * share
    return {"loss": loss.mean().float().reshape(1), "seq_logp": seq.float(),
            "dlogits": _gradient(s, p, target, (c[:, None] * live).float())}


PLAIN = {"attention": _plain_attention, "logprobs": _plain_logprobs, "policy": _plain_policy,
         "preference": _plain_preference}


# ---------------------------------------------------------- the framework's --
def _own(s):
    from paper_2510_14614_amd import fal
    case = s["case"]
    if case["kind"] == "attention":
        shape = {"n_head": case["H"], "n_kv_head": case["kv"], "window": case["window"], "sinks": case["sinks"],
                 "lens": s["lens"]}
        out, lse = fal.window_attention_fwd(s["qkv"], out=s["out"], lse=s["lse"], **shape)
        got = {"out": out, "lse": lse}
        if case["train"]:
            got["dqkv"] = fal.window_attention_bwd(s["qkv"], out, s["dout"], lse, dqkv=s["dqkv"], **shape)
        return got
    rows = {"vocab": case["V"], "mask": s["mask"], "temperature": case["temperature"]}
    if case["kind"] == "logprobs":
        got = fal.token_logprobs(s["logits"], s["targets"], entropy=case["entropy"], **rows)
        return {"logp": got[0], "entropy": got[1]} if case["entropy"] else {"logp": got}
    if case["kind"] == "policy":
        got = fal.policy_loss(s["logits"], s["targets"], s["old_logp"], s["advantages"], ref_logp=s["ref_logp"],
                              dlogits=s["dlogits"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL,
                              sequence_mean=case["sequences"], **rows)
        return {"stats": got.stats, "logp": got.logp, "dlogits": got.dlogits}
    got = fal.preference_loss(s["logits"], s["targets"], s["ref_logp"], dlogits=s["dlogits"], beta=BETA,
                              label_smoothing=0.0 if case["ipo"] else SMOOTHING, ipo=case["ipo"],
                              length_mean=case["mean"], **rows)
    return {"loss": got.loss, "seq_logp": got.seq_logp, "dlogits": got.dlogits}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["kind"]](state)


# -------------------------------------------------------------------- work --
def work(case):
    """Attention: the products over the visible pairs (two forward, five
    backward), packed activations, outputs and gradients once.  Losses: the
    logits of the trained rows read once, every row of their gradient written
    once."""
    es = 2 if case["dtype"] == BF16 else 4
    if case["kind"] == "attention":
        kv, hd, M = case["kv"] or case["H"], case["hd"], case["B"] * case["T"]
        width, dA = (case["H"] + 2 * kv) * hd, case["H"] * hd
        flops = 4.0 * hd * case["H"] * _pairs(case)
        nbytes = M * (es * (width + dA) + 4 * case["H"])
        if case["train"]:
            flops *= 3.5
            nbytes += M * es * (dA + width)
        return {"bytes": nbytes, "flops": flops}
    live, N = sum(hi - lo for lo, hi in _spans(case)), case["B"] * case["T"]
    nbytes = live * case["V"] * es + N * (4 + 4 + (1 if case["answers"] else 0))
    if case["kind"] == "logprobs":
        return {"bytes": nbytes + (4 * N if case["entropy"] else 0), "flops": live * case["V"] * 6.0}
    nbytes += N * (case["V"] + case["pad"]) * es
    if case["kind"] == "policy":
        nbytes += N * (12 if case["ref"] else 8)
    return {"bytes": nbytes, "flops": live * case["V"] * 8.0}


# ------------------------------------------------------------------- exact --
def exact(case, seed):
    def attention(case, s):
        H, kv, hd, T = case["H"], case["kv"] or case["H"], case["hd"], case["T"]
        lens = [T] * case["B"] if s["lens"] is None else s["lens"].tolist()
        out = torch.zeros(case["B"], T, H * hd, dtype=torch.float64, device="cuda")
        lse = torch.full((case["B"], H, T), -math.inf, dtype=torch.float64, device="cuda")
        dqkv = torch.zeros(case["B"], T, (H + 2 * kv) * hd, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            x = s["qkv"][b, :n].double()
            i = torch.arange(n, device="cuda")
            hidden = (i[None] > i[:, None]) | ((i[:, None] - i[None] >= case["window"]) & (i[None] >= case["sinks"]))
            for h in range(H if n else 0):
                j = h * kv // H
                at = [slice(c * hd, (c + 1) * hd) for c in (h, H + j, H + kv + j)]
                q, k, v = (x[:, a] for a in at)
                score = (q @ k.T / math.sqrt(hd)).masked_fill(hidden, -math.inf)
                lse[b, h, :n] = torch.logsumexp(score, -1)
                p = torch.exp(score - lse[b, h, :n, None])
                out[b, :n, at[0]] = p @ v
                if case["train"]:
                    g = s["dout"][b, :n, at[0]].double()
                    dp = g @ v.T
                    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(hd)
                    dqkv[b, :n, at[0]] = ds @ k
                    dqkv[b, :n, at[1]] += ds.T @ q
                    dqkv[b, :n, at[2]] += p.T @ g
        return {"out": out, "lse": lse, **({"dqkv": dqkv} if case["train"] else {})}

    def rows(case, s):
        """Everything but the loss's own part comes from autograd over
        log-softmax in 64 bits, a sequence at a time."""
        B, T, V = case["B"], case["T"], case["V"]
        keep = torch.ones(B, T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]
        logs = [(s["logits"][b, :, :V].double() / case["temperature"]).log_softmax(-1) for b in range(B)]
        pick = [lp.gather(-1, s["targets"][b].long()[:, None])[:, 0] for b, lp in enumerate(logs)]
        logp = torch.stack([torch.where(keep[b], pick[b], 0.0) for b in range(B)])
        if case["kind"] == "logprobs":
            got = {"logp": logp}
            if case["entropy"]:
                got["entropy"] = torch.stack([torch.where(keep[b], -(lp.exp() * lp).sum(-1), 0.0)
                                              for b, lp in enumerate(logs)])
            return got
        leaf = logp.clone().requires_grad_()
        if case["kind"] == "policy":
            n = keep.sum(-1, keepdim=True).double()
            w = keep / n.clamp(min=1) / B if case["sequences"] else keep / n.sum().clamp(min=1)
            r = torch.exp(leaf - s["old_logp"].double())
            a = s["advantages"].double()
            bound = torch.where(a > 0, r.clamp(max=1 + CLIP_HIGH), r.clamp(min=1 - CLIP_LOW))
            kl = torch.zeros_like(leaf)
            if s["ref_logp"] is not None:
                d = s["ref_logp"].double() - leaf
                kl = torch.expm1(d) - d
            parts = [(w * v).sum() for v in (-bound * a, kl, (bound != r).double())]
            loss = parts[0] + KL * parts[1]
            got = {"stats": torch.stack([loss, *parts]).detach(), "logp": logp}
        else:
            n = keep.sum(-1).double()
            seq = leaf.masked_fill(~keep, 0.0).sum(-1) / (n.clamp(min=1) if case["mean"] else 1.0)
            gain = seq - s["ref_logp"].double()
            h = gain[:B // 2] - gain[B // 2:]
            if case["ipo"]:
                loss = ((h - 1 / (2 * BETA)) ** 2).mean()
            else:
                f = torch.nn.functional.logsigmoid
                loss = -((1 - SMOOTHING) * f(BETA * h) + SMOOTHING * f(-BETA * h)).mean()
            got = {"loss": loss.detach().reshape(1), "seq_logp": seq.detach()}
        loss.backward()
        d = torch.zeros(B, T, V + case["pad"], dtype=torch.float64, device="cuda")
        for b, lp in enumerate(logs):
            c = torch.where(keep[b], leaf.grad[b], 0.0)[:, None] / case["temperature"]
            d[b, :, :V] = torch.where(keep[b][:, None], -c * lp.exp(), 0.0)
            d[b].scatter_add_(-1, s["targets"][b].long()[:, None], c)
        return {**got, "dlogits": d}

    if case["kind"] == "attention":
        return attention(case, _attention_inputs(case, seed))
    return rows(case, _rows_inputs(case, seed))
