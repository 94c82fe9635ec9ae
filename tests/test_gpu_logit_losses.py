"""Token log-probabilities, the clipped policy loss and the preference loss
against their formulas in 64 bits.

Tolerances (u = 2^-24, r = 2^-8 half a step of bf16; X the largest |logit /
temperature|, V columns):

* a row's log-sum-exp: each exponential is off by 3 u (X of its argument) + 2 u,
  the sum of V of them by at most (V / 256 + 12) u in the kernels' order, so
      e = (6 X + V / 256 + 24) u
  bounds the error of a log-probability (absolute) and of a probability
  (relative);
* the entropy lse - sum p x adds e (|lse| + sum p|x|);
* a row's coefficient c: the ratio, e^d and their products move by e + 8 u
  relative, all times the row's weight;
* a gradient element |c| p takes err(c) p + |c| p e, and r of itself in bf16.
"""
import math

import pytest
import torch

from paper_2510_14614_amd import fal

from gpu_helpers import log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U, R = 2.0 ** -24, 2.0 ** -8


def rows(B, T, V, dtype, seed, width=None, scale=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.zeros(B, T, width or V, device="cuda")
    x[:, :, :V] = torch.randn(B, T, V, device="cuda", generator=g) * scale
    x = x.to(dtype)
    y = torch.randint(0, V, (B, T), device="cuda", generator=g, dtype=torch.int32)
    return x, y, g


def err_lse(x, V, temp):
    return (6 * float(x[:, :, :V].double().abs().max()) / temp + V / 256 + 24) * U


def exact(x, y, V, temp):
    lp = (x[:, :, :V].double() / temp).log_softmax(-1)
    return lp, lp.gather(-1, y.long()[:, :, None])[:, :, 0]


def within(name, got, want, bound):
    worst = float(((got.double() - want).abs() / (bound + 1e-30)).nan_to_num(nan=math.inf).max()) if got.numel() else 0
    log(f"  {name}: worst error / bound {worst:.3f}")
    assert worst <= 1.0, name


# vocabularies around the vector widths and the kernels' row variants
VOCABS = [1, 2, 7, 8, 9, 255, 256, 1000, 4097, 50257]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("V", VOCABS + [70001, 140003, 270001])
def test_logprobs(V, dtype):
    B, T, temp = 2, 5, 0.8
    x, y, g = rows(B, T, V, dtype, seed=V)
    mask = torch.rand(B, T, device="cuda", generator=g) < 0.7
    mask[0, 0], mask[1, 1] = True, False
    x[1, 1] = math.nan  # not read
    log(f"logprobs V={V} {dtype}")
    clean = torch.where(mask[:, :, None], x, 0.0)
    lp, want = exact(clean, y, V, temp)
    e = err_lse(clean, V, temp)
    logp, ent = fal.token_logprobs(x, y, mask=mask, temperature=temp, entropy=True)
    assert not logp[~mask].any() and not ent[~mask].any()
    within("logp", logp, torch.where(mask, want, 0.0), e + 2 * U * want.abs())
    h = -(lp.exp() * lp).sum(-1)
    spread = (lp.exp() * lp.abs()).sum(-1)
    within("entropy", ent, torch.where(mask, h, 0.0), e * (1 + 2 * spread) + e)
    assert torch.equal(fal.token_logprobs(x, y, mask=mask.to(torch.uint8) * 255, temperature=temp), logp)


def policy_reference(x, y, V, old, adv, ref, mask, low, high, kl, seq, temp):
    lp, logp = exact(x, y, V, temp)
    leaf = logp.clone().requires_grad_()
    n = mask.sum(-1, keepdim=True).double()
    w = mask / n.clamp(min=1) / x.shape[0] if seq else mask / n.sum().clamp(min=1)
    ratio = torch.exp(leaf - old.double())
    a = adv.double()
    surr = torch.minimum(ratio * a, ratio.clamp(1 - low, 1 + high) * a)
    clipped = ((a > 0) & (ratio > 1 + high)) | ((a < 0) & (ratio < 1 - low))
    term = torch.zeros_like(leaf)
    if ref is not None:
        d = ref.double() - leaf
        term = torch.expm1(d) - d
    parts = [(w * v).sum() for v in (-surr, term, clipped.double())]
    loss = parts[0] + kl * parts[1]
    loss.backward()
    c = torch.where(mask, leaf.grad, 0.0)
    onehot = torch.zeros_like(lp).scatter_(-1, y.long()[:, :, None], 1.0)
    grad = c[:, :, None] / temp * (onehot - lp.exp())
    scale = w * (ratio * a.abs() + kl * (term + 2)).detach()
    size = w * ((ratio * a).abs() + kl * term).detach()
    return torch.stack([loss, *parts]).detach(), logp, grad, scale, size, onehot, lp.exp()


def policy_inputs(B, T, V, dtype, seed, low, high, width=None):
    x, y, g = rows(B, T, V, dtype, seed, width)
    _, logp = exact(x, y, V, 1.0)
    move = torch.randn(B, T, device="cuda", generator=g) * 0.3
    for edge in (math.log(1 - low) if low < 1 else -9.0, math.log(1 + high)):
        # off the border, where the clip's choice is one of rounding
        move = torch.where((move - edge).abs() < 1e-2, edge + 2e-2, move)
    old = (logp - move).float()
    ref = (logp + 0.4 * torch.randn(B, T, device="cuda", generator=g)).float()
    adv = torch.randn(B, T, device="cuda", generator=g)
    adv[0, 0] = 0.0
    return x, y, old, adv, ref, g


@pytest.mark.parametrize("seq", [False, True], ids=["token-mean", "sequence-mean"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("V", [2, 9, 256, 1000, 4097, 50257, 70001, 140003])
def test_policy_loss(V, dtype, seq):
    B, T, low, high, kl = 3, 7, 0.2, 0.3, 0.1
    x, y, old, adv, ref, g = policy_inputs(B, T, V, dtype, V + 1, low, high)
    mask = torch.rand(B, T, device="cuda", generator=g) < 0.6
    mask[0, 0], mask[2] = True, False  # a sequence without a counted row
    log(f"policy V={V} {dtype} seq={seq}")
    stats, logp, grad, scale, size, onehot, p = policy_reference(x, y, V, old, adv, ref, mask, low, high, kl, seq, 1.0)
    for t in (x, old, adv, ref):
        t[~mask] = math.nan  # not read
    got = fal.policy_loss(x, y, old, adv, ref_logp=ref, mask=mask, clip_low=low, clip_high=high, kl_coef=kl,
                          sequence_mean=seq)
    e = err_lse(torch.where(mask[:, :, None], x, 0.0), V, 1.0)
    within("logp", got.logp, torch.where(mask, logp, 0.0), e + 2 * U * logp.abs())
    ec = torch.where(mask, scale, 0.0)[:, :, None] * (e + 8 * U)
    bound = ec * (onehot + p) + (e + 4 * U) * grad.abs() + ec * p + (R if dtype == BF16 else U) * grad.abs() * 1.02
    assert not got.dlogits[~mask].any()
    within("dlogits", got.dlogits, torch.where(mask[:, :, None], grad, 0.0), bound)
    total = float(torch.where(mask, scale, 0.0).sum()) * (e + 8 * U) + U * stats.abs()
    within("stats", got.stats, stats, total + 2 * float(torch.where(mask, size, 0.0).sum()) * U)


def test_policy_parts():
    # no reference: no KL; every ratio one: the next-token gradient
    B, T, V = 2, 6, 300
    x, y, g = rows(B, T, V, F32, seed=5)
    old = fal.token_logprobs(x, y)
    one = torch.ones(B, T, device="cuda")
    got = fal.policy_loss(x, y, old, one)
    lp, logp = exact(x, y, V, 1.0)
    onehot = torch.zeros_like(lp).scatter_(-1, y.long()[:, :, None], 1.0)
    e = err_lse(x, V, 1.0)
    within("dlogits", got.dlogits, (lp.exp() - onehot) / (B * T), (lp.exp() + onehot) * (2 * e + 8 * U) / (B * T))
    assert abs(float(got.stats[0]) + 1) <= 2 * e + 4 * U and float(got.stats[2]) == 0 and float(got.stats[3]) == 0
    # nothing counted: zeros, not NaN
    got = fal.policy_loss(x, y, old, one, mask=torch.zeros(B, T, dtype=torch.bool, device="cuda"), ref_logp=old)
    assert not got.stats.any() and not got.dlogits.any() and not got.logp.any()


def test_policy_extreme_ratios():
    # a ratio that overflows under a positive advantage is held by the clip,
    # and a zero advantage adds nothing to it; -inf logits have probability 0
    x, y, g = rows(1, 4, 50, F32, seed=6)
    x[0, :, 10:20] = -math.inf
    x[0, 3] = torch.finfo(F32).min
    y.fill_(3)
    old = fal.token_logprobs(x, y)
    old[0, 0] -= 200.0
    old[0, 1] -= 200.0
    adv = torch.tensor([[1.0, 0.0, 1.0, 1.0]], device="cuda")
    got = fal.policy_loss(x, y, old, adv, clip_low=0.2, clip_high=0.3)
    assert torch.isfinite(got.stats).all() and torch.isfinite(got.dlogits).all()
    assert not got.dlogits[0, :2].any() and not got.dlogits[0, :3, 10:20].any()
    # loss: -(1.3 + 0 + 1 + 1) / 4
    assert abs(float(got.stats[0]) + 3.3 / 4) <= 1e-5
    assert float(got.stats[3]) == 0.25
    # a row of equal lowest values is a uniform row
    assert abs(float(got.logp[0, 3]) + math.log(50)) <= 1e-5


def preference_reference(x, y, V, ref, mask, beta, smooth, ipo, mean, temp):
    lp, logp = exact(x, y, V, temp)
    leaf = logp.clone().requires_grad_()
    n = mask.sum(-1).double()
    seq = torch.where(mask, leaf, 0.0).sum(-1)
    if mean:
        seq = seq / n.clamp(min=1)
    P = x.shape[0] // 2
    gain = seq - ref.double()
    h = gain[:P] - gain[P:]
    if ipo:
        loss = ((h - 0.5 / beta) ** 2).mean()
    else:
        f = torch.nn.functional.logsigmoid
        loss = (-(1 - smooth) * f(beta * h) - smooth * f(-beta * h)).mean()
    loss.backward()
    c = torch.where(mask, leaf.grad, 0.0)
    onehot = torch.zeros_like(lp).scatter_(-1, y.long()[:, :, None], 1.0)
    return loss.detach(), seq.detach(), c, c[:, :, None] / temp * (onehot - lp.exp()), onehot, lp.exp(), h.detach()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("ipo,mean,smooth", [(False, False, 0.0), (False, True, 0.1), (True, False, 0.0),
                                             (True, True, 0.0)])
@pytest.mark.parametrize("B,T,V", [(2, 1, 9), (4, 33, 257), (6, 9, 5000), (2, 70, 50257), (2, 3, 140003)])
def test_preference_loss(B, T, V, ipo, mean, smooth, dtype):
    beta, temp = 0.3, 1.0
    x, y, g = rows(B, T, V, dtype, seed=B * T + V)
    mask = torch.rand(B, T, device="cuda", generator=g) < 0.6
    mask[0, 0] = True
    if B > 4:
        mask[5] = False  # an empty sequence
    _, logp = exact(x, y, V, temp)
    n = mask.sum(-1).clamp(min=1)
    ref = (torch.where(mask, logp, 0.0).sum(-1) / (n if mean else 1)).float()
    ref = ref + torch.randn(B, device="cuda", generator=g)
    log(f"preference {B}x{T}x{V} {dtype} ipo={ipo} mean={mean}")
    loss, seq, c, grad, onehot, p, h = preference_reference(x, y, V, ref, mask, beta, smooth, ipo, mean, temp)
    x[~mask] = math.inf
    got = fal.preference_loss(x, y, ref, mask=mask, beta=beta, label_smoothing=smooth, ipo=ipo, length_mean=mean)
    e = err_lse(torch.where(mask[:, :, None], x, 0.0), V, temp) + 2 * U * float(logp.abs().max())
    e_seq = (mask.sum(-1) * e / (n if mean else 1)).double() + U * seq.abs()
    within("seq_logp", got.seq_logp, seq, e_seq + 1e-12)
    P = B // 2
    e_h = float((e_seq[:P] + e_seq[P:]).max()) + U * float(ref.abs().max())
    slope = 2.0 * float((h - 0.5 / beta).abs().max()) if ipo else beta
    within("loss", got.loss, loss.reshape(1), torch.tensor(slope * e_h + e_h ** 2 + 4 * U * float(loss), device="cuda"))
    curve = 2.0 if ipo else beta * beta / 4  # the largest second derivative
    share = (mask / (n[:, None] if mean else 1)).double()
    ec = ((curve * e_h / P + 4 * U * slope / P) * share)[:, :, None]
    bound = ec * (onehot + p) + (2 * e + 4 * U) * grad.abs() + c.abs()[:, :, None] * p * e
    bound = bound + (R if dtype == BF16 else U) * (grad.abs() * 1.02 + ec)
    assert not got.dlogits[~mask].any()
    within("dlogits", got.dlogits, torch.where(mask[:, :, None], grad, 0.0), bound)


def test_preference_of_impossible_answers():
    # a token of probability zero in one sequence of a pair: an infinite
    # margin, of loss 0 where the model is right and infinite where not
    x, y, _ = rows(4, 2, 30, F32, seed=8)
    y.fill_(3)
    x[2, 1, 3] = -math.inf  # rejected sequence of pair 0
    ref = torch.zeros(4, device="cuda")
    got = fal.preference_loss(x, y, ref)
    lp, logp = exact(x, y, 30, 1.0)
    h = float(logp[1].sum() - logp[3].sum())
    assert abs(float(got.loss) - math.log1p(math.exp(-0.1 * h)) / 2) <= 1e-6
    assert float(got.seq_logp[2]) == -math.inf and torch.isfinite(got.dlogits).all()
    assert not got.dlogits[0].any() and not got.dlogits[2].any()
    x[0, 0, 3], x[2, 1, 3] = -math.inf, 0.0
    got = fal.preference_loss(x, y, ref)
    assert float(got.loss) == math.inf and torch.isfinite(got.dlogits).all() and got.dlogits[0, 1].any()


@pytest.mark.parametrize("temperature", [1e-38, 1e-3, 1e3, 1e38])
def test_extreme_temperatures(temperature):
    x, y, _ = rows(1, 3, 200, F32, seed=15)
    y[0, 0] = int(x[0, 0].argmax())
    logp, ent = fal.token_logprobs(x, y, temperature=temperature, entropy=True)
    lp = (x.double() / float(torch.tensor(temperature))).log_softmax(-1)
    want = lp.gather(-1, y.long()[:, :, None])[:, :, 0].float()
    h = -torch.where(lp.exp() > 0, lp.exp() * lp, 0.0).sum(-1)
    # x / temperature is off by 4 u of itself; sums as in the header
    e = 8 * U * x.double().abs().max() / temperature + (200 / 256 + 24) * U
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(logp), fine)
    assert bool(((logp - want)[fine].abs().double() <= e).all())
    assert bool((ent.double() - h).abs().max() <= e * 6) and not torch.isnan(ent).any()


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_gradients_against_differences(kind):
    B, T, V = 2, 5, 40
    x, y, old, adv, ref, g = policy_inputs(B, T, V, F32, 9, 0.2, 0.3)
    mask = torch.ones(B, T, dtype=torch.bool, device="cuda")
    mask[1, 3:] = False
    step = torch.randn(x.shape, device="cuda", generator=g).double()
    temp = 0.7

    def value(z):
        if kind == "policy":
            return float(policy_reference(z, y, V, old, adv, ref, mask, 0.2, 0.3, 0.1, True, temp)[0][0])
        return float(preference_reference(z, y, V, ref[:, 0], mask, 0.2, 0.1, False, False, temp)[0])

    if kind == "policy":
        got = fal.policy_loss(x, y, old, adv, ref_logp=ref, mask=mask, clip_low=0.2, clip_high=0.3, kl_coef=0.1,
                              sequence_mean=True, temperature=temp)
    else:
        got = fal.preference_loss(x, y, ref[:, 0].contiguous(), mask=mask, beta=0.2, label_smoothing=0.1,
                                  temperature=temp)
    h = 1e-5  # truncation h^2 and 64-bit rounding 1e-16 / h, both under 1e-9
    slope = (value(x.double() + h * step) - value(x.double() - h * step)) / (2 * h)
    d = got.dlogits.double()
    have = float((d * step).sum())
    # fp32: an element is off by the e of the header relative to its own terms
    allowed = 4 * err_lse(x, V, temp) * float((d.abs() * step.abs()).sum()) + 1e-8
    log(f"{kind}: slope {slope:.9f}, gradient {have:.9f}, allowed {allowed:.1e}")
    assert abs(have - slope) <= allowed


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("V,width", [(300, 320), (1001, 1001), (1001, 1024), (50257, 50304), (50257, 50257)])
def test_padding_strides_and_in_place(V, width, dtype):
    # the padded columns of the gradient are zeros, what lies past the width
    # and between rows stays, targets may be a view of longer rows, and the
    # gradient may take the logits' place
    B, T = 2, 6
    x, _, g = rows(B, T, V, dtype, seed=V + width, width=width)
    tokens = torch.randint(0, V, (B, T + 1), device="cuda", generator=g, dtype=torch.int32)
    y = tokens[:, 1:]
    old = fal.token_logprobs(x, y, vocab=V)
    adv = torch.randn(B, T, device="cuda", generator=g)
    mask = torch.tensor([[1, 1, 0, 1, 1, 1], [0, 0, 1, 1, 0, 1]], dtype=torch.bool, device="cuda")
    want = fal.policy_loss(x, y, old, adv, mask=mask, vocab=V)
    assert not want.dlogits[:, :, V:].any()
    for ld, shift in ((width + 7, 0), (width + 24, 3), (width + 1, 1)):
        buf = torch.full((B, T, ld + shift), 9.0, dtype=dtype, device="cuda")
        out = torch.full((B, T, ld + shift), 4.0, dtype=dtype, device="cuda")
        view, grad = buf[:, :, shift:shift + width], out[:, :, shift:shift + width]
        view.copy_(x)
        got = fal.policy_loss(view, y, old, adv, mask=mask, vocab=V, dlogits=grad)
        within("dlogits at another stride", got.dlogits, want.dlogits.double(),
               (R if dtype == BF16 else 1e-5) * want.dlogits.double().abs() * 2 + 1e-12)
        assert bool((out[:, :, :shift] == 4).all()) and bool((out[:, :, shift + width:] == 4).all())
        # in the logits' place
        ours = fal.policy_loss(view, y, old, adv, mask=mask, vocab=V, dlogits=view)
        assert torch.equal(ours.dlogits, got.dlogits) and torch.equal(ours.stats, got.stats)
        assert bool((buf[:, :, :shift] == 9).all()) and bool((buf[:, :, shift + width:] == 9).all())
        ref = torch.zeros(B, device="cuda")
        view.copy_(x)
        a = fal.preference_loss(view, y, ref, mask=mask, vocab=V)
        b = fal.preference_loss(view, y, ref, mask=mask, vocab=V, dlogits=view)
        assert torch.equal(a.dlogits, b.dlogits) and torch.equal(a.loss, b.loss)
    # a gradient of another alignment than the logits'
    out = torch.full((B, T, width + 5), 4.0, dtype=dtype, device="cuda")[:, :, 1:1 + width]
    got = fal.policy_loss(x, y, old, adv, mask=mask, vocab=V, dlogits=out)
    within("dlogits at another alignment", got.dlogits, want.dlogits.double(),
           (R if dtype == BF16 else 1e-5) * want.dlogits.double().abs() * 2 + 1e-12)


def test_offsets_past_32_bits():
    B, T, V, ld = 1, 1100, 40, 1 << 21
    buf = torch.empty(T * ld, dtype=BF16, device="cuda").view(B, T, ld)
    x, y, g = rows(B, T, V, BF16, seed=13)
    far = buf[:, :, :V]
    far.copy_(x)
    old = fal.token_logprobs(far, y)
    assert torch.equal(old, fal.token_logprobs(x, y))
    adv = torch.randn(B, T, device="cuda", generator=g)
    want = fal.policy_loss(x, y, old, adv)
    got = fal.policy_loss(far, y, old, adv, dlogits=far)
    assert torch.equal(got.dlogits, want.dlogits) and torch.equal(got.stats, want.stats)


def test_targets_outside_the_vocabulary_are_clamped():
    x, y, _ = rows(1, 4, 100, F32, seed=14)
    y[0] = torch.tensor([-5, 100, 2 ** 31 - 1, 99], dtype=torch.int32)
    z = torch.tensor([[0, 99, 99, 99]], dtype=torch.int32, device="cuda")
    assert torch.equal(fal.token_logprobs(x, y), fal.token_logprobs(x, z))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_repeats_streams_and_graphs(dtype):
    B, T, V = 4, 50, 3001
    data = []
    for seed in (41, 42):
        x, y, old, adv, ref, g = policy_inputs(B, T, V, dtype, seed, 0.2, 0.2)
        data.append((x, y, old, adv, ref, torch.rand(B, T, device="cuda", generator=g) < 0.5))

    def all_three(x, y, old, adv, ref, mask):
        a = fal.policy_loss(x, y, old, adv, ref_logp=ref, mask=mask, kl_coef=0.1)
        b = fal.preference_loss(x, y, ref[:, 0].contiguous(), mask=mask)
        return [*a, *b, *fal.token_logprobs(x, y, mask=mask, entropy=True)]

    eager = [all_three(*d) for d in data]
    torch.cuda.synchronize()
    got = []
    for d in data:
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            got.append(all_three(*d))
    torch.cuda.synchronize()
    for a, b in zip(eager, got):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    graphs, static = [], []
    for d in data:
        s = [t.clone() for t in d]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = all_three(*s)
        graphs.append(graph)
        static.append((s, held))
    for turn in range(3):
        for i in (0, 1):
            for dst, src in zip(static[i][0], data[(i + turn) % 2]):
                dst.copy_(src)
        for graph in graphs:
            graph.replay()
        again = all_three(*data[turn % 2])
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(p, q) for p, q in zip(static[i][1], eager[(i + turn) % 2]))
        assert all(torch.equal(p, q) for p, q in zip(again, eager[turn % 2]))


def test_rows_past_one_axis_of_the_grid():
    """2^21 + 6 rows, whose last ones lie in the grid's second row: sampled
    rows on both sides against the formula, gradients in place."""
    B, T, V = 2, (1 << 20) + 3, 4104
    g = torch.Generator(device="cuda").manual_seed(11)
    x = torch.empty(B, T, V, dtype=BF16, device="cuda").normal_(generator=g).mul_(3)
    y = torch.randint(0, V, (B, T), device="cuda", generator=g, dtype=torch.int32)
    at = ([0] * 4 + [1] * 12, [0, 1, T // 2, T - 1, 0, 1, *range(T - 10, T)])
    taken, ty = x[at][None].clone(), y[at][None]
    log(f"logprobs, policy and preference, {B * T} rows")
    lp, want = exact(taken, ty, V, 1.0)
    e = err_lse(taken, V, 1.0)
    logp = fal.token_logprobs(x, y)
    within("logp", logp[at][None], want, e + 2 * U * want.abs())
    onehot, p = torch.zeros_like(lp).scatter_(-1, ty.long()[:, :, None], 1.0), lp.exp()

    def check(name, got, c, ec):
        grad = c[:, :, None] * (onehot - p)
        within(name, got[at][None], grad, ec[:, :, None] * (onehot + p) + c.abs()[:, :, None] * p * (e + 4 * U)
               + 1.02 * R * grad.abs())

    adv = torch.randn(B, T, device="cuda", generator=g)
    a = adv[at][None].double() / (B * T)
    # the ratio is that of a row with itself: one to the last bit or two
    got = fal.policy_loss(x, y, logp.clone(), adv, clip_low=0.2, clip_high=0.2, dlogits=x)
    assert torch.equal(got.logp, logp)
    check("policy dlogits", got.dlogits, -a, a.abs() * 8 * U)

    x.normal_(generator=g).mul_(3)
    taken = x[at][None].clone()
    lp, _ = exact(taken, ty, V, 1.0)
    e, p = err_lse(taken, V, 1.0), lp.exp()
    beta, ref = 0.5, torch.tensor([-9.0, -9.5], device="cuda")
    got = fal.preference_loss(x, y, ref, beta=beta, length_mean=True, dlogits=x)
    gain = got.seq_logp.double() - ref.double()
    dh = beta * float(torch.sigmoid(beta * (gain[0] - gain[1])) - 1) / T
    # the means come back rounded: u |mean| each, times a slope of at most beta^2 / 4
    moved = beta * beta / 4 * U * float(got.seq_logp.double().abs().sum()) / T
    c = torch.tensor([dh, -dh], dtype=torch.float64, device="cuda")[at[0]][None]
    check("preference dlogits", got.dlogits, c, c.abs() * 4 * U + moved)
