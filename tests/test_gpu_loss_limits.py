"""Log-probabilities and tuning losses at their limits: terms of no weight that
are infinite, saturated margins, NaN scores, errors that add up over many
rows, batches of very many sequences and rows of every held width."""
import math

import pytest
import torch

from paper_2510_14614_amd import fal

import test_gpu_logit_losses as losses
from gpu_helpers import log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U, R = 2.0 ** -24, 2.0 ** -8  # half a step of fp32 and of bf16


def rows(B, T, V, dtype, seed, scale=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(B, T, V, device="cuda", generator=g) * scale).to(dtype)
    return x, torch.randint(0, V, (B, T), device="cuda", generator=g, dtype=torch.int32), g


def exact(x, y, temp=1.0):
    lp = (x.double() / temp).log_softmax(-1)
    return lp, lp.gather(-1, y.long()[:, :, None])[:, :, 0]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_a_kl_term_without_weight_adds_nothing(dtype):
    # a reference given for its statistic alone (kl_coef 0), infinitely far
    # from the policy in some rows: e^d overflows, a token that the policy
    # cannot give, one that the reference cannot
    x, y, g = rows(1, 8, 50, dtype, seed=1)
    y.fill_(3)
    x[0, 1, 3] = -math.inf
    old = fal.token_logprobs(x, y)
    old[0, 1] = -4.0
    ref = old.clone()
    ref[0, 0] += 120.0
    ref[0, 2] = -math.inf
    adv = torch.randn(1, 8, device="cuda", generator=g)
    want = fal.policy_loss(x, y, old, adv)
    got = fal.policy_loss(x, y, old, adv, ref_logp=ref)
    assert torch.isfinite(want.dlogits).all() and torch.equal(got.dlogits, want.dlogits)
    assert torch.equal(got.stats[[0, 1, 3]], want.stats[[0, 1, 3]]) and torch.isfinite(got.stats[0])
    assert float(got.stats[2]) == math.inf


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("temperature", [1.0, 0.7])
def test_errors_of_many_rows_do_not_add_up(temperature, dtype):
    # A sequence's log-probability adds those of its rows, so what matters is
    # their mean error.  log p lies in (-64, -32), where half a step is 2^-19:
    # rounding once or twice leaves a mean error of 2^-19 / sqrt(3) *
    # sqrt(2 / N) at one standard deviation, here taken six times, and the sum of
    # exponentials one step of 2^-24.  log2(e) and ln 2 as fp32 constants would
    # move every row by 1e-8 of log p, 5e-7.
    N, V = 1 << 14, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    # scores within 3 of each other but for the target's, on a grid that both
    # types hold
    x = torch.randint(-96, 1, (1, N, V), device="cuda", generator=g).float() / 32
    x[0, :, 5] = torch.randint(-56 * 4, -40 * 4, (N,), device="cuda", generator=g).float() / 4
    x = (x * (1 if temperature == 1 else 0.75)).to(dtype)
    y = torch.full((1, N), 5, device="cuda", dtype=torch.int32)
    temp = float(torch.tensor(temperature))
    _, want = exact(x, y, temp)
    assert -64 < float(want.min()) and float(want.max()) < -32
    bound = 6 * 2.0 ** -19 / math.sqrt(3) * math.sqrt(2 / N) + U
    one = torch.ones(1, N, device="cuda")
    for name, got in (("logprobs", fal.token_logprobs(x, y, temperature=temperature)),
                      ("policy", fal.policy_loss(x, y, want.float(), one, temperature=temperature).logp)):
        mean = float((got.double() - want).mean())
        log(f"{name} {dtype} at {temperature}: mean error {mean:.2e}, bound {bound:.2e}")
        assert abs(mean) <= bound


@pytest.mark.parametrize("temperature", [1e-38, 1.0, 1e38])
def test_masked_scores_at_extreme_temperatures(temperature):
    # columns of -inf, whole chunks of them among others, have probability 0
    # whatever the scale of the exponents
    x, y, _ = rows(1, 3, 600, F32, seed=6)
    kept = x[:, :, :20].clone()
    x[:, :, 20:] = -math.inf
    y.fill_(4)
    want = fal.token_logprobs(kept, y, temperature=temperature, entropy=True)
    got = fal.token_logprobs(x, y, temperature=temperature, entropy=True)
    for a, b in zip(got, want):
        assert not torch.isnan(a).any()
        near = torch.isclose(a, b, rtol=4 * U * 24, atol=24 * U)  # another order of the sums
        assert bool((near | (a == b)).all())


@pytest.mark.parametrize("B,T,seq", [(1 << 24, 1, False), (65536, 16, False), (3, 2051, False), (1, 30000, False),
                                     (1 << 14, 1024, True), (5, 1025, True)])
def test_masks_of_many_sequences(B, T, seq):
    # the rows that a mean runs over are counted once, however they are divided
    # into sequences
    V, low, high = 4, 0.2, 0.2
    x, y, g = rows(B, T, V, BF16, seed=5)
    mask = torch.rand(B, T, device="cuda", generator=g) < 0.3
    if B > 1:
        mask[B // 2] = False  # a sequence without a counted row
    mask[0, 0] = True
    _, logp = exact(x, y)
    old = (logp - 0.1 * torch.randn(B, T, device="cuda", generator=g)).float()
    adv = torch.randn(B, T, device="cuda", generator=g)
    got = fal.policy_loss(x, y, old, adv, mask=mask, clip_low=low, clip_high=high, sequence_mean=seq)
    ratio, a = torch.exp(logp - old.double()), adv.double()
    n = mask.sum(-1, keepdim=True).double()
    w = mask / n.clamp(min=1) / B if seq else mask / n.sum().clamp(min=1)
    each = -torch.minimum(ratio * a, ratio.clamp(1 - low, 1 + high) * a) * w
    # a ratio is off by e, a term by three more roundings, all times its size; one
    # on a clip's border moves by no more than that; sums are fp64, rounded once
    e = (6 * float(x.abs().max()) + 24) * U
    bound = float(((ratio * a).abs() * w).sum()) * (e + 4 * U) + U * float(each.sum().abs())
    log(f"{B} x {T}: {int(mask.sum())} rows, loss {float(got.stats[0]):.6e}, wanted {float(each.sum()):.6e}, "
        f"error / bound {abs(float(got.stats[0]) - float(each.sum())) / bound:.3f}")
    assert abs(float(got.stats[0]) - float(each.sum())) <= bound
    assert not got.dlogits[~mask].any() and not got.logp[~mask].any()
    # a row off the clip's borders has its whole weight
    held = ((a > 0) & (ratio > 1 + high)) | ((a < 0) & (ratio < 1 - low))
    near = ((ratio - 1 - high).abs() < 1e-4) | ((ratio - 1 + low).abs() < 1e-4)
    c = torch.where(held, 0.0, -ratio * a) * w
    p = x.double().softmax(-1)
    want = c[:, :, None] * (torch.zeros_like(p).scatter_(-1, y.long()[:, :, None], 1.0) - p)
    size = c.abs()[:, :, None] * (torch.zeros_like(p).scatter_(-1, y.long()[:, :, None], 1.0) + p)
    err = (got.dlogits.double() - want).abs() - size * (2 * e + 8 * U) - 1.02 * R * want.abs()
    assert float(err[~near].max()) <= 1e-38


@pytest.mark.parametrize("beta_h", [-60.0, -5.0, 20.0, 30.0, 45.0, 80.0])
def test_gradients_of_settled_pairs(beta_h):
    # the slope beta (sigmoid(z) - 1) of a pair that the model ranks right is
    # small and no difference of numbers near one: relative accuracy at any z
    B, T, V, beta = 2, 3, 40, 0.5
    x, y, _ = rows(B, T, V, F32, seed=3)
    lp, logp = exact(x, y)
    seq = logp.sum(-1)
    ref = torch.stack((seq[0] - beta_h / beta, seq[1])).float()
    h = (seq[0] - ref[0].double()) - (seq[1] - ref[1].double())
    got = fal.preference_loss(x, y, ref, beta=beta)
    slope = -beta * torch.sigmoid(-beta * h)
    onehot = torch.zeros_like(lp).scatter_(-1, y.long()[:, :, None], 1.0)
    sign = torch.tensor([1.0, -1.0], dtype=torch.float64, device="cuda")[:, None, None]
    want = sign * slope * (onehot - lp.exp())
    # a row's log-probability and probabilities to e, h to 2 T e, the slope to
    # beta of that relative, then three roundings; the smallest step of fp32
    e = (6 * float(x.abs().max()) + 24) * U
    rel = (2 * T * beta * e + 2 * e + 4 * U) * (onehot + lp.exp()) * slope.abs()
    err = (got.dlogits.double() - want).abs()
    log(f"z = {beta_h}: worst error / bound {float((err / (rel + 2.0 ** -148)).max()):.3f}")
    assert bool((err <= rel + 2.0 ** -148).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("masked", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("V", [300, 5003, 40001])
def test_nan_scores_are_not_lost(V, masked, dtype):
    # a run of NaN as long as whole chunks of a row, among scores or among columns
    # of -inf: the row's softmax is NaN, the other rows are what they were
    x, y, g = rows(2, 3, V, dtype, seed=4)
    y.fill_(1)
    clean = fal.token_logprobs(x, y, entropy=True)
    old, adv = clean[0].clone(), torch.ones(2, 3, device="cuda")
    good = fal.policy_loss(x, y, old, adv)
    if masked:
        x[0, 1, 2:] = -math.inf
    x[0, 1, 264:296] = math.nan
    other = torch.ones(2, 3, dtype=torch.bool, device="cuda")
    other[0, 1] = False
    for a, b in zip(fal.token_logprobs(x, y, entropy=True), clean):
        assert torch.isnan(a[0, 1]) and torch.equal(a[other], b[other])
    got = fal.policy_loss(x, y, old, adv)
    assert torch.isnan(got.logp[0, 1]) and torch.isnan(got.dlogits[0, 1]).all() and torch.isnan(got.stats[0])
    assert torch.equal(got.dlogits[other], good.dlogits[other])
    got = fal.preference_loss(x, y, torch.zeros(2, device="cuda"))
    assert torch.isnan(got.loss).all() and torch.isnan(got.seq_logp[0]) and torch.isfinite(got.seq_logp[1])


@pytest.mark.parametrize("seq", [False, True], ids=["token-mean", "sequence-mean"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("V", [500, 1500, 2500, 3999, 7001, 12001, 20011, 32000, 52001])
def test_policy_rows_of_every_held_width(V, dtype, seq):
    # with the widths of the losses' own test, each number of threads a row and
    # of chunks that they hold
    losses.test_policy_loss(V, dtype, seq)
