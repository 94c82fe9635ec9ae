"""Log-probabilities and tuning losses at their limits: terms of no weight that
are infinite, saturated margins, NaN scores, errors that add up over many
rows, batches of very many sequences and rows of every held width."""
import math

import pytest
import torch

from paper_2510_14614_amd import fal

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
