"""The tuning path as a whole: models whose attention is windowed, scored,
trained under the policy and the preference loss and updated, through a
context, against the CPU oracle.  The oracle's attention takes the window's
mask and its head the tuning loss; everything else in it stays."""
import numpy as np
import pytest
import torch

import oracle
from oracle import fal_oracle
from paper_2510_14614_amd import fal, get_config, synth
from paper_2510_14614_amd.config import (ARCH_FAL, ARCH_FALPLUS, ARCH_GPT, ARCH_PARALLEL, SCHED_MERGED, SCHED_SEQ,
                                         SCHED_STREAMS, SCHED_STREAMS_MERGED)

from gpu_helpers import TOL, compare_step, gpu_model_step, gpu_stack_step, log, rel_err

pytestmark = pytest.mark.gpu


def masked(window, sinks):
    """The oracle's attention under the window's mask."""
    def attention(q, k, v, causal=True):
        T, d = q.shape[-2], q.shape[-1]
        s = q @ np.swapaxes(k, -1, -2) / np.sqrt(d)
        t = np.arange(T)
        see = (t[None] <= t[:, None]) & ((t[:, None] - t[None] < window) | (t[None] < sinks))
        s = np.where(see, s, -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        return p @ v, p
    return attention


def log_softmax(x):
    x = x - x.max(-1, keepdims=True)
    return x - np.log(np.exp(x).sum(-1, keepdims=True))


def policy_head(B, T, old, adv, ref, mask, low, high, kl, kept):
    def head(logits, targets):
        lp = log_softmax(logits)
        i = np.arange(len(targets))
        logp = lp[i, targets]
        m = mask.reshape(-1)
        w = m / max(m.sum(), 1)
        r = np.exp(logp - old.reshape(-1))
        a = adv.reshape(-1)
        clipped = ((a > 0) & (r > 1 + high)) | ((a < 0) & (r < 1 - low))
        d = ref.reshape(-1) - logp
        loss = (w * (-np.minimum(r * a, np.clip(r, 1 - low, 1 + high) * a) + kl * (np.exp(d) - d - 1))).sum()
        c = w * (np.where(clipped, 0.0, -r * a) + kl * (1 - np.exp(d)))
        grad = -c[:, None] * np.exp(lp)
        grad[i, targets] += c
        kept["logp"] = logp.reshape(B, T)
        return loss, grad
    return head


def preference_head(B, T, ref, mask, beta, kept):
    def head(logits, targets):
        lp = log_softmax(logits)
        i = np.arange(len(targets))
        seq = (lp[i, targets].reshape(B, T) * mask).sum(-1)
        g = seq - ref
        z = beta * (g[:B // 2] - g[B // 2:])
        loss = np.log1p(np.exp(-z)).mean()
        dh = -beta / (1 + np.exp(z)) / (B // 2)
        c = (np.concatenate([dh, -dh])[:, None] * mask).reshape(-1)
        grad = -c[:, None] * np.exp(lp)
        grad[i, targets] += c
        kept["seq"] = seq
        return loss, grad
    return head


@pytest.mark.parametrize("dtype", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("arch,sched,kw", [
    (ARCH_GPT, SCHED_SEQ, dict()), (ARCH_FAL, SCHED_SEQ, dict()), (ARCH_FAL, SCHED_MERGED, dict(n_kv_head=2)),
    (ARCH_FALPLUS, SCHED_STREAMS, dict(n_layer=3)), (ARCH_PARALLEL, SCHED_STREAMS_MERGED, dict()),
    (ARCH_FAL, SCHED_STREAMS_MERGED, dict(head_dim=64, n_head=2, d_model=128, n_layer=3, seq_len=300)),
])
def test_windowed_model_step(arch, sched, kw, dtype, monkeypatch):
    cfg = get_config("tiny", arch=arch, sched=sched, dtype=dtype, **{"seq_len": 150, **kw})
    window, sinks = 11, 3
    g, blocks = synth.make_params(cfg, seed=2)
    tok = synth.make_tokens(cfg, seed=3)
    F = fal.Fal(cfg)
    full = gpu_model_step(cfg, g, blocks, tok, ctx=F)
    F.set_attention_window(window, sinks)
    got = gpu_model_step(cfg, g, blocks, tok, ctx=F)
    again = gpu_model_step(cfg, g, blocks, tok, ctx=F)
    F.set_attention_window(0)
    back = gpu_model_step(cfg, g, blocks, tok, ctx=F)
    F.close()
    assert back["loss"] == full["loss"] and np.array_equal(back["logits"], full["logits"])
    assert not np.array_equal(got["logits"], full["logits"])
    assert np.array_equal(again["logits"], got["logits"])
    assert all(np.array_equal(a[k], b[k]) for a, b in zip(again["grads_blocks"], got["grads_blocks"]) for k in a)
    monkeypatch.setattr(fal_oracle, "attention", masked(window, sinks))
    compare_step(cfg, got, oracle.train_step(cfg, g, blocks, tok), label=f"window arch={arch} dtype={dtype}")


@pytest.mark.parametrize("dtype", [0, 1], ids=["fp32", "bf16"])
def test_windowed_stack_and_blocks(dtype, monkeypatch):
    # a block stack and its blocks one by one (a window as long as the
    # sequence there: bitwise the first's own full window)
    cfg = get_config("tiny", n_layer=3, seq_len=200, dtype=dtype, has_embed_head=0, vocab=0)
    _, blocks = synth.make_params(cfg, seed=4)
    x, dy = (synth.make_flat(cfg.tokens * cfg.d_model, seed=s).reshape(cfg.tokens, cfg.d_model) for s in (5, 6))
    F = fal.Fal(cfg)
    F.set_attention_window(40, 1)
    got = gpu_stack_step(cfg, blocks, x, dy, ctx=F)
    F.close()
    monkeypatch.setattr(fal_oracle, "attention", masked(40, 1))
    compare_step(cfg, got, oracle.stack_step(cfg, blocks, x, dy), label=f"window stack dtype={dtype}")


def test_set_attention_window_refusals():
    F = fal.Fal(get_config("tiny"))
    for window, sinks, status in ((-1, 0, fal.FAL_ERR_INVALID_ARG), (4, -1, fal.FAL_ERR_INVALID_ARG),
                                  (0, 1, fal.FAL_ERR_INVALID_ARG), (4, 129, fal.FAL_ERR_UNSUPPORTED)):
        with pytest.raises(fal.FalError) as e:
            F.set_attention_window(window, sinks)
        assert e.value.status == status
    F.close()
    F = fal.Fal(get_config("tiny", has_embed_head=0, vocab=0, bidirectional=1))
    with pytest.raises(fal.FalError, match="causal"):
        F.set_attention_window(4)
    with pytest.raises(fal.FalError, match="has_embed_head"):
        t = torch.zeros(F.cfg.batch, F.cfg.seq_len + 1, dtype=torch.int32, device="cuda")
        F.model_logprobs(t)
    F.close()
    # partial sums of 128 sinks of 520 heads exceed the context's scratch; the
    # window set before stays
    F = fal.Fal(get_config("tiny", batch=130, n_head=4, head_dim=128, seq_len=200, has_embed_head=0, vocab=0))
    F.set_attention_window(8, 2)
    with pytest.raises(fal.FalError, match="scratch"):
        F.set_attention_window(8, 128)
    F.close()
    F = fal.Fal(get_config("tiny", batch=3))
    t = torch.zeros(3, 33, dtype=torch.int32, device="cuda")
    with pytest.raises(fal.FalError, match="even"):
        F.preference_step(t, torch.zeros(3, device="cuda"))
    f = torch.zeros(3, 32, device="cuda")
    with pytest.raises(fal.FalError, match="temperature"):
        F.policy_step(t, f, f, temperature=0.0)
    with pytest.raises(fal.FalError, match="clip"):
        F.policy_step(t, f, f, clip_low=2.0)
    with pytest.raises(ValueError, match="old_logp"):
        F.policy_step(t, f[:, :3], f)
    F.close()


def test_window_refuses_a_batch_past_its_grid():
    F = fal.Fal(get_config("tiny", batch=65536, seq_len=1, has_embed_head=0, vocab=0))
    with pytest.raises(fal.FalError, match="65535") as e:
        F.set_attention_window(4)
    assert e.value.status == fal.FAL_ERR_UNSUPPORTED
    F.set_attention_window(0)
    F.close()


def _setup(arch, dtype, **kw):
    cfg = get_config("tiny", arch=arch, dtype=dtype, batch=4, seq_len=70, sched=SCHED_STREAMS, **kw)
    g, blocks = synth.make_params(cfg, seed=7)
    tok = synth.make_tokens(cfg, seed=8)
    rng = np.random.default_rng(9)
    mask = np.zeros((4, 70), dtype=bool)
    for b, (lo, hi) in enumerate(((20, 70), (0, 41), (69, 70), (30, 60))):
        mask[b, lo:hi] = True
    return cfg, g, blocks, tok, rng, mask


@pytest.mark.parametrize("dtype", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("arch", [ARCH_FAL, ARCH_GPT, ARCH_FALPLUS])
def test_windowed_policy_step(arch, dtype, monkeypatch):
    cfg, g, blocks, tok, rng, mask = _setup(arch, dtype)
    B, T, window, sinks = 4, 70, 16, 2
    F = fal.Fal(cfg)
    F.load_params(g, blocks)
    F.set_attention_window(window, sinks)
    tokens, dmask = torch.from_numpy(tok).cuda(), torch.from_numpy(mask).cuda()
    # old log-probabilities from the model itself, as a sampling pass leaves
    # them, moved a little; kept off the clip's borders
    old = F.model_logprobs(tokens)
    move = rng.normal(0, 0.3, (B, T))
    for edge in (np.log(0.8), np.log(1.3)):
        move = np.where(abs(move - edge) < 0.05, edge + 0.1, move)
    old = (old - torch.from_numpy(move).cuda()).float().contiguous()
    ref = (old + torch.from_numpy(rng.normal(0, 0.2, (B, T))).cuda()).float().contiguous()
    adv = torch.from_numpy(rng.normal(0, 1, (B, T)).astype(np.float32)).cuda()
    stats, logp = F.policy_step(tokens, old, adv, ref_logp=ref, mask=dmask, clip_low=0.2, clip_high=0.3, kl_coef=0.1)
    torch.cuda.synchronize()
    gg, gb = F.grads_numpy()
    kept = {}
    monkeypatch.setattr(fal_oracle, "attention", masked(window, sinks))
    monkeypatch.setattr(fal_oracle, "cross_entropy",
                        policy_head(B, T, *(t.double().cpu().numpy() for t in (old, adv, ref)), mask, 0.2, 0.3, 0.1,
                                    kept))
    want = oracle.train_step(cfg, g, blocks, tok)
    want["loss_scale"] = 1.0  # a sum of terms of both signs
    compare_step(cfg, {"loss": float(stats[0]), "grads_global": gg, "grads_blocks": gb}, want,
                 label=f"policy arch={arch} dtype={dtype}")
    assert rel_err(logp.cpu().numpy()[mask], kept["logp"][mask]) <= TOL[dtype]
    # a forward pass alone scores the tokens the same, bit for bit
    assert torch.equal(F.model_logprobs(tokens, mask=dmask), logp)
    F.close()


@pytest.mark.parametrize("dtype", [0, 1], ids=["fp32", "bf16"])
def test_windowed_preference_step(dtype, monkeypatch):
    cfg, g, blocks, tok, rng, mask = _setup(ARCH_FAL, dtype)
    B, T, window, sinks, beta = 4, 70, 16, 2, 0.2
    F = fal.Fal(cfg)
    F.load_params(g, blocks)
    F.set_attention_window(window, sinks)
    tokens, dmask = torch.from_numpy(tok).cuda(), torch.from_numpy(mask).cuda()
    ref = F.model_logprobs(tokens, mask=dmask).double().sum(-1) + torch.from_numpy(rng.normal(0, 2, B)).cuda()
    ref = ref.float().contiguous()
    loss, seq = F.preference_step(tokens, ref, mask=dmask, beta=beta)
    torch.cuda.synchronize()
    gg, gb = F.grads_numpy()
    kept = {}
    monkeypatch.setattr(fal_oracle, "attention", masked(window, sinks))
    monkeypatch.setattr(fal_oracle, "cross_entropy",
                        preference_head(B, T, ref.double().cpu().numpy(), mask, beta, kept))
    want = oracle.train_step(cfg, g, blocks, tok)
    compare_step(cfg, {"loss": float(loss), "grads_global": gg, "grads_blocks": gb}, want, label=f"preference {dtype}")
    assert rel_err(seq.cpu().numpy(), kept["seq"]) <= TOL[dtype]
    F.close()


@pytest.mark.parametrize("dtype", [0, 1], ids=["fp32", "bf16"])
def test_policy_step_of_ones_is_the_training_step(dtype):
    # ratio one and advantage one everywhere: the next-token gradient
    cfg, g, blocks, tok, _, _ = _setup(ARCH_FAL, dtype)
    F = fal.Fal(cfg)
    F.load_params(g, blocks)
    tokens = torch.from_numpy(tok).cuda()
    F.model_step(tokens)
    torch.cuda.synchronize()
    want = F.grads.clone()
    old = F.model_logprobs(tokens)
    F.policy_step(tokens, old, torch.ones_like(old))
    torch.cuda.synchronize()
    # gradients of the logits that are rounded to the dtype in another order
    err = float((F.grads - want).norm() / want.norm())
    log(f"policy of ones against the training step: {err:.2e}")
    assert err <= (1e-5 if dtype == 0 else 1e-2)
    F.close()


@pytest.mark.parametrize("dtype", [0, 1], ids=["fp32", "bf16"])
def test_tuning_steps_captured_and_replayed(dtype):
    # scores, a policy step, a preference step and updates in one graph,
    # replayed among eager work, against eager steps bit for bit
    cfg, g, blocks, tok, rng, mask = _setup(ARCH_FAL, dtype)
    tokens, dmask = torch.from_numpy(tok).cuda(), torch.from_numpy(mask).cuda()
    adv = torch.from_numpy(rng.normal(0, 1, (4, 70)).astype(np.float32)).cuda()
    ref = torch.zeros(4, device="cuda")
    side = torch.cuda.Stream()

    def step(F):
        old = F.model_logprobs(tokens, mask=dmask)
        stats, _ = F.policy_step(tokens, old, adv, ref_logp=old, mask=dmask, kl_coef=0.1)
        held = F.grads.clone()
        loss, seq = F.preference_step(tokens, ref, mask=dmask)
        return stats, held, loss.clone(), seq, F.grads.clone()

    with torch.cuda.stream(side):
        F = fal.Fal(cfg, stream_main=side)
        F.load_params(g, blocks)
        F.set_attention_window(16, 2)
        want = step(F)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step(F)
        for _ in range(3):
            F.grads.fill_(7.0)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            assert all(torch.equal(a, b) for a, b in zip(step(F), want))
    F.close()


def test_policy_training_runs():
    # score, step, update: three rounds of the loop, finite throughout, the
    # weights move, and the profile counts the loss and windowed attention
    cfg, g, blocks, tok, rng, mask = _setup(ARCH_FAL, 1)
    F = fal.Fal(cfg)
    F.load_params(g, blocks)
    F.set_attention_window(16, 2)
    tokens, dmask = torch.from_numpy(tok).cuda(), torch.from_numpy(mask).cuda()
    adv = torch.from_numpy(rng.normal(0, 1, (4, 70)).astype(np.float32)).cuda()
    start = F.params.clone()
    F.profile_enable(True)
    for _ in range(3):
        old = F.model_logprobs(tokens, mask=dmask)
        for _ in range(2):
            stats, _ = F.policy_step(tokens, old, adv, mask=dmask)
            norm = F.adamw_step(lr=1e-3)
            assert torch.isfinite(stats).all() and float(norm) > 0
    prof = F.profile_read()
    assert prof["cross_entropy"]["launches"] == 9 and prof["attn_bwd"]["launches"] == 6 * cfg.n_layer
    assert not torch.equal(start, F.params)
    F.close()
