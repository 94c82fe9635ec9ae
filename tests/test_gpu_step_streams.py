"""Tuning steps of a context whose stream is not the caller's: what a call
reads, and what it returns, stays allocated until both streams are done with
it.  The tests look at the addresses that the allocator hands out while one
stream is kept busy; nothing is written in between."""
import pytest
import torch

from paper_2510_14614_amd import fal, get_config, synth

pytestmark = pytest.mark.gpu

BUSY = 100_000_000  # cycles of a kernel that only waits: tens of ms


def context(side):
    cfg = get_config("tiny", batch=4, seq_len=70)
    g, blocks = synth.make_params(cfg, seed=1)
    F = fal.Fal(cfg, stream_main=side)
    F.load_params(g, blocks)
    tok = torch.from_numpy(synth.make_tokens(cfg, seed=2)).cuda()
    torch.cuda.synchronize()
    return F, tok


def inputs(tok):
    """Tensors of their own, as a caller's temporaries are."""
    B, T = tok.shape[0], tok.shape[1] - 1
    return dict(tokens=tok.clone(), mask=torch.ones(B, T, dtype=torch.bool, device="cuda"),
                old=torch.zeros(B, T, device="cuda"), adv=torch.ones(B, T, device="cuda"),
                ref=torch.zeros(B, T, device="cuda"), seq=torch.zeros(B, device="cuda"))


CALLS = {
    "model_logprobs": lambda F, t: F.model_logprobs(t["tokens"], mask=t["mask"], entropy=True),
    "policy_step": lambda F, t: F.policy_step(t["tokens"], t["old"], t["adv"], ref_logp=t["ref"], mask=t["mask"]),
    "preference_step": lambda F, t: F.preference_step(t["tokens"], t["seq"], mask=t["mask"]),
    "model_step": lambda F, t: F.model_step(t["tokens"]),
    "model_forward": lambda F, t: F.model_forward(t["tokens"]),
}
USED = {"model_logprobs": ("tokens", "mask"), "policy_step": ("tokens", "mask", "old", "adv", "ref"),
        "preference_step": ("tokens", "mask", "seq"), "model_step": ("tokens",), "model_forward": ("tokens",)}


@pytest.mark.parametrize("call", list(CALLS))
def test_inputs_stay_until_the_step_has_read_them(call):
    side = torch.cuda.Stream()
    F, tok = context(side)
    CALLS[call](F, inputs(tok))
    torch.cuda.synchronize()
    t = inputs(tok)
    spec = [(t[k].shape, t[k].dtype) for k in USED[call]]
    read = {t[k].data_ptr() for k in USED[call]}
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    CALLS[call](F, t)
    del t
    again = [torch.empty(s, dtype=d, device="cuda") for s, d in spec for _ in range(4)]
    assert not side.query()  # the step still waits
    assert not read & {x.data_ptr() for x in again}
    torch.cuda.synchronize()
    F.close()


@pytest.mark.parametrize("call", ["model_logprobs", "policy_step"])
def test_results_stay_until_the_caller_has_read_them(call):
    side = torch.cuda.Stream()
    F, tok = context(side)
    t = inputs(tok)
    torch.cuda.synchronize()
    got = CALLS[call](F, t)
    shapes, held = [tuple(x.shape) for x in got], {x.data_ptr() for x in got}
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(BUSY)  # what reads them on the caller's stream
    del got
    again = [F._empty(*s) for s in shapes for _ in range(4)]
    assert not torch.cuda.current_stream().query()
    assert not held & {x.data_ptr() for x in again}
    torch.cuda.synchronize()
    F.close()


def test_steps_refuse_overlapping_and_misaligned_arrays():
    # refused before anything is launched: a loss's rows read what the same
    # rows' outputs would have overwritten
    F, tok = context(torch.cuda.current_stream())
    t = inputs(tok)
    L, B, T = fal.lib(), *t["mask"].shape
    p = {k: v.data_ptr() for k, v in t.items()}
    out, seq = torch.empty(B, T, device="cuda"), torch.empty(B, device="cuda")
    o, s, st = out.data_ptr(), seq.data_ptr(), torch.empty(4, device="cuda")
    P, G = F.params.data_ptr(), F.grads.data_ptr()
    pol, pref = fal.fal_policy_t(0.2, 0.2, 0.1, 0), fal.fal_preference_t(0.1, 0.0, 0, 0)
    torch.cuda.synchronize()

    def policy(old=p["old"], ref=p["ref"], adv=p["adv"], stats=st.data_ptr(), logp=o, mask=p["mask"], tokens=p["tokens"]):
        return L.fal_policy_step(F.ctx, P, fal.byref(pol), tokens, mask, 1.0, old, ref, adv, stats, logp, G)

    def preference(ref=p["seq"], loss=st.data_ptr(), seq=s, mask=p["mask"]):
        return L.fal_preference_step(F.ctx, P, fal.byref(pref), p["tokens"], mask, 1.0, ref, loss, seq, G)

    def scores(logp=o, entropy=None, mask=p["mask"]):
        return L.fal_model_logprobs(F.ctx, P, p["tokens"], mask, 1.0, logp, entropy)

    for call, kws in ((policy, (dict(logp=p["old"]), dict(logp=p["adv"]), dict(logp=p["ref"]), dict(stats=p["adv"]),
                                dict(logp=st.data_ptr()), dict(logp=G), dict(stats=P), dict(logp=p["tokens"]),
                                dict(mask=o), dict(old=p["old"] + 2), dict(logp=o + 1), dict(tokens=p["tokens"] + 1))),
                      (preference, (dict(seq=p["seq"]), dict(loss=s), dict(loss=p["seq"] + 4), dict(mask=s),
                                    dict(seq=s + 2), dict(loss=G))),
                      (scores, (dict(entropy=o), dict(entropy=o + 4), dict(logp=p["tokens"]), dict(mask=o),
                                dict(logp=o + 2)))):
        for kw in kws:
            assert call(**kw) == fal.FAL_ERR_INVALID_ARG, (call.__name__, kw)
            assert L.fal_last_error(F.ctx)
        assert call() == fal.FAL_OK
    torch.cuda.synchronize()
    F.close()
