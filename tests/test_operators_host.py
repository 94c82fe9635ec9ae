"""Host-only checks of the windowed attention, log-probability and loss entry
points: every refusal comes back with its status and a message before anything
is launched, and the workspace sizes are what the header says."""
import ctypes
from ctypes import byref, c_void_p

import pytest
import torch

from paper_2510_14614_amd import fal

# addresses that no call may reach: 1 GiB apart, 256-byte aligned
A, B, C, D, E, F, G, H = (c_void_p((i + 1) << 30) for i in range(8))
BAD, UNSUP, WS = fal.FAL_ERR_INVALID_ARG, fal.FAL_ERR_UNSUPPORTED, fal.FAL_ERR_WORKSPACE


def off(p, n):
    return c_void_p(p.value + n)


def window(**kw):
    v = dict(batch=2, seq_len=300, n_head=4, n_kv_head=2, head_dim=64, dtype=1, window=64, sinks=4, ld_qkv=512,
             ld_out=256)
    v.update(kw)
    return fal.fal_window_attention_t(**v)


def rows(**kw):
    v = dict(batch=4, seq_len=10, vocab=100, dtype=1, ld_logits=100, ld_targets=11, ld_dlogits=104, dlogits_cols=104,
             temperature=1.0)
    v.update(kw)
    return fal.fal_logit_rows_t(**v)


def message():
    return fal.lib().fal_last_error(None).decode()


@pytest.fixture(autouse=True)
def _clear_message():
    yield
    n = ctypes.c_size_t()
    assert fal.lib().fal_window_attention_workspace_bytes(byref(window()), byref(n)) == fal.FAL_OK
    assert message() == ""


@pytest.mark.parametrize("kw,status,word", [
    (dict(batch=0), BAD, "batch"), (dict(batch=65536), BAD, "batch"), (dict(seq_len=0), BAD, "seq_len"),
    (dict(seq_len=(1 << 22) + 1), BAD, "seq_len"), (dict(n_head=0), BAD, "n_head"),
    (dict(n_kv_head=3), BAD, "n_kv_head"), (dict(n_kv_head=-1), BAD, "n_kv_head"), (dict(window=0), BAD, "window"),
    (dict(sinks=-1), BAD, "sinks"), (dict(sinks=129), UNSUP, "sinks"), (dict(head_dim=48), UNSUP, "head_dim"),
    (dict(dtype=2), BAD, "dtype"), (dict(ld_qkv=504), BAD, "ld_qkv"), (dict(ld_out=248), BAD, "ld_out"),
    (dict(ld_qkv=516), BAD, "16 bytes"), (dict(ld_out=260), BAD, "16 bytes"),
    (dict(ld_qkv=1 << 41), BAD, "2^40"),
])
def test_window_attention_refuses_a_shape(kw, status, word):
    L, s, n = fal.lib(), window(**kw), ctypes.c_size_t()
    assert L.fal_window_attention_workspace_bytes(byref(s), byref(n)) == status
    assert word in message()
    assert L.fal_window_attention_fwd(byref(s), A, None, B, C, None) == status
    assert word in message()
    assert L.fal_window_attention_bwd(byref(s), A, None, B, C, D, E, 512, F, 1 << 29, None) == status
    assert word in message()


def test_window_attention_refuses_rows_past_the_address_space():
    # 2^38 rows: products of sizes and strides that pass 64 bits
    L, n = fal.lib(), ctypes.c_size_t()
    for kw in (dict(ld_qkv=1 << 39), dict(ld_out=1 << 39), dict(ld_qkv=1 << 12), dict(ld_out=1 << 12)):
        s = window(batch=65535, seq_len=1 << 22, **kw)
        assert L.fal_window_attention_workspace_bytes(byref(s), byref(n)) == BAD
        assert "address space" in message()
        assert L.fal_window_attention_fwd(byref(s), A, None, B, C, None) == BAD
    s = window(batch=65535, seq_len=1 << 22, n_head=1, n_kv_head=1, head_dim=16, ld_qkv=48, ld_out=16)
    assert L.fal_window_attention_workspace_bytes(byref(s), byref(n)) == fal.FAL_OK
    assert L.fal_window_attention_bwd(byref(s), A, None, B, C, D, E, 1 << 39, F, 1 << 62, None) == BAD
    assert "address space" in message()


def test_window_attention_refuses_pointers():
    L, s = fal.lib(), window()
    assert L.fal_window_attention_fwd(None, A, None, B, C, None) == BAD
    for args in ((None, None, B, C), (A, None, None, C), (A, None, B, None), (off(A, 8), None, B, C),
                 (A, None, off(B, 2), C), (A, off(D, 2), B, C), (A, None, B, off(C, 1)),
                 (A, None, A, C), (A, None, off(A, 512), C), (A, None, B, off(B, 64)), (A, B, B, C)):
        assert L.fal_window_attention_fwd(byref(s), *args, None) == BAD, args
        assert message()

    def bwd(qkv=A, lens=None, out=B, d_out=C, lse=D, d_qkv=E, ld=512, ws=F, n=1 << 29):
        return L.fal_window_attention_bwd(byref(s), qkv, lens, out, d_out, lse, d_qkv, ld, ws, n, None)

    for kw in (dict(qkv=None), dict(out=None), dict(d_out=None), dict(lse=None), dict(d_qkv=None),
               dict(d_qkv=A), dict(d_qkv=C), dict(d_qkv=off(F, 256)), dict(ws=D), dict(ld=504), dict(ld=516),
               dict(ld=1 << 41), dict(d_out=off(C, 4)), dict(lse=off(D, 2))):
        assert bwd(**kw) == BAD, kw
    n = ctypes.c_size_t()
    assert L.fal_window_attention_workspace_bytes(byref(s), byref(n)) == fal.FAL_OK
    for kw in (dict(ws=None), dict(n=n.value - 1), dict(ws=off(F, 128))):
        assert bwd(**kw) == WS, kw
    assert L.fal_window_attention_workspace_bytes(byref(s), None) == BAD


def test_window_attention_workspace():
    # D = rowsum(dO * O), fp32 [B, H, T]; for sinks that later queries see
    # alone, partial sums of their dK and dV; for shared key/value heads, sums
    # of parts of their query heads
    def size(**kw):
        n = ctypes.c_size_t()
        shape = window(**{"n_kv_head": 0, "ld_qkv": 768, **kw})
        assert fal.lib().fal_window_attention_workspace_bytes(byref(shape), byref(n)) == fal.FAL_OK
        return n.value
    stat = (2 * 4 * 300 * 4 + 255) // 256 * 256
    assert size(sinks=0) == stat
    assert size(window=300) == stat  # every key in every window
    assert size() > stat
    assert (size() - stat) % (2 * 4 * 2 * 4 * 64 * 4) == 0  # whole [B, H, chunk, dK | dV, sinks, hd]
    shared = size(sinks=0, n_kv_head=1) - stat
    assert shared > 0 and shared % (2 * 300 * 2 * 64 * 4) == 0  # whole [part, B, T, dK | dV, hd]


@pytest.mark.parametrize("kw,word", [
    (dict(batch=0), "batch"), (dict(seq_len=0), "seq_len"), (dict(batch=1 << 13, seq_len=1 << 12, ld_targets=1 << 12),
                                                              "too large"),
    (dict(vocab=0), "vocab"), (dict(vocab=(1 << 20) + 1), "vocab"), (dict(dtype=-1), "dtype"),
    (dict(ld_logits=99), "ld_logits"), (dict(ld_targets=9), "ld_targets"),
    (dict(temperature=0.0), "temperature"), (dict(temperature=-1.0), "temperature"),
    (dict(temperature=float("nan")), "temperature"), (dict(temperature=float("inf")), "temperature"),
    (dict(temperature=1e-45), "temperature"), (dict(temperature=4e-39), "temperature"),
])
def test_logit_rows_refuse_a_shape(kw, word):
    L, r, n = fal.lib(), rows(**kw), ctypes.c_size_t()
    pol, pref = fal.fal_policy_t(0.2, 0.2, 0.0, 0), fal.fal_preference_t(0.1, 0.0, 0, 0)
    calls = (lambda: L.fal_token_logprobs(byref(r), A, B, None, C, None, None),
             lambda: L.fal_logit_loss_workspace_bytes(byref(r), byref(n)),
             lambda: L.fal_policy_loss(byref(r), byref(pol), A, B, None, C, None, D, E, None, F, G, 1 << 29, None),
             lambda: L.fal_preference_loss(byref(r), byref(pref), A, B, None, C, D, None, E, F, 1 << 29, None))
    for call in calls:
        assert call() == BAD
        assert word in message()


def test_logprobs_refuse_pointers():
    L, r = fal.lib(), rows()
    assert L.fal_token_logprobs(None, A, B, None, C, None, None) == BAD
    for args in ((None, B, None, C, None), (A, None, None, C, None), (A, B, None, None, None),
                 (off(A, 1), B, None, C, None), (A, off(B, 2), None, C, None), (A, B, None, off(C, 2), None),
                 (A, B, None, A, None), (A, B, None, C, C), (A, B, None, C, off(B, 4)), (A, B, C, C, None)):
        assert L.fal_token_logprobs(byref(r), *args, None) == BAD, args


@pytest.mark.parametrize("kw,word", [
    (dict(clip_low=-0.1), "clip"), (dict(clip_low=1.1), "clip"), (dict(clip_high=-0.1), "clip"),
    (dict(kl_coef=-1.0), "kl_coef"), (dict(kl_coef=float("nan")), "non-finite"),
    (dict(sequence_mean=2), "sequence_mean"),
])
def test_policy_refuses_parameters(kw, word):
    hp = fal.fal_policy_t(**{**dict(clip_low=0.2, clip_high=0.2, kl_coef=0.1, sequence_mean=0), **kw})
    assert fal.lib().fal_policy_loss(byref(rows()), byref(hp), A, B, None, C, None, D, E, None, F, G, 1 << 29,
                                     None) == BAD
    assert word in message()


@pytest.mark.parametrize("kw,word", [
    (dict(beta=0.0), "beta"), (dict(beta=float("inf")), "non-finite"), (dict(label_smoothing=0.6), "label_smoothing"),
    (dict(label_smoothing=-0.1), "label_smoothing"), (dict(ipo=2), "ipo"), (dict(length_mean=-1), "length_mean"),
    (dict(ipo=1, label_smoothing=0.1), "squared"),
])
def test_preference_refuses_parameters(kw, word):
    hp = fal.fal_preference_t(**{**dict(beta=0.1, label_smoothing=0.0, ipo=0, length_mean=0), **kw})
    assert fal.lib().fal_preference_loss(byref(rows()), byref(hp), A, B, None, C, D, None, E, F, 1 << 29, None) == BAD
    assert word in message()


def test_losses_refuse_pointers():
    L, r = fal.lib(), rows()
    pol, pref = fal.fal_policy_t(0.2, 0.2, 0.0, 0), fal.fal_preference_t(0.1, 0.0, 0, 0)
    n = ctypes.c_size_t()
    assert L.fal_logit_loss_workspace_bytes(byref(r), byref(n)) == fal.FAL_OK

    def policy(x=A, y=B, mask=None, old=C, ref=None, adv=D, stats=E, logp=None, dx=F, ws=G, size=n.value, hp=pol):
        return L.fal_policy_loss(byref(r), byref(hp) if hp else None, x, y, mask, old, ref, adv, stats, logp, dx, ws,
                                 size, None)

    def preference(x=A, y=B, mask=None, ref=C, loss=D, seq=None, dx=E, ws=F, size=n.value):
        return L.fal_preference_loss(byref(r), byref(pref), x, y, mask, ref, loss, seq, dx, ws, size, None)

    for kw in (dict(x=None), dict(y=None), dict(old=None), dict(adv=None), dict(stats=None), dict(dx=None),
               dict(hp=None), dict(x=off(A, 1)), dict(dx=off(F, 1)), dict(old=off(C, 2)), dict(stats=off(E, 2)),
               dict(dx=A),  # another row stride than the logits': not in place
               dict(dx=off(A, 200)), dict(dx=C), dict(ws=A), dict(stats=D), dict(logp=E), dict(logp=off(F, 400)),
               dict(logp=C), dict(mask=E), dict(mask=F)):
        assert policy(**kw) == BAD, kw
        assert message()
    for kw in (dict(x=None), dict(y=None), dict(ref=None), dict(loss=None), dict(dx=None), dict(dx=B), dict(loss=C),
               dict(seq=D), dict(seq=F)):
        assert preference(**kw) == BAD, kw
    for call in (policy, preference):
        for kw in (dict(ws=None), dict(size=n.value - 1), dict(ws=off(G, 4))):
            assert call(**kw) == WS, kw
    odd = rows(batch=3)
    assert L.fal_preference_loss(byref(odd), byref(pref), A, B, None, C, D, None, E, F, 1 << 29, None) == BAD
    assert "even" in message()
    for cols in (99, 105):
        short = rows(dlogits_cols=cols)
        assert L.fal_policy_loss(byref(short), byref(pol), A, B, None, C, None, D, E, None, F, G, 1 << 29, None) == BAD
        assert "dlogits_cols" in message()


def test_context_calls_refuse_null():
    L = fal.lib()
    assert L.fal_set_attention_window(None, 1, 0) == BAD
    assert L.fal_model_logprobs(None, A, B, None, 1.0, C, None) == BAD
    pol, pref = fal.fal_policy_t(0.2, 0.2, 0.0, 0), fal.fal_preference_t(0.1, 0.0, 0, 0)
    assert L.fal_policy_step(None, A, byref(pol), B, None, 1.0, C, None, D, E, None, F) == BAD
    assert L.fal_preference_step(None, A, byref(pref), B, None, 1.0, C, D, None, E) == BAD


def test_binding_checks_tensors():
    qkv = torch.zeros(2, 8, 3 * 32)
    for kw, word in ((dict(n_head=2), "GPU"), (dict(n_head=5), "last dimension"), (dict(n_head=0), "last dimension"),
                     (dict(n_head=2, lens=torch.zeros(2)), "int32"),
                     (dict(n_head=2, lens=torch.zeros(3, dtype=torch.int32)), "shape")):
        with pytest.raises(ValueError, match=word):
            fal.window_attention_fwd(qkv, window=4, **kw)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        fal.window_attention_fwd(qkv.half(), 2, 4)
    with pytest.raises(ValueError, match="B, T"):
        fal.window_attention_fwd(qkv[0], 2, 4)
    with pytest.raises(ValueError, match="contiguous in its last"):
        fal.window_attention_fwd(torch.zeros(2, 96, 8).transpose(1, 2), 2, 4)
    with pytest.raises(ValueError, match="follow each other"):
        fal.window_attention_fwd(torch.zeros(2, 9, 96)[:, :8], 2, 4)
    x, y = torch.zeros(2, 3, 10), torch.zeros(2, 3, dtype=torch.int32)
    f = torch.zeros(2, 3)
    for args, kw, word in (((x, y.long()), {}, "targets"), ((x, y[:, :2]), {}, "targets"), ((x[0], y), {}, "logits"),
                           ((x, y), dict(vocab=11), "vocab"), ((x, y), dict(mask=f), "mask"), ((x, y), {}, "GPU")):
        with pytest.raises(ValueError, match=word):
            fal.token_logprobs(*args, **kw)
    for args, kw, word in (((x, y, f[:1], f), {}, "old_logp"), ((x, y, f, f.double()), {}, "advantages"),
                           ((x, y, f, f), dict(ref_logp=f[0]), "ref_logp")):
        with pytest.raises(ValueError, match=word):
            fal.policy_loss(*args, **kw)
    with pytest.raises(ValueError, match="ref_logp"):
        fal.preference_loss(x, y, f)
