"""Host-only checks of the entry points of a gated block: every refusal comes
back with its status and a message before anything is launched, and the
workspace sizes are what the header says."""
import ctypes
from ctypes import byref, c_void_p

import pytest
import torch

from paper_2510_14614_amd import fal

# addresses that no call may reach: 1 GiB apart, 256-byte aligned
A, B, C, D, E, F, G, H, I, J, K, L_ = (c_void_p((i + 1) << 30) for i in range(12))
BAD, UNSUP, WS = fal.FAL_ERR_INVALID_ARG, fal.FAL_ERR_UNSUPPORTED, fal.FAL_ERR_WORKSPACE


def off(p, n):
    return c_void_p(p.value + n)


def message():
    return fal.lib().fal_last_error(None).decode()


def refused(call, args, base, status, word):
    """call refuses args changed at some places (index -> value)."""
    full = list(base)
    for i, v in args.items():
        full[i] = v
    assert call(*full) == status
    assert word in message(), message()


# ---------------------------------------------------------------- head norms --
def norm(**kw):
    v = dict(batch=2, seq_len=300, n_head=4, n_kv_head=2, head_dim=64, dtype=1, rotary_dim=64, interleaved=0,
             theta=10000.0, eps=1e-6, ld_qkv=512, ld_out=520)
    v.update(kw)
    return fal.fal_qk_norm_rope_t(**v)


def norm_bytes(s):
    n = ctypes.c_size_t()
    assert fal.lib().fal_qk_norm_rope_workspace_bytes(byref(s), byref(n)) == fal.FAL_OK
    return n.value


@pytest.mark.parametrize("kw,status,word", [
    (dict(batch=0), BAD, "batch"), (dict(seq_len=0), BAD, "seq_len"), (dict(batch=1 << 16, seq_len=1 << 15), BAD, "2^31"),
    (dict(n_head=0), BAD, "n_head"), (dict(n_head=65536), BAD, "n_head"), (dict(n_kv_head=3), BAD, "n_kv_head"),
    (dict(n_kv_head=-1), BAD, "n_kv_head"), (dict(head_dim=48), UNSUP, "head_dim"), (dict(dtype=2), BAD, "dtype"),
    (dict(rotary_dim=-8), BAD, "rotary_dim"), (dict(rotary_dim=72), BAD, "rotary_dim"),
    (dict(rotary_dim=20), UNSUP, "rotary_dim"), (dict(interleaved=2), BAD, "interleaved"),
    (dict(theta=1.0), BAD, "theta"), (dict(theta=float("inf")), BAD, "theta"), (dict(theta=float("nan")), BAD, "theta"),
    (dict(eps=0.0), BAD, "eps"), (dict(eps=float("nan")), BAD, "eps"), (dict(ld_qkv=504), BAD, "smaller"),
    (dict(ld_out=504), BAD, "smaller"), (dict(ld_qkv=516), BAD, "16 bytes"), (dict(ld_out=1 << 41), BAD, "address space"),
    (dict(ld_out=1 << 39), BAD, "address space"),
])
def test_head_norms_refuse_a_shape(kw, status, word):
    L, s, n = fal.lib(), norm(**kw), ctypes.c_size_t()
    assert L.fal_qk_norm_rope_workspace_bytes(byref(s), byref(n)) == status
    assert word in message()
    assert L.fal_qk_norm_rope_fwd(byref(s), A, B, C, None, None, D, None) == status
    assert L.fal_qk_norm_rope_bwd(byref(s), A, B, C, None, None, D, E, 512, None, None, F, 1 << 30, None) == status


@pytest.mark.parametrize("args,word", [
    ({0: None}, "NULL shape"), ({1: None}, "NULL"), ({6: None}, "NULL"), ({1: off(A, 8)}, "16-byte"),
    ({6: off(D, 8)}, "16-byte"), ({2: off(B, 1)}, "misaligned"), ({4: off(E, 2)}, "misaligned"),
    ({5: off(E, 2)}, "misaligned"), ({6: A}, "overlaps"),  # another stride than qkv's
    ({6: off(A, 512)}, "overlaps"), ({6: B}, "overlaps"), ({6: C}, "overlaps"), ({4: D}, "overlaps"), ({5: D}, "overlaps"),
])
def test_head_norms_forward_refuses(args, word):
    s = norm()
    refused(fal.lib().fal_qk_norm_rope_fwd, args, [byref(s), A, B, C, E, F, D, None], BAD, word)


@pytest.mark.parametrize("args,status,word", [
    ({0: None}, BAD, "NULL shape"), ({1: None}, BAD, "NULL"), ({6: None}, BAD, "NULL"), ({7: None}, BAD, "NULL"),
    ({6: off(D, 4)}, BAD, "16-byte"), ({7: off(E, 4)}, BAD, "16-byte"), ({9: off(F, 2)}, BAD, "misaligned"),
    ({8: 511}, BAD, "smaller"), ({8: 516}, BAD, "16 bytes"), ({8: 1 << 41}, BAD, "address space"),
    ({7: D}, BAD, "overlaps"), ({7: A}, BAD, "overlap"), ({7: B}, BAD, "overlap"), ({9: D}, BAD, "overlap"),
    ({9: G}, BAD, "overlap"), ({10: E}, BAD, "overlap"), ({10: H}, BAD, "overlap"), ({11: D}, BAD, "overlap"),
    ({11: None}, WS, "workspace"), ({11: off(H, 64)}, WS, "workspace"), ({12: 1000}, WS, "workspace"),
])
def test_head_norms_backward_refuses(args, status, word):
    s = norm()
    base = [byref(s), A, B, C, I, J, D, E, 512, F, G, H, norm_bytes(s), None]
    refused(fal.lib().fal_qk_norm_rope_bwd, args, base, status, word)


def test_head_norm_workspace():
    # two rows of fp32 a workgroup of four tokens, up to 1024 workgroups
    assert norm_bytes(norm()) == 150 * 2 * 64 * 4
    assert norm_bytes(norm(batch=1, seq_len=1)) == 2 * 64 * 4
    assert norm_bytes(norm(batch=64, seq_len=8192)) == 1024 * 2 * 64 * 4
    assert fal.lib().fal_qk_norm_rope_workspace_bytes(byref(norm()), None) == BAD


def test_head_norm_binding_refuses():
    x = torch.zeros(2, 5, 512, dtype=torch.bfloat16)
    w = torch.zeros(64, dtype=torch.bfloat16)
    call = lambda t=x, **kw: fal.qk_norm_rope_fwd(t, **{"n_head": 4, "n_kv_head": 2, **kw})  # noqa: E731
    for t, kw, word in [(x[0], {}, "qkv must be"), (x.half(), {}, "bfloat16"), (x, {"n_head": 3}, "last dimension"),
                        (x, {"n_kv_head": -1}, "last dimension"), (x, {"q_weight": w[:32]}, "q_weight"),
                        (x, {"k_weight": w.float()}, "k_weight"), (x.transpose(0, 1), {}, "sequences"),
                        (x, {"positions": torch.zeros(2, 5)}, "positions"),
                        (x, {"positions": torch.zeros(2, 4, dtype=torch.int32)}, "positions"),
                        (x, {"lens": torch.zeros(3, dtype=torch.int32)}, "lens"), (x, {}, "GPU")]:
        with pytest.raises(ValueError, match=word):
            call(t, **kw)
    with pytest.raises(ValueError, match="dout"):
        fal.qk_norm_rope_bwd(x, x[:, :4], 4, n_kv_head=2)
