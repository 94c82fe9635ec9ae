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


@pytest.fixture(autouse=True)
def _clear_message():
    yield
    assert fal.lib().fal_qk_norm_rope_workspace_bytes(byref(norm()), byref(ctypes.c_size_t())) == fal.FAL_OK
    assert message() == ""


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
    # two rows of fp32 a workgroup of four tokens, up to 768 workgroups
    assert norm_bytes(norm()) == 150 * 2 * 64 * 4
    assert norm_bytes(norm(batch=1, seq_len=1)) == 2 * 64 * 4
    assert norm_bytes(norm(batch=64, seq_len=8192)) == 768 * 2 * 64 * 4
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


# -------------------------------------------------------------- gated feed-forward --
def ffn(**kw):
    v = dict(rows=300, d_model=64, d_ff=128, activation=0, dtype=1, grad_dtype=1, ld_x=64, ld_y=72, ld_gate=128,
             ld_up=136, ld_down=64, ld_dx=0, ld_dgate=0, ld_dup=0, ld_ddown=0)
    v.update(kw)
    return fal.fal_gated_ffn_t(**v)


def ffn_bytes(s):
    f, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert fal.lib().fal_gated_ffn_workspace_bytes(byref(s), byref(f), byref(b)) == fal.FAL_OK
    return f.value, b.value


@pytest.mark.parametrize("kw,status,word", [
    (dict(rows=0), BAD, "rows"), (dict(d_model=0), BAD, "d_model"), (dict(d_ff=0), BAD, "d_ff"),
    (dict(d_ff=(1 << 20) + 8), BAD, "d_ff"), (dict(activation=3), BAD, "activation"), (dict(activation=-1), BAD, "activation"),
    (dict(dtype=2), BAD, "dtype"), (dict(grad_dtype=2), BAD, "grad_dtype"), (dict(dtype=0), BAD, "grad_dtype"),
    (dict(ld_x=56), BAD, "stride"), (dict(ld_y=56), BAD, "stride"), (dict(ld_gate=120), BAD, "stride"),
    (dict(ld_up=120), BAD, "stride"), (dict(ld_down=56), BAD, "stride"), (dict(ld_dx=56), BAD, "stride"),
    (dict(ld_dgate=8), BAD, "stride"), (dict(ld_dup=120), BAD, "stride"), (dict(ld_ddown=56), BAD, "stride"),
    (dict(ld_dx=-1), BAD, "stride"), (dict(ld_dx=(1 << 40) + 8), BAD, "2^40"),
    (dict(d_model=60), UNSUP, "multiples of 8"), (dict(d_ff=100), UNSUP, "multiples of 8"),
    (dict(ld_x=68), BAD, "multiples of 8"), (dict(ld_dup=132), BAD, "multiples of 8"),
    (dict(ld_x=1 << 24), UNSUP, "2 GiB"), (dict(rows=1 << 23), UNSUP, "2 GiB"), (dict(ld_down=1 << 23), UNSUP, "2 GiB"),
    (dict(dtype=0, grad_dtype=0, rows=1 << 30, d_ff=1 << 10, ld_gate=1 << 10, ld_up=1 << 10), UNSUP, "2^33"),
    (dict(dtype=0, grad_dtype=0, rows=1 << 30), UNSUP, "2^33"),
    (dict(dtype=0, grad_dtype=0, rows=1 << 30, ld_x=1 << 40), BAD, "address space"),
    (dict(dtype=0, grad_dtype=0, rows=1 << 30, ld_dx=1 << 40), BAD, "address space"),
    (dict(dtype=0, grad_dtype=0, rows=1, d_model=1 << 17, d_ff=1 << 17, ld_x=1 << 17, ld_y=1 << 17, ld_down=1 << 17,
          ld_gate=1 << 17, ld_up=1 << 17), UNSUP, "2^33"),
])
def test_gated_ffn_refuses_a_shape(kw, status, word):
    L, s, n = fal.lib(), ffn(**kw), ctypes.c_size_t()
    assert L.fal_gated_ffn_workspace_bytes(byref(s), byref(n), byref(n)) == status
    assert word in message()
    assert L.fal_gated_ffn_fwd(byref(s), A, B, C, D, E, F, G, 1 << 30, None) == status
    assert L.fal_gated_ffn_bwd(byref(s), A, B, C, D, E, F, G, H, I, J, K, 1 << 30, None) == status


@pytest.mark.parametrize("args,status,word", [
    ({0: None}, BAD, "NULL shape"), *(({i: None}, BAD, "NULL") for i in range(1, 6)),
    *(({i: off(A, 8)}, BAD, "misaligned") for i in range(1, 7)),
    *(({5: p}, BAD, "overlaps") for p in (A, B, C, D, F, G)), *(({6: p}, BAD, "overlaps") for p in (A, B, D, E, G)),
    *(({7: p}, BAD, "overlaps") for p in (A, E)),
    ({7: None}, WS, "workspace"), ({7: off(G, 64)}, WS, "workspace"), ({8: 300 * 128 * 2 - 1}, WS, "workspace"),
])
def test_gated_ffn_forward_refuses(args, status, word):
    s = ffn()
    refused(fal.lib().fal_gated_ffn_fwd, args, [byref(s), A, B, C, D, E, F, G, ffn_bytes(s)[0], None], status, word)


@pytest.mark.parametrize("args,status,word", [
    ({0: None}, BAD, "NULL shape"), *(({i: None}, BAD, "NULL") for i in range(1, 7)),
    *(({i: None}, BAD, "all be NULL") for i in (8, 9, 10)), *(({i: off(A, 4)}, BAD, "misaligned") for i in range(1, 11)),
    *(({7: p}, BAD, "overlaps") for p in (A, B, C, D, E, F, H, I, J, K)),
    *(({10: p}, BAD, "overlaps") for p in (A, B, C, D, E, F, G, H, I, K)),
    ({9: H}, BAD, "overlaps"), ({9: off(H, 128)}, BAD, "overlaps"), ({11: E}, BAD, "overlaps"),
    ({11: None}, WS, "workspace"), ({11: off(K, 64)}, WS, "workspace"), ({12: 3 * 300 * 128 * 2}, WS, "workspace"),
])
def test_gated_ffn_backward_refuses(args, status, word):
    s = ffn()
    base = [byref(s), A, B, C, D, E, F, G, H, I, J, K, ffn_bytes(s)[1], None]
    refused(fal.lib().fal_gated_ffn_bwd, args, base, status, word)


def test_gated_ffn_halves_of_one_gradient():
    """Halves of one matrix pass the overlap check; halves that run into each
    other do not."""
    L = fal.lib()
    for ld, apart, fine in ((256, 256, True), (256, 240, False), (256, 272, False), (264, 272, True), (256, 512, False)):
        s = ffn(ld_dgate=ld, ld_dup=ld)
        # a workspace that is too small is found before any launch
        args = [byref(s), A, B, C, D, E, F, G, H, off(H, apart), J, K, ffn_bytes(s)[1], None]
        if fine:
            args[4] = None  # stops the call after its first checks
            assert L.fal_gated_ffn_bwd(*args) == BAD
        else:
            assert L.fal_gated_ffn_bwd(*args) == BAD and "overlaps" in message()


def test_gated_ffn_workspace():
    r = lambda n: (n + 255) // 256 * 256  # noqa: E731
    # h; dg, du and h, and two fp32 parts of dx
    assert ffn_bytes(ffn()) == (300 * 128 * 2, 3 * 300 * 128 * 2 + 2 * 300 * 64 * 4)
    # tiles that fill the chip: dx in one launch
    big = ffn(rows=8192, d_model=2048, ld_x=2048, ld_y=2048, ld_down=2048, d_ff=2048, ld_gate=2048, ld_up=2048)
    assert ffn_bytes(big) == (8192 * 2048 * 2, 3 * 8192 * 2048 * 2)
    assert ffn_bytes(ffn(dtype=0, grad_dtype=0, d_ff=101)) == (3 * r(300 * 101 * 4),) * 2
    # four fp32 parts of y and of dx
    long = ffn(dtype=0, grad_dtype=0, d_ff=5000, ld_gate=5000, ld_up=5000)
    assert ffn_bytes(long) == (3 * r(300 * 5000 * 4) + 4 * 300 * 64 * 4,) * 2
    assert fal.lib().fal_gated_ffn_workspace_bytes(byref(ffn()), None, None) == fal.FAL_OK


def test_gated_ffn_binding_refuses():
    bf = torch.bfloat16
    x, wg, wd = torch.zeros(2, 5, 64, dtype=bf), torch.zeros(64, 128, dtype=bf), torch.zeros(128, 64, dtype=bf)
    for args, kw, word in [((x[0, 0], wg, wg, wd), {}, "x must be"), ((x, wg[0], wg, wd), {}, "x must be"),
                           ((x.half(), wg, wg, wd), {}, "bfloat16"), ((x, wg, wg, wd), {"activation": "relu"}, "activation"),
                           ((x, wg.float(), wg, wd), {}, "w_gate"), ((x, wg, wg[:, :64], wd), {}, "w_up"),
                           ((x, wg, wg, wg), {}, "w_down"), ((x, wg, wg, wg.t()), {}, "w_down"),
                           ((x.transpose(0, 1), wg, wg, wd), {}, "rows of x"), ((x, wg, wg, wd), {}, "GPU")]:
        with pytest.raises(ValueError, match=word):
            fal.gated_ffn_fwd(*args, **kw)
    saved = torch.zeros(10, 256)
    for args, kw, word in [((saved[:9], x), {}, "saved"), ((saved.double(), x), {}, "saved"), ((saved, x[:1]), {}, "dy"),
                           ((saved, x), {"dx": x.float()}, "dx"), ((saved, x), {"dw": (wg, wg)}, "dw"),
                           ((saved, x), {"dw": (wg, wg, wg)}, "dw"), ((saved, x), {"dw": (wg, wg, wd), "grads_f32": True}, "dw"),
                           ((saved, x), {}, "GPU")]:
        with pytest.raises(ValueError, match=word):
            fal.gated_ffn_bwd(x, wg, wg, wd, *args, **kw)


# --------------------------------------------------------------- orthogonal updates --
def schulz(**kw):
    v = dict(count=3, rows=100, cols=200, steps=5, dtype=1, a=3.4444, b=-4.775, c=2.0315, stride=20000, out_stride=0)
    v.update(kw)
    return fal.fal_newton_schulz_t(**v)


def muon(**kw):
    v = dict(lr=0.02, beta=0.95, weight_decay=0.01, scale=1.0, nesterov=1)
    v.update(kw)
    return fal.fal_muon_t(**v)


def schulz_bytes(s):
    n = ctypes.c_size_t()
    assert fal.lib().fal_newton_schulz_workspace_bytes(byref(s), byref(n)) == fal.FAL_OK
    return n.value


@pytest.mark.parametrize("kw,status,word", [
    (dict(count=0), BAD, "count"), (dict(count=(1 << 22) + 1), UNSUP, "2^22"), (dict(rows=0), BAD, "rows"), (dict(cols=0), BAD, "cols"), (dict(steps=0), BAD, "steps"),
    (dict(steps=33), BAD, "steps"), (dict(dtype=2), BAD, "dtype"), (dict(a=float("nan")), BAD, "finite"),
    (dict(b=float("inf")), BAD, "finite"), (dict(a=1e30), BAD, "grow"), (dict(c=10.0), BAD, "grow"),
    (dict(stride=19999), BAD, "stride"), (dict(out_stride=19999), BAD, "stride"), (dict(stride=1 << 46), BAD, "address space"),
    (dict(out_stride=1 << 46), BAD, "address space"), (dict(rows=1 << 15, cols=1 << 15), UNSUP, "2^30"),
    (dict(rows=1, cols=1 << 23), UNSUP, "2^30"),
])
def test_newton_schulz_refuses_a_shape(kw, status, word):
    L, s, n = fal.lib(), schulz(**kw), ctypes.c_size_t()
    assert L.fal_newton_schulz_workspace_bytes(byref(s), byref(n)) == status
    assert word in message()
    assert L.fal_newton_schulz(byref(s), A, B, C, 1 << 30, None) == status
    assert L.fal_muon_step(byref(s), byref(muon()), A, B, C, D, E, 1 << 30, None) == status


@pytest.mark.parametrize("args,status,word", [
    ({0: None}, BAD, "NULL shape"), ({1: None}, BAD, "NULL"), ({2: None}, BAD, "NULL"), ({1: off(A, 1)}, BAD, "misaligned"),
    ({2: off(B, 1)}, BAD, "misaligned"), ({2: off(A, 256)}, BAD, "overlaps"), ({2: C}, BAD, "overlaps"),
    ({1: off(C, 256)}, BAD, "overlaps"), ({3: None}, WS, "workspace"), ({3: off(C, 64)}, WS, "workspace"),
    ({4: 100000}, WS, "workspace"), ({0: byref(schulz(out_stride=20002)), 2: A}, BAD, "overlaps"),
])
def test_newton_schulz_refuses(args, status, word):
    s = schulz()
    refused(fal.lib().fal_newton_schulz, args, [byref(s), A, B, C, schulz_bytes(s), None], status, word)


@pytest.mark.parametrize("args,status,word", [
    ({0: None}, BAD, "NULL shape"), ({1: None}, BAD, "NULL"), *(({i: None}, BAD, "NULL") for i in (2, 4, 5)),
    *(({i: off(A, 2)}, BAD, "misaligned") for i in (2, 4, 5)), ({3: off(B, 1)}, BAD, "misaligned"),
    *(({1: byref(muon(**kw))}, BAD, word) for kw, word in (
        (dict(lr=-1.0), "lr"), (dict(lr=float("nan")), "lr"), (dict(beta=1.0), "beta"), (dict(weight_decay=-0.1), "weight_decay"),
        (dict(scale=float("inf")), "scale"), (dict(nesterov=2), "nesterov"))),
    *(({3: p}, BAD, "overlaps") for p in (A, C, D, E)), ({2: C}, BAD, "overlaps"), ({2: D}, BAD, "overlaps"),
    ({5: off(C, 128)}, BAD, "overlaps"), ({6: D}, BAD, "overlaps"), ({0: byref(schulz(out_stride=20000))}, BAD, "out_stride"),
    ({6: None}, WS, "workspace"), ({6: off(E, 64)}, WS, "workspace"), ({7: 100000}, WS, "workspace"),
])
def test_muon_refuses(args, status, word):
    s = schulz()
    refused(fal.lib().fal_muon_step, args, [byref(s), byref(muon()), A, B, C, D, E, schulz_bytes(s), None], status, word)


def test_newton_schulz_binding_refuses():
    x = torch.zeros(3, 10, 20)
    for t, kw, word in [(x[0, 0], {}, "x must be"), (x.half(), {}, "bfloat16"), (x.transpose(1, 2), {}, "contiguous"),
                        (x, {"coefficients": (1.0, 2.0)}, "three"), (x, {"steps": 0}, "GPU")]:
        with pytest.raises(ValueError, match=word):
            fal.newton_schulz(t, **kw)
    for kw, word in [({"grads": x[:2]}, "grads"), ({"grads": x.bfloat16()}, "grads"), ({"momentum": x.double()}, "momentum"),
                     ({"params": x.half()}, "params"), ({"params": torch.zeros(3, 11, 20)[:, :10]}, "params"),
                     ({"master": x.bfloat16()}, "master"), ({}, "GPU")]:
        with pytest.raises(ValueError, match=word):
            fal.muon_step(**{"master": x, "grads": x, "momentum": x, **kw})


def test_gated_ffn_refuses_more_rows_than_a_launch_has_threads():
    """fp32 rows of one column: 2^29 - 64 of them are 2^23 - 1 tiles of 64 in
    each of two products, 256 threads a tile."""
    L, n = fal.lib(), ctypes.c_size_t()
    one = dict(dtype=0, grad_dtype=0, d_model=1, d_ff=1, ld_x=1, ld_y=1, ld_gate=1, ld_up=1, ld_down=1)
    most = (1 << 29) - 64
    assert 2 * -(-most // 64) * 256 < 1 << 32 <= 2 * -(-(most + 1) // 64) * 256
    assert ffn_bytes(ffn(rows=most, **one))[0] == 3 * 4 * most
    for rows in (most + 1, 1 << 30, (1 << 31) - 1):
        s = ffn(rows=rows, **one)
        assert L.fal_gated_ffn_workspace_bytes(byref(s), byref(n), byref(n)) == UNSUP and "2^29 - 64" in message()
        assert L.fal_gated_ffn_fwd(byref(s), A, B, C, D, E, F, G, 1 << 30, None) == UNSUP
        assert L.fal_gated_ffn_bwd(byref(s), A, B, C, D, E, F, G, H, I, J, K, 1 << 30, None) == UNSUP
