"""Norms of queries and keys with the rotation of their positions, forward and
backward, against the formula in 64 bits.

Tolerances are element by element, from the roundings that the kernels make
(u = 2^-24; r = 2^-8 for bf16 storage, u for fp32):

* the mean square is a sum of hd products: 1 / sqrt of it is off by
  (hd / 2 + 4) u relative, hat = x / rms by one rounding more;
* an angle is a fp64 product of position and rate (rate off by up to 2^-48,
  an exponential and a product), reduced to at most half a turn and rounded to
  fp32 (2^-26 of a turn, 2 u), its sine and cosine off by 2 u more:
  c = 4 u + 2 pi |turns| 2^-48;
* out turns a pair (a, b): (|a| + |b|) ((hd / 2 + 8) u + c) + r |out|;
* dn turns a pair of the gradient: G (c + 2 u), G the pair's absolute sum;
* dx = (dn w - hat m) / rms with m = mean(dn w hat): each part's error times the
  other factors, and the same relative roundings;
* dw sums a wavefront's products in fp32, one after the other, the rest in
  fp64: the products' errors and (terms of a wavefront + 8) u of their sizes.
"""
import math

import pytest
import torch

from paper_2510_14614_amd import fal

from gpu_helpers import log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
EPS = 1e-6


def partner(hd, r, interleaved):
    """Each element's partner, its pair's number and the sine's sign."""
    e = torch.arange(hd)
    if interleaved:
        j, other, sign = e // 2, e ^ 1, torch.where(e % 2 == 0, -1.0, 1.0)
    else:
        half = r // 2
        j = torch.where(e < half, e, e - half)
        other, sign = torch.where(e < half, e + half, e - half), torch.where(e < half, -1.0, 1.0)
    still = e >= r
    return torch.where(still, e, other), torch.where(still, 0, j), torch.where(still, 0.0, sign), still


def rotation(shape, pos, hd, r, theta, interleaved, device):
    """cos, sin [tokens, 1, hd], the partner's index and the angles' error."""
    other, j, sign, still = (t.to(device) for t in partner(hd, r, interleaved))
    rate = theta ** (-2.0 * j.double() / max(r, 1))
    angle = pos.double().reshape(-1, 1, 1) * torch.where(still, 0.0, rate)
    return angle.cos(), angle.sin() * sign, other, 4 * U + angle.abs() * 2.0 ** -48


def formula(x, w, turn, eps=EPS):
    """out in 64 bits: x [tokens, heads, hd], w [heads, hd]."""
    c, s, other, _ = turn
    n = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w
    return n * c + n[..., other] * s


def reference(x, dout, w, turn, terms, r, eps=EPS):
    """{name: (value, bound of the error)} of out, dx and dw [heads, hd]."""
    c, s, other, ec = turn
    hd = x.shape[-1]
    rms = (x.square().mean(-1, keepdim=True) + eps).sqrt()
    hat = x / rms
    n = hat * w
    out = n * c + n[..., other] * s
    e_out = (n.abs() + n[..., other].abs()) * ((hd / 2 + 8) * U + ec) + r * out.abs()
    # the gradient turns back: the sine's sign is the partner's
    dn = dout * c + (dout * s)[..., other]
    G = dout.abs() + dout[..., other].abs()
    e_dn = G * (ec + 2 * U)
    p, P = dn * w, G * w.abs()
    m = (p * hat).mean(-1, keepdim=True)
    rel = (hd / 2 + 8) * U
    e_p = e_dn * w.abs() + 2 * U * P
    e_m = ((e_p + P * (rel + hd * U)) * hat.abs()).mean(-1, keepdim=True)
    dx = (p - hat * m) / rms
    e_dx = (e_p + hat.abs() * e_m + (P + 2 * hat.abs() * m.abs()) * rel) / rms + r * dx.abs()
    d = dn * hat
    size = G * hat.abs()
    dw = d.sum(0)
    e_dw = ((e_dn + G * rel) * hat.abs()).sum(0) + (terms + 8) * U * size.sum(0)
    return {"out": (out, e_out), "dx": (dx, e_dx), "dw": (dw, e_dw)}


def worst(got, want, bound):
    """Largest error over its bound; zero bounds ask for equality."""
    got, want, bound = got.double(), want.double(), bound.double() + 1e-300
    assert torch.isfinite(got).all()
    return float(((got - want).abs() / bound).max()) if got.numel() else 0.0


def make(seed, B, T, H, kv, hd, dtype, pad=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = (H + 2 * kv) * hd
    rows = lambda: torch.randn(B, T, width + pad, generator=g, device="cuda").mul_(scale).to(dtype)[:, :, :width]  # noqa: E731
    weight = lambda: (1 + 0.3 * torch.randn(hd, generator=g, device="cuda")).to(dtype)  # noqa: E731
    return rows(), rows(), weight(), weight()


def check(label, B, T, H, kv, hd, dtype, r=None, interleaved=False, theta=10000.0, pos=None, lens=None, pad=0,
          weights=True, scale=1.0, in_place=False, seed=0):
    qkv, dout, wq, wk = make(seed, B, T, H, kv, hd, dtype, pad, scale)
    log(f"{label}: B {B} T {T} H {H} kv {kv} hd {hd} {dtype} r {r} interleaved {interleaved}")
    width = (H + 2 * kv) * hd
    kw = dict(n_head=H, n_kv_head=0 if kv == H else kv, positions=pos, lens=lens, rotary_dim=r, theta=theta, eps=EPS,
              interleaved=interleaved, q_weight=wq if weights else None, k_weight=wk if weights else None)
    src = qkv.clone()
    if lens is not None:
        # what lies past a sequence is never read
        for b, n in enumerate(lens.tolist()):
            qkv[b, max(n, 0):] = math.nan
            dout[b, max(n, 0):] = math.nan
    if in_place:
        grads = fal.qk_norm_rope_bwd(qkv, dout, **kw)
        out, dx = qkv.clone(), dout.clone()
        fal.qk_norm_rope_fwd(out, out=out, **kw)
        again = fal.qk_norm_rope_bwd(qkv, dx, dqkv=dx, **kw)
        assert torch.equal(again.dqkv, grads.dqkv)
    else:
        out = fal.qk_norm_rope_fwd(qkv, **kw)
        grads = fal.qk_norm_rope_bwd(qkv, dout, **kw)
    turned = H + kv
    place = torch.arange(T, device="cuda").expand(B, T)
    live = torch.ones(B, T, dtype=torch.bool, device="cuda")
    if lens is not None:
        live = place < lens[:, None]
    at = (place if pos is None else pos)[live]
    assert (out[~live] == 0).all() and (grads.dqkv[~live] == 0).all()
    assert torch.equal(out[live][:, turned * hd:], src[live][:, turned * hd:])
    assert torch.equal(grads.dqkv[live][:, turned * hd:], dout[live][:, turned * hd:])
    x = qkv[live][:, :turned * hd].double().unflatten(-1, (turned, hd))
    g = dout[live][:, :turned * hd].double().unflatten(-1, (turned, hd))
    one = torch.ones(hd, device="cuda", dtype=torch.float64)
    w = torch.cat([(v.double() if weights else one).expand(n, hd) for v, n in ((wq, H), (wk, kv))])
    turn = rotation(None, at, hd, hd if r is None else r, theta, interleaved, "cuda")
    terms = math.ceil(B * T / (4 * 768)) * math.ceil(turned / (512 // hd))
    ref = reference(x, g, w, turn, terms, 2.0 ** -8 if dtype == BF16 else U)
    errs = {"out": worst(out[live][:, :turned * hd].unflatten(-1, (turned, hd)), *ref["out"]),
            "dx": worst(grads.dqkv[live][:, :turned * hd].unflatten(-1, (turned, hd)), *ref["dx"])}
    if weights:
        for name, got, s in (("dwq", grads.dq_weight, slice(0, H)), ("dwk", grads.dk_weight, slice(H, None))):
            errs[name] = worst(got, ref["dw"][0][s].sum(0), ref["dw"][1][s].sum(0))
    else:
        assert grads.dq_weight is None and grads.dk_weight is None
    log(f"  errors over their bounds: { {k: round(v, 3) for k, v in errs.items()} }")
    assert all(v <= 1 for v in errs.values()), errs
    return out, grads


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [16, 32, 64, 128])
@pytest.mark.parametrize("part", [1, 2, 0])  # of the head is turned (0: none of it)
@pytest.mark.parametrize("interleaved", [False, True])
def test_every_head_and_pairing(dtype, hd, part, interleaved):
    check("heads", 2, 37, 6, 2, hd, dtype, r=hd // part if part else 0, interleaved=interleaved, seed=hd + part)


@pytest.mark.parametrize("r", [8, 24, 40, 56, 120])
@pytest.mark.parametrize("interleaved", [False, True])
def test_odd_parts_of_a_head(r, interleaved):
    check("part", 1, 19, 3, 3, 128, F32, r=r, interleaved=interleaved, seed=r)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,H,kv", [(1, 1, 1, 1), (3, 1, 7, 7), (1, 2, 12, 1), (64, 1, 16, 2), (1, 4099, 2, 1),
                                      (5, 1700, 5, 5)])
def test_shapes(dtype, B, T, H, kv):
    check("shape", B, T, H, kv, 64, dtype, pad=64, seed=T)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_without_weights_and_in_place(dtype):
    check("no weights", 2, 33, 4, 4, 32, dtype, weights=False)
    check("in place", 2, 33, 4, 2, 64, dtype, in_place=True)


@pytest.mark.parametrize("hd", [16, 128])
def test_ragged_batches_read_nothing_past_a_sequence(hd):
    lens = torch.tensor([20, 0, 1, 300, -5, 7], dtype=torch.int32, device="cuda")
    check("ragged", 6, 20, 3, 1, hd, F32, lens=lens, pad=32)
    check("ragged in place", 6, 20, 3, 1, hd, BF16, lens=lens, in_place=True)


@pytest.mark.parametrize("top", [1000, 1000000, 2147483647])
def test_far_and_negative_positions(top):
    pos = torch.tensor([[0, 1, top // 3, top], [-1, -top, top - 1, 7]], dtype=torch.int32, device="cuda")
    check("far", 2, 4, 2, 2, 128, F32, pos=pos, theta=1e6)
    check("far", 2, 4, 2, 2, 64, F32, pos=pos, theta=1.5, interleaved=True)


@pytest.mark.parametrize("scale", [1e-6, 1e-3, 1e15])
def test_small_and_large_heads(scale):
    """Rows below eps's square root, and squares far above one."""
    check("scale", 1, 50, 2, 2, 64, F32, scale=scale)


def test_a_head_of_zeros():
    qkv, dout, wq, wk = make(1, 1, 3, 2, 2, 32, F32)
    qkv.zero_()
    kw = dict(n_head=2, q_weight=wq, k_weight=wk, eps=EPS)
    assert (fal.qk_norm_rope_fwd(qkv, **kw) == 0).all()
    g = fal.qk_norm_rope_bwd(qkv, dout, **kw)
    assert torch.isfinite(g.dqkv).all() and (g.dq_weight == 0).all() and (g.dk_weight == 0).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_against_differences(interleaved):
    """Along random directions, the change of sum(dout * out) in 64 bits."""
    B, T, H, kv, hd = 2, 9, 3, 1, 32
    qkv, dout, wq, wk = make(3, B, T, H, kv, hd, F32)
    kw = dict(n_head=H, n_kv_head=kv, q_weight=wq, k_weight=wk, eps=EPS, interleaved=interleaved)
    grads = fal.qk_norm_rope_bwd(qkv, dout, **kw)
    turn = rotation(None, torch.arange(T, device="cuda").expand(B, T).flatten(), hd, hd, 10000.0, interleaved, "cuda")
    x0 = qkv.double().reshape(B * T, H + 2 * kv, hd)
    g0 = dout.double().reshape(B * T, H + 2 * kv, hd)
    w0 = torch.stack((wq.double(), wk.double()))

    def value(x, w):
        rows = torch.cat((w[:1].expand(H, hd), w[1:].expand(kv, hd)))
        return float((formula(x[:, :H + kv], rows, turn) * g0[:, :H + kv]).sum() + (x[:, H + kv:] * g0[:, H + kv:]).sum())

    gen = torch.Generator(device="cuda").manual_seed(5)
    step = 1e-5
    for _ in range(4):
        dx = torch.randn(x0.shape, generator=gen, device="cuda", dtype=torch.float64)
        dw = torch.randn(w0.shape, generator=gen, device="cuda", dtype=torch.float64)
        slope = (value(x0 + step * dx, w0 + step * dw) - value(x0 - step * dx, w0 - step * dw)) / (2 * step)
        parts = torch.cat(((grads.dqkv.double().reshape(x0.shape) * dx).flatten(),
                           (torch.stack((grads.dq_weight, grads.dk_weight)).double() * dw).flatten()))
        # each fp32 value is off by under 100 u of its size; the difference by
        # step^2 times a third derivative of this sum's size
        assert abs(slope - float(parts.sum())) <= 100 * U * float(parts.abs().sum()) + step * float(parts.abs().sum())


def test_offsets_past_32_bits():
    """Rows so far apart that their offsets pass 2^31 elements."""
    B, T, H, hd = 1, 3, 1, 16
    ld = 1 << 30
    buf = torch.empty(2 * ld + 3 * hd, dtype=BF16, device="cuda")
    rows = torch.as_strided(buf, (B, T, 3 * hd), (T * ld, ld, 1))
    src, dout, wq, wk = make(2, B, T, H, H, hd, BF16)
    rows.copy_(src)
    kw = dict(n_head=H, q_weight=wq, k_weight=wk)
    want = fal.qk_norm_rope_fwd(src, **kw)
    assert torch.equal(fal.qk_norm_rope_fwd(rows, **kw), want)
    assert torch.equal(fal.qk_norm_rope_bwd(rows, dout, **kw).dqkv, fal.qk_norm_rope_bwd(src, dout, **kw).dqkv)
    fal.qk_norm_rope_fwd(rows, out=rows, **kw)
    assert torch.equal(rows, want)


def test_replayed_graphs_share_nothing():
    a, b = (make(s, 2, 300, 4, 2, 64, BF16) for s in (1, 2))
    kw = dict(n_head=4, n_kv_head=2)

    def both(t):
        qkv, dout, wq, wk = t
        g = fal.qk_norm_rope_bwd(qkv, dout, q_weight=wq, k_weight=wk, **kw)
        return (fal.qk_norm_rope_fwd(qkv, q_weight=wq, k_weight=wk, **kw), *g)

    want = [[t.clone() for t in both(v)] for v in (a, b)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for v in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(both(v))
        graphs.append(g)
    for k in range(4):
        for o in outs:
            for t in o:
                t.zero_()
        for g in graphs if k % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(x, y) for x, y in zip(o, w))
        both(a)


def test_another_stream():
    qkv, dout, wq, wk = make(4, 2, 500, 4, 4, 64, BF16)
    kw = dict(n_head=4, q_weight=wq, k_weight=wk)
    want = fal.qk_norm_rope_bwd(qkv, dout, **kw)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = fal.qk_norm_rope_bwd(qkv, dout, **kw)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
