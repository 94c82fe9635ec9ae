"""Windowed attention with sinks, forward and backward, against the formula in
64 bits.

Tolerances are element by element, from the roundings that the kernels make
(u = 2^-24 for fp32, r = 2^-8 for bf16, half a step each):

* a score is a sum of hd products, a probability the exponential of a score
  difference: its relative error is at most
      e = 2 (hd + 4) u max|q||k| / sqrt(hd) + (n + 8) u
  (n visible keys in the row's sum; |q||k| the sum of absolute products), plus
  r where P is rounded to bf16 for its second product;
* out = sum p v: e sum p|v| + n u sum p|v|, and r|out| for bf16 storage;
* D = rowsum(dO * out) takes out's error: E = sum_d |dO| err(out) + hd u ...;
  dS = P (dP - D): e |dS| + P (E + hd u sum|dO||v|), plus r|dS| (bf16);
* dV, dK and dQ sum those bounds times |dO|, |Q| and |K|, and round once.
"""
import math

import numpy as np
import pytest
import torch

from paper_2510_14614_amd import fal

from gpu_helpers import log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def visible(T, window, sinks, n, device="cuda"):
    t = torch.arange(T, device=device)
    q, k = t[:, None], t[None]
    return (k <= q) & ((q - k < window) | (k < sinks)) & (q < n) & (k < n)


def reference(qkv, H, kv, hd, window, sinks, lens, dout):
    """out, lse, dqkv in 64 bits and the bounds of their errors."""
    B, T = qkv.shape[:2]
    bf = qkv.dtype == BF16
    u, r = 2.0 ** -24, 2.0 ** -8 if bf else 0.0
    x, g = qkv.double(), dout.double()
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device=qkv.device)  # noqa: E731
    W = (H + 2 * kv) * hd
    out, lse, dx = z(B, T, H * hd), z(B, H, T), z(B, T, W)
    e_out, e_lse, e_dx = z(B, T, H * hd), z(B, H, T), z(B, T, W)
    for b in range(B):
        see = visible(T, window, sinks, int(lens[b]), qkv.device)
        keys = int(see.sum(-1).max())
        some = see.any(-1)
        for h in range(H):
            j = h // (H // kv)
            cq, ck, cv = (slice(i * hd, (i + 1) * hd) for i in (h, H + j, H + kv + j))
            # rows past the length may hold anything: they take no part
            dead = ~some[:, None]
            q, k, v = (x[b, :, c].masked_fill(dead, 0.0) for c in (cq, ck, cv))
            go = g[b, :, cq].masked_fill(dead, 0.0)
            sc = 1 / math.sqrt(hd)
            s = (q @ k.T * sc).masked_fill(~see, -math.inf)
            l = torch.logsumexp(s, -1)
            p = torch.where(see, torch.exp(s - l[:, None]), 0.0)
            o = p @ v
            size = torch.where(see, q.abs() @ k.abs().T * sc, 0.0).max()
            e = float(2 * (hd + 4) * u * size + (keys + 8) * u)
            err_o = (e + r + keys * u) * (p @ v.abs()) + r * o.abs()
            out[b, :, cq], lse[b, h] = o, l
            e_out[b, :, cq], e_lse[b, h] = err_o, e + 4 * u * l.abs()
            dp = go @ v.T
            D = (go * o).sum(-1, keepdim=True)
            E = (go.abs() * err_o).sum(-1, keepdim=True) + hd * u * (go.abs() * o.abs()).sum(-1, keepdim=True)
            ds = p * (dp - D)
            err_ds = 2 * (e + r) * ds.abs() + p * (E + hd * u * (go.abs() @ v.abs().T)) * (1 + r)
            sums = keys * u
            dq, dk, dv = ds @ k * sc, ds.T @ q * sc, p.T @ go
            e_dq = (err_ds + sums * ds.abs()) @ k.abs() * sc
            e_dk = (err_ds + T * u * ds.abs()).T @ q.abs() * sc
            e_dv = ((e + r + T * u) * p).T @ go.abs()
            for c, d, ed in ((cq, dq, e_dq), (ck, dk, e_dk), (cv, dv, e_dv)):
                dx[b, :, c] += d
                e_dx[b, :, c] += ed
    return (out, lse, dx), (e_out, e_lse, e_dx + (r + u) * dx.abs())


def inputs(B, T, H, kv, hd, dtype, seed, lens=None, ld=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    W = (H + 2 * kv) * hd
    qkv = torch.randn(B, T, ld or W, device="cuda", generator=g).to(dtype)[:, :, :W]
    dout = torch.randn(B, T, H * hd, device="cuda", generator=g).to(dtype)
    n = torch.full((B,), T, dtype=torch.int32) if lens is None else torch.tensor(lens, dtype=torch.int32)
    return qkv, dout, n


def check(name, got, want, bound):
    # a floor of one part in 2^22 of the tensor's largest value covers sums
    # whose bound cancels to nothing (a gradient that is exactly zero)
    err = (got.double() - want).abs()
    ok = bound * 1.02 + 2.0 ** -22 * want.abs().max()
    worst = float((err / ok).nan_to_num(nan=math.inf).max())
    log(f"  {name}: worst error / bound {worst:.3f}")
    assert worst <= 1.0, name


SHAPES = [
    # B, T, H, kv, hd, window, sinks, lens
    (1, 1, 1, 1, 64, 1, 0, None),          # one token
    (5, 1, 2, 1, 64, 3, 2, (1, 0, 1, 1, 1)),
    (2, 2, 3, 3, 16, 1, 1, None),
    (2, 33, 4, 2, 32, 7, 2, (33, 0)),      # an empty sequence
    (3, 65, 2, 1, 16, 64, 3, (65, 1, 64)),
    (1, 200, 2, 2, 128, 1, 0, None),       # every query sees itself alone
    (1, 130, 2, 2, 64, 1000, 5, None),     # the window holds every key
    (2, 257, 4, 1, 64, 100, 4, (257, 130)),
    (1, 700, 4, 2, 64, 65, 70, None),      # sinks over two key tiles
    (1, 700, 2, 2, 128, 33, 128, None),    # a whole block of sinks
    (1, 513, 2, 1, 32, 128, 37, (400,)),
    (2, 900, 2, 2, 16, 129, 33, (900, 340)),
    (1, 1500, 2, 1, 128, 127, 1, None),
    (3, 385, 6, 3, 64, 64, 0, (385, 128, 129)),
    (1, 129, 8, 2, 128, 128, 2, None),
    # grids that fill the chip, whole blocks of 128 rows (the others halve
    # them): every head_dim, sinks seen from afar, ragged, shared heads
    (16, 280, 32, 16, 64, 40, 3, None),
    (16, 260, 32, 32, 128, 100, 0, (260, 259, 258, 257, 256, 255, 200, 129, 128, 127, 65, 64, 33, 1, 0, 260)),
    (24, 270, 32, 32, 32, 30, 33, None),
    (24, 257, 32, 32, 16, 8, 1, None),
    (8, 256, 16, 16, 128, 40, 3, None),    # ... in fp32 at head_dim 128 too: one round of the chip
    (4, 640, 24, 24, 128, 30, 9, None),    # two and a half rounds of it
    (2, 300, 40, 40, 128, 200, 4, None),   # the full length in most windows
    # few key/value heads: the query heads of a group divided
    (1, 600, 24, 2, 64, 200, 5, (577,)),
    (1, 600, 6, 1, 128, 70, 40, None),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(v) for v in s[:7]))
def test_against_the_formula(shape, dtype):
    B, T, H, kv, hd, window, sinks, lens = shape
    log(f"window attention {shape} {dtype}")
    qkv, dout, n = inputs(B, T, H, kv, hd, dtype, seed=T + hd)
    if lens is not None:
        n = torch.tensor(lens, dtype=torch.int32)
        for b in range(B):  # what lies past a sequence's end must not matter
            qkv[b, lens[b]:] = math.nan
            dout[b, lens[b]:] = math.inf
    want, bound = reference(qkv, H, kv, hd, window, sinks, n.tolist(), dout)
    dev_lens = None if lens is None else n.cuda()
    out, lse = fal.window_attention_fwd(qkv, H, window, sinks, n_kv_head=kv, lens=dev_lens)
    dqkv = fal.window_attention_bwd(qkv, out, dout, lse, H, window, sinks, n_kv_head=kv, lens=dev_lens)
    torch.cuda.synchronize()
    live = torch.arange(T)[None] < n[:, None]
    assert torch.equal(lse.isneginf().cpu(), ~live[:, None].expand(B, H, T))
    assert not out[~live.cuda()].any() and not dqkv[~live.cuda()].any()
    check("out", out, want[0], bound[0])
    check("lse", lse.masked_fill(lse.isneginf(), 0), want[1].masked_fill(want[1].isneginf(), 0),
          bound[1].masked_fill(bound[1].isinf(), 0))
    check("dqkv", dqkv, want[2], bound[2])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_a_full_window_is_the_causal_mask(dtype):
    # the same shapes through a window of T and of far more than T: bitwise
    qkv, dout, _ = inputs(2, 300, 4, 2, 64, dtype, seed=1)
    runs = []
    for window, sinks in ((300, 0), (2 ** 31 - 1, 7), (2 ** 40, 0)):
        out, lse = fal.window_attention_fwd(qkv, 4, window, sinks, n_kv_head=2)
        runs.append((out, lse, fal.window_attention_bwd(qkv, out, dout, lse, 4, window, sinks, n_kv_head=2)))
    for other in runs[1:]:
        for a, b in zip(runs[0], other):
            assert torch.equal(a, b)


def test_gradient_against_differences():
    B, T, H, kv, hd, window, sinks = 1, 90, 2, 1, 32, 20, 3
    qkv, dout, n = inputs(B, T, H, kv, hd, F32, seed=3)
    step = torch.randn(qkv.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)).double()

    def value(x):  # sum(dout * attention(x)) in 64 bits
        q, k, v = x[0].split((H * hd, kv * hd, kv * hd), -1)
        k, v = (t.repeat(1, H // kv) for t in (k, v))
        total = 0.0
        for h in range(H):
            c = slice(h * hd, (h + 1) * hd)
            s = (q[:, c] @ k[:, c].T / math.sqrt(hd)).masked_fill(~visible(T, window, sinks, T), -math.inf)
            total = total + (s.softmax(-1) @ v[:, c] * dout[0, :, c].double()).sum()
        return float(total)

    out, lse = fal.window_attention_fwd(qkv, H, window, sinks, n_kv_head=kv)
    dqkv = fal.window_attention_bwd(qkv, out, dout, lse, H, window, sinks, n_kv_head=kv).double()
    h = 1e-4  # truncation h^2 of the third derivative, 64-bit rounding 1e-16 / h: both under 1e-7
    slope = (value(qkv.double() + h * step) - value(qkv.double() - h * step)) / (2 * h)
    _, bound = reference(qkv, H, kv, hd, window, sinks, [T], dout)
    got = float((dqkv * step).sum())
    allowed = float((bound[2] * step.abs()).sum()) + 1e-6 * float((dqkv * step).abs().sum())
    log(f"slope {slope:.8f}, gradient {got:.8f}, allowed {allowed:.2e}")
    assert abs(got - slope) <= allowed


@pytest.mark.parametrize("dtype,hd", [(BF16, 64), (F32, 128), (BF16, 16)])
def test_strides_and_untouched_memory(dtype, hd):
    # rows inside wider buffers; what lies between them stays as it was
    B, T, H, kv, window, sinks = 2, 170, 4, 2, 50, 6
    W, dA = (H + 2 * kv) * hd, H * hd
    g = torch.Generator(device="cuda").manual_seed(7)
    wide = torch.randn(B, T, W + 32, device="cuda", generator=g).to(dtype)
    qkv = wide[:, :, 16:W + 16]
    dout = torch.randn(B, T, dA + 64, device="cuda", generator=g).to(dtype)[:, :, :dA]
    obuf = torch.full((B, T, dA + 64), 5.0, device="cuda", dtype=dtype)
    gbuf = torch.full((B, T, W + 48), 7.0, device="cuda", dtype=dtype)
    before = wide.clone()
    out, lse = fal.window_attention_fwd(qkv, H, window, sinks, n_kv_head=kv, out=obuf[:, :, :dA])
    fal.window_attention_bwd(qkv, out, dout, lse, H, window, sinks, n_kv_head=kv, dqkv=gbuf[:, :, :W])
    q2, d2 = qkv.contiguous(), dout.contiguous()
    out2, lse2 = fal.window_attention_fwd(q2, H, window, sinks, n_kv_head=kv)
    dq2 = fal.window_attention_bwd(q2, out2, d2, lse2, H, window, sinks, n_kv_head=kv)
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and torch.equal(gbuf[:, :, :W], dq2)
    assert bool((obuf[:, :, dA:] == 5).all()) and bool((gbuf[:, :, W:] == 7).all())
    assert torch.equal(wide, before)


def test_offsets_past_32_bits():
    # 1100 rows spaced 2^21 elements: offsets to 2.3e9 elements, 4.6 GB
    T, H, hd, window, sinks = 1100, 1, 64, 70, 2
    ld = 1 << 21
    buf = torch.empty(T * ld, dtype=BF16, device="cuda")
    far = buf.view(1, T, ld)[:, :, :3 * hd]
    near, dout, _ = inputs(1, T, H, H, hd, BF16, seed=11)
    far.copy_(near)
    out, lse = fal.window_attention_fwd(far, H, window, sinks)
    want, lse2 = fal.window_attention_fwd(near, H, window, sinks)
    assert torch.equal(out, want) and torch.equal(lse, lse2)
    got = fal.window_attention_bwd(far, out, dout, lse, H, window, sinks)
    assert torch.equal(got, fal.window_attention_bwd(near, want, dout, lse2, H, window, sinks))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_repeats_streams_and_graphs(dtype):
    # two calls at once on two streams and a captured pair replayed among
    # eager calls give the eager results, bit for bit
    B, T, H, hd, window, sinks = 2, 600, 4, 64, 90, 9
    sets = [inputs(B, T, H, H, hd, dtype, seed=s)[:2] for s in (21, 22)]

    def both(qkv, dout):
        out, lse = fal.window_attention_fwd(qkv, H, window, sinks)
        return out, lse, fal.window_attention_bwd(qkv, out, dout, lse, H, window, sinks)

    eager = [both(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [None, None]
    for i, st in enumerate(streams):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            got[i] = both(*sets[i])
    torch.cuda.synchronize()
    for a, b in zip(eager, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    graphs, static = [], []
    for qkv, dout in sets:
        s = (qkv.clone(), dout.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = both(*s)
        graphs.append(graph)
        static.append((s, held))
    for turn in range(3):
        for i in (0, 1):
            src = sets[(i + turn) % 2]
            static[i][0][0].copy_(src[0])
            static[i][0][1].copy_(src[1])
        for graph in graphs:
            graph.replay()
        again = both(*sets[turn % 2])
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(x, y) for x, y in zip(static[i][1], eager[(i + turn) % 2]))
        assert all(torch.equal(x, y) for x, y in zip(again, eager[turn % 2]))


def test_causality():
    # a change of token t changes no output before t and none past the window
    T, H, hd, window, sinks, t = 400, 2, 64, 60, 3, 150
    qkv, _, _ = inputs(1, T, H, H, hd, BF16, seed=31)
    base, _ = fal.window_attention_fwd(qkv, H, window, sinks)
    other = qkv.clone()
    other[0, t] = torch.randn(3 * H * hd, device="cuda").to(BF16)
    got, _ = fal.window_attention_fwd(other, H, window, sinks)
    same = (got == base).all(-1)[0].cpu().numpy()
    assert np.array_equal(np.flatnonzero(~same), np.arange(t, t + window))
