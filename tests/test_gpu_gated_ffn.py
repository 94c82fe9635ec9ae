"""The gated feed-forward block, forward and backward, against the formula in
64 bits.

Tolerances are element by element, from the roundings that the kernels make
(u = 2^-24; r = 2^-8 for bf16, half a step; in fp32 blocks r = u).  A sum of K
products in fp32 is off by (K + 2) u times the sum of their absolute values,
whatever its order:

* g and u: E(g) = (d + 2) u |x| |Wg|, E(u) alike;
* a = act(g): |act'| E(g) + s |a| with |act'| <= 1.13, s = 16 u for the
  exponential, reciprocal and products that make it (|g| rounds in the exponent:
  |g| u more), and act' alike with |act''| <= 1.3;
* h = a u: E(a) |u| + |a| E(u), and r |h| as an operand of the next product;
* y: E(h) |Wd| + (f + 2) u |h| |Wd| + r |y|;
* dh = dy Wd^T: (d + 2) u |dy| |Wd|^T; dg = dh u act' and du = dh a by the rule
  of products, and r of themselves as operands;
* dx, dWg, dWu, dWd: operand errors times the other operand, the sums' own
  error, and the result's rounding.
"""
import pytest
import torch

from paper_2510_14614_amd import fal

from gpu_helpers import log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
ACTS = ("silu", "gelu_tanh", "gelu")


def act(kind, g):
    """The activation, its first derivative."""
    g = g.detach().requires_grad_()
    f = torch.nn.functional
    a = f.silu(g) if kind == "silu" else f.gelu(g, approximate="tanh" if kind == "gelu_tanh" else "none")
    return a.detach(), torch.autograd.grad(a.sum(), g)[0]


def reference(x, wg, wu, wd, dy, kind, r, r_grad):
    """{name: (value, bound)} in 64 bits; r_grad: the weight gradients' rounding."""
    M, d = x.shape
    f = wg.shape[1]
    ax, ag, au, ad, ay = (t.abs() for t in (x, wg, wu, wd, dy))
    su = lambda k: (k + 2) * U  # noqa: E731
    g, u = x @ wg, x @ wu
    eg, eu = su(d) * (ax @ ag), su(d) * (ax @ au)
    a, da = act(kind, g)
    s = (16 + g.abs()) * U
    ea = 1.13 * eg + s * a.abs() + U * 1e-3
    eda = 1.3 * eg + s * (da.abs() + 1) + U
    h = a * u
    eh = ea * u.abs() + a.abs() * eu + ea * eu + r * h.abs()
    y = h @ wd
    ey = eh @ ad + su(f) * ((h.abs() + eh) @ ad) + r * y.abs()
    out = {"y": (y, ey)}
    if dy is None:
        return out
    dh = dy @ wd.T
    edh = su(d) * (ay @ ad.T)
    size = dh.abs() + edh
    dg, du = dh * u * da, dh * a
    edg = edh * (u * da).abs() + size * (eu * da.abs() + (u.abs() + eu) * eda) + (r + 3 * U) * dg.abs()
    edu = edh * a.abs() + size * ea + (r + U) * du.abs()
    # errors of rounded operands are relative to the rounded values
    edg, edu = edg * (1 + r), edu * (1 + r)
    dx = dg @ wg.T + du @ wu.T
    edx = edg @ ag.T + edu @ au.T + su(2 * f) * ((dg.abs() + edg) @ ag.T + (du.abs() + edu) @ au.T) + r * dx.abs()
    out["dx"] = (dx, edx)
    for name, p, ep in (("dw_gate", dg, edg), ("dw_up", du, edu)):
        w = x.T @ p
        out[name] = (w, ax.T @ ep + su(M) * (ax.T @ (p.abs() + ep)) + r_grad * w.abs())
    w = h.T @ dy
    out["dw_down"] = (w, eh.T @ ay + su(M) * ((h.abs() + eh).T @ ay) + r_grad * w.abs())
    return out


def worst(got, want, bound):
    got, want, bound = got.double(), want.double(), bound.double() + 1e-300
    assert got.shape == want.shape
    assert torch.isfinite(got).all()
    return float(((got - want).abs() / bound).max())


def wide(t, pad):
    buf = torch.full((*t.shape[:-1], t.shape[-1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    buf[..., :t.shape[-1]] = t
    return buf[..., :t.shape[-1]]


def make(seed, M, d, f, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, dy = n(M, d) * scale, n(M, d)
    return [t.to(dtype) for t in (x, n(d, f) * d ** -0.5, n(d, f) * d ** -0.5, n(f, d) * f ** -0.5, dy)]


def check(label, M, d, f, dtype, kind="silu", pad=0, grads_f32=False, scale=1.0, packed=False, seed=0):
    log(f"{label}: M {M} d {d} f {f} {dtype} {kind} pad {pad} grads_f32 {grads_f32} scale {scale}")
    x, wg, wu, wd, dy = make(seed, M, d, f, dtype, scale)
    r = 2.0 ** -8 if dtype == BF16 else U
    ref = reference(*(t.double() for t in (x, wg, wu, wd, dy)), kind, r, U if grads_f32 else r)
    kw = {}
    if pad:
        x, wg, wu, wd, dy = (wide(t, pad) for t in (x, wg, wu, wd, dy))
        kw = {"dx": wide(x, pad), "dw": [wide(w.to(F32 if grads_f32 else dtype), 2 * pad) for w in (wg, wu, wd)]}
    if packed:
        both = torch.cat((wg, wu), 1)
        wg, wu = both[:, :f], both[:, f:]
        grad = torch.empty(d, 2 * f, dtype=F32 if grads_f32 else dtype, device="cuda")
        kw = {"dw": (grad[:, :f], grad[:, f:], torch.empty(f, d, dtype=grad.dtype, device="cuda"))}
    y, none = fal.gated_ffn_fwd(x, wg, wu, wd, kind)
    assert none is None
    y2, saved = fal.gated_ffn_fwd(x, wg, wu, wd, kind, y=wide(y, pad) if pad else None, save=True)
    assert torch.equal(y, y2)
    grads = fal.gated_ffn_bwd(x, wg, wu, wd, saved, dy, kind, grads_f32=grads_f32, **kw)
    errs = {"y": worst(y, *ref["y"])}
    for name in ("dx", "dw_gate", "dw_up", "dw_down"):
        t = getattr(grads, name)
        assert t.dtype == (F32 if grads_f32 and name != "dx" else dtype)
        errs[name] = worst(t, *ref[name])
    log(f"  errors over their bounds: { {k: round(v, 3) for k, v in errs.items()} }")
    assert all(v <= 1 for v in errs.values()), errs
    return grads


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_activations(dtype, kind):
    check("activation", 70, 64, 136, dtype, kind)
    # gates from deep in the left tail to far on the right
    check("wide gates", 40, 32, 64, dtype, kind, scale=12.0)


@pytest.mark.parametrize("M,d,f", [(1, 8, 8), (1, 64, 256), (2, 72, 40), (3, 8, 520), (5, 1000, 136), (17, 200, 72),
                                   (127, 128, 128), (128, 136, 264), (129, 256, 1000), (300, 1032, 2056)])
def test_bf16_shapes(M, d, f):
    check("bf16", M, d, f, BF16, seed=M)


@pytest.mark.parametrize("M", range(1, 10))
@pytest.mark.parametrize("d,f", [(64, 256), (1000, 72), (136, 2744), (2048, 5504)])
def test_few_rows(M, d, f):
    check("few", M, d, f, BF16, ACTS[M % 3], pad=8 * (M % 2), seed=M)


@pytest.mark.parametrize("M,d,f", [(40, 2048, 256), (40, 256, 2048), (100, 1000, 1096), (500, 1000, 520),
                                   (1501, 1000, 2744), (130, 520, 4096)])
def test_products_cut_along_k(M, d, f):
    """Few tiles and long sums: parts of k in workgroups of their own."""
    check("cut", M, d, f, BF16, ACTS[M % 3], pad=8, seed=M)
    check("cut", M, d + 1, f + 3, F32, ACTS[M % 3], pad=1, seed=M)


@pytest.mark.parametrize("M,d,f", [(33, 67, 5001), (300, 260, 8192), (700, 1500, 4097)])
def test_long_fp32_sums(M, d, f):
    """Sums over f in four parts, also held in the norm."""
    x, wg, wu, wd, dy = make(M, M, d, f, F32)
    y, saved = fal.gated_ffn_fwd(x, wg, wu, wd, save=True)
    dx = fal.gated_ffn_bwd(x, wg, wu, wd, saved, dy, weight_grads=False).dx
    ref = reference(*(t.double() for t in (x, wg, wu, wd, dy)), "silu", U, U)
    assert worst(y, *ref["y"]) <= 1 and worst(dx, *ref["dx"]) <= 1
    # independent roundings of a sum in four parts: sqrt(f / 4) halves of u a term's
    # mean size, and as many again from h and its factors
    for got, want in ((y, ref["y"][0]), (dx, ref["dx"][0])):
        assert float((got.double() - want).norm() / want.norm()) <= 2 * (f / 4) ** 0.5 * U


def test_more_elements_than_one_axis_of_a_grid():
    """2^32 elements of h and more, a thread each: the last rows against fp64."""
    M, d, f = (1 << 32) // 8193 + 131, 16, 8193
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB")
    x, wg, wu, wd, dy = make(5, M, d, f, F32)
    y, saved = fal.gated_ffn_fwd(x, wg, wu, wd, save=True)
    dx = fal.gated_ffn_bwd(x, wg, wu, wd, saved, dy, weight_grads=False).dx
    del saved
    for rows in (slice(0, 9), slice(M - 200, M)):
        ref = reference(*(t.double() for t in (x[rows], wg, wu, wd, dy[rows])), "silu", U, U)
        assert worst(y[rows], *ref["y"]) <= 1 and worst(dx[rows], *ref["dx"]) <= 1
    del x, y, dx, dy
    torch.cuda.empty_cache()


def test_few_rows_of_long_products():
    """Ranges of k cut by what LDS holds of their rows, past 16 of them too."""
    check("long", 8, 8, 20000, BF16)
    check("long", 8, 24000, 8, BF16)
    check("long", 8, 8, 24000, BF16)


@pytest.mark.parametrize("M,d,f", [(1, 1, 1), (1, 63, 257), (2, 7, 33), (65, 65, 65), (130, 100, 301), (300, 33, 1000)])
def test_fp32_shapes(M, d, f):
    check("fp32", M, d, f, F32, seed=M)


@pytest.mark.parametrize("M,d,f", [(2500, 64, 2304), (2048, 512, 2048), (4096, 768, 2048)])
def test_large_tiles(M, d, f):
    """Sizes whose launches take the larger tiles, whole and ragged."""
    check("large", M, d, f, BF16, grads_f32=M == 2048)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(dtype):
    check("pad", 37, 72, 136, dtype, pad=8)
    check("pad", 2, 64, 72, dtype, pad=24, grads_f32=True)
    if dtype == F32:
        check("pad", 37, 71, 133, dtype, pad=3)
    check("packed", 50, 64, 120, dtype, packed=True)


def test_leading_dimensions_and_partial_gradients():
    x, wg, wu, wd, dy = make(1, 30, 64, 128, BF16)
    y, saved = fal.gated_ffn_fwd(x, wg, wu, wd, save=True)
    y3, saved3 = fal.gated_ffn_fwd(x.view(5, 6, 64), wg, wu, wd, save=True)
    assert y3.shape == (5, 6, 64) and torch.equal(y3.view(30, 64), y) and torch.equal(saved3, saved)
    full = fal.gated_ffn_bwd(x, wg, wu, wd, saved, dy)
    only_x = fal.gated_ffn_bwd(x.view(5, 6, 64), wg, wu, wd, saved, dy.view(5, 6, 64), weight_grads=False)
    assert torch.equal(only_x.dx.view(30, 64), full.dx) and only_x.dw_gate is None
    only_w = fal.gated_ffn_bwd(x, wg, wu, wd, saved, dy, input_grad=False)
    assert only_w.dx is None
    assert all(torch.equal(a, b) for a, b in zip(only_w[1:], full[1:]))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gates_past_the_exponentials_range(dtype):
    """Gates of +-200 and +-1e30: the activation is the gate or zero, and
    nothing becomes NaN."""
    d = f = 8
    for big in (200.0, 1e30):
        x = torch.eye(8, device="cuda", dtype=dtype)
        x[1] *= -1
        wg = torch.full((d, f), big, device="cuda", dtype=dtype)
        wu = torch.full((d, f), 0.5, device="cuda", dtype=dtype)
        wd = torch.eye(8, device="cuda", dtype=dtype)
        for kind in ACTS:
            y, saved = fal.gated_ffn_fwd(x, wg, wu, wd, kind, save=True)
            want = torch.full((8, f), float(wg[0, 0].double() * 0.5), device="cuda", dtype=torch.float64)
            want[1] = 0  # act(-big) * -0.5
            assert ((y.double() - want).abs() <= want.abs() * 2.0 ** -7).all(), kind
            g = fal.gated_ffn_bwd(x, wg, wu, wd, saved, torch.ones_like(x), kind)
            assert all(torch.isfinite(t).all() for t in g), kind


@pytest.mark.parametrize("kind", ACTS)
def test_gradients_against_differences(kind):
    """Along random directions, the change of sum(dy * y) in 64 bits."""
    t = make(2, 20, 24, 40, F32)
    x, wg, wu, wd, dy = t
    y, saved = fal.gated_ffn_fwd(x, wg, wu, wd, kind, save=True)
    grads = fal.gated_ffn_bwd(x, wg, wu, wd, saved, dy, kind)
    base = [v.double() for v in t[:4]]

    def value(leaves):
        a, _ = act(kind, leaves[0] @ leaves[1])
        return float(((a * (leaves[0] @ leaves[2])) @ leaves[3] * dy).sum())

    gen = torch.Generator(device="cuda").manual_seed(3)
    step = 1e-5
    for _ in range(4):
        way = [torch.randn(v.shape, generator=gen, device="cuda", dtype=torch.float64) for v in base]
        slope = (value([v + step * w for v, w in zip(base, way)]) -
                 value([v - step * w for v, w in zip(base, way)])) / (2 * step)
        parts = torch.cat([(g.double() * w).flatten() for g, w in zip(grads, way)])
        # fp32 values off by under 200 u of their sums' sizes, and the
        # difference by step^2 of a third derivative
        assert abs(slope - float(parts.sum())) <= (200 * U + 1e-6) * float(parts.abs().sum())


def test_replayed_graphs_share_nothing():
    sets = [make(s, 130, 64, 256, BF16) for s in (1, 2)]

    def both(t):
        y, saved = fal.gated_ffn_fwd(*t[:4], save=True)
        return (y, *fal.gated_ffn_bwd(*t[:4], saved, t[4]))

    want = [[v.clone() for v in both(t)] for t in sets]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for t in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(both(t))
        graphs.append(g)
    for k in range(4):
        for o in outs:
            for v in o:
                v.zero_()
        for g in graphs if k % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w))
        both(sets[k % 2])


def test_another_stream():
    t = make(5, 200, 128, 256, BF16)
    y, saved = fal.gated_ffn_fwd(*t[:4], save=True)
    want = fal.gated_ffn_bwd(*t[:4], saved, t[4])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got_y, got_saved = fal.gated_ffn_fwd(*t[:4], save=True)
        got = fal.gated_ffn_bwd(*t[:4], got_saved, t[4])
    s.synchronize()
    assert torch.equal(got_y, y) and all(torch.equal(a, b) for a, b in zip(got, want))


def right_half(t):
    """t as the right-hand columns of a matrix that ends with it, NaN beside."""
    buf = torch.full((t.shape[0], 2 * t.shape[1]), float("nan"), dtype=t.dtype, device=t.device)
    buf[:, t.shape[1]:] = t
    return buf[:, t.shape[1]:]


@pytest.mark.parametrize("M,d,f", [(5, 72, 200), (50, 64, 120), (300, 1000, 1096), (1501, 1000, 2744), (2500, 72, 2312)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_right_hand_columns(dtype, M, d, f):
    """Every operand the right-hand columns of a matrix of its own, on ragged
    tiles, products in parts and the larger tiles."""
    x, wg, wu, wd, dy = make(M + d, M, d, f, dtype)
    r = 2.0 ** -8 if dtype == BF16 else U
    ref = reference(*(t.double() for t in (x, wg, wu, wd, dy)), "silu", r, r)
    x, wg, wu, wd, dy = (right_half(t) for t in (x, wg, wu, wd, dy))
    y, saved = fal.gated_ffn_fwd(x, wg, wu, wd, save=True)
    grads = fal.gated_ffn_bwd(x, wg, wu, wd, saved, dy)
    errs = {k: worst(y if k == "y" else getattr(grads, k), *v) for k, v in ref.items()}
    log(f"{(M, d, f)} {dtype}: errors over their bounds { {k: round(v, 3) for k, v in errs.items()} }")
    assert all(v <= 1 for v in errs.values()), errs


def test_as_many_rows_as_a_call_takes():
    """fp32 rows of one column, as many tiles as a launch holds."""
    M = (1 << 29) - 64
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    x, wg, wu, wd, dy = make(4, M, 1, 1, F32)
    y, saved = fal.gated_ffn_fwd(x, wg, wu, wd, save=True)
    dx = fal.gated_ffn_bwd(x, wg, wu, wd, saved, dy, weight_grads=False).dx
    del saved
    for rows in (slice(0, 200), slice(M // 2, M // 2 + 200), slice(M - 200, M)):
        ref = reference(*(t.double() for t in (x[rows], wg, wu, wd, dy[rows])), "silu", U, U)
        assert worst(y[rows], *ref["y"]) <= 1 and worst(dx[rows], *ref["dx"]) <= 1
    del x, y, dx, dy
    torch.cuda.empty_cache()


# (columns of one matrix, first column of dw_gate and of dw_up) for f = 120
LAYOUTS = [(240, 0, 120), (240, 120, 0), (264, 0, 136), (264, 8, 144), (272, 152, 16)]


@pytest.mark.parametrize("width,at_gate,at_up", LAYOUTS)
@pytest.mark.parametrize("dtype,grads_f32", [(F32, False), (BF16, False), (BF16, True)])
def test_gradients_in_one_matrix(dtype, grads_f32, width, at_gate, at_up):
    """dw_gate and dw_up side by side in either order, with and without columns
    beside and between them, which stay as they are."""
    M, d, f = 70, 64, 120
    x, wg, wu, wd, dy = make(6, M, d, f, dtype)
    _, saved = fal.gated_ffn_fwd(x, wg, wu, wd, save=True)
    want = fal.gated_ffn_bwd(x, wg, wu, wd, saved, dy, grads_f32=grads_f32)
    both = torch.full((d, width), 7.0, dtype=want.dw_gate.dtype, device="cuda")
    halves = both[:, at_gate:at_gate + f], both[:, at_up:at_up + f]
    got = fal.gated_ffn_bwd(x, wg, wu, wd, saved, dy, dw=(*halves, torch.empty_like(want.dw_down)), grads_f32=grads_f32)
    assert got.dw_gate is halves[0] and got.dw_up is halves[1]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for h in halves:
        h.fill_(7.0)
    assert (both == 7.0).all()
    # columns that both would write
    with pytest.raises(fal.FalError, match="overlap"):
        fal.gated_ffn_bwd(x, wg, wu, wd, saved, dy, dw=(both[:, :f], both[:, f - 8:2 * f - 8], got.dw_down),
                          grads_f32=grads_f32)
