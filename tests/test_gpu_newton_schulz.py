"""Newton-Schulz products and the update round them, against 64 bits.

Tolerances, in the Frobenius norm (u = 2^-24 for fp32, r the result's rounding):

* stored X, A and B are sums of two fp16 values: off by R = 2^-22 of each
  element;
* a product of K terms leaves out the products of the two low parts (2^-22 of
  the absolute sum S) and rounds 3 K sums in fp32, which as independent
  roundings stay within 4 sqrt(3 K) u of S;
* A = X X^T so is off by fA, B = a I + b A + c A^2 by
  fB = (|b| + 2 |c| |A|_2) fA + its own product's and storage's, B X by
  fB |X|_2 + its own;
* an earlier error E goes through the polynomial, whose slope on the singular
  values' range is at most L: E <- L E + the step's.

The slope bound takes every error for one of the smallest singular values, so
the results are also held to four times the error of the same products in
fp32 (22 bits of storage against 24), plus the result's rounding.
"""
import math

import pytest
import torch

from paper_2510_14614_amd import fal
from paper_2510_14614_amd.config import get_config

from gpu_helpers import log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U, R = 2.0 ** -24, 2.0 ** -22
COEF = fal.NEWTON_SCHULZ


def f(m):
    return float(torch.linalg.matrix_norm(m))


def exact(x, steps, coef):
    """The polynomial of each matrix in 64 bits, and the bound of the kernels'
    error in the Frobenius norm."""
    a, b, c = coef
    done, bounds = [], []
    for m in x.double():
        z = m if m.shape[0] <= m.shape[1] else m.T
        p, q = z.shape
        size = f(z)
        z = z / size if size > 0 else z
        E = f(z) * (R + 2 * U)
        acc = lambda k: R + 4 * math.sqrt(3 * k) * U  # noqa: E731
        for _ in range(steps):
            s = float(torch.linalg.matrix_norm(z, 2)) + E
            t = torch.linspace(0, s, 1001, dtype=torch.float64)
            L = float((a + 3 * b * t ** 2 + 5 * c * t ** 4).abs().max()) * 1.01
            A = z @ z.T
            fA = acc(q) * f(z.abs() @ z.abs().T) + R * f(A)
            B = a * torch.eye(p, dtype=z.dtype, device=z.device) + b * A + c * A @ A
            fB = (abs(b) + 2 * abs(c) * s * s) * fA + abs(c) * acc(p) * f(A.abs() @ A.abs()) + (R + 4 * U) * f(B) \
                + 4 * U * (abs(b) * f(A) + abs(c) * f(A @ A))
            new = B @ z
            E = L * E + fB * s + acc(p) * f(B.abs() @ z.abs()) + R * f(new)
            z = new
        done.append(z if m.shape[0] <= m.shape[1] else z.T)
        bounds.append(E)
    return torch.stack(done), bounds


def in_fp32(x, steps, coef):
    a, b, c = coef
    done = []
    for m in x.float():
        z = m if m.shape[0] <= m.shape[1] else m.T.contiguous()
        z = (z.double() / torch.linalg.matrix_norm(z.double())).float()
        for _ in range(steps):
            A = z @ z.T.contiguous()
            z = a * z + (b * A + c * (A @ A)) @ z
        done.append(z if m.shape[0] <= m.shape[1] else z.T)
    return torch.stack(done)


def make(seed, count, rows, cols, dtype, scale=1e-3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(count, rows, cols, generator=g, device="cuda").mul_(scale).to(dtype)


def hold(got, want, bounds, plain, r):
    assert got.shape == want.shape and torch.isfinite(got).all()
    for i in range(len(want)):
        err, mine = f(got[i].double() - want[i]), r * f(want[i])
        near = 4 * f(plain[i].double() - want[i])
        log(f"  matrix {i}: error {err:.3e}, bound {bounds[i] + mine:.3e}, four times fp32's {near:.3e}, "
            f"norm {f(want[i]):.3e}")
        assert err <= bounds[i] + mine
        assert err <= near + mine + 4 * U * f(want[i])


def check(count, rows, cols, dtype, steps=5, coef=COEF, seed=0, scale=1e-3):
    log(f"count {count} {rows} x {cols} {dtype} steps {steps} coefficients {coef}")
    x = make(seed, count, rows, cols, dtype, scale)
    keep = x.clone()
    got = fal.newton_schulz(x, steps, coef)
    assert torch.equal(x, keep) and got.dtype == dtype
    want, bounds = exact(x, steps, coef)
    hold(got, want, bounds, in_fp32(x, steps, coef), 2.0 ** -8 if dtype == BF16 else U)
    return x, got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (5, 1), (3, 3), (16, 40), (64, 64), (65, 63), (127, 300),
                                       (128, 128), (128, 160), (161, 128), (31, 1100), (129, 257), (300, 129),
                                       (256, 512), (2, 3000), (100, 700), (901, 70)])
def test_shapes(dtype, rows, cols):
    check(2, rows, cols, dtype, seed=rows + cols)


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
def test_steps(steps):
    check(1, 100, 200, F32, steps=steps)


@pytest.mark.parametrize("coef", [(1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5), (1.0, 0.0, 0.0),
                                  (4.0848, -6.8946, 2.9270), (0.5, 0.25, 0.0)])
def test_coefficients(coef):
    check(1, 96, 130, F32, coef=coef, steps=4)


def test_more_matrices_than_one_batch_holds():
    """2.6 MB of parts a matrix: 900 of them pass the 2 GiB that go through
    together, so they go in two batches of 450."""
    x = make(0, 900, 200, 1000, BF16)
    got = fal.newton_schulz(x)
    some = [0, 1, 449, 450, 899]
    want, bounds = exact(x[some], 5, COEF)
    hold(got[some], want, bounds, in_fp32(x[some], 5, COEF), 2.0 ** -8)
    # (orthogonal rows: every matrix has its norm, within the polynomial's band)
    norms = torch.linalg.matrix_norm(got.float())
    assert ((norms > 0.6 * 200 ** 0.5) & (norms < 1.3 * 200 ** 0.5)).all()


@pytest.mark.parametrize("count,rows,cols", [(1, 200, 4000), (3, 1001, 333), (1, 640, 700), (1, 1024, 1024), (2, 130, 9000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products_cut_along_k(count, rows, cols, dtype):
    """Few tiles and long sums: ranges of k in workgroups of their own."""
    check(count, rows, cols, dtype, seed=rows)


@pytest.mark.parametrize("count", [2, 8])  # 72 and 288 tiles of 256 x 256
def test_products_on_large_tiles(count):
    x = make(9, count, 2000, 5000, F32)
    got = fal.newton_schulz(x, steps=3)
    some = [0, count - 1]
    want, bounds = exact(x[some], 3, COEF)
    hold(got[some], want, bounds, in_fp32(x[some], 3, COEF), U)
    norms = torch.linalg.matrix_norm(got)
    assert ((norms - norms.mean()).abs() < 0.02 * norms.mean()).all()


def test_large():
    check(1, 700, 2100, BF16)
    check(1, 1000, 640, F32)


@pytest.mark.parametrize("count,rows,cols", [(1, 1401, 1503), (2, 1503, 1400), (1, 130, 130), (3, 900, 1700), (12, 260, 390)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products_on_every_tile(count, rows, cols, dtype):
    """B X of 144 and 288 tiles of 128 x 128, of 336, and of 64 x 64."""
    check(count, rows, cols, dtype, steps=3, seed=rows)


@pytest.mark.parametrize("case", [(1, 1401, 1503), (1, 1503, 1400), (3, 200, 333)])
def test_update_on_every_tile(case):
    test_update(case, BF16, True)


def test_tall_matrices_are_wide_ones_transposed():
    x = make(3, 3, 150, 90, F32)
    got = fal.newton_schulz(x)
    assert torch.equal(got, fal.newton_schulz(x.transpose(1, 2).contiguous()).transpose(1, 2))


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e30])
def test_any_scale(scale):
    """The norm is taken in fp64, and only the direction counts."""
    check(1, 40, 60, F32, scale=scale)


def test_diagonal_matrices_stay_diagonal():
    n, (a, b, c) = 200, COEF
    d = torch.linspace(0.1, 1, n, device="cuda", dtype=torch.float64)
    got = fal.newton_schulz(torch.diag(d.float()))
    s = d.float().double()
    s = s / s.norm()
    for _ in range(5):
        s = s * (a + b * s ** 2 + c * s ** 4)
    off = got - torch.diag(got.diagonal())
    assert (off == 0).all()
    # each step: a factor off by at most 2^-20 of its largest value, slope 3.5
    assert ((got.diagonal().double() - s).abs() <= 3.5 ** 5 * 2.0 ** -20 * s.abs().clamp(min=1e-2)).all()


def test_zeros_and_values_that_are_not_finite():
    x = make(4, 4, 33, 70, F32)
    x[1] = 0
    x[2, 5, 7] = math.nan
    x[3, 0, 0] = math.inf
    got = fal.newton_schulz(x)
    assert torch.equal(got[0], fal.newton_schulz(x[0]))
    assert (got[1] == 0).all() and torch.isnan(got[2]).all() and torch.isnan(got[3]).all()


@pytest.mark.parametrize("rows,cols", [(40, 90), (90, 40)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_batches_with_gaps_and_in_place(rows, cols, dtype):
    x = make(5, 3, rows, cols, dtype)
    want = fal.newton_schulz(x)
    n = rows * cols
    buf = torch.full((3 * (n + 13),), 7.0, dtype=dtype, device="cuda")
    view = torch.as_strided(buf, (3, rows, cols), (n + 13, cols, 1))
    view.copy_(x)
    out = torch.full((3 * (n + 5),), 9.0, dtype=dtype, device="cuda")
    other = torch.as_strided(out, (3, rows, cols), (n + 5, cols, 1))
    assert fal.newton_schulz(view, out=other) is other and torch.equal(other, want)
    assert torch.equal(fal.newton_schulz(view), want)
    fal.newton_schulz(view, out=view)
    assert torch.equal(view, want)
    for b, step, v in ((buf, n + 13, 7.0), (out, n + 5, 9.0)):
        for i in range(3):
            assert (b[i * step + n:(i + 1) * step] == v).all()


def update(case, master, grads, momentum, hp):
    """The step in 64 bits: master and momentum, and the bound of master's
    error."""
    g, m = grads.double(), momentum.double()
    beta = float(torch.tensor(hp["beta"], dtype=F32))
    m = beta * m + g
    u = g + beta * m if hp["nesterov"] else m
    x, bounds = exact(u, hp["steps"], COEF)
    scale = hp["scale"] if hp["scale"] is not None else max(1.0, case[2] / case[1]) ** 0.5
    w = master.double() * (1 - hp["lr"] * hp["weight_decay"]) - hp["lr"] * scale * x
    # momentum and U round three times more, before the products' slope (at most
    # 4 a step); master twice, its hyper-parameters once each
    bounds = [hp["lr"] * scale * (b + 4.0 ** hp["steps"] * 4 * U + 4 * U * f(v)) + 4 * U * f(master[i].double())
              for i, (b, v) in enumerate(zip(bounds, x))]
    return w, m, bounds


@pytest.mark.parametrize("case", [(2, 64, 192), (1, 257, 130), (3, 100, 100), (1, 7, 1)])
@pytest.mark.parametrize("dtype", [None, F32, BF16])
@pytest.mark.parametrize("nesterov", [True, False])
def test_update(case, dtype, nesterov):
    grads, momentum, master = (make(s, *case, F32, scale) for s, scale in ((1, 1e-3), (2, 1e-2), (3, 0.02)))
    params = None if dtype is None else torch.zeros(case, dtype=dtype, device="cuda")
    hp = {"lr": 0.02, "beta": 0.95, "weight_decay": 0.1, "nesterov": nesterov, "scale": None, "steps": 5}
    w, m, bounds = update(case, master, grads, momentum, hp)
    keep = grads.clone()
    fal.muon_step(master, grads, momentum, params, **hp)
    assert torch.equal(grads, keep)
    assert ((momentum.double() - m).abs() <= 2 * U * (m.abs() + momentum.abs())).all()
    for i in range(case[0]):
        err = f(master[i].double() - w[i])
        log(f"{case} {dtype} nesterov {nesterov}: error {err:.3e}, bound {bounds[i]:.3e}")
        assert err <= bounds[i]
    if params is not None:
        assert torch.equal(params, master.to(dtype))


def test_updates_go_on():
    """Three steps in a row, with another scale and without decay."""
    case = (2, 48, 80)
    grads, momentum, master = (make(s, *case, F32, 1e-2) for s in (1, 2, 3))
    momentum.zero_()
    hp = {"lr": 0.1, "beta": 0.9, "weight_decay": 0.0, "nesterov": True, "scale": 0.3, "steps": 3}
    for k in range(3):
        w, m, bounds = update(case, master, grads, momentum, hp)
        fal.muon_step(master, grads, momentum, **hp)
        assert all(f(master[i].double() - w[i]) <= bounds[i] for i in range(2))
        grads = make(10 + k, *case, F32, 1e-2)


def test_update_in_a_models_buffers():
    """Every layer's up-projection where the model keeps it: nothing else
    moves."""
    cfg = get_config("tiny", dtype=1)
    F = fal.Fal(cfg)
    gen = torch.Generator(device="cuda").manual_seed(1)
    F.params.copy_(torch.randn(F.params.shape, generator=gen, device="cuda") * 0.02)
    F.init_optimizer()
    tokens = torch.randint(0, cfg.vocab, (cfg.batch, cfg.seq_len + 1), generator=gen, device="cuda", dtype=torch.int32)
    F.model_step(tokens)
    lay, k = F.layout, fal.BLOCK_TENSORS.index("w_fc")
    d, ff = cfg.d_model, cfg.d_ff
    at = lay["block_base"] + lay["block"][k]

    def view(flat):
        return torch.as_strided(flat, (cfg.n_layer, d, ff), (lay["block_stride"], ff, 1), at)

    before = {n: getattr(F, n).clone() for n in ("master", "m", "params", "grads")}
    hp = {"lr": 0.02, "beta": 0.95, "weight_decay": 0.0, "nesterov": True, "scale": None, "steps": 5}
    w, m, bounds = update((cfg.n_layer, d, ff), view(F.master), view(F.grads), view(F.m), hp)
    fal.muon_step(view(F.master), view(F.grads), view(F.m), view(F.params), **hp)
    for i in range(cfg.n_layer):
        assert f(view(F.master)[i].double() - w[i]) <= bounds[i]
    assert torch.equal(view(F.params), view(F.master).to(BF16))
    for n, old in before.items():
        new = getattr(F, n).clone()
        if n != "grads":
            assert not torch.equal(view(new), view(old))
            view(new).copy_(view(old))
        assert torch.equal(new, old), n
    F.close()


def test_replayed_graphs_share_nothing():
    sets = [make(s, 2, 100, 180, F32) for s in (1, 2)]
    want = [fal.newton_schulz(x).clone() for x in sets]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(fal.newton_schulz(x))
        graphs.append(g)
    for k in range(4):
        for o in outs:
            o.zero_()
        for g in graphs if k % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
        fal.newton_schulz(sets[k % 2])


def test_another_stream():
    x = make(6, 2, 200, 300, BF16)
    want = fal.newton_schulz(x)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = fal.newton_schulz(x)
    s.synchronize()
    assert torch.equal(got, want)


def test_as_many_small_matrices_as_a_call_takes():
    """2^22 of them, a workgroup of 1024 threads each: more threads than one
    axis of a grid holds."""
    n = 1 << 22
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(n, 2, 3, generator=g, device="cuda")
    got = fal.newton_schulz(x, steps=2)
    for some in (slice(0, 3), slice((1 << 20) - 2, (1 << 20) + 2), slice(n - 3, n)):
        want, bounds = exact(x[some], 2, COEF)
        hold(got[some], want, bounds, in_fp32(x[some], 2, COEF), U)
    # the larger of two singular values starts at 0.7 at least, and the polynomial
    # takes 0.7 .. 1.2 to 0.68 .. 1.2
    assert (torch.linalg.matrix_norm(got) > 0.67).all()


@pytest.mark.parametrize("count,rows,cols", [(2, 40, 60), (2, 150, 700), (1, 900, 200)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_polynomial_of_zeros(dtype, count, rows, cols):
    """a = b = c = 0: X is 0 after the first step, and the update nothing but
    the weights' decay."""
    x = make(7, count, rows, cols, dtype)
    for steps in (1, 3):
        assert (fal.newton_schulz(x, steps, (0.0, 0.0, 0.0)) == 0).all()
    master, momentum = (make(s, count, rows, cols, F32) for s in (8, 9))
    want = master * torch.tensor(1 - 0.1 * 0.5, device="cuda")
    fal.muon_step(master, x.float(), momentum, lr=0.1, weight_decay=0.5, coefficients=(0.0, 0.0, 0.0))
    assert torch.equal(master, want)


def uneven(kind, seed, count, rows, cols, dtype):
    """Matrices whose singular values differ much."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(count, *s, generator=g, device="cuda")  # noqa: E731
    p = min(rows, cols)
    if kind == "rank":
        # rank 5 at most, exactly so in bf16: whole numbers up to 20
        whole = lambda *s: torch.randint(-2, 3, (count, *s), generator=g, device="cuda").float()  # noqa: E731
        return torch.matmul(whole(rows, min(5, p)), whole(min(5, p), cols)).to(dtype)
    if kind == "one":
        return torch.matmul(n(rows, 1), n(1, cols)).to(dtype)
    if kind == "decay":
        # singular values from 1 down to 1e-6, evenly in their logarithm
        s = torch.logspace(0, -6, p, device="cuda")
        left, right = torch.linalg.qr(n(rows, p))[0], torch.linalg.qr(n(cols, p))[0]
        return torch.matmul(left * s, right.transpose(1, 2).contiguous()).to(dtype)
    # a few strong directions over noise, as gradients have them
    few = min(8, p)
    s = torch.arange(1, few + 1, device="cuda", dtype=F32).pow(-0.7)
    return (torch.matmul(n(rows, few) * s, n(few, cols)) + 0.03 * n(rows, cols)).mul_(1e-3).to(dtype)


# one launch; tiles of 64; X X^T cut along k; tiles of 128; of 256
@pytest.mark.parametrize("count,rows,cols", [(3, 64, 192), (2, 160, 100), (3, 1001, 333), (1, 256, 4096), (1, 1401, 1503),
                                             (1, 2000, 5000)])
@pytest.mark.parametrize("kind", ["rank", "one", "decay", "strong"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_uneven_singular_values(dtype, kind, count, rows, cols):
    x = uneven(kind, rows, count, rows, cols, dtype)
    got = fal.newton_schulz(x)
    want, bounds = exact(x, 5, COEF)
    hold(got, want, bounds, in_fp32(x, 5, COEF), 2.0 ** -8 if dtype == BF16 else U)
