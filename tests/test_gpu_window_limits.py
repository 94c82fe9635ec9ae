"""Windowed attention where its paths differ: rows of few keys under a long
window, divided head groups with whole key blocks, scores that keep raising a
row's maximum, and block calls of a context."""
import math

import pytest
import torch

from oracle import fal_oracle
from paper_2510_14614_amd import fal, synth

import test_gpu_block_abi as blocks_abi
import test_gpu_tuning_steps as steps
import test_gpu_window_attention as attention
from gpu_helpers import TOL, log, rel_err

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


@pytest.mark.parametrize("B,T,H,hd", [(2, 300, 3, 64), (40, 257, 8, 64), (3, 129, 2, 128), (40, 257, 16, 128),
                                      (1, 200, 2, 16), (64, 140, 16, 32)])
def test_first_rows_of_a_long_window(B, T, H, hd):
    # The first rows of a sequence see few keys, here of values so alike that
    # dS = P (dP - D) is a small difference: D from an output rounded to bf16
    # would be off by 2^-9 of D, as much as dS itself.  With D from products in
    # fp32 what is left is the rounding of dS and of the result.
    g = torch.Generator(device="cuda").manual_seed(hd)
    rows, r = 8, 2.0 ** -8
    x = torch.randn(B, T, 3, H, hd, device="cuda", generator=g)
    x[:, :rows, 2] = x[:, :1, 2] * (1 + torch.randn(B, rows, H, hd, device="cuda", generator=g) / 64)
    qkv = x.to(BF16).view(B, T, 3 * H * hd)
    dout = torch.randn(B, T, H * hd, device="cuda", generator=g).to(BF16)
    out, lse = fal.window_attention_fwd(qkv, H, T)
    got = fal.window_attention_bwd(qkv, out, dout, lse, H, T)[:, :rows, :H * hd].double()
    got = got.view(B, rows, H, hd).transpose(1, 2)
    # [B, H, rows, hd] each
    q, k, v = (t.transpose(1, 2) for t in qkv[:, :rows].double().view(B, rows, 3, H, hd).unbind(2))
    go = dout[:, :rows].double().view(B, rows, H, hd).transpose(1, 2)
    sc = 1 / math.sqrt(hd)
    see = torch.ones(rows, rows, dtype=torch.bool, device="cuda").tril()
    kt, vt = (t.transpose(-1, -2).contiguous() for t in (k, v))
    p = (q @ kt * sc).masked_fill(~see, -math.inf).softmax(-1)
    dp = go @ vt
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    # P is off by its score's two sums and its exponentials, D and dP - D by the
    # sums of hd products in fp32
    e = 2 * (hd + 4) * U * float((q.abs() @ kt.abs()).max()) * sc + (rows + 8) * U
    sums = (go.abs() @ vt.abs()).amax(-1, keepdim=True)
    err = (2 * e + r) * ds.abs() + p * (2 * e + (hd + 8) * U) * sums
    want = ds @ k * sc
    bound = (err @ k.abs() * sc + r * want.abs()) * 1.01
    worst = float(((got - want).abs() / (bound + 1e-30)).max())
    log(f"{B} x {T} x {H} x {hd}: worst error / bound {worst:.3f}")
    assert worst <= 1.0


def plan(B, T, H, kv, hd, window, dtype):
    """Parts that a group's query heads are divided into, from the workspace
    (without sinks: rowsum(dO * O), then the parts' fp32 sums of dK and dV)."""
    code = 1 if dtype == BF16 else 0
    n = fal._window_workspace(B, T, H, kv, hd, code, window, 0, (H + 2 * kv) * hd, H * hd)
    stat = (B * H * T * 4 + 255) // 256 * 256
    return (n - stat) // (B * T * 2 * kv * hd * 4)


@pytest.mark.parametrize("dtype,shape,parts", [
    # enough parts of long sequences that whole blocks of 128 keys fill the chip,
    # with and without sinks; in fp32 at head_dim 128 one round of them
    (BF16, (1, 4096, 16, 1, 64, 300, 5, (4001,)), 16),
    (F32, (1, 4096, 16, 1, 64, 300, 0, None), 16),
    (BF16, (1, 4096, 24, 1, 32, 1000, 37, (4096,)), 24),
    (F32, (1, 4096, 24, 1, 16, 90, 2, (3900,)), 24),
    (BF16, (16, 60, 32, 2, 128, 40, 3, tuple(range(60, 28, -2))), 16),
    (F32, (1, 2100, 8, 1, 128, 300, 5, (2051,)), 8),
    # halved blocks
    (BF16, (1, 4096, 16, 2, 128, 1024, 16, (4096,)), 4),
    (F32, (2, 600, 16, 2, 64, 100, 3, (600, 430)), 8),
], ids=lambda v: "x".join(map(str, v[:7])) if isinstance(v, tuple) else str(v).replace("torch.", ""))
def test_divided_head_groups(dtype, shape, parts):
    B, T, H, kv, hd, window = shape[:6]
    assert plan(B, T, H, kv, hd, window, dtype) == parts
    attention.test_against_the_formula(shape, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("B,H,hd", [(1, 2, 64), (2, 2, 128), (40, 8, 64), (20, 16, 128)])
@pytest.mark.parametrize("kind", ["rising", "falling", "sinks"])
def test_scores_that_move_the_maximum(kind, B, H, hd, dtype):
    # Every 32 keys the scores of all rows move by 7: a row's maximum passes its
    # reference by 10 log2 units at every half tile, with sums that still count
    # for 1e-3 of what follows ("falling": never again after the first; "sinks":
    # by 40 from the window to the sinks and back).
    T, window, sinks = 300, 140, 3 if kind == "sinks" else 0
    g = torch.Generator(device="cuda").manual_seed(hd + len(kind))
    x = torch.randn(B, T, 3, H, hd, device="cuda", generator=g)
    t = torch.arange(T, device="cuda")
    level = {"rising": 7.0 * (t // 32), "falling": -7.0 * (t // 32), "sinks": torch.where(t < 3, 40.0, 0.0) +
             torch.where(t % 64 < 32, 0.0, 7.0)}[kind]
    x[:, :, 0, :, 0] = math.sqrt(hd)  # the score's part of dim 0 is the key's level
    x[:, :, 1, :, 0] = level[None, :, None]
    qkv = x.to(dtype).view(B, T, 3 * H * hd)
    dout = torch.randn(B, T, H * hd, device="cuda", generator=g).to(dtype)
    want, bound = attention.reference(qkv, H, H, hd, window, sinks, [T] * B, dout)
    out, lse = fal.window_attention_fwd(qkv, H, window, sinks)
    dqkv = fal.window_attention_bwd(qkv, out, dout, lse, H, window, sinks)
    for name, got, i in (("out", out, 0), ("lse", lse, 1), ("dqkv", dqkv, 2)):
        attention.check(name, got, want[i], bound[i])


@pytest.mark.parametrize("dtype", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("arch,block1_mode", blocks_abi.CASES)
def test_windowed_block_calls(arch, block1_mode, dtype, monkeypatch):
    # fal_block_fwd / fal_block_bwd under a window against the oracle, and
    # bitwise against the stack step under the same window
    window, sinks = 37, 2
    init = fal.Fal.__init__

    def windowed(self, *args, **kw):
        init(self, *args, **kw)
        self.set_attention_window(window, sinks)

    monkeypatch.setattr(fal.Fal, "__init__", windowed)
    monkeypatch.setattr(fal_oracle, "attention", steps.masked(window, sinks))
    blocks_abi.test_block_calls_match_oracle_and_stack_step(arch, block1_mode, dtype)


def test_windowed_blocks_differ_from_the_full_mask():
    # (the window above reaches the block calls)
    cfg = blocks_abi._cfg(blocks_abi.ARCH_GPT, 0, 0)
    _, params = synth.make_params(cfg, seed=70)
    x1, gout = synth.make_stack_inputs(cfg, seed=71)
    F = fal.Fal(cfg)
    F.load_params({}, params)
    full = blocks_abi._run_blocks(F, cfg, x1, gout)
    F.set_attention_window(37, 2)
    got = blocks_abi._run_blocks(F, cfg, x1, gout)
    F.set_attention_window(cfg.seq_len)
    all_of_it = blocks_abi._run_blocks(F, cfg, x1, gout)
    F.close()
    for a, b, c in zip(full, got, all_of_it):
        assert rel_err(b, a) > 1e-3 and rel_err(c, a) <= TOL[0]
