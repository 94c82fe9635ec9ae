"""Windowed attention where its paths differ: rows of few keys under a long
window, divided head groups with whole key blocks, scores that keep raising a
row's maximum, and block calls of a context."""
import math

import numpy as np
import pytest
import torch

from paper_2510_14614_amd import fal

from gpu_helpers import log

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
