"""Host-only checks of the operators' limits: sizes that the library's 32-bit
fields and column counts do not hold are refused before anything is launched."""
import ctypes
from ctypes import byref, c_void_p

import pytest
import torch

from paper_2510_14614_amd import fal

# addresses that no call may reach: 1 TiB apart
A, B, C, D, E, F, G = (c_void_p((i + 1) << 40) for i in range(7))
BAD = fal.FAL_ERR_INVALID_ARG


def message():
    return fal.lib().fal_last_error(None).decode()


@pytest.mark.parametrize("cols", [(1 << 30) + 1, (1 << 31) - 16, (1 << 31) - 1])
def test_gradient_rows_past_the_column_count(cols):
    # columns are counted in 32 bits, a workgroup's stride past the last one
    # included
    L, n = fal.lib(), ctypes.c_size_t()
    r = fal.fal_logit_rows_t(1, 2, 100, 1, 100, 2, 1 << 31, cols, 1.0)
    pol, pref = fal.fal_policy_t(0.2, 0.2, 0.0, 0), fal.fal_preference_t(0.1, 0.0, 0, 0)
    assert L.fal_logit_loss_workspace_bytes(byref(r), byref(n)) == BAD
    assert "dlogits_cols" in message()
    assert L.fal_policy_loss(byref(r), byref(pol), A, B, None, C, None, D, E, None, F, G, 1 << 29, None) == BAD
    assert "dlogits_cols" in message()
    r.batch = 2
    assert L.fal_preference_loss(byref(r), byref(pref), A, B, None, C, D, None, E, F, 1 << 29, None) == BAD
    assert "dlogits_cols" in message()
    r.dlogits_cols = 1 << 30
    assert L.fal_logit_loss_workspace_bytes(byref(r), byref(n)) == fal.FAL_OK


def test_binding_keeps_sizes_past_32_bits():
    # sizes reach the library as they are or larger than it allows, never cut
    # to their last 32 bits
    def rows(B, T, V, vocab=None):
        x = torch.empty(B, T, V, dtype=torch.bfloat16, device="meta")
        y = torch.empty(B, T, dtype=torch.int32, device="meta")
        return x, fal._logit_rows(x, y, None, vocab, 1.0)

    most = (1 << 31) - 1
    for args, field in (((2 ** 32 + 1, 1, 8), "batch"), ((1, 2 ** 32 + 1, 8), "seq_len"), ((1, 1, 2 ** 32 + 8), "vocab")):
        _, r = rows(*args)
        assert getattr(r, field) == most
        assert fal.lib().fal_token_logprobs(byref(r), A, B, None, C, None, None) == BAD
    x, r = rows(1, 2, 2 ** 32 + 8, vocab=8)
    assert r.vocab == 8 and r.dlogits_cols == most
    with pytest.raises(ValueError, match="2\\^30"):
        fal._gradient_rows(r, x, None)
    with pytest.raises(ValueError, match="2\\^30"):
        fal._gradient_rows(rows(1, 2, (1 << 30) + 1, vocab=8)[1], x, x)
