"""append and attend built for the CPU (as in test_attn_emulated.py) at the ends of what their arguments may hold: scales
that are no numbers, zero or infinite, windows as long as an int, slices of one buffer."""
import ctypes
import math

import pytest
import torch

import test_emulated_kernels as base
from _attn_plain import append_plain, values
from test_attn_blocks_emulated import attend, case
from test_attn_emulated import TYPE, Box, batch_args, emu, make_pool  # noqa: F401  (a fixture)

pytestmark = pytest.mark.skipif(not base.os.path.exists(base.CXX), reason="no clang++ (the sources use its vector types)")


@pytest.mark.parametrize("which,odd", [("v", math.nan), ("v", math.inf), ("v", -math.inf), ("k", math.nan)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("new", [4, 70])
def test_a_hidden_tokens_scale_has_no_effect(emu, new, dtype, which, odd):  # noqa: F811
    """The last token's page, of one token, has such a scale: the rows before it stay as they are, bit for bit."""
    c = case(dtype, 8, 1, 2, 64, 1, [(20, new), (40, 3)], seed=new)
    out, lse = attend(emu, c)
    page = int(c["table"][0, 20 + new - 1])
    c["scales"][1 if which == "v" else 0, page, 0] = odd
    got, got_lse = attend(emu, c)                    # holds the last row to its infinities or NaN, too
    assert torch.equal(got[:new - 1], out[:new - 1]) and torch.equal(got[new:], out[new:])
    assert torch.equal(got_lse[:new - 1], lse[:new - 1]) and torch.equal(got_lse[new:], lse[new:])
    assert not bool(got[new - 1].isfinite().all())


@pytest.mark.parametrize("odd", [math.nan, math.inf])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("new", [2, 70])
def test_scales_that_all_rows_see(emu, new, dtype, odd):  # noqa: F811
    """Values times such a scale are infinite, or NaN (largest codes are made NaN, too): held to the definition's."""
    c = case(dtype, 8, 1, 1, 64, 32, [(130, new)], seed=new)
    page = int(c["table"][0, 1])
    c["pool"].view(torch.uint8)[1, page * 32:page * 32 + 32, 0] &= 0x7f     # of one sign in each dim: their sum is an infinity
    c["pool"].view(torch.uint8)[1, page * 32:page * 32 + 32, 0, ::2] |= 0x81
    c["pool"].view(torch.uint8)[1, page * 32:page * 32 + 32, 0, 1::2] |= 1
    c["scales"][1, page, 0] = odd
    out, _ = attend(emu, c)
    out = out[:new]
    assert bool(out.isnan().all()) if math.isnan(odd) else bool((out[..., ::2] == -math.inf).any() and (out[..., 1::2] == math.inf).any())
