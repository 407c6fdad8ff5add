"""kvio_check after attend, built for the CPU (as in test_attn_emulated.py): pages outside the pool are reported where some row
sees a token of theirs, and only there."""
import pytest
import torch

import test_emulated_kernels as base
from test_attn_blocks_emulated import case
from test_attn_emulated import emu  # noqa: F401  (a fixture)
from test_attn_precision_emulated import call

pytestmark = pytest.mark.skipif(not base.os.path.exists(base.CXX), reason="no clang++ (the sources use its vector types)")


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("new", [1, 4, 90])
@pytest.mark.parametrize("where,window,seen", [("first", 0, True), ("first", 20, False), ("last", 0, True), ("last", 20, True),
                                               ("behind", 0, False), ("edge", 20, True), ("no rows", 0, False)])
def test_pages_outside_the_pool_are_reported(emu, new, bits, where, window, seen):  # noqa: F811
    """Where some row sees a token of theirs, and only there, with the sequence and its page."""
    c = case(torch.bfloat16, bits, 2, 2, 64, 4, [(30, 2), (80, new), (0, 0), (33, new)], window=window, seed=new)
    c["max_query"] = max(2, new)
    ctx = 80 + new
    first_seen = max(0, 80 - window + 1) if window else 0
    b, j = {"first": (1, 0), "last": (1, (ctx - 1) // 4), "behind": (1, (ctx - 1) // 4 + 1), "edge": (1, first_seen // 4), "no rows": (2, 0)}[where]
    c["table"][b, j] = 1000
    out, lse, said = call(emu, c)
    if seen:
        assert said is not None and f"span {b}, context page {j}:" in said
    else:
        assert said is None
        c["table"][b, j] = 0 if where != "first" else c["table"][b, 1]
        again = call(emu, c)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
