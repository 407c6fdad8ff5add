"""What attend loses on an MI355X, as test_attn_precision_emulated.py holds it on the CPU, and over many short contexts."""
import pytest

from _attn_plain import STEP
from test_attn_blocks_emulated import case
from test_attn_precision_emulated import exact
from test_gpu_attn import kv, on_gpu  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G,new", [(1, 1), (4, 1), (2, 4), (4, 12), (2, 70), (3, 90)])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("bits", [8, 16])
def test_what_probabilities_lose(kv, bits, dtype, D, G, new):  # noqa: F811
    import torch
    dtype = getattr(torch, dtype)
    c = case(dtype, bits, 2, G, D, 16, [(b % 7 + 1, new if b % 2 else max(1, new - b)) for b in range(24)], seed=D + new)
    c["max_query"] = new
    c["q"] = c["q"] * 0.125
    if bits == 8:
        c["scales"][1] *= 2.0 ** torch.randint(-6, 7, c["scales"][1].shape, generator=torch.Generator().manual_seed(new))
    steps = new * G <= (64 if D <= 128 else 32)
    half = STEP[torch.float16 if bits == 8 else dtype]
    loss = half * half if steps and not (bits == 8 and dtype == torch.bfloat16) else half
    g, pool, batch = on_gpu(kv, c)
    N = int(c["starts"][-1])
    out = pool.attend(0, batch, g["q"], out=g["q_out"]).cpu()
    want, reach, off, least = exact(c)
    tol = want.abs() * STEP[dtype] + reach * (loss + 2 * off) * 1.01 + least
    bad = ~((out.double() - want).abs() <= tol)[:N]
    assert not bool(bad.any()), (int(bad.sum()), bad.numel())
    assert bool((out[N:] == -2.5).all())
    pool.check()
    pool.close()
