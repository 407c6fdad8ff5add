"""What attend, built for the CPU (as in test_attn_emulated.py), loses: short contexts, whose results show the rounding of
single probabilities wherever values cancel, held to what each kernel carries."""
import ctypes
import math

import pytest
import torch

import test_emulated_kernels as base
from _attn_plain import STEP, page_at, rows_of, values
from test_attn_blocks_emulated import case
from test_attn_emulated import TYPE, Box, batch_args, emu, make_pool  # noqa: F401  (a fixture)

pytestmark = pytest.mark.skipif(not base.os.path.exists(base.CXX), reason="no clang++ (the sources use its vector types)")


def call(emu, c):  # noqa: F811
    """out, lse and what kvio_check says (None: nothing)."""
    kv, lib, A = emu
    box = Box(kv)
    _, h = make_pool(kv, box, c)
    N, Hq, D = c["q"].shape
    a = A.kvio_attend_args(batch=batch_args(A, box, c, c["table"], c["ctx"], c["starts"], N, c["max_query"]),
                           dtype=TYPE[c["dtype"]], cache_dtype=TYPE[c["dtype"]] if c["scales"] is None else 2,
                           num_q_heads=Hq, window=c["window"], softmax_scale=1 / math.sqrt(D), q_stride=Hq * D, out_stride=Hq * D)
    a.q = box.put(c["q"])[1]
    out, a.out = box.put(c["q_out"])
    lse, a.lse = box.put(torch.full((N, Hq), 7.0))
    if c["scales"] is not None:
        a.k_scale = box.put(c["scales"])[1]
        a.v_scale, a.scale_stride = a.k_scale + 4 * c["scales"][0].numel(), c["scales"].shape[2]
    need = ctypes.c_size_t()
    assert lib.kvio_attend_workspace(h, ctypes.byref(a), ctypes.byref(need)) == 0, kv.kvio_last_error()
    if need.value:
        a.workspace, a.workspace_bytes = box.put(torch.full((need.value,), 255, dtype=torch.uint8))[1], need.value
    assert lib.kvio_attend(h, 0, ctypes.byref(a), None) == 0, kv.kvio_last_error()
    said = None
    try:
        kv.kvio_check(h)
    except kv.KvioError as e:
        assert e.status == kv.KVIO_ERANGE
        said = str(e)
    got = out.clone(), lse.clone(), said
    kv.kvio_pool_destroy(h)
    box.free()
    return got


def exact(c):
    """out in 64 bits, and the tolerance by what a probability loses (`loss`, relative)."""
    G, D, P, is8 = c["Hq"] // c["H"], c["D"], c["P"], c["scales"] is not None
    pool = values(c["pool"]) if is8 else c["pool"].double()
    want, reach, off, least = (torch.zeros(c["q"].shape, dtype=torch.float64) for _ in range(4))
    for b, r0, rows, first, ctx in rows_of(c):
        at = torch.tensor([page_at(c, b, t) * P + t % P for t in range(ctx)])
        k, v = pool[0, at], pool[1, at]
        unit = torch.ones(c["H"])
        if is8:
            k, v = (x * c["scales"][i, at // P].double()[:, :, None] for i, x in ((0, k), (1, v)))
            unit = c["scales"][1, at // P].amax(0) / 64          # a ValueUnit is at most that
        for h in range(c["Hq"]):
            q = c["q"][r0:r0 + rows, h].double()
            dot = q @ k[:, h // G].t() / math.sqrt(D)
            size = (q.abs() @ k[:, h // G].abs().t() / math.sqrt(D)).amax(1, keepdim=True)
            dot.masked_fill_(torch.arange(ctx) > first + torch.arange(rows)[:, None], -math.inf)
            p = torch.softmax(dot, 1)
            want[r0:r0 + rows, h], reach[r0:r0 + rows, h] = p @ v[:, h // G], p @ v[:, h // G].abs()
            # scores: sums of D products in 32 bits, and the exponent's; the sums of probabilities and values; constants
            off[r0:r0 + rows, h] = size * (D + 8) * 2.0 ** -24 + dot.amax(1, keepdim=True).abs() * 2.0 ** -22 + ctx * 2.0 ** -23 + 2.0 ** -20
            if is8 or c["dtype"] == torch.float16:               # fp16 has steps of 2^-24 at least
                size = v[:, h // G].abs().sum(0) if not is8 else pool[1, at][:, h // G].abs().sum(0) * unit[h // G]
                least[r0:r0 + rows, h] = size * 2.0 ** -25 + (2.0 ** -25 if c["dtype"] == torch.float16 else 0)
    return want, reach, off, least


@pytest.mark.parametrize("G,new", [(1, 1), (2, 4), (4, 12), (2, 70), (3, 90)])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [8, 16])
def test_what_probabilities_lose(emu, bits, dtype, D, G, new):  # noqa: F811
    """Half a step of their type, or with a second term (steps, but for bf16 queries over e4m3) half a step of half a step."""
    if new > 16 and D == 256 and bits == 8 and dtype == torch.float16:
        new = 40                                                   # time; more than 32 rows all the same
    c = case(dtype, bits, 2, G, D, 16, [(b % 4 + 1, new if b % 2 else max(1, new - b)) for b in range(6)], seed=D + new)
    c["max_query"] = new
    c["q"] = c["q"] * 0.125                                         # scores near each other: several keys count, and scores are exact enough
    if bits == 8:
        c["scales"][1] *= 2.0 ** torch.randint(-6, 7, c["scales"][1].shape, generator=torch.Generator().manual_seed(new))
    steps = new * G <= (64 if D <= 128 else 32)
    half = STEP[torch.float16 if bits == 8 else dtype]
    loss = half * half if steps and not (bits == 8 and dtype == torch.bfloat16) else half
    out, _, said = call(emu, c)
    want, reach, off, least = exact(c)
    N = int(c["starts"][-1])
    tol = want.abs() * STEP[dtype] + reach * (loss + 2 * off) * 1.01 + least
    bad = ~((out.double() - want).abs() <= tol)[:N]
    assert not bool(bad.any()), (int(bad.sum()), bad.numel())
    assert said is None and bool((out[N:] == -2.5).all())


@pytest.mark.parametrize("new,window", [(1, 0), (12, 0), (90, 0), (90, 350)])
def test_small_fp16_probabilities_that_add_up(emu, new, window):  # noqa: F811
    """One token takes nearly all of a row's probability, its value is small; hundreds that have 2^-27 of it and large values
    make the result."""
    c = case(torch.float16, 16, 1, 2, 64, 16, [(400, new)], window=window, seed=new)
    c["max_query"] = new
    ctx = 400 + new
    place = torch.arange(ctx)
    slots = c["table"][0, place // 16].long() * 16 + place % 16
    gen = torch.Generator().manual_seed(1)
    c["pool"][0, slots] = 0
    c["pool"][1, slots] = (1000 + torch.rand(ctx, 1, 64, generator=gen) * 500).half()
    strong = slots[max(0, ctx - new - 30)]                          # in every row's window
    c["pool"][0, strong, 0, 0], c["pool"][1, strong] = 8, 2.0 ** -10
    c["q"][:] = 0
    c["q"][..., 0] = 27 * math.log(2)                               # times 8 / sqrt(64)
    out, lse, _ = call(emu, c)
    k, v = c["pool"][0, slots, 0].double(), c["pool"][1, slots, 0].double()
    for i in range(new):
        seen = torch.arange(max(0, 400 + i - window + 1) if window else 0, 400 + i + 1)
        s = k[seen] @ c["q"][i, 0].double() / 8
        p = torch.softmax(s, 0)
        want = p @ v[seen]
        # a probability is exact here but for half a step of fp16, its exponent's error (2^-24 of 27), and 2^-32 of the largest
        tol = want * (2 * STEP[torch.float16] + 27 * 2.0 ** -23 + len(seen) * 2.0 ** -23) + len(seen) * 2.0 ** -32 * 1500 + 2.0 ** -25
        assert bool(((out[i].double() - want).abs() <= tol).all()), (i, out[i, 0, :3], want[:3])
        assert abs(float(lse[i, 0]) - float(torch.logsumexp(s, 0))) <= 2.0 ** -18
