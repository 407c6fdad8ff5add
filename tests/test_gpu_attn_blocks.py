"""attend's two kernels on an MI355X where they meet, work shared by many workgroups, calls side by side and graphs in turn."""
import math

import pytest

from test_gpu_attn import filled, hold, kv, on_gpu  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("D,G,new", [(128, 1, 63), (128, 1, 64), (128, 1, 65), (128, 16, 4), (128, 13, 5), (64, 7, 9), (64, 7, 10), (128, 6, 8), (128, 3, 11),
                                     (256, 4, 8), (256, 3, 11), (256, 1, 128), (256, 1, 129), (64, 256, 1), (128, 250, 2), (128, 5, 52)])
def test_rows_at_the_borders(kv, D, G, new, bits):  # noqa: F811
    """As many rows to a KV head as a wave, three quarters of one, a block hold, and one more."""
    import torch
    c = filled(bits, torch.bfloat16, 2 * G, 2, D, 16, [(500, new), (0, new), (37, max(1, new - 1))], seed=D + G + new)
    g, pool, batch = on_gpu(kv, c)
    for window in (0, 33):
        hold(c, pool.attend(0, batch, g["q"], window=window), g, window)
    pool.close()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("D,H,G,lens,window", [
    (128, 1, 4, [(30000, 70)], 0), (64, 1, 8, [(20000, 100), (5, 300)], 0), (256, 2, 4, [(9000, 50)], 0),
    (128, 8, 1, [(3 * b, 65 + b % 26) for b in range(40)], 0), (128, 2, 5, [(0, 700), (2000, 90)], 300),
    (64, 2, 3, [(0, 2000)], 1), (128, 1, 1, [(0, 4097)], 0)])
def test_blocks_that_workgroups_share(kv, D, H, G, lens, window, bits):  # noqa: F811
    import torch
    c = filled(bits, torch.float16, H * G, H, D, 24, lens, seed=len(lens) + D)
    g, pool, batch = on_gpu(kv, c)
    lse = torch.empty(g["q"].shape[:2], device="cuda")
    out = pool.attend(0, batch, g["q"], window=window, lse=lse)
    hold(c, out, g, window)
    again = torch.empty_like(lse)
    assert torch.equal(out, pool.attend(0, batch, g["q"], window=window, lse=again)) and torch.equal(lse, again)
    # lse is off by no more than the scores' exponents and sums in 32 bits are (hold's `off`): looked at for one head
    ctx, n = lens[0][0] + lens[0][1], lens[0][1]
    t = torch.arange(ctx, device="cuda")
    slot = g["table"][0].long()[t // 24] * 24 + t % 24
    k = g["pool"][0, 0, :, 0].view(torch.uint8 if bits == 8 else torch.float16)[slot]
    k = k.view(torch.float8_e4m3fn).float().double() * g["scales"][0, 0, :, 0].double()[slot // 24][:, None] if bits == 8 else k.double()
    q = g["q"][:n, 0].double()
    dot = q @ k.t().contiguous() / math.sqrt(D)
    place = (ctx - n + torch.arange(n, device="cuda"))[:, None]
    hidden = (t > place) | (t <= place - window) if window else t > place
    want = torch.logsumexp(dot.masked_fill(hidden, -math.inf), 1)
    size = (q.abs() @ k.abs().t().contiguous()).amax(1) / math.sqrt(D)
    off = size * (D + 8) * 2.0 ** -24 + size * 2.0 ** -22 + ctx * 2.0 ** -23 + 2.0 ** -20 + want.abs() * 2.0 ** -22
    assert bool(((lse[:n, 0].double() - want).abs() <= 2 * off).all())
    pool.close()


def test_calls_side_by_side(kv):  # noqa: F811
    """Prompts and steps on two streams at once, each with its own workspace, give what they give one after the other."""
    import torch
    c = filled(16, torch.bfloat16, 16, 4, 128, 16, [(4000, 200), (100, 300)], seed=31)
    d = filled(16, torch.bfloat16, 16, 4, 128, 16, [(9000, 1), (20, 1), (3000, 1)], seed=32)
    (gc, pc, bc), (gd, pd, bd) = on_gpu(kv, c), on_gpu(kv, d)
    want = pc.attend(0, bc, gc["q"]), pd.attend(0, bd, gd["q"])
    spaces = [torch.full((kv.attend_workspace(p, b, g["q"]) + 16,), 255, dtype=torch.uint8, device="cuda") for p, b, g in ((pc, bc, gc), (pd, bd, gd))]
    outs = [[torch.empty_like(gc["q"]) for _ in range(6)], [torch.empty_like(gd["q"]) for _ in range(6)]]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(6):
        pc.attend(0, bc, gc["q"], out=outs[0][i], workspace=spaces[0], stream=streams[0])
        pd.attend(0, bd, gd["q"], out=outs[1][i], workspace=spaces[1], stream=streams[1])
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for o, w in zip(outs, want) for x in o)
    pc.close()
    pd.close()


def test_two_graphs_in_turn(kv):  # noqa: F811
    """Two captured calls that share a workspace, replayed one after the other with eager calls between."""
    import torch
    c = filled(8, torch.bfloat16, 8, 2, 128, 16, [(3000, 90), (50, 40)], seed=33)
    g, pool, batch = on_gpu(kv, c)
    steps = kv.Batch(g["table"], g["ctx"])
    qs = g["q"][:2].clone()
    space = torch.empty(max(kv.attend_workspace(pool, batch, g["q"]), kv.attend_workspace(pool, steps, qs)), dtype=torch.uint8, device="cuda")
    calls = [(batch, g["q"], torch.empty_like(g["q"])), (steps, qs, torch.empty_like(qs))]
    graphs = []
    for b, q, o in calls:
        pool.attend(0, b, q, out=o, workspace=space)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pool.attend(0, b, q, out=o, workspace=space)
        graphs.append(graph)
    for rep in range(3):
        g["q"].add_(0.25)
        qs.mul_(0.75)
        for i in ((0, 1), (1, 0), (0, 1))[rep]:
            graphs[i].replay()
        torch.cuda.synchronize()
        space.fill_(255)
        for b, q, o in calls:
            assert torch.equal(o, pool.attend(0, b, q))
    del graphs
    pool.close()


@pytest.mark.parametrize("new", [1, 3, 80])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_fp16_keeps_its_precision_over_an_8_bit_cache(kv, D, new):  # noqa: F811
    """Scales that grow and shrink by 2^20 along the context; probabilities lose half a step of fp16, 2^-11, not of bf16."""
    import torch
    ctx, P, G = 3000, 16, 4
    c = filled(8, torch.float16, 2 * G, 2, D, P, [(ctx - new, new)], seed=D + new)
    pages = c["scales"].shape[1]
    gen = torch.Generator().manual_seed(5)
    c["scales"][1] *= 2.0 ** torch.randint(-10, 11, (pages, 2), generator=gen)
    g, pool, batch = on_gpu(kv, c)
    out = pool.attend(0, batch, g["q"])
    t = torch.arange(ctx, device="cuda")
    slot = g["table"][0].long()[t // P] * P + t % P
    for h in range(2 * G):
        k, v = (g["pool"][i, 0, :, h // G].view(torch.uint8)[slot].view(torch.float8_e4m3fn).float().double() *
                g["scales"][i, 0, :, h // G].double()[slot // P][:, None] for i in (0, 1))
        q = g["q"][:, h].double()
        place = (ctx - new + torch.arange(new, device="cuda"))[:, None]
        p = torch.softmax((q @ k.t().contiguous() / math.sqrt(D)).masked_fill(t > place, -math.inf), 1)
        want, reach = p @ v, p @ v.abs()
        size = (q.abs() @ k.abs().t().contiguous()).amax(1, keepdim=True) / math.sqrt(D)
        off = size * (D + 8) * 2.0 ** -24 + size * 2.0 ** -22 + ctx * 2.0 ** -23 + 2.0 ** -20
        # steps of 2^-24 times a unit of at most 2^-6 of the largest scale, for each key's share
        least = ctx * 2.0 ** -31 * float(g["scales"][1].max()) * 448
        tol = want.abs() * 2.0 ** -11 + reach * (2.0 ** -11 + 2 * off) * 1.01 + least + 2.0 ** -25
        assert bool(((out[:, h].double() - want).abs() <= tol).all()), h
    pool.close()
