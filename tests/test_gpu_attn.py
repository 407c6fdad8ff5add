"""append and attend on an MI355X, through KVPool, against plain 64-bit computations."""
import math

import pytest

from _attn_plain import STEP, append_plain, attend_plain, random_batch, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an AMD GPU"
    import paper_2508_18572_amd as kv
    return kv


def on_gpu(kv, c):
    """The case's tensors on the GPU, a pool handle over them (one layer) and the batch."""
    import torch
    g = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in c.items()}
    _, S, H, D = c["pool"].shape
    g["pool"] = g["pool"].view(2, 1, S, H, D)
    if c["scales"] is not None:
        g["scales"] = g["scales"].unsqueeze(1).contiguous()
    pool = kv.KVPool(g["pool"], c["P"], scales=g["scales"])
    return g, pool, kv.Batch(g["table"], g["ctx"], g["starts"], c["max_query"])


@pytest.mark.parametrize("seed", range(40))
def test_append_random(kv, seed):
    import torch
    c = random_batch(seed, "append")
    g, pool, batch = on_gpu(kv, c)
    pool.append(0, batch, g["k"], g["v"], q=g["q"], q_out=g["q_out"], inv_freq=g["inv_freq"] if c["rot"] else None,
                positions=g["positions"], interleaved=c["interleaved"])
    torch.cuda.synchronize()
    append_plain(c, g["pool"].cpu().squeeze(1), None if c["scales"] is None else g["scales"].cpu().squeeze(1),
                 g["q_out"].cpu())
    if c["bad"]:
        with pytest.raises(kv.KvioError) as e:
            pool.check()
        assert e.value.status == kv.KVIO_ERANGE
    pool.check()
    pool.close()


@pytest.mark.parametrize("seed", range(64))
def test_attend_random(kv, seed):
    import torch
    c = random_batch(seed, "attend")
    g, pool, batch = on_gpu(kv, c)
    lse = torch.full(c["q"].shape[:2], 7.0, device="cuda")
    pool.attend(0, batch, g["q"], out=g["q_out"], lse=lse, window=c["window"])
    torch.cuda.synchronize()
    attend_plain(c, g["q_out"].cpu(), lse.cpu())
    pool.close()


def filled(bits, dtype, Hq, H, D, P, lens, seed=0, spare=3):
    """A case of (cached, new) lengths without oddities, as random_batch gives them."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    counts = [-(-(a + b) // P) for a, b in lens]
    pages = sum(counts) + spare
    order, at = torch.randperm(pages, generator=gen).int(), 0
    table = torch.full((len(lens), max(max(counts), 1)), -1, dtype=torch.int32)
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    N = sum(n for _, n in lens)
    x = torch.randn(2, pages * P, H, D, generator=gen)
    scales = None
    if bits == 8:
        x = (x * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
        scales = 0.02 * (0.5 + torch.rand(2, pages, H, generator=gen))
    else:
        x = x.to(dtype)
    return {"dtype": dtype, "H": H, "Hq": Hq, "D": D, "P": P, "pool": x, "scales": scales, "table": table,
            "ctx": torch.tensor([a + b for a, b in lens], dtype=torch.int32), "max_query": max(n for _, n in lens),
            "starts": torch.tensor([sum(n for _, n in lens[:b]) for b in range(len(lens) + 1)], dtype=torch.int32),
            "q": (torch.randn(N, Hq, D, generator=gen) * 1.5).to(dtype), "q_out": torch.full((N, Hq, D), -2.5, dtype=dtype),
            "window": 0}


def hold(c, out, g, window=0):
    """out against 64 bits, on the GPU: attend_plain's bounds with the seen values' sizes, by sequence and head."""
    import torch
    P, G, at = c["P"], c["Hq"] // c["H"], 0
    p_eps = STEP[torch.bfloat16 if c["scales"] is not None else c["dtype"]]
    new = (c["starts"][1:] - c["starts"][:-1]).tolist()
    for b, (ctx, n) in enumerate(zip(c["ctx"].tolist(), new)):
        t = torch.arange(ctx, device="cuda")
        slot = g["table"][b].long()[t // P] * P + t % P
        for h in range(c["H"]):
            k, v = (g["pool"][i, 0, :, h].view(torch.uint8 if c["scales"] is not None else c["dtype"])[slot] for i in (0, 1))
            if c["scales"] is not None:
                k, v = (values(x) * g["scales"][i, 0, :, h].double()[slot // P][:, None] for i, x in ((0, k), (1, v)))
            k, v = k.double(), v.double()
            q = g["q"][at:at + n, h * G:(h + 1) * G].double().reshape(n * G, -1)
            place = (ctx - n + torch.arange(n, device="cuda")).repeat_interleave(G)[:, None]
            hidden = (t > place) | (t <= place - window) if window else t > place
            dot = (q @ k.t().contiguous() / math.sqrt(c["D"]))
            size = (q.abs() @ k.abs().t().contiguous()).amax(1, keepdim=True) / math.sqrt(c["D"])
            p = torch.softmax(dot.masked_fill(hidden, -math.inf), 1)
            want, reach = p @ v, p @ v.abs()
            off = size * (c["D"] + 8) * 2.0 ** -24 + size * 2.0 ** -22 + ctx * 2.0 ** -23 + 2.0 ** -20
            got = out[at:at + n, h * G:(h + 1) * G].double().reshape(n * G, -1)
            tol = want.abs() * STEP[c["dtype"]] + reach * (p_eps + 2 * off) * 1.01 + (ctx * 2.0 ** -25 * 6 if c["dtype"] == torch.float16 else 0)
            bad = ~((got - want).abs() <= tol)
            assert not bool(bad.any()), (b, h, int(bad.sum()), [float(x.expand_as(bad)[bad][0]) for x in (got, want, tol)])
        at += n


LENGTHS = {
    "one_long": [(70001, 1)],
    "ragged_steps": [(5000, 1), (3, 1), (0, 1), (20000, 1), (63, 1), (64, 1), (999, 1)],
    "drafts": [(4096, 5), (77, 5), (0, 5), (9000, 5)],
    "rest": [(6000, 300), (130, 64), (1, 500)],
    "prompts": [(0, 1500), (0, 1), (0, 129), (10, 777)],
}


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("heads", [(8, 8, 64, 16, "fp16"), (14, 2, 128, 1, "bf16"), (32, 2, 128, 24, "bf16"), (6, 3, 256, 64, "fp16"),
                                   (8, 2, 128, 256, "fp16"), (20, 1, 64, 5, "bf16")], ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("lengths", list(LENGTHS))
def test_attend_lengths(kv, lengths, heads, bits):
    import torch
    Hq, H, D, P, dt = heads
    c = filled(bits, {"bf16": torch.bfloat16, "fp16": torch.float16}[dt], Hq, H, D, P, LENGTHS[lengths], seed=len(lengths))
    g, pool, batch = on_gpu(kv, c)
    for window in (0, 200):
        out = pool.attend(0, batch, g["q"], window=window)
        hold(c, out, g, window)
        # the same bits again, also where nothing says how many new tokens a sequence has at most
        assert torch.equal(out, pool.attend(0, batch, g["q"], window=window))
        hold(c, pool.attend(0, kv.Batch(g["table"], g["ctx"], g["starts"]), g["q"], window=window), g, window)
    pool.close()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("new", [1, 4, 90])
def test_what_hidden_tokens_hold_has_no_effect(kv, new, bits):
    """NaN and infinities in tokens that some rows see and others do not: the others' results stay as they are."""
    import torch
    c = filled(bits, torch.bfloat16, 8, 2, 128, 16, [(150, new), (40, new)], seed=3)
    g, pool, batch = on_gpu(kv, c)
    clean = pool.attend(0, batch, g["q"], out=torch.empty_like(g["q"])).clone()
    last = int(c["ctx"][0]) - 1
    slot = int(c["table"][0, last // 16]) * 16 + last % 16
    raw = g["pool"].view(torch.uint8 if bits == 8 else torch.int16)
    raw[1, 0, slot, 0, 5] = 0x7f if bits == 8 else 0x7f80          # V: NaN in e4m3, else +inf, in one dim
    got = pool.attend(0, batch, g["q"], out=torch.empty_like(g["q"]))
    assert torch.equal(got[:new - 1], clean[:new - 1]) and torch.equal(got[new:], clean[new:])
    row = got[new - 1, :4]                                         # the last row's heads on KV head 0
    assert bool(row[:, 5].isnan().all() if bits == 8 else (row[:, 5] == math.inf).all())
    keep = [d for d in range(128) if d != 5]
    assert torch.equal(row[:, keep], clean[new - 1, :4][:, keep]) and torch.equal(got[new - 1, 4:], clean[new - 1, 4:])
    raw[0, 0, slot, 0, 9] = 0x7f if bits == 8 else 0x7fc0          # K: NaN
    got = pool.attend(0, batch, g["q"], out=torch.empty_like(g["q"]))
    assert torch.equal(got[:new - 1], clean[:new - 1]) and torch.equal(got[new:], clean[new:])
    assert bool(got[new - 1, :4].isnan().all()) and torch.equal(got[new - 1, 4:], clean[new - 1, 4:])
    pool.close()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("new", [1, 40])
def test_graph_replays_follow_the_lengths(kv, new, bits):
    """append and attend captured once and replayed with other tokens, lengths and pages, eager work in between."""
    import torch
    H, Hq, D, P, B = 2, 8, 128, 16, 3
    gen = torch.Generator().manual_seed(5)
    c = filled(bits, torch.bfloat16, Hq, H, D, P, [(900, new), (300, new), (0, new)], seed=9, spare=80)
    g, pool, _ = on_gpu(kv, c)
    table = torch.randperm(g["pool"].shape[2] // P, generator=gen)[:B * 35].view(B, 35).int().cuda()
    ctx, starts = torch.zeros(B, dtype=torch.int32, device="cuda"), (torch.arange(B + 1, dtype=torch.int32) * new).cuda()
    batch = kv.Batch(table, ctx, starts, max_query=new)
    N = B * new
    fused = torch.zeros(N, (Hq + 2 * H) * D, dtype=torch.bfloat16, device="cuda")
    q, k, v = (x.view(N, -1, D) for x in fused.split((Hq * D, H * D, H * D), 1))
    inv = (10000.0 ** (-torch.arange(0, D, 2) / D)).float().cuda()

    def step(q_out=None, out=None):
        q_out = pool.append(0, batch, k, v, q=q, q_out=q_out, inv_freq=inv)
        return q_out, pool.attend(0, batch, q_out, out=out)

    ctx.fill_(new)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qg, og = step()
    pool_before = g["pool"].clone()
    for rep in range(4):
        fused.copy_(torch.randn(fused.shape, generator=gen))
        ctx.copy_(torch.tensor([new, new + rep * 130, min(560, new + 1 + rep * 90)], dtype=torch.int32))
        keep_pool, keep_scales = g["pool"].clone(), None if bits == 16 else g["scales"].clone()
        graph.replay()
        torch.cuda.synchronize()
        after, qa, oa = g["pool"].clone(), qg.clone(), og.clone()
        after_scales = None if bits == 16 else g["scales"].clone()
        g["pool"].copy_(keep_pool)
        if bits == 8:
            g["scales"].copy_(keep_scales)
        qe, oe = step()
        torch.cuda.synchronize()
        assert torch.equal(after.view(torch.uint8), g["pool"].view(torch.uint8)) and torch.equal(qa, qe) and torch.equal(oa, oe), rep
        assert bits == 16 or torch.equal(after_scales, g["scales"])
    assert not torch.equal(pool_before.view(torch.uint8), g["pool"].view(torch.uint8))
    del graph
    pool.close()


def test_append_attend_offload_load(kv):
    """A conversation: a prompt, a few steps; its codes and scales offloaded, loaded into other pages of another
    pool, where the next step gives the same bits."""
    import torch
    L, Hq, H, D, P, S = 2, 16, 4, 128, 16, 1024
    gen = torch.Generator(device="cuda").manual_seed(11)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    inv = (500000.0 ** (-torch.arange(0, D, 2) / D)).float().cuda()
    pools = []
    for _ in range(2):
        codes = torch.randint(0, 127, (2, L, S, H, D), dtype=torch.uint8, device="cuda", generator=gen)
        scales = rnd(2, L, S // P, H).abs()
        pools.append((kv.KVPool(codes, P, scales=scales), kv.KVPool(scales.view(2, L, S // P, H, 1), 1)))
    pages = [torch.randperm(S // P, device="cuda", generator=gen)[:12].to(torch.int32) for _ in range(2)]
    length = torch.zeros(1, dtype=torch.int32, device="cuda")
    places = [(0, 131)] + [(131 + i, 1) for i in range(20)]
    dense = [[], []]
    for cached, new in places:
        length.fill_(cached + new)
        batch = kv.Batch(pages[0][None], length, torch.tensor([0, new], dtype=torch.int32, device="cuda"), max_query=new)
        for layer in range(L):
            q, k, v = rnd(new, Hq, D).bfloat16(), rnd(new, H, D).bfloat16(), rnd(new, H, D).bfloat16()
            q = pools[0][0].append(layer, batch, k, v, q=q, inv_freq=inv)
            out = pools[0][0].attend(layer, batch, q)
            ang = torch.arange(cached, cached + new, device="cuda").double()[:, None, None] * inv.double()
            a, b = k.double().chunk(2, -1)
            dense[layer].append((torch.cat((a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()), -1), v.double()))
            kk, vv = (torch.cat([x[i] for x in dense[layer]]).repeat_interleave(Hq // H, 1) for i in (0, 1))
            dot = torch.matmul(q.double().transpose(0, 1), kk.permute(1, 2, 0).contiguous()) / math.sqrt(D)
            hidden = torch.arange(cached + new, device="cuda") > torch.arange(cached, cached + new, device="cuda")[:, None]
            want = torch.matmul(torch.softmax(dot.masked_fill(hidden, -math.inf), -1), vv.transpose(0, 1).contiguous()).transpose(0, 1)
            # 8 bits move each key and value by up to 2^-4: the norm of the difference stays well under twice that of the result's
            assert float((out.double() - want).norm() / want.norm()) < 2.0 ** -3
    T = int(length)
    with kv.HostBuffer(L * 2 * 192 * H * D) as chunk, kv.HostBuffer(L * 2 * 12 * H * 4) as scale_chunk:
        n = -(-T // P)
        pools[0][0].offload([(chunk.ptr, 192, T, pages[0].data_ptr())])
        pools[0][1].offload([(scale_chunk.ptr, 12, n, pages[0].data_ptr())])
        pools[1][0].load([(chunk.ptr, 192, T, pages[1].data_ptr())])
        pools[1][1].load([(scale_chunk.ptr, 12, n, pages[1].data_ptr())])
        torch.cuda.synchronize()
    length.fill_(T + 1)
    for layer in range(L):
        q, k, v = rnd(1, Hq, D).bfloat16(), rnd(1, H, D).bfloat16(), rnd(1, H, D).bfloat16()
        outs = []
        for (pool, _), p in zip(pools, pages):
            batch = kv.Batch(p[None], length)
            outs.append(pool.attend(layer, batch, pool.append(layer, batch, k, v, q=q, inv_freq=inv)))
        assert torch.equal(*outs)
    for pool, sp in pools:
        pool.check()
        pool.close()
        sp.close()


def test_strided_in_place_and_on_another_stream(kv):
    """Slices of one fused projection, queries rotated in place, everything on a stream of its own."""
    import torch
    c = filled(16, torch.float16, 6, 3, 64, 16, [(100, 30), (0, 2)], seed=21)
    g, pool, batch = on_gpu(kv, c)
    twin = kv.KVPool(g["pool"].clone(), 16)
    N, D = 32, 64
    fused = torch.randn(N + 1, 12 * D, device="cuda").half()
    inv = (10000.0 ** (-torch.arange(0, D, 2) / D)).float().cuda()
    split = lambda f: [x.view(-1, x.shape[1] // D, D) for x in f[:N].split((6 * D, 3 * D, 3 * D), 1)]  # noqa: E731
    q, k, v = (x.contiguous() for x in split(fused))
    want_q = twin.append(0, batch, k, v, q=q, inv_freq=inv)
    want = twin.attend(0, batch, want_q)
    q2, k2, v2 = split(fused)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    wide = torch.full((N, 8, D), 3.0, device="cuda", dtype=torch.float16)
    got_q = pool.append(0, batch, k2, v2, q=q2, q_out=q2, inv_freq=inv, stream=side)
    assert got_q is q2
    pool.attend(0, batch, q2, out=wide[:, 1:7], stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(q2, want_q) and torch.equal(wide[:, 1:7], want)
    assert bool((wide[:, 0] == 3).all()) and bool((wide[:, 7] == 3).all())
    assert torch.equal(g["pool"].view(torch.int16), twin.tensor.view(torch.int16))
    pool.close()
    twin.close()


def test_offsets_past_32_bits(kv):
    """A layer of more than 4 GiB: its last pages take and give tokens."""
    import torch
    H, D, P, S = 32, 128, 16, 600_000
    pool_t = torch.zeros(2, 1, S, H, D, dtype=torch.bfloat16, device="cuda")
    pool = kv.KVPool(pool_t, P)
    table = torch.tensor([[S // P - 1, 7, S // P - 2]], dtype=torch.int32, device="cuda")
    batch = kv.Batch(table, torch.tensor([40], dtype=torch.int32, device="cuda"),
                     torch.tensor([0, 40], dtype=torch.int32, device="cuda"))
    q, k, v = (torch.randn(40, H, D, device="cuda").bfloat16() for _ in range(3))
    pool.append(0, batch, k, v)
    assert torch.equal(pool_t[:, 0, S - P:], torch.stack((k, v))[:, :P])
    assert torch.equal(pool_t[:, 0, S - 2 * P:S - P][:, :8], torch.stack((k, v))[:, 2 * P:])
    assert torch.count_nonzero(pool_t[:, 0].amax(dim=(2, 3))) <= 2 * 40
    out = pool.attend(0, batch, q)
    p = torch.softmax((torch.matmul(q.float().transpose(0, 1), k.float().permute(1, 2, 0).contiguous()) / math.sqrt(D)).masked_fill(
        torch.ones(40, 40, device="cuda", dtype=torch.bool).triu(1), -math.inf), -1)
    want = torch.matmul(p, v.float().transpose(0, 1).contiguous()).transpose(0, 1)
    assert float((out.float() - want).abs().max()) < 2.0 ** -8 * 2 * float(v.abs().max()) + 1e-4
    pool.close()


def test_python_refusals(kv):
    import torch
    c = filled(8, torch.bfloat16, 4, 2, 64, 16, [(20, 2)], seed=1)
    g, pool, batch = on_gpu(kv, c)
    bare = kv.KVPool(g["pool"], 16)
    k = torch.zeros(2, 2, 64, device="cuda", dtype=torch.bfloat16)
    bad = [lambda: pool.append(0, batch, k.float(), k), lambda: pool.append(0, batch, k, k[:1]), lambda: pool.append(1, batch, k, k),
           lambda: pool.append(0, batch, k[:, :1], k), lambda: pool.append(0, batch, k.transpose(0, 1), k), lambda: bare.append(0, batch, k, k),
           lambda: pool.append(0, batch, k, k, q_out=g["q"]), lambda: pool.attend(0, batch, g["q"].cpu()),
           lambda: pool.attend(0, batch, g["q"][:, :3]), lambda: pool.attend(0, batch, g["q"], out=g["q"]),
           lambda: pool.attend(0, batch, g["q"], scale=0.0), lambda: pool.attend(0, batch, g["q"], window=-1),
           lambda: kv.Batch(g["table"].long(), g["ctx"]), lambda: kv.Batch(g["table"], g["ctx"][:0]),
           lambda: kv.Batch(g["table"].cpu(), g["ctx"]), lambda: kv.Batch(g["table"], g["ctx"], g["starts"][:1]),
           lambda: pool.append(0, batch, k, k, inv_freq=torch.ones(4, device="cuda"))]
    for i, f in enumerate(bad):
        with pytest.raises(kv.KvioError) as e:
            f()
        assert e.value.status in (kv.KVIO_EINVAL, kv.KVIO_EALIGN), i
    assert pool.attend(0, batch, g["q"][:0]).shape == (0, 4, 64)
    pool.close()
    bare.close()
