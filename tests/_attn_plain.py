"""Random batches on a paged cache, and what kvio_append and kvio_attend make of them, in 64 bits, token by token
and row by row.  Tolerances follow from the roundings that the operators' descriptions name."""
import math
import random

import torch

LARGEST = 448.0
STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step of each type, relative


def values(codes):
    """e4m3 codes (uint8 or float8) as float64."""
    return codes.view(torch.float8_e4m3fn).to(torch.float32).double()


def random_batch(seed, op, device="cpu", small=True):
    """A case: heads, a pool of one layer with garbage (NaN and infinities too) wherever no context has a token,
    sequences of no, one and several tokens, rows of no sequence, offsets and lengths that make no sense, pages
    outside the pool."""
    rng = random.Random(seed * 7919 + (op == "append"))
    gen = torch.Generator().manual_seed(seed)
    c = {"dtype": rng.choice((torch.bfloat16, torch.float16)), "H": rng.choice((1, 2, 3, 4)), "P": rng.choice((1, 2, 5, 16, 32, 64, 100))}
    G = rng.choice((1, 2, 3, 4, 7, 8, 16, 20)) if op == "attend" else rng.choice((1, 2, 3))
    c["D"] = rng.choice((64, 128, 256)) if op == "attend" else rng.choice((16, 48, 64, 80, 128, 256))
    c["Hq"], H, D, P, dt = G * c["H"], c["H"], c["D"], c["P"], c["dtype"]
    if (H * D) % 16:
        raise AssertionError
    e4m3 = bool(seed & 1)
    B = rng.choice((1, 2, 3, 7)) if rng.random() < 0.85 else 70
    single = rng.random() < 0.3
    cached = [rng.choice((0, 1, 3, rng.randint(0, 40), rng.randint(0, 200))) for _ in range(B)]
    new = [1 if single else rng.choice((0, 1, 2, 5, rng.randint(0, 80 if B < 8 else 3))) for _ in range(B)]
    ctx = [a + b for a, b in zip(cached, new)]
    N = sum(new) + rng.choice((0, 0, 3))
    starts = [sum(new[:b]) for b in range(B + 1)]
    max_pages = max(1, max(-(-t // P) for t in ctx) + rng.choice((0, 1)))
    if rng.random() < 0.15 and not single:                        # more new tokens than the context has
        ctx[0] = new[0] // 2
    pages = sum(-(-t // P) for t in ctx) + 2
    order = torch.randperm(pages, generator=gen)
    table, at = torch.full((B, max_pages), -5, dtype=torch.int32), 0
    for b, t in enumerate(ctx):
        n = -(-t // P)
        table[b, :n] = order[at:at + n].int()
        at += n
    c["bad"] = rng.random() < 0.15 and max(ctx) > P
    if c["bad"]:
        b = max(range(B), key=lambda i: ctx[i])
        j = rng.randrange(max(0, ctx[b] - new[b]) // P, -(-ctx[b] // P)) if op == "append" else rng.randrange(-(-ctx[b] // P))
        c["bad"] = op == "attend" or new[b] > 0
        table[b, j] = pages + 3 if c["bad"] else table[b, j]
    c["table"], c["ctx"] = table, torch.tensor(ctx, dtype=torch.int32)
    c["starts"] = None if single else torch.tensor(starts, dtype=torch.int32)
    if single:
        N = B + rng.choice((0, 2))
    N = max(N, 1)
    c["max_query"] = rng.choice((0, max(max(new), 1), max(max(new), 1) + 5))
    S = pages * P
    k = torch.randn(2, S, H, D, generator=gen) * 1.5
    if e4m3:
        c["pool"] = (k * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
        c["scales"] = 2.0 ** torch.randint(-9, -5, (2, pages, H), generator=gen).float()
        if op == "attend":
            c["scales"] *= 0.5 + torch.rand(2, pages, H, generator=gen)
    else:
        c["pool"], c["scales"] = k.to(dt), None
    c["window"] = rng.choice((0, 0, 1, 7, 64, 100000)) if op == "attend" else 0
    # garbage where no token lies
    used = torch.zeros(S, dtype=torch.bool)
    for b in range(B):
        for t in range(ctx[b]):
            if 0 <= table[b, t // P] < pages:
                used[int(table[b, t // P]) * P + t % P] = True
    raw = c["pool"].view(torch.uint8)
    raw[:, ~used] = 0x7f if e4m3 else 0xff
    c["k"], c["v"] = torch.randn(N, H, D, generator=gen).to(dt), (torch.randn(N, H, D, generator=gen) * 3).to(dt)
    c["q"] = (torch.randn(N, c["Hq"], D, generator=gen) * 2).to(dt)
    c["q_out"] = torch.full((N, c["Hq"], D), -2.5, dtype=dt)
    c["rot"] = rng.choice((0, 16, D // 32 * 16, D)) if D >= 32 else rng.choice((0, 16))
    c["interleaved"] = rng.random() < 0.4
    c["inv_freq"] = (10000.0 ** (-torch.arange(0, max(c["rot"], 2), 2).double() / max(c["rot"], 2))).float()
    c["positions"] = torch.randint(0, 1 << 20, (N,), generator=gen, dtype=torch.int32) if rng.random() < 0.3 else None
    return {n: x.to(device) if isinstance(x, torch.Tensor) else x for n, x in c.items()}


CASES = random_batch


def rows_of(c):
    """(sequence, first row, rows, place of the first row, context length) of every sequence."""
    N = c["q"].shape[0]
    most = c["max_query"] or N
    for b in range(len(c["ctx"])):
        r0, r1 = (b, b + 1) if c["starts"] is None else (int(c["starts"][b]), int(c["starts"][b + 1]))
        ctx = int(c["ctx"][b])
        yield b, r0, min(r1 - r0, 1 if c["starts"] is None else most), ctx - (r1 - r0), ctx


def page_at(c, b, t):
    page = int(c["table"][b, t // c["P"]])
    return page if 0 <= page < c["pool"].shape[1] // c["P"] else -1


def near(got, want, tol, what):
    got, want = got.double(), want.double()
    assert torch.equal(got.isnan(), want.isnan()), what
    ok = ~want.isnan()
    off = ~((got[ok] == want[ok]) | ((got[ok] - want[ok]).abs() <= tol[ok]))
    assert not bool(off.any()), (what, int(off.sum()), "values off, the first: got, wanted, tolerance",
                                 [float(x[ok][off][0]) for x in (got, want, tol)])


def rotate(c, x, row, place):
    x = x.double().clone()
    half = c["rot"] // 2
    if half:
        pos = place if c["positions"] is None else int(c["positions"][row])
        ang = pos * c["inv_freq"].double()
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if c["interleaved"] else (slice(0, half), slice(half, 2 * half))
        u, v = x[..., a].clone(), x[..., b].clone()
        x[..., a], x[..., b] = u * ang.cos() - v * ang.sin(), v * ang.cos() + u * ang.sin()
    return x


def append_plain(c, pool, scales, q_out):
    """Hold pool, scales and q_out, as the call left them, to what it is described to do from c's."""
    P, dt, before = c["P"], c["dtype"], c["pool"]
    eps = STEP[dt]
    # One rounding, and the rotation's in 32 bits: three roundings of a 32-bit product sum and an angle off by at most
    # 2^-24 turns (2 pi 2^-24 radians), relative to the pair's size, at most 2^-20 of it.
    exp_q, tol_q = c["q_out"].double().clone(), torch.zeros(c["q_out"].shape, dtype=torch.float64, device=q_out.device)
    is8 = scales is not None
    exp = values(before).clone() if is8 else before.double().clone()
    tol = torch.zeros_like(exp)
    exp_scales = c["scales"].double().clone() if is8 else None
    loose = None if not is8 else torch.zeros_like(exp_scales, dtype=torch.bool)
    slots = {}
    for b, r0, rows, first, ctx in rows_of(c):
        for i in range(rows):
            place, row = first + i, r0 + i
            if place < 0:
                continue
            exp_q[row] = rotate(c, c["q"][row], row, place)
            tol_q[row] = exp_q[row].abs() * eps + c["q"][row].double().abs().max() * 2.0 ** -20
            page = page_at(c, b, place)
            if page < 0:
                continue
            k = rotate(c, c["k"][row], row, place)
            new = torch.stack((k, c["v"][row].double()))
            slot = page * P + place % P
            if not is8:
                exp[:, slot] = new
                tol[0, slot] = k.abs() * eps + c["k"][row].double().abs().max() * 2.0 ** -20
            else:
                slots.setdefault((page, place // P, b), []).append((slot, new, place))
    if is8:
        for (page, j, b), got in slots.items():
            lead = got[0][2] - j * P                               # rows the page had
            for i in range(2):
                x = torch.stack([n[i] for _, n, _ in got])          # tokens, H, D
                if i == 0:
                    x = x.to(dt).double()                          # keys pass through the model's type
                top = torch.where(x.isfinite(), x.abs(), 0).amax(dim=(0, 2))
                need = torch.where(top > 0, 2.0 ** torch.ceil(torch.log2(top / LARGEST)), 0).clamp(min=2.0 ** -100)
                was = c["scales"][i, page].double()
                now = torch.maximum(was, need) if lead else need
                if lead:
                    now = torch.where(top <= LARGEST * was, was, need)
                exp_scales[i, page] = now
                if i == 0 and c["rot"]:                            # a key right at a scale's edge may fall on either side of it
                    edge = torch.log2(top / LARGEST)
                    loose[i, page] = (edge - edge.round()).abs() < 2 * eps
                if lead:
                    old = slice(page * P, page * P + lead)
                    grown = now != was
                    r = exp[i, old] * (was / now)[:, None]
                    exp[i, old] = torch.where(grown[:, None], r, exp[i, old])
                    tol[i, old] = torch.where(grown[:, None], (r.abs() * 2.0 ** -4).clamp(min=2.0 ** -10) * 1.0001, 0)
                for (slot, n, _), y in zip(got, x):
                    z = y / now[:, None]
                    exp[i, slot] = torch.where(z.isnan(), z, z.clamp(-LARGEST, LARGEST))
                    # half a step of e4m3, 2^-4 relative, 2^-10 below its normal range, and for keys half a step of the
                    # model's type more where their rounding to it fell to the other side
                    tol[i, slot] = (exp[i, slot].abs() * 2.0 ** -4).clamp(min=2.0 ** -10) * 1.0001 + (z.abs() * 2 * eps if i == 0 else 0)
        ok = (scales.double() == exp_scales) | loose
        assert bool(ok.all()), "scales"
        strict = ~loose.repeat_interleave(P, dim=1)
        near(values(pool)[strict], exp[strict], tol[strict], "pool")
    else:
        near(pool, exp, tol, "pool")
    near(q_out, exp_q, tol_q, "q_out")


def attend_plain(c, out, lse):
    """Hold out and lse to the attention of c."""
    P, dt, G, D = c["P"], c["dtype"], c["Hq"] // c["H"], c["D"]
    is8 = c["scales"] is not None
    pool = values(c["pool"]) if is8 else c["pool"].double()
    exp = c["q_out"].double().clone()
    exp_lse = torch.full(lse.shape, 7.0, dtype=torch.float64, device=lse.device)
    tol, tol_lse = torch.zeros_like(exp), torch.zeros_like(exp_lse)
    # A probability is off by half a step of its 16-bit type (bf16 beside an e4m3 cache) and by its score's error; a score's
    # sum of D products in 32 bits by at most D 2^-24 of the sum of their sizes, its exponent by the same; the result is
    # rounded once.
    p_eps = STEP[torch.bfloat16 if is8 else dt]
    # fp16 probabilities below 2^-14 of the largest keep steps of 2^-24
    p_abs = 0.0 if is8 or dt == torch.bfloat16 else 2.0 ** -25
    for b, r0, rows, first, ctx in rows_of(c):
        slots = [page_at(c, b, t) * P + t % P if page_at(c, b, t) >= 0 else -1 for t in range(ctx)]
        for i in range(rows):
            place = first + i
            seen = [t for t in range(max(0, place - c["window"] + 1) if c["window"] else 0, place + 1) if slots[t] >= 0]
            if not seen:
                exp[r0 + i], exp_lse[r0 + i] = 0, -math.inf
                continue
            at = torch.tensor([slots[t] for t in seen], device=out.device)
            k, v = pool[0, at], pool[1, at]
            if is8:
                k = k * c["scales"][0, at // P].double()[:, :, None]
                v = v * c["scales"][1, at // P].double()[:, :, None]
            k, v = k.repeat_interleave(G, dim=1), v.repeat_interleave(G, dim=1)
            q = c["q"][r0 + i].double()
            score = (k * q).sum(-1) / math.sqrt(D)                  # T, Hq
            size = ((k * q).abs().sum(-1) / math.sqrt(D)).amax(0)
            m = score.amax(0)
            p = (score - m).exp()
            total = p.sum(0)
            exp[r0 + i] = (p[:, :, None] * v).sum(0) / total[:, None]
            exp_lse[r0 + i] = m + total.log()
            off = size * (D + 8) * 2.0 ** -24 + m.abs() * 2.0 ** -22 + len(seen) * 2.0 ** -23 + 2.0 ** -20
            reach = (p[:, :, None] * v.abs()).sum(0) / total[:, None]
            tol[r0 + i] = exp[r0 + i].abs() * STEP[dt] + reach * (p_eps + 2 * off[:, None]) * 1.01 + p_abs * v.abs().sum(0) / total[:, None] + (2.0 ** -25 if dt == torch.float16 else 0)
            tol_lse[r0 + i] = 2 * off + exp_lse[r0 + i].abs() * 2.0 ** -22
    near(out, exp, tol, "out")
    near(lse, exp_lse, tol_lse, "lse")
