"""The operators that work on the cache in the pool's pages, as a serving program calls them:

  append  new tokens' keys and values into the pages of their sequences, keys and queries rotated by
          their positions on the way; the cache in 16 bits, or in e4m3 with a scale for each page and head
  attend  causal attention of new tokens over the pages of their sequences: single tokens, a few drafted
          ones, the rest of a partly cached prompt, whole prompts; with or without a sliding window

A case names the operator, the heads, the cache, how many sequences have how many cached and new tokens
(several: ragged, their mean), and the window (0: none).  Lengths follow from "lengths" alone.
"""
import math
import random

import torch

own = False

LAYERS, LAYER = 2, 1                 # a pool of two layers, the second one used
LARGEST = 448.0                      # of e4m3
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
FIELDS = ("op", "dtype", "bits", "Hq", "H", "D", "P", "seqs", "cached", "new", "window", "lengths")


def _case(op, dtype, bits, Hq, H, D, P, seqs, cached, new, window=0, lengths=0, name=None):
    c = dict(zip(FIELDS, (op, dtype, bits, Hq, H, D, P, seqs, cached, new, window, lengths)))
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # One token of one sequence on the smallest pool: what a step costs at least.
        _case("append", "fp16", 16, 8, 4, 64, 16, 1, 1000, 1, name="append_one"),
        # A decoding step of a full batch on an 8-bit cache: pages partly filled, some of whose scales grow.
        _case("append", "bf16", 8, 32, 8, 128, 16, 128, 4096, 1, lengths=1, name="append_step_8bit"),
        # The new parts of five prompts, into single-token pages.
        _case("append", "bf16", 16, 28, 4, 128, 1, 5, 1000, 1600, lengths=2, name="append_prompts"),
        # Eight long prompts into an 8-bit cache.
        _case("append", "bf16", 8, 64, 8, 128, 64, 8, 100, 2048, lengths=3, name="append_prompts_8bit"),
        # The next token of one short context on the smallest pool.
        _case("attend", "fp16", 16, 8, 4, 64, 16, 1, 1000, 1, name="decode_one"),
        # The next token of one long context: work has to be split along it.
        _case("attend", "bf16", 8, 32, 8, 128, 16, 1, 131071, 1, name="decode_long_8bit"),
        # A decoding step of a batch of ragged contexts.
        _case("attend", "bf16", 8, 32, 8, 128, 16, 64, 8000, 1, lengths=4, name="decode_batch_8bit"),
        # The same on a 16-bit cache whose tokens lie scattered, seven query heads to a KV head.
        _case("attend", "bf16", 16, 28, 4, 128, 1, 16, 16000, 1, lengths=5, name="decode_scattered"),
        # Drafted tokens of a batch, checked in one step.
        _case("attend", "bf16", 8, 64, 8, 128, 32, 32, 4096, 5, lengths=6, name="verify_8bit"),
        # Questions about documents whose cache was loaded: the case that loading caches is for.
        _case("attend", "bf16", 8, 32, 8, 128, 64, 4, 16384, 512, lengths=7, name="extend_8bit"),
        # A whole prompt with nothing cached.
        _case("attend", "bf16", 16, 32, 8, 128, 16, 1, 0, 8192, name="prefill"),
        # Ragged prompts, wide heads, a sliding window.
        _case("attend", "fp16", 16, 16, 4, 256, 16, 3, 200, 2500, window=1024, lengths=8, name="prefill_window"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more of these: one to 256 sequences, nothing to 128K tokens cached, one to 8192 new ones, 1 to 16 query
    heads to a KV head, heads of 64 to 256 dims, pages of 1 to 256 tokens, caches of both widths."""
    op, dtype, bits = rng.choice(("append", "attend", "attend")), rng.choice(("bf16", "bf16", "fp16")), rng.choice((8, 16))
    H, G, D = rng.choice((1, 2, 4, 5, 8, 8, 16)), rng.choice((1, 2, 3, 4, 4, 7, 8, 16)), rng.choice((64, 128, 128, 256))
    P, Hq = rng.choice((1, 1, 5, 16, 16, 24, 32, 64, 256)), H * G
    if op == "append":
        total = _log_uniform(rng, 1, min(16384, (64 * 128 * 16384) // (Hq * D)))
        seqs = min(total, _log_uniform(rng, 1, 256))
        cached, window = _log_uniform(rng, 1, 4096) - 1, 0
        new = max(1, total // seqs)
    else:
        kind = rng.choice(("step", "step", "draft", "rest", "prompt"))
        window = rng.choice((0, 0, 0, _log_uniform(rng, 16, 4096)))
        if kind in ("step", "draft"):
            most = (600 << 20) // (2 * H * D * bits // 8)          # tokens of all contexts
            seqs = _log_uniform(rng, 1, 128)
            cached = _log_uniform(rng, 1, max(2, min(131072, most // seqs)))
            new = 1 if kind == "step" else rng.randint(2, 8)
        else:
            pairs = (8192 * 8192 * 32 // 4 * 128) // (Hq * D)        # query tokens times keys, of all sequences, padded
            seqs = rng.randint(1, 6)
            new = _log_uniform(rng, 16, 512) if kind == "rest" else _log_uniform(rng, 128, 4096)
            new = max(1, min(new, int((pairs / (2.5 * seqs)) ** 0.5)))
            cached = min(_log_uniform(rng, 256, 32768), max(0, pairs // (3 * seqs * new) - new)) if kind == "rest" else 0
    return _case(op, dtype, bits, Hq, H, D, P, seqs, cached, new, window, rng.randrange(1 << 20))


def _lengths(case):
    """(cached, new) tokens of each sequence: the case's own for one, about its mean for several (single new tokens
    stay single)."""
    if case["seqs"] == 1:
        return [(case["cached"], case["new"])]
    rng = random.Random(case["lengths"])
    out = []
    for _ in range(case["seqs"]):
        new = case["new"]
        if case["op"] == "append" or new > 16:
            new = max(1, int(new * rng.uniform(0.5, 1.5)))
        out.append((int(case["cached"] * rng.uniform(0.25, 1.75)), new))
    return out


def work(case):
    """Each new row read once and written once, every cached row that some query sees read once, with its scales and
    its page; two products of D for each query head and key that it sees."""
    Hq, H, D, P, elem, w = case["Hq"], case["H"], case["D"], case["P"], case["bits"] // 8, case["window"]
    nbytes, flops = 0, 0
    for cached, new in _lengths(case):
        ctx = cached + new
        if case["op"] == "append":
            rows, first = new, cached // P
            nbytes += new * D * (2 * 2 * Hq + 2 * H * (2 + elem))
            flops += new * D * 3 * (Hq + H)
        else:
            rows = min(ctx, new - 1 + w) if w else ctx
            first = (ctx - rows) // P
            nbytes += new * D * 2 * 2 * Hq + rows * D * 2 * H * elem
            n = min(w, ctx) if w else ctx                        # keys the last query sees
            full = min(new, ctx - n + 1) if w else 1             # queries that see as many
            pairs = full * n + sum(range(n - (new - full), n))
            flops += 4 * D * Hq * pairs
        pages = (ctx - 1) // P - first + 1
        nbytes += pages * (4 + (2 * H * 4 if elem == 1 else 0))
    return {"bytes": nbytes, "flops": flops}


class _State:
    pass


def prepare(case, seed):
    Hq, H, D, P, dtype = case["Hq"], case["H"], case["D"], case["P"], TYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    s = _State()
    s.op, s.H, s.Hq, s.D, s.P, s.dtype, s.window = case["op"], H, Hq, D, P, dtype, case["window"]
    lens = _lengths(case)
    s.max_new, s.max_ctx = max(n for _, n in lens), max(c + n for c, n in lens)
    s.lens = lens
    B, N = len(lens), sum(n for _, n in lens)
    # a pool that also holds other contexts, pages in no order
    counts = [-(-(c + n) // P) for c, n in lens]
    pages = sum(counts) + sum(counts) // 4 + 3
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    s.table = torch.full((B, max(counts)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(counts):
        s.table[b, :n] = order[at:at + n]
        at += n
    s.ctx_len = torch.tensor([c + n for c, n in lens], dtype=torch.int32, device="cuda")
    s.q_start = torch.tensor([sum(n for _, n in lens[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda")
    # keys have a few strong channels, as models' do
    strong = 1.0 + 3.0 * (torch.rand(D, device="cuda", generator=gen) < 0.05)
    S = pages * P
    s.pool = torch.empty(2, LAYERS, S, H, D, dtype=torch.float8_e4m3fn if case["bits"] == 8 else dtype, device="cuda")
    s.scales = None
    if case["bits"] == 8:
        s.scales = torch.empty(2, LAYERS, pages, H, device="cuda")
        for i in range(2):                                       # the codes of a page and head reach 224 to 448
            for j in range(LAYERS):
                codes = (randn(S, H, D) * (strong if i == 0 else 1) * 80.0).clamp_(-LARGEST, LARGEST)
                s.pool[i, j] = codes.to(torch.float8_e4m3fn)
                s.scales[i, j] = 2.0 ** torch.randint(-8, -5, (pages, H), device="cuda", generator=gen)
        if s.op == "attend":                                     # a cache that came from elsewhere
            s.scales *= 0.75 + 0.5 * torch.rand(s.scales.shape, device="cuda", generator=gen)
    else:
        for i in range(2):
            for j in range(LAYERS):
                s.pool[i, j] = randn(S, H, D) * (strong if i == 0 else 1)
    if s.op == "append":
        fused = randn(N, (Hq + 2 * H) * D).to(dtype)              # what one projection gives
        s.q, s.k, s.v = (x.view(N, -1, D) for x in fused.split((Hq * D, H * D, H * D), dim=1))
        s.inv_freq = (500000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)).float()
        s.q_out = torch.empty(N, Hq, D, dtype=dtype, device="cuda")
    else:
        s.q = (randn(N, Hq, D) * 1.5).to(dtype)
        s.out = torch.empty(N, Hq, D, dtype=dtype, device="cuda")
    if own:
        import paper_2508_18572_amd as kv
        s.handle = kv.KVPool(s.pool, P, scales=s.scales)
        s.batch = kv.Batch(s.table, s.ctx_len, s.q_start if N > B else None, max_query=s.max_new)
    return s


def _rows(s):
    """Of each new token its sequence and its place in the context."""
    n = torch.arange(s.q.shape[0], device="cuda")
    seq = torch.searchsorted(s.q_start[1:].contiguous(), n.to(torch.int32), right=True)
    return seq, s.ctx_len[seq].long() - s.q_start[seq + 1] + n


def _rotate(x, cos, sin):
    """Pairs (i, i + D / 2) of each head turned by their angles, in 32 bits."""
    a, b = x.float().chunk(2, dim=-1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)


def _append_plain(s):
    seq, place = _rows(s)
    angle = (place.double()[:, None] * s.inv_freq.double()).unsqueeze(1)
    cos, sin = angle.cos().float(), angle.sin().float()
    s.q_out.copy_(_rotate(s.q, cos, sin))
    k, page = _rotate(s.k, cos, sin), s.table[seq, place // s.P].long()
    slot = page * s.P + place % s.P
    if s.scales is None:
        s.pool[0, LAYER, slot], s.pool[1, LAYER, slot] = k.to(s.dtype), s.v
        return
    # Keys and values pass through the model's type.  A page's scale is the smallest power of two that holds its rows,
    # and only grows while the page fills; rows that are there are rounded again where it does.
    num_pages = s.scales.shape[2]                                # of each page, how many rows it had: P where none is new
    had = torch.full((num_pages,), s.P, device="cuda").scatter_reduce_(0, page, place % s.P, "amin")
    touched, begun = had < s.P, had == 0
    before = torch.arange(s.P, device="cuda") < had[:, None]
    for i, x in enumerate((k.to(s.dtype).float(), s.v.float())):
        cache, scales = s.pool[i, LAYER].view(num_pages, s.P, s.H, s.D), s.scales[i, LAYER]
        top = torch.zeros(num_pages, s.H, device="cuda").index_reduce_(0, page, x.abs().amax(dim=-1), "amax")
        part, power = torch.frexp(top / LARGEST)                  # the quotient is part * 2 ** power, part in [1/2, 1)
        need = torch.exp2(torch.where(top > 0, power - (part == 0.5).int(), -100).clamp(-100).float())
        new = torch.where(begun[:, None], need, torch.maximum(scales, need))
        new = torch.where(touched[:, None], new, scales)
        at, head = (touched[:, None] & ~begun[:, None] & (new > scales)).nonzero().unbind(1)
        old = cache.view(torch.uint8)[at, :, head]
        again = (old.view(torch.float8_e4m3fn).float() * (scales / new)[at, head][:, None, None]).to(torch.float8_e4m3fn)
        cache.view(torch.uint8)[at, :, head] = torch.where(before[at][:, :, None], again.view(torch.uint8), old)
        scales.copy_(new)
        codes = (x / new[page][:, :, None]).clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
        s.pool[i, LAYER].view(torch.uint8)[slot] = codes.view(torch.uint8)


def _gathered(s, i, slot):
    """Rows of K (i = 0) or V (1) at these slots, in 32 bits, heads before tokens."""
    x = s.pool[i, LAYER].view(torch.uint8 if s.scales is not None else s.dtype)[slot]
    if s.scales is not None:
        x = x.view(torch.float8_e4m3fn).float() * s.scales[i, LAYER][slot // s.P].unsqueeze(-1)
    return x.float().transpose(1, 2).contiguous()                # B, H, T, D


def _attend_plain(s):
    B, T, Q, G = len(s.lens), s.max_ctx, s.max_new, s.Hq // s.H
    t, i = torch.arange(T, device="cuda"), torch.arange(Q, device="cuda")
    there = t < s.ctx_len[:, None]                               # B, T
    slot = torch.where(there, s.table[:, t // s.P].long() * s.P + t % s.P, 0)
    new = (s.q_start[1:] - s.q_start[:-1])[:, None].long()
    row = torch.where(i < new, s.q_start[:-1, None] + i, 0)      # B, Q
    place = s.ctx_len[:, None] - new + i
    seen = there[:, None, :] & (t <= place[:, :, None])
    if s.window:
        seen &= t > place[:, :, None] - s.window
    q = s.q.float()[row].view(B, Q, s.H, G, s.D).permute(0, 2, 1, 3, 4).reshape(B, s.H, Q * G, s.D).contiguous()
    score = torch.matmul(q, _gathered(s, 0, slot).transpose(2, 3).contiguous()).mul_(s.D ** -0.5).view(B, s.H, Q, G, T)
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    score.sub_(score.amax(dim=-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = score.sum(dim=-1, keepdim=True)
    out = torch.matmul(score.view(B, s.H, Q * G, T), _gathered(s, 1, slot)).view(B, s.H, Q, G, s.D)
    out = torch.where(total > 0, out / total, 0).permute(0, 2, 1, 3, 4).reshape(B, Q, s.Hq, s.D)
    s.out[row[i < new]] = out[i < new].to(s.dtype)


def run(s):
    if s.op == "append":
        if own:
            s.handle.append(LAYER, s.batch, s.k, s.v, q=s.q, q_out=s.q_out, inv_freq=s.inv_freq)
        else:
            _append_plain(s)
        return {"pool": s.pool[:, LAYER], "q": s.q_out, **({} if s.scales is None else {"scales": s.scales[:, LAYER]})}
    if own:
        s.handle.attend(LAYER, s.batch, s.q, out=s.out, window=s.window)
    else:
        _attend_plain(s)
    return s.out


def _exact_append(s):
    pool, q_out, at = s.pool[:, LAYER].double(), torch.empty_like(s.q_out, dtype=torch.float64), 0
    half = s.D // 2
    scales = None if s.scales is None else s.scales[:, LAYER].double().clone()

    def turned(x, place):
        z = torch.complex(x[..., :half].double(), x[..., half:].double())
        z = z * torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), place.double()[:, None, None] * s.inv_freq.double())
        return torch.cat((z.real, z.imag), dim=-1)

    for b, (cached, new) in enumerate(s.lens):
        place = torch.arange(cached, cached + new, device="cuda")
        q_out[at:at + new] = turned(s.q[at:at + new], place)
        for i, x in enumerate((turned(s.k[at:at + new], place), s.v[at:at + new].double())):
            table = s.table[b].long()
            if scales is None:
                pool[i, table[place // s.P] * s.P + place % s.P] = x
                continue
            x = x.to(s.dtype).double()
            first, last = cached // s.P, (cached + new - 1) // s.P
            pages = table[first:last + 1]
            grid = torch.zeros((last + 1 - first) * s.P, s.H, s.D, dtype=torch.float64, device="cuda")
            off = cached - first * s.P
            grid[off:off + new] = x
            grid = grid.view(-1, s.P, s.H, s.D)
            top = grid.abs().amax(dim=(1, 3))
            sc = 2.0 ** torch.ceil(torch.log2(top / LARGEST)).clamp(min=-100)
            rows = pool[i].view(-1, s.P, s.H, s.D)
            if off:                                              # the first page is begun
                was = scales[i, pages[0]]
                sc[0] = torch.maximum(sc[0], was)
                rows[pages[0], :off] *= (was / sc[0])[:, None]
            scales[i, pages] = sc
            pool[i, table[place // s.P] * s.P + place % s.P] = (x.view(new, s.H, s.D) / sc[(place // s.P) - first][:, :, None]).clamp(-LARGEST, LARGEST)
        at += new
    return {"pool": pool, "q": q_out, **({} if scales is None else {"scales": scales})}


def exact(case, seed):
    s = prepare(case, seed)
    if s.op == "append":
        return _exact_append(s)
    out, at = torch.empty(s.q.shape, dtype=torch.float64, device="cuda"), 0
    for b, (cached, new) in enumerate(s.lens):
        ctx = cached + new
        t = torch.arange(ctx, device="cuda")
        slot = s.table[b].long()[t // s.P] * s.P + t % s.P
        if s.scales is None:
            k, v = s.pool[0, LAYER][slot].double(), s.pool[1, LAYER][slot].double()
        else:
            codes = s.pool.view(torch.uint8)[:, LAYER, slot].view(torch.float8_e4m3fn).double()
            k, v = (codes[i] * s.scales[i, LAYER].double()[slot // s.P][:, :, None] for i in range(2))
        for h in range(s.Hq):
            for a in range(0, new, 2048):                        # so many queries at a time
                n = min(2048, new - a)
                end = cached + a + n                             # keys behind the last of them are masked for all
                dot = s.q[at + a:at + a + n, h].double() @ k[:end, h * s.H // s.Hq].t().contiguous() / math.sqrt(s.D)
                back = torch.arange(end - n, end, device="cuda")[:, None] - t[:end]
                hidden = (back < 0) | (back >= s.window) if s.window else back < 0
                p = torch.softmax(dot.masked_fill(hidden, -math.inf), dim=-1)
                out[at + a:at + a + n, h] = p @ v[:end, h * s.H // s.Hq]
        at += new
    return out
