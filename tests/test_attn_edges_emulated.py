"""append and attend built for the CPU (as in test_attn_emulated.py) at the ends of what their arguments may hold: scales
that are no numbers, zero or infinite, windows as long as an int, slices of one buffer."""
import ctypes
import math

import pytest
import torch

import test_emulated_kernels as base
from _attn_plain import values
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


BEGUN = [(0.0, 0.0), (0.0, 1.5), (-0.0, 0.0), (2.0 ** -140, 0.0), (2.0 ** -128, 0.0), (2.0 ** -127, 2.0 ** -130), (2.0 ** -101, 0.0), (2.0 ** -100, 0.0),
         (2.0 ** -99, 2.0 ** -92), (0.75, 300.0), (0.75, 340.0), (-0.5, 100.0), (-0.5, 300.0), (2.0 ** 127, 1.0), (math.inf, 1.0), (math.inf, 0.0),
         (math.nan, 2.0), (math.nan, 0.0)]


@pytest.mark.parametrize("was,top", BEGUN)
@pytest.mark.parametrize("new", [1, 9])
def test_append_to_a_begun_page_of_any_scale(emu, new, was, top):  # noqa: F811
    """A page whose scale came from elsewhere keeps it where it is a number of at least 2^-100 in size whose 448-fold holds the new
    rows; else the rows that are there are rounded again under the new one."""
    kv, lib, A = emu
    H, D, P, had = 2, 64, 16, 5
    gen = torch.Generator().manual_seed(new)
    codes = torch.randint(0, 256, (2, P, H, D), generator=gen).to(torch.uint8)
    box = Box(kv)
    pool, h = make_pool(kv, box, {"H": H, "D": D, "P": P, "pool": codes.view(torch.float8_e4m3fn)})
    rows = torch.rand(2, new, H, D, generator=gen) * 2 - 1
    rows[:, -1, :, 7] = -1
    rows = (rows * top).bfloat16()
    a = A.kvio_append_args(batch=batch_args(A, box, None, torch.zeros(1, 1, dtype=torch.int32), torch.tensor([had + new], dtype=torch.int32),
                                            torch.tensor([0, new], dtype=torch.int32), new), dtype=0, cache_dtype=2)
    (_, a.k), (_, a.v) = box.put(rows[0]), box.put(rows[1])
    a.k_stride = a.v_stride = H * D
    scales, a.k_scale = box.put(torch.full((2, 1, H), was))
    a.v_scale, a.scale_stride = a.k_scale + 4 * H, H
    assert lib.kvio_append(h, 0, ctypes.byref(a), None) == 0, kv.kvio_last_error()
    top = float(rows.double().abs().max())
    need = 2.0 ** max(-100, math.ceil(math.log2(top / 448))) if top else 2.0 ** -100
    now = was if 2.0 ** -100 <= abs(was) < math.inf and top <= 448 * abs(was) else need
    assert bool((scales == now).all()), (scales, now)
    want = torch.cat((values(codes[:, :had]) * was, rows.double()), 1) / now
    want = torch.where(want.isnan(), want, want.clamp(-448, 448))
    got = values(pool)[:, :had + new]
    assert torch.equal(got.isnan(), want.isnan())
    # half a step of e4m3: 2^-4 relative, 2^-10 below its normal range; a quotient in 32 bits is off by 2^-23 of itself
    ok = (got - want).abs() <= want.abs().clamp(min=2.0 ** -6) * 2.0 ** -4 * (1 + 2.0 ** -19)
    assert bool((ok | want.isnan()).all())
    assert now != was or torch.equal(pool.view(torch.uint8)[:, :had], codes[:, :had])
    assert torch.equal(pool.view(torch.uint8)[:, had + new:], codes[:, had + new:])
    kv.kvio_pool_destroy(h)
    box.free()


LONGEST = 2 ** 31 - 1


@pytest.mark.parametrize("window", [LONGEST, LONGEST - 40, 91, 90])
@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("G", [1, 8])
def test_windows_longer_than_the_context(emu, G, bits, window):  # noqa: F811
    """More new tokens than the context has, 64 or fewer rows to a KV head and more: as without a window, bit for bit."""
    c = case(torch.bfloat16, bits, 1, G, 64, 16, [(0, 60), (30, 20), (0, 5)], seed=12)
    c["ctx"][0], c["ctx"][2] = 30, 1
    c["max_query"] = 60
    out, lse = attend(emu, c)
    assert bool((out[30:60] != 0).any(2).all()) and bool((out[84] != 0).any())
    c["window"] = window
    got, got_lse = attend(emu, c)
    assert torch.equal(got, out) and torch.equal(got_lse, lse)


def small_attend(kv, lib, A, width=4 * 64, rows=6):
    """One context of 40 tokens, 5 of them new, over a 16-bit pool; q and out in one buffer of `width` elements a row."""
    box, H, Hq, D, P, pages, N = Box(kv), 2, 4, 64, 16, 3, 5
    gen = torch.Generator().manual_seed(3)
    codes = torch.randn(2, pages * P, H, D, generator=gen).bfloat16()
    _, h = make_pool(kv, box, {"H": H, "D": D, "P": P, "pool": codes})
    a = A.kvio_attend_args(batch=batch_args(A, box, None, torch.tensor([[0, 1, 2]], dtype=torch.int32), torch.tensor([40], dtype=torch.int32),
                                            torch.tensor([0, N], dtype=torch.int32), N), num_q_heads=Hq, softmax_scale=0.125)
    fused, at = box.put(torch.randn(rows, width, generator=gen).bfloat16())
    a.q, a.out, a.q_stride, a.out_stride = at, at, width, width
    need = ctypes.c_size_t()
    assert lib.kvio_attend_workspace(h, ctypes.byref(a), ctypes.byref(need)) == 0
    a.workspace, a.workspace_bytes = box.put(torch.zeros(max(need.value, 16), dtype=torch.uint8))[1], need.value
    return a, h, box, fused


@pytest.mark.parametrize("scale,fits", [(2.3e38, True), (2.4e38, False), (3.4e38, False), (1e-45, True), (-1.0, False), (math.nan, False)])
def test_softmax_scales(emu, scale, fits):  # noqa: F811
    """Scores are kept in powers of two: the scale times log2(e) has to be finite too (it would make NaN of a score of 0)."""
    kv, lib, A = emu
    a, h, box, _ = small_attend(kv, lib, A, width=8 * 64)
    a.out = a.q + 2 * 4 * 64 * 6
    a.q_stride = a.out_stride = 4 * 64
    a.softmax_scale = scale
    assert lib.kvio_attend(h, 0, ctypes.byref(a), None) == (0 if fits else kv.KVIO_EINVAL), kv.kvio_last_error()
    assert fits or "softmax_scale" in kv.kvio_last_error()
    need = ctypes.c_size_t()
    assert lib.kvio_attend_workspace(h, ctypes.byref(a), ctypes.byref(need)) == (0 if fits else kv.KVIO_EINVAL)
    kv.kvio_pool_destroy(h)
    box.free()


@pytest.mark.parametrize("q_at,out_at,fits", [(0, 256, True), (256, 0, True), (0, 512, True), (512, 0, True), (128, 400, True), (0, 248, False), (256, 8, False),
                                              (0, 768 + 8, False), (0, 768 + 256, True), (768 + 512, 248, True), (520, 768, False), (512, 768, True), (0, 0, False)])
def test_slices_of_one_buffer(emu, q_at, out_at, fits):  # noqa: F811
    """q and out as slices of rows of 768 elements, 256 each: apart from each other in every row, or refused."""
    kv, lib, A = emu
    a, h, box, fused = small_attend(kv, lib, A, width=768, rows=7)
    clean = fused.clone()
    at = a.q
    a.q, a.out = at + 2 * q_at, at + 2 * out_at
    assert lib.kvio_attend(h, 0, ctypes.byref(a), None) == (0 if fits else kv.KVIO_EINVAL), kv.kvio_last_error()
    assert fits or "overlaps" in kv.kvio_last_error()
    got, flat = fused.view(-1)[out_at:][:4 * 768 + 256].clone(), clean.view(-1)
    for i in range(5):                               # the same from a buffer of its own; nothing else is written
        assert torch.equal(fused.view(-1)[q_at + i * 768:][:256], flat[q_at + i * 768:][:256])
    if fits:
        fused.copy_(clean)
        a.out, a.out_stride = box.put(torch.zeros(5, 256, dtype=torch.bfloat16))[1], 256
        own = torch.from_numpy(box.all[-1].array).view(torch.bfloat16).view(5, 256)
        assert lib.kvio_attend(h, 0, ctypes.byref(a), None) == 0
        for i in range(5):
            assert torch.equal(got[i * 768:][:256], own[i])
    # of append, the same check
    b = A.kvio_append_args(batch=a.batch, num_q_heads=4, q=at + 2 * q_at, q_out=at + 2 * out_at, q_stride=768, q_out_stride=768, k_stride=128, v_stride=128)
    b.k, b.v = (box.put(torch.zeros(5, 2, 64, dtype=torch.bfloat16))[1] for _ in range(2))
    assert lib.kvio_append(h, 0, ctypes.byref(b), None) == (0 if fits or q_at == out_at else kv.KVIO_EINVAL), kv.kvio_last_error()
    b.q_out, b.q_out_stride = b.q + 2 * 256, 776                  # strides that differ: by the whole ranges
    assert lib.kvio_append(h, 0, ctypes.byref(b), None) == kv.KVIO_EINVAL
    kv.kvio_pool_destroy(h)
    box.free()


@pytest.mark.parametrize("starts", [[0, 5, 3, 8], [0, 90, 1, 2], [6, 2, 90, 40], [90, 90, 0, 90], [-5, 200, -7, 3], [2 ** 31 - 1, -2 ** 31, 0, 90]])
@pytest.mark.parametrize("bits", [8, 16])
def test_falling_offsets_touch_nothing_else(emu, bits, starts):  # noqa: F811
    """Which rows such a call works on is not defined; rows, slots and scales of no sequence stay, every access is in bounds (the
    buffers lie against inaccessible pages), and the call ends."""
    kv, lib, A = emu
    N, P, H, D = 92, 16, 2, 64
    for max_query in (0, 12):
        c = case(torch.bfloat16, bits, H, 2, D, P, [(10, 80), (0, 95), (30, 60)], seed=5)
        c["q"], c["q_out"] = c["q"][:N].contiguous(), c["q_out"][:N].contiguous()
        c["max_query"] = max_query
        box = Box(kv)
        pool, h = make_pool(kv, box, c)
        batch = batch_args(A, box, c, c["table"], c["ctx"], torch.tensor(starts, dtype=torch.int32), N, max_query)
        a = A.kvio_attend_args(batch=batch, dtype=0, cache_dtype=2 if bits == 8 else 0, num_q_heads=4, softmax_scale=0.125, q_stride=256, out_stride=256)
        b = A.kvio_append_args(batch=batch, dtype=0, cache_dtype=2 if bits == 8 else 0, num_q_heads=4, k_stride=128, v_stride=128, q_stride=256, q_out_stride=256)
        a.q = b.q = box.put(c["q"])[1]
        out, a.out = box.put(c["q_out"])
        q_out, b.q_out = box.put(c["q_out"])
        b.k, b.v = (box.put(torch.randn(N, H, D).bfloat16())[1] for _ in range(2))
        if bits == 8:
            scales, a.k_scale = box.put(c["scales"])
            a.v_scale, a.scale_stride = a.k_scale + 4 * c["scales"][0].numel(), c["scales"].shape[2]
            b.k_scale, b.v_scale, b.scale_stride = a.k_scale, a.v_scale, a.scale_stride
        need = ctypes.c_size_t()
        assert lib.kvio_attend_workspace(h, ctypes.byref(a), ctypes.byref(need)) == 0
        a.workspace, a.workspace_bytes = box.put(torch.zeros(max(need.value, 16), dtype=torch.uint8))[1], need.value
        assert lib.kvio_attend(h, 0, ctypes.byref(a), None) == 0, kv.kvio_last_error()
        assert lib.kvio_append(h, 0, ctypes.byref(b), None) == 0, kv.kvio_last_error()
        cut = [min(max(s, 0), N) for s in starts]
        named = torch.zeros(N, dtype=torch.bool)
        for i in range(3):
            named[cut[i]:cut[i + 1]] = True
        assert bool((out[~named] == -2.5).all()) and bool((q_out[~named] == -2.5).all())
        pages = torch.zeros(c["pool"].shape[1] // P, dtype=torch.bool)
        pages[c["table"][c["table"] >= 0].long()] = True
        same = pool.view(torch.uint8).view(2, -1, P * H * D * pool.element_size()) == c["pool"].view(torch.uint8).view(2, -1, P * H * D * pool.element_size())
        assert bool(same[:, ~pages].all())
        kv.kvio_pool_destroy(h)
        box.free()


@pytest.mark.parametrize("rot", [0, 16])
def test_append_to_a_page_of_a_billion_tokens(emu, rot):  # noqa: F811
    """Places past 2^30 in one page: steps through it stay below 2^31 (a layer of 17.6 GB, of which little is touched)."""
    kv, lib, A = emu
    P, D, ctx, new = 1_100_000_000, 16, 1_099_999_990, 3
    box = Box(kv)
    layers = [base.Memory(kv, P * D, 1, 1) for _ in range(2)]
    h = kv.kvio_pool_create(1, 1, D, 1, P, P, [layers[0].ptr], [layers[1].ptr])
    x = torch.arange(2 * new * D).view(2, new, 1, D).bfloat16() - 40
    a = A.kvio_append_args(batch=batch_args(A, box, None, torch.zeros(1, 1, dtype=torch.int32), torch.tensor([ctx], dtype=torch.int32),
                                            torch.tensor([0, new], dtype=torch.int32), new), dtype=0, cache_dtype=2, rot_dim=rot)
    (_, a.k), (_, a.v) = box.put(x[0]), box.put(x[1])
    a.k_stride = a.v_stride = D
    if rot:
        a.inv_freq = box.put(torch.zeros(rot // 2))[1]
    scales, a.k_scale = box.put(torch.ones(2, 1, 1))
    a.v_scale, a.scale_stride = a.k_scale + 4, 1
    assert lib.kvio_append(h, 0, ctypes.byref(a), None) == 0, kv.kvio_last_error()
    assert bool((scales == 1).all())
    for i in range(2):
        got = torch.from_numpy(layers[i].array[(ctx - new - 1) * D:(ctx + 1) * D].copy()).view(torch.float8_e4m3fn).double().view(new + 2, D)
        assert bool((got[0] == 0).all()) and bool((got[-1] == 0).all())
        want = x[i, :, 0].double()
        assert bool(((got[1:-1] - want).abs() <= want.abs() * 2.0 ** -4).all())
    kv.kvio_check(h)
    kv.kvio_pool_destroy(h)
    for m in layers:
        m.free()
    box.free()
