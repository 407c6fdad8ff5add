"""kvio_attend's blocks of rows built for the CPU (as in test_attn_emulated.py): contexts that several workgroups
share, odd groups of query heads, windows, values that are not finite in hidden tokens; and what is refused there."""
import ctypes
import math

import pytest
import torch

import test_emulated_kernels as base
from _attn_plain import attend_plain
from test_attn_emulated import TYPE, Box, batch_args, emu, make_pool  # noqa: F401  (a fixture)

pytestmark = pytest.mark.skipif(not base.os.path.exists(base.CXX), reason="no clang++ (the sources use its vector types)")


def case(dtype, bits, H, G, D, P, lens, window=0, seed=0):
    gen = torch.Generator().manual_seed(seed)
    counts = [-(-(a + b) // P) for a, b in lens]
    pages = sum(counts) + 2
    order, at = torch.randperm(pages, generator=gen).int(), 0
    table = torch.full((len(lens), max(counts) + 1), -7, dtype=torch.int32)
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    N = sum(n for _, n in lens)
    x = torch.randn(2, pages * P, H, D, generator=gen) * 1.5
    c = {"dtype": dtype, "H": H, "Hq": H * G, "D": D, "P": P, "window": window, "table": table, "max_query": 0,
         "ctx": torch.tensor([a + b for a, b in lens], dtype=torch.int32),
         "starts": torch.tensor([sum(n for _, n in lens[:b]) for b in range(len(lens) + 1)], dtype=torch.int32),
         "q": (torch.randn(N + 1, H * G, D, generator=gen) * 2).to(dtype), "q_out": torch.full((N + 1, H * G, D), -2.5, dtype=dtype),
         "scales": None, "pool": x.to(dtype)}
    if bits == 8:
        c["pool"] = (x * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
        c["scales"] = 0.01 * (0.5 + torch.rand(2, pages, H, generator=gen))
    return c


def attend(emu, c):  # noqa: F811
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
    attend_plain(c, out, lse)
    got = out.clone(), lse.clone()
    kv.kvio_pool_destroy(h)
    box.free()
    return got


@pytest.mark.parametrize("name,c", [
    ("shared by two", case(torch.bfloat16, 16, 1, 1, 64, 16, [(1500, 70)], seed=1)),
    ("shared, a window", case(torch.float16, 8, 1, 3, 64, 5, [(900, 30)], window=700, seed=2)),
    ("rows of one sequence in two blocks", case(torch.bfloat16, 8, 1, 7, 128, 1, [(40, 38)], seed=3)),
    ("a block of one row", case(torch.float16, 16, 1, 2, 64, 16, [(0, 129)], seed=4)),
    ("a window of one token", case(torch.bfloat16, 16, 2, 16, 64, 24, [(3, 5), (0, 17)], window=1, seed=5)),
    ("wide heads", case(torch.bfloat16, 8, 1, 4, 256, 16, [(70, 33)], seed=6)),
    ("a group as large as a block", case(torch.bfloat16, 16, 1, 256, 64, 16, [(20, 2)], seed=7)),
], ids=lambda x: x if isinstance(x, str) else "")
def test_blocks(emu, name, c):  # noqa: F811
    attend(emu, c)


@pytest.mark.parametrize("bits", [8, 16])
def test_more_new_tokens_than_the_context_has(emu, bits):  # noqa: F811
    """Rows whose place comes out below zero see nothing: zeros, and minus infinity."""
    c = case(torch.bfloat16, bits, 1, 4, 64, 16, [(10, 90), (2, 20)], seed=8)
    c["ctx"][0] = 30
    out, lse = attend(emu, c)
    assert bool((out[:60] == 0).all()) and bool((lse[:60] == -math.inf).all()) and bool((out[60:110] != 0).any())


@pytest.mark.parametrize("D,group,fits", [(64, 256, True), (64, 257, False), (128, 300, False), (256, 128, True), (256, 129, False)])
def test_more_query_heads_than_a_block_has_rows(emu, D, group, fits):  # noqa: F811
    kv, lib, A = emu
    box = Box(kv)
    ptr = box.put(torch.zeros(2, 16, 1, D, dtype=torch.bfloat16))[1]
    h = kv.kvio_pool_create(1, 1, D, 2, 16, 16, [ptr], [ptr + 16 * D * 2])
    a = A.kvio_attend_args(batch=A.kvio_batch(1, 1, 1, 0, 1), num_q_heads=group, softmax_scale=1.0)
    need = ctypes.c_size_t()
    got = lib.kvio_attend_workspace(h, ctypes.byref(a), ctypes.byref(need))
    assert got == (0 if fits else kv.KVIO_EINVAL)
    assert fits or "query heads to a KV head" in kv.kvio_last_error()
    kv.kvio_pool_destroy(h)
    box.free()


def test_more_tokens_than_a_launch_holds(emu):  # noqa: F811
    """2^26 rows of single tokens, whose partial results would be joined by 2^32 threads, are refused."""
    kv, lib, A = emu
    box = Box(kv)
    ptr = box.put(torch.zeros(2, 16, 1, 64, dtype=torch.bfloat16))[1]
    h = kv.kvio_pool_create(1, 1, 64, 2, 16, 16, [ptr], [ptr + 16 * 64 * 2])
    a = A.kvio_attend_args(batch=A.kvio_batch(1 << 24, 1 << 24, 1, 0, 1), num_q_heads=4, softmax_scale=1.0)
    need = ctypes.c_size_t()
    assert lib.kvio_attend_workspace(h, ctypes.byref(a), ctypes.byref(need)) == kv.KVIO_EINVAL and "too many" in kv.kvio_last_error()
    kv.kvio_pool_destroy(h)
    box.free()
