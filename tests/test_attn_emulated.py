"""kvio_append and kvio_attend, their kernels included, built for the CPU (tests/c/emu, tests/c/emu_attn: every
buffer lies against an inaccessible page, lanes and waves have to meet where the kernels say they do): against
plain 64-bit computations, over cache types, head counts, page sizes, ragged, empty and senseless batches, and
what the calls refuse."""
import ctypes
import math
import os
import shutil

import numpy as np
import pytest
import torch

import test_emulated_kernels as base
from _attn_plain import append_plain, attend_plain, random_batch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(base.CXX), reason="no clang++ (the sources use its vector types)")


@pytest.fixture(scope="module")
def emu(tmp_path_factory):
    """(binding of the emulated kvio.h, library with the structs of kvio_attn.h, the structs' module)"""
    import paper_2508_18572_amd.attn as A
    out = str(tmp_path_factory.mktemp("attn"))
    for where in (os.path.join(ROOT, "tests", "c", "emu_attn"), os.path.join(ROOT, "paper_2508_18572_amd", "csrc_attn")):
        for f in os.listdir(where):
            if not os.path.exists(os.path.join(out, f)):          # the emulation's kvio_lane.h comes first
                shutil.copy(os.path.join(where, f), out)
    base.build(out, extra=("-mf16c",))
    kv = base.load(out)
    for name in ("kvio_append", "kvio_attend", "kvio_attend_workspace"):
        getattr(kv._lib, name).argtypes = getattr(A._lib, name).argtypes
        getattr(kv._lib, name).restype = ctypes.c_int
    return kv, kv._lib, A


class Box:
    """Buffers of one case in guarded memory, seen as torch tensors."""

    def __init__(self, kv):
        self.kv, self.all = kv, []

    def put(self, t, skip=0):
        n = max(t.numel() * t.element_size(), 1)
        m = base.Memory(self.kv, n, 1, 1, skip)
        self.all.append(m)
        if t.numel():
            m.array[:] = t.contiguous().view(-1).view(torch.uint8).numpy()
        out = torch.from_numpy(m.array)[:t.numel() * t.element_size()].view(t.dtype).view(t.shape)
        return out, m.ptr

    def free(self):
        for m in self.all:
            m.free()


def make_pool(kv, box, c):
    pool, ptr = box.put(c["pool"])
    H, D, S = c["H"], c["D"], c["pool"].shape[1]
    e = c["pool"].element_size()
    h = kv.kvio_pool_create(1, H, D, e, c["P"], S, [ptr], [ptr + S * H * D * e])
    return pool, h


def batch_args(A, box, c, table, ctx, starts, N, max_query=0):
    t, tp = box.put(table)
    cl, cp = box.put(ctx)
    qp = box.put(starts)[1] if starts is not None else None
    return A.kvio_batch(len(ctx), N, table.shape[1], max_query, table.shape[1], tp, cp, qp)


TYPE = {torch.bfloat16: 0, torch.float16: 1}


@pytest.mark.parametrize("seed", range(48))
def test_append(emu, seed):
    kv, lib, A = emu
    c = random_batch(seed, "append")
    box = Box(kv)
    pool, h = make_pool(kv, box, c)
    N, Hq, H, D = c["k"].shape[0], c["Hq"], c["H"], c["D"]
    a = A.kvio_append_args(batch=batch_args(A, box, c, c["table"], c["ctx"], c["starts"], N, c["max_query"]),
                           dtype=TYPE[c["dtype"]], cache_dtype=TYPE[c["dtype"]] if c["scales"] is None else 2,
                           num_q_heads=Hq, rot_dim=c["rot"], flags=int(c["interleaved"]))
    (_, a.k), (_, a.v) = box.put(c["k"]), box.put(c["v"])
    q_out, a.q_out = box.put(c["q_out"])
    a.q = box.put(c["q"])[1]
    a.k_stride = a.v_stride = H * D
    a.q_stride = a.q_out_stride = Hq * D
    if c["rot"]:
        a.inv_freq = box.put(c["inv_freq"])[1]
    if c["positions"] is not None:
        a.positions = box.put(c["positions"])[1]
    scales = None
    if c["scales"] is not None:
        scales, a.k_scale = box.put(c["scales"])
        a.v_scale, a.scale_stride = a.k_scale + 4 * c["scales"][0].numel(), c["scales"].shape[2]
    assert lib.kvio_append(h, 0, ctypes.byref(a), None) == 0, kv.kvio_last_error()
    append_plain(c, pool, scales, q_out)
    if c["bad"]:
        with pytest.raises(kv.KvioError) as e:
            kv.kvio_check(h)
        assert e.value.status == kv.KVIO_ERANGE
    else:
        kv.kvio_check(h)
    kv.kvio_pool_destroy(h)
    box.free()


@pytest.mark.parametrize("seed", range(64))
def test_attend(emu, seed):
    kv, lib, A = emu
    c = random_batch(seed, "attend")
    box = Box(kv)
    _, h = make_pool(kv, box, c)
    N, Hq, D = c["q"].shape[0], c["Hq"], c["D"]
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
    kv.kvio_pool_destroy(h)
    box.free()


# What is refused: a field's value (or several), the status, and a word of the text.
BATCH = [
    ({"batch.num_seqs": -1}, "EINVAL", "negative"), ({"batch.num_tokens": -1}, "EINVAL", "negative"),
    ({"batch.max_query": -1}, "EINVAL", "negative"), ({"batch.max_pages": 0}, "EINVAL", "max_pages"),
    ({"batch.table_stride": 1}, "EINVAL", "table_stride"), ({"batch.max_pages": 1 << 30, "batch.table_stride": 1 << 30}, "EINVAL", "2^31"),
    ({"batch.page_table": None}, "EINVAL", "page_table is null"), ({"batch.page_table": +2}, "EALIGN", "page_table"),
    ({"batch.table_stride": 1000}, "EINVAL", "allocation"), ({"batch.ctx_len": None}, "EINVAL", "ctx_len is null"),
    ({"batch.q_start": None, "batch.num_tokens": 1}, "EINVAL", "without q_start"), ({"batch.num_tokens": 4000}, "EINVAL", "allocation"),
    ({"dtype": 2}, "EINVAL", "dtype"), ({"cache_dtype": 1}, "EINVAL", "cache_dtype"), ({"cache_dtype": 0}, "EINVAL", "bytes"),
    ({"k_scale": None}, "EINVAL", "k_scale is null"), ({"v_scale": +2}, "EALIGN", "v_scale"), ({"scale_stride": 1}, "EINVAL", "scale_stride"),
    ({"scale_stride": 100}, "EINVAL", "allocation"), ({"q": +8}, "EALIGN", "q is not 16"), ({"q_stride": 4 * 64 + 4}, "EINVAL", "multiple of 8"),
    ({"q_stride": 64}, "EINVAL", "at least"), ({"reserved": 1}, "EINVAL", "reserved"),
]
APPEND = BATCH + [
    ({"k": None}, "EINVAL", "k is null"), ({"v": +8}, "EALIGN", "v is not"), ({"k_stride": 120}, "EINVAL", "k: tokens"),
    ({"num_q_heads": 0}, "EINVAL", "num_q_heads"), ({"q": None}, "EINVAL", "num_q_heads"), ({"rot_dim": 24}, "EINVAL", "rot_dim"),
    ({"rot_dim": 128}, "EINVAL", "rot_dim"), ({"rot_dim": 64}, "EINVAL", "inv_freq is null"), ({"flags": 2}, "EINVAL", "flags"),
    ({"q_out": "q+16"}, "EINVAL", "overlaps"), ({"q_out_stride": 8 * 64}, "EINVAL", "allocation"),
]
ATTEND = BATCH + [
    ({"num_q_heads": 3}, "EINVAL", "query heads"), ({"num_q_heads": 0}, "EINVAL", "query heads"), ({"window": -1}, "EINVAL", "window"),
    ({"softmax_scale": 0.0}, "EINVAL", "softmax_scale"), ({"softmax_scale": float("nan")}, "EINVAL", "softmax_scale"),
    ({"softmax_scale": float("inf")}, "EINVAL", "softmax_scale"), ({"out": "q"}, "EINVAL", "overlaps"), ({"out": None}, "EINVAL", "out is null"),
    ({"workspace": None}, "EINVAL", "workspace is null"), ({"workspace_bytes": 100}, "EINVAL", "are needed"), ({"workspace": +8}, "EALIGN", "workspace"),
    ({"lse": +2}, "EALIGN", "lse"),
]


def refusal_case(kv, lib, A, op):
    """Two contexts of 40 and 30 tokens, 3 and 2 of them new, on an e4m3 pool: (arguments, handle, box)"""
    box, H, Hq, D, P, pages, N = Box(kv), 2, 4, 64, 16, 6, 5
    ptr = box.put(torch.zeros(2, pages * P, H, D, dtype=torch.uint8))[1]
    h = kv.kvio_pool_create(1, H, D, 1, P, pages * P, [ptr], [ptr + pages * P * H * D])
    c = {"H": H}
    a = (A.kvio_append_args if op == "append" else A.kvio_attend_args)()
    a.batch = batch_args(A, box, c, torch.tensor([[0, 1, 2], [3, 4, 5]], dtype=torch.int32), torch.tensor([40, 30], dtype=torch.int32),
                         torch.tensor([0, 3, 5], dtype=torch.int32), N)
    a.dtype, a.cache_dtype, a.num_q_heads, a.q_stride, a.scale_stride = 0, 2, Hq, Hq * D, H
    half = torch.zeros(N + 1, Hq, D, dtype=torch.bfloat16)
    a.q, a.k_scale, a.v_scale = box.put(half)[1], box.put(torch.ones(pages, H))[1], box.put(torch.ones(pages, H))[1]
    if op == "append":
        a.k, a.v, a.q_out = (box.put(x)[1] for x in (half[:, :H], half[:, :H], half))
        a.k_stride, a.v_stride, a.q_out_stride = H * D, H * D, Hq * D
    else:
        a.out, a.out_stride, a.softmax_scale, a.lse = box.put(half)[1], Hq * D, 0.125, box.put(torch.zeros(N, Hq))[1]
        need = ctypes.c_size_t()
        assert lib.kvio_attend_workspace(h, ctypes.byref(a), ctypes.byref(need)) == 0
        a.workspace, a.workspace_bytes = box.put(torch.zeros(max(need.value, 16), dtype=torch.uint8))[1], need.value
    return a, h, box


@pytest.mark.parametrize("op,changed,status,word", [("append", *x) for x in APPEND] + [("attend", *x) for x in ATTEND])
def test_refusals(emu, op, changed, status, word):
    kv, lib, A = emu
    a, h, box = refusal_case(kv, lib, A, op)
    call = getattr(lib, "kvio_" + op)
    assert call(h, 0, ctypes.byref(a), None) == 0, kv.kvio_last_error()
    for field, value in changed.items():
        of = a.batch if field.startswith("batch.") else a
        name = field.split(".")[-1]
        if isinstance(value, str):
            value = a.q + (16 if value == "q+16" else 0)
        elif isinstance(value, int) and isinstance(getattr(of, name), int) and getattr(of, name) > 1 << 20:
            value += getattr(of, name)                             # a pointer moved by so many bytes
        setattr(of, name, value)
    assert call(h, 0, ctypes.byref(a), None) == getattr(kv, "KVIO_" + status), kv.kvio_last_error()
    assert word in kv.kvio_last_error()
    kv.kvio_pool_destroy(h)
    box.free()


def test_null_and_empty_calls(emu):
    kv, lib, A = emu
    for op in ("append", "attend"):
        a, h, box = refusal_case(kv, lib, A, op)
        call = getattr(lib, "kvio_" + op)
        assert call(None, 0, ctypes.byref(a), None) == kv.KVIO_EINVAL and "null pool" in kv.kvio_last_error()
        assert call(h, 0, None, None) == kv.KVIO_EINVAL and "null arguments" in kv.kvio_last_error()
        assert call(h, 1, ctypes.byref(a), None) == call(h, -1, ctypes.byref(a), None) == kv.KVIO_EINVAL
        for field in ("num_seqs", "num_tokens"):
            b = type(a).from_buffer_copy(a)
            setattr(b.batch, field, 0)
            b.batch.page_table = b.q = None                        # nothing of an empty batch is looked at
            if op == "append":
                b.num_q_heads, b.q_out = 0, None
            assert call(h, 0, ctypes.byref(b), None) == 0, kv.kvio_last_error()
        kv.kvio_pool_destroy(h)
        box.free()
    n = ctypes.c_size_t()
    assert lib.kvio_attend_workspace(None, ctypes.byref(a), ctypes.byref(n)) == kv.KVIO_EINVAL


def test_heads_that_are_not_built(emu):
    kv, lib, A = emu
    box = Box(kv)
    for D, op in ((80, "attend"), (24, "append")):
        ptr = box.put(torch.zeros(2, 16, 2, D, dtype=torch.bfloat16))[1]
        h = kv.kvio_pool_create(1, 2, D, 2, 16, 16, [ptr], [ptr + 16 * 2 * D * 2])
        a = (A.kvio_append_args if op == "append" else A.kvio_attend_args)(batch=A.kvio_batch(1, 1, 1, 0, 1), num_q_heads=2 if op == "attend" else 0)
        assert getattr(lib, "kvio_" + op)(h, 0, ctypes.byref(a), None) == kv.KVIO_EINVAL and "dims" in kv.kvio_last_error()
        kv.kvio_pool_destroy(h)
    box.free()
