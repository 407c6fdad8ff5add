"""append and attend on an MI355X at the ends of what their arguments may hold."""
import math

import pytest

from test_gpu_attn import filled, kv, on_gpu  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("odd", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("D,new", [(64, 4), (64, 90), (128, 5), (128, 12), (128, 100), (256, 3), (256, 70)])
def test_a_hidden_tokens_scale_has_no_effect(kv, D, new, dtype, odd):  # noqa: F811
    """The last token's page, of one token, gets such a scale of values: the rows before it stay as they are."""
    import torch
    c = filled(8, getattr(torch, dtype), 8, 2, D, 1, [(700, new), (40, 3)], seed=new)
    g, pool, batch = on_gpu(kv, c)
    lses = [torch.empty(g["q"].shape[:2], device="cuda") for _ in range(2)]
    clean = pool.attend(0, batch, g["q"], lse=lses[0])
    page = int(c["table"][0, 700 + new - 1])
    g["scales"][1, 0, page, 0] = odd
    got = pool.attend(0, batch, g["q"], lse=lses[1])
    assert torch.equal(got[:new - 1], clean[:new - 1]) and torch.equal(got[new:], clean[new:]) and torch.equal(*lses)
    assert torch.equal(got[new - 1, 4:], clean[new - 1, 4:])
    code = g["pool"].view(torch.float8_e4m3fn)[1, 0, page, 0].float()
    want = (code * odd).to(got.dtype)                              # nothing finite counts beside it
    row = got[new - 1, :4]
    assert bool(((row == want) | (row.isnan() & want.isnan())).all())
    pool.close()


@pytest.mark.parametrize("was,now", [(0.0, 2.0 ** -100), (2.0 ** -140, 2.0 ** -100), (2.0 ** -101, 2.0 ** -100), (math.inf, 2.0 ** -100),
                                     (2.0 ** -100, 2.0 ** -100), (0.75, 0.75)])
def test_append_zeros_to_a_begun_page_of_any_scale(kv, was, now):  # noqa: F811
    """Rows of zeros stay zeros, and a scale that codes cannot be divided by is replaced."""
    import torch
    H, D, P = 4, 128, 16
    codes = torch.full((2, 1, 2 * P, H, D), 0x38, dtype=torch.uint8, device="cuda")                # 1.0
    scales = torch.full((2, 1, 2, H), was, device="cuda")
    pool = kv.KVPool(codes, P, scales=scales)
    batch = kv.Batch(torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"), torch.tensor([7], dtype=torch.int32, device="cuda"))
    zeros = torch.zeros(1, H, D, dtype=torch.bfloat16, device="cuda")
    pool.append(0, batch, zeros, zeros)
    assert bool((scales[:, 0, 1] == now).all()) and bool((scales[:, 0, 0] == was).all())
    assert bool((codes[:, 0, P + 6] == 0).all())                   # the seventh token
    old = {True: 0x38}.get(was == now, 0x7e if was == math.inf else None)
    rest = codes[:, 0, P:P + 6]
    if old is not None:
        assert bool((rest == old).all())
    else:                                                          # 1.0 times `was`, under 2^-100
        want = torch.tensor(was / now).to(torch.float8_e4m3fn).view(torch.uint8).item()
        assert bool((rest == want).all())
    assert bool((codes[:, 0, :P] == 0x38).all()) and bool((codes[:, 0, P + 7:] == 0x38).all())
    pool.close()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("D,new", [(64, 16), (128, 7), (128, 90), (256, 70)])
def test_windows_longer_than_the_context(kv, D, new, bits):  # noqa: F811
    """A window that hides nothing gives the bits of none, also where contexts have fewer tokens than are new."""
    import torch
    c = filled(bits, torch.bfloat16, 8, 2, D, 16, [(300, new), (0, new), (0, new)], seed=D + new)
    c["ctx"][1] = new // 2
    g, pool, batch = on_gpu(kv, c)
    want = pool.attend(0, batch, g["q"])
    row = new + new - new // 2
    assert bool((want[new:row] == 0).all()) and bool((want[row:] != 0).any(2).all())
    for window in (300 + new, 2 ** 31 - 1):
        assert torch.equal(want, pool.attend(0, batch, g["q"], window=window))
    pool.close()


def test_numbers_and_shapes_that_no_call_takes(kv):  # noqa: F811
    """Numbers that 32 bits do not hold are refused, not cut to their lowest 32 bits; so are tensors of other ranks."""
    import torch
    c = filled(16, torch.bfloat16, 4, 2, 64, 16, [(20, 2)], seed=1)
    g, pool, batch = on_gpu(kv, c)
    q, k = g["q"], torch.zeros(2, 2, 64, device="cuda", dtype=torch.bfloat16)
    bad = [lambda: pool.attend(0, batch, q, window=2 ** 32 + 5), lambda: pool.attend(0, batch, q, window=2 ** 31),
           lambda: pool.attend(2 ** 32, batch, q), lambda: pool.append(2 ** 32, batch, k, k), lambda: pool.attend(-1, batch, q),
           lambda: kv.Batch(g["table"], g["ctx"], g["starts"], 2 ** 32 + 1), lambda: kv.Batch(g["table"], g["ctx"], g["starts"], -1),
           lambda: kv.attend_workspace(pool, batch, q, window=2 ** 32), lambda: kv.attend_workspace(pool, batch, q[0]),
           lambda: kv.attend_workspace(pool, batch, q.sum()), lambda: pool.attend(0, batch, q.sum()), lambda: pool.attend(0, batch, q[0]),
           lambda: pool.append(0, batch, k.sum(), k), lambda: pool.append(0, batch, k, k.sum()), lambda: pool.append(0, batch, k, k, q=q[0])]
    for i, f in enumerate(bad):
        with pytest.raises(kv.KvioError) as e:
            f()
        assert e.value.status == kv.KVIO_EINVAL, i
    pool.attend(0, batch, q, window=2 ** 31 - 1)
    pool.close()


def test_tensors_that_want_gradients(kv):  # noqa: F811
    """Neither call has a backward pass: refused where autograd records, ordinary calls where it does not."""
    import torch
    c = filled(16, torch.bfloat16, 4, 2, 64, 16, [(20, 2)], seed=1)
    g, pool, batch = on_gpu(kv, c)
    q, k = g["q"], torch.zeros(2, 2, 64, device="cuda", dtype=torch.bfloat16)
    want = pool.attend(0, batch, q)
    before = pool.tensor.clone()
    qg, kg = q.clone().requires_grad_(), k.clone().requires_grad_()
    for f in (lambda: pool.attend(0, batch, qg), lambda: pool.attend(0, batch, qg * 1.0), lambda: pool.attend(0, batch, q, out=qg),
              lambda: pool.append(0, batch, kg, k), lambda: pool.append(0, batch, k, kg * 1.0), lambda: pool.append(0, batch, k, k, q=qg)):
        with pytest.raises(kv.KvioError, match="no backward pass"):
            f()
    assert torch.equal(pool.tensor.view(torch.int16), before.view(torch.int16))
    with torch.no_grad():
        assert torch.equal(pool.attend(0, batch, qg), want)
    assert torch.equal(pool.attend(0, batch, (qg * 1.0).detach()), want)
    with torch.inference_mode():
        assert torch.equal(pool.attend(0, batch, q.clone()), want)
    assert not pool.attend(0, batch, q).requires_grad
    pool.close()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("new", [1, 5, 90])
def test_pages_outside_the_pool_are_reported(kv, new, bits):  # noqa: F811
    """By kvio_check, with the sequence and its page, where some row sees a token of theirs; not outside a window or behind a
    context."""
    import torch
    c = filled(bits, torch.bfloat16, 8, 2, 128, 16, [(100, new), (3000, new)], seed=new)
    g, pool, batch = on_gpu(kv, c)
    pool.attend(0, batch, g["q"])
    pool.check()
    last = (3000 + new - 1) // 16
    for j, window, seen in ((0, 0, True), (last, 0, True), (last, 10, True), (90, 1000, False), ((3000 - 999) // 16, 1000, True)):
        keep = g["table"][1, j].item()
        g["table"][1, j] = -1 if j else 1 << 30
        pool.attend(0, batch, g["q"], window=window)
        if seen:
            with pytest.raises(kv.KvioError, match=f"span 1, context page {j}:"):
                pool.check()
        pool.check()
        g["table"][1, j] = keep
    pool.close()
