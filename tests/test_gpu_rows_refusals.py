"""Calls on plain rows that would drop a gradient are refused, whichever of their tensors asks for it."""
import pytest
import torch

import paper_2511_07427_b200 as P

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def _things():
    x = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(3, 4, 128, dtype=torch.bfloat16, device="cuda")
    at = torch.arange(3, **I32)
    return x, q, at


@pytest.mark.parametrize("which", ["inv_freq", "q_weight", "k_weight"])
def test_an_embedding_whose_constants_want_a_gradient(which):
    x, q, at = _things()
    c = P.RowCache.allocate(1, 2, 128, P.BF16)
    t = dict(inv_freq=torch.ones(64, device="cuda"), q_weight=torch.nn.Parameter(torch.ones(128, device="cuda"), requires_grad=False),
             k_weight=torch.nn.Parameter(torch.ones(128, device="cuda"), requires_grad=False))
    ro = P.HeadRotary(4, 2, 128, **t)
    for f in (lambda: ro.apply(q, x, at), lambda: ro.store(q, x, x, at, c, at)):
        f()
        t[which].requires_grad_()
        with pytest.raises(P.DynaKVError, match="gradient"):
            f()
        with torch.no_grad():
            f()
        with torch.inference_mode():
            f()
        t[which].requires_grad_(False)
    assert c.get_status() == 0


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_cache_whose_rows_want_a_gradient(which, dtype):
    x, q, at = (t.to(dtype) if t.is_floating_point() else t for t in _things())
    pools = dict(k=torch.zeros(1, 2, 32, 128, dtype=dtype, device="cuda"), v=torch.zeros(1, 2, 32, 128, dtype=dtype, device="cuda"))
    c = P.RowCache(**pools)
    ro = P.HeadRotary(4, 2, 128, torch.ones(64, device="cuda"))
    table, lens, start = torch.zeros(1, 1, **I32), torch.full((1,), 3, **I32), torch.tensor([0, 3], **I32)
    for f in (lambda: c.write(x, x, at), lambda: c.read(table, lens, 3), lambda: ro.store(q, x, x, at, c, at), lambda: c.attend_tree(q, table, lens, start, 3)):
        f()
        pools[which].requires_grad_()
        with pytest.raises(P.DynaKVError, match="gradient"):
            f()
        with torch.no_grad():
            f()
        pools[which].requires_grad_(False)
    out = torch.zeros_like(q, requires_grad=True)
    with pytest.raises(P.DynaKVError, match="gradient"):
        c.attend_tree(q, table, lens, start, 3, out=out)
    assert c.get_status() == 0


def test_tensors_whose_memory_was_replaced():
    x, q, at = _things()
    w = torch.nn.Parameter(torch.ones(128, device="cuda"), requires_grad=False)
    ro = P.HeadRotary(4, 2, 128, torch.ones(64, device="cuda"), q_weight=w)
    k, v = (torch.zeros(1, 2, 32, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = P.RowCache(k, v)
    table, lens, start = torch.zeros(1, 1, **I32), torch.full((1,), 3, **I32), torch.tensor([0, 3], **I32)
    before = ro.apply(q + 1, x + 1, at)[0]
    w.mul_(2.0)                                   # the same memory: fine
    assert torch.equal(ro.apply(q + 1, x + 1, at)[0], (before.float() * 2).bfloat16())
    w.data = torch.ones(128, device="cuda")
    for f in (lambda: ro.apply(q, x, at), lambda: ro.store(q, x, x, at, c, at)):
        with pytest.raises(P.DynaKVError, match="memory"):
            f()
    ro = P.HeadRotary(4, 2, 128, torch.ones(64, device="cuda"), q_weight=w)
    v.untyped_storage().resize_(0)
    for f in (lambda: c.write(x, x, at), lambda: c.read(table, lens, 3), lambda: ro.store(q, x, x, at, c, at), lambda: c.attend_tree(q, table, lens, start, 3)):
        with pytest.raises(P.DynaKVError, match="memory"):
            f()


@pytest.mark.parametrize("cache", [P.F32, P.BF16, P.FP8])
def test_a_negative_length_is_read_as_zeros_and_reported(cache):
    c = P.RowCache.allocate(2, 2, 64, cache)
    x = torch.ones(64, 2, 64, device="cuda")
    c.write(x, x, torch.arange(64, **I32))
    table = torch.tensor([[0], [1]], **I32)
    K, V = c.read(table, torch.tensor([0, 32], **I32), 40)
    assert c.get_status() == 0 and float(K[0].abs().max()) == 0 and float(K[1, :, :32].min()) == 1
    K, V = c.read(table, torch.tensor([32, -1], **I32), 40)
    assert float(K[0, :, :32].min()) == 1 and float(K[1].abs().max()) == 0 and float(V[1].abs().max()) == 0
    assert c.get_status() == P.ST_BOUNDS          # as attend_tree reports it
