"""The joint call (norm, rotation, rows into slots) in all its forms: equal, bit for bit, to the separate calls, which are tested
against 64-bit references; slots that skip their token or lie outside the cache."""
import pytest
import torch

import paper_2511_07427_b200 as P

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
# head dim, rotary_dim, interleaved
FORMS = [(128, 128, False), (64, 64, False), (128, 64, False), (128, 64, True), (128, 48, False), (128, 128, True), (64, 0, False), (64, 64, True), (64, 16, True), (64, 32, False)]


def _joint(n, h, hk, d, dtype, layout):
    g = torch.Generator(device="cuda").manual_seed(n + d)
    if layout == "outer":
        return [torch.randn(k, n, d, generator=g, device="cuda").to(dtype).transpose(0, 1) for k in (h, hk, hk)]
    pad = 3 if layout == "odd" else 0             # rows that start at odd elements
    x = torch.randn(n, h + 2 * hk, d + pad, generator=g, device="cuda").to(dtype)[..., pad // 2:pad // 2 + d]
    return x[:, :h], x[:, h:h + hk], x[:, h + hk:]


@pytest.mark.parametrize("cache_type", [P.F32, P.BF16, P.FP8])
@pytest.mark.parametrize("d,rot,inter", FORMS)
@pytest.mark.parametrize("src,layout,norm,n,h,hk", [("bf16", "joint", True, 21, 6, 2), ("f32", "odd", False, 21, 5, 5), ("bf16", "odd", True, 700, 7, 1), ("f32", "outer", True, 700, 12, 3),
                                                    ("bf16", "outer", False, 1, 1, 1)])
def test_store_equals_apply_and_write(cache_type, d, rot, inter, src, layout, norm, n, h, hk):
    q, k, v = _joint(n, h, hk, d, DT[src], layout)
    g = torch.Generator(device="cuda").manual_seed(5)
    inv_freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().cuda()
    wq, wk = (torch.rand(d, generator=g, device="cuda") + 0.5 for _ in range(2)) if norm else (None, None)
    ro = P.HeadRotary(h, hk, d, inv_freq, q_weight=wq, k_weight=wk, interleaved=inter)
    pos = torch.randint(0, 1 << 17, (n,), generator=g, device="cuda", dtype=torch.int32)
    pages = (n + 31) // 32 + 2
    a, b = (P.RowCache.allocate(pages, hk, d, cache_type) for _ in range(2))
    for c in (a, b):
        for t in (c.k, c.v, c.k_exp, c.v_exp):
            if t is not None:
                t.view(torch.uint8).fill_(17)
    slots = torch.randperm(pages * 32, generator=g, device="cuda")[:n].to(torch.int32)
    skipped = [i for i in (3, 11) if i < n]
    outside = [i for i in (0, n - 1) if n > 1]
    slots[skipped] = -1
    if outside:
        slots[outside[0]], slots[outside[1]] = pages * 32, (1 << 31) - 1
    for q_dtype in (torch.float32, torch.bfloat16):
        got = ro.store(q, k, v, pos, a, slots, q_dtype=q_dtype)
        qo, ko = ro.apply(q, k, pos, q_dtype=q_dtype, k_dtype=torch.float32)
        assert torch.equal(got, qo)                # tokens that are not stored included
    b.write(ko, v.float(), slots)                  # fp32 keys: rounded once, as the joint call does
    for x, y in ((a.k, b.k), (a.v, b.v), (a.k_exp, b.k_exp), (a.v_exp, b.v_exp)):
        if x is not None:
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    used = torch.zeros(pages * 32, dtype=torch.bool)
    live = [i for i in range(n) if i not in skipped + outside]
    used[slots.cpu()[live].long()] = True
    rest = a.k.view(torch.uint8).cpu().view(pages, hk, 32, -1).permute(0, 2, 1, 3).reshape(pages * 32, -1)[~used]
    assert bool((rest == 17).all())
    want = P.ST_BOUNDS if outside else 0
    assert a.get_status() == want and b.get_status() == want


@pytest.mark.parametrize("d,rot,inter", [(128, 128, False), (128, 64, True)])
def test_values_that_are_no_numbers_stay_in_their_rows(d, rot, inter):
    """A NaN or an infinity of one head's row reaches no other row, and v is stored as it is."""
    n, h, hk = 40, 3, 2
    q, k, v = (x.clone() for x in _joint(n, h, hk, d, torch.bfloat16, "joint"))
    inv_freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()
    ro = P.HeadRotary(h, hk, d, inv_freq, q_weight=torch.ones(d, device="cuda"), k_weight=torch.ones(d, device="cuda"), interleaved=inter)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    slots = pos.clone()
    clean, wild = (P.RowCache.allocate(2, hk, d, P.BF16) for _ in range(2))
    want = ro.store(q, k, v, pos, clean, slots)
    q[5, 1, 3], k[6, 0, 7], v[7, 1, 0], v[8, 0, 1] = float("nan"), float("inf"), float("nan"), -float("inf")
    got = ro.store(q, k, v, pos, wild, slots)
    rows = torch.ones(n, h, dtype=torch.bool)
    rows[5, 1] = False
    assert torch.equal(got.cpu()[rows], want.cpu()[rows]) and bool(torch.isnan(got[5, 1]).any())
    kept = lambda c, x: x.permute(0, 2, 1, 3).reshape(64, hk, d)[:n].cpu()
    rows = torch.ones(n, hk, dtype=torch.bool)
    rows[6, 0] = False
    assert torch.equal(kept(wild, wild.k)[rows], kept(clean, clean.k)[rows])
    assert torch.equal(torch.nan_to_num(kept(wild, wild.v), nan=7.0), torch.nan_to_num(v.cpu(), nan=7.0))


@pytest.mark.parametrize("cache_type", [P.F32, P.BF16, P.FP8])
@pytest.mark.parametrize("d,rot,inter", FORMS)
def test_values_are_stored_as_the_write_stores_them(cache_type, d, rot, inter):
    """Zeros of either sign included."""
    n, h, hk = 33, 3, 2
    q, k, v = (x.clone() for x in _joint(n, h, hk, d, torch.bfloat16, "joint"))
    v[:, :, ::3] = -0.0
    v[5], v[6] = -0.0, 0.0
    inv_freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().cuda()
    ro = P.HeadRotary(h, hk, d, inv_freq, interleaved=inter)
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    a, b = (P.RowCache.allocate(2, hk, d, cache_type) for _ in range(2))
    for c in (a, b):
        c.v.view(torch.uint8).zero_()
        if c.v_exp is not None:
            c.v_exp.zero_()
    ro.store(q, k, v, at, a, at)
    b.write(k, v, at)
    assert torch.equal(a.v.view(torch.uint8), b.v.view(torch.uint8))
    assert a.v_exp is None or torch.equal(a.v_exp, b.v_exp)
