"""Norm and rotary embedding of heads, and rows written to and read from a paged cache, against 64-bit references.

Tolerances count roundings.  A half step of a type is finfo.eps / 2 relative to the value.  In the norm and rotation, with
u = 2^-24: the mean of squares takes at most 12 roundings (8 in a lane, 4 across lanes), which the square root halves; the
square root, the division, the products with the factor and the weight add 4; the angle's rounding to fp32 (|half turns|
<= 1: pi u / 2 absolute) and the sine's own error another 4; the two products of the rotation 2: at most 16 u relative to
|a| + |b| of the pair.  24 u leaves room for no more than the constants' own roundings."""
import math

import numpy as np
import pytest
import torch

import paper_2511_07427_b200 as P

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TORCH = {P.F32: torch.float32, P.BF16: torch.bfloat16, P.FP8: torch.float8_e4m3fn}


def _half_step(t):
    return torch.finfo(t).eps / 2


def _rotated(x, w, eps, positions, inv_freq, rot, interleaved):
    """The formula in 64 bits; with it |a| + |b| of every element's pair."""
    x = x.double().cpu()
    if w is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w.double().cpu()
    out, size = x.clone(), x.abs()
    ang = positions.double().cpu()[:, None] * inv_freq.double().cpu()
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    ia = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    ib = ia + 1 if interleaved else ia + rot // 2
    a, b = x[..., ia], x[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return out, size


def _inputs(n, h, hk, d, dtype, seed, layout="joint"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if layout == "joint":           # slices of one projection
        x = torch.randn(n, h + 2 * hk, d, generator=g, device="cuda").to(dtype)
        return x[:, :h], x[:, h:h + hk], x[:, h + hk:]
    if layout == "odd":             # rows that start at odd elements: no 16-byte loads
        x = torch.randn(n, h + 2 * hk, d + 3, generator=g, device="cuda").to(dtype)[..., 1:d + 1]
        return x[:, :h], x[:, h:h + hk], x[:, h + hk:]
    x = [torch.randn(k, n, d, generator=g, device="cuda").to(dtype).transpose(0, 1) for k in (h, hk, hk)]      # heads outermost
    return x


def _freq(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().cuda()


def _check(got, want, size, extra=0.0):
    tol = 24 * U * size + extra + _half_step(got.dtype) * want.abs() + torch.finfo(got.dtype).tiny
    bad = ((got.double().cpu() - want).abs() - tol).max().item() if got.numel() else -1.0
    assert bad <= 0, bad


CASES = [
    # tokens, heads, KV heads, d, rotary_dim, interleaved, norm, input, q out, k out, layout
    (1, 28, 4, 128, 128, False, True, "bf16", "f32", "bf16", "joint"),
    (17, 32, 8, 128, 128, False, True, "bf16", "bf16", "bf16", "joint"),
    (5, 4, 1, 64, 64, False, False, "f32", "f32", "f32", "joint"),
    (33, 5, 5, 64, 32, True, True, "f32", "bf16", "f32", "odd"),
    (7, 3, 1, 128, 48, False, True, "bf16", "f32", "f32", "odd"),
    (7, 3, 1, 128, 48, True, True, "bf16", "f32", "f32", "outer"),
    (3, 1, 2, 128, 0, False, True, "f32", "f32", "bf16", "outer"),
    (2500, 12, 4, 64, 64, False, True, "bf16", "bf16", "bf16", "joint"),
    (2369, 9, 3, 128, 112, False, True, "bf16", "f32", "bf16", "odd"),
]
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("n,h,hk,d,rot,inter,norm,src,qd,kd,layout", CASES)
def test_norm_rope(n, h, hk, d, rot, inter, norm, src, qd, kd, layout):
    q, k, _ = _inputs(n, h, hk, d, DT[src], 3, layout)
    g = torch.Generator(device="cuda").manual_seed(9)
    wq, wk = (torch.randn(d, generator=g, device="cuda") for _ in range(2)) if norm else (None, None)
    pos = torch.randint(0, 1 << 20, (n,), generator=g, device="cuda", dtype=torch.int32)
    ro = P.HeadRotary(h, hk, d, _freq(rot), q_weight=wq, k_weight=wk, eps=1e-5, interleaved=inter)
    qo, ko = ro.apply(q, k, pos, q_dtype=DT[qd], k_dtype=DT[kd])
    for got, x, w in ((qo, q, wq), (ko, k, wk)):
        want, size = _rotated(x, w, 1e-5, pos, _freq(rot), rot, inter)
        _check(got, want, size)


def test_norm_of_one_side_only_and_far_and_negative_positions():
    q, k, _ = _inputs(6, 4, 2, 128, torch.float32, 5)
    w = torch.rand(128, device="cuda")
    pos = torch.tensor([0, 1, -1, -123456, (1 << 31) - 1, -(1 << 31)], dtype=torch.int32, device="cuda")
    ro = P.HeadRotary(4, 2, 128, _freq(128), k_weight=w)
    qo, ko = ro.apply(q, k, pos)
    # the 64-bit angle itself is off by its roundings: 2^-51 of it
    extra = (pos.double().abs().cpu() * 2.0 ** -51)[:, None, None]
    for got, x, ww in ((qo, q, None), (ko, k, w)):
        want, size = _rotated(x, ww, 1e-6, pos, _freq(128), 128, False)
        _check(got, want, size, extra * size)


def test_norm_rope_of_zero_rows_and_no_tokens():
    ro = P.HeadRotary(2, 1, 64, _freq(64), q_weight=torch.ones(64, device="cuda"), k_weight=torch.ones(64, device="cuda"))
    z = torch.zeros(3, 3, 64, device="cuda")
    qo, ko = ro.apply(z[:, :2], z[:, 2:], torch.arange(3, device="cuda", dtype=torch.int32))
    assert float(qo.abs().max()) == 0.0 and float(ko.abs().max()) == 0.0
    qo, ko = ro.apply(z[:0, :2], z[:0, 2:], torch.zeros(0, device="cuda", dtype=torch.int32))
    assert qo.shape == (0, 2, 64) and ko.shape == (0, 1, 64)


def _fp8_reference(x):
    """e4m3 values (before the row's scale) and exponents of rows, from the format's definition, in 64 bits."""
    x = x.double().cpu().numpy()
    top = np.abs(np.where(np.isnan(x), 0, x)).max(-1)
    e = np.zeros(top.shape)
    pos = top > 0
    with np.errstate(divide="ignore", invalid="ignore"):
        e[pos] = np.where(np.isinf(top[pos]), 120, np.ceil(np.log2(top[pos] / 448)))
        e = np.clip(np.nan_to_num(e, posinf=120), -120, 120)
        for _ in range(2):        # the logarithm may be off next to a whole number
            e = np.where(pos & (top > 448 * 2.0 ** e) & (e < 120), e + 1, e)
            e = np.where(pos & (top <= 448 * 2.0 ** (e - 1)) & (e > -120), e - 1, e)
        y = x / 2.0 ** e[..., None]
        grid = 2.0 ** (np.maximum(np.floor(np.log2(np.abs(y))), -6) - 3)
        grid = np.where(np.isfinite(grid) & (grid > 0), grid, 2.0 ** -9)
        r = np.clip(np.rint(y / grid) * grid, -448, 448)
    return np.where(np.isnan(x), np.nan, r), e.astype(np.int64)


def _special_rows(n, heads, d, dtype, seed):
    """Rows with what the rounding can go wrong at: zeros, tiny and huge rows, maxima on and next to 448 * 2^e, ties, NaN, Inf."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, heads, d, generator=g, device="cuda")
    s = torch.exp2(torch.randint(-100, 100, (n, heads, 1), generator=g, device="cuda").float())
    x = torch.where(torch.rand(n, heads, 1, generator=g, device="cuda") < 0.5, x * s, x)
    x[0, 0] = 0
    if n > 8:
        x[1, 0, 3] = 448 * 8.0
        x[2, 0] = x[2, 0].clamp(-1, 1); x[2, 0, 5] = -1.75
        x[3, 0] = x[3, 0].clamp(-1, 1); x[3, 0, 5] = 1.7578125                  # one bf16 step above 448 / 256
        x[4, 0] = 2.0 ** -130; x[4, 0, 1] = 2.0 ** -126
        x[5, 0] = 3e38
        x[6, 0, 2] = float("nan")
        x[7, 0, 9] = float("inf"); x[7, 0, 10] = -float("inf")
        x[8, 0] = (torch.arange(d, device="cuda") + 0.5) * 4                    # ties of the grid
    return x.to(dtype)


@pytest.mark.parametrize("cache_type", [P.F32, P.BF16, P.FP8])
@pytest.mark.parametrize("d,hk,n,src,layout", [(128, 4, 16, "bf16", "plain"), (128, 1, 1, "bf16", "plain"), (64, 3, 77, "f32", "odd"),
                                               (128, 8, 3001, "bf16", "plain"), (64, 5, 6001, "bf16", "outer"), (128, 2, 129, "f32", "plain")])
def test_write_and_read(cache_type, d, hk, n, src, layout):
    g = torch.Generator(device="cuda").manual_seed(n)
    k, v = (_special_rows(n, hk, d, DT[src], s) for s in (1, 2))
    if layout == "odd":
        k, v = (torch.cat([x, x[..., :3]], -1)[..., :d] for x in (k, v))
    elif layout == "outer":
        k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (k, v))
    pages = (n + 31) // 32 + 5
    shape = (pages, hk, 32, d)
    c = P.RowCache.allocate(pages, hk, d, cache_type)
    for t in (c.k, c.v, c.k_exp, c.v_exp):
        if t is not None:
            t.view(torch.uint8).fill_(17)
    slots = torch.randperm(pages * 32, generator=g, device="cuda")[:n].to(torch.int32)
    if n > 2:
        slots[n // 2] = -1
    c.write(k, v, slots)
    page, row = slots.long().cpu() // 32, slots.long().cpu() % 32
    used = torch.zeros(pages, 32, dtype=torch.bool)
    used[page[slots.cpu() >= 0], row[slots.cpu() >= 0]] = True
    live = slots.cpu() >= 0
    for x, pool, exp in ((k, c.k, c.k_exp), (v, c.v, c.v_exp)):
        rows = pool.view(torch.uint8).cpu().view(pages, hk, 32, -1).permute(0, 2, 1, 3)[page[live], row[live]].contiguous().view(TORCH[cache_type])      # [n, hk, d]
        if cache_type == P.FP8:
            want, e = _fp8_reference(x.cpu()[live])
            assert np.array_equal(exp.cpu().permute(0, 2, 1)[page[live], row[live]].numpy(), e)
            assert np.array_equal(rows.double().numpy(), want, equal_nan=True)
        else:
            want = x.cpu()[live].to(TORCH[cache_type])
            assert torch.equal(torch.nan_to_num(rows.double(), nan=7.5), torch.nan_to_num(want.double(), nan=7.5))
        # rows of no slot are as they were
        rest = pool.view(torch.uint8).cpu().view(pages, hk, 32, -1).permute(0, 2, 1, 3)[~used]
        assert bool((rest == 17).all())
        if exp is not None:
            assert bool((exp.cpu().permute(0, 2, 1)[~used] == 17).all())
    assert c.get_status() == 0
    assert tuple(c.k.shape) == shape


def _paged(case_seed, lens, hk, d, cache_type, spare=3):
    """A cache with sequences of the given lengths on shuffled pages; returns it, the page table and the rows as stored."""
    g = torch.Generator(device="cuda").manual_seed(case_seed)
    per = [(n + 31) // 32 for n in lens]
    width = max(per + [1])
    total = sum(per) + spare
    c = P.RowCache.allocate(total, hk, d, cache_type)
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    for t in (c.k, c.v, c.k_exp, c.v_exp):
        if t is not None:
            t.view(torch.uint8).fill_(0x7f)          # NaN rows (and large exponents) wherever nothing is written
    at, kept = 0, []
    for b, n in enumerate(lens):
        table[b, :per[b]] = order[at:at + per[b]]
        at += per[b]
        k, v = (torch.randn(n, hk, d, generator=g, device="cuda").to(torch.float32 if cache_type == P.F32 else torch.bfloat16) for _ in range(2))
        if n:
            slots = (table[b].long()[torch.arange(n, device="cuda") // 32] * 32 + torch.arange(n, device="cuda") % 32).to(torch.int32)
            c.write(k, v, slots)
        if cache_type == P.FP8:
            k, v = ((torch.from_numpy(y) * 2.0 ** torch.from_numpy(e).double()[..., None]).to(torch.bfloat16).cuda() for y, e in (_fp8_reference(k), _fp8_reference(v)))
        kept.append((k, v))
    return c, table, kept


@pytest.mark.parametrize("cache_type", [P.F32, P.BF16, P.FP8])
@pytest.mark.parametrize("lens,hk,d,first,n", [([1], 1, 128, 0, 1), ([0, 31, 32, 33, 100], 3, 64, 0, 100), ([257, 64, 5], 2, 128, 33, 90), ([40], 2, 128, 100, 7)])
def test_read(cache_type, lens, hk, d, first, n):
    c, table, kept = _paged(4, lens, hk, d, cache_type)
    K, V = c.read(table, torch.tensor(lens, dtype=torch.int32, device="cuda"), n, first=first)
    for got, i in ((K, 0), (V, 1)):
        want = torch.zeros_like(got)
        for b, m in enumerate(lens):
            part = kept[b][i][first:min(m, first + n)].transpose(0, 1)
            want[b, :, :part.shape[1]] = part
        assert torch.equal(got, want)
    assert c.get_status() == 0


@pytest.mark.parametrize("cache_type", [P.F32, P.BF16, P.FP8])
@pytest.mark.parametrize("d,n", [(128, 21), (64, 2400)])
def test_store_is_apply_and_write(cache_type, d, n):
    h, hk = 6, 2
    q, k, v = _inputs(n, h, hk, d, torch.bfloat16, 8)
    ro = P.HeadRotary(h, hk, d, _freq(d), q_weight=torch.rand(d, device="cuda"), k_weight=torch.rand(d, device="cuda"))
    pos = torch.arange(n, device="cuda", dtype=torch.int32) * 7
    a, b = (P.RowCache.allocate((n + 31) // 32, hk, d, cache_type) for _ in range(2))
    slots = torch.randperm(a.n_pages * 32, device="cuda")[:n].to(torch.int32)
    for c in (a, b):
        for t in (c.k, c.v, c.k_exp, c.v_exp):
            if t is not None:
                t.view(torch.uint8).zero_()
    got = ro.store(q, k, v, pos, a, slots, q_dtype=torch.float32)
    qo, ko = ro.apply(q, k, pos, q_dtype=torch.float32, k_dtype=torch.float32)
    b.write(ko, v.float(), slots)                  # fp32 keys: rounded once, as the joint call does
    assert torch.equal(got, qo)
    for x, y in ((a.k, b.k), (a.v, b.v), (a.k_exp, b.k_exp), (a.v_exp, b.v_exp)):
        if x is not None:
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_slots_and_pages_out_of_range_are_skipped_and_reported():
    c = P.RowCache.allocate(2, 1, 128, P.FP8)
    for t in (c.k, c.v, c.k_exp, c.v_exp):
        t.view(torch.uint8).zero_()
    x = torch.randn(3, 1, 128, device="cuda")
    c.write(x, x, torch.tensor([-5, 3, -(1 << 31)], dtype=torch.int32, device="cuda"))
    assert c.get_status() == 0
    before = c.k.view(torch.uint8).clone()
    c.write(x, x, torch.tensor([64, 1 << 30, (1 << 31) - 1], dtype=torch.int32, device="cuda"))
    assert c.get_status() == P.ST_BOUNDS and torch.equal(before, c.k.view(torch.uint8))
    c = P.RowCache(c.k, c.v, c.k_exp, c.v_exp)
    table = torch.tensor([[0, 2], [-1, 0]], dtype=torch.int32, device="cuda")
    K, _ = c.read(table, torch.tensor([64, 64], dtype=torch.int32, device="cuda"), 64)
    assert c.get_status() == P.ST_BOUNDS
    assert float(K[0, 0, 3].abs().max()) > 0 and float(K[0, 0, 32:].abs().max()) == 0 and float(K[1, 0, :32].abs().max()) == 0
    assert torch.equal(K[1, 0, 32:], K[0, 0, :32])
    c = P.RowCache(c.k, c.v, c.k_exp, c.v_exp)
    K, _ = c.read(table[:1, :1].contiguous(), torch.tensor([40], dtype=torch.int32, device="cuda"), 40)         # a length past the page table
    assert c.get_status() == P.ST_BOUNDS and float(K[0, 0, 32:].abs().max()) == 0


def test_binding_refusals():
    c = P.RowCache.allocate(4, 2, 128, P.BF16)
    ro = P.HeadRotary(4, 2, 128, _freq(128))
    x = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(3, 4, 128, dtype=torch.bfloat16, device="cuda")
    i = torch.zeros(3, dtype=torch.int32, device="cuda")
    E = P.DynaKVError
    for f in (lambda: c.write(x.half(), x.half(), i), lambda: c.write(x, x.float(), i), lambda: c.write(x, x, i.long()), lambda: c.write(x, x, i[:2]),
              lambda: c.write(x[:, :1], x[:, :1], i), lambda: c.write(x.transpose(1, 2), x.transpose(1, 2), i), lambda: c.write(x.cpu(), x, i),
              lambda: c.read(i, i, 4), lambda: c.read(i[None], i, 4), lambda: c.read(i[None], i[:1], -1), lambda: c.read(i[None].long(), i[:1], 4),
              lambda: ro.apply(q, x, i.float()), lambda: ro.apply(q, q, i), lambda: ro.apply(q, x, i, q_dtype=torch.float16),
              lambda: ro.apply(q.clone().requires_grad_(), x, i), lambda: ro.store(q, x, x, i, P.RowCache.allocate(4, 1, 128), i),
              lambda: P.RowCache(c.k, c.v[:, :, :, :64].contiguous()), lambda: P.RowCache(c.k, c.v, i, i), lambda: P.RowCache(c.k.transpose(0, 1), c.v.transpose(0, 1)),
              lambda: P.RowCache(c.k.view(torch.uint8)[..., :128].contiguous(), c.v.view(torch.uint8)[..., :128].contiguous()),
              lambda: P.RowCache.allocate(4, 2, 96), lambda: P.RowCache.allocate(4, 2, 128, 5), lambda: P.HeadRotary(4, 2, 128, _freq(128).double())):
        with pytest.raises(E):
            f()
    with torch.no_grad():
        ro.apply(q.clone().requires_grad_(), x, i)


def test_rows_on_a_side_stream_and_in_a_graph():
    h, hk, d, n = 8, 2, 128, 40
    ro = P.HeadRotary(h, hk, d, _freq(d))
    c = P.RowCache.allocate(4, hk, d, P.FP8)
    table = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    x = torch.empty(n, h + 2 * hk, d, dtype=torch.bfloat16, device="cuda")
    pos = torch.empty(n, dtype=torch.int32, device="cuda")

    def step():
        q = ro.store(x[:, :h], x[:, h:h + hk], x[:, h + hk:], pos, c, slots)
        return (q, *c.read(table, lens, n))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x.normal_(); pos.fill_(3)
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (1, 2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x.copy_(torch.randn(x.shape, generator=g, device="cuda")); pos.copy_(torch.randint(0, 1000, (n,), generator=g, device="cuda"))
        graph.replay()
        held = [t.clone() for t in got]
        for a, b in zip(held, step()):
            assert torch.equal(a, b)
