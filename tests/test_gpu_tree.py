"""Tree attention over a paged cache against a 64-bit reference.

Tolerances, with u = 2^-24.  A logit of d products summed in fp32 is off by at most (d + 4) u sum |q_e k_e| scale; the
exponential of a difference adds 4 u of the logits' size, and 2^-21 for the approximate instruction and the merges: eps, the
relative error of a weight, doubled because the sum of weights has it too.  Weights enter the products as bf16 hi + lo (2^-16),
f16 (2^-11 of the weight, 2^-25 of the largest weight times scale when subnormal) or fp32; a sum over n rows adds n u; the
output's own rounding half a step."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2511_07427_b200 as P

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
KV = {"f32": P.F32, "bf16": P.BF16, "fp8": P.FP8}


class Problem:
    """Sequences of given lengths on shuffled pages, drafted tokens, optional trees; NaN wherever nothing was written."""

    def __init__(self, lens, drafts, heads, hk, d, cache, tree=False, seed=0, spare=2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.drafts, self.heads, self.hk, self.d, self.cache = lens, drafts, heads, hk, d, cache
        per = [(n + 31) // 32 for n in lens]
        total = sum(per) + spare
        self.c = P.RowCache.allocate(total, hk, d, KV[cache])
        for t in (self.c.k, self.c.v, self.c.k_exp, self.c.v_exp):
            if t is not None:
                t.view(torch.uint8).fill_(0xff)
        order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((len(lens), max(per + [0])), 1 << 30, dtype=torch.int32, device="cuda")
        at = 0
        io = torch.float32 if cache == "f32" else torch.bfloat16
        for b, n in enumerate(lens):
            self.table[b, :per[b]] = order[at:at + per[b]]
            at += per[b]
            if n:
                k, v = (torch.randn(n, hk, d, generator=g, device="cuda").to(io) for _ in range(2))
                v = v * torch.exp2(torch.randint(-6, 4, (n, 1, 1), generator=g, device="cuda").float()).to(io)
                self.c.write(k, v, self.slots(b, 0, n))
        self.q = torch.randn(sum(drafts), heads, d, generator=g, device="cuda").to(io)
        self.q_start = torch.tensor(np.concatenate([[0], np.cumsum(drafts)]), dtype=torch.int32, device="cuda")
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.most = max(drafts + [1])
        self.sees = [torch.ones(t, t, dtype=torch.bool).tril() for t in drafts]
        self.mask = None
        if tree:
            rng = np.random.default_rng(seed)
            for t, s in zip(drafts, self.sees):
                s.zero_()
                for i in range(t):
                    p = int(rng.integers(-1, i)) if i else -1
                    if p >= 0:
                        s[i] = s[p]
                    s[i, i] = True
            self.pack()

    def slots(self, b, first, n):
        i = torch.arange(first, first + n, device="cuda")
        return (self.table[b].long()[i // 32] * 32 + i % 32).to(torch.int32)

    def pack(self):
        words = (self.most + 63) // 64
        m = np.zeros((sum(self.drafts), words), dtype=np.uint64)
        at = 0
        for t, s in zip(self.drafts, self.sees):
            for i in range(t):
                for j in np.nonzero(s[i].numpy())[0]:
                    m[at + i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
            at += t
        self.mask = torch.from_numpy(m.view(np.int64)).cuda()

    def run(self, **kw):
        return self.c.attend_tree(self.q, self.table, self.kv_len, self.q_start, self.most, tree_mask=self.mask, **kw)

    def check(self, out, lse, scale=None):
        scale = scale if scale is not None else self.d ** -0.5
        group, half = self.heads // self.hk, torch.finfo(out.dtype).eps / 2
        at = 0
        for b, (n, t) in enumerate(zip(self.lens, self.drafts)):
            sees = torch.ones(t, n, dtype=torch.bool)
            for j in range(max(0, n - t), n):
                sees[:, j] = self.sees[b][:, j - (n - t)]
            if n == 0:
                assert not out[at:at + t].any() and bool((lse[at:at + t] == -math.inf).all())
            for h in range(self.hk if n and t else 0):
                pages = self.table[b].long()[:(n + 31) // 32]
                def rows(pool, exp):
                    x = pool.view(torch.uint8)[pages, h].contiguous().view(pool.dtype).double().reshape(-1, self.d)[:n].cpu()
                    e = exp[pages, h].reshape(-1)[:n].double().cpu() if exp is not None else torch.zeros(n, dtype=torch.float64)
                    return x, torch.exp2(e)[:, None]
                (k8, ke), (v8, ve) = rows(self.c.k, self.c.k_exp), rows(self.c.v, self.c.v_exp)
                k, v = k8 * ke, v8 * ve
                q = self.q[at:at + t, h * group:(h + 1) * group].double().cpu()
                s = torch.einsum("tgd,nd->tgn", q, k) * scale
                size = torch.einsum("tgd,nd->tgn", q.abs(), k.abs()) * abs(scale)
                see = sees[:, None].expand(-1, group, -1)
                s = torch.where(see, s, -math.inf)
                want_lse = torch.logsumexp(s, -1)
                w = torch.exp(s - torch.where(torch.isfinite(want_lse), want_lse, 0.0)[..., None])
                w = torch.where(see, w, 0.0)
                vv = torch.where(see[..., None], v, 0.0)                     # rows not seen do not count, whatever they hold
                want = (w[..., None] * vv).sum(-2)
                weight = (w[..., None] * vv.abs()).sum(-2)
                size = torch.where(see, torch.nan_to_num(size, posinf=0.0), 0.0)
                eps = ((self.d + 4) * U * size.amax(-1) + 4 * U * size.amax(-1) + 2.0 ** -21)[..., None]
                tol = (2 * eps + n * U) * weight + half * want.abs()
                if self.cache == "bf16":
                    tol += 2.0 ** -16 * weight
                if self.cache == "fp8":
                    top = torch.where(see, w * ve[:, 0], 0.0).amax(-1)[..., None]
                    tol += 2.0 ** -11 * weight + 2.0 ** -25 * top * torch.where(see[..., None], v8.abs(), 0.0).sum(-2)
                got = out[at:at + t, h * group:(h + 1) * group].double().cpu()
                got_lse = lse[at:at + t, h * group:(h + 1) * group].double().cpu()
                fine = torch.isfinite(want)
                assert torch.equal(torch.isnan(got), torch.isnan(want)), (b, h)
                assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
                bad = ((got - want).abs() - tol)[fine]
                assert bad.numel() == 0 or bad.max().item() <= 0, (b, h, bad.max().item(), (got - want).abs()[fine].max().item())
                empty = ~see.any(-1)
                assert bool((got_lse[empty] == -math.inf).all()) and not got[empty].any()
                d = (got_lse - want_lse).abs() - eps[..., 0] * 2 - 4 * U * want_lse.abs()
                d = d[~empty & torch.isfinite(want_lse)]
                assert d.numel() == 0 or d.max().item() <= 0, (b, h, d.max().item())
            at += t
        assert self.c.get_status() == 0


LENGTHS = [([1], [1]), ([31, 32, 33], [1, 1, 1]), ([5, 0, 100, 64], [3, 2, 0, 4]), ([700], [1]), ([129, 1025], [7, 2])]


@pytest.mark.parametrize("cache", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,drafts", LENGTHS)
@pytest.mark.parametrize("heads,hk", [(4, 1), (7, 1), (6, 3)])
def test_chains(cache, d, lens, drafts, heads, hk):
    p = Problem(lens, drafts, heads, hk, d, cache)
    p.check(*p.run())


@pytest.mark.parametrize("cache", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("d,lens,drafts,heads,hk", [
    (128, [40, 300, 65], [5, 16, 33], 8, 2), (128, [1000], [64], 4, 1), (64, [130, 500], [70, 65], 8, 1), (128, [256, 300], [256, 200], 2, 2),
    (64, [20, 9], [20, 9], 16, 2), (128, [4000, 33], [12, 3], 7, 1)])
def test_trees(cache, d, lens, drafts, heads, hk):
    p = Problem(lens, drafts, heads, hk, d, cache, tree=True, seed=5)
    p.check(*p.run())


@pytest.mark.parametrize("cache", ["f32", "bf16", "fp8"])
def test_long_rows_are_shared_out_and_merged(cache):
    p = Problem([20000, 3, 9001], [2, 1, 1], 8, 2, 128, cache, seed=2)
    p.check(*p.run())


@pytest.mark.parametrize("cache,tree", [("bf16", False), ("fp8", True), ("f32", False)])
def test_many_short_sequences(cache, tree):
    lens = [(b * 37) % 90 for b in range(333)]
    p = Problem(lens, [min(n, 1 + b % 3) for b, n in enumerate(lens)], 4, 2, 64, cache, tree=tree, seed=3)
    p.check(*p.run())


@pytest.mark.parametrize("cache", ["f32", "bf16", "fp8"])
def test_rows_whose_mask_leaves_nothing(cache):
    p = Problem([6, 40], [6, 3], 4, 2, 128, cache, tree=True)
    p.sees[0][2] = False                      # no context either: sees no row at all
    p.sees[0][4] = False
    p.sees[1][0] = False                      # sees its context only
    p.pack()
    out, lse = p.run()
    p.check(out, lse)
    assert not out[2].any() and bool((lse[2] == -math.inf).all())


@pytest.mark.parametrize("cache,d,heads", [("f32", 128, 4), ("bf16", 128, 4), ("bf16", 64, 8), ("bf16", 128, 16), ("fp8", 128, 4), ("fp8", 64, 2)])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_nan_and_infinities_in_rows_not_seen(cache, d, heads, what):
    if cache == "fp8" and what == "inf":
        pytest.skip("an e4m3 byte holds no infinity")
    p = Problem([45, 70], [8, 5], heads, 2, d, cache, tree=True, seed=11)
    for b, j, which in ((0, 2, "v"), (0, 5, "k"), (1, 4, "v"), (1, 1, "k")):
        s = p.sees[b]
        s[:, j] = False                       # a branch of its own: seen by nobody but (here) one token
        s[j, j] = True
        n = p.lens[b] - p.drafts[b] + j
        pool = getattr(p.c, which)
        row = pool[p.table[b, n // 32].item(), :, n % 32] if cache != "fp8" else pool.view(torch.uint8)[p.table[b, n // 32].item(), :, n % 32]
        row[:, 3] = {"nan": float("nan"), "inf": float("inf")}[what] if cache != "fp8" else 0x7f
    p.pack()
    out, lse = p.run()
    # every token but the two whose own key is no number; those that see a bad V row among them
    for b, at, rows in ((0, 0, [0, 1, 2, 3, 4, 6, 7]), (1, 8, [0, 2, 3, 4])):
        _check_rows(p, b, at, out, lse, rows)


@pytest.mark.parametrize("cache,d", [("fp8", 128), ("fp8", 64), ("bf16", 128), ("f32", 64)])
def test_drafted_nan_rows_with_few_query_rows(cache, d):
    p = Problem([45, 70], [4, 3], 2, 1, d, cache, tree=True, seed=12)       # at most 8 query rows
    for b, j, which in ((0, 1, "v"), (0, 3, "k"), (1, 2, "v")):
        p.sees[b][:, j] = False
        p.sees[b][j, j] = True
        n = p.lens[b] - p.drafts[b] + j
        pool = getattr(p.c, which)
        row = pool[p.table[b, n // 32].item(), :, n % 32] if cache != "fp8" else pool.view(torch.uint8)[p.table[b, n // 32].item(), :, n % 32]
        row[:, 3] = float("nan") if cache != "fp8" else 0x7f
    p.pack()
    out, lse = p.run()
    for b, at, rows in ((0, 0, [0, 1, 2]), (1, 4, [0, 1, 2])):
        _check_rows(p, b, at, out, lse, rows)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,drafts", [(7, 1), (2, 4), (4, 4), (8, 8), (8, 16)])
def test_fp8_rows_of_very_different_scales(d, heads, drafts):
    p = Problem([333, 64], [drafts, 1], heads, 1, d, "fp8", seed=13)
    g = torch.Generator(device="cuda").manual_seed(14)
    p.c.v_exp.copy_(torch.randint(-120, 100, p.c.v_exp.shape, generator=g, device="cuda"))
    p.c.k_exp.sub_(torch.randint(0, 30, p.c.k_exp.shape, generator=g, device="cuda").to(torch.int8))
    p.check(*p.run())


def _check_rows(p, b, at, out, lse, rows):
    """Some tokens of sequence b (its first one is packed row `at`) against the formula over the rows they see, and only those."""
    n, t, group = p.lens[b], p.drafts[b], p.heads // p.hk
    pages = p.table[b].long()[:(n + 31) // 32]
    for h in range(p.hk):
        def get(pool, exp):
            x = pool.view(torch.uint8)[pages, h].contiguous().view(pool.dtype).double().reshape(-1, p.d)[:n].cpu()
            return x if exp is None else x * torch.exp2(exp[pages, h].reshape(-1)[:n].double().cpu())[:, None]
        k, v = get(p.c.k, p.c.k_exp), get(p.c.v, p.c.v_exp)
        for i in rows:
            see = torch.cat([torch.ones(n - t, dtype=torch.bool), p.sees[b][i]])
            for g in range(group):
                s = (p.q[at + i, h * group + g].double().cpu() @ k[see].T) * p.d ** -0.5
                w = torch.softmax(s, -1)
                want = w @ v[see]
                got = out[at + i, h * group + g].double().cpu()
                assert torch.equal(torch.isnan(want), torch.isnan(got)) and torch.equal(want[torch.isinf(want)], got[torch.isinf(got)]), (h, i, g)
                assert abs(lse[at + i, h * group + g].item() - torch.logsumexp(s, -1).item()) < 1e-4
                fine = torch.isfinite(want)
                # weights: f16 or bf16 hi + lo, with the bounds of the header; 70 rows keep the fp32 terms below 2^-13
                tol = (2.0 ** -10 if p.cache == "fp8" else 2.0 ** -13) * (w @ torch.nan_to_num(v[see], posinf=0.0).abs()) + torch.finfo(out.dtype).eps / 2 * want.abs()
                assert bool(((got - want).abs() <= tol)[fine].all()), (h, i, g)


def test_infinite_and_nan_logits_of_seen_rows():
    p = Problem([50], [1], 2, 1, 128, "bf16")
    p.c.k[p.table[0, 0].item(), 0, 3, 0] = float("inf")
    out, lse = p.run()
    for head in range(2):                      # a logit of +inf: inf - inf; one of -inf: a weight of 0
        if p.q[0, head, 0].item() > 0:
            assert bool(torch.isnan(out[0, head]).all()) and not math.isfinite(lse[0, head].item())
        else:
            assert bool(torch.isfinite(out[0, head]).all()) and math.isfinite(lse[0, head].item())
    p.c.k[p.table[0, 0].item(), 0, 3, 0] = float("nan")
    out, lse = p.run()
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())


@pytest.mark.parametrize("cache", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 2.5])
def test_scales(cache, scale):
    p = Problem([77, 40], [3, 1], 4, 2, 64, cache)
    p.check(*p.run(scale=scale), scale=scale)


def test_tokens_behind_the_last_sequence_are_left():
    p = Problem([50, 20], [3, 2], 4, 2, 128, "bf16")
    q = torch.cat([p.q, torch.full((4, 4, 128), float("nan"), dtype=torch.bfloat16, device="cuda")])
    out = torch.full_like(q, 7.0)
    o, lse = p.c.attend_tree(q, p.table, p.kv_len, p.q_start, 3, out=out)
    assert o is out and bool((out[5:] == 7.0).all())
    p.check(out[:5], lse[:5])


def test_same_bits_every_time_and_under_a_graph():
    p = Problem([3000, 700, 5], [4, 4, 4], 8, 2, 128, "fp8", tree=True)
    a = p.run()
    for _ in range(3):
        b = p.run()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = p.run()
    side.synchronize()
    assert torch.equal(a[0], c[0])
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = p.run()
        graphs.append((g, r))
    # the lengths are read on the device: the captured call follows a cache that grows
    p.kv_len.copy_(torch.tensor([2999, 650, 4], dtype=torch.int32))
    want = p.run()
    for g, r in graphs:
        with torch.cuda.stream(side):
            g.replay()
    for g, r in graphs:
        with torch.cuda.stream(side):
            g.replay()
    torch.cuda.synchronize()
    for g, r in graphs:
        assert torch.equal(r[0], want[0]) and torch.equal(r[1], want[1])


@pytest.mark.parametrize("cache,lens,drafts,heads,hk,d", [("bf16", [2, 40], [5, 60], 2, 1, 128), ("fp8", [50, 3], [200, 3], 4, 4, 64), ("fp8", [70], [100], 4, 2, 128),
                                                          ("f32", [7], [9], 6, 3, 64), ("bf16", [33, 90], [256, 7], 3, 1, 64)])
@pytest.mark.parametrize("tree", [False, True])
def test_more_drafts_than_rows(cache, lens, drafts, heads, hk, d, tree):
    """The rows are the tree's last ones: those that would lie before the cache's first row do not exist."""
    p = Problem(lens, drafts, heads, hk, d, cache, tree=tree, seed=9)
    p.check(*p.run())


@pytest.mark.parametrize("cache", ["f32", "bf16", "fp8"])
def test_two_streams_at_once(cache):
    a, b = (Problem([4000, 900], [3, 20], 8, 2, 128, cache, seed=s) for s in (1, 2))
    want = [x.run() for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(5):
        for st, x in zip(streams, (a, b)):
            with torch.cuda.stream(st):
                got.append(x.run())
    torch.cuda.synchronize()
    for i, (o, l) in enumerate(got):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(l, want[i % 2][1])


@pytest.mark.parametrize("cache,heads", [(P.BF16, 2), (P.FP8, 2), (P.BF16, 8)])
def test_a_cache_of_more_than_2_to_the_31_elements(cache, heads):
    hk, d, pages = 1, 128, (1 << 31) // (32 * 128) + 40
    c = P.RowCache.allocate(pages, hk, d, cache)
    g = torch.Generator(device="cuda").manual_seed(6)
    n, t = 70, 8
    table = torch.tensor([[pages - 1, 3, pages - 30]], dtype=torch.int32, device="cuda")
    k, v = (torch.randn(n, hk, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    i = torch.arange(n, device="cuda")
    c.write(k, v, (table[0].long()[i // 32] * 32 + i % 32).to(torch.int32))
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    K, V = c.read(table, lens, n)
    if cache == P.BF16:
        assert torch.equal(K[0, 0], k[:, 0]) and torch.equal(V[0, 0], v[:, 0])
    else:
        assert (K[0, 0].float() - k[:, 0].float()).abs().max().item() <= 2.0 ** -4 * k.float().abs().max().item()
    q = torch.randn(t, heads, d, generator=g, device="cuda").to(torch.bfloat16)
    out, _ = c.attend_tree(q, table, lens, torch.tensor([0, t], dtype=torch.int32, device="cuda"), t)
    small = P.RowCache.allocate(3, hk, d, cache)
    near = torch.arange(3, dtype=torch.int32, device="cuda")[None]
    small.write(k, v, i.to(torch.int32))
    want, _ = small.attend_tree(q, near, lens, torch.tensor([0, t], dtype=torch.int32, device="cuda"), t)
    assert torch.equal(out, want) and c.get_status() == 0


def test_first_call_of_a_process_under_capture():
    code = ("import torch, sys; sys.path.insert(0, %r); import paper_2511_07427_b200 as P\n"
            "i = dict(dtype=torch.int32, device='cuda')\n"
            "for cache, heads in ((P.BF16, 4), (P.FP8, 8), (P.BF16, 8)):\n"
            "    c = P.RowCache.allocate(3, 1, 128, cache)\n"
            "    x = torch.ones(80, 1, 128, dtype=torch.bfloat16, device='cuda'); s = torch.arange(80, **i)\n"
            "    q = torch.ones(16, heads, 128, dtype=torch.bfloat16, device='cuda'); t = torch.arange(3, **i)[None]; n = torch.tensor([80], **i); b = torch.tensor([0, 16], **i)\n"
            "    g = torch.cuda.CUDAGraph()\n"
            "    with torch.cuda.graph(g):\n"
            "        c.write(x, x, s); o, l = c.attend_tree(q, t, n, b, 16); k, v = c.read(t, n, 80)\n"
            "    g.replay(); torch.cuda.synchronize()\n"
            "    assert bool((o == 1).all()) and bool((k == 1).all()) and c.get_status() == 0\n") % os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_bad_pages_lengths_and_token_ranges_are_skipped_and_reported():
    p = Problem([100], [2], 4, 2, 128, "bf16")
    p.check(*p.run())
    good = p.table.clone()
    p.table[0, 1] = 1 << 30
    out, lse = p.run()
    assert p.c.get_status() == P.ST_BOUNDS and bool(torch.isfinite(out).all())
    # what a missing page holds is not seen: the same as a cache without those 32 rows
    q = Problem([68], [2], 4, 2, 128, "bf16")
    q.table = good[:, [0, 2, 3]].contiguous()
    q.c, q.q, q.kv_len = P.RowCache(p.c.k, p.c.v), p.q, torch.tensor([68], dtype=torch.int32, device="cuda")
    q.check(out, lse)
    for kw in (dict(kv_len=[1000]), dict(kv_len=[-3]), dict(q_start=[0, 5]), dict(q_start=[1, 0]), dict(q_start=[-1, 1]), dict(q_start=[1, 3])):
        c = P.RowCache(p.c.k, p.c.v)
        args = dict(kv_len=[100], q_start=[0, 2])
        args.update(kw)
        out, lse = c.attend_tree(p.q, good, torch.tensor(args["kv_len"], dtype=torch.int32, device="cuda"), torch.tensor(args["q_start"], dtype=torch.int32, device="cuda"), 2,
                                 out=torch.zeros_like(p.q))
        assert c.get_status() == P.ST_BOUNDS, kw


@pytest.mark.parametrize("cache,heads,d,drafts", [("fp8", 4, 128, 1), ("fp8", 4, 64, 1), ("fp8", 4, 128, 9), ("fp8", 8, 128, 40), ("f32", 4, 64, 1), ("bf16", 8, 128, 40)])
def test_missing_pages_in_a_long_table(cache, heads, d, drafts):
    p = Problem([3000], [drafts], heads, 2, d, cache, seed=21)
    good, gone = p.table.clone(), [1, 5, 6, 40, 90]
    for i, x in zip(gone, (1 << 30, -1, -(1 << 31), p.c.k.shape[0], 1 << 30)):
        p.table[0, i] = x
    out, lse = p.run()
    assert p.c.get_status() == P.ST_BOUNDS
    q = Problem([3000 - 32 * len(gone)], [drafts], heads, 2, d, cache, seed=21)
    q.table = good[:, [i for i in range(good.shape[1]) if i not in gone]].contiguous()
    q.c, q.q = P.RowCache(p.c.k, p.c.v, p.c.k_exp, p.c.v_exp), p.q         # the same rows, a status of its own
    q.check(out, lse)


def test_refusals():
    p = Problem([50], [3], 4, 2, 128, "bf16")
    i32 = dict(dtype=torch.int32, device="cuda")
    E = P.DynaKVError
    ok = dict(q=p.q, page_table=p.table, kv_len=p.kv_len, q_start=p.q_start, max_tree=3, tree_mask=None)
    p.c.attend_tree(**ok)
    for bad in (dict(q=p.q.float()), dict(q=p.q[:, :3].contiguous()), dict(q=p.q.transpose(0, 1)), dict(q=p.q[..., :64].contiguous()), dict(q=p.q.cpu()),
                dict(q=torch.zeros(3, 18, 128, dtype=torch.bfloat16, device="cuda")), dict(max_tree=0), dict(max_tree=257), dict(page_table=p.table[0]),
                dict(page_table=p.table.long()), dict(kv_len=torch.zeros(2, **i32)), dict(q_start=torch.zeros(1, **i32)), dict(scale=float("nan")),
                dict(tree_mask=torch.zeros(3, 5, dtype=torch.int64, device="cuda")), dict(tree_mask=torch.zeros(3, 1, **i32)),
                dict(tree_mask=torch.zeros(2, 1, dtype=torch.int64, device="cuda")), dict(out=torch.zeros(3, 4, 128, device="cuda")),
                dict(q=p.q.clone().requires_grad_())):
        with pytest.raises(E):
            p.c.attend_tree(**{**ok, **bad})
    out, lse = p.c.attend_tree(p.q[:0], p.table, p.kv_len, torch.zeros(2, **i32), 3)
    assert out.shape == (0, 4, 128) and lse.shape == (0, 4)


@pytest.mark.parametrize("cache", [P.F32, P.BF16, P.FP8])
def test_a_run_as_used(cache):
    """Prompt into the cache, one decode step over it, its rows read back for an index, and the index's own decode step: the
    dense attention and the retrieval with a budget that covers everything answer alike."""
    B, hk, group, d, n = 2, 2, 4, 128, 300
    g = torch.Generator(device="cuda").manual_seed(1)
    io = torch.float32 if cache == P.F32 else torch.bfloat16
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ro = P.HeadRotary(hk * group, hk, d, (10000.0 ** (-torch.arange(0, d, 2, device="cuda") / d)).float(),
                          q_weight=torch.ones(d, device="cuda"), k_weight=torch.ones(d, device="cuda"))
        c = P.RowCache.allocate(B * 10 + 1, hk, d, cache)
        table = torch.randperm(B * 10 + 1, generator=g, device="cuda")[:B * 10].view(B, 10).to(torch.int32)
        x = torch.randn(B, n, hk * group + 2 * hk, d, generator=g, device="cuda").to(io)
        i = torch.arange(n, device="cuda")
        for b in range(B):
            slots = (table[b].long()[i // 32] * 32 + i % 32).to(torch.int32)
            q = ro.store(x[b, :, :hk * group], x[b, :, hk * group:hk * group + hk], x[b, :, hk * group + hk:], i.to(torch.int32), c, slots, q_dtype=io)
            x[b, -1, :hk * group] = q[-1]                    # the query of the newest token
        newest = x[:, -1, :hk * group].contiguous()
        lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
        out, _ = c.attend_tree(newest, table, lens, torch.arange(B + 1, dtype=torch.int32, device="cuda"), 1)
        K, V = c.read(table, lens, n)
        index = P.DynaKV(P.DynaKVConfig(n_units=B * hk, gqa_group=group, head_dim=d, kv_dtype=cache, max_tokens=n + 8, max_clusters=16, kmeans_iters=2))
        index.build_index(K.view(B * hk, n, d), V.view(B * hk, n, d), 8, 1)
        want = index.decode_step(newest.float().view(B * hk, group, d), 10 ** 9)
    side.synchronize()
    assert c.get_status() == 0
    got, want = out.float().view(B * hk, group, d), want
    assert (got - want).abs().max().item() <= 2e-3 + (torch.finfo(io).eps / 2) * want.abs().max().item()     # the attention tolerance of the parity tests
    index.destroy()
