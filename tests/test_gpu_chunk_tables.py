"""Chunk attention and the width of its page table."""
import math

import pytest
import torch

import paper_2511_07427_b200 as P
from test_gpu_chunk_strict import Strict

KV = {"f32": P.F32, "bf16": P.BF16, "fp8": P.FP8}


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("most", [1, 20, 200, 4000])
def test_a_table_of_no_pages(cache, d, most):
    """Every kernel, and FP8 rows that would be turned into bf16 first: tokens that see nothing get zeros and -infinity."""
    c = P.RowCache.allocate(3, 2, d, KV[cache])
    io = torch.float32 if cache == "f32" else torch.bfloat16
    for new in ([most], [most, 0, 1], [0, 0]):
        n = sum(new)
        q = torch.randn(n + 3, 8, d, device="cuda").to(io)
        start = torch.tensor([0] + [sum(new[:i + 1]) for i in range(len(new))], dtype=torch.int32, device="cuda")
        table, lens = torch.zeros(len(new), 0, dtype=torch.int32, device="cuda"), torch.zeros(len(new), dtype=torch.int32, device="cuda")
        out, lse = torch.full_like(q, 7.0), torch.full((n + 3, 8), 9.0, device="cuda")
        c.attend_chunk(q, table, lens, start, most, out=out, lse=lse)
        assert c.get_status() == 0
        assert not out[:n].any() and bool((lse[:n] == -math.inf).all()) and bool((out[n:] == 7.0).all()) and bool((lse[n:] == 9.0).all())


def wide_table(table, columns):
    """The table with so many columns, the new ones naming nothing."""
    more = torch.full((table.shape[0], columns - table.shape[1]), 1 << 30, dtype=torch.int32, device="cuda")
    return torch.cat([table, more], 1).contiguous()


@pytest.mark.gpu
@pytest.mark.parametrize("d,hk", [(64, 4), (128, 2)])
@pytest.mark.parametrize("kind", ["causal", "window", "documents", "prefix"])
def test_long_chunks_over_fp8_rows_and_wide_tables(d, hk, kind):
    """Tables made for long sequences change no bit of the results of short ones, and scratch goes by the cache's pages."""
    p = Strict([900, 2000, 130, 0, 700], [900, 700, 130, 0, 300], 4 * hk, hk, d, "fp8", seed=31)
    kw = dict(window=150) if kind == "window" else {}
    if kind == "documents":
        p.see(low=lambda b, place, n: place // 200 * 200)
    if kind == "prefix":
        p.see(high=lambda b, place, n: (place + 1).clamp(min=n // 3))
    want = p.run(**kw)
    p.check(*want, **kw)
    narrow = p.table
    for columns in (narrow.shape[1] + 1, 5000):
        p.table = wide_table(narrow, columns)
        got = p.run(**kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and p.c.get_status() == 0
        size = p.c._workspace[4 * hk, p.most, p.n, 5, columns]
        assert size < (100 << 20) + p.c.n_pages * hk * 32 * d * 4


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_pages_that_many_sequences_share(d):
    """More pages in the tables than in the cache: rows are turned into bf16 as they are read, with the same results."""
    p = Strict([1500, 1500, 1500, 200], [700, 700, 650, 200], 8, 2, d, "fp8", seed=32)
    p.table[1, :47], p.table[2, :47] = p.table[0, :47], p.table[0, :47]
    want = p.run()
    p.check(*want)
    # a cache of the pages that are used and no more: the tables' pages are three times as many
    used = torch.unique(torch.cat([p.table[0, :47], p.table[3, :7]])).long()
    place = torch.full((p.c.n_pages,), 1 << 30, dtype=torch.int32, device="cuda")
    place[used] = torch.arange(len(used), dtype=torch.int32, device="cuda")
    small = P.RowCache(p.c.k[used].contiguous(), p.c.v[used].contiguous(), p.c.k_exp[used].contiguous(), p.c.v_exp[used].contiguous())
    table = torch.where(p.table < p.c.n_pages, place[p.table.clamp(max=p.c.n_pages - 1).long()], 1 << 30).to(torch.int32)
    p.c, p.table = small, wide_table(table, 2000)
    for _ in range(2):
        got = p.run()
        p.check(*got)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
def test_wide_tables_under_a_graph():
    """One graph, lengths that change: pages that are turned into bf16 find room, then none, then room again."""
    p = Strict([600, 600], [600, 600], 8, 2, 128, "fp8", seed=34)
    p.table[1, :19] = p.table[0, :19]
    keep = p.table[0, :19].long()
    small = P.RowCache(*[t[keep].contiguous() for t in (p.c.k, p.c.v, p.c.k_exp, p.c.v_exp)])
    p.c = small
    p.table = wide_table(torch.arange(19, dtype=torch.int32, device="cuda").repeat(2, 1), 40)
    full = p.kv_len.clone(), p.q_start.clone()
    less = torch.tensor([600, 0], dtype=torch.int32, device="cuda"), torch.tensor([0, 600, 600], dtype=torch.int32, device="cuda")
    p.run()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        out, lse = p.run()
    for lens, starts in (full, less, full, less):
        p.kv_len.copy_(lens)
        p.q_start.copy_(starts)
        p.lens, p.new = lens.tolist(), (starts[1:] - starts[:-1]).tolist()
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        p.check(out, lse)
