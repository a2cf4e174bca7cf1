"""Chunk attention and the width of its page table."""
import math

import pytest
import torch

import paper_2511_07427_b200 as P

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
