"""Chunk attention with more tiles than the planning launch keeps in shared memory, and the C entry without lse."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2511_07427_b200 as P
from paper_2511_07427_b200 import rows as R
from test_gpu_chunk_strict import Strict

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("kind", ["causal", "window", "documents"])
def test_thousands_of_tiles(cache, kind):
    """5000 short sequences and one long: more than 4096 tiles of 64 or 128 query rows."""
    rng = np.random.default_rng(2)
    lens = [int(x) for x in rng.integers(0, 70, 5000)]
    lens[2500] = 6000
    new = [int(min(n, rng.integers(0, 50))) for n in lens]
    new[2500] = 4000
    p = Strict(lens, new, 2, 1, 64, cache, seed=41)
    kw = dict(window=33) if kind == "window" else {}
    if kind == "documents":
        p.see(low=lambda b, place, n: place // 40 * 40, high=lambda b, place, n: (place // 40 * 40 + 40).clamp(max=n))
    out, lse = p.run(**kw)
    again = p.run(**kw)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1]) and torch.isfinite(out).all()
    starts = p.q_start.tolist()
    for b in [2500] + list(np.flatnonzero(np.array(new))[::250]):
        sub = Strict([lens[b]], [new[b]], 2, 1, 64, cache)
        sub.c, sub.table, sub.q = p.c, p.table[b:b + 1], p.q[starts[b]:starts[b + 1]]
        sub.low, sub.high = p.low[starts[b]:starts[b + 1]], p.high[starts[b]:starts[b + 1]]
        sub.most = p.most
        sub.check(out[starts[b]:starts[b + 1]], lse[starts[b]:starts[b + 1]], **kw)


@pytest.mark.parametrize("cache", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("new", [2, 200])
@pytest.mark.parametrize("spoilt", [False, True])
def test_the_c_entry_without_lse(cache, new, spoilt):
    p = Strict([3000, 400], [new, new], 8, 2, 128, cache, seed=42)
    if spoilt:
        v = p.c.v.view(torch.uint8) if cache == "fp8" else p.c.v
        v[int(p.table[0, 90]), 1, 7] = 0x7f if cache == "fp8" else math.nan
    p.see(low=lambda b, place, n: torch.where(torch.arange(len(place), device="cuda") % 2 == 0, 2890, 0) if n == 3000 else torch.zeros_like(place))
    want, _ = p.run()
    out = torch.full_like(p.q, 7.0)
    size = p.c._workspace[8, new, p.n, 2, p.table.shape[1]]
    space = torch.empty(size, dtype=torch.uint8, device="cuda")
    scores = R._Scores(128 ** -0.5, 0.0, 0, None, p.from_to["rows_from"].data_ptr(), None)
    rc = R._library().dynakv_attend_chunk(p.c._ref, p.q.data_ptr(), 8, p.n, p.q_start.data_ptr(), 2, new, p.table.data_ptr(), p.table.shape[1], p.kv_len.data_ptr(),
                                          C.byref(scores), out.data_ptr(), None, space.data_ptr(), size, None, torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    same = (out == want) | (out.isnan() & want.isnan())
    assert bool(same.all()) and bool(torch.isnan(out[new - 1, 4:]).all()) == spoilt             # row 2887, which the last token sees
