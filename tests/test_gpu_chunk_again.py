"""Chunk attention over rows of V that hold no numbers, or numbers near the end of fp32: who does not see them has the results of the
other rows, in sequences long enough that taking rows again costs more than any wait inside a kernel allows, and no other unit is touched.

What is compared with the 64-bit reference goes by the tolerances of test_gpu_chunk (through the check of test_gpu_chunk_strict)."""
import math

import pytest
import torch

import paper_2511_07427_b200 as P
from test_gpu_chunk_strict import Strict

pytestmark = pytest.mark.gpu
TYPES = ["f32", "bf16", "fp8"]


def spoil(p, b, h, place, value=math.nan, columns=None):
    """Columns of the row of V at `place` of sequence b and KV head h become `value` (FP8: the byte of NaN); returns what undoes it."""
    page, row = int(p.table[b, place // 32]), place % 32
    v = p.c.v.view(torch.uint8) if p.cache == "fp8" else p.c.v
    at = (page, h, row) if columns is None else (page, h, row, columns)
    old = v[at].clone()
    v[at] = 0x7f if p.cache == "fp8" else value

    def undo(keep=0):
        v[at] = old if keep is None else keep
    return undo


def compare(p, spoilt, **kw):
    """The run with the rows spoilt against the same with zeros in their places: where a token sees one, its columns are NaN; all else
    goes by the 64-bit reference, and what has nothing to do with the sequence and KV head keeps its bits.  spoilt: (sequence, KV head, place, columns)."""
    group = p.heads // p.hk
    undo = [spoil(p, b, h, at, columns=c) for b, h, at, c in spoilt]
    out, lse = p.run(**kw)
    torch.cuda.synchronize()
    assert p.c.get_status() == 0
    for u in undo:
        u()
    clean, clean_lse = p.run(**kw)
    mend = out.clone()
    touched = torch.zeros(p.n, p.heads, dtype=torch.bool, device="cuda")
    window = kw.get("window", 0)
    starts = p.q_start.tolist()
    for b, h, at, c in spoilt:
        mine = slice(starts[b], starts[b + 1])
        low = torch.maximum(p.low[mine], p.place[mine] + 1 - window) if window else p.low[mine]
        sees = (low <= at) & (at < p.high[mine]) & (at < p.lens[b])
        touched[mine, h * group:(h + 1) * group] = True
        cols = torch.arange(p.d, device="cuda") if c is None else torch.tensor(c, device="cuda").view(-1)
        for hq in range(h * group, (h + 1) * group):
            rows = torch.arange(p.n, device="cuda")[mine][sees]
            got = out[rows[:, None], hq, cols[None]]
            assert torch.isnan(got).all(), (b, h, at, hq)
            mend[rows[:, None], hq, cols[None]] = clean[rows[:, None], hq, cols[None]]
    p.check(mend, lse, **kw)
    assert torch.equal(out[~touched], clean[~touched]) and torch.equal(lse, clean_lse)
    return out


@pytest.mark.parametrize("cache", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 3, 9, 150])
def test_short_sequences(cache, d, new):
    p = Strict([400, 333], [new, new], 8, 2, d, cache, seed=1)
    compare(p, [(0, 1, 400 - new // 2 - 1, [d - 1])])
    compare(p, [(0, 1, 400 - 1, None), (1, 0, 5, [0, 3, 17])])
    p.see(low=lambda b, place, n: torch.full_like(place, 20))
    compare(p, [(0, 0, 19, None), (0, 1, 3, [7]), (1, 1, 20, [8])])


@pytest.mark.parametrize("cache", TYPES)
@pytest.mark.parametrize("new", [4, 200])
@pytest.mark.parametrize("kind", ["window", "documents", "prefix", "cap", "biases"])
def test_masks_and_scores(cache, new, kind):
    p = Strict([900, 500], [new, new], 8, 4, 128, cache, seed=2)
    kw = {}
    if kind == "window":
        kw = dict(window=77)
    if kind == "documents":
        p.see(low=lambda b, place, n: place // 61 * 61)
    if kind == "prefix":
        p.see(high=lambda b, place, n: (place + 1).clamp(min=n - 20))
    if kind == "cap":
        kw = dict(softcap=7.0)
    if kind == "biases":
        p.slopes = torch.tensor([2.0 ** -i for i in range(8)], device="cuda")
    compare(p, [(0, 0, 900 - new // 2, [5]), (0, 3, 900 - 60, None), (0, 2, 100, [1, 2]), (1, 1, 499, [127]), (1, 1, 470, [126])], **kw)


@pytest.mark.parametrize("cache", TYPES)
@pytest.mark.parametrize("kv,new", [(131000, 1), (40000, 4), (40000, 8), (100000, 100), (24000, 1000)])
def test_one_long_sequence_leaves_the_others(cache, kv, new):
    """In all columns of a long sequence's rows: every unit of a KV head is taken again.  The other sequences keep their bits."""
    lens = [kv, 700, 5, 3000]
    p = Strict(lens, [min(new, n) for n in lens], 4, 2, 128, cache, seed=3)
    compare(p, [(0, 1, kv - 1, None), (0, 1, kv - 2, None), (0, 1, kv - new // 2 - 1, None)])


@pytest.mark.parametrize("cache", TYPES)
@pytest.mark.parametrize("new", [2, 160])
def test_all_rows_of_a_sequence(cache, new):
    p = Strict([20000, 900], [new, new], 8, 2, 64, cache, seed=4)
    want, want_lse = p.run()
    pages = p.table[0].long()[:625]
    p.c.v.view(torch.uint8)[pages] = 0x7f if cache == "fp8" else 0xff
    out, lse = p.run()
    assert p.c.get_status() == 0
    assert torch.isnan(out[:new]).all() and torch.equal(out[new:], want[new:]) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("cache", TYPES)
@pytest.mark.parametrize("new", [2, 160])
def test_queries_and_seen_keys_that_hold_no_numbers(cache, new):
    p = Strict([9000, 900], [new, new], 8, 2, 128, cache, seed=5)
    want, want_lse = p.run()
    p.q[1, 5, 17] = math.nan
    out, lse = p.run()
    assert torch.isnan(out[1, 5]).all() and torch.isnan(lse[1, 5])
    out[1, 5], lse[1, 5] = want[1, 5], want_lse[1, 5]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    p.q[1, 5, 17] = 0.5
    want, want_lse = p.run()
    page = int(p.table[0, 0])
    k = p.c.k.view(torch.uint8) if cache == "fp8" else p.c.k
    k[page, 1, 3, 9] = 0x7f if cache == "fp8" else math.nan
    out, lse = p.run()
    assert p.c.get_status() == 0
    assert torch.isnan(out[:new, 4:]).all() and torch.isnan(lse[:new, 4:]).all()
    assert torch.equal(out[:new, :4], want[:new, :4]) and torch.equal(out[new:], want[new:]) and torch.equal(lse[new:], want_lse[new:])


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("new", [2, 160])
def test_infinities(cache, new):
    """One that a token sees makes its column infinite; two of opposite signs make it NaN; unseen ones do nothing."""
    p = Strict([5000], [new], 8, 2, 128, cache, seed=6)
    p.see(low=lambda b, place, n: torch.full_like(place, 40))
    undo = [spoil(p, 0, 0, 4000, math.inf, [3, 4]), spoil(p, 0, 0, 100, -math.inf, [4, 5]), spoil(p, 0, 0, 39, math.inf, [6])]
    out, lse = p.run()
    assert p.c.get_status() == 0
    mine = out[:, :4].float()
    assert bool((mine[:, :, 3] == math.inf).all()) and torch.isnan(mine[:, :, 4]).all() and bool((mine[:, :, 5] == -math.inf).all())
    for u in undo:
        u()
    clean, _ = p.run()
    out[:, :4, 3:6] = clean[:, :4, 3:6]
    p.check(out, lse)


@pytest.mark.parametrize("cache", TYPES)
@pytest.mark.parametrize("new", [3, 200])
def test_under_a_graph_and_again(cache, new):
    p = Strict([3000, 400], [new, new], 8, 2, 64, cache, seed=7)
    clean = p.run()
    undo = spoil(p, 0, 1, 3000 - 1, columns=[9])
    want = p.run()
    undo(None)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        out, lse = p.run()
    for spoilt in (False, True, False, True):
        undo = spoil(p, 0, 1, 3000 - 1, columns=[9]) if spoilt else (lambda keep: None)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((out, lse), want if spoilt else clean):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        undo(None)


def test_a_long_prompt_is_slow_but_comes_to_an_end():
    """16384 tokens of one prompt, one row of V with a NaN in each of 2 KV heads: what does not see it is taken again, the rest is NaN as it stands."""
    p = Strict([16384, 64], [16384, 64], 8, 2, 128, "bf16", seed=8)
    clean, clean_lse = p.run()
    undo = [spoil(p, 0, 0, 9001, columns=[5]), spoil(p, 0, 1, 16383)]
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    out, lse = p.run()
    end.record()
    torch.cuda.synchronize()
    assert p.c.get_status() == 0 and begin.elapsed_time(end) < 2000
    assert torch.isnan(out[9001:16384, :4, 5]).all() and torch.isnan(out[16383, 4:]).all()
    out[9001:16384, :4, 5], out[16383, 4:] = clean[9001:16384, :4, 5], clean[16383, 4:]
    assert torch.equal(lse, clean_lse) and torch.equal(out[16384:], clean[16384:])
    away = (out.float() - clean.float()).abs()                   # rows taken again differ by how weights are rounded, 2^-8, and two roundings of results
    assert bool((away <= 2.0 ** -6 * clean.float().abs() + 2.0 ** -6).all())
    for u in undo:
        u()


@pytest.mark.parametrize("cache", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new", [([5000, 300], [1, 1]), ([5000, 300], [3, 3]), ([3000, 300], [8, 2]), ([5000, 300], [200, 100]), ([900, 40, 9000], [900, 40, 30])])
def test_values_near_the_end_of_fp32(cache, d, lens, new):
    """V of one sign around 2^120: the sum of the weighted rows leaves fp32, the weighted mean does not."""
    p = Strict(lens, new, 8, 2, d, cache, seed=9)
    if cache == "fp8":
        p.c.v.view(torch.uint8).bitwise_and_(0x7f)
        p.c.v_exp += 118                                          # about 2^-8 for these rows
    else:
        p.c.v.abs_().mul_(2.0 ** 120)
    p.check(*p.run())
    p.check(*p.run(window=500), window=500)
    p.check(*p.run(softcap=3.0), softcap=3.0)


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("new", [3, 300])
@pytest.mark.parametrize("kind", ["causal", "documents", "weights of nothing"])
def test_which_of_them_a_token_sees(cache, new, kind):
    """NaN and infinities of both signs in one column, at several rows: the column is what the token sees of them makes it.  Slopes of 30 and 1000 make
    weights of e^-1000 and less, which are 0 in fp32, and 0 times infinity is NaN: there a column with an infinity may be either."""
    p = Strict([2000], [new], 4, 2, 64, cache, seed=10)
    if kind == "documents":
        p.see(low=lambda b, place, n: place // 50 * 50, high=lambda b, place, n: (place // 50 * 50 + 50).clamp(max=n))
    if kind == "weights of nothing":
        p.slopes = torch.tensor([1.0, 4.0, 30.0, 1000.0], device="cuda")
    marks = [(2000 - new + x * (new - 1) // 12, 11 + x % 3, v) for x, v in enumerate([math.inf, math.inf, math.inf, math.nan, -math.inf, math.inf, math.inf, -math.inf, math.nan, math.inf, math.inf, -math.inf, math.nan])]
    marks += [(1000, 20, math.inf), (1500, 20, math.inf), (1100, 21, -math.inf), (900, 22, math.nan), (1600, 22, math.inf)]
    undo = [spoil(p, 0, 1, at, v, [c]) for at, c, v in marks]
    out, lse = p.run()
    assert p.c.get_status() == 0
    held = {}
    for at, c, v in marks:                                        # the last one written is what a place holds
        held[at, c] = v
    want = torch.zeros(new, 64, dtype=torch.float64, device="cuda")
    for (at, c), v in held.items():
        want[:, c] += torch.where((p.low <= at) & (at < p.high), v, 0.0)
    odd = want != 0                                               # NaN != 0 too
    got = out[:, 2:].double()
    for h in range(2):
        x = got[:, h]
        nothing = kind == "weights of nothing"
        assert bool(((x == want) | (x.isnan() & (want.isnan() | nothing)))[odd].all()) and bool(torch.isfinite(x[~odd]).all())
    for u in reversed(undo):
        u()
    clean, _ = p.run()
    out[:, 2:] = torch.where(odd[:, None], clean[:, 2:], out[:, 2:])
    p.check(out, lse)


@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_a_long_prompt_over_one_odd_row(what):
    """32768 tokens that nearly all see one row with such a value, in a few of its columns: no query row but those around it is taken again."""
    p = Strict([32768], [32768], 4, 1, 128, "bf16", seed=11)
    clean, clean_lse = p.run()
    spoil(p, 0, 0, 70, what, [5, 6])
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    out, lse = p.run()
    end.record()
    torch.cuda.synchronize()
    assert p.c.get_status() == 0 and begin.elapsed_time(end) < 400
    seen = out[70:, :, 5:7].float()
    assert bool((seen.isnan() if math.isnan(what) else seen == what).all()) and torch.equal(lse, clean_lse)
    out[70:, :, 5:7] = clean[70:, :, 5:7]
    assert bool(((out.float() - clean.float()).abs() <= 2.0 ** -6 * clean.float().abs() + 2.0 ** -6).all())
