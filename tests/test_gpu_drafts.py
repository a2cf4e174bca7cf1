"""Pages and slots for new tokens, verification of drafted tokens, and rows of accepted drafts moved together, against plain
restatements.  All results are whole numbers or copied rows: they have to be equal."""
import math

import numpy as np
import pytest
import torch

import paper_2511_07427_b200 as P

pytestmark = pytest.mark.gpu
PAGE = 32


def ints(x):
    return torch.tensor(np.ascontiguousarray(x), dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------- pages

class Pages:
    """The pool and the tables as plain lists."""

    def __init__(self, n_pages, table, lens, seed):
        used = table[table >= 0].tolist()
        self.free = [int(x) for x in np.random.default_rng(seed).permutation(n_pages) if x not in set(used)]
        self.n_pages, self.table, self.lens = n_pages, table.copy(), lens.copy()

    def extend(self, add, room):
        per = self.table.shape[1]
        starts, places, slots, status, stop = [0], [], [], 0, False
        used_pages = used_tokens = 0
        for b, t in enumerate(int(x) for x in add):
            old = int(self.lens[b])
            valid = old >= 0 and t >= 0 and old + t <= per * PAGE
            if stop:
                starts.append(len(places))
                continue
            if not valid:
                status |= P.ST_BOUNDS
                starts.append(len(places))
                continue
            need = -(-(old + t) // PAGE) - -(-old // PAGE)
            if used_pages + need > len(self.free) + used_pages or used_tokens + t > room:
                status |= P.ST_PAGE_POOL if need > len(self.free) else P.ST_BOUNDS
                stop = True
                starts.append(len(places))
                continue
            for i in range(need):
                self.table[b, -(-old // PAGE) + i] = self.free.pop()
            used_pages += need
            used_tokens += t
            for r in range(old, old + t):
                places.append(r)
                slots.append(int(self.table[b, r // PAGE]) * PAGE + r % PAGE)
            self.lens[b] += t
            starts.append(len(places))
        pad = room - len(places)
        return starts, places + [0] * pad, slots + [-1] * pad, status

    def trim(self, drop):
        status, back = 0, []
        for b, t in enumerate(int(x) for x in drop):
            old = int(self.lens[b])
            if not (0 <= old <= self.table.shape[1] * PAGE and 0 <= t <= old):
                status |= P.ST_BOUNDS
                continue
            for column in range(-(-(old - t) // PAGE), -(-old // PAGE)):
                back.append(int(self.table[b, column]))
                self.table[b, column] = -1
            self.lens[b] -= t
        self.free += back[::-1]
        return status


def pool_for(ref):
    free = np.full(ref.n_pages, -1, np.int32)
    free[:len(ref.free)] = ref.free
    return P.PagePool(ints(free), ints([len(ref.free)]))


def same(pool, ref, table, lens):
    n = int(pool.count)
    assert n == len(ref.free) and pool.free[:n].tolist() == ref.free
    assert np.array_equal(table.cpu().numpy(), ref.table) and lens.tolist() == ref.lens.tolist()


@pytest.mark.parametrize("batch,per,most", [(1, 1, 1), (3, 4, 70), (64, 20, 1), (64, 20, 40), (700, 9, 100), (1024, 3, 33), (1025, 3, 33), (2500, 4, 60), (2, 600, 9000)])
def test_extend_and_trim(batch, per, most):
    rng = np.random.default_rng(batch + most)
    table, lens = np.full((batch, per), -1, np.int32), np.zeros(batch, np.int32)
    ref = Pages(batch * per + 7, table, lens, 1)
    pool, t, n = pool_for(ref), ints(table), ints(lens)
    for step in range(5):
        add = rng.integers(0, most + 1, batch)
        if step % 2:                                              # within bounds, or some of them not
            add = np.minimum(add, per * PAGE - ref.lens)
        room = int(np.maximum(add, 0).sum()) + int(rng.integers(0, 40))
        status = int(pool.get_status())
        starts, places, slots, want = ref.extend(add, room)
        got = pool.extend(t, n, ints(add), room)
        assert got[0].tolist() == starts and got[1].tolist() == places and got[2].tolist() == slots
        assert pool.get_status() == status | want
        same(pool, ref, t, n)
        drop = rng.integers(0, ref.lens + 1)
        ref.trim(drop)
        pool.trim(t, n, ints(drop))
        same(pool, ref, t, n)


@pytest.mark.parametrize("batch", [5, 1500])
def test_pages_or_places_that_run_out(batch):
    rng = np.random.default_rng(3)
    table, lens = np.full((batch, 8), -1, np.int32), np.zeros(batch, np.int32)
    for pages, places in ((batch, 10 ** 6), (8 * batch, 60 * batch), (1, 10 ** 6), (8 * batch, 0)):
        ref = Pages(pages, table, lens, 2)
        pool, t, n = pool_for(ref), ints(table), ints(lens)
        add = rng.integers(0, 200, batch)
        starts, where, slots, want = ref.extend(add, places if places < 10 ** 6 else int(add.sum()))
        got = pool.extend(t, n, ints(add), places if places < 10 ** 6 else int(add.sum()))
        assert want and pool.get_status() == want
        assert got[0].tolist() == starts and got[1].tolist() == where and got[2].tolist() == slots
        same(pool, ref, t, n)


def test_numbers_out_of_range_leave_their_sequences():
    ref = Pages(50, np.full((6, 4), -1, np.int32), np.array([0, -3, 10 ** 6, 128, 20, 0], np.int32), 4)
    pool, t, n = pool_for(ref), ints(ref.table), ints(ref.lens)
    add = [3, 2, 2, 1, -1, 40]
    starts, where, slots, want = ref.extend(add, 50)
    got = pool.extend(t, n, ints(add), 50)
    assert want == P.ST_BOUNDS == pool.get_status()
    assert got[0].tolist() == starts and got[1].tolist() == where and got[2].tolist() == slots
    same(pool, ref, t, n)
    ref.trim([4, 0, 0, 129, 21, 3])
    pool.trim(t, n, ints([4, 0, 0, 129, 21, 3]))
    same(pool, ref, t, n)
    # lengths as far as they go: sums of changes pass 32 bits
    m = 3000
    pool = P.PagePool.allocate(10)
    t, n = ints(np.full((m, 1), -1)), ints(np.zeros(m))
    got = pool.extend(t, n, ints(np.full(m, 2 ** 31 - 1)), 5)
    assert not got[0].any() and pool.get_status() == P.ST_BOUNDS and int(pool.count) == 10 and not n.any()
    pool.trim(t, n, ints(np.full(m, 2 ** 31 - 1)))
    assert int(pool.count) == 10 and not n.any()


def test_a_full_pool_takes_no_more_pages_back():
    pool = P.PagePool.allocate(4)
    t, n = ints([[0, 1], [2, 3]]), ints([64, 64])
    pool.trim(t, n, ints([64, 64]))
    assert pool.get_status() == P.ST_PAGE_POOL and int(pool.count) == 4 and n.tolist() == [64, 64]


def test_empty_calls_of_the_pool():
    pool = P.PagePool.allocate(4)
    got = pool.extend(ints(np.zeros((0, 3))), ints([]), ints([]), 5)
    assert got[0].tolist() == [0] and got[1].tolist() == [0] * 5 and got[2].tolist() == [-1] * 5
    got = pool.extend(ints(np.zeros((2, 0))), ints([0, 0]), ints([0, 0]), 0)
    assert got[0].tolist() == [0, 0, 0]
    pool.trim(ints(np.zeros((0, 3))), ints([]), ints([]))
    assert pool.get_status() == 0 and int(pool.count) == 4


def test_steps_of_a_captured_graph():
    batch, per = 40, 6
    ref = Pages(batch * per, np.full((batch, per), -1, np.int32), np.zeros(batch, np.int32), 5)
    pool, t, n, add = pool_for(ref), ints(ref.table), ints(ref.lens), ints(np.ones(batch))
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        got = pool.extend(t, n, add, batch)
    for step in range(100):
        graph.replay()
        want = ref.extend([1] * batch, batch)
    torch.cuda.synchronize()
    assert got[2].tolist() == want[2]
    same(pool, ref, t, n)


def test_refusals_of_the_pool():
    free, count = ints(np.arange(5)), ints([5])
    for bad in (dict(free=free.long()), dict(free=free.view(1, 5)), dict(free=free[:0]), dict(free=free.cpu()), dict(count=ints([5, 5])), dict(count=count.cpu()),
                dict(count=count.long())):
        with pytest.raises(P.DynaKVError):
            P.PagePool(**{**dict(free=free, count=count), **bad})
    pool = P.PagePool(free, count)
    ok = dict(page_table=ints(np.zeros((2, 3))), kv_len=ints([1, 2]), new_len=ints([1, 1]), n_tokens=2)
    for bad in (dict(page_table=ints([1])), dict(page_table=ok["page_table"].long()), dict(kv_len=ints([1])), dict(new_len=ints([1, 1]).cpu()), dict(n_tokens=-1),
                dict(n_tokens=1 << 31), dict(page_table=ints(np.zeros((3, 2))).T)):
        with pytest.raises(P.DynaKVError):
            pool.extend(**{**ok, **bad})
    with pytest.raises(P.DynaKVError, match="kv_len"):
        pool.trim(ok["page_table"], ok["kv_len"], ok["kv_len"])


# ------------------------------------------------------------------------------------------------- verification

def verified(logits, tokens, starts, most, uniform, heat, parent=None, draft=None):
    """The rule, one sequence and one draft after the other, in 64 bits."""
    logits, tokens, uniform, heat = (x.cpu().numpy() if x.dtype != torch.bfloat16 else x.float().cpu().numpy() for x in (logits, tokens, uniform, heat))
    draft = draft.cpu().numpy().astype(np.float64) if draft is not None else None
    kept, path, following = [], np.full((len(starts) - 1, most), -1), []
    vocab = logits.shape[1]

    def weights(row, t):
        x = logits[row].astype(np.float64)
        if not np.isfinite(x.max()):
            return np.zeros(vocab)
        if t <= 0:
            return (np.arange(vocab) == int(np.argmax(x))).astype(np.float64)
        return np.exp((x - x.max()) / np.float64(t))

    for b in range(len(starts) - 1):
        first, size = starts[b], starts[b + 1] - starts[b]
        if size == 0:
            kept.append(0)
            following.append(-1)
            continue
        at, walk = 0, [0]
        p = weights(first, heat[b])
        going = True
        while going:
            going = False
            for c in range(at + 1, size):
                up = int(parent[first + c]) if parent is not None else c - 1
                if up != at:
                    continue
                x = int(tokens[first + c])
                if not 0 <= x < vocab:
                    continue
                q = draft[first + c] if draft is not None else (np.arange(vocab) == x).astype(np.float64)
                if (p[x] > 0 and heat[b] <= 0) or (heat[b] > 0 and float(uniform[first + c]) * q[x] * p.sum() < p[x]):
                    at, going = c, True
                    walk.append(c)
                    p = weights(first + c, heat[b])
                    break
                if heat[b] > 0:
                    left = np.maximum(p / p.sum() - q, 0) if draft is not None else np.where(q > 0, 0, p)
                    p = left if left.sum() > 0 or draft is None else p
        runs = np.cumsum(p)
        chosen = int(np.searchsorted(runs, float(uniform[first]) * runs[-1], side="right")) if runs[-1] > 0 else -1
        following.append(min(chosen, int(np.flatnonzero(p)[-1])) if chosen >= 0 else -1)
        kept.append(len(walk))
        path[b, :len(walk)] = walk
    return kept, path, following


def drafts(sizes, vocab, dtype, shape, drawn, seed, spread=3.0, like=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    n = sum(sizes)
    starts = np.concatenate([[0], np.cumsum(sizes)])
    parent = None
    if shape == "tree":
        parent = np.concatenate([[-1] + [int(rng.integers(max(0, i - 5), i)) for i in range(1, t)] for t in sizes if t])
    logits = (spread * torch.randn(n, vocab, generator=g, device="cuda")).to(dtype)
    up = np.concatenate([np.arange(t) - 1 if parent is None else parent[s:s + t] for s, t in zip(starts, sizes) if t] or [np.zeros(0)]).clip(min=0).astype(np.int64)
    above = torch.tensor(up + np.repeat(starts[:-1], sizes), device="cuda")
    near = torch.softmax(logits[above].float() + like * torch.randn(n, vocab, generator=g, device="cuda"), -1)
    tokens = torch.multinomial(near, 1, generator=g)[:, 0].to(torch.int32) if n else ints([])
    return dict(logits=logits, tokens=tokens, q_start=ints(starts), max_tree=max(max(sizes), 1), uniform=torch.rand(n, generator=g, device="cuda"),
                parent=ints(parent) if parent is not None else None, draft_probs=near if drawn else None)


def compare(a, heat):
    got = P.verify_drafts(**a, temperature=heat)
    starts = a["q_start"].tolist()
    kept, path, following = verified(a["logits"], a["tokens"], starts, a["max_tree"], a["uniform"], heat, a["parent"].cpu() if a["parent"] is not None else None, a["draft_probs"])
    assert got[0].tolist() == kept
    assert got[1].tolist() == [t - k for t, k in zip(np.diff(starts).tolist(), kept)]
    assert np.array_equal(got[2].cpu().numpy(), path)
    assert got[3].tolist() == following
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 2, 7, 33, 1000, 4097, 20011, 70000])
@pytest.mark.parametrize("shape,drawn", [("chain", False), ("chain", True), ("tree", False)])
def test_verification(dtype, vocab, shape, drawn):
    sizes = [1, 5, 0, 8, 2, 13, 1, 6]
    a = drafts(sizes, vocab, dtype, shape, drawn, vocab)
    heat = torch.tensor([1.0, 0.0, 1.0, 0.6, 1.5, 1.0, 0.0, 4.0], device="cuda")
    compare(a, heat)


@pytest.mark.parametrize("batch", [1, 20, 300])
@pytest.mark.parametrize("shape,drawn", [("chain", True), ("tree", False)])
def test_batches(batch, shape, drawn):
    rng = np.random.default_rng(batch)
    a = drafts([int(x) for x in rng.integers(0, 9, batch)] + [3], 3001, torch.bfloat16, shape, drawn, batch)
    compare(a, torch.tensor(rng.choice([0.0, 0.5, 1.0], batch + 1), dtype=torch.float32, device="cuda"))


@pytest.mark.parametrize("batch,vocab", [(200, 9001), (1100, 37), (64, 20011)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape,drawn", [("chain", True), ("tree", False)])
def test_more_sequences_than_processors_and_long_slices(batch, vocab, dtype, shape, drawn):
    rng = np.random.default_rng(batch)
    a = drafts([int(x) for x in rng.integers(0, 4, batch)], vocab, dtype, shape, drawn, batch)
    compare(a, torch.tensor(rng.choice([0.0, 0.7, 1.0], batch), dtype=torch.float32, device="cuda"))


def test_wide_and_deep_trees():
    for width in (1, 255):                                        # a chain of 256; 255 drafts behind the root
        a = drafts([256], 500, torch.float32, "tree", False, 3, spread=1.0)
        a["parent"] = ints([-1] + [0 if width == 255 else i for i in range(255)])
        for seed in range(4):
            a["uniform"] = torch.rand(256, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * (1.0 if width == 255 else 0.01)
            compare(a, torch.tensor([1.0], device="cuda"))


def test_the_same_token_twice_and_tokens_that_are_none():
    logits = torch.log(torch.tensor([[0.5, 0.3, 0.2, 0.0]], device="cuda")).repeat(6, 1)
    base = dict(logits=logits, q_start=ints([0, 6]), max_tree=6, parent=ints([-1, 0, 0, 0, 0, 0]), draft_probs=None)
    for tokens in ([0, 0, 0, 1, 0, 1], [0, 3, 3, 3, 3, 3], [0, -1, 4, 10 ** 9, 1, 1], [0, 0, 1, 2, 3, 0]):
        for u in (0.0, 0.3, 0.55, 0.7, 0.999):
            a = dict(base, tokens=ints(tokens), uniform=torch.full((6,), u, device="cuda"))
            for heat in (1.0, 0.0):
                compare(a, torch.tensor([heat], device="cuda"))
    # a parent that is none: never reached
    a = dict(base, parent=ints([-1, -1, 2, 7, -9, 4]), tokens=ints([0] * 6), uniform=torch.zeros(6, device="cuda"))
    kept, dropped, path, _ = P.verify_drafts(**a, temperature=torch.ones(1, device="cuda"))
    assert kept.tolist() == [1] and dropped.tolist() == [5] and path.tolist() == [[0, -1, -1, -1, -1, -1]]


def test_masked_logits_and_the_ends_of_the_draw():
    vocab = 5000
    a = drafts([2, 3, 1, 1], vocab, torch.float32, "chain", False, 9)
    a["logits"][:, 100:4900] = -math.inf
    a["logits"][5] = -math.inf                                    # the last two sequences: nothing, one token
    a["logits"][6] = -math.inf
    a["logits"][6, 4321] = 3.0
    for u in (0.0, 2.0 ** -24, 0.5, 1 - 2.0 ** -24):
        a["uniform"] = torch.full((7,), u, device="cuda")
        got = compare(a, torch.ones(4, device="cuda"))
        assert got[3].tolist()[2:] == [-1, 4321]
        compare(a, torch.zeros(4, device="cuda"))
    # more than 1, which is not asked for: the last token that has a weight
    a["uniform"] = torch.full((7,), 1.5, device="cuda")
    got = P.verify_drafts(**a, temperature=torch.ones(4, device="cuda"))
    assert got[0].tolist() == [1, 1, 1, 1] and all(x == -1 or x >= 4900 or x == 4321 for x in got[3].tolist())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drawn", [False, True])
def test_temperatures_near_zero_and_without_end(dtype, drawn):
    vocab, n = 5000, 6
    a = drafts([4, 2], vocab, dtype, "chain", drawn, 21)
    a["logits"].clamp_(max=19.0)
    best = torch.tensor([7, 4999, 0, 2500, 1234, 4095], device="cuda")
    a["logits"][torch.arange(n, device="cuda"), best] = 20.0
    a["logits"][:, 3000:4000] = -math.inf
    a["tokens"][1:3] = best[:2].to(torch.int32)                   # the first two drafts are the largest, the third and the other sequence's are not
    a["tokens"][3] = a["tokens"][5] = 1
    a["uniform"] = torch.tensor([0.25, 0.5, 0.75, 0.3, 0.6, 0.9], device="cuda")
    for heat in (1e-6, 1e-9, 1e-12, 1e-30, 2.0 ** -126, 1e-44):
        got = P.verify_drafts(**a, temperature=torch.full((2,), heat, device="cuda"))
        assert got[0].tolist() == [3, 1] and got[3].tolist() == [0, 1234], heat
    # all that is not masked weighs the same: the draw counts through the 4000 tokens
    a["draft_probs"] = None
    a["tokens"][1] = a["tokens"][5] = 3500                        # masked: refused
    a["uniform"][0], a["uniform"][4] = (3100 + 0.5) / 4000, (1000 + 0.5) / 4000
    for heat in (2.0 ** 90, 2.0 ** 120, math.inf):
        got = P.verify_drafts(**a, temperature=torch.full((2,), heat, device="cuda"))
        assert got[0].tolist() == [1, 1] and got[3].tolist() == [4100, 1000], heat


def test_a_draft_that_covers_the_target():
    # equal logits, so that the target's probabilities are quarters exactly (those of ln 0.25 in fp32 are off by 2e-8, and 2e-8 would be left)
    p = torch.tensor([[0.25, 0.25, 0.25, 0.25, 0.0]] * 2, device="cuda")
    a = dict(logits=torch.where(p > 0, 0.0, -math.inf), tokens=ints([0, 4]), q_start=ints([0, 2]), max_tree=2, draft_probs=p.clone(), parent=None)
    for u in (0.1, 0.3, 0.6):                                     # token 4 has no chance and is refused; what is left is nothing, so p stays
        got = P.verify_drafts(**a, uniform=torch.full((2,), u, device="cuda"), temperature=torch.ones(1, device="cuda"))
        assert got[0].tolist() == [1] and got[3].tolist() == [int(4 * u)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_odd_addresses(dtype):
    a = drafts([4, 5], 1001, dtype, "chain", True, 11)
    wide = torch.zeros(9, 1311, dtype=dtype, device="cuda")
    odd = torch.zeros(9, 1201, device="cuda")
    for first in (0, 1, 3, 6):
        wide[:, first:first + 1001] = a["logits"]
        odd[:, first:first + 1001] = a["draft_probs"]
        compare(dict(a, logits=wide[:, first:first + 1001], draft_probs=odd[:, first:first + 1001]), torch.tensor([1.0, 0.7], device="cuda"))


def test_ranges_of_tokens_that_are_none():
    a = drafts([3, 3, 3], 50, torch.float32, "chain", False, 12)
    good = P.verify_drafts(**a, temperature=torch.ones(3, device="cuda"))
    for starts, bad in (([-2, 3, 6, 9], 0), ([0, 3, 6, 10], 2), ([4, 3, 6, 9], 0), ([0, 3, 6, 2 ** 31 - 1], 2)):
        got = P.verify_drafts(**{**a, "q_start": ints(starts)}, temperature=torch.ones(3, device="cuda"))
        assert got[0][bad] == 0 and got[1][bad] == -1 and got[3][bad] == -1 and bool((got[2][bad] == -1).all())
        for b in range(3):
            if b != bad and starts[b:b + 2] == [3 * b, 3 * b + 3]:
                assert all(torch.equal(x[b], y[b]) for x, y in zip(got, good))
    got = P.verify_drafts(**{**a, "max_tree": 2}, temperature=torch.ones(3, device="cuda"))
    assert got[0].tolist() == [0, 0, 0] and got[1].tolist() == [-1] * 3
    empty = P.verify_drafts(a["logits"][:0], a["tokens"][:0], ints([0, 0]), 4, a["uniform"][:0], torch.ones(1, device="cuda"))
    assert empty[0].tolist() == [0] and empty[1].tolist() == [0] and empty[3].tolist() == [-1]
    assert P.verify_drafts(a["logits"][:0], a["tokens"][:0], ints([0]), 4, a["uniform"][:0], torch.ones(0, device="cuda"))[2].shape == (0, 4)


@pytest.mark.parametrize("drawn", [True, False])
def test_kept_tokens_are_distributed_as_the_target_s(drawn):
    """A chain of one draft, 60000 times: the first new token has the target's distribution whatever drafted it, the one behind an accepted
    draft that of its row.  Counts of n draws are off by less than 5.5 standard deviations (7 tokens, twice: a chance of 1e-6)."""
    n, vocab = 60000, 7
    g = torch.Generator(device="cuda").manual_seed(1)
    two = torch.randn(2, vocab, generator=g, device="cuda") * 1.5
    p = torch.softmax(two.double() / 0.8, -1).cpu().numpy()
    q = torch.softmax(torch.randn(vocab, generator=g, device="cuda"), -1)
    tokens = torch.zeros(n, 2, dtype=torch.int32, device="cuda")
    tokens[:, 1] = torch.multinomial(q, n, replacement=True, generator=g).to(torch.int32) if drawn else int(p[0].argmax())      # likely enough to be accepted often
    kept, _, _, following = P.verify_drafts(two.repeat(n, 1), tokens.view(-1), ints(2 * np.arange(n + 1)), 2, torch.rand(2 * n, generator=g, device="cuda"),
                                            torch.full((n,), 0.8, device="cuda"), draft_probs=q.repeat(2 * n, 1) if drawn else None)
    first = torch.where(kept == 2, tokens[:, 1], following).cpu().numpy()
    second = following[kept == 2].cpu().numpy()
    assert len(second) > 2000
    for got, want in ((first, p[0]), (second, p[1])):
        counts, m = np.bincount(got, minlength=vocab), len(got)
        assert (np.abs(counts - m * want) <= 5.5 * np.sqrt(m * want * (1 - want)) + 1).all(), (counts / m, want)


def test_verification_under_a_graph_and_on_two_streams():
    problems = [(drafts([6] * 8, 9001, torch.bfloat16, "chain", True, s), torch.full((8,), 0.9, device="cuda")) for s in (1, 2)]
    want = [P.verify_drafts(**a, temperature=h) for a, h in problems]
    streams, graphs, got = [torch.cuda.Stream() for _ in problems], [torch.cuda.CUDAGraph() for _ in problems], [None, None]
    torch.cuda.synchronize()
    for i, (a, h) in enumerate(problems):
        with torch.cuda.stream(streams[i]), torch.cuda.graph(graphs[i], stream=streams[i]):
            got[i] = P.verify_drafts(**a, temperature=h)
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
                P.verify_drafts(**problems[i][0], temperature=problems[i][1])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for w, r in zip(want, got) for x, y in zip(w, r))


def test_refusals_of_the_verification():
    a = drafts([3, 3], 50, torch.float32, "chain", True, 13)
    a["temperature"] = torch.ones(2, device="cuda")
    L, D = a["logits"], a["draft_probs"]
    for bad in (dict(logits=L[0]), dict(logits=L.double()), dict(logits=L.T), dict(logits=L.cpu()), dict(tokens=a["tokens"].long()), dict(tokens=a["tokens"][:5]),
                dict(q_start=a["q_start"].long()), dict(q_start=a["q_start"].view(1, 3)), dict(max_tree=0), dict(max_tree=257), dict(uniform=a["uniform"].double()),
                dict(uniform=a["uniform"][:5]), dict(temperature=torch.ones(3, device="cuda")), dict(temperature=torch.ones(2)), dict(parent=ints([0] * 6)),
                dict(parent=ints([0] * 5), draft_probs=None), dict(draft_probs=D.bfloat16()), dict(draft_probs=D[:, :49]), dict(draft_probs=D.cpu()),
                dict(logits=L.clone().requires_grad_()), dict(draft_probs=D.clone().requires_grad_()), dict(uniform=a["uniform"].clone().requires_grad_())):
        with pytest.raises(P.DynaKVError):
            P.verify_drafts(**{**a, **bad})
    with torch.no_grad():
        P.verify_drafts(**{**a, "logits": L.clone().requires_grad_()})


# ------------------------------------------------------------------------------------------------- rows of accepted drafts

@pytest.mark.parametrize("cache", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,trees", [([1], [1]), ([40, 300, 7, 0], [9, 256, 7, 0]), ([64, 65, 33], [33, 32, 31])])
def test_kept_rows(cache, d, lens, trees):
    rng = np.random.default_rng(d)
    hk, per = 3, max((n + 31) // 32 for n in lens) + 1
    c = P.RowCache.allocate(per * len(lens) + 1, hk, d, {"f32": P.F32, "bf16": P.BF16, "fp8": P.FP8}[cache])
    pools = [t.view(torch.uint8) for t in (c.k, c.v, c.k_exp, c.v_exp) if t is not None]
    for t in pools:
        t.copy_(torch.randint(0, 256, t.shape, device="cuda", dtype=torch.uint8))
    before = [t.clone() for t in pools]
    table = torch.randperm(per * len(lens) + 1, device="cuda")[:per * len(lens)].view(len(lens), per).to(torch.int32)
    width = max(trees) + 2
    path, kept = rng.integers(-5, 500, (len(lens), width)), []
    for b, t in enumerate(trees):
        chosen = [0] + [i for i in range(1, t) if rng.random() < 0.4] if t else []
        if b == 0 and t > 2:
            chosen = list(range(t))                               # all of it: nothing moves
        path[b, :len(chosen)] = chosen
        kept.append(len(chosen))
    starts = np.concatenate([[0], np.cumsum(trees)])
    c.keep(table, ints(lens), ints(starts), ints(path), ints(kept))
    want = [t.clone() for t in before]
    for b, (n, t) in enumerate(zip(lens, trees)):
        for i in range(kept[b]):
            to, of = n - t + i, n - t + int(path[b, i])
            for x, y in zip(want, before):
                x[int(table[b, to // 32]), :, to % 32] = y[int(table[b, of // 32]), :, of % 32]
    assert all(torch.equal(x, y) for x, y in zip(pools, want)) and c.get_status() == 0


def test_paths_and_pages_that_are_none():
    def fresh():
        c = P.RowCache.allocate(5, 2, 64, P.BF16)
        c.k.normal_()
        c.v.normal_()
        return c, c.k.clone()
    table, lens, starts = ints([[0, 1], [2, 3]]), ints([40, 60]), ints([0, 10, 20])
    for bad in (dict(kept=[11, 1]), dict(kept=[-1, 1]), dict(path=[[0, 0, 3], [0, 1, 2]], kept=[3, 1]), dict(path=[[0, 10, 11], [0, 1, 2]], kept=[2, 1]),
                dict(path=[[0, -4, 5], [0, 1, 2]], kept=[2, 1]), dict(lens=[-1, 60]), dict(lens=[65, 60]), dict(lens=[9, 60]), dict(starts=[10, 0, 10]),
                dict(kept=[4, 1]), dict(table=[[0, -1], [2, 3]], path=[[0, 3, 4], [0, 1, 2]], kept=[3, 1]), dict(table=[[0, 5], [2, 3]], path=[[0, 3, 4], [0, 1, 2]], kept=[3, 1])):
        c, before = fresh()
        use = dict(table=table, lens=lens, starts=starts, path=ints([[0, 2, 5], [0, 1, 2]]), kept=ints([3, 1]))
        use.update({k: ints(v) for k, v in bad.items()})
        c.keep(use["table"], use["lens"], use["starts"], use["path"], use["kept"])
        assert c.get_status() == P.ST_BOUNDS, bad
        assert torch.equal(c.k[4], before[4]) and torch.equal(c.k[2:4], before[2:4])


def test_refusals_of_keep():
    c = P.RowCache.allocate(4, 2, 64, P.BF16)
    ok = dict(page_table=ints([[0, 1]]), kv_len=ints([40]), q_start=ints([0, 4]), path=ints([[0, 2]]), kept=ints([2]))
    for bad in (dict(page_table=ints([0, 1])), dict(kv_len=ints([40]).long()), dict(q_start=ints([0])), dict(path=ints([0, 2])), dict(path=ints([[0, 2], [0, 1]])),
                dict(kept=ints([2]).cpu()), dict(page_table=ok["page_table"].float())):
        with pytest.raises(P.DynaKVError):
            c.keep(**{**ok, **bad})
    c.k.requires_grad_()
    with pytest.raises(P.DynaKVError, match="gradient"):
        c.keep(**ok)


# ------------------------------------------------------------------------------------------------- all of them together

class Toy:
    """One layer of attention over tokens: q, k and v from tables, the next token from the attention's result.  fp32, so that two ways
    to the same logits differ by less than any two logits."""

    def __init__(self, vocab=40, heads=4, hk=2, d=64, cache=P.F32):
        g = torch.Generator(device="cuda").manual_seed(3)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.vocab, self.heads, self.hk, self.d = vocab, heads, hk, d
        self.tq, self.tk, self.tv = rand(vocab, heads, d), rand(vocab, hk, d), rand(vocab, hk, d)
        self.w = rand(heads * d, vocab)
        self.rotary = P.HeadRotary(heads, hk, d, (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().cuda())
        self.cache, self.pool = P.RowCache.allocate(64, hk, d, cache), P.PagePool.allocate(64)

    def rows(self, tokens, positions, slots):
        t = tokens.long()
        return self.rotary.store(self.tq[t], self.tk[t], self.tv[t], positions, self.cache, slots)

    def logits(self, out):
        return out.reshape(len(out), -1) @ self.w


def test_a_run_as_used():
    """Prompts in chunks, then trees of drafts verified, kept and trimmed: the same tokens as one at a time."""
    prompts, steps = [[3, 17, 5, 29, 8, 11, 2], list(np.arange(90) * 7 % 40), [1]], 24
    batch = len(prompts)

    def start():
        toy = Toy()
        table, lens = torch.full((batch, 8), -1, dtype=torch.int32, device="cuda"), ints([0] * batch)
        done = [0] * batch
        while any(x < len(p) for x, p in zip(done, prompts)):     # chunks of at most 40 tokens
            new = [min(40, len(p) - x) for x, p in zip(done, prompts)]
            tokens = ints(np.concatenate([p[x:x + t] for x, p, t in zip(done, prompts, new)]))
            q_start, positions, slots = toy.pool.extend(table, lens, ints(new), sum(new))
            q = toy.rows(tokens, positions, slots)
            out, _ = toy.cache.attend_chunk(q, table, lens, q_start, 40)
            for b in range(batch):
                if new[b]:
                    last = toy.logits(out[int(q_start[b + 1]) - 1:int(q_start[b + 1])]).argmax()
                    if done[b] + new[b] == len(prompts[b]):
                        first[b] = int(last)
            done = [x + t for x, t in zip(done, new)]
        return toy, table, lens

    first = [0] * batch
    toy, table, lens = start()
    plain, now = [[x] for x in first], ints(first)
    for _ in range(steps):
        q_start, positions, slots = toy.pool.extend(table, lens, ints([1] * batch), batch)
        out, _ = toy.cache.attend_chunk(toy.rows(now, positions, slots), table, lens, q_start, 1)
        now = toy.logits(out).argmax(-1).to(torch.int32)
        for b in range(batch):
            plain[b].append(int(now[b]))
    assert toy.pool.get_status() == 0

    toy, table, lens = start()
    said, rng, longest = [[x] for x in first], np.random.default_rng(5), 0
    mask_of = lambda parent: [sum(1 << j for j in chain) for chain in ([i] + ancestors(parent, i) for i in range(len(parent)))]
    def ancestors(parent, i):
        got = []
        while parent[i] >= 0:
            i = parent[i]
            got.append(i)
        return got
    while min(len(x) for x in said) <= steps:
        tokens, parents, sizes = [], [], []
        for b in range(batch):
            # a tree: the last certain token, some right drafts, some wrong ones beside them
            truth = (plain[b] + [0] * 8)[len(said[b]):len(said[b]) + 3]
            mine, up, tip = [said[b][-1]], [-1], 0
            for t in truth[:int(rng.integers(0, 4))]:
                for x in [(t + 1 + int(rng.integers(0, 38))) % 40] * int(rng.integers(0, 2)) + [t]:
                    mine.append(int(x))
                    up.append(tip)
                tip = len(mine) - 1
            tokens += mine
            parents += up
            sizes.append(len(mine))
        most = max(sizes)
        n = sum(sizes) + 3                                        # a padded batch
        q_start, positions, slots = toy.pool.extend(table, lens, ints(sizes), n)
        # a draft's position is its depth's, not its place in the tree
        depth = torch.tensor(np.concatenate([[len(ancestors(parents[s:s + t], i)) - i for i in range(t)] for s, t in zip(np.cumsum([0] + sizes[:-1]), sizes)] + [[0] * 3]), device="cuda")
        all_tokens = ints(tokens + [0] * 3)
        q = toy.rows(all_tokens, (positions + depth).to(torch.int32), slots)
        mask = torch.tensor(np.concatenate([mask_of(parents[s:s + t]) for s, t in zip(np.cumsum([0] + sizes[:-1]), sizes)] + [[0] * 3]), dtype=torch.int64, device="cuda")[:, None]
        out, _ = toy.cache.attend_tree(q, table, lens, q_start, most, tree_mask=mask)
        kept, dropped, path, following = P.verify_drafts(toy.logits(torch.nan_to_num(out)), all_tokens, q_start, most, torch.rand(n, device="cuda"), torch.zeros(batch, device="cuda"),
                                                         parent=ints(parents + [0] * 3))
        toy.cache.keep(table, lens, q_start, path, kept)
        toy.pool.trim(table, lens, dropped)
        for b in range(batch):
            s = int(q_start[b])
            said[b] += [tokens[s + int(i)] for i in path[b, 1:int(kept[b])]] + [int(following[b])]
            longest = max(longest, int(kept[b]))
    assert toy.pool.get_status() == 0 and toy.cache.get_status() == 0 and longest >= 3
    for b in range(batch):
        assert said[b][:steps] == plain[b][:steps]
    toy.pool.trim(table, lens, lens.clone())
    assert int(toy.pool.count) == 64 and not lens.any()
