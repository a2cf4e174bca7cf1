"""Measured cases of the operators around the paged row cache: attention of a chunk of new tokens over it, page tables and
slots made on the device, verification of drafted tokens, and moving the rows of the accepted ones.

Each case is what a serving program does in one place of its loop.  ``run`` has two forms of every operator: the plain one in
elementary torch operations (``own = False``) and the framework's entry points (``own = True``); ``exact`` restates the
operators in 64 bits, one sequence and head at a time.
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 32                                    # rows of a cache page
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


# ------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one decode step of 16 ragged sequences in a layer with a sliding window and capped scores: the smallest attention call
        dict(name="chunk step 16 x 8192, window, cap", op="chunk", batch=16, heads=28, kv_heads=4, d=128, kv=8192, chunk=1, cache="bf16",
             mask="window", window=4096, cap=50.0, slopes=False),
        # chunks of four prompts that share a batch, capped scores: ordinary chunked prefill
        dict(name="chunk 4 x 512 over 16384, cap", op="chunk", batch=4, heads=32, kv_heads=8, d=128, kv=16384, chunk=512, cache="bf16",
             mask="causal", window=0, cap=50.0, slopes=False),
        # the last quarter of a long prompt: the most arithmetic
        dict(name="chunk 4096 over 16384", op="chunk", batch=1, heads=32, kv_heads=8, d=128, kv=16384, chunk=4096, cache="bf16",
             mask="causal", window=0, cap=0.0, slopes=False),
        # two packs of short documents of odd lengths, each seen by its own tokens only, over FP8 rows
        dict(name="documents 2 x 4001 fp8", op="chunk", batch=2, heads=28, kv_heads=4, d=128, kv=4001, chunk=4001, cache="fp8",
             mask="documents", window=0, cap=0.0, slopes=False),
        # prompts whose first part is seen by all of it, with a bias by distance, in 32 bits
        dict(name="prefix 3 x 777 f32, distances", op="chunk", batch=3, heads=8, kv_heads=8, d=64, kv=777, chunk=777, cache="f32",
             mask="prefix", window=0, cap=0.0, slopes=True),
        # a decode step of 64 sequences: a row each, now and then a page
        dict(name="pages step 64", op="pages", batch=64, per=640, new=1, spare=64, ragged=False),
        # the prompts of 512 requests taken in at once
        dict(name="pages 512 prompts", op="pages", batch=512, per=640, new=256, spare=1 << 13, ragged=True),
        # one sequence with four drafts that were looked up, not drawn: the smallest verification
        dict(name="verify 1 x 5, 32000", op="verify", batch=1, tree=5, vocab=32000, logits="f32", shape="chain", drawn=False),
        # a large batch with five drawn drafts each: the most bytes
        dict(name="verify 64 x 6, 128256, drawn", op="verify", batch=64, tree=6, vocab=128256, logits="bf16", shape="chain", drawn=True),
        # trees of likely tokens, an odd vocabulary
        dict(name="verify 16 trees of 32, 50257", op="verify", batch=16, tree=32, vocab=50257, logits="bf16", shape="tree", drawn=False),
        # rows of small trees written, and those of the accepted path moved together
        dict(name="keep 4 x 16 bf16", op="keep", batch=4, kv_heads=8, d=128, kv=2048, tree=16, cache="bf16"),
        # the same for a large batch of wide trees over FP8 rows
        dict(name="keep 48 x 128 fp8", op="keep", batch=48, kv_heads=8, d=128, kv=1024, tree=128, cache="fp8"),
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], even over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


_HEADS = [(4, 1), (8, 8), (28, 4), (32, 8), (16, 2), (12, 4), (5, 5)]


def draw(rng):
    op = rng.choice(["chunk", "chunk", "chunk", "chunk", "pages", "verify", "verify", "keep"])
    heads, kv_heads = rng.choice(_HEADS)
    d = rng.choice([64, 128, 128])
    cache = rng.choice(["f32", "bf16", "bf16", "bf16", "fp8", "fp8"])
    if op == "chunk":
        batch, chunk = _spread(rng, 1, 16), rng.choice([1, _spread(rng, 2, 4096), _spread(rng, 16, 4096)])
        # the largest listed case is 32 heads x 4096 tokens x 16384 rows; fp32 rows are kept below it by a factor
        most = 32 * 4096 * 16384 // (16 if cache == "f32" else 1)
        most_kv = max(16, min(20000, most // (batch * heads * chunk), 400_000 // (batch * kv_heads) + 1))
        kv = max(_spread(rng, 1, most_kv), 1)
        mask = rng.choice(["causal", "causal", "window", "prefix", "documents", "both ways"])
        return dict(op=op, batch=batch, heads=heads, kv_heads=kv_heads, d=d, kv=kv, chunk=min(chunk, kv), cache=cache, mask=mask,
                    window=_spread(rng, 1, 5000) if mask == "window" or rng.random() < 0.1 else 0,
                    cap=rng.choice([0.0, 0.0, 30.0, 50.0, 8.0]), slopes=rng.random() < 0.25)
    if op == "pages":
        batch = _spread(rng, 1, 1000)
        new = rng.choice([1, _spread(rng, 1, 300), _spread(rng, 1, max(1, 130000 // batch))])
        per = (new + PAGE - 1) // PAGE + _spread(rng, 1, 300)
        return dict(op=op, batch=batch, per=per, new=new, spare=_spread(rng, 1, 2 * batch * ((new + PAGE - 1) // PAGE + 1)), ragged=rng.random() < 0.7)
    if op == "verify":
        shape = rng.choice(["chain", "tree"])
        batch, tree = _spread(rng, 1, 64), _spread(rng, 1, 8 if shape == "chain" else 64)
        vocab = _spread(rng, 100, max(200, min(150000, 64 * 6 * 128256 // (batch * tree))))
        return dict(op=op, batch=batch, tree=tree, vocab=vocab, logits=rng.choice(["f32", "bf16"]), shape=shape,
                    drawn=shape == "chain" and rng.random() < 0.6)
    batch, tree = _spread(rng, 1, 48), _spread(rng, 1, 128)
    return dict(op=op, batch=batch, kv_heads=kv_heads, d=d, kv=max(tree, _spread(rng, 1, 1024)), tree=tree, cache=cache)


def _sizes(case):
    """Rows in the cache and new tokens of every sequence of a case: ragged, the first sequence the longest."""
    kv, new = case["kv"], case.get("chunk", case.get("tree"))
    lens = [kv - (b * 977) % (kv // 2 + 1) for b in range(case["batch"])]
    return lens, [min(n, new - (b * 5) % ((new + 1) // 2)) for b, n in enumerate(lens)]


def _seen(case):
    """First row and end of the rows that every token of every sequence sees, as the masks say, before windows: two lists of arrays."""
    lens, new = _sizes(case)
    low, high = [], []
    for b, (n, t) in enumerate(zip(lens, new)):
        place = np.arange(n - t, n)
        first, end = np.zeros(t, np.int64), place + 1
        if case["mask"] == "prefix":                     # the first third is seen by every token
            end = np.maximum(end, n // 3)
        if case["mask"] in ("documents", "both ways"):   # documents of 37 to 1060 rows, their borders at odd places
            borders = np.cumsum(37 + (np.arange(n // 37 + 2) * 389 + b * 61) % 1024)
            owner = np.searchsorted(borders, place, side="right")
            first = np.concatenate([[0], borders])[owner]
            if case["mask"] == "both ways":
                end = np.minimum(borders[owner], n)
        low.append(first)
        high.append(end)
    return low, high


def work(case):
    """What a pass cannot do without: inputs read once, outputs written once, products and sums of the formulas."""
    size = {"f32": 4, "bf16": 2, "fp8": 1}
    op = case["op"]
    if op == "pages":
        tokens = case["batch"] * case["new"]
        pages = tokens // (2 if case["ragged"] else 1) // PAGE + 1
        # lengths in and out twice, the pages taken and given back, and for every token (or place for one) its position and slot
        return {"bytes": case["batch"] * 24 + pages * 16 + tokens * 8, "flops": 0}
    if op == "verify":
        n, v, es = sum(_trees(case)), case["vocab"], size[case["logits"]]
        # all rows of logits once; of a drawn draft its probabilities at the one place where a sequence may stop
        return {"bytes": n * v * es + (case["batch"] * v * 4 if case["drawn"] else 0) + n * 16, "flops": 3 * n * v}
    d = case["d"]
    row = d * size[case["cache"]] + (case["cache"] == "fp8")
    lens, new = _sizes(case)
    if op == "keep":
        moved = sum(new) * case["kv_heads"]
        # drafted rows in, stored; about half of them read and written once more
        return {"bytes": moved * 2 * (d * (4 if case["cache"] == "f32" else 2) + 2 * row), "flops": 0}
    h, hk, io = case["heads"], case["kv_heads"], 4 if case["cache"] == "f32" else 2
    low, high = _seen(case)
    pairs = rows = 0
    for n, t, lo, hi in zip(lens, new, low, high):
        if case["window"]:
            lo = np.maximum(lo, np.arange(n - t, n) + 1 - case["window"])
        pairs += int(np.maximum(hi - lo, 0).sum())
        rows += int(hi.max(initial=0) - lo.min(initial=n)) if t else 0
    return {"bytes": 2 * hk * rows * row + sum(new) * h * (2 * d * io + 4), "flops": 4 * d * h * pairs}


# ------------------------------------------------------------------------------------------------- inputs

def _rows(g, *shape):
    """Keys as a cache holds them: a mixture of 64 directions with noise, four channels eight times as large as the others."""
    d = shape[-1]
    n = math.prod(shape[:-1])
    means = torch.randn(64, d, generator=g, device="cuda")
    x = means[torch.randint(64, (n,), generator=g, device="cuda")] + 0.5 * torch.randn(n, d, generator=g, device="cuda")
    scale = torch.ones(d, device="cuda")
    scale[torch.randperm(d, generator=g, device="cuda")[:4]] = 8.0
    return (x * scale).view(shape)


def _two(e):
    """2^e of whole numbers e of [-126, 127], from the bits of the result."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _to_fp8(x):
    """Rows as e4m3 values and one exponent each: the smallest 2^e (e in [-120, 120]) with max|x| / 2^e <= 448."""
    x = x.float()
    top = x.abs().amax(-1)
    part, e = torch.frexp(top)
    e = torch.where(top > 0, e - 9 + (part > 0.875), torch.zeros_like(e)).clamp(-120, 120)
    return (x * _two(-e)[..., None]).to(torch.float8_e4m3fn), e.to(torch.int8)


def _pools(state, g, pages, case):
    """A cache of `pages` pages that earlier sequences have written over: [pages, KV heads, 32, d], FP8 with exponents."""
    shape = (pages, case["kv_heads"], PAGE, case["d"])
    for name, x in (("k", _rows(g, *shape)), ("v", torch.randn(shape, generator=g, device="cuda"))):
        if case["cache"] == "fp8":
            state[name + "_pool"], state[name + "_exp"] = _to_fp8(x)
        else:
            state[name + "_pool"], state[name + "_exp"] = x.to(_TYPES[case["cache"]]), None


def _trees(case):
    """Tokens of every sequence's tree: the last token that is certain, and drafts."""
    tree = case["tree"]
    return [tree - (b * 3) % ((tree + 1) // 2) for b in range(case["batch"])]


def _ints(x):
    return torch.tensor(np.ascontiguousarray(x), dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    state = dict(case=case)
    if op in ("chunk", "keep"):
        lens, new = _sizes(case)
        b, per = case["batch"], (case["kv"] + PAGE - 1) // PAGE
        _pools(state, g, b * per + 3, case)
        state["page_table"] = torch.randperm(b * per + 3, generator=g, device="cuda")[: b * per].view(b, per).to(torch.int32)
        state["kv_len"] = _ints(lens)
        state["q_start"] = _ints(np.cumsum([0] + new))
        state["most"] = max(new)
        n, d, hk = sum(new), case["d"], case["kv_heads"]
    if op == "chunk":
        io = torch.float32 if case["cache"] == "f32" else torch.bfloat16
        state["q"] = torch.randn(n, case["heads"], d, generator=g, device="cuda").to(io)
        low, high = _seen(case)
        state["rows_from"] = _ints(np.concatenate(low)) if case["mask"] in ("documents", "both ways") else None
        state["rows_to"] = _ints(np.concatenate(high)) if case["mask"] in ("prefix", "both ways") else None
        state["slopes"] = torch.pow(2.0, -8.0 * torch.arange(1, case["heads"] + 1, device="cuda") / case["heads"]) if case["slopes"] else None
    if op == "keep":
        src = torch.float32 if case["cache"] == "f32" else torch.bfloat16
        kv = torch.randn(n, 2 * hk, d, generator=g, device="cuda")
        kv[:, :hk] = _rows(g, n, hk, d)
        kv = kv.to(src)
        state.update(k=kv[:, :hk], v=kv[:, hk:])
        # every tree's rows lie at its sequence's end
        rng = np.random.default_rng(seed)
        place = np.concatenate([np.arange(n - t, n) for n, t in zip(lens, new)])
        owner = np.repeat(np.arange(len(new)), new)
        at = torch.as_tensor(place, device="cuda"), torch.as_tensor(owner, device="cuda")
        state["slots"] = (state["page_table"][at[1], at[0] // PAGE] * PAGE + at[0] % PAGE).to(torch.int32)
        # accepted paths: the root, and every later token with even chances, in order
        path, kept = np.zeros((len(new), max(new)), np.int32), np.zeros(len(new), np.int32)
        for b, t in enumerate(new):
            chosen = np.flatnonzero(np.concatenate([[True], rng.random(t - 1) < 0.5])) if t else np.zeros(0, np.int64)
            path[b, :len(chosen)], kept[b] = chosen, len(chosen)
        state.update(path=_ints(path), kept=_ints(kept))
    if op == "pages":
        rng = np.random.default_rng(seed)
        b, per, new = case["batch"], case["per"], case["new"]
        add = rng.integers(1, new + 1, b) if case["ragged"] else np.full(b, new)
        old = rng.integers(0, np.maximum(per * PAGE - add, 0) + 1)
        held = (old + PAGE - 1) // PAGE
        pages = b * per + case["spare"]
        ids = rng.permutation(pages).astype(np.int32)
        table = np.full((b, per), -1, np.int32)
        table[np.arange(per) < held[:, None]] = ids[case["spare"]:][:held.sum()]
        free = np.full(pages, -1, np.int32)
        free[:case["spare"]] = ids[:case["spare"]]
        state.update(page_table=_ints(table), kv_len=_ints(old), new_len=_ints(add), free=_ints(free), count=_ints([case["spare"]]), tokens=b * new + 5)          # room for the longest prompts
    if op == "verify":
        rng = np.random.default_rng(seed)
        sizes = _trees(case)
        n, v = sum(sizes), case["vocab"]
        starts = np.cumsum([0] + sizes)
        parent = np.concatenate([np.concatenate([[-1], [rng.integers(max(0, i - 6), i) if case["shape"] == "tree" else i - 1 for i in range(1, t)]]) for t in sizes]).astype(np.int64)
        above = torch.as_tensor(np.where(parent < 0, 0, parent) + np.repeat(starts[:-1], sizes), device="cuda")      # packed row of the parent
        heat = rng.choice([0.0, 0.7, 1.0, 1.0, 1.3], len(sizes)).astype(np.float32)
        # a model's logits: a few tokens stand out of many that hardly matter
        logits = 2.0 * torch.randn(n, v, generator=g, device="cuda") - 1.5 * torch.log(1 + torch.randperm(v, generator=g, device="cuda").float())
        state["logits"] = logits.to(_TYPES[case["logits"]])
        # the drafting model sees nearly the same
        draft = logits[above] + 0.4 * torch.randn(n, v, generator=g, device="cuda")
        state["draft"] = None
        if case["drawn"]:
            t = torch.tensor(heat, device="cuda").clamp(min=0.5).repeat_interleave(torch.tensor(sizes, device="cuda"))
            state["draft"] = torch.softmax(draft / t[:, None], -1)
            race = state["draft"] / torch.empty_like(draft).exponential_(generator=g).clamp(min=1e-30)
            tokens = race.argmax(-1)
        else:                                            # likely tokens, a place further down for every sibling
            best = draft.topk(min(8, v), -1).indices
            rank, seen = [], {}
            for i, p in enumerate(zip(np.repeat(np.arange(len(sizes)), sizes).tolist(), parent.tolist())):
                rank.append(seen.get(p, 0))
                seen[p] = rank[-1] + 1
            tokens = best.gather(1, torch.tensor(rank, device="cuda").remainder(best.shape[1])[:, None])[:, 0]
        state.update(tokens=tokens.to(torch.int32), q_start=_ints(starts), parent=_ints(parent) if case["shape"] == "tree" else None, most=max(sizes),
                     uniform=torch.rand(n, generator=g, device="cuda"), temperature=torch.tensor(heat, device="cuda"))
    return state


# ------------------------------------------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _held(s):
    """The cache's own buffers: rows, and with FP8 their exponents."""
    return [s[n] for n in ("k_pool", "v_pool", "k_exp", "v_exp") if s[n] is not None]


def _run_own(s):
    import paper_2511_07427_b200 as dk
    case = s["case"]
    op = case["op"]
    if "handle" not in s:            # what a program makes once: the cache around its pools, the pool of free pages
        s["handle"] = dk.RowCache(s["k_pool"], s["v_pool"], s["k_exp"], s["v_exp"]) if "k_pool" in s else dk.PagePool(s["free"], s["count"]) if op == "pages" else None
    if op == "chunk":
        return s["handle"].attend_chunk(s["q"], s["page_table"], s["kv_len"], s["q_start"], s["most"], window=case["window"], softcap=case["cap"],
                                        slopes=s["slopes"], rows_from=s["rows_from"], rows_to=s["rows_to"])
    if op == "keep":
        s["handle"].write(s["k"], s["v"], s["slots"])
        s["handle"].keep(s["page_table"], s["kv_len"], s["q_start"], s["path"], s["kept"])
        return _held(s)
    if op == "pages":                # rows for new tokens, and when the step is taken back their pages
        q_start, positions, slots = s["handle"].extend(s["page_table"], s["kv_len"], s["new_len"], s["tokens"])
        s["handle"].trim(s["page_table"], s["kv_len"], q_start[1:] - q_start[:-1])
        return q_start, positions, slots, s["page_table"], s["kv_len"], s["free"], s["count"]
    return dk.verify_drafts(s["logits"], s["tokens"], s["q_start"], s["most"], s["uniform"], s["temperature"], parent=s["parent"], draft_probs=s["draft"])


def _run_plain(s):
    op = s["case"]["op"]
    return _attend(s) if op == "chunk" else _keep(s) if op == "keep" else _pages(s) if op == "pages" else _verify(s)


def _got(s, name):
    """Rows of every sequence in order, [sequences, KV heads, rows, d] in 32 bits, zeros behind a sequence's length."""
    table = s["page_table"].long()
    pool = s[name + "_pool"]
    if s[name + "_exp"] is None:
        x = pool[table].float()
    else:
        x = pool.view(torch.uint8)[table].view(pool.dtype).float() * _two(s[name + "_exp"][table])[..., None]
    x = x.transpose(1, 2).flatten(2, 3)[:, :, :s["case"]["kv"]]
    there = torch.arange(x.shape[2], device=x.device) < s["kv_len"][:, None]
    return torch.where(there[:, None, :, None], x, 0.0)


def _attend(s):
    case = s["case"]
    b, h, hk, d, most = case["batch"], case["heads"], case["kv_heads"], case["d"], s["most"]
    group = h // hk
    k, v = _got(s, "k"), _got(s, "v")
    n = k.shape[2]
    starts = s["q_start"].long()
    token = torch.arange(most, device=k.device)
    spot = (starts[:-1, None] + token).clamp(max=s["q"].shape[0] - 1)           # packed row of (sequence, token)
    q = s["q"][spot].float().view(b, most, hk, group, d).permute(0, 2, 1, 3, 4).reshape(b, hk, most * group, d)
    logits = (q @ k.transpose(-1, -2) / math.sqrt(d)).view(b, hk, most, group, n)
    if case["cap"]:
        logits = case["cap"] * torch.tanh(logits / case["cap"])
    # the token's own row, and the rows that it sees
    place = (s["kv_len"].long() - (starts[1:] - starts[:-1]))[:, None] + token
    row = torch.arange(n, device=k.device)
    if s["slopes"] is not None:
        away = (place[:, :, None] - row).abs().float()
        logits = logits - s["slopes"].view(hk, 1, group, 1) * away[:, None, :, None]
    first = s["rows_from"][spot].long() if s["rows_from"] is not None else torch.zeros_like(place)
    if case["window"]:
        first = torch.maximum(first, place + 1 - case["window"])
    end = s["rows_to"][spot].long() if s["rows_to"] is not None else place + 1
    sees = (row >= first[:, :, None]) & (row < torch.minimum(end, s["kv_len"][:, None])[:, :, None])
    logits = torch.where(sees[:, None, :, None], logits, -torch.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    out = ((p.view(b, hk, most * group, n) @ v).view(b, hk, most, group, d) / total).nan_to_num()
    lse = (torch.log(total) + top).squeeze(-1)
    lse = torch.where(sees.any(-1)[:, None, :, None], lse, -torch.inf)
    out = out.permute(0, 2, 1, 3, 4).reshape(b * most, h, d)
    lse = lse.permute(0, 2, 1, 3).reshape(b * most, h)
    # back to packed rows
    index = torch.arange(s["q"].shape[0], device=k.device)
    owner = torch.searchsorted(starts, index, right=True) - 1
    back = owner * most + index - starts[owner]
    return out[back].to(s["q"].dtype), lse[back]


def _keep(s):
    """Drafted rows into their slots, then row path[i] of every tree to the tree's row i."""
    page, row = s["slots"].long() // PAGE, s["slots"].long() % PAGE
    for name in ("k", "v"):
        pool = s[name + "_pool"]
        if s[name + "_exp"] is None:
            pool[page, :, row] = s[name].to(pool.dtype)
        else:
            x, e = _to_fp8(s[name])
            pool.view(torch.uint8)[page, :, row] = x.view(torch.uint8)
            s[name + "_exp"][page, :, row] = e
    starts = s["q_start"].long()
    first = s["kv_len"].long() - (starts[1:] - starts[:-1])
    i = torch.arange(s["most"], device=first.device).expand(len(first), -1)
    take = i < s["kept"][:, None]
    owner = torch.arange(len(first), device=first.device)[:, None].expand_as(i)[take]
    to, source = (first[:, None] + i)[take], (first[:, None] + s["path"])[take]
    table = s["page_table"].long()
    at, of = (table[owner, to // PAGE], to % PAGE), (table[owner, source // PAGE], source % PAGE)
    for pool in _held(s):
        pool = pool.view(torch.uint8) if pool.dtype == torch.float8_e4m3fn else pool
        pool[at[0], :, at[1]] = pool[of[0], :, of[1]]
    return _held(s)


def _pages(s):
    """Rows for new tokens at the ends of the sequences, pages from the top of the stack of free ones; then all of it back."""
    table, lens, free, count = s["page_table"], s["kv_len"], s["free"], s["count"]
    b, per = table.shape
    old, add = lens.long(), s["new_len"].long()
    pages = lambda rows: torch.div(rows + PAGE - 1, PAGE, rounding_mode="floor")
    fits = (add >= 0) & (old >= 0) & (old + add <= per * PAGE)
    want = torch.where(fits, add, 0)
    need = torch.where(fits, pages(old + add) - pages(old), 0)
    # sequences are served in order, up to the first one for which pages or places are short
    served = fits & (need.cumsum(0) <= count) & (want.cumsum(0) <= s["tokens"])
    want, need = torch.where(served, want, 0), torch.where(served, need, 0)
    q_start = torch.cat([torch.zeros_like(want[:1]), want.cumsum(0)])
    before = need.cumsum(0) - need
    column = torch.arange(per, device=table.device)
    rank = column - pages(old)[:, None]                                  # a column's place among the sequence's new pages
    fresh = (rank >= 0) & (rank < need[:, None])
    taken = (count.long() - 1 - before[:, None] - rank).clamp(min=0, max=len(free) - 1)
    table.copy_(torch.where(fresh, free[taken], table))
    lens.add_(want.to(torch.int32))
    count.sub_(need.sum().to(torch.int32))
    index = torch.arange(s["tokens"], device=table.device)
    owner = (torch.searchsorted(q_start, index, right=True) - 1).clamp(max=b - 1)
    place = old[owner] + index - q_start[owner]
    real = index < q_start[-1]
    page = table[owner, (place // PAGE).clamp(max=per - 1)]
    positions = torch.where(real, place, 0).to(torch.int32)
    slots = torch.where(real, page * PAGE + place % PAGE, -1).to(torch.int32)
    # taken back: the pages behind the old lengths return in the order in which they lay
    fewer = lens.long() - want
    gone = (column >= pages(fewer)[:, None]) & (column < pages(lens.long())[:, None])
    number = gone.flatten().cumsum(0).view(b, per) - 1
    total = gone.sum()
    free[(count + total - 1 - number)[gone]] = table[gone]
    table.masked_fill_(gone, -1)
    lens.copy_(fewer)
    count.add_(total.to(torch.int32))
    return q_start.to(torch.int32), positions, slots, table, lens, free, count


def _verify(s):
    starts = s["q_start"].long()
    sizes = starts[1:] - starts[:-1]
    b, most = len(sizes), s["most"]
    n, vocab = s["logits"].shape
    index = torch.arange(n, device=starts.device)
    owner = torch.searchsorted(starts, index, right=True) - 1
    root = index == starts[owner]
    above = torch.where(root, index, index - 1 if s["parent"] is None else starts[owner] + s["parent"])      # packed row of the parent
    heat = s["temperature"].double()[owner]
    logits = s["logits"].double()
    top, best = logits.max(-1, keepdim=True)                            # the first of equals
    p = torch.softmax((logits - top) / torch.where(heat > 0, heat, 1.0)[:, None], -1)
    p = torch.where(heat[:, None] > 0, p, torch.zeros_like(p).scatter_(1, best, 1.0))
    token = s["tokens"].long()
    mine = p[above, token]
    # earlier siblings (rows and columns: tokens of one tree), whose tokens are out of question once they were refused
    spot = (starts[:-1, None] + torch.arange(most, device=starts.device)).clamp(max=n - 1)
    there = torch.arange(most, device=starts.device) < sizes[:, None]
    up, tok, pm = above[spot], token[spot], mine[spot]
    drafted = there & ~root[spot]
    older = torch.ones(most, most, dtype=torch.bool, device=starts.device).tril(-1)
    sibling = (up[:, :, None] == up[:, None, :]) & drafted[:, :, None] & drafted[:, None, :] & older
    again = sibling & (tok[:, :, None] == tok[:, None, :])
    repeat = again.any(-1)                                              # this token was refused before
    out = (sibling & ~repeat[:, None, :]).double() @ pm[:, :, None]
    u = s["uniform"].double()[spot]
    if s["draft"] is None:
        passes = (u * (1 - out[..., 0]) < pm) & ~repeat
    else:
        passes = u * s["draft"][index, token].double()[spot] < pm
    passes = torch.where(heat[spot] > 0, passes, (best[above, 0][spot] == tok) & ~repeat) & drafted
    chosen = passes & ~(sibling & passes[:, None, :]).any(-1)
    # a token is kept if it and all above it are chosen: the reach of the links upward doubles
    good = chosen | (there & root[spot])
    link = up - starts[:-1, None]
    for _ in range(max(1, most).bit_length()):
        good, link = good & good.gather(1, link.clamp(min=0)), link.gather(1, link.clamp(min=0))
    good = good & there
    kept = good.sum(-1)
    path = torch.where(torch.arange(most, device=starts.device) < kept[:, None], torch.argsort((~good).to(torch.int8), dim=-1, stable=True), -1)
    # the next token, from what is left of the last kept token's distribution
    last = starts[:-1] + path.gather(1, (kept - 1).clamp(min=0)[:, None])[:, 0].clamp(min=0)
    last = last.clamp(max=n - 1)
    left = p[last]
    refused = drafted & (up == last[:, None]) & ~good
    if s["draft"] is None:
        gone = torch.zeros_like(left).scatter_add_(1, tok, refused.double()) > 0
        left = torch.where(gone & (heat[last] > 0)[:, None], 0.0, left)
    else:
        child = (spot * refused).amax(-1)
        rest = (left - s["draft"][child].double()).clamp(min=0)
        use = refused.any(-1) & (heat[last] > 0) & (rest.sum(-1) > 0)
        left = torch.where(use[:, None], rest, left)
    run_sum = left.cumsum(-1)
    goal = s["uniform"].double()[starts[:-1].clamp(max=n - 1)] * run_sum[:, -1]
    chosen = torch.searchsorted(run_sum, goal[:, None], right=True)[:, 0]
    none = (sizes == 0) | ~(run_sum[:, -1] > 0)
    next_token = torch.where(none, -1, chosen)
    return kept.to(torch.int32), (sizes - kept).to(torch.int32), path.to(torch.int32), next_token.to(torch.int32)


# ------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"chunk": _exact_chunk, "keep": _exact_keep, "pages": _exact_pages, "verify": _exact_verify}[case["op"]](case, s)


def _power(e):
    """2^e of whole numbers in 64 bits, from the bits of the result: a power function may be off in its last place."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _all_rows(s, name):
    """The pool in 64 bits."""
    x = s[name + "_pool"].float().double()
    if s[name + "_exp"] is not None:
        x = x * _power(s[name + "_exp"])[..., None]
    return x


def _exact_chunk(case, s):
    lens, new = _sizes(case)
    d, group = case["d"], case["heads"] // case["kv_heads"]
    low, high = _seen(case)
    out = torch.zeros(sum(new), case["heads"], d, dtype=torch.float64, device="cuda")
    lse = torch.full((sum(new), case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    pool_k, pool_v = s["k_pool"], s["v_pool"]
    begin = 0
    for b, (n, t) in enumerate(zip(lens, new)):
        mine = dict(k_pool=pool_k.view(torch.uint8)[s["page_table"][b].long()].view(pool_k.dtype) if case["cache"] == "fp8" else pool_k[s["page_table"][b].long()],
                    v_pool=pool_v.view(torch.uint8)[s["page_table"][b].long()].view(pool_v.dtype) if case["cache"] == "fp8" else pool_v[s["page_table"][b].long()],
                    k_exp=s["k_exp"][s["page_table"][b].long()] if case["cache"] == "fp8" else None,
                    v_exp=s["v_exp"][s["page_table"][b].long()] if case["cache"] == "fp8" else None)
        ks, vs = (_all_rows(mine, x).transpose(0, 1).reshape(case["kv_heads"], -1, d)[:, :n] for x in ("k", "v"))
        own_row = torch.arange(n - t, n, device="cuda")
        row = torch.arange(n, device="cuda")
        first = torch.as_tensor(low[b], device="cuda")
        if case["window"]:
            first = torch.maximum(first, own_row - case["window"] + 1)
        sees = (first[:, None] <= row) & (row < torch.as_tensor(high[b], device="cuda")[:, None])
        for head in range(case["heads"]):
            w = (s["q"][begin:begin + t, head].double() @ ks[head // group].T) / math.sqrt(d)
            if case["cap"]:
                w = torch.tanh(w / case["cap"]) * case["cap"]
            if case["slopes"]:
                w -= s["slopes"][head].double() * (own_row[:, None] - row).abs()
            w.masked_fill_(~sees, -math.inf)
            lse[begin:begin + t, head] = torch.logsumexp(w, -1)
            out[begin:begin + t, head] = torch.softmax(w, -1).nan_to_num(0.0) @ vs[head // group]
        begin += t
    return out, lse


def _exact_keep(case, s):
    """FP8 rows before their rounding to e4m3, and their exponents."""
    lens, new = _sizes(case)
    results = []
    table, path, kept = (s[x].tolist() for x in ("page_table", "path", "kept"))
    exps = []
    for name in ("k", "v"):
        pool = s[name + "_pool"].float().double()
        exp = s[name + "_exp"].clone() if s[name + "_exp"] is not None else None
        begin = 0
        for b, (n, t) in enumerate(zip(lens, new)):
            x = s[name][begin:begin + t].double()
            begin += t
            e = None
            if exp is not None:
                top = x.abs().amax(-1)
                e = torch.ceil(torch.log2(top / 448)).nan_to_num(neginf=0.0)
                # the logarithm may be off by one step next to a whole number
                e = torch.where(top > 448 * _power(e), e + 1, torch.where(top <= 448 * _power(e - 1), e - 1, e))
                e = torch.where(top > 0, e, 0.0).clamp(-120, 120)
                x = x / _power(e)[..., None]
            source = path[b][:kept[b]] + list(range(kept[b], t))
            place = [n - t + i for i in range(t)]
            at = (torch.tensor([table[b][r // PAGE] for r in place], device="cuda"), torch.tensor([r % PAGE for r in place], device="cuda"))
            pool[at[0], :, at[1]] = x[source]
            if exp is not None:
                exp[at[0], :, at[1]] = e[source].to(torch.int8)
        results.append(pool)
        exps += [exp] if exp is not None else []
    return results + exps


def _exact_pages(case, s):
    table, lens, add, free = (s[x].cpu().numpy().copy() for x in ("page_table", "kv_len", "new_len", "free"))
    count, room = int(s["count"][0]), s["tokens"]
    starts, positions, slots, used = [0], [], [], 0
    open_ = True
    for b in range(case["batch"]):
        pages, rows = -(-int(lens[b]) // PAGE), int(lens[b]) + int(add[b])
        need = -(-rows // PAGE) - pages
        open_ = open_ and used + need <= count and starts[-1] + int(add[b]) <= room
        if open_:
            here = list(table[b, :pages]) + [free[count - 1 - used - i] for i in range(need)]
            used += need
            positions += range(int(lens[b]), rows)
            slots += [here[r // PAGE] * PAGE + r % PAGE for r in range(int(lens[b]), rows)]
        starts.append(len(positions))
    pad = room - len(positions)
    return (np.array(starts, np.int32), np.array(positions + [0] * pad, np.int32), np.array(slots + [-1] * pad, np.int32), table, lens, free, np.array([count], np.int32))


def _exact_verify(case, s):
    starts, tokens, uniform, heat = (s[x].cpu().numpy() for x in ("q_start", "tokens", "uniform", "temperature"))
    parent = s["parent"].cpu().numpy() if s["parent"] is not None else None
    kept, path, following = [], np.full((case["batch"], s["most"]), -1, np.int32), []

    def chances(row, t):
        x = s["logits"][row].double().cpu().numpy()
        if t == 0:
            p = np.zeros_like(x)
            p[int(np.argmax(x))] = 1.0
            return p
        p = np.exp((x - x.max()) / float(t))
        return p / p.sum()

    for b in range(case["batch"]):
        first, size = int(starts[b]), int(starts[b + 1] - starts[b])
        at, walked = 0, [0]
        p = chances(first, heat[b])
        going = True
        while going:
            going = False
            for c in range(at + 1, size):
                if (parent[first + c] if parent is not None else c - 1) != at:
                    continue
                x = int(tokens[first + c])
                drawn = s["draft"][first + c].double().cpu().numpy() if s["draft"] is not None else None
                q = drawn[x] if drawn is not None else 1.0
                if (p[x] == 1.0) if heat[b] == 0 else float(uniform[first + c]) * q * p.sum() < p[x]:
                    at, going = c, True
                    walked.append(c)
                    p = chances(first + c, heat[b])
                    break
                if heat[b] > 0:
                    if drawn is None:
                        p[x] = 0.0
                    elif np.maximum(p - drawn, 0).sum() > 0:
                        p = np.maximum(p - drawn, 0)
        runs = np.cumsum(p)
        following.append(int(np.searchsorted(runs, float(uniform[first]) * runs[-1], side="right")))
        kept.append(len(walked))
        path[b, :len(walked)] = walked
    kept = np.array(kept, np.int32)
    return kept, (np.diff(starts) - kept).astype(np.int32), path, np.array(following, np.int32)


if __name__ == "__main__":
    draws = random.Random(0)
    for c in listed() + [draw(draws) for _ in range(10)]:
        print(c, work(c))
