"""Measured cases of the row operators: head norms with the rotary embedding, rows written to and read from a paged cache,
and attention for trees of drafted tokens over it.

Each case is one call as a serving program makes it.  ``run`` has two forms of every operator: the plain one in elementary
torch operations (``own = False``) and the framework's entry point (``own = True``); ``exact`` restates the operators in
64 bits, one sequence and head at a time.
"""
import math
import random

import torch

own = False

PAGE = 32                                    # rows of a cache page
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


# ------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one decode step of a batch of 16 sequences, 28 query and 4 KV heads: the smallest call, latency counts
        dict(name="rope step 16", op="rope", tokens=16, heads=28, kv_heads=4, d=128, rot=128, interleaved=False, norm=True,
             src="bf16", dst="bf16", far=20480),
        # prefill of 8192 tokens, 32 query and 8 KV heads: bandwidth
        dict(name="rope prefill 8192", op="rope", tokens=8192, heads=32, kv_heads=8, d=128, rot=128, interleaved=False,
             norm=True, src="bf16", dst="bf16", far=8192),
        # a prefill chunk of odd length whose rows go straight into the paged cache, q, k and v as slices of one projection
        dict(name="rope store 1777", op="store", tokens=1777, heads=32, kv_heads=8, d=128, rot=64, interleaved=True,
             norm=True, src="bf16", dst="bf16", cache="bf16", far=1 << 20),
        # one token of each of 16 sequences into an FP8 cache
        dict(name="write step 16 fp8", op="write", tokens=16, kv_heads=4, d=128, src="bf16", cache="fp8"),
        # a whole prompt into an FP8 cache
        dict(name="write prompt 16384 fp8", op="write", tokens=16384, kv_heads=8, d=128, src="bf16", cache="fp8"),
        # the rows of a few short, ragged sequences read back for an index build
        dict(name="read 3 x 777 bf16", op="read", batch=3, kv_heads=8, d=128, kv=777, cache="bf16"),
        # the rows of a batch of long sequences read back from FP8
        dict(name="read 16 x 16384 fp8", op="read", batch=16, kv_heads=4, d=128, kv=16384, cache="fp8"),
        # plain decoding of one sequence: the smallest attention call
        dict(name="attend 1 x 2048 f32", op="attend", batch=1, heads=4, kv_heads=1, d=64, kv=2048, tree=1, shape="chain", cache="f32"),
        # decoding of one sequence at 8192 rows
        dict(name="attend 1 x 8192 bf16", op="attend", batch=1, heads=32, kv_heads=8, d=128, kv=8192, tree=1, shape="chain", cache="bf16"),
        # batched decoding of ragged sequences over FP8 rows
        dict(name="attend 16 x 20480 fp8", op="attend", batch=16, heads=28, kv_heads=4, d=128, kv=20480, tree=1, shape="chain", cache="fp8"),
        # four sequences, trees of up to 16 drafted tokens over long caches
        dict(name="tree 16, 4 x 32768 bf16", op="attend", batch=4, heads=32, kv_heads=8, d=128, kv=32768, tree=16, shape="tree", cache="bf16"),
        # wide trees of up to 64 drafted tokens: the most arithmetic per row read
        dict(name="tree 64, 2 x 34816 bf16", op="attend", batch=2, heads=32, kv_heads=8, d=128, kv=34816, tree=64, shape="tree", cache="bf16"),
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], even over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


_HEADS = [(4, 1), (8, 8), (28, 4), (32, 8), (16, 2), (12, 4), (5, 5)]


def draw(rng):
    op = rng.choice(["rope", "store", "write", "read", "attend", "attend", "attend"])
    heads, kv_heads = rng.choice(_HEADS)
    d = rng.choice([64, 128, 128])
    cache = rng.choice(["f32", "bf16", "bf16", "fp8", "fp8"])
    if op in ("rope", "store"):
        case = dict(op=op, tokens=_spread(rng, 1, 8000), heads=heads, kv_heads=kv_heads, d=d, rot=rng.choice([d, d, d // 2, 48]),
                    interleaved=rng.random() < 0.3, norm=rng.random() < 0.7, src=rng.choice(["bf16", "bf16", "f32"]),
                    dst=rng.choice(["bf16", "f32"]), far=_spread(rng, 8, 1 << 20))
        if op == "store":
            case["cache"] = cache
        return case
    if op == "write":
        return dict(op=op, tokens=_spread(rng, 1, 16000), kv_heads=kv_heads, d=d, src=rng.choice(["bf16", "bf16", "f32"]), cache=cache)
    batch = _spread(rng, 1, 16)
    if op == "read":
        return dict(op=op, batch=batch, kv_heads=kv_heads, d=d, kv=_spread(rng, 1, max(1, min(16384, 1_000_000 // (batch * kv_heads)))), cache=cache)
    tree = rng.choice([1, 1, _spread(rng, 2, 64), _spread(rng, 2, 200)])
    # the largest listed case is 2 sequences x 32 heads x 64 drafts x 34816 rows; fp32 rows are kept below it by a factor
    most = 2 * 32 * 64 * 34816 // (4 if cache == "f32" else 1)
    most_kv = max(16, min(34816, most // (batch * heads * tree), 500_000 // (batch * kv_heads) + 1))
    return dict(op=op, batch=batch, heads=heads, kv_heads=kv_heads, d=d, kv=max(_spread(rng, 1, most_kv), 1), tree=tree,
                shape=rng.choice(["chain", "tree"]), cache=cache)


def _sizes(case):
    """Rows in the cache and drafted tokens of every sequence of a case: ragged, the first sequence the longest."""
    kv, tree = case["kv"], case.get("tree", 1)
    lens = [kv - (b * 977) % (kv // 2 + 1) for b in range(case["batch"])]
    return lens, [min(n, tree - (b * 5) % ((tree + 1) // 2)) for b, n in enumerate(lens)]


def work(case):
    """What a pass cannot do without: inputs read once, outputs written once, products and sums of the formulas."""
    size = {"f32": 4, "bf16": 2, "fp8": 1}
    op, d = case["op"], case["d"]
    if op in ("rope", "store"):
        t, h, hk = case["tokens"], case["heads"], case["kv_heads"]
        src, dst = size[case["src"]], size[case["dst"]]
        if op == "rope":
            n = t * (h + hk) * d * (src + dst) + 4 * t
        else:
            row = d * size[case["cache"]] + (case["cache"] == "fp8")
            n = t * (h * d * (src + dst) + 2 * hk * (d * src + row)) + 8 * t
        return {"bytes": n, "flops": t * (h + hk) * ((4 * d if case["norm"] else 0) + 3 * case["rot"])}
    row = d * size[case["cache"]] + (case["cache"] == "fp8")
    if op == "write":
        t, hk = case["tokens"], case["kv_heads"]
        return {"bytes": 2 * t * hk * (d * size[case["src"]] + row) + 4 * t, "flops": 4 * t * hk * d}
    lens, drafts = _sizes(case)
    hk = case["kv_heads"]
    if op == "read":
        out = d * (4 if case["cache"] == "f32" else 2)
        return {"bytes": 2 * hk * (sum(lens) * row + case["batch"] * case["kv"] * out), "flops": 2 * sum(lens) * hk * d}
    h, io = case["heads"], 4 if case["cache"] == "f32" else 2
    return {"bytes": 2 * hk * sum(lens) * row + sum(drafts) * h * (2 * d * io + 4), "flops": 4 * d * h * sum(n * t for n, t in zip(lens, drafts))}


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


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, d = case["op"], case["d"]
    state = dict(case=case)
    if op in ("rope", "store", "write"):
        t, h, hk = case["tokens"], case.get("heads", 0), case["kv_heads"]
        # q, k and v are slices of one projection's output, as a model has them
        qkv = torch.randn(t, h + 2 * hk, d, generator=g, device="cuda")
        qkv[:, h:h + hk] = _rows(g, t, hk, d)
        qkv = qkv.to(_TYPES[case["src"]])
        state.update(q=qkv[:, :h], k=qkv[:, h:h + hk], v=qkv[:, h + hk:])
    if op in ("rope", "store"):
        r = case["rot"]
        state["inv_freq"] = (500000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float().cuda()
        state["q_weight"] = 1 + 0.1 * torch.randn(d, generator=g, device="cuda") if case["norm"] else None
        state["k_weight"] = 1 + 0.1 * torch.randn(d, generator=g, device="cuda") if case["norm"] else None
        if t <= 64:          # a decode step: every token is at its own place
            state["positions"] = torch.randint(case["far"], (t,), generator=g, device="cuda", dtype=torch.int32)
        else:                # a chunk of a prompt that ends at `far` or begins at 0
            state["positions"] = torch.arange(t, device="cuda", dtype=torch.int32) + max(0, case["far"] - t)
    if op in ("store", "write"):
        pages = (t + PAGE - 1) // PAGE + 8
        _pools(state, g, pages, case)
        order = torch.randperm(pages, generator=g, device="cuda")
        # a prompt fills pages one after the other, a decode step one row of many pages
        spots = torch.arange(t, device="cuda")
        rows = torch.randperm(pages * PAGE, generator=g, device="cuda")[:t] if t <= 64 else order[spots // PAGE] * PAGE + spots % PAGE
        state["slots"] = rows.to(torch.int32)
    if op in ("read", "attend"):
        lens, drafts = _sizes(case)
        b, per = case["batch"], (case["kv"] + PAGE - 1) // PAGE
        _pools(state, g, b * per + 3, case)
        state["page_table"] = torch.randperm(b * per + 3, generator=g, device="cuda")[: b * per].view(b, per).to(torch.int32)
        state["kv_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if op == "attend":
        n, most = sum(drafts), max(drafts)
        io = torch.float32 if case["cache"] == "f32" else torch.bfloat16
        state["q"] = torch.randn(n, case["heads"], d, generator=g, device="cuda").to(io)
        state["q_start"] = torch.tensor([0] + drafts, device="cuda").cumsum(0).to(torch.int32)
        state["most"] = most
        state["tree_mask"] = None
        if case["shape"] == "tree":
            state["tree_mask"] = _tree(g, drafts, most)
    return state


def _tree(g, drafts, most):
    """Random trees: every token's parent is one of the four before it, or the last token of the context.  Bit j of a token's
    words: it sees token j of its tree (itself and its ancestors)."""
    b = len(drafts)
    index = torch.arange(most, device="cuda")
    parent = index - 1 - torch.randint(4, (b, most), generator=g, device="cuda")
    sees = (parent[:, :, None] == index) | (index[:, None] == index)
    steps = 1
    while steps < most:                          # ancestors of ancestors: the reach doubles
        sees = torch.bmm(sees.float(), sees.float()) > 0
        steps *= 2
    words = (most + 63) // 64
    bits = torch.zeros(b, most, words * 64, dtype=torch.int64, device="cuda")
    bits[:, :, :most] = sees.to(torch.int64)
    packed = (bits.view(b, most, words, 64) << torch.arange(64, device="cuda")).sum(-1)
    keep = index < torch.tensor(drafts, device="cuda")[:, None]
    return packed[keep].contiguous()


# ------------------------------------------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2511_07427_b200 as dk
    case = s["case"]
    op = case["op"]
    if "handles" not in s:          # what a program makes once: the cache around its pools, the rotary embedding's constants
        s["handles"] = (
            dk.RowCache(s["k_pool"], s["v_pool"], s["k_exp"], s["v_exp"]) if "k_pool" in s else None,
            dk.HeadRotary(case["heads"], case["kv_heads"], case["d"], s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                          eps=1e-6, interleaved=case["interleaved"]) if "inv_freq" in s else None)
    cache, rotary = s["handles"]
    if op == "rope":
        return rotary.apply(s["q"], s["k"], s["positions"], q_dtype=_TYPES[case["dst"]], k_dtype=_TYPES[case["dst"]])
    if op == "store":
        return [rotary.store(s["q"], s["k"], s["v"], s["positions"], cache, s["slots"], q_dtype=_TYPES[case["dst"]])] + _held(s)
    if op == "write":
        cache.write(s["k"], s["v"], s["slots"])
        return _held(s)
    if op == "read":
        return cache.read(s["page_table"], s["kv_len"], case["kv"])
    return cache.attend_tree(s["q"], s["page_table"], s["kv_len"], s["q_start"], s["most"], tree_mask=s["tree_mask"])


def _held(s):
    """The cache's own buffers: rows, and with FP8 their exponents."""
    return [s[n] for n in ("k_pool", "v_pool", "k_exp", "v_exp") if s[n] is not None]


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "rope":
        to = _TYPES[case["dst"]]
        return _turn(s, s["q"], s["q_weight"]).to(to), _turn(s, s["k"], s["k_weight"]).to(to)
    if op == "store":
        _put(s, "k", _turn(s, s["k"], s["k_weight"]))
        _put(s, "v", s["v"])
        return [_turn(s, s["q"], s["q_weight"]).to(_TYPES[case["dst"]])] + _held(s)
    if op == "write":
        _put(s, "k", s["k"])
        _put(s, "v", s["v"])
        return _held(s)
    if op == "read":
        return tuple(_got(s, n).to(torch.float32 if case["cache"] == "f32" else torch.bfloat16) for n in ("k", "v"))
    return _attend(s)


def _turn(s, x, weight):
    """RMS norm of every head with its weight, then the rotation by position * inv_freq, the angles in 64 bits."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight
    r = s["case"]["rot"]
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    c, n = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if s["case"]["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * c - b * n, b * c + a * n], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _put(s, name, x):
    """Rows of every token and head into the cache's slots."""
    page, row = s["slots"].long() // PAGE, s["slots"].long() % PAGE
    pool = s[name + "_pool"]
    if s[name + "_exp"] is None:
        pool[page, :, row] = x.to(pool.dtype)
    else:
        x, e = _to_fp8(x)
        pool.view(torch.uint8)[page, :, row] = x.view(torch.uint8)
        s[name + "_exp"][page, :, row] = e


def _paged(s, name, table):
    pool = s[name + "_pool"]
    return pool[table] if s[name + "_exp"] is None else pool.view(torch.uint8)[table].view(pool.dtype)


def _got(s, name):
    """Rows of every sequence in order, [sequences, KV heads, rows, d] in 32 bits, zeros behind a sequence's length."""
    table = s["page_table"].long()
    x = _paged(s, name, table).float()
    if s[name + "_exp"] is not None:
        x = x * _two(s[name + "_exp"][table])[..., None]
    x = x.transpose(1, 2).flatten(2, 3)[:, :, :s["case"]["kv"]]
    there = torch.arange(x.shape[2], device=x.device) < s["kv_len"][:, None]
    return torch.where(there[:, None, :, None], x, 0.0)


def _attend(s):
    case = s["case"]
    b, h, hk, d, most = case["batch"], case["heads"], case["kv_heads"], case["d"], s["most"]
    k, v = _got(s, "k"), _got(s, "v")
    n = k.shape[2]
    starts = s["q_start"].long()
    token = torch.arange(most, device=k.device)
    spot = (starts[:-1, None] + token).clamp(max=s["q"].shape[0] - 1)           # packed row of (sequence, drafted token)
    q = s["q"][spot].float().view(b, most, hk, h // hk, d).permute(0, 2, 1, 3, 4).reshape(b, hk, most * (h // hk), d)
    logits = (q @ k.transpose(-1, -2) / math.sqrt(d)).view(b, hk, most, h // hk, n)
    # which cache row a token sees: all of the context, and of its tree the tokens that its mask names
    place = torch.arange(n, device=k.device) - (s["kv_len"] - (starts[1:] - starts[:-1]))[:, None]   # row's index in the tree
    if s["tree_mask"] is None:
        sees = place[:, None] <= token[:, None]
    else:
        bit = place.clamp(min=0, max=most - 1)
        words = s["tree_mask"][spot]                                              # [b, most, words]
        word = torch.gather(words, 2, (bit // 64)[:, None].expand(-1, most, -1))
        sees = ((word >> (bit % 64)[:, None]) & 1).bool() | (place < 0)[:, None]
    sees = sees & (torch.arange(n, device=k.device) < s["kv_len"][:, None])[:, None]
    logits = torch.where(sees[:, None, :, None], logits, -torch.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    out = (p / total).view(b, hk, most * (h // hk), n) @ v
    lse = (torch.log(total) + top).squeeze(-1)
    out = out.view(b, hk, most, h // hk, d).permute(0, 2, 1, 3, 4).reshape(b * most, h, d)
    lse = lse.permute(0, 2, 1, 3).reshape(b * most, h)
    # back to packed rows
    owner = torch.searchsorted(starts, torch.arange(s["q"].shape[0], device=k.device), right=True) - 1
    back = owner * most + torch.arange(s["q"].shape[0], device=k.device) - starts[owner]
    return out[back].to(s["q"].dtype), lse[back]


# ------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op, d = case["op"], case["d"]
    if op in ("rope", "store"):
        r = case["rot"]
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["inv_freq"].double())

        def turned(x, w):
            x = x.double()
            if w is not None:
                x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / d + 1e-6) * w.double()
            out = x.clone()
            pairs = torch.complex(x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else torch.complex(x[..., :r // 2], x[..., r // 2:r])
            pairs = pairs * z[:, None]
            if case["interleaved"]:
                out[..., 0:r:2], out[..., 1:r:2] = pairs.real, pairs.imag
            else:
                out[..., :r // 2], out[..., r // 2:r] = pairs.real, pairs.imag
            return out

        q, k = turned(s["q"], s["q_weight"]), turned(s["k"], s["k_weight"])
        return (q, k) if op == "rope" else [q] + _held_exactly(s, k, s["v"].double())
    if op == "write":
        return _held_exactly(s, s["k"].double(), s["v"].double())
    lens, drafts = _sizes(case)
    hk, group = case["kv_heads"], case.get("heads", 0) // case["kv_heads"]
    rows = {}
    for name in ("k", "v"):
        for b, n in enumerate(lens):
            x = _paged(s, name, s["page_table"][b].long()).float().double()
            if s[name + "_exp"] is not None:
                x = x * torch.pow(torch.tensor(2.0, dtype=torch.float64, device="cuda"), s[name + "_exp"][s["page_table"][b].long()].double())[..., None]
            rows[name, b] = x.transpose(0, 1).reshape(hk, -1, d)[:, :n]
    if op == "read":
        got = []
        for name in ("k", "v"):
            whole = torch.zeros(len(lens), hk, case["kv"], d, dtype=torch.float64, device="cuda")
            for b, n in enumerate(lens):
                whole[b, :, :n] = rows[name, b]
            got.append(whole)
        return tuple(got)
    out = torch.zeros(sum(drafts), case["heads"], d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(sum(drafts), case["heads"], dtype=torch.float64, device="cuda")
    first = 0
    for b, (n, t) in enumerate(zip(lens, drafts)):
        sees = torch.ones(t, n, dtype=torch.bool, device="cuda")
        if s["tree_mask"] is None:
            sees[:, n - t:] = torch.ones(t, t, dtype=torch.bool, device="cuda").tril()
        else:
            at = torch.arange(t, device="cuda")
            sees[:, n - t:] = (s["tree_mask"][first:first + t][:, at // 64] >> (at % 64)) & 1 == 1
        for head in range(case["heads"]):
            k, v = rows["k", b][head // group], rows["v", b][head // group]
            w = (s["q"][first:first + t, head].double() @ k.T) / math.sqrt(d)
            w[~sees] = -torch.inf
            lse[first:first + t, head] = torch.logsumexp(w, -1)
            out[first:first + t, head] = torch.softmax(w, -1) @ v
        first += t
    return out, lse


def _held_exactly(s, k, v):
    """The cache after the write: FP8 rows before their rounding to e4m3, and their exponents."""
    page, row = torch.div(s["slots"].long(), PAGE, rounding_mode="floor"), s["slots"].long() % PAGE
    pools, exps = [], []
    for name, x in (("k", k), ("v", v)):
        pool = s[name + "_pool"].float().double()
        if s[name + "_exp"] is not None:
            top = x.abs().amax(-1)
            e = torch.ceil(torch.log2(top / 448)).nan_to_num(neginf=0.0)
            # the logarithm may be off by one step next to a whole number
            e = torch.where(top > 448 * torch.pow(2.0, e), e + 1, torch.where(top <= 448 * torch.pow(2.0, e - 1), e - 1, e))
            e = torch.where(top > 0, e, 0.0).clamp(-120, 120)
            x = x / torch.pow(2.0, e)[..., None]
            held = s[name + "_exp"].clone()
            held[page, :, row] = e.to(torch.int8)
            exps.append(held)
        pool[page, :, row] = x
        pools.append(pool)
    return pools + exps


if __name__ == "__main__":
    draws = random.Random(0)
    for c in listed() + [draw(draws) for _ in range(10)]:
        print(c, work(c))
