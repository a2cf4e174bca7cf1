"""Verification of drafts where sums in 32 bits do not tell: siblings that have all of the weight between them, and random numbers next to a draft's chance."""
import math

import numpy as np
import pytest
import torch

import paper_2511_07427_b200 as P
from test_gpu_drafts import compare, drafts, ints, verified

pytestmark = pytest.mark.gpu
LAST = 1 - 2.0 ** -24                                             # the largest number below 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [40, 5003, 128256])
@pytest.mark.parametrize("open_tokens", [2, 3, 30])
def test_siblings_that_hold_all_the_weight(dtype, vocab, open_tokens):
    """All tokens that are not masked are drafted behind the root, with the largest random number: the last one is accepted, whatever the others leave."""
    g = torch.Generator(device="cuda").manual_seed(vocab + open_tokens)
    for seed in range(6):
        batch, size = 5, open_tokens + 3
        logits = torch.full((batch * size, vocab), -math.inf, device="cuda")
        tokens, parent = torch.zeros(batch, size, dtype=torch.int32, device="cuda"), [-1] + [0] * open_tokens + [open_tokens] * 2
        for b in range(batch):
            at = torch.randperm(vocab, generator=g, device="cuda")[:open_tokens]
            logits[b * size, at] = torch.randn(open_tokens, generator=g, device="cuda") * (3.0 if seed % 2 else 0.5)
            tokens[b, 1:open_tokens + 1] = at[torch.randperm(open_tokens, generator=g, device="cuda")].to(torch.int32)
            logits[b * size + 1:(b + 1) * size] = torch.randn(size - 1, vocab, generator=g, device="cuda")
        a = dict(logits=logits.to(dtype), tokens=tokens.view(-1), q_start=ints(np.arange(batch + 1) * size), max_tree=size, parent=ints(parent * batch), draft_probs=None,
                 uniform=torch.full((batch * size,), LAST, device="cuda"))
        kept, _, path, following = compare(a, torch.tensor([1.0, 0.3, 2.0, 7.0, 1.0], device="cuda"))
        assert bool((kept >= 2).all()) and bool((following >= 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [33, 4097, 50257])
@pytest.mark.parametrize("shape,drawn", [("chain", False), ("chain", True), ("tree", False)])
def test_random_numbers_next_to_the_chance(dtype, vocab, shape, drawn):
    """Every draft's number is one of the two fp32 numbers around p(x) / (q(x) sum(p)), the sum without its older siblings' tokens."""
    sizes = [5, 8, 2, 13, 6, 3]
    a = drafts(sizes, vocab, dtype, shape, drawn, 3 * vocab)
    heat = torch.tensor([1.0, 0.7, 1.0, 0.6, 1.5, 4.0], device="cuda")
    starts, L = a["q_start"].tolist(), a["logits"].double().cpu().numpy()
    x, parent = a["tokens"].tolist(), a["parent"].tolist() if a["parent"] is not None else None
    chance = np.zeros(sum(sizes))
    for b, size in enumerate(sizes):
        gone = {}
        for i in range(1, size):
            at = starts[b] + i
            up = parent[at] if parent else i - 1
            row = L[starts[b] + up]
            w = np.exp((row - row.max()) / float(heat[b]))
            before = gone.setdefault(up, set())
            left = w.sum() - sum(w[t] for t in before)
            q = float(a["draft_probs"][at, x[at]]) if drawn else 1.0
            chance[at] = min(w[x[at]] / (q * left), LAST)
            before.add(x[at])
    near = chance.astype(np.float32)
    rng = np.random.default_rng(vocab)
    for seed in range(8):
        u = np.where(rng.random(len(near)) < 0.5, near, np.nextafter(near, np.float32(0) if seed % 2 else np.float32(1))).clip(0, np.float32(LAST)).astype(np.float32)
        compare(dict(a, uniform=torch.tensor(u, device="cuda")), heat)


def test_many_open_tests_in_one_tree():
    """Each of 255 siblings has the number next to its chance."""
    vocab, n = 3001, 256
    g = torch.Generator(device="cuda").manual_seed(4)
    logits = torch.randn(n, vocab, generator=g, device="cuda")
    tokens = torch.randperm(vocab, generator=g, device="cuda")[:n].to(torch.int32)
    w = np.exp(logits[0].double().cpu().numpy() - float(logits[0].max()))
    t = tokens.cpu().numpy()
    left = w.sum() - np.concatenate([[0.0], np.cumsum(w[t[1:]])])[:-1]
    chance = np.concatenate([[0.5], w[t[1:]] / left])
    for above in (True, False):
        u = np.nextafter(chance.astype(np.float32), np.float32(1 if above else 0))
        u = np.where(above & (u.astype(np.float64) <= chance), np.nextafter(u, np.float32(1)), u).astype(np.float32)
        a = dict(logits=logits, tokens=tokens, q_start=ints([0, n]), max_tree=n, parent=ints([-1] + [0] * 255), draft_probs=None, uniform=torch.tensor(u, device="cuda"))
        kept, _, path, _ = compare(a, torch.ones(1, device="cuda"))
        assert int(kept) == (1 if above else 2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,moved", [(50257, 1e-5), (4001, 1e-5), (4001, 1e-3), (128256, 1e-4)])
def test_a_draft_that_was_drawn_from_nearly_the_target(dtype, vocab, moved):
    """q is the target's own softmax in fp32 but for a little weight moved onto the draft: what a refused draft leaves is that little and the roundings of q."""
    batch = 48
    g = torch.Generator(device="cuda").manual_seed(vocab)
    logits = (2.0 * torch.randn(2 * batch, vocab, generator=g, device="cuda")).to(dtype)
    q = torch.softmax(logits.float(), -1)[::2].repeat_interleave(2, 0)
    x = torch.randint(vocab, (batch,), generator=g, device="cuda")
    rows = torch.arange(batch, device="cuda")
    from_ = q[1::2].argmax(-1)
    from_ = torch.where(from_ == x, (from_ + 1) % vocab, from_)
    q[1 + 2 * rows, from_] -= moved
    q[1 + 2 * rows, x] += moved
    tokens = torch.stack([torch.zeros_like(x), x], 1).view(-1).to(torch.int32)
    u = torch.rand(2 * batch, generator=g, device="cuda")
    u[1::2] = LAST
    a = dict(logits=logits, tokens=tokens, q_start=ints(2 * np.arange(batch + 1)), max_tree=2, parent=None, draft_probs=q.contiguous(), uniform=u)
    for seed in range(4):
        u[0::2] = torch.rand(batch, generator=g, device="cuda")
        kept, _, _, _ = compare(a, torch.ones(batch, device="cuda"))
        assert int((kept == 1).sum()) > batch // 2
