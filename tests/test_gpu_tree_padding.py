"""Tree attention of padded batches: tokens of no sequence, in results that the caller passes in."""
import pytest
import torch

import paper_2511_07427_b200 as P

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def _batch(cache, heads, tokens, padding, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = P.RowCache.allocate(8, 2, 128, cache)
    x = torch.randn(250, 2, 128, generator=g, device="cuda")
    c.write(x, x.flip(0), torch.arange(250, **I32))
    io = torch.float32 if cache == P.F32 else torch.bfloat16
    q = torch.randn(tokens + padding, heads, 128, generator=g, device="cuda").to(io)
    q[tokens:] = float("nan")
    return c, q, torch.arange(8, **I32).view(2, 4), torch.tensor([120, 97], **I32)


@pytest.mark.parametrize("cache", [P.F32, P.BF16, P.FP8])
@pytest.mark.parametrize("heads,tree", [(4, 3), (4, 20), (16, 20), (16, 40)])
def test_tokens_of_no_sequence_keep_what_out_and_lse_held(cache, heads, tree):
    """One captured call, replayed while q_start shrinks and moves: 5 and more tokens belong to no sequence."""
    n = 2 * tree
    c, q, table, lens = _batch(cache, heads, n, 5)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 9.0, device="cuda")
    start = torch.tensor([0, tree, n], **I32)

    def call(**kw):
        return c.attend_tree(q, table, lens, start, tree, **kw)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    for s in ([0, tree, n], [0, tree - 1, n - 2], [2, tree, tree], [1, 1, 2], [0, 0, 0]):
        start.copy_(torch.tensor(s))
        out.fill_(7.0)
        lse.fill_(9.0)
        graph.replay()
        want = call()
        own = slice(s[0], s[-1])
        assert torch.equal(out[own], want[0][own]) and torch.equal(lse[own], want[1][own])
        assert bool(torch.isfinite(out[own]).all()) and bool(torch.isfinite(lse[own]).all())
        for rest in (slice(0, s[0]), slice(s[-1], None)):
            assert bool((out[rest] == 7.0).all()) and bool((lse[rest] == 9.0).all())
    assert c.get_status() == 0


def test_refusals_of_results():
    c, q, table, lens = _batch(P.F32, 4, 6, 0)
    start = torch.tensor([0, 3, 6], **I32)
    flat = torch.zeros(2 * q.numel(), device="cuda")
    for kw in (dict(lse=torch.zeros(6, 4, dtype=torch.bfloat16, device="cuda")), dict(lse=torch.zeros(4, 6, device="cuda")), dict(lse=torch.zeros(6, 4)),
               dict(lse=torch.zeros(4, 6, device="cuda").t()), dict(out=q), dict(lse=q.view(-1)[:24].view(6, 4)),
               dict(out=flat[:q.numel()].view(q.shape), lse=flat[q.numel() - 4:q.numel() + 20].view(6, 4))):
        with pytest.raises(P.DynaKVError):
            c.attend_tree(q, table, lens, start, 3, **kw)
    with pytest.raises(P.DynaKVError, match="gradient"):
        c.attend_tree(q, table, lens, start, 3, lse=torch.zeros(6, 4, device="cuda", requires_grad=True))
    out, lse = c.attend_tree(q, table, lens, start, 3, out=flat[:q.numel()].view(q.shape), lse=flat[q.numel():q.numel() + 24].view(6, 4))
    want = c.attend_tree(q, table, lens, start, 3)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    shifted = flat[q.numel() // 2:][:q.numel()].view(q.shape)
    shifted.copy_(q)
    with pytest.raises(P.DynaKVError, match="memory"):
        c.attend_tree(shifted, table, lens, start, 3, out=flat[:q.numel()].view(q.shape))
