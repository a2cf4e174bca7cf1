"""Tree attention over FP8 rows where a few rows outweigh all others by 2^14 to 2^26 and hold nothing in some columns: those
columns are made of small weights alone.

Tolerance, relative to sum w |v| of the element.  The weights' f16 half step, 2^-12, which is relative as long as a weight is
a normal f16 value; every logit is one product (off by 4 * 2^-24 of at most 18.1, twice because the sum of weights has it
too: 2^-16), the exponential 2^-21, the merge of at most 296 records 2^-15: together below 2^-12 + 2^-13.  The fp32 sums over
`share` rows that one warp sees: share / 16 products of 16 rows, each off by 2^-23 at most, and share / 4 additions of
weights per lane.  The output's own rounding is half a step."""
import math

import pytest
import torch

import paper_2511_07427_b200 as P

pytestmark = pytest.mark.gpu

# head dim, query heads, tokens: 1, 4, 16, 32, 64 and 64 query rows on mma.sync, 80 on tcgen05
FORMS = [(128, 1, 1), (64, 4, 1), (128, 8, 2), (128, 8, 4), (64, 8, 8), (128, 8, 8), (128, 8, 10)]


def _run(d, heads, tokens, n, every, gap, v_up, seqs, share):
    g = torch.Generator(device="cuda").manual_seed(31)
    pages = (n + 31) // 32
    c = P.RowCache.allocate(pages, 1, d, P.FP8)
    large = torch.arange(n, device="cuda") % every == 5
    k = torch.zeros(n, 1, d, device="cuda")
    k[large, :, 0] = 16.0
    v = 0.5 + 0.5 * torch.rand(n, 1, d, generator=g, device="cuda")
    v[large] *= 2.0 ** v_up
    v[large, :, :9] = 0.0                     # columns that the large rows do not touch
    c.write(k, v, torch.arange(n, dtype=torch.int32, device="cuda"))
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None].repeat(seqs, 1)         # all sequences have the same rows
    lens = torch.full((seqs,), n, dtype=torch.int32, device="cuda")
    q = torch.zeros(tokens, heads, d, dtype=torch.bfloat16, device="cuda")
    # the whole gap, or parts of it
    q[..., 0] = torch.tensor([1.0, 0.75, 1.0, 0.5], dtype=torch.bfloat16, device="cuda")[torch.arange(tokens * heads, device="cuda") % 4].view(tokens, heads)
    scale = gap * math.log(2.0) / 16
    q_start = torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * tokens
    out, lse = c.attend_tree(q.repeat(seqs, 1, 1), table, lens, q_start, tokens, scale=scale)
    assert c.get_status() == 0
    K, V = c.read(table[:1], lens[:1], n)
    K, V = K[0, 0].double(), V[0, 0].double()
    sees = torch.arange(n, device="cuda") < n - tokens + 1 + torch.arange(tokens, device="cuda")[:, None]
    s = (q.double().view(-1, d) @ K.T).view(tokens, heads, n) * torch.tensor(scale, dtype=torch.float32).double().item()
    s = torch.where(sees[:, None], s, -math.inf)
    want_lse = torch.logsumexp(s, -1)
    want = torch.exp(s - want_lse[..., None]) @ V             # no value is negative: also the sum of w |v|
    sums = share * (2.0 ** -27 + 2.0 ** -26)
    tol = (2.0 ** -12 + 2.0 ** -13 + sums + torch.finfo(out.dtype).eps / 2) * want
    worst = ((out.double().view(seqs, tokens, heads, d) - want).abs() / tol).amax().item()
    assert worst <= 1, worst
    assert (lse.double().view(seqs, tokens, heads) - want_lse).abs().max().item() <= 2.0 ** -15 + sums + 2.0 ** -22 * want_lse.abs().max().item()


@pytest.mark.parametrize("d,heads,tokens", FORMS)
@pytest.mark.parametrize("gap,v_up", [(14.0, 0), (24.6, 0), (25.5, 0), (26.0, 0), (14.5, 11), (5.5, 20)])
def test_small_weights_beside_a_large_one_in_every_page(d, heads, tokens, gap, v_up):
    _run(d, heads, tokens, 4100, 32, gap, v_up, 1, 160)


@pytest.mark.parametrize("d,heads,tokens", FORMS)
@pytest.mark.parametrize("gap", [24.6, 25.5])
def test_one_row_beside_many(d, heads, tokens, gap):
    """As many sequences as blocks run at once, so that one warp sees a third of a sequence's rows or all of them."""
    _run(d, heads, tokens, 1 << 17, 1 << 17, gap, 0, 296, 1 << 17)
