"""Tree attention of more sequences than a warp plans at once, on every kernel."""
import pytest

from test_gpu_tree import Problem

pytestmark = pytest.mark.gpu


# query rows per KV head (drafts x heads per KV head): tcgen05 in tiles of 128 and of 256, then 32 and 64 rows and few rows
@pytest.mark.parametrize("cache,most,heads,hk,d", [("bf16", 20, 4, 1, 128), ("bf16", 40, 4, 1, 128), ("bf16", 40, 8, 1, 64), ("fp8", 20, 4, 1, 128), ("fp8", 40, 4, 1, 128),
                                                   ("fp8", 70, 2, 1, 64), ("fp8", 16, 8, 2, 64), ("fp8", 4, 8, 1, 128), ("bf16", 4, 8, 1, 64), ("f32", 12, 4, 1, 64), ("f32", 1, 4, 2, 128)])
@pytest.mark.parametrize("seqs,tree", [(33, True), (400, False), (600, True)])
def test_many_sequences(cache, most, heads, hk, d, seqs, tree):
    lens = [0 if b % 11 == 4 else 1 + (b * 37) % 90 for b in range(seqs)]
    lens[seqs // 2] = 1500                                   # one long one, cut between several blocks
    drafts = [0 if b % 7 == 3 else 1 + (b * 5) % most for b in range(seqs)]
    drafts[-1] = most
    p = Problem(lens, drafts, heads, hk, d, cache, tree=tree, seed=17)
    p.check(*p.run())
