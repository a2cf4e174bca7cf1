"""Sines and cosines of the rotary embedding, taken out of it by rotating unit pairs.

Tolerance.  The reduced angle is good to 2^-51 of the whole one.  sincospif is off by at most one unit in the last place (its
documented bound), 2^-24 for results of [0.5, 1) and less below; adding the angle's remainder rounds once more, 2^-25.  The
products with 1 and 0 are exact.  Together 1.5 * 2^-24."""
import pytest
import torch

import paper_2511_07427_b200 as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,rot,interleaved", [(128, 128, False), (64, 64, False), (128, 128, True), (128, 48, False), (64, 16, True)])
@pytest.mark.parametrize("far", [1, 64, 32768, 1 << 20, (1 << 31) - 1])
def test_sines_and_cosines(d, rot, interleaved, far):
    n = 2000
    g = torch.Generator(device="cuda").manual_seed(far % 1000 + d)
    inv_freq = (500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()
    pos = torch.randint(-far, far + 1, (n,), generator=g, device="cuda").to(torch.int32)
    a = torch.arange(0, rot, 2, device="cuda") if interleaved else torch.arange(rot // 2, device="cuda")
    b = a + 1 if interleaved else a + rot // 2
    q = torch.zeros(n, 1, d, device="cuda")
    q[..., a] = 1.0                                # (1, 0) becomes (cos, sin)
    k = torch.zeros(n, 1, d, device="cuda")
    k[..., b] = 1.0                                # (0, 1) becomes (-sin, cos)
    qo, ko = P.HeadRotary(1, 1, d, inv_freq, interleaved=interleaved).apply(q, k, pos)
    angle = pos.double()[:, None] * inv_freq.double()
    c, s = torch.cos(angle), torch.sin(angle)
    tol = 1.5 * 2.0 ** -24 + 2.0 ** -51 * angle.abs()
    for got, want in ((qo[:, 0, a], c), (qo[:, 0, b], s), (ko[:, 0, a], -s), (ko[:, 0, b], c)):
        assert ((got.double() - want).abs() - tol).max().item() <= 0, ((got.double() - want).abs().max().item() * 2 ** 24)
    assert not qo[..., rot:].any() and not ko[..., rot:].any()
