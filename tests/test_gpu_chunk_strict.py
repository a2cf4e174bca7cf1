"""The tests of chunk attention once more, with a comparison that a NaN cannot pass.

`Chunk.check` asks that no difference is above its bound, which a NaN is not: 0 * NaN of a row that nobody sees (rows that were not
written hold NaN there) would go unnoticed in the results.  Here every value of a token of a sequence is finite and every difference at most its bound,
with the tolerances derived in test_gpu_chunk."""
import math

import pytest
import torch

import test_gpu_chunk as base
from test_gpu_chunk import *                                      # noqa: F401,F403  (its tests, collected here with the class below)

pytestmark = pytest.mark.gpu
U = base.U


class Strict(base.Chunk):
    def check(self, out, lse, scale=None, softcap=0.0, window=0):
        scale = scale if scale is not None else self.d ** -0.5
        group, half = self.heads // self.hk, torch.finfo(out.dtype).eps / 2
        many = self.most * group > (32 if self.d == 128 else 64)
        grain = {"f32": 0.0, "bf16": 2.0 ** -8 if many else 2.0 ** -16, "fp8": 2.0 ** -8 if many else 2.0 ** -11}[self.cache]
        at = self.lead
        for b, (n, t) in enumerate(zip(self.lens, self.new)):
            place = self.place[at:at + t]
            low = torch.maximum(self.low[at:at + t], place + 1 - window) if window else self.low[at:at + t]
            row = torch.arange(n, device="cuda")
            for h in range(self.hk if t else 0):
                k, v, known = self.rows(b, h)
                see = (row >= low[:, None]) & (row < self.high[at:at + t, None]) & known
                k, v = (torch.where(torch.isfinite(x), x, 0.0) for x in (k, v))            # what no token sees; the tests have none that one does
                for hq in range(h * group, (h + 1) * group):
                    q = self.q[at:at + t, hq].double()
                    s = (q @ k.T) * scale
                    err = (self.d + 4) * U * (q.abs() @ k.abs().T) * abs(scale)
                    if softcap:
                        s = softcap * torch.tanh(s / softcap)
                        err = err + 2.0 ** -22 * softcap
                    if self.slopes is not None:
                        away = self.slopes[hq].double() * (place[:, None] - row).abs()
                        s = s - away
                        err = err + 6 * U * (away.abs() + self.slopes[hq].double().abs() * 128)
                    seen_err = torch.where(see, err + 4 * U * s.abs(), 0.0)
                    s = torch.where(see, s, -math.inf)
                    none = ~see.any(-1)
                    want_lse = torch.logsumexp(s, -1) if n else torch.full((t,), -math.inf, dtype=torch.float64, device="cuda")
                    w = torch.exp(s - torch.where(none, 0.0, want_lse)[:, None])
                    want, weight = w @ v, w @ v.abs()
                    eps = 2 * (seen_err.amax(-1) if n else torch.zeros(t, dtype=torch.float64, device="cuda")) + 2.0 ** -20
                    got, got_lse = out[at:at + t, hq].double(), lse[at:at + t, hq].double()
                    bound = (eps + grain + n * U)[:, None] * weight + half * want.abs() + 1e-30
                    assert bool(torch.isfinite(bound).all()) and bool(torch.isfinite(got).all()), (b, hq, int((~torch.isfinite(got)).sum()))
                    assert bool(((got - want).abs() <= bound).all()), (b, hq, float(((got - want).abs() / bound).max()))
                    assert not got[none].any() and bool((got_lse[none] == -math.inf).all())
                    assert bool(((got_lse - want_lse).abs() <= eps + n * U + 2 * U * want_lse.abs())[~none].all()), (b, hq)
            at += t
        assert self.c.get_status() == 0


@pytest.fixture(autouse=True)
def strict(monkeypatch):
    monkeypatch.setattr(base, "Chunk", Strict)


def test_the_check_refuses_nan():
    p = Strict([40], [3], 2, 1, 64, "f32")
    out, lse = p.run()
    p.check(out, lse)
    out[1, 1, 5] = math.nan
    with pytest.raises(AssertionError):
        p.check(out, lse)
