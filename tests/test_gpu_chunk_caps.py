"""Caps and scales at the ends of what chunk attention takes, with the comparison of test_gpu_chunk_strict."""
import pytest

from test_gpu_chunk_strict import Strict

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 3, 200])
@pytest.mark.parametrize("scale,cap", [(2.0 ** 26, 2.0 ** -100), (-2.0 ** 26, 2.0 ** -100), (2.0 ** 120, 2.0 ** -6), (2.0 ** -20, 2.0 ** 100), (2.0 ** -26, 2.0 ** 60), (0.0, 2.0 ** -100)])
def test_quotients_of_scale_and_cap_at_the_ends(cache, d, new, scale, cap):
    """scale / cap up to 2^126: queries times that leave fp32, the capped logits do not."""
    p = Strict([300, 130], [new, 100 if new > 2 else 1], 8, 2, d, cache, seed=20)
    p.q[:, 1] = 0                                                 # logits of 0 beside those at the cap
    # logits saturate, whatever their products' rounding: what is summed is exact enough without its term in the tolerance
    out, lse = p.run(scale=scale, softcap=cap)
    assert bool(out.isfinite().all()) and bool(lse.isfinite().all())
    if abs(scale) <= 1.0:
        p.check(out, lse, scale=scale, softcap=cap)
    elif cap < 1.0:
        # at most 2^-6 * 1.0002 either way: exp of that, against equal weights
        want, want_lse = p.run(scale=0.0)
        assert bool(((lse - want_lse).abs() <= 1.01 * cap + 2.0 ** -18).all())
        assert bool(((out.float() - want.float()).abs() <= 2.0 ** -3 * want.float().abs() + 2.0 ** -3).all())
