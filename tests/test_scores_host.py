"""Plans with scores of their own, on the CPU: refusals, position tables' limits, the order of the stream."""
import numpy as np
import pytest

from attention_reference import layout
from paper_2508_08895_b200 import binding as B

STEP = [(37, [(5, 1), (0, 2)], 0), (100, [(7, 1)], 0)]


def plan(step=STEP, mode=B.MODE_BRANCH, q_pos=None, page=16, heads=(4, 2), sm_scale=0.125, **kw):
    tune = {k: kw.pop(k) for k in ("mma_m", "mask", "n_ctas", "wide_rows") if k in kw}
    desc, n_pool, _ = layout(step, page)
    shape = B.make_shape(*heads, 128, page, "bf16", 1e4, sm_scale)
    return B.Plan(shape, desc, n_pool, mode, q_pos=q_pos, host_only=True, scores=B.Scores(**kw), **tune)


def status(**kw):
    with pytest.raises(B.AspdError) as e:
        plan(**kw)
    return e.value.status


def test_refusals():
    nan, inf = float("nan"), float("inf")
    for cap in (-1.0, nan, inf, -inf, 2e30, 1e-33):
        assert status(cap=cap) == -1, cap
    for bad in (nan, inf, -inf, 1e30, -32.1):
        assert status(slopes=[0.5, bad, 0.1, 0.1]) == -1, bad
    assert status(rotated=True, q_pos=np.zeros(4, np.int32)) == -1
    assert status(cap=30.0, mma_m=64) == -3 and status(slopes=[0.5] * 4, mma_m=64) == -3
    with pytest.raises(ValueError):
        plan(slopes=[0.5] * 3)
    for ok in (dict(), dict(cap=1e30), dict(cap=1e-20), dict(slopes=[32, -32, 0, 1e-40]), dict(rotated=True, mma_m=64), dict(cap=50.0, slopes=[1] * 4, mma_m=96)):
        assert plan(**ok).n_new == 4


def test_positions_of_a_bias():
    slopes = dict(slopes=[0.5] * 4)
    shared = [(20, [(9, -1), (0, 1)], 0)]
    assert status(step=shared, **slopes) == -2                            # an earlier stage's positions are the caller's to give
    assert plan(step=shared, cap=3.0).n_new == 1                          # (without a bias nobody needs them)
    assert plan(step=[(20, [(9, -1, 20), (0, 1)], 0)], **slopes).n_new == 1
    assert plan(step=[(20, [(0, -1), (0, 1)], 0)], **slopes).n_new == 1   # (an empty one has none)
    far = (1 << 24) - 5
    assert plan(step=[(20, [(4, 1, far)], 0)], **slopes).n_new == 1
    assert status(step=[(20, [(5, 1, far)], 0)], **slopes) == -7
    assert plan(step=[(20, [(5, 1, far)], 0)], cap=3.0).n_new == 1
    assert status(step=[(20, [(6, 0, far)], 3)], mode=B.MODE_SERIAL, **slopes) == -7
    assert plan(step=[(20, [(5, 0)], 3)], mode=B.MODE_SERIAL, **slopes).n_new == 1


@pytest.mark.parametrize("kw", [dict(), dict(n_ctas=1, wide_rows=128), dict(n_ctas=1, wide_rows=256)], ids=str)
def test_prefix_is_walked_from_its_end_with_a_bias(kw):
    """... and what the step reads and sees stays the same: pages, valid rows, ranges."""
    step = [(200, [(5, 30), (0, 20)], 0), (37, [(7, 1)], 0)]
    a, b = plan(step, **kw), plan(step, slopes=[0.5] * 4, **kw)
    pa, pb = a.stream_pages(), b.stream_pages()
    assert sorted(zip(*pa)) == sorted(zip(*pb))
    n = 13                                                                # pages of the first request's prefix
    np.testing.assert_array_equal(pa[0][:n][::-1], pb[0][:n])
    np.testing.assert_array_equal(pa[1][:n][::-1], pb[1][:n])
    for x, y in zip(a.token_ranges(), b.token_ranges()):
        np.testing.assert_array_equal(x, y)
    np.testing.assert_array_equal(a.items(), b.items())
