"""Which form the plans of capped scores take -- dealt whole, in row blocks of 256, 128 or 64, or cut -- on the CPU; and the one-tile wide kernel, which
takes them where queries come rotated only, on the GPU."""
import pytest

from attention_reference import alibi, layout
from paper_2508_08895_b200 import binding as B

OPEN = [(130, [(0, 5), (7, 3)], 0), (16, [(0, 9)], 0)]                    # (tests of the variants: test_gpu_scores.py)
WHOLE = [(70, [(0, 33), (4, 40), (0, 1)], 0), (200, [(0, 20)], 0)]
SMALL = [(70, [(0, 9), (4, 9)], 0)]                                       # 18 query tokens of seven heads: one tile
RISING = [-0.01] * 28


def form(step, d=128, page=16, cap=20.0, slopes=None, rotated=False, **kw):
    """(dealt, rows of a row block)"""
    desc, n_pool, _ = layout(step, page)
    plan = B.Plan(B.make_shape(28, 4, d, page, "bf16", 1e4, d ** -0.5), desc, n_pool, B.MODE_BRANCH, host_only=True, n_ctas=1,
                  scores=B.Scores(cap, slopes, rotated), **kw)
    return plan.info.dealt, plan.info.max_rows_per_item


@pytest.mark.parametrize("step,wide_rows,inside,turned,moving", [
    (WHOLE, 0, (1, 256), (1, 256), (0, 64)), (WHOLE, 256, (1, 256), (1, 256), (0, 64)), (WHOLE, 128, (0, 64), (1, 128), (0, 64)),
    (OPEN, 0, (0, 64), (1, 128), (0, 64)), (OPEN, 256, (1, 256), (1, 256), (0, 64)), (SMALL, 0, (0, 64), (1, 128), (0, 64)), (SMALL, 128, (0, 64), (1, 128), (0, 64))])
def test_forms_of_capped_plans(step, wide_rows, inside, turned, moving):
    """inside: the attention rotates the queries; moving: the same where references move (caps above 55, a bias that raises scores)."""
    for kw in (dict(), dict(slopes=alibi(28))):
        assert form(step, wide_rows=wide_rows, **kw) == inside
        assert form(step, wide_rows=wide_rows, rotated=True, **kw) == turned
    for kw in (dict(cap=57.0), dict(slopes=RISING)):
        assert form(step, wide_rows=wide_rows, **kw) == moving
        assert form(step, wide_rows=wide_rows, rotated=True, **kw) == (1, 128)


def test_forms_of_other_plans():
    """No cap: as plain plans; other heads and pages have row blocks of 64."""
    for kw in (dict(), dict(slopes=alibi(28)), dict(rotated=True)):
        assert form(WHOLE, cap=0.0, **kw) == (1, 256) and form(WHOLE, cap=0.0, wide_rows=128, **kw) == (1, 128)
    for kw in (dict(d=64), dict(page=8), dict(page=32)):
        assert form(WHOLE, **kw) == (1, 64) and form(WHOLE, rotated=True, **kw) == (1, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [dict(cap=20.0), dict(cap=20.0, slopes=alibi(28)), dict(cap=57.0), dict(cap=20.0, slopes=alibi(28) * -0.02), dict(slopes=alibi(28))], ids=str)
@pytest.mark.parametrize("step,wide_rows,n_ctas", [(OPEN, 0, 1), (SMALL, 0, 1), (WHOLE, 128, 2)])
def test_the_one_tile_wide_kernel(step, wide_rows, n_ctas, kw):
    from attention_reference import Scene
    s = Scene("bf16", 128, 16, (28, 4), step, rotated=True, q_scale=5.0 if kw.get("cap") else 1.0, **kw)
    plan = s.plan(wide_rows=wide_rows, n_ctas=n_ctas)
    assert (plan.info.dealt, plan.info.max_rows_per_item) == (1, 128)
    s.step(plan)
    s.check()
