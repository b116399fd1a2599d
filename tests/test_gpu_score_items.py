"""The two-tile kernel with capped scores, many items to a CTA: of one half of 64 keys and of several, with the second query tile and without.
An item's scores go over the weights of the item before it in tensor memory, and a half's over those of two halves before."""
import pytest

from attention_reference import Scene, alibi

pytestmark = pytest.mark.gpu

STEP = [(prefix, [(0, n), *more], 0) for prefix, n, more in (
    (0, 1, []), (0, 20, []), (5, 19, [(3, 2)]), (70, 40, []), (200, 3, []), (0, 36, []), (64, 37, []), (16, 2, [(0, 1), (30, 1)]), (0, 19, []), (130, 65, [(1, 8)]),
    (3, 1, []), (48, 30, []), (0, 64, []), (333, 1, []))]


@pytest.mark.parametrize("n_ctas", [1, 3])
@pytest.mark.parametrize("kw", [dict(cap=20.0), dict(cap=20.0, rotated=True), dict(cap=50.0, slopes=alibi(28)), dict(cap=50.0, slopes=alibi(28), rotated=True)], ids=str)
def test_items_in_a_row(kw, n_ctas):
    s = Scene("bf16", 128, 16, (28, 4), STEP, q_scale=5.0, **kw)
    plan = s.plan(wide_rows=256, n_ctas=n_ctas)
    assert (plan.info.dealt, plan.info.max_rows_per_item) == (1, 256)
    s.step(plan)
    s.check()
    want = s.out.clone()
    for _ in range(20):
        s.out.zero_()
        s.step(plan)
        assert s.torch.equal(s.out, want)
