"""A capped row's output is made of what the row sees and of nothing else: bit for bit the same whatever ran before, whatever lies in keys that it
does not see (sibling branches, rows of a page that nobody has written), and whatever the other rows of its tile ask.  (References that move are
moved a tile at a time, for all of its rows: there the last two are asked of steps of a single tile.)"""
import numpy as np
import pytest

from attention_reference import Scene, alibi
from paper_2508_08895_b200 import binding as B
from pool_format import elements

pytestmark = pytest.mark.gpu

# odd numbers of pages, pages that end early
SHORT = [(20, [(3, 1), (9, 1), (5, 1)], 0), (5, [(3, 1)], 0)]
DECODE = [(37, [(20, 1), (9, 1), (33, 1)], 0), (5, [(3, 1)], 0)]
LONG = [(1500, [(40, 1), (0, 1), (15, 1), (129, 1)], 0)]
WHOLE = [(70, [(0, 33), (4, 40), (0, 1)], 0), (200, [(0, 20)], 0)]
TC = ("bf16", 128, 16, (28, 4))
CASES = [(TC, DECODE, {}), (TC, DECODE, dict(n_ctas=1)), (TC, LONG, {}), (TC, LONG, dict(n_ctas=2)), (TC, WHOLE, {}), (TC, WHOLE, dict(n_ctas=1, wide_rows=256)),
         (TC, WHOLE, dict(n_ctas=2, wide_rows=128)), (("bf16", 128, 16, (8, 1)), DECODE, {}), (("bf16", 64, 16, (14, 2)), DECODE, {}),
         (("bf16", 128, 8, (28, 4)), DECODE, {}), (("bf16", 128, 32, (8, 1)), LONG, {}), (("bf16", 64, 32, (64, 1)), WHOLE, {}), (("f32", 64, 16, (4, 1)), DECODE, {})]
# scores on both sides of 0.6 of the cap and of the cap; above 55 (references that move), with a bias that raises logits
ONE_TILE = [(x, SHORT, {}) for x in (TC, ("bf16", 128, 16, (8, 1)), ("bf16", 64, 16, (14, 2)), ("bf16", 128, 8, (28, 4)), ("bf16", 64, 32, (64, 1)))]
KINDS = {"cap": dict(cap=20.0, q_scale=5.0), "turned": dict(cap=20.0, q_scale=5.0, rotated=True), "both": dict(cap=12.0, bias=1, q_scale=5.0),
         "both-turned": dict(cap=30.0, bias=1, q_scale=15.0, rotated=True), "moving": dict(cap=57.0, q_scale=30.0), "rising": dict(cap=12.0, bias=-0.03, q_scale=5.0, rotated=True),
         "bias": dict(bias=1)}
FIXED = [(*x, k) for x in CASES for k in ("cap", "turned", "both", "both-turned")]
SEEN = FIXED + [(*x, k) for x in ONE_TILE for k in ("moving", "rising", "bias")]


def scene(shape, step, kind, **more):
    kw = dict(KINDS[kind])
    bias = kw.pop("bias", 0)
    if bias:
        kw["slopes"] = bias * alibi(shape[3][0])
    return Scene(*shape, step, **{**kw, **more})


def unseen(s, request, region):
    """Element numbers of that region's keys and of every row behind a region's end."""
    at = []
    for r, regions in enumerate(s.reqs):
        ids = s.desc["page_ids"][s.desc["page_begin"][r]:]
        for i, (first, length, _, _) in enumerate(regions):
            end = -(-length // s.page) * s.page
            for slot in range(first if (r, i) == (request, region) else first + length, first + end):
                at.append(elements([ids[slot // s.page]], [slot % s.page], s.hkv, s.page, s.d, B._esize(s.shape)).reshape(-1))
    return s.torch.from_numpy(np.concatenate(at)).cuda()


def tokens(s):
    """(request, region) of every new token."""
    return [(r, i) for r, regions in enumerate(s.reqs) for i, x in enumerate(regions) for _ in range(max(0, x[3]))]


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("shape,step,kw", CASES, ids=str)
def test_launches_repeat(shape, step, kw, kind):
    """... with steps of far larger and far smaller scores in between, which leave theirs in tensor and shared memory."""
    s = scene(shape, step, kind)
    others = [scene(shape, x, k, q_scale=scale, seed=8) for x, k, scale in ((WHOLE, kind, 80.0), (DECODE, "turned", 1e-3), (LONG, kind, 20.0))]
    plan, plans = s.plan(**kw), [x.plan(**kw) for x in others]
    s.step(plan)
    want = s.out.clone()
    for other, p in zip(others, plans):
        other.step(p)
        s.out.zero_()
        s.step(plan)
        assert s.torch.equal(s.out, want)


@pytest.mark.parametrize("shape,step,kw,kind", SEEN, ids=str)
def test_keys_that_a_row_does_not_see(shape, step, kw, kind):
    """One branch's keys and values, and what lies behind the regions' ends, are others: the other branches' rows stay."""
    s = scene(shape, step, kind)
    plan = s.step(s.plan(**kw))
    want = s.out.clone()
    gen = s.torch.Generator().manual_seed(3)
    at = unseen(s, 0, 2)
    mine = [t for t, x in enumerate(tokens(s)) if x == (0, 2)]
    rest = [t for t, x in enumerate(tokens(s)) if x != (0, 2)]
    for scale in (30.0, 1e-3):
        for pool in (s.k_pool, s.v_pool):
            pool[at] = (s.torch.randn(at.numel(), generator=gen) * scale).to(pool.dtype).cuda()
        s.k[mine] = (s.torch.randn(s.k[mine].shape, generator=gen) * scale).to(s.k.dtype).cuda()
        s.step(plan)
        assert s.torch.equal(s.out[rest], want[rest])
        assert not s.torch.equal(s.out[mine], want[mine])


@pytest.mark.parametrize("shape,step,kw,kind", SEEN, ids=str)
def test_the_other_rows_of_a_tile(shape, step, kw, kind):
    """One token's queries are others, and one head's: the other rows stay."""
    s = scene(shape, step, kind)
    plan = s.step(s.plan(**kw))
    want, was = s.out.clone(), s.q.clone()
    for scale in (40.0, 1e-3):
        s.q.copy_(was)
        s.q[1] *= scale
        s.q[:, 1] *= scale
        s.step(plan)
        same = [t for t in range(s.n) if t != 1]
        heads = [h for h in range(s.hq) if h != 1]
        assert s.torch.equal(s.out[same][:, heads], want[same][:, heads])
        assert not s.torch.equal(s.out[1], want[1]) or KINDS[kind].get("cap") is None
