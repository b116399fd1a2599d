"""Plans whose scores are capped by a tanh, get a distance bias, or whose queries and keys come rotated: every attention kernel,
step and call against the definition in 64 bits (bounds: attention_reference.py)."""
import numpy as np
import pytest

from attention_reference import Scene, alibi
from paper_2508_08895_b200 import binding as B

pytestmark = pytest.mark.gpu

DECODE = [(37, [(5, 1), (0, 1), (30, 1)], 0), (300, [(16, 1)], 0), (0, [(3, 1), (8, 0)], 0)]
LONG = [(1500, [(40, 1), (0, 1), (15, 1), (129, 1)], 0)]
OPEN = [(130, [(0, 5), (7, 3)], 0), (16, [(0, 9)], 0)]
WHOLE = [(70, [(0, 33), (4, 40), (0, 1)], 0), (200, [(0, 20)], 0)]
SERIAL = [(129, [(40, 0), (3, 0)], 5), (0, [], 1), (333, [(17, 0)], 40)]
ONE = [(0, [(0, 1)], 0)]
STEPS = dict(decode=DECODE, long=LONG, open=OPEN, whole=WHOLE, serial=SERIAL, one=ONE)
KINDS = {"cap": dict(cap=20.0, q_scale=5.0), "bias": dict(bias=True), "both": dict(cap=30.0, bias=True, q_scale=5.0),
         "both-rotated": dict(cap=20.0, bias=True, rotated=True, q_scale=5.0), "rotated": dict(rotated=True)}
TC = ("bf16", 128, 16, (28, 4))
# shape -> what its kernel rounds (turned queries, weights): only the kernel of heads of 128 in pages of 16
SMALL = [("bf16", 64, 16, (14, 2)), ("bf16", 128, 8, (28, 4)), ("bf16", 128, 32, (8, 1)), ("bf16", 64, 8, (4, 4)), ("bf16", 64, 32, (64, 1))]
CORES = [("f32", 64, 16, (4, 1)), ("f32", 128, 8, (28, 4)), ("f32", 64, 32, (16, 8)), ("f32", 128, 32, (64, 2))]


def scene(shape, step, kind, **more):
    kw = dict(KINDS[kind])
    if kw.pop("bias", False):
        kw["slopes"] = alibi(shape[3][0])
    return Scene(*shape, step, **{**kw, **more})


def bits(shape, **kw):
    tc = shape[0] == "bf16" and shape[1:3] == (128, 16) and kw.get("kernel") != B.KERNEL_GENERIC
    return dict(q_bits=8, p_bits=8) if tc else dict(q_bits=0, p_bits=0)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("step", list(STEPS))
@pytest.mark.parametrize("shape", [TC, ("bf16", 128, 16, (64, 1)), ("bf16", 128, 16, (4, 4)), *SMALL, *CORES], ids=str)
def test_steps(shape, step, kind):
    s = scene(shape, STEPS[step], kind)
    s.step()
    s.check(**bits(shape))


@pytest.mark.parametrize("kind", ["cap", "both", "both-rotated"])
@pytest.mark.parametrize("step,kw", [("long", dict(n_ctas=1)), ("long", dict(n_ctas=5)), ("long", dict(mma_m=128)), ("long", dict(combine=B.COMBINE_FUSED)),
                                     ("decode", dict(combine=B.COMBINE_FUSED, n_ctas=3)), ("long", dict(chunk_tokens=64)), ("long", dict(kernel=B.KERNEL_GENERIC)),
                                     ("whole", dict(n_ctas=2)), ("whole", dict(n_ctas=2, wide_rows=128)), ("whole", dict(n_ctas=1, wide_rows=256)),
                                     ("open", dict(n_ctas=1, wide_rows=128)), ("open", dict(n_ctas=2, stable_cache=True)), ("serial", dict(n_ctas=2)),
                                     ("decode", dict(stable_cache=True)), ("whole", dict(kernel=B.KERNEL_GENERIC))], ids=str)
def test_variants_of_the_tensor_core_kernel(step, kw, kind):
    s = scene(TC, STEPS[step], kind)
    s.step(**kw)
    s.check(**bits(TC, **kw))


@pytest.mark.parametrize("kw", [dict(n_ctas=1), dict(n_ctas=2), dict(chunk_tokens=32)], ids=str)
@pytest.mark.parametrize("shape", [SMALL[0], SMALL[1], CORES[1]], ids=str)
def test_cuts_of_the_other_kernels(shape, kw):
    for step in ("long", "whole"):
        s = scene(shape, STEPS[step], "both")
        s.step(**kw)
        s.check(**bits(shape))


@pytest.mark.parametrize("shape", [TC, SMALL[0], CORES[0]], ids=str)
def test_shared_mask(shape):
    s = scene(shape, [(50, [(20, 3), (5, 1), (30, 0), (0, 2)], 0)], "both", mask=B.MASK_SHARED)
    s.step()
    s.check(**bits(shape))


@pytest.mark.parametrize("shape", [TC, SMALL[1], CORES[0]], ids=str)
@pytest.mark.parametrize("kw", [dict(), dict(n_ctas=1)], ids=str)
def test_regions_of_earlier_stages_and_given_positions(shape, kw):
    """Their positions are the caller's; branches with positions of their own (far ones too)."""
    for step in ([(20, [(9, -1, 20), (5, -1, 20), (18, -1, 34), (0, 3), (4, 1)], 0)], [(33, [(9, -1, 33), (20, 0, 5000), (3, 0)], 7)],
                 [(40, [(5, 2, 100), (0, 1, 3000000), (9, 1)], 0)]):
        s = scene(shape, step, "both")
        s.step(**kw)
        s.check(**bits(shape))


@pytest.mark.parametrize("shape", [TC, SMALL[0], CORES[1]], ids=str)
def test_steep_flat_and_rising_slopes(shape):
    """Slopes that leave a row only its nearest keys, none, and ones that favour the far end."""
    hq = shape[3][0]
    slopes = np.resize([30.0, 0.0, -0.02, 1e-6, 32.0, -0.5, 2.0], hq)
    for step in ("long", "whole", "serial"):
        for kw in (dict(), dict(n_ctas=2)):
            s = Scene(*shape, STEPS[step], slopes=slopes)
            s.step(**kw)
            s.check(**bits(shape))


@pytest.mark.parametrize("shape", [TC, SMALL[1], CORES[1]], ids=str)
@pytest.mark.parametrize("cap,q_scale", [(0.5, 20.0), (2.0, 300.0), (50.0, 40.0)])
def test_saturated_caps(shape, cap, q_scale):
    """Scores far beyond the cap: tanh at its ends."""
    s = Scene(*shape, STEPS["long"], cap=cap, q_scale=q_scale, v_mean=1.0)
    s.step()
    s.check(**bits(shape))


@pytest.mark.parametrize("shape", [TC, *SMALL[:2], CORES[0]], ids=str)
def test_calls_apart_host_step_static_and_graph(shape):
    """kv_append + attention, the step from host memory, the static scratch, an updated plan in a replayed graph: the fused
    step's outputs."""
    import torch
    for kind in ("both", "both-rotated"):
        s = scene(shape, STEPS["decode"], kind)
        pools = s.k_pool.clone(), s.v_pool.clone()
        plan = s.step()
        want = s.out.clone()
        same = lambda: (s.out.double() - want.double()).abs().max().item() <= 2.0 ** -7 * want.abs().max().item()   # noqa: E731
        pos = B.positions(s.desc, s.mode)[0] * (0 if s.rotated else 1)

        s.k_pool, s.v_pool = (x.clone() for x in pools)
        s.out.zero_()
        B.kv_append(plan, s.k, s.v, torch.from_numpy(pos.copy()).cuda(), s.k_pool, s.v_pool)
        B.branch_attn(plan, s.q, s.k_pool, s.v_pool, s.out)
        torch.cuda.synchronize()
        assert same()
        s.check(**bits(shape))

        s.k_pool, s.v_pool = (x.clone() for x in pools)
        host = [x.cpu().pin_memory() for x in (s.q, s.k, s.v)]
        out = torch.zeros_like(host[0]).pin_memory()
        B.step_host(plan, *host, B.positions(s.desc, s.mode)[0].copy(), s.k_pool, s.v_pool, out)      # (rotated: whatever they are)
        s.out.copy_(out)
        assert same()

        s.out.zero_()
        B.attn_static(s.plan(host_only=True), s.q, s.k_pool, s.v_pool, s.out)
        torch.cuda.synchronize()
        assert B.static_status() == 0 and same()


def test_updated_plan_in_a_graph():
    import torch
    s = scene(TC, [(100, [(20, 1), (7, 1)], 0), (700, [(33, 1)], 0)], "both")
    plan = s.plan(updatable=True)
    s.step(plan)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.branch_step(plan, s.q, s.k, s.v, s.k_pool, s.v_pool, s.out)
    later = scene(TC, [(100, [(24, 1), (11, 1)], 0), (700, [(37, 1)], 0)], "both", seed=6)
    assert later.n_pool == s.n_pool
    for name in ("q", "k", "v", "k_pool", "v_pool"):
        getattr(s, name).copy_(getattr(later, name))
    plan.update(later.desc)
    s.out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert plan.status() == 0
    later.k_pool, later.v_pool, later.out = s.k_pool, s.v_pool, s.out
    later.check(**bits(TC))


def test_refused_updates_leave_the_plan_as_it_is():
    """q_pos for rotated queries; positions with which the references can no longer be fixed (another kernel instance)."""
    s = scene(TC, DECODE, "rotated")
    plan = s.plan(updatable=True)
    with pytest.raises(B.AspdError) as e:
        plan.update(s.desc, q_pos=np.zeros(s.n, np.int32))
    assert e.value.status == -1
    s.step(plan)
    s.check(**bits(TC))

    s = scene(TC, [(100, [(20, -1, 100), (7, 1, 300)], 0)], "both")
    plan = s.plan(updatable=True)
    later = scene(TC, [(100, [(20, -1, 400), (7, 1, 300)], 0)], "both")       # keys later than the query
    with pytest.raises(B.AspdError) as e:
        plan.update(later.desc)
    assert e.value.status == -3
    s.step(plan)
    s.check(**bits(TC))
    later.step()
    later.check(**bits(TC))


@pytest.mark.parametrize("shape", [TC, SMALL[0], SMALL[1], CORES[0]], ids=str)
@pytest.mark.parametrize("cap", [1e-3, 54.0, 57.0, 1e4, 1e30])
def test_the_smallest_and_largest_caps(shape, cap):
    """Caps around the limit of fixed references, ones that the scores never come near, one that leaves weights all alike."""
    for step in ("long", "whole"):
        for kw in (dict(), dict(n_ctas=2)):
            s = Scene(*shape, STEPS[step], cap=cap, q_scale=5.0)
            s.step(**kw)
            s.check(**bits(shape))


def test_branches_that_start_at_different_positions_under_the_shared_mask():
    for shape in (TC, SMALL[0], CORES[0]):
        s = scene(shape, [(50, [(20, 3), (5, 1, 900), (30, 0, 4), (0, 2)], 0)], "both", mask=B.MASK_SHARED)
        s.step()
        s.check(**bits(shape))


@pytest.mark.parametrize("shape", [TC, SMALL[1], CORES[1]], ids=str)
def test_pages_beyond_four_gigabytes(shape):
    """Pools whose byte offsets pass 32 bits: the same step with its pages at their far ends, norms and all."""
    import torch
    near = Scene(*shape, OPEN, cap=20.0, slopes=alibi(shape[3][0]), rotated=True, q_scale=5.0)
    page = B.pool_bytes(near.shape, 1)
    n_pool = (9 << 29) // page + near.n_pool                      # 4.5 GiB and a step
    dt = near.q.dtype
    pools = [torch.zeros(n_pool * page // near.q.element_size(), dtype=dt, device="cuda") for _ in "kv"]
    first = n_pool - near.n_pool
    for big, small in zip(pools, (near.k_pool, near.v_pool)):
        big[first * page // near.q.element_size():] = small
    far = dict(near.desc, page_ids=near.desc["page_ids"] + np.int32(first))
    plan = B.Plan(near.shape, far, n_pool, near.mode, scores=near.scores)
    nm = B.QkNorm(near.shape, torch.ones(near.d, dtype=dt, device="cuda"), None, 1e-6)
    pos = torch.from_numpy(B.positions(far, near.mode)[0].copy()).cuda()
    q = near.q.clone()
    B.qk_norm_append(plan, nm, q, near.k, near.v, pos, *pools, near.q)
    B.branch_attn(plan, near.q, *pools, near.out)
    torch.cuda.synchronize()
    assert plan.status() == 0
    near.k_pool, near.v_pool = (big[first * page // near.q.element_size():].clone() for big in pools)
    assert all(not big[:first * page // near.q.element_size()].any() for big in pools)
    near.check(**bits(shape))


def test_two_streams_and_a_replayed_graph_of_whole_branches():
    """The two-tile kernel's instances side by side on two streams, each with a plan of its own; the same, captured and replayed."""
    import torch
    scenes = [Scene(*TC, WHOLE, q_scale=5.0, cap=cap, slopes=sl, seed=seed) for cap, sl, seed in ((20.0, None, 1), (30.0, alibi(28), 2))]
    streams = [torch.cuda.Stream() for _ in scenes]
    plans = [s.plan(n_ctas=2, stream=st) for s, st in zip(scenes, streams)]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, p, st in zip(scenes, plans, streams):
            B.branch_step(p, s.q, s.k, s.v, s.k_pool, s.v_pool, s.out, stream=st)
    torch.cuda.synchronize()
    for s, p in zip(scenes, plans):
        assert p.status() == 0
        s.check(**bits(TC))
        s.out.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for s, p in zip(scenes, plans):
            B.branch_step(p, s.q, s.k, s.v, s.k_pool, s.v_pool, s.out)
    for s in scenes:
        s.q.neg_()
    graph.replay()
    torch.cuda.synchronize()
    for s in scenes:
        s.check(**bits(TC))


def test_a_step_without_queries():
    s = scene(TC, [(40, [(20, 0), (9, 0)], 0)], "both")
    plan = s.plan()
    assert plan.n_new == 0
    B.branch_step(plan, s.q, s.k, s.v, s.k_pool, s.v_pool, s.out)
    import torch
    nm = B.QkNorm(s.shape)
    B.qk_norm_append(plan, nm, s.q, s.k, s.v, torch.zeros(1, 0, dtype=torch.int32, device="cuda"), s.k_pool, s.v_pool, s.out)
    torch.cuda.synchronize()


@pytest.mark.parametrize("shape", [TC, *SMALL, *CORES], ids=str)
@pytest.mark.parametrize("kind", ["cap", "both"])
def test_infinities_and_nan_of_keys_that_a_row_does_not_see(shape, kind):
    """A sibling branch's keys (and, but in the kernel of heads of 128 in pages of 16, its values), rows of a page that nobody has
    written: rows that do not see them do not change."""
    step = [(40, [(20, 1), (9, 1), (33, 1)], 0)]
    for kw in (dict(), dict(n_ctas=1)):
        clean, dirty = (scene(shape, step, kind) for _ in range(2))
        clean.step(**kw)
        first, length = dirty.reqs[0][2][:2]
        ids = dirty.desc["page_ids"]
        from pool_format import elements
        for slot, value in ((first + 2, float("nan")), (first + 4, float("inf")), (first + 5, -float("inf"))):
            at = elements([ids[slot // dirty.page]], [slot % dirty.page], dirty.hkv, dirty.page, dirty.d, B._esize(dirty.shape))
            at = dirty.torch.from_numpy(at.reshape(-1)).cuda()
            dirty.k_pool[at] = value
            if shape != TC:
                dirty.v_pool[at] = value
        dirty.step(**kw)
        for t in (0, 2):                # the tokens of the other branches (one each)
            a, b = clean.out[t].double(), dirty.out[t].double()
            assert dirty.torch.isfinite(b).all()
            assert (a - b).abs().max() <= 2.0 ** -7 * a.abs().max()
        assert not dirty.torch.isfinite(dirty.out[1]).all()


def test_plain_scores_are_the_plain_plan():
    """cap 0, no slopes, not rotated: bit for bit the plan without scores."""
    s = Scene(*TC, DECODE)
    s.step()
    want = s.out.clone()
    s.scores = None
    s.step()
    assert s.torch.equal(want, s.out)


def test_a_layer_with_normalised_heads_and_three_axes():
    """qk_norm_append and the attention over what it wrote: a packed projection, turned queries, capped scores."""
    import torch
    import test_gpu_qk_norm as N
    for shape in (N.SHAPES[0], N.SHAPES[1], N.SHAPES[6]):
        c = N.Case(shape, "ragged")
        s = Scene(c.dtype, c.d, c.page, (c.hq, c.hkv), [(p, list(b), 0) for p, b in N.STEPS["ragged"]], cap=15.0, slopes=alibi(c.hq), rotated=True)
        s.desc["page_ids"], s.n_pool = c.desc["page_ids"], c.n_pool
        s.shape = c.shape                        # (its theta)
        c.plan = s.plan()
        c.call()
        out = torch.empty_like(c.q_out)
        B.branch_attn(c.plan, c.q_out, *c.pool, out)
        c.check()
        s.q, s.k_pool, s.v_pool, s.out = c.q_out, *c.pool, out
        s.check(**bits(shape))
