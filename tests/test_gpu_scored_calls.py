"""Calls around plans with scores of their own: norms, rotation and append in a serial plan, a layer before and after its branches close, records
and their merge as calls of their own, and the checking build."""
import subprocess
import sys

import numpy as np
import pytest

import test_gpu_debug_bounds as D
import test_gpu_qk_norm as N
from attention_reference import THETA
from paper_2508_08895_b200 import binding as B
from pool_format import elements
from test_gpu_scores import CORES, DECODE, SERIAL, SMALL, TC, WHOLE, bits, scene

pytestmark = pytest.mark.gpu

SHAPES = [TC, SMALL[0], SMALL[1], CORES[0]]


def normed_append(s, plan, axes, rotate_q=True, stream=None):
    """qk_norm_append of the scene's tokens with so many position axes; the scene's queries are then what came out.  Checked against 64 bits: queries, the written rows, and that nothing else was written."""
    import torch
    gen = torch.Generator().manual_seed(11)
    wq, wk = ((1 + 0.3 * torch.randn(s.d, generator=gen)).to(s.q.dtype).cuda() for _ in "qk")
    half = s.d // 2
    axis = np.asarray([i % axes for i in range(half)])
    own, slot, req = B.positions(s.desc, s.mode)
    pos = np.stack([own + 7 * a for a in range(axes)]).astype(np.int32)
    before = s.k_pool.clone(), s.v_pool.clone()
    q_out = torch.full_like(s.q, 7.0)
    norm = B.QkNorm(s.shape, wq, wk, 1e-6, axis, rotate_q)
    B.qk_norm_append(plan, norm, s.q, s.k, s.v, torch.from_numpy(pos).cuda(), s.k_pool, s.v_pool, q_out, stream=stream)
    torch.cuda.synchronize()
    host = lambda x: x.detach().double().cpu().numpy()   # noqa: E731

    def turned(x):
        ang = pos[axis].T.astype(np.float64) * THETA ** (-2.0 * np.arange(half) / s.d)
        c, sn = np.cos(ang)[:, None], np.sin(ang)[:, None]
        a, b = x[..., :half], x[..., half:]
        return np.concatenate([a * c - b * sn, b * c + a * sn], -1)

    qn, kn = N.normed(host(s.q), host(wq), 1e-6), N.normed(host(s.k), host(wk), 1e-6)
    N.close(host(q_out), turned(qn) if rotate_q else qn, qn, s.dtype)
    page = s.desc["page_ids"][s.desc["page_begin"][req] + slot // s.page]
    at = elements(page, slot % s.page, s.hkv, s.page, s.d, B._esize(s.shape))
    N.close(host(s.k_pool)[at], turned(kn), kn, s.dtype)
    np.testing.assert_array_equal(host(s.v_pool)[at], host(s.v))
    for now, was in zip((s.k_pool, s.v_pool), before):
        now, was = host(now), host(was)
        now[at] = was[at]
        np.testing.assert_array_equal(now, was)
    s.q = q_out


@pytest.mark.parametrize("kind", ["cap", "both", "rotated"])
@pytest.mark.parametrize("axes", [1, 3])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_norms_in_a_serial_plan(shape, axes, kind):
    s = scene(shape, SERIAL, kind, rotated=True, q_scale=2.0)
    plan = s.plan()
    normed_append(s, plan, axes)
    B.serial_attn(plan, s.q, s.k_pool, s.v_pool, s.out)
    s.torch.cuda.synchronize()
    assert plan.status() == 0
    s.check(**bits(shape))


@pytest.mark.parametrize("kind", ["cap", "both"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_a_layer_before_and_after_its_branches_close(shape, kind):
    """The last tokens of two branches, then the first one behind them, over one cache."""
    s = scene(shape, [(129, [(39, 1), (2, 1)], 0), (40, [(16, 1)], 0)], kind, rotated=True)
    closed = scene(shape, [(129, [(40, 0), (3, 0)], 1), (40, [(17, 0)], 1)], kind, rotated=True, seed=6)
    s.n_pool, s.k_pool, s.v_pool = closed.n_pool, closed.k_pool, closed.v_pool
    for name in ("page_ids", "page_begin", "n_pages"):
        s.desc[name] = closed.desc[name]
    for x, call in ((s, B.branch_attn), (closed, B.serial_attn)):
        plan = x.plan(stable_cache=True)
        normed_append(x, plan, 3)
        call(plan, x.q, x.k_pool, x.v_pool, x.out)
        x.torch.cuda.synchronize()
        assert plan.status() == 0
        x.check(**bits(shape))


@pytest.mark.parametrize("kind", ["cap", "both", "both-rotated"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_records_and_their_merge(shape, kind):
    """attn_partials, step_partials and attn_combine against branch_attn, which is made of them."""
    s = scene(shape, DECODE, kind)
    plan = s.step()
    s.check(**bits(shape))
    B.branch_attn(plan, s.q, s.k_pool, s.v_pool, s.out)
    want = s.out.clone()
    s.out.zero_()
    B.attn_partials(plan, s.q, s.k_pool, s.v_pool)
    B.attn_combine(plan, s.out)
    s.torch.cuda.synchronize()
    assert s.torch.equal(s.out, want)
    s.out.zero_()
    if shape[0] == "bf16" and plan.info.fused_append:
        B.step_partials(plan, s.q, s.k, s.v, s.k_pool, s.v_pool)
        B.attn_combine(plan, s.out)
        s.torch.cuda.synchronize()
        assert plan.status() == 0
        s.check(**bits(shape))
    else:
        with pytest.raises(B.AspdError):
            B.step_partials(plan, s.q, s.k, s.v, s.k_pool, s.v_pool)


CHILD = r"""
import sys
sys.path[:0] = [ROOT, ROOT + "/tests"]
import torch
from paper_2508_08895_b200 import binding as B
import test_gpu_qk_norm as N
import test_gpu_scored_calls as C
for shape in C.SHAPES:
    for kind in ("cap", "both", "both-rotated"):
        for step in (C.DECODE, C.WHOLE):
            s = C.scene(shape, step, kind)
            kw = dict(n_ctas=2) if step is C.WHOLE else {}
            s.step(**kw)                                                 # the status word is looked at
            s.check(**C.bits(shape))
            # a lowered limit: page ids of the step are now "outside"; the kernels flag and skip
            plan = s.plan(**kw)
            assert B.debug_pool_limit(plan, s.n_pool + 1) == -1 and B.debug_pool_limit(plan, 1) == 0
            B.branch_step(plan, s.q, s.k, s.v, s.k_pool, s.v_pool, s.out)
            torch.cuda.synchronize()
            assert plan.status() == -2, plan.status()
            s.step(**kw)
            s.check(**C.bits(shape))
for shape in (N.SHAPES[0], N.SHAPES[4], N.SHAPES[6]):
    c = N.Case(shape, "ragged")
    c.call()
    c.check()
    assert c.plan.status() == 0
    c = N.Case(shape, "ragged")
    assert B.debug_pool_limit(c.plan, 1) == 0
    c.call()
    torch.cuda.synchronize()
    assert c.plan.status() == -2
    first = B.pool_bytes(c.shape, 1) // B._esize(c.shape)                # page 0 is inside
    assert all(torch.equal(a[first:], b[first:]) for a, b in zip(c.pool, c.before))
    other = N.Case(shape, "ragged")
    assert (c.q_out == other.q_out).sum() < other.q_out.numel()          # queries need no page
    other.call()
    other.check()
    assert torch.equal(c.q_out, other.q_out) and other.plan.status() == 0
print("CHILD-OK")
"""


def test_the_checking_build():
    res = subprocess.run([sys.executable, "-c", f"ROOT = {D.ROOT!r}\n" + CHILD], env=D._child_env(), capture_output=True, text=True, timeout=600, cwd=D.ROOT)
    assert res.returncode == 0 and "CHILD-OK" in res.stdout, res.stdout[-2000:] + res.stderr[-3000:]
