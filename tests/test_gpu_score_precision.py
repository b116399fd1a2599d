"""What the kernel of heads of 128 in pages of 16 keeps of capped scores: queries that it rotates in two bf16 pieces, rows divided by the sum of
their weights as P.V takes them.  Neither shows in a bound element by element, which allows one piece; both show in the root mean square over
thousands of rows.  Outputs are compared with 64 bits, and so is a 64-bit computation with the kernel's roundings and no others: the kernel may
be 4 % further off than that (fp32 sums and a tanh off by 3e-6 move a weight of such logits by 1e-4 of itself at most, 2 % of a step of bf16, so
that one rounding in fifty falls the other way), while one piece, and unrounded sums, have to be beyond it."""
import numpy as np
import pytest

from attention_reference import THETA, Scene
from paper_2508_08895_b200 import binding as B
from pool_format import elements

pytestmark = pytest.mark.gpu

SHAPE = ("bf16", 128, 16, (28, 4))
CUT = [(500, [(i, 1) for i in (3, 17, 40, 0, 64, 90)], 0), (200, [(i, 2) for i in (11, 31, 5)], 0)]
WHOLE = [(90, [(0, 40), (7, 30), (0, 3)], 0), (33, [(0, 50)], 0)]
MORE = 1.04


def bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def outputs(s, pieces, round_weights, round_sums):
    """Branch steps of capped scores in 64 bits; roundings as asked, and the output's own."""
    host = lambda x: x.detach().double().cpu().numpy()   # noqa: E731
    q, kp, vp = host(s.q), host(s.k_pool), host(s.v_pool)
    if not s.rotated:
        pos, half = B.positions(s.desc, s.mode)[0], s.d // 2
        ang = pos[:, None] * THETA ** (-2.0 * np.arange(half) / s.d)
        c, sn = np.cos(ang)[:, None], np.sin(ang)[:, None]
        a, b = q[..., :half], q[..., half:]
        q = np.concatenate([a * c - b * sn, b * c + a * sn], -1)
    if pieces:
        first = bf16(q)
        q = first + (bf16(q - first) if pieces == 2 else 0)
    out, G, t = np.zeros_like(q), s.hq // s.hkv, 0
    for r, regions in enumerate(s.reqs):
        ids = s.desc["page_ids"][s.desc["page_begin"][r]:]
        for first, length, _, new in regions[1:]:
            slot = np.concatenate([np.arange(regions[0][1]), first + np.arange(length)])
            at = elements(ids[slot // s.page], slot % s.page, s.hkv, s.page, s.d, 2)
            k, v = kp[at], vp[at]
            for j in range(new):
                n = len(slot) - new + j + 1
                for h in range(s.hq):
                    w = np.exp(s.cap * np.tanh(s.scale * (k[:n, h // G] @ q[t, h]) / s.cap))
                    p = bf16(w) if round_weights else w
                    out[t, h] = (p @ v[:n, h // G]) / (p if round_sums else w).sum()
                t += 1
    return out if not round_weights else bf16(out)


def off(a, b):
    return float(np.linalg.norm(a - b) / np.linalg.norm(b))


@pytest.mark.parametrize("cap", [20.0, 50.0])
@pytest.mark.parametrize("rotated", [False, True], ids=["turned-inside", "come-turned"])
@pytest.mark.parametrize("step,kw,rows", [(CUT, {}, 64), (CUT, dict(combine=B.COMBINE_FUSED), 64), (WHOLE, dict(n_ctas=2, wide_rows=256), 256)], ids=["cut", "merged-inside", "two-tiles"])
def test_roundings(step, kw, rows, rotated, cap):
    s = Scene(*SHAPE, step, cap=cap, q_scale=5.0, rotated=rotated)
    plan = s.plan(**kw)
    assert plan.info.max_rows_per_item == rows
    s.step(plan)
    got, exact = s.out.double().cpu().numpy(), outputs(s, 0, False, False)
    pieces = 0 if rotated else 2
    allowed = MORE * off(outputs(s, pieces, True, True), exact)
    others = [outputs(s, pieces, True, False)] + ([] if rotated else [outputs(s, 1, True, True)])
    assert all(off(x, exact) > allowed for x in others)
    assert off(got, exact) <= allowed, (off(got, exact), allowed)


@pytest.mark.parametrize("shape", [("bf16", 64, 16, (14, 2)), ("bf16", 128, 8, (28, 4))], ids=str)
def test_heads_of_64_and_other_pages(shape):
    """Their kernel keeps queries and weights in several pieces: nothing but the output's own rounding."""
    s = Scene(*shape, CUT, cap=20.0, q_scale=5.0)
    s.step()
    got, exact = s.out.double().cpu().numpy(), outputs(s, 0, False, False)
    allowed = MORE * off(bf16(exact), exact)
    assert all(off(bf16(outputs(s, *x)), exact) > allowed for x in ((1, False, False), (0, True, True)))
    assert off(got, exact) <= allowed, (off(got, exact), allowed)
