"""Requests of very many branches, on the CPU: what a plan costs grows with their number, not with its square."""
import time

import numpy as np
import pytest

from paper_2508_08895_b200 import binding as B


def seconds(n, pos_start, scores):
    """The quickest of several plans of one request with n branches of one token each."""
    shape = B.make_shape(4, 2, 128, 16, "bf16", 1e4, 0.125)
    desc = dict(prefix_len=[16], n_branches=[n], branch_begin=[0], page_begin=[0], n_pages=[1 + n], tail_off=[0], tail_len=[0], br_kv_off=16 + 16 * np.arange(n),
                br_kv_len=np.ones(n), br_q_len=np.ones(n), br_pos_start=np.full(n, pos_start), page_ids=np.arange(1 + n))
    desc = {k: np.asarray(v, dtype=np.int32) for k, v in desc.items()}
    best = np.inf
    for _ in range(5):
        start = time.perf_counter()
        plan = B.Plan(shape, desc, n + 1, B.MODE_BRANCH, host_only=True, scores=scores)
        best = min(best, time.perf_counter() - start)
        plan.destroy()
    return best


@pytest.mark.parametrize("scores", [None, B.Scores(cap=30.0), B.Scores(slopes=[0.5] * 4)], ids=["plain", "cap", "bias"])
def test_positions_that_the_library_numbers_cost_no_more_than_given_ones(scores):
    """8 000 branches: 2 ms of planning either way.  (A walk over all of them for each one's first position: 95 to 160 ms.)"""
    assert seconds(8000, B.POS_AUTO, scores) < 8 * seconds(8000, 16, scores)
