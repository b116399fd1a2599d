"""What the binding of aspd_qk_norm_append takes for positions and gains.  On the CPU: calls that pass its checks end at the
host-only plan, which the library refuses, and nothing is launched."""
import pytest
import torch

from paper_2508_08895_b200 import binding as B
from test_gpu_qk_norm import STEPS, layout


class Call:
    def __init__(self, dtype="bf16", d=64):
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        desc, n_pool = layout(STEPS["ragged"], 16)
        self.shape = B.make_shape(4, 2, d, 16, dtype, 1e4, 0.125)
        self.plan = B.Plan(self.shape, desc, n_pool, B.MODE_BRANCH, host_only=True)
        self.n = self.plan.n_new
        self.q, self.k, self.pool = torch.zeros(self.n, 4, d, dtype=self.dt), torch.zeros(self.n, 2, d, dtype=self.dt), torch.zeros(1, dtype=self.dt)

    def __call__(self, norm, pos):
        B.qk_norm_append(self.plan, norm, self.q, self.k, self.k, pos, self.pool, self.pool, self.q)

    def axes(self, n):
        return B.QkNorm(self.shape, axis_of_pair=[i % n for i in range(self.shape.head_dim // 2)])


def test_positions_of_several_axes_lie_a_row_of_the_step_apart():
    """A buffer made for more tokens than the step has would have axes 1 and 2 turn by other tokens' positions."""
    c = Call()
    for rows in ((3, c.n + 5), (c.n, 3), (2, c.n), (3, c.n - 1), (3 * c.n + 15,), (2 * c.n,), (1, 3, c.n), (3 * c.n, 1), ()):
        with pytest.raises(ValueError):
            c(c.axes(3), torch.zeros(rows, dtype=torch.int32))
    for rows in ((3, c.n + 5), (c.n + 1,), (c.n, 1)):
        with pytest.raises(ValueError):
            c(c.axes(1), torch.zeros(rows, dtype=torch.int32))
    for bad in (torch.zeros(3, c.n, dtype=torch.int64), torch.zeros(c.n, 3, dtype=torch.int32).T):
        with pytest.raises(ValueError):
            c(c.axes(3), bad)
    for axes, rows in ((3, (3, c.n)), (3, (4, c.n)), (3, (3 * c.n,)), (1, (1, c.n)), (1, (c.n,)), (1, (3, c.n))):
        with pytest.raises(B.AspdError):
            c(c.axes(axes), torch.zeros(rows, dtype=torch.int32))


@pytest.mark.parametrize("dtype,others", [("bf16", (torch.float16, torch.int16, torch.float32)), ("f32", (torch.int32, torch.bfloat16, torch.float64))])
def test_gains_are_of_the_storage_type(dtype, others):
    c = Call(dtype)
    for other in others:
        for name in ("q_weight", "k_weight"):
            with pytest.raises(ValueError):
                B.QkNorm(c.shape, **{name: torch.ones(64, dtype=other)})
    with pytest.raises(B.AspdError):
        c(B.QkNorm(c.shape, torch.ones(64, dtype=c.dt), torch.ones(64, dtype=c.dt)), torch.zeros(1, c.n, dtype=torch.int32))


def test_a_norm_made_for_another_shape():
    """Its gains would be read beyond their end, or as another type."""
    c = Call()
    for other in (Call("f32"), Call("bf16", 128)):
        with pytest.raises(ValueError):
            c(B.QkNorm(other.shape, torch.ones(other.shape.head_dim, dtype=other.dt)), torch.zeros(1, c.n, dtype=torch.int32))
