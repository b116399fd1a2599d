"""aspd_qk_norm_append: norms of queries and keys, rotation by one or several axes, paged append -- against 64 bits."""
import numpy as np
import pytest

from paper_2508_08895_b200 import binding as B
from pool_format import elements

THETA = 1.0e6
# dtype, head_dim, page size, (query heads, KV heads)
SHAPES = [("bf16", 128, 16, (28, 4)), ("bf16", 64, 16, (14, 2)), ("bf16", 128, 8, (3, 1)), ("bf16", 128, 32, (64, 1)), ("bf16", 64, 8, (1, 1)),
          ("f32", 128, 16, (28, 4)), ("f32", 64, 8, (4, 1)), ("f32", 64, 32, (5, 5)), ("f32", 128, 16, (160, 8))]
# per request: prefix, (cached, new) of its branches
STEPS = {"one": [(0, [(0, 1)])], "ragged": [(37, [(5, 1), (0, 3), (31, 1), (8, 0)]), (0, [(15, 2)]), (160, [(0, 9), (7, 1)])], "whole": [(3, [(0, 65), (2, 40)]), (64, [(0, 17)])]}


def layout(step, page):
    up = lambda n: -(-n // page) * page   # noqa: E731
    d = {k: [] for k in ("prefix_len", "n_branches", "branch_begin", "page_begin", "n_pages", "tail_off", "tail_len", "br_kv_off", "br_kv_len", "br_q_len")}
    pages = 0
    for prefix, branches in step:
        at = up(prefix)
        d["prefix_len"].append(prefix), d["n_branches"].append(len(branches)), d["branch_begin"].append(len(d["br_kv_off"]))
        for cached, new in branches:
            d["br_kv_off"].append(at), d["br_kv_len"].append(cached + new), d["br_q_len"].append(new)
            at += up(max(1, cached + new))
        d["tail_off"].append(at), d["tail_len"].append(0), d["page_begin"].append(pages), d["n_pages"].append(at // page)
        pages += at // page
    desc = {k: np.asarray(v, dtype=np.int32) for k, v in d.items()}
    n_pool = pages + 5
    desc["page_ids"] = np.random.default_rng(7).permutation(n_pool)[:pages].astype(np.int32)
    return desc, n_pool


def places(desc, page):
    pos, slot, req = B.positions(desc, B.MODE_BRANCH)
    return pos, desc["page_ids"][desc["page_begin"][req] + slot // page], slot % page


def turned(x, pos, axis):
    """x [n][heads][d] in 64 bits, pair i turned by pos[axis[i]]."""
    half = x.shape[-1] // 2
    ang = pos[axis].T.astype(np.float64) * THETA ** (-2.0 * np.arange(half) / x.shape[-1])
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def normed(x, w, eps):
    return x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w


def close(got, ref, before, dtype):
    """got: one rounding to the storage type (half a step, 2^-8 or 2^-24 of the value) of a fp32 computation.  Its own error
    counts relative to |a| + |b| of the pair that was turned: sum of squares (33 additions and products at most in a row, half of which
    counts under the root), root and division (2 steps), three products, sine and cosine (2 steps of a value up to 1, and an angle in
    [-pi, pi] rounded to fp32: 2^-22 at most), two products and an addition: less than 40 roundings of 2^-24."""
    half = ref.shape[-1] // 2
    mag = np.abs(before[..., :half]) + np.abs(before[..., half:])
    own = 40 * 2.0 ** -24 * np.concatenate([mag, mag], -1)
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    err = np.abs(got - ref)
    bound = (np.abs(ref) + own) * step + own + 1e-37
    assert (err <= bound).all(), (err / bound).max()


class Case:
    def __init__(self, shape, step="ragged", axes=3, interleaved=False, norm="qk", rotate_q=True, packed=True, seed=3, scale=3.0):
        import torch
        self.torch = torch
        self.dtype, self.d, self.page, (self.hq, self.hkv) = shape
        dt = torch.bfloat16 if self.dtype == "bf16" else torch.float32
        self.desc, self.n_pool = layout(STEPS[step], self.page)
        self.shape = B.make_shape(self.hq, self.hkv, self.d, self.page, self.dtype, THETA, self.d ** -0.5)
        self.plan = B.Plan(self.shape, self.desc, self.n_pool, B.MODE_BRANCH)
        n = self.n = self.plan.n_new
        gen = torch.Generator().manual_seed(seed)
        qkv = (torch.randn(n, self.hq + 2 * self.hkv, self.d, generator=gen) * scale).to(dt).cuda()
        cut = [qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv], qkv[:, self.hq + self.hkv:]]
        self.q, self.k, self.v = cut if packed else [x.contiguous() for x in cut]
        weight = lambda: (1 + 0.3 * torch.randn(self.d, generator=gen)).to(dt).cuda()   # noqa: E731
        self.wq, self.wk = (weight() if c in norm else None for c in "qk")
        half = self.d // 2
        self.axis = np.asarray(B.axes_of_pairs([half - 2 * (3 * half // 8), 3 * half // 8, 3 * half // 8], interleaved) if axes == 3 else
                               [i % axes for i in range(half)])
        rng = np.random.default_rng(seed)
        own, self.pages, self.rows = places(self.desc, self.page)
        self.pos = np.stack([own + (rng.integers(-50, 5000, n) if a else 0) for a in range(axes)]).astype(np.int32)
        self.eps, self.rotate_q = 1e-6, rotate_q
        self.pool = [torch.randn(B.pool_bytes(self.shape, self.n_pool) // B._esize(self.shape), generator=gen).to(dt).cuda() for _ in "kv"]
        self.before = [x.clone() for x in self.pool]
        self.q_out = torch.full((n, self.hq, self.d), 7.0, dtype=dt, device="cuda")
        self.norm = B.QkNorm(self.shape, self.wq, self.wk, self.eps, self.axis, rotate_q)

    def call(self, **kw):
        B.qk_norm_append(self.plan, self.norm, self.q, self.k, self.v, self.torch.from_numpy(self.pos).cuda(), *self.pool, self.q_out, **kw)

    def check(self, q_in=None):
        host = lambda x: None if x is None else x.detach().double().cpu().numpy()   # noqa: E731
        self.torch.cuda.synchronize()
        q, k, v = host(self.q if q_in is None else q_in), host(self.k), host(self.v)
        qn, kn = normed(q, host(self.wq), self.eps), normed(k, host(self.wk), self.eps)
        close(host(self.q_out), turned(qn, self.pos, self.axis) if self.rotate_q else qn, qn, self.dtype)
        at = elements(self.pages, self.rows, self.hkv, self.page, self.d, B._esize(self.shape))
        kp, vp = (host(x) for x in self.pool)
        close(kp[at], turned(kn, self.pos, self.axis), kn, self.dtype)
        np.testing.assert_array_equal(vp[at], v)
        for now, was in zip((kp, vp), self.before):             # and nothing else was written
            now, was = now.copy(), host(was)
            now[at] = was[at]
            np.testing.assert_array_equal(now, was)


@pytest.mark.gpu
@pytest.mark.parametrize("step", list(STEPS))
@pytest.mark.parametrize("shape", SHAPES)
def test_against_64_bits(shape, step):
    c = Case(shape, step)
    c.call()
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [dict(axes=1), dict(axes=2), dict(axes=4), dict(interleaved=True), dict(norm="q"), dict(norm="k"), dict(norm=""),
                                dict(rotate_q=False), dict(rotate_q=False, norm="k"), dict(packed=False)], ids=str)
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[6]])
def test_options(shape, kw):
    c = Case(shape, **kw)
    c.call()
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[5]])
def test_queries_in_place(shape):
    c = Case(shape, "whole", packed=False)
    was = c.q.clone()
    c.q_out = c.q
    c.call()
    c.check(was)


@pytest.mark.gpu
def test_far_and_negative_positions_and_small_and_large_heads():
    c = Case(SHAPES[0], "ragged", axes=2)
    c.pos[0], c.pos[1] = 2 ** 31 - 1 - np.arange(c.n), -(2 ** 31) + 17 * np.arange(c.n)
    c.q[0], c.k[0] = 0.0, 0.0                                   # a head of zeros stays one
    c.q[1] *= 1e12
    c.k[1] *= 1e-20                                             # below eps: scaled by 1 / sqrt(eps)
    c.call()
    c.check()


@pytest.mark.gpu
def test_the_key_that_kv_append_writes():
    """Without norms and with one axis the cache is aspd_kv_append's, bit for bit."""
    for shape in (SHAPES[0], SHAPES[1], SHAPES[6]):
        c = Case(shape, "whole", axes=1, norm="")
        c.call()
        other = [x.clone() for x in c.before]
        B.kv_append(c.plan, c.k.contiguous(), c.v.contiguous(), c.torch.from_numpy(c.pos[0].copy()).cuda(), *other)
        c.torch.cuda.synchronize()
        assert all(c.torch.equal(x, y) for x, y in zip(c.pool, other))


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_head():
    c = Case(SHAPES[0], "ragged")
    c.q[2, 3, 5], c.k[1, 2, 9], c.v[0, 0, 0] = float("nan"), float("inf"), float("nan")
    c.call()
    c.torch.cuda.synchronize()
    out, kp = c.q_out.float().cpu(), c.pool[0].float().cpu().numpy()
    bad = ~np.isfinite(out.numpy())
    assert bad[2, 3].all() and bad.sum() == c.d
    at = elements(c.pages, c.rows, c.hkv, c.page, c.d, 2)
    bad = ~np.isfinite(kp[at])
    assert bad[1, 2].any() and not np.delete(bad.reshape(-1, c.d), 1 * c.hkv + 2, 0).any()


@pytest.mark.gpu
def test_another_stream_and_a_replayed_graph():
    c = Case(SHAPES[0], "whole")
    torch = c.torch
    pos = torch.from_numpy(c.pos).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.qk_norm_append(c.plan, c.norm, c.q, c.k, c.v, pos, *c.pool, c.q_out, stream=side)
    side.synchronize()
    c.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.qk_norm_append(c.plan, c.norm, c.q, c.k, c.v, pos, *c.pool, c.q_out)
    c.q.mul_(0.5), c.k.add_(1.0), pos.add_(3)
    c.pos += 3
    c.q_out.zero_()
    graph.replay()
    c.check()


@pytest.mark.gpu
def test_refusals():
    c = Case(SHAPES[0], packed=False)
    torch, L = c.torch, B.lib()
    import ctypes
    pos = torch.from_numpy(c.pos).cuda()
    row, kv = c.hq * c.d, c.hkv * c.d

    def rc(norm=None, q=c.q, qs=row, k=c.k, ks=kv, v=c.v, vs=kv, p=pos, kp=c.pool[0], vp=c.pool[1], out=c.q_out, plan=c.plan, **fields):
        nm = type(c.norm.c).from_buffer_copy(c.norm.c)
        for name, value in fields.items():
            setattr(nm, name, value)
        ptr = lambda x: x if x is None or isinstance(x, int) else x.data_ptr()   # noqa: E731
        return L.aspd_qk_norm_append(plan._h if plan else None, ctypes.addressof(nm) if norm is None else None, ptr(q), qs, ptr(k), ks, ptr(v), vs, ptr(p),
                                     ptr(kp), ptr(vp), ptr(out), B._stream(None))

    was = [x.clone() for x in (*c.pool, c.q_out)]
    assert rc(plan=None) == -1 and rc(norm=False) == -1
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(p=None), dict(kp=None), dict(vp=None), dict(out=None)):
        assert rc(**kw) == -1, kw
    for kw in (dict(q=c.q.data_ptr() + 2), dict(out=c.q_out.data_ptr() + 8), dict(q_weight=c.wq.data_ptr() + 2)):
        assert rc(**kw) == -1, kw
    for kw in (dict(qs=row - 8), dict(qs=row + 1), dict(ks=kv - 8), dict(vs=0), dict(ks=-kv), dict(q=c.q_out, qs=row + 8)):
        assert rc(**kw) == -1, kw
    for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(n_axes=0), dict(n_axes=5), dict(n_axes=2)):   # (a pair of axis 2)
        assert rc(**kw) == -1, kw
    host = B.Plan(c.shape, c.desc, c.n_pool, B.MODE_BRANCH, host_only=True)
    assert rc(plan=host) == -1
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((*c.pool, c.q_out), was))
    assert rc() == 0
    c.check()


def test_binding_refuses_what_does_not_fit():
    """On the CPU: nothing is launched."""
    import torch
    desc, n_pool = layout(STEPS["ragged"], 16)
    shape = B.make_shape(4, 2, 64, 16, "f32", THETA, 0.125)
    plan = B.Plan(shape, desc, n_pool, B.MODE_BRANCH, host_only=True)
    n = plan.n_new
    q, k, pos = torch.zeros(n, 4, 64), torch.zeros(n, 2, 64), torch.zeros(1, n, dtype=torch.int32)
    pool = torch.zeros(B.pool_bytes(shape, n_pool) // 4)
    nm = B.QkNorm(shape)
    for bad in (torch.zeros(n, 64, 4).transpose(1, 2), torch.zeros(n + 1, 4, 64), torch.zeros(n, 4, 64, dtype=torch.bfloat16), torch.zeros(n, 8, 64)[:, ::2]):
        with pytest.raises(ValueError):
            B.qk_norm_append(plan, nm, bad, k, k, pos, pool, pool, q)
    with pytest.raises(ValueError):
        B.qk_norm_append(plan, B.QkNorm(shape, axis_of_pair=[0, 1] * 16), q, k, k, pos, pool, pool, q)      # one position each, two axes
    with pytest.raises(B.AspdError):
        B.qk_norm_append(plan, nm, q, k, k, pos, pool, pool, q)                                             # a host-only plan
    for kw in (dict(axis_of_pair=[0] * 31), dict(axis_of_pair=[4] * 32), dict(q_weight=torch.zeros(63)), dict(k_weight=torch.zeros(64, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            B.QkNorm(shape, **kw)
    assert B.axes_of_pairs([16, 24, 24]) == [0] * 16 + [1] * 24 + [2] * 24
    assert B.axes_of_pairs([3, 2, 1], True) == [0, 1, 2, 0, 1, 0]
