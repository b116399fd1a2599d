"""Attention over a paged branch cache in 64 bits from its definition, with how far a kernel may be off, for the tests of plans
whose scores are not the plain products.  A step is a list of requests: (prefix, regions, tail), a region (cached, new[, pos_start])
with new = -1 for one of an earlier stage; tail > 0: a serial step."""
import numpy as np

from paper_2508_08895_b200 import binding as B
from pool_format import elements

THETA = 1.0e4


def layout(step, page, seed=7):
    """(descriptors, pool pages, per request [(first slot, length, first position, new tokens at its end)], prefix first)."""
    up = lambda n: -(-n // page) * page   # noqa: E731
    keys = ("prefix_len", "n_branches", "branch_begin", "page_begin", "n_pages", "tail_off", "tail_len", "br_kv_off", "br_kv_len", "br_q_len", "br_pos_start")
    d, reqs, pages = {k: [] for k in keys}, [], 0
    for prefix, regions, tail in step:
        at, out = up(prefix), [(0, prefix, 0, 0)]
        stage = prefix + sum(r[0] for r in regions if r[1] == -1)
        d["prefix_len"].append(prefix), d["n_branches"].append(len(regions)), d["branch_begin"].append(len(d["br_kv_off"]))
        for cached, new, *start in regions:
            n = cached + max(0, new)
            d["br_kv_off"].append(at), d["br_kv_len"].append(n), d["br_q_len"].append(new), d["br_pos_start"].append(start[0] if start else B.POS_AUTO)
            out.append((at, n, start[0] if start else stage, new))
            at += up(max(1, n))
        d["tail_off"].append(at), d["tail_len"].append(tail)
        if tail:
            out.append((at, tail, prefix + sum(r[1] for r in out[1:]), 1))
        d["page_begin"].append(pages), d["n_pages"].append((at + up(tail)) // page)
        pages += d["n_pages"][-1]
        reqs.append(out)
    desc = {k: np.asarray(v, dtype=np.int32) for k, v in d.items()}
    n_pool = pages + 3
    desc["page_ids"] = np.random.default_rng(seed).permutation(n_pool)[:pages].astype(np.int32)
    return desc, n_pool, reqs


class Scene:
    """A step's inputs on the device, and the reference of its outputs."""

    def __init__(self, dtype, d, page, heads, step, cap=0.0, slopes=None, rotated=False, mask=0, q_scale=1.0, seed=5, v_mean=0.0):
        import torch
        self.torch, self.dtype, self.d, self.page, (self.hq, self.hkv) = torch, dtype, d, page, heads
        dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.desc, self.n_pool, self.reqs = layout(step, page)
        self.mode = B.MODE_SERIAL if step[0][2] else B.MODE_BRANCH
        self.shape = B.make_shape(*heads, d, page, dtype, THETA, d ** -0.5)
        self.scale, self.cap, self.rotated, self.mask = d ** -0.5, cap, rotated, mask
        self.slopes = None if slopes is None else np.asarray(slopes, dtype=np.float32)
        self.scores = B.Scores(cap, self.slopes, rotated)
        gen = torch.Generator().manual_seed(seed)
        normal = lambda *size: torch.randn(*size, generator=gen)   # noqa: E731
        n = self.n = B.count_new_tokens(self.desc, self.mode)
        self.q, self.k, self.v = ((normal(n, h, d) * s + m).to(dt).cuda() for h, s, m in ((self.hq, q_scale, 0), (self.hkv, 1, 0), (self.hkv, 1, v_mean)))
        size = B.pool_bytes(self.shape, self.n_pool) // B._esize(self.shape)
        self.k_pool, self.v_pool = normal(size).to(dt).cuda(), (normal(size) + v_mean).to(dt).cuda()
        self.out = torch.full((n, self.hq, d), 77.0, dtype=dt, device="cuda")

    def plan(self, **kw):
        return B.Plan(self.shape, self.desc, self.n_pool, self.mode, scores=self.scores, mask=self.mask, **kw)

    def step(self, plan=None, stream=None, **kw):
        plan = plan or self.plan(**kw)
        (B.serial_step if self.mode == B.MODE_SERIAL else B.branch_step)(plan, self.q, self.k, self.v, self.k_pool, self.v_pool, self.out, stream=stream)
        self.torch.cuda.synchronize()
        assert plan.status() == 0
        return plan

    def reference(self, q_bits, p_bits, own):
        """(outputs, bound) in 64 bits over the keys that the cache holds now.  q_bits: the kernel rounds turned queries by half a
        step 2^-q_bits, p_bits: weights before P.V (0: not rounded); own: relative error of the rest of a logit and of a sum (fp32)."""
        host = lambda x: x.detach().double().cpu().numpy()   # noqa: E731
        q, kp, vp = host(self.q), host(self.k_pool), host(self.v_pool)
        pos, _, _ = B.positions(self.desc, self.mode)
        if not self.rotated:
            half = self.d // 2
            ang = pos[:, None] * THETA ** (-2.0 * np.arange(half) / self.d)
            c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
            a, b = q[..., :half], q[..., half:]
            q = np.concatenate([a * c - b * s, b * c + a * s], -1)
        G, t = self.hq // self.hkv, 0
        out, bound = np.zeros_like(q), np.zeros_like(q)
        for r, regions in enumerate(self.reqs):
            ids = self.desc["page_ids"][self.desc["page_begin"][r]:]
            ks, vs, ps, reg, place = [], [], [], [], []
            for i, (first, length, p0, _) in enumerate(regions):
                slot = first + np.arange(length)
                at = elements(ids[slot // self.page], slot % self.page, self.hkv, self.page, self.d, B._esize(self.shape))
                ks.append(kp[at]), vs.append(vp[at]), ps.append(p0 + np.arange(length)), reg.append(np.full(length, i)), place.append(np.arange(length))
            k, v, kpos, reg, place = (np.concatenate(x) for x in (ks, vs, ps, reg, place))
            for i, (first, length, p0, new) in enumerate(regions):
                for j in range(max(0, new)):
                    own_place = length - new + j
                    if self.mode == B.MODE_SERIAL:
                        seen = np.ones(len(reg), bool)
                    else:
                        shared = [m for m, x in enumerate(regions) if m == 0 or x[3] == -1]
                        seen = np.isin(reg, shared) | ((reg == i) & (place <= own_place))
                        if self.mask == B.MASK_SHARED:
                            seen |= ~np.isin(reg, shared) & (reg != i) & (place < own_place)
                    dist = p0 + own_place - kpos[seen]
                    for h in range(self.hq):
                        kk, vv = k[seen][:, h // G], v[seen][:, h // G]
                        x = self.scale * (kk @ q[t, h])
                        size = self.scale * (np.abs(kk) @ np.abs(q[t, h]))
                        delta = size * ((2.0 ** -q_bits if q_bits and not self.rotated else 0) + own)
                        y = self.cap * np.tanh(x / self.cap) if self.cap else x
                        if self.cap:
                            delta = delta + 4 * own * np.abs(y)
                        if self.slopes is not None:
                            y = y - float(self.slopes[h]) * dist
                            delta = delta + own * np.abs(float(self.slopes[h]) * dist)
                        z = np.exp(y - y.max()).sum()
                        w = np.exp(y - y.max()) / z
                        out[t, h] = w @ vv
                        # logits off by delta take a weight w = e^y / z to at most e^(y + delta) / z (not as w e^delta: a key at a steep
                        # slope's far end has a weight of 0 and a delta beyond any exponent), against the weights' own mean; then rounded
                        # weights, sums and the output
                        more = np.exp(y - y.max() + (delta + 4 * own)) / z - w
                        bound[t, h] = 1.1 * (more @ (np.abs(vv) + np.abs(out[t, h]))) + ((2.0 ** -p_bits if p_bits else 0) + 8 * own) * (w @ np.abs(vv))
                    t += 1
        step = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24
        return out, bound * (1 + step) + step * np.abs(out) + 1e-30

    def check(self, q_bits=8, p_bits=8, own=2.0 ** -18):
        """bf16: turned queries and weights are rounded to bf16 (half a step, 2^-8); `own` covers fp32 sums of up to 2^6 roundings
        of 2^-24 in a row (d / 16 MMA steps, tiles, parts) and the approximations of 2^x, 1 / x and tanh."""
        got = self.out.double().cpu().numpy()
        ref, bound = self.reference(q_bits, p_bits, own)
        assert np.isfinite(got).all()
        err = np.abs(got - ref)
        assert (err <= bound).all(), float((err / bound).max())
        # and far inside on the whole: roundings are independent, so that the bound's sum over hundreds of keys is never met
        return float(np.linalg.norm(got - ref) / np.linalg.norm(ref))


def alibi(n):
    return 2.0 ** (-8.0 * (np.arange(n) + 1) / n)
