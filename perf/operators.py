"""Operators around the attention step for models whose attention is not the plain one, as timed cases:

  norm    ``qk_norm_append``: RMS norms of queries and keys for each head, the rotation (one position ID per
          token or three, as vision-language models use), K and V rows into the paged cache, in one pass
  step    ``branch_step`` / ``serial_step`` of a plan whose scores are capped by a tanh, get a bias that
          falls with the distance of the position IDs, or both
  layer   both in sequence, as a layer of such a model calls them

The plain forms compute the same in elementary torch operations, 32 bits, one rounding at the end; angles of
positions in 64 bits.  ``exact`` states each operator once more in 64 bits.

A case: requests with a shared prefix and branches of ``prior`` cached tokens and ``new`` new ones (more than 24:
whole branches of up to that many), lengths drawn from ``lens``.  Cache values are N(0, 1); the pools keep a token row
of a page as 16-byte chunks, XOR-ed by the row's number modulo 8 inside 128-byte spans, eight rows to a block.
"""
import math
import random

import numpy as np
import torch

own = False

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
_ES = {"bf16": 2, "f32": 4}
_THETA = 1.0e6
_EPS = 1.0e-6


def _case(name, op, step="branch", n_req=1, prefix=(256, 256), branches=(4, 4), prior=(1, 1), new=1, tail=0, lens=1, heads=(28, 4), d=128, page=16,
          dtype="bf16", cap=0.0, bias=False, norm=False, axes=1, interleaved=False, rope=True):
    c = {"op": op, "step": step, "n_req": n_req, "prefix_lo": prefix[0], "prefix_hi": prefix[1], "branches_lo": branches[0], "branches_hi": branches[1],
         "prior_lo": prior[0], "prior_hi": prior[1], "new": new, "tail": tail, "lens": lens, "hq": heads[0], "hkv": heads[1], "d": d, "page": page,
         "dtype": dtype, "cap": cap, "bias": bias, "norm": norm, "axes": axes, "interleaved": interleaved, "rope": rope}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one chat request decoding four branches: the smallest call of a model with normalised heads, all latency
        _case("norm-one-request", "norm", n_req=1, prefix=(2048, 2048), prior=(128, 128), norm=True),
        # a serving batch in mixed states, text and images: three position axes
        _case("norm-serving", "norm", n_req=32, prefix=(128, 512), branches=(1, 8), prior=(1, 256), norm=True, axes=3),
        # teacher forcing / prefill: thousands of new tokens, interleaved axes
        _case("norm-prefill", "norm", n_req=32, prefix=(128, 512), branches=(1, 8), prior=(0, 0), new=256, norm=True, axes=3, interleaved=True),
        # fp32, heads of 64, pages of 8, a model that turns three axes but does not normalise
        _case("axes-f32", "norm", n_req=5, prefix=(37, 201), branches=(3, 7), prior=(0, 29), new=13, heads=(14, 2), d=64, page=8, dtype="f32", axes=3),
        # a small fp32 step with both
        _case("both-f32", "step", n_req=1, prefix=(256, 256), branches=(3, 3), prior=(9, 23), heads=(4, 1), d=64, dtype="f32", cap=30.0, bias=True),
        # one chat request, capped scores
        _case("cap-one-request", "step", n_req=1, prefix=(2048, 2048), prior=(128, 128), cap=50.0),
        # a serving batch in mixed states, capped scores
        _case("cap-serving", "step", n_req=32, prefix=(512, 8192), branches=(1, 8), prior=(1, 256), cap=50.0),
        # one request over a long context, a model without rotation whose scores fall with distance
        _case("bias-long", "step", n_req=1, prefix=(16384, 16384), branches=(8, 8), prior=(32, 256), bias=True, rope=False),
        # a serving batch after its segments closed: one token per request over the merged cache
        _case("bias-serving-serial", "step", "serial", n_req=32, prefix=(512, 8192), branches=(1, 8), prior=(1, 256), bias=True, rope=False),
        # whole branches of a batch in one step (masked prefill), capped scores: compute-bound
        _case("cap-prefill", "step", n_req=32, prefix=(512, 8192), branches=(1, 8), prior=(0, 0), new=256, cap=50.0),
        # heads of 64, two KV heads, both
        _case("both-d64", "step", n_req=8, prefix=(512, 4096), branches=(1, 8), prior=(1, 256), heads=(14, 2), d=64, cap=50.0, bias=True),
        # a layer: norms, rotation and append, then attention with capped scores over that cache
        _case("layer-serving", "layer", n_req=32, prefix=(512, 4096), branches=(1, 8), prior=(1, 256), norm=True, axes=3, cap=30.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case of the ranges above."""
    op = rng.choice(["norm", "norm", "step", "step", "step", "layer"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([128, 128, 64])
    heads = rng.choice([(28, 4), (32, 8), (16, 2), (8, 1)] if d == 128 else [(14, 2), (16, 8), (32, 4), (4, 1)])
    page = rng.choice([16, 16, 16, 8, 32])
    common = dict(lens=rng.randrange(1, 1 << 20), heads=heads, d=d, page=page, dtype=dtype, tail=rng.randint(0, 40))
    which = rng.choice(["cap", "bias", "both"])
    scores = dict(cap=rng.choice([20.0, 30.0, 50.0]) if which != "bias" else 0.0, bias=which != "cap", rope=which == "cap" or rng.random() < 0.5)
    axes = rng.choice([1, 3, 3])
    norms = dict(norm=rng.random() < 0.75 or axes == 1, axes=axes, interleaved=axes == 3 and rng.random() < 0.5)
    # whole branches: compute-bound on the tensor cores; the CUDA-core and small-shape kernels get short ones
    wide = dtype == "bf16" and d == 128 and page == 16
    kind = rng.choice(["decode", "decode", "open", "whole"])
    new = 1 if kind == "decode" else rng.randint(2, 24) if kind == "open" or not wide else rng.randint(25, 256)
    n_req = _log_int(rng, 1, 32 if kind == "decode" else 10) if wide else _log_int(rng, 1, 8 if dtype == "bf16" else 3)
    lo = _log_int(rng, 30, 4000 if wide else 1000)
    hi = min(8192, lo * rng.randint(1, 4))
    if op == "norm":
        return _case(None, "norm", n_req=n_req, prefix=(min(lo, 400), min(hi, 800)), branches=(1, 8), prior=(0, rng.choice([0, 100])), new=new, **common, **norms)
    if op == "step":
        step = "serial" if kind == "decode" and rng.random() < 0.4 else "branch"
        return _case(None, "step", step, n_req=n_req, prefix=(lo, hi), branches=(1, 8), prior=(1, 200), new=new, **common, **scores)
    return _case(None, "layer", n_req=n_req, prefix=(lo, hi), branches=(1, 8), prior=(1, 200), new=new, **common, **norms, cap=scores["cap"], bias=scores["bias"])


# ------------------------------------------------------------------------------------ lengths and layout
def _lengths(case):
    """Per request: prefix length, tokens of every branch before the step, new tokens of every branch."""
    rng = random.Random(case["lens"])
    out = []
    for _ in range(case["n_req"]):
        prefix = _log_int(rng, case["prefix_lo"], case["prefix_hi"])
        n_br = rng.randint(case["branches_lo"], case["branches_hi"])
        prior = [rng.randint(case["prior_lo"], case["prior_hi"]) for _ in range(n_br)]
        new = [case["new"] if case["new"] <= 24 else rng.randint(1, case["new"]) for _ in range(n_br)]
        out.append((prefix, prior, new if case["step"] == "branch" else [0] * n_br))
    return out


def _layout(case, seed):
    """Descriptor arrays of the step (page-aligned branches and tail, pages scattered by the seed), and per
    request what the masks come from: the region, the place in it and the position ID of every slot and new token."""
    ps, serial = case["page"], case["step"] == "serial"
    up = lambda n: -(-n // ps) * ps   # noqa: E731
    keys = ("prefix_len", "n_branches", "branch_begin", "page_begin", "n_pages", "tail_off", "tail_len", "br_kv_off", "br_kv_len", "br_q_len")
    desc, reqs, pages = {k: [] for k in keys}, [], 0
    for prefix, prior, new in _lengths(case):
        regions, at = [(0, prefix, 0, 0)], up(prefix)              # (first slot, length, first position, new tokens at its end)
        desc["prefix_len"].append(prefix)
        desc["n_branches"].append(len(prior))
        desc["branch_begin"].append(len(desc["br_kv_off"]))
        for p, n in zip(prior, new):
            desc["br_kv_off"].append(at)
            desc["br_kv_len"].append(p + n)
            desc["br_q_len"].append(n)
            regions.append((at, p + n, prefix, n))                 # branches of a stage share the position IDs
            at += up(max(1, p + n))
        tail = case["tail"] + 1 if serial else 0
        if serial:
            regions.append((at, tail, prefix + sum(prior), 1))
        desc["tail_off"].append(at)
        desc["tail_len"].append(tail)
        desc["page_begin"].append(pages)
        desc["n_pages"].append((at + up(tail)) // ps)
        pages += desc["n_pages"][-1]
        reqs.append(regions)
    desc = {k: np.asarray(v, dtype=np.int32) for k, v in desc.items()}
    n_pool = pages + 3
    desc["page_ids"] = np.random.default_rng(seed).permutation(n_pool)[:pages].astype(np.int32)
    return desc, n_pool, reqs


def _slopes(case):
    return [2.0 ** (-8.0 * (h + 1) / case["hq"]) for h in range(case["hq"])]


def _axis_of_pair(case):
    half = case["d"] // 2
    if case["axes"] == 1:
        return [0] * half
    hw = 3 * half // 8                                              # 16 / 24 / 24 of 64 pairs, 8 / 12 / 12 of 32
    if not case["interleaved"]:
        return [0] * (half - 2 * hw) + [1] * hw + [2] * hw
    return [i % 3 if i < 3 * hw and i % 3 else 0 for i in range(half)]


def _inputs(case, seed):
    desc, n_pool, reqs = _layout(case, seed)
    hq, hkv, d, ps, dt = case["hq"], case["hkv"], case["d"], case["page"], _DTYPE[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    normal = lambda *size: torch.randn(*size, dtype=dt, device="cuda", generator=gen)   # noqa: E731
    s = {"case": case, "desc": desc, "n_pool": n_pool, "reqs": reqs}
    s["k_pool"], s["v_pool"] = normal(n_pool * hkv * ps * d), normal(n_pool * hkv * ps * d)
    tok = [(r, first + length - n + i, pos + length - n + i) for r, regions in enumerate(reqs) for first, length, pos, n in regions for i in range(n)]
    n = len(tok)
    s["n"], s["tok_pos"] = n, np.asarray([t[2] for t in tok], dtype=np.int32)
    slot, begin = np.asarray([t[1] for t in tok]), desc["page_begin"][[t[0] for t in tok]]
    s["tok_page"] = torch.from_numpy(desc["page_ids"][begin + slot // ps].astype(np.int64)).cuda()
    s["tok_row"] = torch.from_numpy((slot % ps).astype(np.int64)).cuda()
    if case["op"] == "step":
        # capped models have logits that come near the cap; without one they are of order 1
        s["q"] = normal(n, hq, d) * (5.0 if case["cap"] else 1.0)
        s["k"], s["v"] = normal(n, hkv, d), normal(n, hkv, d)
        s["pos"] = torch.from_numpy(s["tok_pos"])[None].cuda()
    else:
        # one projection's output, its three parts views of it
        packed = normal(n, hq + 2 * hkv, d) * 3.0
        s["q"], s["k"], s["v"] = packed[:, :hq], packed[:, hq:hq + hkv], packed[:, hq + hkv:]
        rng = np.random.default_rng(seed + 1)
        pos = np.stack([s["tok_pos"]] * case["axes"])
        if case["axes"] > 1:                                       # a third of the tokens are image patches
            image = rng.random(n) < 0.33
            pos = np.where(image[None], pos + rng.integers(0, 48, pos.shape), pos)
        s["pos"] = torch.from_numpy(pos.astype(np.int32)).cuda()
        if case["norm"]:
            gain = 5.0 if case["op"] == "layer" and case["cap"] else 1.0
            s["wq"], s["wk"] = ((1.0 + 0.2 * torch.randn(d, device="cuda", generator=gen)) * g for g in (gain, 1.0))
            s["wq"], s["wk"] = s["wq"].to(dt), s["wk"].to(dt)
        else:
            s["wq"] = s["wk"] = None
    return s


# ------------------------------------------------------------------------------------------ the program
def prepare(case, seed):
    s = _inputs(case, seed)
    n, hq, d, dt = s["n"], case["hq"], case["d"], _DTYPE[case["dtype"]]
    s["q_out"] = torch.empty(n, hq, d, dtype=dt, device="cuda")
    s["out"] = torch.empty(n, hq, d, dtype=dt, device="cuda")
    if own:
        from paper_2508_08895_b200 import binding as B
        s["B"] = B
        shape = B.make_shape(hq, case["hkv"], d, case["page"], case["dtype"], _THETA, d ** -0.5)
        mode = B.MODE_SERIAL if case["step"] == "serial" else B.MODE_BRANCH
        scores = B.Scores(cap=case["cap"], slopes=_slopes(case) if case["bias"] else None, rotated=case["op"] != "step" or not case["rope"])
        s["plan"] = B.Plan(shape, s["desc"], s["n_pool"], mode, stable_cache=True, scores=scores)
        s["step"] = B.serial_step if case["step"] == "serial" else B.branch_step
        if case["op"] != "step":
            s["norm"] = B.QkNorm(shape, s["wq"], s["wk"], _EPS, axis_of_pair=_axis_of_pair(case), rotate_q=True)
        return s
    # what the plan says, for the plain form: the angle of every pair, per request its pages, new tokens, and the
    # region, place and position of every slot
    s["freq"] = torch.tensor([_THETA ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64, device="cuda")
    s["axis"] = torch.tensor(_axis_of_pair(case), device="cuda")
    s["slopes"] = torch.tensor(_slopes(case), device="cuda")
    s["plain"], t0 = [], 0
    for r, regions in enumerate(s["reqs"]):
        b, e = int(s["desc"]["page_begin"][r]), int(s["desc"]["page_begin"][r] + s["desc"]["n_pages"][r])
        slots = (e - b) * case["page"]
        region, place, pos = np.full(slots, -1), np.zeros(slots, int), np.zeros(slots, int)
        tr, tp = [], []
        for i, (first, length, p0, n_new) in enumerate(regions):
            region[first:first + length], place[first:first + length] = i, np.arange(length)
            pos[first:first + length] = p0 + np.arange(length)
            tr += [i] * n_new
            tp += range(length - n_new, length)
        dev = lambda x: torch.from_numpy(np.asarray(x, dtype=np.int64)).cuda()   # noqa: E731
        s["plain"].append((dev(s["desc"]["page_ids"][b:e]), dev(region), dev(place), dev(pos), dev(tr), dev(tp), dev(s["tok_pos"][t0:t0 + len(tr)]), t0, t0 + len(tr)))
        t0 += len(tr)
    return s


def run(s):
    case = s["case"]
    if own:
        B, plan = s["B"], s["plan"]
        if case["op"] == "step":
            s["step"](plan, s["q"], s["k"], s["v"], s["k_pool"], s["v_pool"], s["out"])
            return {"out": s["out"], "k": s["k_pool"], "v": s["v_pool"]}
        B.qk_norm_append(plan, s["norm"], s["q"], s["k"], s["v"], s["pos"], s["k_pool"], s["v_pool"], s["q_out"])
        if case["op"] == "norm":
            return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}
        B.branch_attn(plan, s["q_out"], s["k_pool"], s["v_pool"], s["out"])
        return {"out": s["out"], "q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}
    q, k = s["q"].float(), s["k"].float()
    if case["op"] != "step" and case["norm"]:
        q, k = _rms(q, s["wq"]), _rms(k, s["wk"])
    if case["op"] != "step" or case["rope"]:
        angle = s["pos"].double()[s["axis"]].T * s["freq"]         # [n][d / 2]
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        q, k = _turn(q, cos, sin), _turn(k, cos, sin)
    _put(s, s["k_pool"], k)
    _put(s, s["v_pool"], s["v"])
    if case["op"] != "step":
        s["q_out"].copy_(q)
        if case["op"] == "norm":
            return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}
        q = s["q_out"].float()                                     # the queries between the two calls are of the storage type
    _attend(s, q)
    outs = {"out": s["out"], "k": s["k_pool"], "v": s["v_pool"]}
    return dict(outs, q=s["q_out"]) if case["op"] == "layer" else outs


# ------------------------------------------------------------------------------------ the plain forms
def _rms(x, w):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * w.float()


def _turn(x, cos, sin):
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _blocks(case, pool):
    """The pool as [page][KV head][8 rows][128-byte span][row][16-byte chunk][element]."""
    es = _ES[case["dtype"]]
    return pool.view(-1, case["hkv"], case["page"] // 8, case["d"] * es // 128, 8, 8, 16 // es)


def _put(s, pool, rows):
    """Token rows into their places of the pool."""
    case, es = s["case"], _ES[s["case"]["dtype"]]
    hkv, d = case["hkv"], case["d"]
    dev = pool.device
    x = rows.to(pool.dtype).reshape(-1, hkv, d * es // 128, 8, 16 // es)
    page, row = s["tok_page"][:, None, None, None], s["tok_row"][:, None, None, None]
    h = torch.arange(hkv, device=dev)[:, None, None]
    span = torch.arange(d * es // 128, device=dev)[:, None]
    _blocks(case, pool)[page, h, row // 8, span, row % 8, torch.arange(8, device=dev) ^ (row % 8)] = x


def _get(case, pool, pages):
    """The token rows of these pages: [slots][KV heads][head_dim]."""
    t, c = torch.arange(8, device=pool.device)[:, None], torch.arange(8, device=pool.device)
    x = _blocks(case, pool)[pages][:, :, :, :, t, c ^ t]
    return x.permute(0, 2, 4, 1, 3, 5, 6).reshape(-1, case["hkv"], case["d"])


def _attend(s, q):
    case = s["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g, scale, cap = hq // hkv, case["d"] ** -0.5, case["cap"]
    for pages, region, place, pos, tok_region, tok_place, tok_pos, t0, t1 in s["plain"]:
        k, v = _get(case, s["k_pool"], pages).float(), _get(case, s["v_pool"], pages).float()
        x = q[t0:t1].view(-1, hkv, g, d).permute(1, 2, 0, 3)                           # [KV head][g][token][d]
        p = torch.matmul(x, k.permute(1, 2, 0)[:, None]) * scale                       # [KV head][g][token][slot]
        if cap:
            p = torch.tanh(p / cap) * cap
        if case["bias"]:
            p = p - s["slopes"].view(hkv, g, 1, 1) * (tok_pos[:, None] - pos).float()
        # a branch's token sees the prefix and its own branch up to itself, a serial token everything
        seen = (region == 0) | ((region == tok_region[:, None]) & (place <= tok_place[:, None]))
        if case["step"] == "serial":
            seen = (region >= 0).expand(t1 - t0, -1)
        p = torch.where(seen, p, -math.inf)
        p = torch.exp(p - p.amax(-1, keepdim=True))
        o = torch.matmul(p / p.sum(-1, keepdim=True), v.permute(1, 0, 2)[:, None])
        s["out"][t0:t1] = o.permute(2, 0, 1, 3).reshape(-1, hq, d).to(s["out"].dtype)


# ------------------------------------------------------------------------------------ in 64 bits, from the definition
def exact(case, seed):
    s = _inputs(case, seed)
    hq, hkv, d, ps, es, n = case["hq"], case["hkv"], case["d"], case["page"], _ES[case["dtype"]], s["n"]
    g, dt = hq // hkv, _DTYPE[case["dtype"]]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    if case["op"] != "step" and case["norm"]:
        q = q / (q.pow(2).sum(2, keepdim=True) / d + _EPS).sqrt() * s["wq"].double()
        k = k / (k.pow(2).sum(2, keepdim=True) / d + _EPS).sqrt() * s["wk"].double()
    if case["op"] != "step" or case["rope"]:
        i = torch.arange(d // 2, dtype=torch.float64, device="cuda")
        which = torch.tensor(_axis_of_pair(case), device="cuda")
        theta = s["pos"].double().index_select(0, which).t() / torch.pow(torch.tensor(_THETA, dtype=torch.float64, device="cuda"), 2 * i / d)
        w = torch.polar(torch.ones_like(theta), theta).unsqueeze(1)
        turned = lambda x: torch.view_as_real(torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous()) * w).transpose(-1, -2).reshape(x.shape)  # noqa: E731
        q, k = turned(q), turned(k)
    # byte b of row r of a (page, head) tile: (r / 8) 8 d es + (b / 128) 1024 + (r mod 8) 128 + ((b mod 128 / 16) ^ (r mod 8)) 16 + b mod 16
    b = torch.arange(d, device="cuda") * es

    def where(page, row):                                           # [rows][hkv][d] element numbers
        page, row = page.view(-1, 1, 1), row.view(-1, 1, 1)
        head = torch.arange(hkv, device="cuda").view(1, -1, 1)
        inside = (row // 8) * (8 * d * es) + (b // 128) * 1024 + (row % 8) * 128 + (((b % 128) // 16) ^ (row % 8)) * 16 + b % 16
        return ((page * hkv + head) * (ps * d * es) + inside) // es

    places = where(s["tok_page"], s["tok_row"])
    kp, vp = s["k_pool"].double(), s["v_pool"].double()
    kp[places.reshape(-1)] = k.reshape(-1)
    vp[places.reshape(-1)] = v.reshape(-1)
    outs = {"k": kp, "v": vp}
    if case["op"] != "step":
        outs["q"] = q
        if case["op"] == "norm":
            return outs
        q = q.to(dt).double()
    # the cache holds keys of the storage type
    held = kp.clone()
    held[places.reshape(-1)] = k.reshape(-1).to(dt).double()
    out = torch.empty(n, hq, d, dtype=torch.float64, device="cuda")
    slopes = torch.tensor(_slopes(case), dtype=torch.float64, device="cuda").view(hkv, g, 1, 1)
    t = 0
    for r, regions in enumerate(s["reqs"]):
        ids = torch.from_numpy(s["desc"]["page_ids"][int(s["desc"]["page_begin"][r]):][:int(s["desc"]["n_pages"][r])].astype(np.int64)).cuda()

        def rows(region):                                           # keys, values and positions of a region's tokens
            slot = torch.arange(region[0], region[0] + region[1], device="cuda")
            at = where(ids[slot // ps], slot % ps)
            return held[at], vp[at], region[2] + torch.arange(region[1], device="cuda")

        parts = [rows(x) for x in regions]
        for i, region in enumerate(regions):
            m = region[3]
            if m == 0:
                continue
            read = parts if case["step"] == "serial" else [parts[0], parts[i]]
            keys, values, pos = (torch.cat([x[j] for x in read]) for j in range(3))
            mine = parts[i][2][region[1] - m:]
            x = q[t:t + m].reshape(m, hkv, g, d).permute(1, 2, 0, 3).reshape(hkv, g * m, d)
            y = (x @ keys.permute(1, 2, 0)).reshape(hkv, g, m, -1) / math.sqrt(d)
            if case["cap"]:
                y = case["cap"] * torch.tanh(y / case["cap"])
            if case["bias"]:
                y = y - slopes * (mine.view(-1, 1) - pos).double()
            hidden = torch.arange(keys.shape[0], device="cuda") > torch.arange(keys.shape[0] - m, keys.shape[0], device="cuda").view(-1, 1)
            y = torch.softmax(y.masked_fill(hidden, -math.inf), -1).reshape(hkv, g * m, -1)
            out[t:t + m] = (y @ values.permute(1, 0, 2)).reshape(hkv, g, m, d).permute(2, 0, 1, 3).reshape(m, hq, d)
            t += m
    return dict(outs, out=out)


# --------------------------------------------------------------------------------- what a pass must move
def work(case):
    hq, hkv, d, es = case["hq"], case["hkv"], case["d"], _ES[case["dtype"]]
    cached, pairs, n = 0, 0, 0
    for prefix, prior, new in _lengths(case):
        if case["step"] == "serial":
            cached += prefix + sum(prior) + case["tail"]
            pairs += prefix + sum(prior) + case["tail"] + 1
            n += 1
        else:
            cached += prefix + sum(prior)
            pairs += sum(m * (prefix + p) + m * (m + 1) // 2 for p, m in zip(prior, new))
            n += sum(new)
    # q, k_new, v_new in; q or out, and the new cache rows, out
    ends = 2 * n * (hq + 2 * hkv) * d * es
    norm = n * (hq + hkv) * d * ((4 if case["norm"] else 0) + 3) if case["op"] != "step" else 0
    if case["op"] == "norm":
        return {"bytes": ends, "flops": norm}
    # cached K and V once
    rows = 2 * hkv * d * es * cached
    return {"bytes": ends + rows + (2 * n * hq * d * es if case["op"] == "layer" else 0), "flops": norm + 4 * d * hq * pairs}
