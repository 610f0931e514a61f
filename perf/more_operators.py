"""The operators of a stage whose cache holds one latent vector a token, as cases that can be timed and compared.

  rotate     rotary positions of rows of heads: pairs in halves or interleaved, all of a head's columns or its first ones,
             frequencies plain or scaled for long contexts; `inverse` turns back
  append     the latent's norm, the rotation of the part that all heads' keys share and of the query heads' parts, and the
             cache append, in one pass over a call's rows
  product    products head by head: queries into the latent space, attention results out of it
  attention  tree attention of query rows in the latent space over the cache, every head over the same rows

With `own` the cases run through the library's entry points, else in plain torch in 32 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
THETA, EPS = 500000.0, 1e-5
# columns of the latent, of the rotated part beside it, of a query head's other part, of a value head
SPACES = {"wide": (512, 64, 128, 128), "slim": (256, 32, 64, 64)}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
FACTOR, ORIGINAL = 8.0, 8192.0              # of the scaled frequencies: the context grew from 8192 by this factor
BAND = (1.0, 4.0)                           # turns within the original context between which the bands blend
RAMP = (32.0, 1.0)                          # ... between which the ramp goes
RAMP_GAIN = 0.1 * math.log(FACTOR) + 1.0


def listed():
    return [
        # a drafted token's query heads: the smallest rotation
        {"name": "rotate_one", "kind": "rotate", "rows": 1, "heads": 32, "d": 128, "dims": 128, "layout": "half", "scaling": "bands", "type": "bf16", "inverse": False},
        # the keys of a long committed context on their way into the cache, an odd number of them, half of every head rotated
        {"name": "rotate_context", "kind": "rotate", "rows": 32749, "heads": 8, "d": 128, "dims": 64, "layout": "interleaved", "scaling": "ramp", "type": "bf16", "inverse": False},
        # one new node: the smallest append
        {"name": "append_one", "kind": "append", "space": "wide", "heads": 16, "layout": "interleaved", "scaling": "ramp", "requests": 1, "t_lo": 1, "t_hi": 1, "p_lo": 512, "p_hi": 512, "page": 0, "sizes": 1},
        # 32 requests whose trees are all new
        {"name": "append_batch32", "kind": "append", "space": "wide", "heads": 64, "layout": "half", "scaling": "none", "requests": 32, "t_lo": 8, "t_hi": 32, "p_lo": 512, "p_hi": 4096, "page": 0, "sizes": 2},
        # the queries of a single node into the latent space: the smallest product
        {"name": "absorb_one", "kind": "product", "rows": 1, "heads": 16, "n": 512, "k": 128},
        # a level's results out of it
        {"name": "values_level64", "kind": "product", "rows": 64, "heads": 64, "n": 128, "k": 512},
        # the queries of a cold batch
        {"name": "absorb_batch", "kind": "product", "rows": 637, "heads": 64, "n": 512, "k": 128},
        # a stall: the true token alone behind a short context, where latency counts
        {"name": "attn_one_512", "kind": "attention", "space": "wide", "heads": 16, "requests": 1, "t_lo": 1, "t_hi": 1, "p_lo": 512, "p_hi": 512, "page": 0, "sizes": 3},
        # the benchmark's step: a level's width of 64 nodes behind 2048 slots
        {"name": "attn_tree64_2k", "kind": "attention", "space": "wide", "heads": 32, "requests": 1, "t_lo": 64, "t_hi": 64, "p_lo": 2048, "p_hi": 2048, "page": 0, "sizes": 4},
        # a long context fed a few nodes per step; a length that fills no tile
        {"name": "attn_few_32k", "kind": "attention", "space": "wide", "heads": 16, "requests": 1, "t_lo": 5, "t_hi": 5, "p_lo": 32749, "p_hi": 32749, "page": 0, "sizes": 5},
        # dynamic batching in steady state, ragged, the cache in pages
        {"name": "attn_batch32_paged", "kind": "attention", "space": "wide", "heads": 16, "requests": 32, "t_lo": 1, "t_hi": 8, "p_lo": 512, "p_hi": 4096, "page": 64, "sizes": 6},
        # many heads and a tree of two levels' width
        {"name": "attn_tree128_64heads", "kind": "attention", "space": "wide", "heads": 64, "requests": 1, "t_lo": 128, "t_hi": 128, "p_lo": 4096, "p_hi": 4096, "page": 0, "sizes": 7},
    ]


def _log_int(r, lo, hi):
    return int(round(math.exp(r.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    r = rng
    kind = r.choice(["attention", "attention", "attention", "append", "product", "product", "rotate"])
    while True:
        if kind == "rotate":
            d = r.choice([64, 128, 128])
            case = {"kind": kind, "rows": _log_int(r, 1, 32768), "heads": r.choice([1, 3, 8, 32, 64]), "d": d, "dims": r.choice([d, d, d // 2]),
                    "layout": r.choice(["half", "interleaved"]), "scaling": r.choice(["none", "linear", "bands", "ramp"]),
                    "type": r.choice(["bf16", "bf16", "f32"]), "inverse": r.random() < 0.25}
            if case["rows"] * case["heads"] * d <= 32749 * 8 * 128:
                return case
            continue
        if kind == "product":
            n, k = r.choice([(512, 128), (128, 512), (256, 64), (64, 256)])
            case = {"kind": kind, "rows": _log_int(r, 1, 1024), "heads": r.choice([8, 16, 32, 64, 128]), "n": n, "k": k}
            if case["rows"] * case["heads"] <= 637 * 64:
                return case
            continue
        R = 1 if r.random() < 0.5 else _log_int(r, 2, 32)
        p_lo = _log_int(r, 1, 32768 if R == 1 else 4096)
        t_lo = _log_int(r, 1, 128 if R == 1 else 16)
        case = {"kind": kind, "space": r.choice(["wide", "wide", "slim"]), "heads": r.choice([8, 16, 32, 64, 128]), "requests": R, "t_lo": t_lo,
                "t_hi": t_lo if R == 1 else 2 * t_lo, "p_lo": p_lo, "p_hi": p_lo if R == 1 else 2 * p_lo, "page": r.choice([0, 32, 64, 256]), "sizes": r.randrange(1 << 20)}
        if kind == "append":
            case["page"] = 0
            case["layout"], case["scaling"] = r.choice(["half", "interleaved"]), r.choice(["none", "linear", "bands", "ramp"])
            return case
        w = work(case)
        if w["flops"] <= max(work(c)["flops"] for c in listed()) and w["bytes"] <= max(work(c)["bytes"] for c in listed()):
            return case


# ---- inputs: values from the seed, sizes and the shapes of the trees from the case --------------------------------
def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + what) % (1 << 62))


def _normal(seed, what, *size, dtype=torch.bfloat16):
    return torch.randn(*size, generator=_gen(seed, what), device=DEV, dtype=dtype)


def _sizes(case):
    """(context lengths, new nodes) of the requests."""
    r = random.Random("sizes %d" % case["sizes"])
    R = range(case["requests"])
    return [r.randint(case["p_lo"], case["p_hi"]) for _ in R], [r.randint(case["t_lo"], case["t_hi"]) for _ in R]


def _trees(case):
    """Parents of every request's nodes: sequential attachment, at most four children and twelve levels."""
    r, out = random.Random("trees %d" % case["sizes"]), []
    for n in _sizes(case)[1]:
        parents, lev, kids = [], [], {-1: 0}
        for i in range(n):
            p = r.choice([j for j in range(-1, i) if kids[j] < 4 and (j < 0 or lev[j] < 11)] or [-1])
            kids[p] += 1
            kids[i] = 0
            lev.append(0 if p < 0 else lev[p] + 1)
            parents.append(p)
        out.append(parents)
    return out


def _ancestors(parents):
    up = np.zeros((len(parents), len(parents)), bool)
    for i, p in enumerate(parents):
        if p >= 0:
            up[i] = up[p]
        up[i, i] = True
    return up


def _positions(case):
    depth = [int(u.sum()) - 1 for p in _trees(case) for u in _ancestors(p)]
    Ps, Ts = _sizes(case)
    return np.repeat(Ps, Ts) + np.asarray(depth)


def _cache_rows(case, seed, q, n):
    """What a request's n slots hold: normed latents with a few strong channels, and rotated key parts."""
    c, rope, _, _ = SPACES[case["space"]]
    g = _gen(seed, 1000 + q)
    x = torch.randn(n, c + rope, generator=g, device=DEV)
    return (x * torch.exp(0.3 * torch.randn(c + rope, generator=g, device=DEV))).to(torch.bfloat16)


# ---- what the program holds before the call --------------------------------------------------------------------
def _rope(case, dims):
    """The frequencies of a case's rotation as a program hands them to the library."""
    import paper_2504_04104_amd as sp
    kind = case["scaling"]
    scaling = {"none": None, "linear": ("linear", FACTOR), "bands": ("bands", FACTOR, ORIGINAL, *BAND), "ramp": ("ramp", FACTOR, ORIGINAL, *RAMP)}[kind]
    return sp.Rope(case["layout"], dims, THETA, scaling=scaling, gain=RAMP_GAIN if kind == "ramp" else 1.0)


def _stage(case, Ps, Ts, gain=None):
    """A stage with one layer of latent cache, its requests initialised and their trees inserted."""
    import paper_2504_04104_amd as sp
    c, rope, n, _ = SPACES[case["space"]]
    page, base, off = case["page"], [], 0
    for P, T in zip(Ps, Ts):
        base.append(0 if page else off)
        off += -(-(P + T) // page) * page if page else P + T
    st = sp.LatentStage(1, case["heads"], c, rope, scale=1 / math.sqrt(n + rope), rms_eps=EPS, kv_slots=off, max_requests=len(Ps) + 2, max_batch_nodes=sum(Ts),
                        page_slots=page, norms=None if gain is None else [gain], rope=_rope(case, rope) if "scaling" in case else None)
    if page:                # two requests that came and went: the pages are handed out of order from here on
        third = max(1, off // page // 3) * page
        for q in (len(Ps), len(Ps) + 1):
            if third * 2 <= off:
                st.request_init(q, 0, third, third)
        for q in (len(Ps), len(Ps) + 1):
            if third * 2 <= off:
                st.request_release(q)
    for q, (P, T) in enumerate(zip(Ps, Ts)):
        st.request_init(q, base[q], P + T, P)
    st.tree_insert_batch(list(range(len(Ps))), _trees(case))
    return st, base


def prepare(case, seed):
    s = {"case": case}
    if case["kind"] == "rotate":
        dt = TYPES[case["type"]]
        s["x"] = _normal(seed, 1, case["rows"], case["heads"], case["d"], dtype=torch.float32).to(dt)
        # a context's rows in order, from somewhere in a long one
        start = int(torch.randint(0, 1 << 17, (1,), generator=_gen(seed, 2), device=DEV))
        s["pos"] = torch.arange(start, start + case["rows"], dtype=torch.int32, device=DEV)
        if own:
            s["rope"] = _rope(case, case["dims"])
        return s
    if case["kind"] == "product":
        s["x"] = _normal(seed, 3, case["rows"], case["heads"], case["k"])
        s["w"] = _normal(seed, 4, case["heads"], case["n"], case["k"]).mul_(case["k"] ** -0.5)
        return s
    c, rope, n, _ = SPACES[case["space"]]
    Ps, Ts = _sizes(case)
    s["ids"], s["first"], s["n"], M = list(range(len(Ps))), [0] * len(Ps), Ts, sum(Ts)
    if case["kind"] == "append":
        s["q"] = _normal(seed, 5, M, case["heads"], n + rope)
        s["kv"] = _normal(seed, 6, M, c + rope, dtype=torch.float32).mul_(1.7).to(torch.bfloat16)
        s["gain"] = (1 + 0.1 * _normal(seed, 7, c, dtype=torch.float32)).to(torch.bfloat16)
        if own:
            s["stage"], base = _stage(case, Ps, Ts, s["gain"])
            s["rows"] = [s["stage"].kv_view()[0, b + P:b + P + T] for b, P, T in zip(base, Ps, Ts)]
        else:
            s["pos"] = torch.from_numpy(_positions(case)).to(DEV)
        return s
    s["q"] = _normal(seed, 8, M, case["heads"], c + rope)
    if own:
        s["stage"], _ = _stage(case, Ps, Ts)
        for q, (P, T) in enumerate(zip(Ps, Ts)):
            s["stage"].kv_store(q, 0, 0, _cache_rows(case, seed, q, P + T))
        return s
    # one block for every request, as long as the longest
    R, n, S = len(Ps), max(Ts), max(P + T for P, T in zip(Ps, Ts))
    s["cache"] = torch.zeros(R, S, c + rope, dtype=torch.bfloat16, device=DEV)
    seen, row = np.zeros((R, n, S), bool), np.zeros((R, n), np.int64)
    seen[:, :, 0] = True
    at = 0
    for q, (P, T, parents) in enumerate(zip(Ps, Ts, _trees(case))):
        s["cache"][q, :P + T] = _cache_rows(case, seed, q, P + T)
        seen[q, :T, :P], seen[q, :T, P:P + T] = True, _ancestors(parents)
        row[q, :T] = np.arange(at, at + T)
        at += T
    s["seen"], s["row"] = torch.from_numpy(seen).to(DEV), torch.from_numpy(row).to(DEV)
    s["real"] = torch.from_numpy(np.flatnonzero(np.arange(n)[None] < np.asarray(Ts)[:, None])).to(DEV)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if case["kind"] == "rotate":
        if own:
            import paper_2504_04104_amd as sp
            return sp.rotate(s["x"], s["pos"], s["rope"], inverse=case["inverse"])
        return _turn(s["x"].float(), s["pos"], case, case["dims"], case["inverse"]).to(s["x"].dtype)
    if case["kind"] == "product":
        if own:
            import paper_2504_04104_amd as sp
            return sp.head_product(s["x"], s["w"])
        y = torch.bmm(s["x"].float().transpose(0, 1).contiguous(), s["w"].float().transpose(1, 2).contiguous())
        return y.transpose(0, 1).contiguous().to(torch.bfloat16)
    c, rope, n, _ = SPACES[case["space"]]
    if case["kind"] == "append":
        if own:
            q = s["stage"].append(0, s["ids"], s["first"], s["n"], s["q"][..., n:], s["kv"])
            return {"q": q, "rows": s["rows"]}
        kv = s["kv"].float()
        latent = kv[:, :c] * torch.rsqrt(kv[:, :c].square().mean(-1, keepdim=True) + EPS) * s["gain"].float()
        rows = torch.cat([latent, _turn(kv[:, None, c:], s["pos"], case, rope)[:, 0]], -1).to(torch.bfloat16)
        return {"q": _turn(s["q"][..., n:].float(), s["pos"], case, rope).to(torch.bfloat16), "rows": list(rows.split(s["n"]))}
    if own:
        return s["stage"].attention(0, s["ids"], s["first"], s["n"], s["q"])
    R, T, S = s["seen"].shape
    H = case["heads"]
    rows = s["cache"].float()
    q = s["q"].float()[s["row"]].reshape(R, T * H, c + rope)
    sc = torch.bmm(q, rows.transpose(1, 2).contiguous()) / math.sqrt(n + rope)
    sc = sc.reshape(R, T, H, S).masked_fill(~s["seen"][:, :, None], -math.inf)
    p = torch.exp(sc - sc.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = torch.bmm(p.reshape(R, T * H, S), rows[..., :c].contiguous())
    return o.reshape(R * T, H, c)[s["real"]].to(torch.bfloat16)


def _frequencies(case, dims):
    """Angle per position of every pair, in 64 bits."""
    t = torch.arange(dims // 2, device=DEV, dtype=torch.float64)
    f = THETA ** (-2 * t / dims)
    if case["scaling"] == "linear":
        f = f / FACTOR
    if case["scaling"] == "bands":
        turns = ORIGINAL * f / (2 * math.pi)
        keep = ((turns - BAND[0]) / (BAND[1] - BAND[0])).clamp(0, 1)
        f = keep * f + (1 - keep) * f / FACTOR
    if case["scaling"] == "ramp":
        lo, hi = (dims * math.log(ORIGINAL / (b * 2 * math.pi)) / (2 * math.log(THETA)) for b in RAMP)
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), dims - 1)
        away = ((t - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = (1 - away) * f + away * f / FACTOR
    return f


def _turn(x, pos, case, dims, inverse=False):
    """x [rows, heads, d] with its first dims columns turned; the angles of far positions lose what matters in 32 bits."""
    ang = pos.double()[:, None, None] * _frequencies(case, dims)
    gain = RAMP_GAIN if case["scaling"] == "ramp" else 1.0
    cos, sin = (torch.cos(ang) * gain).float(), (torch.sin(ang) * (-gain if inverse else gain)).float()
    part = x[..., :dims]
    if case["layout"] == "half":
        a, b = part[..., :dims // 2], part[..., dims // 2:]
        part = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        part = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([part, x[..., dims:]], -1)


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "rotate":
        values, e = case["rows"] * case["heads"] * case["d"], 4 if case["type"] == "f32" else 2
        return {"bytes": 2 * values * e + 4 * case["rows"], "flops": 3 * case["rows"] * case["heads"] * case["dims"]}
    if case["kind"] == "product":
        m, h, n, k = case["rows"], case["heads"], case["n"], case["k"]
        return {"bytes": 2 * h * (n * k + m * (n + k)), "flops": 2 * m * h * n * k}
    c, rope, _, _ = SPACES[case["space"]]
    H = case["heads"]
    Ps, Ts = _sizes(case)
    M = sum(Ts)
    if case["kind"] == "append":
        return {"bytes": 4 * M * (c + rope + H * rope) + 2 * c, "flops": M * (4 * c + 3 * rope * (H + 1))}
    spans = [P + T for P, T in zip(Ps, Ts)]
    return {"bytes": 2 * (c + rope) * sum(spans) + 2 * M * H * (2 * c + rope), "flops": 2 * H * (2 * c + rope) * sum(s * t for s, t in zip(spans, Ts))}


# ---- the same pass in 64 bits -------------------------------------------------------------------------------------
def _angles(case, dims, pos):
    """[rows, pairs] in 64 bits, a pair at a time."""
    out = []
    for t in range(dims // 2):
        f = math.exp(-2 * t / dims * math.log(THETA))
        slow, wave = f / FACTOR, 2 * math.pi / f
        if case["scaling"] == "linear":
            f = slow
        elif case["scaling"] == "bands":
            if wave > ORIGINAL / BAND[0]:
                f = slow
            elif wave >= ORIGINAL / BAND[1]:
                part = (ORIGINAL / wave - BAND[0]) / (BAND[1] - BAND[0])
                f = slow + part * (f - slow)
        elif case["scaling"] == "ramp":
            at = [dims / 2 * math.log(ORIGINAL / (2 * math.pi * b)) / math.log(THETA) for b in RAMP]
            first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), dims - 1)
            part = min(max((t - first) / max(last - first, 0.001), 0.0), 1.0)
            f = f + part * (slow - f)
        out.append(f)
    return pos.double()[:, None] * torch.tensor(out, dtype=torch.float64, device=DEV)


def _spun(x, pos, case, dims, inverse=False):
    """The rotation as products of complex numbers."""
    gain = RAMP_GAIN if case["scaling"] == "ramp" else 1.0
    ang = _angles(case, dims, pos)[:, None]
    spin = torch.polar(torch.full_like(ang, gain), -ang if inverse else ang)
    y = x.clone()
    if case["layout"] == "half":
        z = torch.complex(x[..., :dims // 2].contiguous(), x[..., dims // 2:dims].contiguous()) * spin
        y[..., :dims // 2], y[..., dims // 2:dims] = z.real, z.imag
    else:
        z = torch.view_as_complex(x[..., :dims].unflatten(-1, (-1, 2)).contiguous()) * spin
        y[..., :dims] = torch.view_as_real(z).flatten(-2)
    return y


def exact(case, seed):
    if case["kind"] == "rotate":
        s = prepare(case, seed)
        return _spun(s["x"].double(), s["pos"], case, case["dims"], case["inverse"])
    if case["kind"] == "product":
        s = prepare(case, seed)
        return torch.stack([s["x"][:, h].double() @ s["w"][h].double().T for h in range(case["heads"])], 1)
    c, rope, n, _ = SPACES[case["space"]]
    Ps, Ts = _sizes(case)
    M = sum(Ts)
    if case["kind"] == "append":
        s = prepare(case, seed)
        pos = torch.from_numpy(_positions(case)).to(DEV)
        kv = s["kv"].double()
        latent = kv[:, :c] / torch.sqrt((kv[:, :c] ** 2).sum(-1, keepdim=True) / c + EPS) * s["gain"].double()
        key = _spun(kv[:, None, c:], pos, case, rope)[:, 0]
        return {"q": _spun(s["q"][..., n:].double(), pos, case, rope), "rows": list(torch.cat([latent, key], 1).split(Ts))}
    q, out, at = _normal(seed, 8, M, case["heads"], c + rope).double(), [], 0
    for r, (P, T, parents) in enumerate(zip(Ps, Ts, _trees(case))):
        rows = _cache_rows(case, seed, r, P + T).double()
        seen = torch.ones(T, P + T, dtype=torch.bool, device=DEV)
        seen[:, P:] = torch.from_numpy(_ancestors(parents)).to(DEV)
        heads = []
        for h in range(case["heads"]):
            sc = (q[at:at + T, h] @ rows.T) / math.sqrt(n + rope)
            heads.append(torch.softmax(sc.masked_fill(~seen, -math.inf), -1) @ rows[:, :c])
        out.append(torch.stack(heads, 1))
        at += T
    return torch.cat(out)
