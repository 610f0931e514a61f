"""The operators of a stage whose weights and cache are held in 4 bits, as cases that can be timed and compared.

  attention  tree attention of a call's query rows over a cache in 4 bits
  append     norms of the query and key heads, position rotation and the cache append, in one pass over the rows of the
             QKV projection; the cache in 4 bits, bfloat16 or float32
  product    rows times a matrix of 4-bit weights with a scale for every 32 columns; `gated`: silu(gate) * up

4 bits: groups of 32 consecutive values (of a head, of a weight row) share a power of two, the smallest 2^e (-100 <= e <= 125)
with max |x| <= 6 * 2^e; a value is sign * {0, 0.5, 1, 1.5, 2, 3, 4, 6} * 2^e, rounded to nearest, ties to the even code.

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
HEADS = {                                   # query heads, KV heads, head size
    "8b": (32, 8, 128),
    "70b": (64, 8, 128),
    "narrow": (16, 4, 64),
    "tiny": (4, 4, 64),
}
TYPES = {"fp4": torch.bfloat16, "bf16": torch.bfloat16, "f32": torch.float32}      # storage of the cache -> of the rows


def listed():
    return [
        # a stall: the true token alone behind a short context, where latency counts
        {"name": "attn_one_512", "kind": "attention", "heads": "8b", "requests": 1, "t_lo": 1, "t_hi": 1, "p_lo": 512, "p_hi": 512, "page": 0, "sizes": 1},
        # the benchmark's step: a level's width of 64 nodes behind 2048 slots
        {"name": "attn_tree64_2k", "kind": "attention", "heads": "8b", "requests": 1, "t_lo": 64, "t_hi": 64, "p_lo": 2048, "p_hi": 2048, "page": 0, "sizes": 2},
        # a long context fed a few nodes per step; a length that fills no tile
        {"name": "attn_few_32k", "kind": "attention", "heads": "8b", "requests": 1, "t_lo": 5, "t_hi": 5, "p_lo": 32749, "p_hi": 32749, "page": 0, "sizes": 3},
        # dynamic batching in steady state, ragged, the cache in pages
        {"name": "attn_batch32_paged", "kind": "attention", "heads": "8b", "requests": 32, "t_lo": 1, "t_hi": 8, "p_lo": 512, "p_hi": 4096, "page": 64, "sizes": 4},
        # the 70B shape with a tree of two levels' width
        {"name": "attn_tree128_70b", "kind": "attention", "heads": "70b", "requests": 1, "t_lo": 128, "t_hi": 128, "p_lo": 4096, "p_hi": 4096, "page": 0, "sizes": 5},
        # one new node: the smallest append
        {"name": "append_one_fp4", "kind": "append", "heads": "8b", "cache": "fp4", "norms": True, "requests": 1, "t_lo": 1, "t_hi": 1, "p_lo": 512, "p_hi": 512, "sizes": 6},
        # a level of the tree behind a long context, into a cache in 4 bits
        {"name": "append_level64_fp4", "kind": "append", "heads": "8b", "cache": "fp4", "norms": True, "requests": 1, "t_lo": 64, "t_hi": 64, "p_lo": 32749, "p_hi": 32749, "sizes": 7},
        # 32 requests whose trees are all new, a cache in bfloat16
        {"name": "append_batch32_bf16", "kind": "append", "heads": "8b", "cache": "bf16", "norms": True, "requests": 32, "t_lo": 8, "t_hi": 32, "p_lo": 512, "p_hi": 4096, "sizes": 8},
        # the output projection of a single row: the smallest product
        {"name": "product_1_4096", "kind": "product", "rows": 1, "n": 4096, "k": 4096, "gated": False},
        # the down projection of a few nodes
        {"name": "product_9_down", "kind": "product", "rows": 9, "n": 4096, "k": 14336, "gated": False},
        # gate and up of a level's 64 nodes
        {"name": "gated_64", "kind": "product", "rows": 64, "n": 14336, "k": 4096, "gated": True},
        # gate and up of the 70B shape over the rows of a cold batch
        {"name": "gated_200_70b", "kind": "product", "rows": 200, "n": 28672, "k": 8192, "gated": True},
    ]


def _log_int(r, lo, hi):
    return int(round(math.exp(r.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    r = rng
    kind = r.choice(["attention", "attention", "append", "product", "product"])
    while True:
        if kind == "product":
            gated = r.random() < 0.5
            case = {"kind": kind, "rows": _log_int(r, 1, 256), "n": 16 * _log_int(r, 16, 1792), "k": 32 * _log_int(r, 8, 896), "gated": gated}
            if case["rows"] * case["n"] * case["k"] * (2 if gated else 1) > 200 * 28672 * 8192 or case["n"] * case["k"] > 28672 * 8192:
                continue
            return case
        R = 1 if r.random() < 0.5 else _log_int(r, 2, 32)
        p_lo = _log_int(r, 1 if kind == "append" else 16, 32768 if R == 1 else 4096)
        t_lo = _log_int(r, 1, 128 if R == 1 else 16)
        case = {"kind": kind, "heads": r.choice(["8b", "8b", "70b", "narrow"]), "requests": R, "t_lo": t_lo,
                "t_hi": t_lo if R == 1 else 2 * t_lo, "p_lo": p_lo, "p_hi": p_lo if R == 1 else 2 * p_lo, "sizes": r.randrange(1 << 20)}
        if kind == "append":
            case["cache"] = "bf16" if R > 1 else r.choice(["fp4", "fp4", "bf16", "f32"])
            case["norms"] = r.random() < 0.75
            return case
        case["page"] = r.choice([0, 32, 64, 256])
        w = work(case)
        if w["flops"] <= work(_MOST_ROWS)["flops"] and w["bytes"] <= work(_MOST_BYTES)["bytes"]:
            return case


_MOST_ROWS = {"kind": "attention", "heads": "70b", "requests": 1, "t_lo": 128, "t_hi": 128, "p_lo": 4096, "p_hi": 4096, "page": 0, "sizes": 5}
_MOST_BYTES = {"kind": "attention", "heads": "8b", "requests": 32, "t_lo": 1, "t_hi": 8, "p_lo": 4096, "p_hi": 4096, "page": 64, "sizes": 4}


# ---- inputs: values from the seed, sizes and the shapes of the trees from the case --------------------------------
def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + what) % (1 << 62))


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


def _cache_rows(case, seed, q, n):
    """K and V of a request's n slots, [2, n, n_kv, d_head]: keys with a few strong channels, as models have them."""
    _, kv, dh = HEADS[case["heads"]]
    g = _gen(seed, 1000 + q)
    x = torch.randn(2, n, kv, dh, generator=g, device=DEV)
    x[0] *= torch.exp(0.5 * torch.randn(kv, dh, generator=g, device=DEV))
    return x.to(torch.bfloat16)


def _query_rows(case, seed, M):
    nq, _, dh = HEADS[case["heads"]]
    return torch.randn(M, nq * dh, generator=_gen(seed, 1), device=DEV, dtype=torch.bfloat16)


def _qkv_rows(case, seed, M):
    """Rows of the QKV projection and the gains of the head norms."""
    nq, kv, dh = HEADS[case["heads"]]
    g, dt = _gen(seed, 2), TYPES[case["cache"]]
    x = torch.randn(M, (nq + 2 * kv) * dh, generator=g, device=DEV) * 1.3
    gains = 1 + 0.1 * torch.randn(2, dh, generator=g, device=DEV)
    return x.to(dt), gains.to(dt)


def _matrix(case, seed):
    rows = case["n"] * (2 if case["gated"] else 1)
    w = torch.randn(rows, case["k"], generator=_gen(seed, 3), device=DEV, dtype=torch.bfloat16)
    return w.mul_(0.02)


def _rows(case, seed):
    return torch.randn(case["rows"], case["k"], generator=_gen(seed, 4), device=DEV, dtype=torch.bfloat16)


# ---- 4 bits in plain torch: two codes a byte (low half first), a biased exponent a group ----------------------------
_EDGES = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))
_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _to_fp4(x):
    x = x.float().unflatten(-1, (-1, 32))
    bits = x.abs().amax(-1, keepdim=True).view(torch.int32)
    biased = ((bits >> 23) - 2 + ((bits & 0x7fffff) > 0x400000).int()).clamp(27, 252)
    v = x * ((254 - biased) << 23).view(torch.float32)
    a = v.abs()
    code = torch.zeros(a.shape, dtype=torch.uint8, device=a.device)
    for edge, even in _EDGES:
        code += (a >= edge) if even else (a > edge)
    code += (torch.signbit(v)).to(torch.uint8) * 8
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), biased.squeeze(-1).to(torch.uint8)


def _from_fp4(codes, biased):
    table = torch.tensor(_VALUES, device=codes.device)
    v = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).flatten(-2)
    scale = (biased.int() << 23).view(torch.float32)
    return (v.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


# ---- what the program holds before the call --------------------------------------------------------------------
def _stage(case, Ps, Ts, page, dtype, flags, gains=None):
    """A stage with one layer of these heads, its requests initialised and their trees inserted."""
    import paper_2504_04104_amd as sp
    from workloads import ModelShape
    nq, kv, dh = HEADS[case["heads"]]
    sh = ModelShape(1, 256, nq, kv, dh, 256, EPS, THETA, "f32" if dtype == torch.float32 else "bf16")
    w = {"wqkv": ((nq + 2 * kv) * dh, 256), "wo": (256, nq * dh), "wgu": (512, 256), "wd": (256, 256), "norm1": (256,), "norm2": (256,)}
    layer = {k: torch.zeros(*v, device=DEV, dtype=dtype) for k, v in w.items()}
    base, off = [], 0
    for P, T in zip(Ps, Ts):
        base.append(0 if page else off)
        off += -(-(P + T) // page) * page if page else P + T
    st = sp.Stage(sh, [layer], kv_slots=off, max_requests=len(Ps) + 2, max_batch_nodes=sum(Ts), flags=flags | (sp.SP_FLAG_PAGED_KV if page else 0),
                  page_slots=page, head_norms=None if gains is None else [{"q": gains[0], "k": gains[1]}])
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
    if case["kind"] == "product":
        w = _matrix(case, seed)
        s["x"] = _rows(case, seed)
        if own:
            import paper_2504_04104_amd as sp
            s["w"] = sp.fp4_pack_matrix(w)
        else:
            s["w"] = _to_fp4(w)
        return s
    Ps, Ts = _sizes(case)
    s["ids"], s["first"], s["n"], M = list(range(len(Ps))), [0] * len(Ps), Ts, sum(Ts)
    if case["kind"] == "append":
        s["x"], s["gains"] = _qkv_rows(case, seed, M)
        dt = TYPES[case["cache"]]
        if own:
            import paper_2504_04104_amd as sp
            s["stage"], base = _stage(case, Ps, Ts, 0, dt, sp.SP_FLAG_FP4_KV if case["cache"] == "fp4" else 0, s["gains"] if case["norms"] else None)
            s["P"] = Ps[0]
            s["kv"] = None if case["cache"] == "fp4" else [s["stage"].kv_view()[0, :, :, b + P:b + P + T] for b, P, T in zip(base, Ps, Ts)]
        else:
            depth = [int(u.sum()) - 1 for p in _trees(case) for u in _ancestors(p)]
            at = np.repeat(Ps, Ts) + np.asarray(depth)
            s["pos"] = torch.from_numpy(at).to(DEV)
        return s
    s["q"] = _query_rows(case, seed, M)
    if own:
        import paper_2504_04104_amd as sp
        s["stage"], _ = _stage(case, Ps, Ts, case["page"], torch.bfloat16, sp.SP_FLAG_FP4_KV)
        for q, (P, T) in enumerate(zip(Ps, Ts)):
            k, v = _cache_rows(case, seed, q, P + T)
            s["stage"].kv_store(q, 0, 0, k, v)
        return s
    # one block for every request, as long as the longest
    _, kv, dh = HEADS[case["heads"]]
    R, n, S = len(Ps), max(Ts), max(P + T for P, T in zip(Ps, Ts))
    s["codes"] = torch.zeros(2, R, kv, S, dh // 2, dtype=torch.uint8, device=DEV)
    s["scales"] = torch.full((2, R, kv, S, dh // 32), 127, dtype=torch.uint8, device=DEV)
    seen, row = np.zeros((R, n, S), bool), np.zeros((R, n), np.int64)
    seen[:, :, 0] = True
    at = 0
    for q, (P, T, parents) in enumerate(zip(Ps, Ts, _trees(case))):
        c, b = _to_fp4(_cache_rows(case, seed, q, P + T).transpose(1, 2))
        s["codes"][:, q, :, :P + T], s["scales"][:, q, :, :P + T] = c, b
        seen[q, :T, :P], seen[q, :T, P:P + T] = True, _ancestors(parents)
        row[q, :T] = np.arange(at, at + T)
        at += T
    s["seen"], s["row"] = torch.from_numpy(seen).to(DEV), torch.from_numpy(row).to(DEV)
    s["real"] = torch.from_numpy(np.flatnonzero(np.arange(n)[None] < np.asarray(Ts)[:, None])).to(DEV)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if case["kind"] == "product":
        if own:
            import paper_2504_04104_amd as sp
            return sp.fp4_product(s["x"], s["w"], gated=case["gated"])
        y = s["x"].float() @ _from_fp4(*s["w"]).T
        if case["gated"]:
            gate, up = y[:, :case["n"]], y[:, case["n"]:]
            y = gate / (1 + torch.exp(-gate)) * up
        return y.to(torch.bfloat16)
    if case["kind"] == "append":
        if own:
            st = s["stage"]
            q = st.append(0, s["ids"], s["first"], s["n"], s["x"])
            return {"q": q, "kv": list(st.kv_load(0, 0, s["P"], s["n"][0])) if s["kv"] is None else s["kv"]}
        return _append_plain(s)
    if own:
        return s["stage"].attention(0, s["ids"], s["first"], s["n"], s["q"])
    nq, kv, dh = HEADS[case["heads"]]
    R, n, S = s["seen"].shape
    K, V = _from_fp4(s["codes"], s["scales"])
    q = s["q"].float()[s["row"]].reshape(R, n, kv, nq // kv, dh).permute(0, 2, 3, 1, 4).reshape(R * kv, nq // kv * n, dh)
    sc = torch.bmm(q, K.reshape(R * kv, S, dh).transpose(1, 2).contiguous()) / math.sqrt(dh)
    sc = sc.reshape(R, kv * (nq // kv), n, S).masked_fill(~s["seen"][:, None], -math.inf)
    p = torch.exp(sc - sc.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = torch.bmm(p.reshape(R * kv, nq // kv * n, S), V.reshape(R * kv, S, dh))
    o = o.reshape(R, nq, n, dh).transpose(1, 2).reshape(R * n, nq * dh)[s["real"]]
    return o.to(torch.bfloat16)


def _append_plain(s):
    case, x = s["case"], s["x"]
    nq, kv, dh = HEADS[case["heads"]]
    M, dt = x.shape[0], x.dtype
    x = x.float().reshape(M, nq + 2 * kv, dh)
    qk, v = x[:, :nq + kv], x[:, nq + kv:]
    if case["norms"]:
        g = s["gains"].float()
        gain = torch.cat([g[:1].expand(nq, dh), g[1:].expand(kv, dh)])
        qk = qk * torch.rsqrt(qk.square().mean(-1, keepdim=True) + EPS) * gain
    # the angles of far positions lose what matters in 32 bits
    freq = THETA ** (-torch.arange(dh // 2, device=DEV, dtype=torch.float64) * 2 / dh)
    ang = s["pos"].double()[:, None, None] * freq
    cos, sin = torch.cos(ang).float(), torch.sin(ang).float()
    a, b = qk[..., :dh // 2], qk[..., dh // 2:]
    qk = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    q, k = qk[:, :nq].reshape(M, nq * dh).to(dt), qk[:, nq:]
    if case["cache"] == "fp4":
        return {"q": q, "kv": [_from_fp4(*_to_fp4(k)).to(dt), _from_fp4(*_to_fp4(v)).to(dt)]}
    rows = torch.stack([k, v]).transpose(1, 2).to(dt)
    return {"q": q, "kv": list(rows.split(s["n"], 2))}


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "product":
        m, n, k = case["rows"], case["n"], case["k"]
        cols = n * (2 if case["gated"] else 1)
        return {"bytes": cols * k * 17 // 32 + 2 * m * (k + n), "flops": 2 * m * cols * k}
    nq, kv, dh = HEADS[case["heads"]]
    Ps, Ts = _sizes(case)
    M = sum(Ts)
    if case["kind"] == "append":
        e = 4 if case["cache"] == "f32" else 2
        row = 2 * kv * (dh * 17 // 32 if case["cache"] == "fp4" else dh * e)
        return {"bytes": M * ((nq + 2 * kv) * dh * e + nq * dh * e + row), "flops": 10 * M * (nq + kv) * dh}
    spans = [P + T for P, T in zip(Ps, Ts)]
    return {"bytes": 2 * kv * (dh * 17 // 32) * sum(spans) + 4 * M * nq * dh, "flops": 4 * nq * dh * sum(s * t for s, t in zip(spans, Ts))}


# ---- the same pass in 64 bits -------------------------------------------------------------------------------------
def _held(x):
    """The values that 4 bits hold for x, in 64 bits: the grid point of the group's power of two nearest to each value."""
    x = x.double().unflatten(-1, (-1, 32))
    mant, expo = torch.frexp(x.abs().amax(-1, keepdim=True))           # max = mant * 2^expo, mant in [0.5, 1)
    e = torch.where(mant <= 0.75, expo - 3, expo - 2).clamp(-100, 125)
    e = torch.where(mant == 0, torch.full_like(e, -100), e)
    a = torch.ldexp(x.abs(), -e)
    # spacing of the grid: 0.5 below 2, 1 from 2 to 4, 2 from there; torch.round goes to even, as the codes do
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    return torch.ldexp(torch.copysign(a, x), e).flatten(-2)


def exact(case, seed):
    if case["kind"] == "product":
        x, out = _rows(case, seed).double(), []
        w = _matrix(case, seed)
        for part in w.split(8192):
            out.append(x @ _held(part).T)
        y = torch.cat(out, 1)
        if case["gated"]:
            y = torch.sigmoid(y[:, :case["n"]]) * y[:, :case["n"]] * y[:, case["n"]:]
        return y
    nq, kv, dh = HEADS[case["heads"]]
    Ps, Ts = _sizes(case)
    M, trees = sum(Ts), _trees(case)
    if case["kind"] == "attention":
        q, out, at = _query_rows(case, seed, M).double().reshape(M, nq, dh), [], 0
        for r, (P, T, parents) in enumerate(zip(Ps, Ts, trees)):
            k, v = _held(_cache_rows(case, seed, r, P + T))
            seen = torch.ones(T, P + T, dtype=torch.bool, device=DEV)
            seen[:, P:] = torch.from_numpy(_ancestors(parents)).to(DEV)
            heads = []
            for h in range(nq):
                c = h // (nq // kv)
                sc = (q[at:at + T, h] @ k[:, c].T) / math.sqrt(dh)
                heads.append(torch.softmax(sc.masked_fill(~seen, -math.inf), -1) @ v[:, c])
            out.append(torch.stack(heads, 1).reshape(T, nq * dh))
            at += T
        return torch.cat(out)
    x, gains = _qkv_rows(case, seed, M)
    x, gains = x.double().reshape(M, nq + 2 * kv, dh), gains.double()
    parts = [x[:, :nq], x[:, nq:nq + kv], x[:, nq + kv:]]
    if case["norms"]:
        for i in range(2):
            parts[i] = parts[i] / torch.sqrt(parts[i].pow(2).mean(-1, keepdim=True) + EPS) * gains[i]
    pos = torch.tensor([P + int(u.sum()) - 1 for P, p in zip(Ps, trees) for u in _ancestors(p)], device=DEV, dtype=torch.float64)
    turn = torch.polar(torch.ones(M, 1, dh // 2, device=DEV, dtype=torch.float64),
                       (pos[:, None] / THETA ** (torch.arange(0, dh, 2, device=DEV, dtype=torch.float64) / dh))[:, None])
    for i in range(2):
        z = torch.complex(parts[i][..., :dh // 2].contiguous(), parts[i][..., dh // 2:].contiguous()) * turn
        parts[i] = torch.cat([z.real, z.imag], -1)
    q = parts[0].reshape(M, nq * dh)
    if case["cache"] == "fp4":
        return {"q": q, "kv": [_held(parts[1]), _held(parts[2])]}
    return {"q": q, "kv": list(torch.stack(parts[1:]).transpose(1, 2).split(Ts, 2))}
