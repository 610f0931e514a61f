"""Rotary positions, latent append and latent attention in float64, written from their formulas; stages to hold against them."""
import math

import numpy as np
import torch

import paper_2504_04104_amd as sp
from fp4_reference import ancestors, random_tree


def frequencies(dims, theta, scaling=None):
    out = []
    for t in range(dims // 2):
        f = theta ** (-2.0 * t / dims)
        if scaling is None:
            pass
        elif scaling[0] == "linear":
            f /= scaling[1]
        elif scaling[0] == "bands":
            _, factor, original, first, second = scaling
            turns = original * f / (2 * math.pi)
            if turns <= first:
                f /= factor
            elif turns < second:
                s = (turns - first) / (second - first)
                f = (1 - s) * f / factor + s * f
        else:
            _, factor, original, first, second = scaling
            c = [dims * math.log(original / (2 * math.pi * n)) / (2 * math.log(theta)) for n in (first, second)]
            lo, hi = max(math.floor(c[0]), 0), min(math.ceil(c[1]), dims - 1)
            away = min(max((t - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f = f * (1 - away) + f / factor * away
        out.append(f)
    return np.array(out)


def turn(x, pos, freq, layout, gain=1.0, inverse=False):
    """x [rows, heads, d] (float64 numpy) with its first 2 * len(freq) columns turned at pos [rows]."""
    ang = np.asarray(pos, np.float64)[:, None, None] * np.asarray(freq)
    c, s = gain * np.cos(ang), gain * np.sin(ang) * (-1 if inverse else 1)
    y, n = x.copy(), len(freq)
    at = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = x[..., at[0]], x[..., at[1]]
    y[..., at[0]], y[..., at[1]] = a * c - b * s, b * c + a * s
    return y


def pair_lengths(x, n, layout):
    """Length of the pair that every rotated column belongs to, zero in the others."""
    r = np.zeros_like(x)
    at = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    r[..., at[0]] = r[..., at[1]] = np.hypot(x[..., at[0]], x[..., at[1]])
    return r


def attend(q, rows, c, seen, scale):
    """q [n, heads, D], rows [slots, D], seen [n, slots], all on the GPU -> (out [n, heads, c], sum of weight * |latent|, sum of
    |q row| * scale at its largest): the result in float64, the last two for error bounds."""
    n, heads, D = q.shape
    q, rows = q.double(), rows.double()
    s = (q.reshape(n * heads, D) @ rows.T).reshape(n, heads, -1) * scale
    p = torch.softmax(s.masked_fill(~seen[:, None], -math.inf), -1)
    out, mag = (p.reshape(n * heads, -1) @ t for t in (rows[:, :c], rows[:, :c].abs()))
    big = ((q.abs().reshape(n * heads, D) @ rows.abs().T) * scale).amax(-1)
    return out.reshape(n, heads, c), mag.reshape(n, heads, c), big.reshape(n, heads, 1)


def make(heads, c, r, trees, *, page=0, layers=1, seed=0, flags=0, rows=None, extra=1, scale=None, spread=1.0, layer=0, **kw):
    """A latent stage with the requests of trees [(context, nodes)], their caches full of random rows; pages out of order."""
    unit = page or 32
    room = [-(-(P + T) // unit) * unit for P, T in trees]
    st = sp.LatentStage(layers, heads, c, r, scale=scale or (c // 4 + r) ** -0.5, kv_slots=sum(room) + unit, max_requests=len(trees) + extra,
                        max_batch_nodes=rows or max(64, sum(T for _, T in trees)), page_slots=page, flags=flags, **kw)
    if page:
        st.request_init(len(trees), 0, room[0], room[0])
        st.request_release(len(trees))
    st.trees, st.parents, st.held, st.base = trees, [], [], []
    base = 0 if page else 3
    g = torch.Generator().manual_seed(seed)
    for i, (P, T) in enumerate(trees):
        st.request_init(i, base, room[i], P)
        st.base.append(base)
        base += 0 if page else room[i]
        st.parents.append(random_tree(T, seed + i))
        st.tree_insert(i, st.parents[-1])
        x = (spread * torch.randn(P + T, c + r, generator=g)).to(torch.bfloat16).cuda()
        st.kv_store(i, layer, 0, x)
        st.held.append(x)
    return st


def seen_by(st, i, first=0):
    P, T = st.trees[i]
    seen = torch.ones(T - first, P + T, dtype=torch.bool, device="cuda")
    seen[:, P:] = torch.from_numpy(ancestors(st.parents[i])[first:]).cuda()
    return seen


def positions(st):
    return np.concatenate([P + ancestors(p).sum(1) - 1 for (P, _), p in zip(st.trees, st.parents)])
