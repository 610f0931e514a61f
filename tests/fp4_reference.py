"""4-bit storage, head norms, rotation and tree attention in float64, written from their formulas."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def group_exponent(x):
    """e of every group of 32 along the last axis: the smallest in [-100, 125] with max |x| <= 6 * 2^e."""
    with np.errstate(invalid="ignore"):
        amax = np.nanmax(np.where(np.isnan(x), 0.0, np.abs(x)).reshape(*x.shape[:-1], -1, 32), axis=-1)
    e = np.full(amax.shape, -100)
    for k in range(-100, 125):                      # (a plain search, one exponent after the other)
        e = np.where(amax > 6.0 * 2.0 ** k, k + 1, e)
    return e


def held(x, e=None):
    """The values that 4 bits hold for x (float64, last axis in groups of 32)."""
    x = np.asarray(x, np.float64)
    if e is None:
        e = group_exponent(x)
    g = np.where(np.isnan(x), 0.0, x).reshape(*x.shape[:-1], -1, 32)
    a = np.minimum(np.abs(g) / 2.0 ** e[..., None], 6.0)
    hi = np.searchsorted(GRID, a.reshape(-1)).reshape(a.shape)       # first grid point >= a
    lo = np.maximum(hi - 1, 0)
    up, down = GRID[hi] - a, a - GRID[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return (np.copysign(GRID[code], g) * 2.0 ** e[..., None]).reshape(x.shape)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def head_norm(x, gain, eps):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain


def rotate(x, pos, theta):
    """x [rows, heads, d], pos [rows]."""
    d = x.shape[-1]
    ang = np.asarray(pos, np.float64)[:, None, None] * theta ** (-2.0 * np.arange(d // 2) / d)
    a, b = x[..., :d // 2], x[..., d // 2:]
    return np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], -1)


def ancestors(parents):
    m = np.zeros((len(parents), len(parents)), bool)
    for i, p in enumerate(parents):
        if p >= 0:
            m[i] = m[p]
        m[i, i] = True
    return m


def attend(q, k, v, seen):
    """q [rows, n_q, d], k / v [slots, n_kv, d], seen [rows, slots] -> (out, sum of weight * |v|, sum of |q k| / sqrt(d) at
    its largest), the last two for error bounds."""
    g, d = q.shape[1] // k.shape[1], q.shape[-1]
    out, mag, big = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[:2])
    for h in range(q.shape[1]):
        s = np.where(seen, q[:, h] @ k[:, h // g].T / np.sqrt(d), -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        out[:, h], mag[:, h] = p @ v[:, h // g], p @ np.abs(v[:, h // g])
        big[:, h] = (np.abs(q[:, h]) @ np.abs(k[:, h // g]).T / np.sqrt(d)).max(-1)
    return out, mag, big


def random_tree(n, seed, wide=4):
    r, parents = np.random.default_rng(seed), []
    for i in range(n):
        parents.append(int(r.integers(max(-1, i - 3 * wide), i)) if i else -1)
    return parents


def stage(sp, shape, *, slots, flags=0, requests=1, rows=64, page=0, norms=False, seed=0, layers=None):
    """A stage with weights of the right shapes (random where `layers` asks for them: float64-friendly bf16 / float32)."""
    dt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(seed)
    nqkv = (shape.n_q_heads + 2 * shape.n_kv_heads) * shape.d_head
    size = {"wqkv": (nqkv, shape.d_model), "wo": (shape.d_model, shape.n_q_heads * shape.d_head), "wgu": (2 * shape.d_ff, shape.d_model),
            "wd": (shape.d_model, shape.d_ff)}
    if layers is None:
        layers = []
        for _ in range(shape.n_layers):
            w = {n: (0.05 * torch.randn(*s, generator=g)).to("cuda", dt) for n, s in size.items()}
            for n in ("norm1", "norm2"):
                w[n] = (1 + 0.05 * torch.randn(shape.d_model, generator=g)).to("cuda", dt)
            layers.append(w)
    gains = [{n: (1 + 0.2 * torch.randn(shape.d_head, generator=g)).to("cuda", dt) for n in "qk"} for _ in range(shape.n_layers)] if norms else None
    if page:
        flags |= sp.SP_FLAG_PAGED_KV
    packed = sp.fp4_pack_weights(shape, layers) if flags & sp.SP_FLAG_FP4_WEIGHTS else layers
    st = sp.Stage(shape, packed, kv_slots=slots, max_requests=requests, max_batch_nodes=rows, flags=flags, page_slots=page, head_norms=gains)
    st.plain_layers, st.gains = layers, gains
    return st
