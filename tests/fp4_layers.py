"""Layers in float64 on the device, with the roundings that a stage makes between its products."""
import torch

import paper_2504_04104_amd as sp
from fp4_reference import ancestors


def bf16(t):
    return t.to(torch.bfloat16).double()


def matrix(w):
    """The values of a matrix, held in 4 bits or not, in float64."""
    return (sp.fp4_unpack_matrix(w) if isinstance(w, sp.Fp4Matrix) else w).double()


def tree(P, parents):
    """(positions, who sees which of the P + n slots) of a tree's nodes behind P slots."""
    up = torch.from_numpy(ancestors(parents)).cuda()
    return P + up.sum(1).double() - 1, torch.cat([torch.ones(len(parents), P, dtype=torch.bool, device="cuda"), up], 1)


def rotated(t, pos, theta, r):
    dh = t.shape[-1]
    ang = pos[:, None, None] * theta ** (-2.0 * torch.arange(dh // 2, device="cuda", dtype=torch.float64) / dh)
    a, b = t[..., :dh // 2], t[..., dh // 2:]
    return r(torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], -1))


def normed(v, gain, eps):
    return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + eps) * gain.double()


def attended(q, k, v, seen):
    n, nq, dh = q.shape
    out = torch.empty_like(q)
    for h in range(nq):
        c = h * k.shape[1] // nq
        s = (q[:, h] @ k[:, c].T.contiguous()) / dh ** 0.5
        out[:, h] = torch.softmax(s.masked_fill(~seen, float("-inf")), -1) @ v[:, c]
    return out


def layer(w, x, pos, seen, cache, sh, r=bf16, gains=None):
    """Rows x of one request through a layer.  cache: of the nodes' new K and V, what the attention reads.  r: what the rows between
    the products, the queries and the new K and V are rounded by.  gains: of the head norms."""
    nq, kv, dh, n = sh.n_q_heads, sh.n_kv_heads, sh.d_head, len(x)
    qkv = (r(normed(x, w["norm1"], sh.rms_eps)) @ matrix(w["wqkv"]).T).view(n, nq + 2 * kv, dh)
    q, k, v = qkv[:, :nq], qkv[:, nq:nq + kv], qkv[:, nq + kv:]
    if gains is not None:
        q, k = normed(q, gains["q"], sh.rms_eps), normed(k, gains["k"], sh.rms_eps)
    k_all, v_all = cache(rotated(k, pos, sh.rope_theta, r), r(v))
    att = r(attended(rotated(q, pos, sh.rope_theta, r), k_all, v_all, seen))
    h = x + att.reshape(n, nq * dh) @ matrix(w["wo"]).T
    gu = r(normed(h, w["norm2"], sh.rms_eps)) @ matrix(w["wgu"]).T
    return h + r(torch.nn.functional.silu(gu[:, :sh.d_ff]) * gu[:, sh.d_ff:]) @ matrix(w["wd"]).T
