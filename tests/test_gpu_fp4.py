"""4-bit storage and the operators on it, against float64: conversion, products, cache rows, append, attention, the whole stage.

Tolerances count roundings: u = 2^-8 is half a step of bf16 relative to the value, 2^-24 of float32, and a float32 sum of n
terms in any order is off by at most n * 2^-24 times the sum of their magnitudes."""
import numpy as np
import pytest
import torch

import workloads as wl
import paper_2504_04104_amd as sp
from fp4_reference import ancestors, attend, f64, group_exponent, head_norm, held, random_tree, rotate, stage
from gpu_harness import use_own_stream

pytestmark = pytest.mark.gpu
U, F = 2.0 ** -8, 2.0 ** -24


def rnd(seed, *size, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*size, generator=g)).to(torch.bfloat16).cuda()


def shape(nq=8, nkv=2, dh=128, layers=1, d=256, ff=256, dtype="bf16"):
    return wl.ModelShape(layers, d, nq, nkv, dh, ff, 1e-5, 500000.0, dtype)


# ---- conversion ------------------------------------------------------------------------------------
def test_every_kind_of_value_is_held_as_its_definition_says():
    rows = []
    r = np.random.default_rng(1)
    for k in (-140, -120, -101, -100, -99, -30, -1, 0, 1, 17, 120, 124, 125, 126):
        rows.append(r.uniform(-8, 8, 256) * 2.0 ** k)                          # scales inside and beyond their range
    rows.append(np.tile(np.arange(-32, 32) / 4.0, 4))                          # all ties: quarters up to 8
    rows.append(np.tile(np.concatenate([np.arange(-16, 16) / 4.0, np.full(32, 6.0)]), 4))
    zero = np.zeros(256)
    zero[64] = -0.0
    rows.append(zero)
    odd = r.standard_normal(256)
    odd[[3, 40, 41]] = [np.inf, np.nan, -np.nan]
    odd[96:128] = np.nan
    odd[200] = -np.inf
    rows.append(odd)
    x = np.array(rows)
    x = np.concatenate([x, r.standard_normal(((-len(x)) % 16, 256))])
    t = torch.from_numpy(x).to(torch.bfloat16).cuda()
    want = held(f64(t))
    got = f64(sp.fp4_unpack_matrix(sp.fp4_pack_matrix(t)))
    assert np.isfinite(got).all()
    assert np.array_equal(got, want)


@pytest.mark.parametrize("n,k", [(16, 32), (16, 256), (48, 288), (32, 8192 + 32), (4096, 96)])
def test_matrices_of_any_shape_come_back_as_held(n, k):
    w = rnd(n + k, n, k, scale=0.02)
    assert np.array_equal(f64(sp.fp4_unpack_matrix(sp.fp4_pack_matrix(w))), held(f64(w)))


# ---- products ----------------------------------------------------------------------------------------
def product_case(m, n, k, gated, seed=0):
    x, w = rnd(seed + 1, m, k), rnd(seed + 2, n * (2 if gated else 1), k, scale=0.05)
    p = sp.fp4_pack_matrix(w)
    y = f64(sp.fp4_product(x, p, gated=gated))
    xr, wr = f64(x), held(f64(w))
    ref, mag = xr @ wr.T, k * F * (np.abs(xr) @ np.abs(wr).T)
    if gated:
        a, b, ea, eb = ref[:, :n], ref[:, n:], mag[:, :n], mag[:, n:]
        s = a / (1 + np.exp(-a))
        # silu changes by at most 1.1 per unit; its exponential and quotient are good to a few float32 steps
        ref, mag = s * b, 1.1 * ea * (np.abs(b) + eb) + np.abs(s) * eb + 2.0 ** -20 * np.abs(s * b)
    assert y.shape == ref.shape
    assert (np.abs(y - ref) <= U * np.abs(ref) + 1.01 * mag + 1e-30).all()


@pytest.mark.parametrize("m", [1, 2, 8, 9, 16, 17, 31, 33, 48, 64, 65, 100, 128, 129, 257])
@pytest.mark.parametrize("gated", [False, True])
def test_products_of_any_number_of_rows(m, gated):
    product_case(m, 272, 544, gated, seed=m)


@pytest.mark.parametrize("m,n,k,gated", [(1, 16, 32, False), (5, 16, 32, True), (1, 4096, 4096, False), (7, 1040, 14336, False),
                                         (64, 4096, 1024, True), (20, 28672, 288, False), (3, 64, 131072, False), (130, 4112, 2048, False),
                                         (200, 2064, 4096, True), (33, 8192, 512, True), (70, 16, 8192, False)])
def test_products_of_many_shapes(m, n, k, gated):
    product_case(m, n, k, gated)


@pytest.mark.parametrize("m,n,k,gated", [(100, 14336, 544, True), (160, 14416, 288, True), (200, 14320, 800, True), (12, 10256, 4096, False),
                                         (5, 10256, 1056, False), (16, 1040, 14336, True), (300, 4112, 14336, False), (13, 2064, 14304, False),
                                         (65, 10256, 8288, False), (16, 14416, 1312, True), (2, 6160, 4096, False), (3, 6160, 4096, True)])
def test_products_of_every_cut(m, n, k, gated):
    """Tiles of one to seven, kernels for few and many rows, whole and in slices, columns that end inside a unit or a chunk."""
    product_case(m, n, k, gated)


@pytest.mark.parametrize("m,n,k,gated", [(1 << 17, 16, 32, False), (40000, 48, 96, True), (1 << 16, 32, 288, False)])
def test_products_of_very_many_rows(m, n, k, gated):
    product_case(m, n, k, gated)


@pytest.mark.parametrize("m,n", [(1, 4096), (12, 1024), (30, 4096), (64, 4096), (100, 28672), (150, 28672), (200, 28672)])
def test_columns_past_the_end_count_as_nothing(m, n):
    """Storage goes on to a multiple of 256 columns.  Whatever was in shared memory before: here NaN, out of a product before."""
    x, w = rnd(m, m, 1056), rnd(n, n, 1056, scale=0.05)
    nan = torch.full((m, 1056), float("nan"), dtype=torch.bfloat16, device="cuda")
    full = sp.fp4_pack_matrix(w)
    for k in (32, 160, 288, 1056):
        xk, p = x[:, :k].contiguous(), sp.fp4_pack_matrix(w[:, :k].contiguous())
        first = sp.fp4_product(xk, p)
        assert torch.isfinite(first).all()
        assert torch.isnan(sp.fp4_product(nan, full)).all()
        assert torch.equal(sp.fp4_product(xk, p), first)


def test_a_gated_product_of_a_matrix_past_2_gb():
    """Gate and up rows more than 2 GB apart: one strip of both is not zero."""
    n, k = 65536, 131072
    units = k // 256
    w = sp.Fp4Matrix(torch.zeros(sp.load_library().sp_fp4_matrix_bytes(2 * n, k), dtype=torch.uint8, device="cuda"), 2 * n, k)
    gate, up, x = rnd(1, 16, k, scale=0.02), rnd(2, 16, k, scale=0.02), rnd(3, 3, k)
    at = [s * units * 2176 for s in (n // 16 - 1, 2 * n // 16 - 1)]
    for part, o in zip((gate, up), at):
        piece = sp.fp4_pack_matrix(part).data
        w.data[o:o + piece.numel()] = piece
    y = f64(sp.fp4_product(x, w, gated=True))
    assert not y[:, :n - 16].any()
    small = sp.fp4_pack_matrix(torch.cat([gate, up]))
    assert np.allclose(y[:, n - 16:], f64(sp.fp4_product(x, small, gated=True)), rtol=2.0 ** -7, atol=2.0 ** -7)


def test_a_row_that_is_not_finite_stays_alone():
    """Columns are padded to 256 in storage; what lies behind a row of x is the next row, here NaN and infinity."""
    for m in (3, 20, 70):
        x, w = rnd(1, m, 288), rnd(2, 64, 288)
        p = sp.fp4_pack_matrix(w)
        clean = sp.fp4_product(x, p)
        bad = x.clone()
        bad[1] = float("nan")
        bad[m - 1, 0] = float("inf")
        y = sp.fp4_product(bad, p)
        keep = [i for i in range(m) if i not in (1, m - 1)]
        assert torch.equal(y[keep], clean[keep])
        assert torch.isnan(y[1]).all() and not torch.isfinite(y[m - 1]).any()


def test_product_writes_its_rows_only_and_takes_no_row():
    for m, gated in ((5, False), (37, True), (130, False)):
        x, w = rnd(1, m, 256), rnd(2, 128, 256)
        p = sp.fp4_pack_matrix(w)
        n = 64 if gated else 128
        room = torch.full((m + 20, n), 7.0, dtype=torch.bfloat16, device="cuda")
        sp.fp4_product(x, p, gated=gated, out=room[:m])
        assert (room[m:] == 7).all()
        assert torch.equal(room[:m], sp.fp4_product(x, p, gated=gated))
    assert sp.fp4_product(x[:0].contiguous(), p).shape == (0, 128)


# ---- cache rows -----------------------------------------------------------------------------------------
CACHES = {"fp4_128": (shape(), sp.SP_FLAG_FP4_KV), "fp4_64": (shape(4, 4, 64), sp.SP_FLAG_FP4_KV), "bf16_128": (shape(), 0),
          "bf16_64": (shape(4, 2, 64), 0), "f32_64": (shape(4, 4, 64, dtype="f32"), 0)}


@pytest.mark.parametrize("page", [0, 32])
@pytest.mark.parametrize("cache", sorted(CACHES))
def test_stored_rows_come_back_as_the_cache_holds_them(cache, page):
    sh, flags = CACHES[cache]
    st = stage(sp, sh, slots=512, flags=flags, requests=2, page=page)
    for q, (base, P) in enumerate(((0, 71), (128, 90))):
        st.request_init(q, 0 if page else base, 128, P)
    ref = []
    for q, P in ((0, 71), (1, 90)):
        k, v = (rnd(10 * q + i, P, sh.n_kv_heads, sh.d_head).to(st.tdtype) for i in range(2))
        st.kv_store(q, 0, 0, k[:40], v[:40])
        st.kv_store(q, 0, 40, k[40:], v[40:])
        ref.append((k, v))
    for q, P in ((0, 71), (1, 90)):
        for first, n in ((0, P), (P - 1, 1), (33, 17), (5, 0)):
            for got, want in zip(st.kv_load(q, 0, first, n), ref[q]):
                w = f64(want)[first:first + n]
                assert np.array_equal(f64(got), held(w) if flags and n else w)


@pytest.mark.parametrize("mode", [sp.SP_ACCEPT, sp.SP_DROP])
@pytest.mark.parametrize("page", [0, 32])
@pytest.mark.parametrize("dh", [64, 128])
def test_compaction_moves_codes_and_scales_together(dh, page, mode):
    sh = shape(4, 2, dh, layers=2)
    st = stage(sp, sh, slots=1024, flags=sp.SP_FLAG_FP4_KV, requests=2, rows=256, page=page)
    P, T = 45, 200
    st.request_init(0, 0 if page else 7, 300, P)
    st.request_init(1, 0 if page else 307, 300, 20)
    parents = random_tree(T, 3)
    st.tree_insert(0, parents)
    zero = st.kv_load(0, 1, P, T)
    assert not f64(zero[0]).any() and not f64(zero[1]).any()          # inserted rows hold zeros until they are written
    for l in range(2):
        for q, n in ((0, P + T), (1, 20)):
            k, v = (rnd(7 + l + 10 * i + q, n, 2, dh) * torch.exp2(torch.arange(n, device="cuda") % 23 - 11.0)[:, None, None].to(torch.bfloat16) for i in range(2))
            st.kv_store(q, l, 0, k, v)
    before = [[f64(t) for t in st.kv_load(0, l, 0, P + T)] for l in range(2)]
    other = [[f64(t) for t in st.kv_load(1, l, 0, 20)] for l in range(2)]
    node = 60
    anc = ancestors(parents)
    if mode == sp.SP_ACCEPT:
        # (the committed path has to count as forwarded: an append to the last layer does that)
        st.append(1, [0], [0], [T], torch.zeros(T, (4 + 4) * dh, dtype=torch.bfloat16, device="cuda"))
        before[1] = [f64(t) for t in st.kv_load(0, 1, 0, P + T)]
        keep = [j for j in range(T) if anc[node, j] or anc[j, node]]
    else:
        keep = [j for j in range(T) if not anc[j, node]]
    st.tree_prune(0, mode, node)
    st.kv_compact(0)
    p, t, _ = st.request_info(0)
    assert p + t == P + len(keep)
    src = list(range(P)) + [P + j for j in keep]
    for l in range(2):
        for i, got in enumerate(st.kv_load(0, l, 0, p + t)):
            assert np.array_equal(f64(got), before[l][i][src])
        for i, got in enumerate(st.kv_load(1, l, 0, 20)):
            assert np.array_equal(f64(got), other[l][i])


# ---- append -----------------------------------------------------------------------------------------------
def check_held(got, x, off):
    """got is what 4 bits hold of some value within `off` of x: codes and scales may differ where a border lies in between."""
    lo, hi = held(x - off), held(x + off)
    e = group_exponent(x)
    near = np.abs(np.log2(np.maximum(np.abs(x).reshape(*x.shape[:-1], -1, 32).max(-1), 1e-300) / 6.0) % 1.0)
    near = np.minimum(near, 1 - near) < 1e-4                          # the group's scale itself is on a border
    ok = (got >= np.minimum(lo, hi)) & (got <= np.maximum(lo, hi))
    ok |= np.repeat(near, 32, -1).reshape(x.shape) & ((got == held(x, e + 1)) | (got == held(x, e - 1)))
    assert ok.all(), np.argwhere(~ok)[:4]


@pytest.mark.parametrize("norms", [False, True])
@pytest.mark.parametrize("cache", sorted(CACHES))
@pytest.mark.parametrize("trees", [[(1, 1)], [(512, 1)], [(40, 37)], [(100000, 256)], [(3, 5), (700, 64), (31, 1), (32, 33)]])
def test_append_norms_rotates_and_writes_the_cache(cache, norms, trees):
    sh, flags = CACHES[cache]
    page = 32 if len(trees) > 1 else 0
    room = [-(-(P + T) // 32) * 32 for P, T in trees]
    st = stage(sp, sh, slots=sum(room), flags=flags, requests=len(trees), rows=1024, page=page, norms=norms)
    base, pos, par = 0, [], []
    for q, (P, T) in enumerate(trees):
        st.request_init(q, 0 if page else base, room[q], P)
        base += room[q]
        par.append(random_tree(T, q))
        st.tree_insert(q, par[-1])
        pos += [P + int(a.sum()) - 1 for a in ancestors(par[-1])]
    ids, n = list(range(len(trees))), [T for _, T in trees]
    M, nq, kv, dh = sum(n), sh.n_q_heads, sh.n_kv_heads, sh.d_head
    x = (1.5 * torch.randn(M, (nq + 2 * kv) * dh, generator=torch.Generator().manual_seed(M))).to("cuda", st.tdtype)
    got = f64(st.append(0, ids, [0] * len(ids), n, x)).reshape(M, nq, dh)
    rows = f64(x).reshape(M, nq + 2 * kv, dh)
    q, k, v = rows[:, :nq], rows[:, nq:nq + kv], rows[:, nq + kv:]
    if norms:
        q, k = head_norm(q, f64(st.gains[0]["q"]), sh.rms_eps), head_norm(k, f64(st.gains[0]["k"]), sh.rms_eps)
    q, k = rotate(q, pos, sh.rope_theta), rotate(k, pos, sh.rope_theta)
    # float32 on the way: norm (d_head terms and a reciprocal root), gain, sine and cosine, two products and a sum, relative to
    # the pair's length; 32 steps and the sum's d_head / 2 are more than all of them
    half = dh // 2
    def off(y):
        r = np.hypot(y[..., :half], y[..., half:])
        return (32 + half) * F * np.concatenate([r, r], -1)
    u = U if st.tdtype == torch.bfloat16 else F
    assert (np.abs(got - q) <= u * np.abs(q) + off(q)).all()
    at = 0
    for i, (P, T) in enumerate(trees):
        kk, vv = (f64(t) for t in st.kv_load(i, 0, P, T))
        if flags:
            check_held(kk, k[at:at + T], off(k[at:at + T]))
            assert np.array_equal(vv, held(v[at:at + T]))
        else:
            assert (np.abs(kk - k[at:at + T]) <= u * np.abs(k[at:at + T]) + off(k[at:at + T])).all()
            assert np.array_equal(vv, v[at:at + T])
        at += T


def test_append_of_some_nodes_leaves_the_others_and_counts_them_as_forwarded_in_the_last_layer():
    sh = shape(layers=2)
    st = stage(sp, sh, slots=256, flags=sp.SP_FLAG_FP4_KV)
    st.request_init(0, 0, 200, 50)
    st.tree_insert(0, [-1, 0, 1, -1])
    x = rnd(1, 2, 12 * 128)
    for l in range(2):
        with pytest.raises(sp.SpError) as err:
            st.append(l, [0], [2], [2], x)                            # its parent is not there yet
        assert err.value.status == -6
    st.append(0, [0], [0], [2], x)
    assert st.request_info(0)[2] == 0
    st.append(1, [0], [0], [2], x)
    assert st.request_info(0)[2] == 2
    held_k = f64(st.kv_load(0, 1, 50, 4)[0])
    assert held_k[:2].any() and not held_k[2:].any()
    st.append(1, [0], [2], [2], x)
    assert st.request_info(0)[2] == 4
    assert np.array_equal(f64(st.kv_load(0, 1, 50, 2)[0]), held_k[:2])


# ---- attention -------------------------------------------------------------------------------------------------
def attention_case(sh, trees, *, flags=sp.SP_FLAG_FP4_KV, page=0, layer=0, first=None, spread=1.0, seed=0):
    """trees: [(context, nodes)]; first: per request the first node whose row is computed."""
    unit = page or 32
    room = [-(-(P + T) // unit) * unit for P, T in trees]
    st = stage(sp, sh, slots=sum(room) + unit, flags=flags, requests=len(trees) + 1, rows=max(64, sum(T for _, T in trees)), page=page)
    if page:                                        # pages out of order
        st.request_init(len(trees), 0, room[0], room[0])
        st.request_release(len(trees))
    first = first or [0] * len(trees)
    base, ref, qs, n = 3, [], [], []
    if page:
        base = 0
    for i, (P, T) in enumerate(trees):
        st.request_init(i, 0 if page else base, room[i], P)
        base += room[i]
        par = random_tree(T, seed + i)
        st.tree_insert(i, par)
        k, v = (rnd(seed + 100 * i + j, P + T, sh.n_kv_heads, sh.d_head, scale=spread if j == 0 else 1.0).to(st.tdtype) for j in range(2))
        st.kv_store(i, layer, 0, k, v)
        rows = T - first[i]
        q = rnd(seed + 100 * i + 7, rows, sh.n_q_heads * sh.d_head).to(st.tdtype)
        seen = np.ones((rows, P + T), bool)
        seen[:, P:] = ancestors(par)[first[i]:]
        hk, hv = (held(f64(t)) if flags & sp.SP_FLAG_FP4_KV else f64(t) for t in (k, v))
        ref.append(attend(f64(q).reshape(rows, sh.n_q_heads, sh.d_head), hk, hv, seen))
        qs.append(q)
        n.append(rows)
    ids = list(range(len(trees)))
    # nodes in front of the call's count as forwarded after an append to the last layer; here their rows are stored already
    for i in ids:
        if first[i]:
            keep = st.kv_load(i, sh.n_layers - 1, trees[i][0], first[i])
            st.append(sh.n_layers - 1, [i], [0], [first[i]], torch.zeros(first[i], (sh.n_q_heads + 2 * sh.n_kv_heads) * sh.d_head, dtype=st.tdtype, device="cuda"))
            st.kv_store(i, sh.n_layers - 1, trees[i][0], *keep)
    q = torch.cat(qs)
    out = st.attention(layer, ids, first, n, q)
    got, at = f64(out), 0
    u = U if st.tdtype == torch.bfloat16 else F
    for i, rows in enumerate(n):
        y, mag, big = ref[i]
        g = got[at:at + rows].reshape(y.shape)
        # the result's rounding; every weight rounded to the storage type, against their exact sum; scores off by d_head float32
        # steps and the exponential, the sums and the chunks' rescaling by as many again
        off = u * np.abs(y) + (1.01 * u + (8 + 2 * sh.d_head) * F * (1 + big[..., None]) + 64 * F) * mag
        assert np.isfinite(g).all()
        assert (np.abs(g - y) <= off).all(), (i, np.max(np.abs(g - y) / off))
        at += rows
    return st, ids, first, n, q, out


HEADS = [(8, 2, 128), (32, 8, 128), (64, 8, 128), (4, 4, 128), (3, 1, 128), (16, 4, 64), (4, 4, 64), (14, 2, 64)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("P,T", [(1, 1), (1, 40), (31, 1), (32, 2), (33, 31), (63, 64), (257, 9), (1000, 256)])
def test_attention_of_one_request(heads, P, T):
    attention_case(shape(*heads), [(P, T)], seed=P + T)


@pytest.mark.parametrize("heads", [(32, 8, 128), (16, 4, 64)])
@pytest.mark.parametrize("P,T", [(5000, 1), (16383, 3), (40000, 20)])
def test_attention_over_long_contexts(heads, P, T):
    attention_case(shape(*heads), [(P, T)])


@pytest.mark.parametrize("heads", [(8, 1, 128), (2, 1, 64)])
@pytest.mark.parametrize("P,T", [(20000, 1), (52000, 3)])
def test_attention_in_more_chunks_than_a_wave_has_lanes(heads, P, T):
    """One KV head over a long range: a chunk for most of the CUs."""
    attention_case(shape(*heads), [(P, T)])


@pytest.mark.parametrize("page", [0, 32, 64, 256])
@pytest.mark.parametrize("heads", [(32, 8, 128), (16, 4, 64)])
def test_attention_of_ragged_batches(heads, page):
    attention_case(shape(*heads), [(1, 1), (900, 7), (64, 30), (33, 1), (511, 12), (2000, 3)], page=page)
    attention_case(shape(*heads), [(300 + 37 * i, 1 + i % 5) for i in range(33)], page=page)


def test_attention_of_peaked_scores_and_of_the_last_nodes_only():
    attention_case(shape(), [(500, 60)], spread=12.0)
    attention_case(shape(layers=2), [(100, 60), (40, 9)], layer=1, first=[44, 8])


@pytest.mark.parametrize("cache", ["bf16_128", "bf16_64", "f32_64"])
def test_attention_over_the_other_caches(cache):
    sh, flags = CACHES[cache]
    attention_case(sh, [(70, 20)], flags=flags)
    attention_case(sh, [(300, 5), (31, 9)], flags=flags, page=32)
    if cache == "bf16_64":
        attention_case(sh, [(70, 20)], flags=flags | sp.SP_FLAG_SIMPLE_KERNELS)


def test_what_is_not_finite_stays_with_those_that_see_it():
    """NaN and infinities in the K and V of nodes, and in query rows: 4 bits hold finite values, so nothing reaches the other
    rows through a masked weight of zero; a query row of NaN is NaN itself."""
    sh = shape()
    st = stage(sp, sh, slots=256, flags=sp.SP_FLAG_FP4_KV)
    st.request_init(0, 0, 128, 40)
    parents = [-1, -1, 0, 1]
    st.tree_insert(0, parents)
    k, v = rnd(1, 44, 2, 128), rnd(2, 44, 2, 128)
    k[40], v[40] = float("nan"), float("inf")                          # node 0, seen by nodes 0 and 2
    st.kv_store(0, 0, 0, k, v)
    q = rnd(3, 4, 1024)
    y = st.attention(0, [0], [0], [4], q)
    seen = np.ones((4, 44), bool)
    seen[:, 40:] = ancestors(parents)
    ref, mag, _ = attend(f64(q).reshape(4, 8, 128), held(f64(k)), held(f64(v)), seen)
    got = f64(y).reshape(4, 8, 128)
    assert (np.abs(got - ref)[[1, 3]] <= U * np.abs(ref)[[1, 3]] + 1.02 * U * mag[[1, 3]]).all()
    q2 = q.clone()
    q2[0] = float("nan")
    y2 = st.attention(0, [0], [0], [4], q2)
    assert torch.isnan(y2[0]).all() and torch.equal(y2[[1, 3]], y[[1, 3]])


def test_rows_behind_the_call_are_left_and_scores_of_a_fresh_slab_do_not_show():
    """A slab full of NaN codes: nothing outside the request's live slots is used, nothing outside the call's rows written."""
    sh = shape(32, 8, 128)
    st = stage(sp, sh, slots=4096, flags=sp.SP_FLAG_FP4_KV)
    st.kv.fill_(255)
    st.request_init(0, 100, 3000, 700)
    st.tree_insert(0, [-1] * 5)
    k, v = rnd(1, 705, 8, 128), rnd(2, 705, 8, 128)
    st.kv_store(0, 0, 0, k, v)
    room = torch.full((9, 4096), 3.0, dtype=torch.bfloat16, device="cuda")
    st.attention(0, [0], [0], [5], rnd(3, 5, 4096), room[:5])
    assert torch.isfinite(room).all() and (room[5:] == 3).all()
    st.append(0, [0], [0], [5], rnd(4, 5, 48 * 128), room[:5])
    assert (room[5:] == 3).all()


# ---- refusals -----------------------------------------------------------------------------------------------------
def test_refusals_leave_the_stage_as_it_was():
    sh = shape(layers=2)
    st = stage(sp, sh, slots=256, flags=sp.SP_FLAG_FP4_KV, rows=8)
    st.request_init(0, 0, 128, 40)
    st.tree_insert(0, [-1, 0, 1, 2])
    q, x = rnd(1, 4, 1024), rnd(2, 4, 12 * 128)

    def refused(status, call):
        with pytest.raises(sp.SpError) as err:
            call()
        assert err.value.status == status

    for layer in (-1, 2):
        refused(-1, lambda: st.append(layer, [0], [0], [4], x))
        refused(-1, lambda: st.attention(layer, [0], [0], [4], q))
    refused(-4, lambda: st.attention(0, [1], [0], [4], q))
    refused(-5, lambda: st.attention(0, [0], [1], [4], q))
    refused(-1, lambda: st.attention(0, [0], [0], [4], q, q))
    refused(-1, lambda: st.attention(0, [0, 0], [0, 0], [2, 2], q))
    both = torch.zeros(7, 1024, dtype=torch.bfloat16, device="cuda")
    refused(-1, lambda: st.attention(0, [0], [0], [4], both[:4], both[3:]))
    wide = torch.zeros(4 * 12 * 128, dtype=torch.bfloat16, device="cuda")
    refused(-1, lambda: st.append(0, [0], [0], [4], wide.view(4, -1), wide[:4096].view(4, -1)))
    refused(-2, lambda: st.kv_load(0, 0, 40, 5))
    refused(-1, lambda: st.kv_load(0, 0, -1, 2))
    refused(-1, lambda: st.kv_load(0, 2, 0, 2))
    refused(-2, lambda: st.kv_store(0, 0, 43, rnd(1, 2, 2, 128), rnd(1, 2, 2, 128)))
    refused(-4, lambda: st.kv_store(3, 0, 0, rnd(1, 2, 2, 128), rnd(1, 2, 2, 128)))
    with pytest.raises(ValueError):
        st.kv_view()
    st.tree_insert(0, [-1] * 5)
    refused(-2, lambda: st.attention(0, [0], [0], [9], rnd(1, 9, 1024)))      # more rows than the stage's calls carry
    st.tree_prune(0, sp.SP_DROP, 4)
    refused(-7, lambda: st.append(0, [0], [0], [4], x))
    refused(-7, lambda: st.kv_load(0, 0, 0, 2))
    st.kv_compact(0)
    assert st.request_info(0) == (40, 8, 0)
    with pytest.raises(sp.SpError):
        stage(sp, shape(4, 4, 64, dtype="f32"), slots=256, flags=sp.SP_FLAG_FP4_KV)
    with pytest.raises(sp.SpError):
        sp.fp4_pack_matrix(rnd(1, 17, 64))
    with pytest.raises(sp.SpError):
        sp.fp4_product(rnd(1, 2, 64), sp.fp4_pack_matrix(rnd(1, 48, 64)), gated=True)
    square, room = sp.fp4_pack_matrix(rnd(1, 64, 64)), torch.zeros(5, 64, dtype=torch.bfloat16, device="cuda")
    refused(-1, lambda: sp.fp4_product(room[:3], square, out=room[2:]))
    with pytest.raises(AssertionError):
        sp.fp4_product(room.cpu(), square)


def test_a_cache_past_32_bits():
    """A slab of 5 GB: the last heads' codes and scales lie past 4 GB, the last request's slots past 2^32 bytes of its planes' start."""
    sh, slots = shape(8, 8, 128), 4600 * 1000
    st = stage(sp, sh, slots=slots, flags=sp.SP_FLAG_FP4_KV, requests=2)
    P = 500
    for i, base in enumerate((0, slots - 600)):
        st.request_init(i, base, 600, P)
        st.tree_insert(i, [-1, 0])
        k, v = rnd(10 + i, P, 8, 128), rnd(20 + i, P, 8, 128)
        st.kv_store(i, 0, 0, k, v)
        qkv = rnd(30 + i, 2, 24 * 128)
        q = st.append(0, [i], [0], [2], qkv)
        out = st.attention(0, [i], [0], [2], q)
        hk, hv = (f64(t) for t in st.kv_load(i, 0, 0, P + 2))
        assert np.array_equal(hk[:P], held(f64(k))) and np.array_equal(hv[:P], held(f64(v)))
        assert np.array_equal(hv[P:], held(f64(qkv[:, 16 * 128:]).reshape(2, 8, 128)))
        seen = np.ones((2, P + 2), bool)
        seen[0, P + 1] = False
        y, mag, big = attend(f64(q).reshape(2, 8, 128), hk, hv, seen)
        off = U * np.abs(y) + (1.01 * U + (8 + 256) * F * (1 + big[..., None]) + 64 * F) * mag
        assert (np.abs(f64(out).reshape(y.shape) - y) <= off).all()


# ---- the whole stage ---------------------------------------------------------------------------------------------------
def forward_reference(st, sh, weights, x, q_seen, pos, cache):
    """float64 layers with the weights given and the K and V that the cache holds; returns the rows and, per layer, the K and V
    of the call's nodes before they are put into the cache."""
    h, made = x, []
    nq, kv, dh = sh.n_q_heads, sh.n_kv_heads, sh.d_head
    for l, w in enumerate(weights):
        def norm(v, gain):
            return v / np.sqrt((v * v).mean(-1, keepdims=True) + sh.rms_eps) * gain
        qkv = (norm(h, w["norm1"]) @ w["wqkv"].T).reshape(len(h), nq + 2 * kv, dh)
        q, k, v = qkv[:, :nq], qkv[:, nq:nq + kv], qkv[:, nq + kv:]
        if st.gains:
            q, k = head_norm(q, f64(st.gains[l]["q"]), sh.rms_eps), head_norm(k, f64(st.gains[l]["k"]), sh.rms_eps)
        made.append((rotate(k, pos, sh.rope_theta), v))
        a = attend(rotate(q, pos, sh.rope_theta), *cache[l], q_seen)[0].reshape(len(h), nq * dh)
        h = h + a @ w["wo"].T
        gu = norm(h, w["norm2"]) @ w["wgu"].T
        gate, up = gu[:, :sh.d_ff], gu[:, sh.d_ff:]
        h = h + (gate / (1 + np.exp(-gate)) * up) @ w["wd"].T
    return h, made


STAGES = {
    "fp4_cache": (shape(8, 2, 128, 2, 512, 768), sp.SP_FLAG_FP4_KV, False),
    "fp4_cache_norms": (shape(8, 2, 128, 2, 512, 768), sp.SP_FLAG_FP4_KV, True),
    "fp4_cache_64": (shape(4, 2, 64, 2, 320, 264), sp.SP_FLAG_FP4_KV, True),
    "fp4_weights": (shape(8, 2, 128, 2, 512, 768), sp.SP_FLAG_FP4_WEIGHTS, False),
    "fp4_both_norms": (shape(8, 4, 128, 4, 768, 1280), sp.SP_FLAG_FP4_WEIGHTS | sp.SP_FLAG_FP4_KV, True),
    "norms": (shape(8, 2, 128, 2, 512, 768), 0, True),
    "norms_64": (shape(4, 4, 64, 2, 256, 512), 0, True),
    "norms_f32": (shape(4, 4, 64, 2, 256, 512, "f32"), 0, True),
}


@pytest.mark.parametrize("n", [1, 7, 16, 30, 64, 150])
@pytest.mark.parametrize("kind", sorted(STAGES))
def test_forward_of_a_stage_with_4_bit_storage_or_head_norms(kind, n):
    """Against float64 on the values held.  The rows are compared as everywhere in these tests (largest distance over largest
    value: 2e-2 in bf16, 2e-4 in float32); the cache rows by what 4 bits are off, a third of the group's largest value, or
    the same bar."""
    use_own_stream()
    sh, flags, norms = STAGES[kind]
    page = 64 if n == 30 else 0
    st = stage(sp, sh, slots=1024, flags=flags, rows=256, page=page, norms=norms, seed=n)
    P = 75
    st.request_init(0, 0, 512, P)
    par = random_tree(n, n)
    for l in range(sh.n_layers):
        k, v = (rnd(l + 10 * i, P, sh.n_kv_heads, sh.d_head).to(st.tdtype) for i in range(2))
        st.kv_store(0, l, 0, k, v)
    x = rnd(5, n, sh.d_model).to(st.tdtype)
    weights = [{name: held(f64(t)) if flags & sp.SP_FLAG_FP4_WEIGHTS and not name.startswith("norm") else f64(t) for name, t in w.items()}
               for w in st.plain_layers]
    seen = np.ones((n, P + n), bool)
    seen[:, P:] = ancestors(par)
    pos = [P + int(a.sum()) - 1 for a in ancestors(par)]
    bar = 2e-4 if sh.dtype == "f32" else 2e-2
    first = None
    for turn in range(4):                           # calls of many launches replay a graph from the third on
        st.request_init(0, 0, 512, P)
        st.tree_insert(0, par)
        y = st.stage_forward([0], [0], [n], x)
        if first is None:
            first = y.clone()
            cache = [[f64(t) for t in st.kv_load(0, l, 0, P + n)] for l in range(sh.n_layers)]
            ref, made = forward_reference(st, sh, weights, f64(x), seen, pos, cache)
            assert np.abs(f64(y) - ref).max() <= bar * np.abs(ref).max()
            assert np.abs((f64(y) - f64(x)) - (ref - f64(x))).max() <= 2 * bar * np.abs(ref - f64(x)).max()
            for l in range(sh.n_layers):
                for got, want in zip(cache[l], made[l]):
                    err, big = np.abs(got[P:] - want), np.abs(want)
                    if flags & sp.SP_FLAG_FP4_KV:
                        top = np.repeat(big.reshape(*big.shape[:-1], -1, 32).max(-1), 32, -1)
                        assert (err <= top / 3 + bar * big.max()).all()
                    else:
                        assert err.max() <= bar * big.max()
        else:
            assert torch.equal(y, first)


def test_pieces_give_what_the_forward_call_gives():
    """A layer put together by the caller: projection, append, attention, output projection, gate and up, down, from the
    operators, against sp_stage_forward of the same stage."""
    sh = shape(8, 2, 128, 2, 512, 768)
    st = stage(sp, sh, slots=1024, flags=sp.SP_FLAG_FP4_KV | sp.SP_FLAG_FP4_WEIGHTS, requests=2, rows=64, norms=True)
    P, par = 130, random_tree(23, 4)
    st.request_init(0, 0, 512, P)
    st.request_init(1, 512, 512, P)
    for q in (0, 1):
        for l in range(2):
            st.kv_store(q, l, 0, rnd(l, P, 2, 128), rnd(5 + l, P, 2, 128))
        st.tree_insert(q, par)
    x = rnd(9, 23, 512)
    y = st.stage_forward([0], [0], [23], x)
    h = x.float()
    for l, w in enumerate(st.layers):
        def norm(v, gain):
            return (v * torch.rsqrt(v.square().mean(-1, keepdim=True) + sh.rms_eps) * gain.float()).to(torch.bfloat16)
        q = st.append(l, [1], [0], [23], sp.fp4_product(norm(h, w["norm1"]), w["wqkv"]))
        a = st.attention(l, [1], [0], [23], q)
        h = h + sp.fp4_product(a, w["wo"]).float()
        h = h + sp.fp4_product(sp.fp4_product(norm(h, w["norm2"]), w["wgu"], gated=True), w["wd"]).float()
    assert st.request_info(1)[2] == 23
    # the pieces round the projections to bf16 where the call keeps float32 sums, and 4 bits may then hold a neighbour
    assert (h - y.float()).abs().max() <= 5e-2 * y.float().abs().max()
    st.tree_prune(0, sp.SP_ACCEPT, 0)
    st.kv_compact(0)
    st.tree_prune(1, sp.SP_ACCEPT, 0)
    st.kv_compact(1)
    assert st.request_info(0)[:2] == st.request_info(1)[:2]


def test_captured_pieces_replay_with_the_values_of_the_time():
    sh = shape(32, 8, 128)
    use_own_stream()
    st = stage(sp, sh, slots=2048, flags=sp.SP_FLAG_FP4_KV, norms=True)
    st.request_init(0, 0, 2000, 1500)
    st.tree_insert(0, random_tree(20, 1))
    st.kv_store(0, 0, 0, rnd(1, 1500, 8, 128), rnd(2, 1500, 8, 128))
    w = sp.fp4_pack_matrix(rnd(3, 48 * 128, 512, scale=0.05))
    wo = sp.fp4_pack_matrix(rnd(4, 512, 4096, scale=0.05))
    x = rnd(5, 20, 512)
    q, a = torch.empty(20, 4096, dtype=torch.bfloat16, device="cuda"), torch.empty(20, 4096, dtype=torch.bfloat16, device="cuda")
    y = torch.empty(20, 512, dtype=torch.bfloat16, device="cuda")

    def step():
        st.append(0, [0], [0], [20], sp.fp4_product(x, w), q)
        st.attention(0, [0], [0], [20], q, a)
        sp.fp4_product(a, wo, out=y)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        x.copy_(rnd(50 + turn, 20, 512))
        graph.replay()
        torch.cuda.synchronize()
        replayed = y.clone()
        rows = [t.clone() for t in st.kv_load(0, 0, 1500, 20)]
        step()
        torch.cuda.synchronize()
        assert torch.equal(replayed, y)
        assert all(torch.equal(r, t) for r, t in zip(rows, st.kv_load(0, 0, 1500, 20)))


def test_calls_on_two_streams_do_not_share_what_they_write():
    """Products own nothing but their arguments: two of them at once on two streams, each with its workspace."""
    x, w = rnd(1, 3, 8192), sp.fp4_pack_matrix(rnd(2, 256, 8192))
    want = sp.fp4_product(x, w)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for turn in range(10):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(sp.fp4_product(x, w))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
