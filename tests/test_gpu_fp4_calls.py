"""Calls of the 4-bit operators and of stages on them that the documentation allows, in forms that test_gpu_fp4.py does not make."""
import random

import numpy as np
import pytest
import torch

import paper_2504_04104_amd as sp
from fp4_layers import bf16, layer, tree
from fp4_reference import ancestors, attend, f64, held, random_tree, stage
from gpu_harness import use_own_stream
from test_gpu_fp4 import F, U, rnd, shape

pytestmark = pytest.mark.gpu


def test_calls_without_a_row():
    """No request, or requests without nodes: nothing to do, as in the forward call."""
    st = stage(sp, shape(layers=2), slots=256, flags=sp.SP_FLAG_FP4_KV)
    st.request_init(0, 0, 128, 40)
    st.tree_insert(0, [-1, 0])
    qkv, q, x = rnd(1, 0, 12 * 128), rnd(1, 0, 1024), rnd(1, 0, 256)
    for ids, first, n in (([], [], []), ([0], [0], [0]), ((), (), ()), (np.zeros(0, int), np.zeros(0, int), np.zeros(0, int))):
        for layer in range(2):
            assert st.append(layer, ids, first, n, qkv).shape == (0, 1024)
            assert st.attention(layer, ids, first, n, q).shape == (0, 1024)
        assert st.stage_forward(ids, first, n, x).shape == (0, 256)
        assert st.request_info(0) == (40, 2, 0)


# ---- forward calls in the other forms ------------------------------------------------------------------------------------
KV, W, PACKED, SIMPLE = sp.SP_FLAG_FP4_KV, sp.SP_FLAG_FP4_WEIGHTS, sp.SP_FLAG_PACKED_WEIGHTS, sp.SP_FLAG_SIMPLE_KERNELS
KINDS = {                                           # shape, flags, head norms, page
    "cache": (shape(8, 2, 128, 2, 512, 768), KV, False, 0),
    "cache_packed": (shape(8, 2, 128, 2, 512, 768), KV | PACKED, False, 64),
    "cache_packed_norms": (shape(8, 2, 128, 2, 512, 768), KV | PACKED, True, 0),
    "cache_simple": (shape(8, 2, 128, 2, 512, 768), KV | SIMPLE, False, 0),
    "cache_64": (shape(8, 2, 64, 2, 320, 264), KV, True, 32),
    "both_norms": (shape(8, 2, 128, 2, 512, 768), KV | W, True, 32),
    "weights": (shape(8, 2, 128, 2, 512, 768), W, False, 64),
    "packed_norms": (shape(8, 2, 128, 2, 512, 768), PACKED, True, 0),
    "norms": (shape(8, 2, 128, 2, 512, 768), 0, True, 64),
    "norms_f32": (shape(4, 4, 64, 2, 256, 512, "f32"), 0, True, 32),
}
# requests of a call: (context, nodes in front of the call's, nodes of the call)
CALLS = {
    "short": [(40, 0, 3), (33, 5, 1), (200, 0, 12), (1, 2, 2)],
    "cut": [(2100, 0, 2), (2600, 3, 1)],            # few blocks over ranges of more than eight rounds: chunks and a merge
    "cut_shared": [(3400, 0, 30)],                  # blocks that share a range
    "one_row": [(60, 0, 1)],
    "wide": [(70, 0, 90), (100, 10, 40)],
}


def plain_and_packed(sh, flags, seed):
    """Weights of the right shapes as they are, and as the stage takes them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if sh.dtype == "bf16" else torch.float32
    size = {"wqkv": ((sh.n_q_heads + 2 * sh.n_kv_heads) * sh.d_head, sh.d_model), "wo": (sh.d_model, sh.n_q_heads * sh.d_head),
            "wgu": (2 * sh.d_ff, sh.d_model), "wd": (sh.d_model, sh.d_ff)}
    layers = []
    for _ in range(sh.n_layers):
        w = {n: (0.05 * torch.randn(*s, generator=g, device="cuda")).to(dt) for n, s in size.items()}
        for n in ("norm1", "norm2"):
            w[n] = (1 + 0.05 * torch.randn(sh.d_model, generator=g, device="cuda")).to(dt)
        layers.append(w)
    if flags & W:
        return sp.fp4_pack_weights(sh, layers), sp.fp4_pack_weights(sh, layers)
    return layers, sp.pack_weights(sh, layers) if flags & PACKED else layers


def make(sh, flags, norms, page, slots, requests, rows, seed=0):
    plain, packed = plain_and_packed(sh, flags, seed)
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if sh.dtype == "bf16" else torch.float32
    gains = [{n: (1 + 0.2 * torch.randn(sh.d_head, generator=g)).to("cuda", dt) for n in "qk"} for _ in range(sh.n_layers)] if norms else None
    st = sp.Stage(sh, packed, kv_slots=slots, max_requests=requests, max_batch_nodes=rows, flags=flags | (sp.SP_FLAG_PAGED_KV if page else 0),
                  page_slots=page, head_norms=gains)
    return st, plain, gains


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("kind", sorted(KINDS))
def test_forward_of_several_requests(kind, name):
    """Against float64 layers that round where the stage keeps bfloat16, over the K and V that the cache holds after the call (what
    4 bits make of the new ones is checked by itself): 1e-2 of the largest value, half of the bar of the other forward calls (2e-4 in
    float32).  The new rows: a third of the group's largest value in 4 bits, and the same bar."""
    sh, flags, norms, page = KINDS[kind]
    reqs = CALLS[name]
    r = bf16 if sh.dtype == "bf16" else (lambda t: t)
    bar = 1e-2 if sh.dtype == "bf16" else 2e-4
    cap = [-(-(P + a + n) // 64) * 64 for P, a, n in reqs]
    st, plain, gains = make(sh, flags, norms, page, sum(cap), len(reqs), 256)
    base = 0
    for q, (P, before, n) in enumerate(reqs):
        st.request_init(q, 0 if page else base, cap[q], P)
        base += cap[q]
        for l in range(sh.n_layers):
            st.kv_store(q, l, 0, *(rnd(100 * q + 10 * l + i, P, sh.n_kv_heads, sh.d_head).to(st.tdtype) for i in range(2)))
    ids = list(range(len(reqs)))
    parents = [random_tree(a + n, 3 + q) for q, (_, a, n) in enumerate(reqs)]
    st.tree_insert_batch(ids, parents)
    first, count = [a for _, a, _ in reqs], [n for _, _, n in reqs]
    x = rnd(7, sum(a + n for _, a, n in reqs), sh.d_model).to(st.tdtype)
    if any(first):
        ahead = [q for q in ids if first[q]]
        rows = torch.cat([x[:first[q]] for q in ahead])
        st.stage_forward(ahead, [0] * len(ahead), [first[q] for q in ahead], rows)
    x = x[:sum(count)].contiguous()
    y, at = st.stage_forward(ids, first, count, x).double(), 0
    for q, (P, before, n) in enumerate(reqs):
        pos, seen = tree(P, parents[q])
        pos, seen = pos[before:], seen[before:]
        h = x[at:at + n].double()
        for l, w in enumerate(plain):
            kept = [t.double() for t in st.kv_load(q, l, 0, P + before + n)]

            def cache(k, v):
                for new, old in ((k, kept[0]), (v, kept[1])):
                    off, big = (old[P + before:] - new).abs(), new.abs()
                    if flags & KV:
                        top = big.unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32, -1)
                        assert (off <= top / 3 + bar * big.max()).all()
                    else:
                        assert off.max() <= bar * big.max()
                return kept
            h = layer(w, h, pos, seen, cache, sh, r, gains[l] if norms else None)
        got = y[at:at + n]
        assert (got - h).abs().max() <= bar * h.abs().max()
        assert (got - h).abs().max() <= 2 * bar * (h - x[at:at + n].double()).abs().max()
        at += n


REPLAYED = {                                        # flags, head norms, page, rows of a call's requests, their contexts
    "cache": (KV | PACKED, False, 0, [4, 1, 3, 2, 4, 2], [33, 1, 257, 31, 128, 300]),
    "cache_cut": (KV | PACKED, False, 64, [3, 2, 4], [1900, 2000, 2040]),
    "cache_shared": (KV, True, 32, [9, 12, 5, 20], [33, 130, 257, 64]),
    "cache_shared_cut": (KV, False, 0, [9, 12], [3400, 3500]),
    "both": (KV | W, True, 32, [9, 12, 5, 20], [33, 130, 257, 64]),
    "both_cut": (KV | W, False, 0, [3, 2, 4], [1900, 2000, 2040]),
    "weights": (W, False, 64, [1, 2, 1], [33, 130, 257]),
    "packed_norms": (PACKED, True, 0, [3, 2, 4], [33, 130, 257]),
    "norms_cut": (0, True, 32, [3, 2, 4], [1040, 1100, 1222]),
}


@pytest.mark.parametrize("name", sorted(REPLAYED))
def test_replays_under_changing_plans(name):
    """Calls of one shape again and again (four layers: more launches than are made one by one), with other requests, contexts, first
    nodes, rows and result tensors: a replayed graph gives the bits of a stage that may not replay, and writes the same cache."""
    flags, norms, page, rows, contexts = REPLAYED[name]
    sh = shape(8, 2, 128, 4, 512, 512)
    use_own_stream()
    rng = random.Random(31)
    nodes = max(rows) + 3
    ids = list(range(len(rows)))
    cap = -(-(max(contexts) + nodes) // 64) * 64
    stages = [make(sh, flags | f, norms, page, cap * len(rows), len(rows), nodes * len(rows), 4)[0] for f in (0, sp.SP_FLAG_NO_GRAPHS)]
    kv = stages[0].kv
    if flags & KV:
        kv.random_(0, 256)
        scales = kv[-sh.n_layers * 2 * sh.n_kv_heads * cap * len(rows) * 4:]
        scales.random_(124, 130)                    # the groups' powers of two, about one
    else:
        stages[0].kv_view().normal_()
    stages[1].kv.copy_(kv)
    parents = [random_tree(nodes, 31 + q) for q in ids]
    results = []
    for rep in range(7):
        calls, lengths, first = rng.sample(ids, len(ids)), rng.sample(contexts, len(ids)), [rng.randint(0, nodes - n) for n in rows]
        x_all, x = rnd(rep, nodes * len(rows), 512), rnd(50 + rep, sum(rows), 512)
        ys = []
        for st in stages:
            for q in ids:
                st.request_init(q, 0 if page else cap * q, cap, lengths[q])
            st.tree_insert_batch(ids, parents)
            st.stage_forward(ids, [0] * len(ids), [nodes] * len(ids), x_all)
            y = torch.full_like(x, float("nan"))
            st.stage_forward(calls, first, rows, x, y)
            ys.append(y)
        assert torch.isfinite(ys[1]).all()
        assert torch.equal(ys[0], ys[1]), rep
        assert torch.equal(stages[0].kv, stages[1].kv), rep
        results.append((ys[0], ys[1].clone()))
    for y, want in results:
        assert torch.equal(y, want)


def test_new_head_norms_are_those_of_the_next_call():
    """Replayed calls too: gains set, changed and taken away between calls of a shape that has its graph."""
    use_own_stream()
    sh = shape(8, 2, 128, 4, 512, 512)
    st, plain, gains = make(sh, KV, True, 0, 512, 1, 64)
    other = [{n: t * 0.5 for n, t in g.items()} for g in gains]
    x, par = rnd(1, 20, 512), random_tree(20, 2)

    def call(norms):
        st.set_head_norms(norms)
        for _ in range(3):
            st.request_init(0, 0, 300, 50)
            for l in range(4):
                st.kv_store(0, l, 0, rnd(l, 50, 2, 128), rnd(9 + l, 50, 2, 128))
            st.tree_insert(0, par)
            y = st.stage_forward([0], [0], [20], x)
        return y
    a, b, none = call(gains), call(other), call(None)
    for norms, y in ((gains, a), (None, none), (other, b), (gains, a)):
        fresh = make(sh, KV | sp.SP_FLAG_NO_GRAPHS, False, 0, 512, 1, 64)[0]
        fresh.set_head_norms(norms)
        fresh.request_init(0, 0, 300, 50)
        for l in range(4):
            fresh.kv_store(0, l, 0, rnd(l, 50, 2, 128), rnd(9 + l, 50, 2, 128))
        fresh.tree_insert(0, par)
        assert torch.equal(fresh.stage_forward([0], [0], [20], x), y)
        assert torch.equal(call(norms), y)
    assert not torch.equal(a, b) and not torch.equal(a, none)


def test_gains_that_are_replaced_may_go():
    """Calls that were made with them have run when the call returns, also those that no graph replays."""
    use_own_stream()
    st, _, gains = make(shape(8, 2, 128, 1, 512, 512), KV | sp.SP_FLAG_NO_GRAPHS, True, 0, 512, 1, 64)
    st.request_init(0, 0, 300, 50)
    st.tree_insert(0, [-1, 0])
    big = torch.randn(8192, 8192, device="cuda", dtype=torch.bfloat16)
    for norms in (None, gains, [{n: t + 1 for n, t in g.items()} for g in gains], gains):
        had = st.head_norms is not None
        for _ in range(40):                         # some 30 ms in front of the call
            big @ big
        st.stage_forward([0], [0], [2], rnd(1, 2, 512))
        st.set_head_norms(norms)
        assert torch.cuda.current_stream().query() or not had
        torch.cuda.synchronize()


# ---- products and pieces at the same time, and at the limits --------------------------------------------------------------
def test_products_that_cut_their_columns_on_two_streams():
    """Each has a workspace, which the other must not write: other rows on either stream."""
    m, n, k = 20, 256, 8192
    assert sp.load_library().sp_fp4_product_workspace(m, n, k, 0) > 0 and sp.load_library().sp_fp4_product_workspace(m, n // 2, k, 1) > 0
    w = sp.fp4_pack_matrix(rnd(1, n, k))
    xs = [rnd(2 + i, m, k) for i in range(2)]
    want = [(sp.fp4_product(x, w), sp.fp4_product(x, w, gated=True)) for x in xs]
    assert not torch.equal(want[0][0], want[1][0])
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for turn in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs.append((i, sp.fp4_product(xs[i], w), sp.fp4_product(xs[i], w, gated=True)))
    torch.cuda.synchronize()
    for i, y, z in outs:
        assert torch.equal(y, want[i][0]) and torch.equal(z, want[i][1])


def test_two_captured_graphs_of_one_stage_replay_in_turn():
    """Attention over cut ranges and cut products, captured for two requests: the stage's workspace is theirs in turn."""
    use_own_stream()
    sh = shape(32, 8, 128)
    st = stage(sp, sh, slots=16384, flags=KV, requests=2, norms=True)
    for q, P in ((0, 6000), (1, 7000)):
        st.request_init(q, 8192 * q, 8000, P)
        st.kv_store(q, 0, 0, rnd(q, P, 8, 128), rnd(5 + q, P, 8, 128))
        st.tree_insert(q, random_tree(4 + q, q))
    w, wo = sp.fp4_pack_matrix(rnd(3, 48 * 128, 512, scale=0.05)), sp.fp4_pack_matrix(rnd(4, 512, 4096, scale=0.05))
    x = [rnd(20 + q, 4 + q, 512) for q in (0, 1)]
    y = [torch.empty(4 + q, 512, dtype=torch.bfloat16, device="cuda") for q in (0, 1)]

    def step(q):
        a = st.attention(0, [q], [0], [4 + q], st.append(0, [q], [0], [4 + q], sp.fp4_product(x[q], w)))
        sp.fp4_product(a, wo, out=y[q])
    graphs = []
    for q in (0, 1):
        step(q)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(q)
        graphs.append(g)
    for turn in range(4):
        for q in (0, 1):
            x[q].copy_(rnd(40 + 2 * turn + q, 4 + q, 512))
        for q in (1, 0) if turn % 2 else (0, 1):
            graphs[q].replay()
        replayed = [t.clone() for t in y]
        for q in (0, 1):
            step(q)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, y))


@pytest.mark.parametrize("page", [0, 4096])
def test_the_last_slots_of_the_largest_cache(page):
    """A plane of just under 2 GB: offsets inside it up to 2^31, and a last tile that ends with it."""
    sh = shape(4, 1, 128)
    slots = (1 << 25) - (page or 1)
    st = stage(sp, sh, slots=slots, flags=KV, requests=2, page=page)
    P, parents = 33, [-1, 0, -1, 1]
    if page:                                        # all pages but the last belong to another request
        st.request_init(1, 0, slots - page, slots - page)
        st.request_init(0, 0, page, P)
    else:
        st.request_init(0, slots - P - 4, P + 4, P)
    st.tree_insert(0, parents)
    k, v = rnd(1, P, 1, 128), rnd(2, P, 1, 128)
    st.kv_store(0, 0, 0, k, v)
    qkv = rnd(3, 4, 6 * 128)
    q = st.append(0, [0], [0], [4], qkv)
    out = st.attention(0, [0], [0], [4], q)
    hk, hv = (f64(t) for t in st.kv_load(0, 0, 0, P + 4))
    assert np.array_equal(hk[:P], held(f64(k))) and np.array_equal(hv[:P], held(f64(v)))
    assert np.array_equal(hv[P:], held(f64(qkv[:, 5 * 128:]).reshape(4, 1, 128)))
    if not page:                                    # codes of the last slot are the last bytes of their plane
        codes = st.kv[:2 * slots * 64].view(2, slots, 64)
        assert codes[:, -1].any() and not codes[:, slots - P - 5].any()
    seen = np.ones((4, P + 4), bool)
    seen[:, P:] = ancestors(parents)
    y, mag, big = attend(f64(q).reshape(4, 4, 128), hk, hv, seen)
    off = U * np.abs(y) + (1.01 * U + (8 + 256) * F * (1 + big[..., None]) + 64 * F) * mag
    assert (np.abs(f64(out).reshape(y.shape) - y) <= off).all()
