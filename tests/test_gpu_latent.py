"""A stage with a cache of latent vectors against float64: rows, append, attention, trees, and a layer's run of them.

u = 2^-8 is half a step of bf16 relative to the value, 2^-24 of float32."""
import math

import numpy as np
import pytest
import torch

import workloads as wl
import paper_2504_04104_amd as sp
from fp4_reference import ancestors, f64
from gpu_harness import use_own_stream
from latent_reference import attend, frequencies, make, pair_lengths, positions, seen_by, turn

pytestmark = pytest.mark.gpu
U, F = 2.0 ** -8, 2.0 ** -24


def rnd(seed, *size, scale=1.0):
    return (scale * torch.randn(*size, generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16).cuda()


def refused(status, call):
    with pytest.raises(sp.SpError) as err:
        call()
    assert err.value.status == status


# ---- attention -------------------------------------------------------------------------------------------
def check_rows(got, q, rows, c, seen, scale):
    y, mag, big = attend(q, rows, c, seen, scale)
    # the result's rounding; every weight rounded to bf16, against their exact sum; scores off by a float32 step of every column's
    # product and the exponential, the sums and the chunks' rescaling by as many again
    off = U * y.abs() + (1.01 * U + (8 + 2 * q.shape[-1]) * F * (1 + big) + 64 * F) * mag
    assert torch.isfinite(got).all()
    bad = (got.double() - y).abs() / off
    assert (bad <= 1).all(), bad.max().item()


def attention_case(heads, c, r, trees, first=None, layer=0, layers=1, seed=0, **kw):
    st = make(heads, c, r, trees, layers=layers, layer=layer, seed=seed, **kw)
    first = first or [0] * len(trees)
    for i, f in enumerate(first):           # nodes in front of the call's count as forwarded after an append to the last layer
        if f:
            keep = st.kv_load(i, layers - 1, trees[i][0], f)
            st.append(layers - 1, [i], [0], [f], rnd(1, f, heads, r), rnd(2, f, c + r))
            st.kv_store(i, layers - 1, trees[i][0], keep)
    n = [T - f for (_, T), f in zip(trees, first)]
    q = rnd(seed + 9, sum(n), heads, c + r)
    got, at, scale = st.attention(layer, list(range(len(trees))), first, n, q), 0, (c // 4 + r) ** -0.5
    for i, rows in enumerate(n):
        check_rows(got[at:at + rows], q[at:at + rows], st.held[i], c, seen_by(st, i, first[i]), scale)
        at += rows
    return st, q, got


DIMS = [(512, 64), (256, 32), (512, 32), (256, 64)]


@pytest.mark.parametrize("heads", [1, 3, 16, 24, 128])
@pytest.mark.parametrize("P,T", [(1, 1), (1, 40), (31, 1), (32, 2), (33, 31), (63, 64), (257, 9), (1000, 256)])
def test_attention_of_one_request(heads, P, T):
    attention_case(heads, 512, 64, [(P, T)], seed=P + T)


@pytest.mark.parametrize("c,r", DIMS)
@pytest.mark.parametrize("heads,P,T", [(16, 100, 1), (5, 333, 7), (64, 500, 33), (128, 2100, 3)])
def test_attention_of_every_covered_space(c, r, heads, P, T):
    attention_case(heads, c, r, [(P, T)], seed=P)
    attention_case(heads, c, r, [(P, T), (P // 2 + 1, T + 1)], seed=P, page=32)


@pytest.mark.parametrize("c,r", [(512, 64), (64, 16), (1024, 128), (136, 8), (8, 24)])
@pytest.mark.parametrize("trees", [[(1, 1)], [(300, 9)], [(63, 64), (5, 2)]])
def test_attention_by_plain_kernels(c, r, trees):
    attention_case(6, c, r, trees, flags=sp.SP_FLAG_SIMPLE_KERNELS)
    attention_case(6, c, r, trees, page=64, flags=sp.SP_FLAG_SIMPLE_KERNELS)
    attention_case(6, c, r, trees)


@pytest.mark.parametrize("heads,P,T", [(1, 20000, 1), (16, 40000, 1), (16, 32749, 5), (128, 9000, 2), (64, 16383, 20), (8, 70000, 3)])
def test_attention_over_long_contexts(heads, P, T):
    attention_case(heads, 512, 64, [(P, T)])


@pytest.mark.parametrize("page", [0, 32, 64, 256])
@pytest.mark.parametrize("heads,c,r", [(16, 512, 64), (40, 256, 32)])
def test_attention_of_ragged_batches(heads, c, r, page):
    attention_case(heads, c, r, [(1, 1), (900, 7), (64, 30), (33, 1), (511, 12), (2000, 3)], page=page)
    attention_case(heads, c, r, [(300 + 37 * i, 1 + i % 5) for i in range(33)], page=page)
    attention_case(heads, c, r, [(9000, 2), (31, 1), (4000, 40)], page=page)


@pytest.mark.parametrize("heads", [16, 64])
def test_attention_of_many_rows(heads):
    attention_case(heads, 512, 64, [(300, 200), (1500, 256), (77, 150)], page=64)
    attention_case(heads, 512, 64, [(700 + 11 * i, 40 + i) for i in range(20)])


def test_attention_of_peaked_scores_and_of_the_last_nodes_only():
    attention_case(16, 512, 64, [(500, 60)], spread=6.0)
    attention_case(40, 256, 32, [(3000, 60)], spread=8.0)
    attention_case(16, 512, 64, [(100, 60), (40, 9)], first=[44, 8], layer=1, layers=2)


def test_scores_that_rise_and_fall_along_the_context():
    """Rows whose scores grow slot by slot, so that every tile raises the maximum, and rows where the first slot outweighs all."""
    P, H = 3000, 16
    st = make(H, 512, 64, [(P, 2)])
    ramp = torch.linspace(-60, 60, P + 2, device="cuda")
    rows = st.held[0].clone()
    rows[:, 0] = ramp.to(torch.bfloat16)
    st.kv_store(0, 0, 0, rows)
    q = rnd(3, 2, H, 576, scale=0.2)
    scale = (128 + 64) ** -0.5
    for v in (20.0, -20.0, 0.0):
        q[:, :, 0] = v
        check_rows(st.attention(0, [0], [0], [2], q), q, rows, 512, seen_by(st, 0), scale)


@pytest.mark.parametrize("heads", [4, 16, 64])
def test_what_is_not_finite_stays_with_those_that_see_it(heads):
    """A node's row of NaN or of infinities, a query row of NaN: whoever does not see the slot is as without it."""
    for bad in (float("nan"), float("inf"), -float("inf")):
        for col in (0, 300, 511, 540):
            st = make(heads, 512, 64, [(40, 5)])
            st.tree_prune(0, sp.SP_CLEAR, 0)
            st.kv_compact(0)
            st.tree_insert(0, [-1, -1, 0, 1, 1])
            rows = st.held[0].clone()
            st.kv_store(0, 0, 0, rows)
            q = rnd(3, 5, heads, 576)
            clean = st.attention(0, [0], [0], [5], q)
            rows[40, col] = bad                                       # node 0, seen by nodes 0 and 2
            st.kv_store(0, 0, 0, rows)
            y = st.attention(0, [0], [0], [5], q)
            assert torch.equal(y[[1, 3, 4]], clean[[1, 3, 4]]), (bad, col)
            if math.isnan(bad):
                assert torch.isnan(y[[0, 2]]).all()
            q2 = q.clone()
            q2[3, heads // 2] = float("nan")
            y2 = st.attention(0, [0], [0], [5], q2)
            assert torch.isnan(y2[3, heads // 2]).all()
            y2[3, heads // 2] = y[3, heads // 2]
            assert torch.equal(y2[[1, 3, 4]], y[[1, 3, 4]])


@pytest.mark.parametrize("heads", [16, 80])
def test_rows_behind_the_call_are_left_and_what_lies_around_does_not_show(heads):
    """A slab full of NaN: nothing outside the request's live slots is used, nothing outside the call's rows written."""
    for P, T in ((700, 5), (95, 1), (40, 30)):
        st = sp.LatentStage(1, heads, 512, 64, scale=0.07, kv_slots=4096, max_batch_nodes=64)
        st.kv_view().fill_(float("nan"))
        st.workspace.fill_(255)
        st.request_init(0, 101, 3000, P)
        st.tree_insert(0, [-1] * T)
        rows = rnd(1, P + T, 576)
        st.kv_store(0, 0, 0, rows)
        room = torch.full((T + 4, heads, 512), 3.0, dtype=torch.bfloat16, device="cuda")
        q = rnd(3, T, heads, 576)
        st.attention(0, [0], [0], [T], q, room[:T])
        seen = torch.ones(T, P + T, dtype=torch.bool, device="cuda")
        seen[:, P:] = torch.eye(T, dtype=torch.bool)
        check_rows(room[:T], q, rows, 512, seen, 0.07)
        assert (room[T:] == 3).all()


def test_a_cache_past_32_bits():
    """Slots whose bytes, and values, lie beyond 2^32 and 2^31 from the layer's first."""
    slots = 4_200_000                                                 # 4.8 GB a layer
    st = sp.LatentStage(2, 16, 512, 64, scale=0.07, kv_slots=slots, max_requests=2, max_batch_nodes=64)
    P, T = 900, 4
    for layer in (0, 1):
        st.request_init(0, slots - 1000, 1000, P)
        st.tree_insert(0, [-1, 0, 1, 0])
        rows, q = rnd(1 + layer, P + T, 576), rnd(3, T, 16, 576)
        st.kv_store(0, layer, 0, rows)
        assert torch.equal(st.kv_load(0, layer, 0, P + T), rows)
        seen = torch.ones(T, P + T, dtype=torch.bool, device="cuda")
        seen[:, P:] = torch.from_numpy(ancestors([-1, 0, 1, 0])).cuda()
        check_rows(st.attention(layer, [0], [0], [T], q), q, rows, 512, seen, 0.07)
        kv = rnd(5, T, 576)
        st.append(layer, [0], [0], [T], rnd(6, T, 16, 64), kv)
        assert torch.equal(st.kv_load(0, layer, P, T)[:, :512], kv[:, :512])
        assert torch.equal(st.kv_load(0, layer, 0, P), rows[:P])


# ---- append, rows, trees ------------------------------------------------------------------------------------
@pytest.mark.parametrize("layout,dims", [("half", 64), ("half", 32), ("half", 24), ("interleaved", 64), ("interleaved", 16), (None, 64)])
@pytest.mark.parametrize("normed", [False, True])
@pytest.mark.parametrize("trees", [[(1, 1)], [(512, 1)], [(40, 37)], [(100000, 256)], [(3, 5), (700, 64), (31, 1), (32, 33), (5, 2)]])
def test_append(layout, dims, normed, trees):
    for heads, c, r in ((16, 512, 64), (5, 256, 64), (3, 136, 64), (128, 1024, 64)):
        gains = [(1 + 0.2 * torch.randn(c, generator=torch.Generator().manual_seed(l))).to(torch.bfloat16).cuda() for l in range(2)] if normed else None
        rope = None if layout is None else sp.Rope(layout, dims, 10000.0, ("ramp", 16.0, 4096.0, 32.0, 1.0), gain=1.2)
        st = make(heads, c, r, trees, page=32 if len(trees) > 1 else 0, layers=2, norms=gains, rope=rope, rms_eps=1e-5, rope_theta=500000.0)
        M = sum(T for _, T in trees)
        q, kv = rnd(1, M, heads, 128 + r), rnd(2, M, c + r + 8, scale=1.5)
        q_out = torch.full((M, heads, c + r), 5.0, dtype=torch.bfloat16, device="cuda")
        before = [st.kv_load(i, 1, 0, P) for i, (P, _) in enumerate(trees)]
        st.append(1, list(range(len(trees))), [0] * len(trees), [T for _, T in trees], q[..., 128:], kv[:, :c + r], q_out[..., c:])
        assert (q_out[..., :c] == 5).all()
        pos = positions(st)
        freq, lay, gain = (frequencies(r, 500000.0), "half", 1.0) if rope is None else (rope.freq, layout, 1.2)

        def near(got, x):
            want = turn(x, pos, freq, lay, gain)
            off = U * np.abs(want) + 16 * F * gain * pair_lengths(x, len(freq), lay)
            return (np.abs(got - want) <= off).all()
        assert near(f64(q_out[..., c:]), f64(q[..., 128:]))
        latent = f64(kv[:, :c])
        if normed:
            latent = latent / np.sqrt((latent ** 2).mean(-1, keepdims=True) + 1e-5) * f64(gains[1])
        got, at = [], 0
        for i, (P, T) in enumerate(trees):
            got.append(f64(st.kv_load(i, 1, P, T)))
            assert torch.equal(st.kv_load(i, 1, 0, P), before[i])
            assert st.request_info(i)[2] == T                         # the last layer: the nodes count as forwarded
        got = np.concatenate(got)
        # a float32 sum of c squares, its root's reciprocal, two products
        assert (np.abs(got[:, :c] - latent) <= (U + (16 + c / 2) * F) * np.abs(latent)).all()
        assert near(got[:, None, c:], f64(kv[:, None, c:c + r]))


def test_append_in_place_and_of_some_nodes():
    st = make(4, 256, 32, [(50, 4)], layers=2)
    st.tree_prune(0, sp.SP_CLEAR, 0)
    st.kv_compact(0)
    st.tree_insert(0, [-1, 0, 1, -1])
    q, kv = rnd(1, 2, 4, 288), rnd(2, 2, 288)
    for l in range(2):
        refused(-6, lambda: st.append(l, [0], [2], [2], q[..., 256:], kv))           # its parent is not there yet
        refused(-6, lambda: st.attention(l, [0], [2], [2], q))
    plain = st.append(0, [0], [0], [2], q[..., 256:], kv)
    assert st.request_info(0)[2] == 0
    keep = q.clone()
    st.append(1, [0], [0], [2], q[..., 256:], kv, q[..., 256:])
    assert torch.equal(q[..., 256:], plain) and torch.equal(q[..., :256], keep[..., :256])
    assert st.request_info(0)[2] == 2
    held = st.kv_load(0, 1, 50, 4)
    assert held[:2].any() and not held[2:].any()
    st.append(1, [0], [2], [2], q[..., 256:], kv)
    assert st.request_info(0)[2] == 4 and torch.equal(st.kv_load(0, 1, 50, 2), held[:2])


@pytest.mark.parametrize("page", [0, 32])
@pytest.mark.parametrize("mode", [sp.SP_ACCEPT, sp.SP_DROP, sp.SP_CLEAR])
def test_compaction_moves_rows(page, mode):
    st = make(4, 256, 32, [(61, 90), (20, 3)], page=page, layers=2)
    both = [[rnd(10 * l + i, P + T, 288) for l in range(2)] for i, (P, T) in enumerate(st.trees)]
    for i in range(2):
        for l in range(2):
            st.kv_store(i, l, 0, both[i][l])
    held = st.kv_load(0, 1, 61, 90)
    st.append(1, [0], [0], [90], rnd(1, 90, 4, 32), rnd(2, 90, 288))                     # forwarded
    st.kv_store(0, 1, 61, held)
    up, node = ancestors(st.parents[0]), 7
    x = rnd(5, 90, 256)
    xr = x.clone()
    st.tree_prune(0, mode, node)
    n, _ = st.kv_compact(0, xr, list(range(90)))
    if mode == sp.SP_ACCEPT:
        keep = np.flatnonzero(up[node] | up[:, node])
        rows = np.flatnonzero(up[:, node])
    else:
        keep = rows = np.flatnonzero(~up[:, node]) if mode == sp.SP_DROP else np.zeros(0, int)
    assert n == len(rows) and torch.equal(xr[:n], x[torch.from_numpy(rows).cuda()])
    P, T, _ = st.request_info(0)
    assert P + T == 61 + len(keep)
    src = torch.from_numpy(np.concatenate([np.arange(61), 61 + keep])).cuda()
    for l in range(2):
        assert torch.equal(st.kv_load(0, l, 0, P + T), both[0][l][src])
        assert torch.equal(st.kv_load(1, l, 0, 23), both[1][l])


def test_the_output_head_and_pruning_by_its_result():
    """The last stage's verification on a latent stage gives what it gives on another with the same hidden rows."""
    V, d = 512, 256
    head = {"norm": (1 + 0.1 * torch.randn(d, generator=torch.Generator().manual_seed(1))).to(torch.bfloat16).cuda(), "wvocab": rnd(2, V, d)}
    from fp4_reference import stage
    other = stage(sp, wl.ModelShape(1, d, 2, 1, 128, 256, 1e-5, 500000.0, "bf16"), slots=256)
    st = sp.LatentStage(1, 4, 256, 32, scale=0.1, kv_slots=256, d_model=d, rms_eps=1e-5)
    x = rnd(3, 6, d)
    got = []
    for s in (other, st):
        s.request_init(0, 0, 100, 30)
        s.tree_insert(0, [-1, -1, 0, 1, 1, 2], tokens=[5, 6, 7, 8, 9, 10])
        if s is other:
            s.stage_forward([0], [0], [6], x)
        else:
            s.append(0, [0], [0], [6], rnd(4, 6, 4, 32), rnd(5, 6, 288))
        pred = s.verify_head(head, [0], [0], [6], x)
        out = (torch.zeros(6, dtype=torch.int32, device="cuda"), None)
        s.verify_head(head, [0], [0], [6], x, noalloc=True, out=out)
        assert torch.equal(out[0], pred)
        s.set_root_pred(0, 6)
        s.tree_prune_verified([0], s.tree_match_dev([0]))
        got.append((pred.tolist(), s.request_info(0)[:2], s.tree_read(0)["token"].tolist(), s.verify_sample(head, [0], x[1:2], 0.7, 0.9, 20, [0.4])))
    assert got[0] == got[1] and got[1][1] == (31, 2)


# ---- a run of them ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("page", [0, 64])
def test_a_layer_against_keys_and_values_written_out(page):
    """Queries absorbed, appended, attended and brought to values: as attention over every head's own keys [W_k c | r] and values W_v c."""
    H, c, r, dn, dv, trees = 6, 512, 64, 128, 128, [(200, 9), (33, 4)]
    gain = (1 + 0.1 * torch.randn(c, generator=torch.Generator().manual_seed(3))).to(torch.bfloat16).cuda()
    rope = sp.Rope("interleaved", r, 10000.0)
    scale = (dn + r) ** -0.5
    st = make(H, c, r, trees, page=page, scale=scale, norms=[gain], rope=rope)
    w_k, w_v = rnd(1, H, dn, c, scale=c ** -0.5), rnd(2, H, dv, c, scale=c ** -0.5)
    M, n = 13, [9, 4]
    q, kv = rnd(3, M, H, dn + r), rnd(4, M, c + r)
    q_lat = torch.empty(M, H, c + r, dtype=torch.bfloat16, device="cuda")
    sp.head_product(q[..., :dn], w_k.transpose(1, 2).contiguous(), out=q_lat[..., :c])
    st.append(0, [0, 1], [0, 0], n, q[..., dn:], kv, q_lat[..., c:])
    out = sp.head_product(st.attention(0, [0, 1], [0, 0], n, q_lat), w_v)
    pos, at = positions(st), 0
    qr = torch.from_numpy(turn(f64(q[..., dn:]), pos, rope.freq, "interleaved")).cuda()
    for i, (P, T) in enumerate(trees):
        rows = st.kv_load(i, 0, 0, P + T).double()
        seen = seen_by(st, i)
        for h in range(H):
            k, v = rows[:, :c] @ w_k[h].double().T, rows[:, :c] @ w_v[h].double().T
            s = (q[at:at + T, h, :dn].double() @ k.T + qr[at:at + T, h] @ rows[:, c:].T) * scale
            p = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
            y = p @ v
            # Three roundings to bf16 lie between: of the absorbed query's columns (scores off by a step of |q_lat| |row|, and the
            # weights by as much of themselves, on top and in the sum), of the weights and the latent result (steps of what they
            # multiply in W_v), and of the result.  The same bounds as sums of magnitudes.
            ql = (q[at:at + T, h, :dn].double() @ w_k[h].double()).abs()
            ds = ((U * ql) @ rows[:, :c].abs().T + U * qr[at:at + T, h].abs() @ rows[:, c:].abs().T) * scale
            ds = 1.05 * ds.masked_fill(~seen, 0).amax(-1, keepdim=True) + 0.002
            lat = p @ rows[:, :c].abs()
            off = U * y.abs() + (2 * torch.expm1(ds) + 2.1 * U + 0.002) * (lat @ w_v[h].double().abs().T)
            err = (out[at:at + T, h].double() - y).abs()
            assert (err <= off).all()
            assert err.square().mean().sqrt() <= 0.02 * y.square().mean().sqrt()
        at += T


def test_captured_pieces_replay_with_the_values_of_the_time():
    use_own_stream()
    H, c, r = 16, 512, 64
    st = make(H, c, r, [(2000, 9)])
    q, kv = rnd(1, 9, H, c + r), rnd(2, 9, c + r)
    out = torch.zeros(9, H, c, dtype=torch.bfloat16, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        st.append(0, [0], [0], [9], q[..., c:], kv, q[..., c:])
        st.attention(0, [0], [0], [9], q, out)
    for k in range(3):
        q.copy_(rnd(20 + k, 9, H, c + r))
        kv.copy_(rnd(30 + k, 9, c + r))
        q2 = q.clone()
        g.replay()
        got = out.clone()
        st.append(0, [0], [0], [9], q2[..., c:], kv, q2[..., c:])
        assert torch.equal(st.attention(0, [0], [0], [9], q2), got)
        check_rows(got, q2, st.kv_load(0, 0, 0, 2009), c, seen_by(st, 0), (c // 4 + r) ** -0.5)


@pytest.mark.parametrize("page", [0, 64])
def test_requests_without_nodes_in_a_call(page):
    """They are passed over: the others' bits, cache rows and what counts as forwarded are those of a call without them."""
    trees = [(70, 3), (500, 4), (9, 2), (1300, 1)]
    got = []
    for ids in ([0, 1, 2, 3], [0, 2, 3]):
        st = make(16, 512, 64, trees, page=page, seed=3)
        n = [trees[i][1] if i != 1 else 0 for i in ids]
        q, kv = rnd(5, 6, 16, 576), rnd(6, 6, 576)
        st.append(0, ids, [0] * len(ids), n, q[..., 512:], kv, q[..., 512:])
        y = st.attention(0, ids, [0] * len(ids), n, q)
        got.append((q, y, torch.cat([st.kv_load(i, 0, 0, P + T) for i, (P, T) in enumerate(trees)])))
        assert [st.request_info(i)[2] for i in range(4)] == [3, 0, 2, 1]
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_two_stages_on_two_streams_and_repeated_calls():
    """Calls that overlap in time on stages of their own, and the same call over and over: equal bits."""
    sts = [make(16, 512, 64, [(6000, 3)], seed=s) for s in (1, 2)]
    qs = [rnd(s, 3, 16, 576) for s in (5, 6)]
    torch.cuda.synchronize()
    want = [st.attention(0, [0], [0], [3], q) for st, q in zip(sts, qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sts]
    outs = [[], []]
    for _ in range(10):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                outs[i].append(sts[i].attention(0, [0], [0], [3], qs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in outs[i])


# ---- refusals -----------------------------------------------------------------------------------------------------
def test_refusals_leave_the_stage_as_it_was():
    st = sp.LatentStage(2, 4, 256, 32, scale=0.1, kv_slots=256, max_requests=2, max_batch_nodes=8)
    st.request_init(0, 0, 128, 40)
    st.tree_insert(0, [-1, 0, 1, 2])
    q, kv, qr = rnd(1, 4, 4, 288), rnd(2, 4, 288), rnd(3, 4, 4, 32)
    for layer in (-1, 2):
        refused(-1, lambda: st.append(layer, [0], [0], [4], qr, kv))
        refused(-1, lambda: st.attention(layer, [0], [0], [4], q))
        refused(-1, lambda: st.kv_load(0, layer, 0, 2))
    refused(-4, lambda: st.attention(0, [1], [0], [4], q))
    refused(-5, lambda: st.attention(0, [0], [1], [4], q))
    refused(-1, lambda: st.attention(0, [0, 0], [0, 0], [2, 2], q))
    both = torch.zeros(4 * 4 * (288 + 256) - 64, dtype=torch.bfloat16, device="cuda")
    refused(-1, lambda: st.attention(0, [0], [0], [4], both[:4 * 4 * 288].view(4, 4, 288), both[-4 * 4 * 256:].view(4, 4, 256)))
    wide = rnd(4, 4, 4, 40)
    refused(-1, lambda: st.append(0, [0], [0], [4], wide[..., :32], kv, wide[..., 8:]))
    refused(-1, lambda: st.append(0, [0], [0], [4], qr, kv, kv[:, None, :128].unflatten(2, (4, 32))[:, 0]))
    refused(-9, lambda: st.append(0, [0], [0], [4], qr, kv, qr[:, :1].expand(4, 4, 32)))
    refused(-9, lambda: st.append(0, [0], [0], [4], rnd(1, 4, 4, 36)[..., :32], kv))
    refused(-2, lambda: st.kv_load(0, 0, 40, 5))
    refused(-1, lambda: st.kv_load(0, 0, -1, 2))
    refused(-4, lambda: st.kv_store(1, 0, 0, rnd(1, 2, 288)))
    refused(-9, lambda: st.stage_forward([0], [0], [4], rnd(1, 4, 256)))
    refused(-9, lambda: st.set_head_norms(None))
    refused(-9, lambda: sp.Stage.kv_load.__get__(_Plain(st))(0, 0, 0, 2))
    refused(-1, lambda: st.set_rope(sp.Rope("half", 64, 10000.0)))
    st.tree_insert(0, [-1] * 5)
    refused(-2, lambda: st.attention(0, [0], [0], [9], rnd(1, 9, 4, 288)))
    st.tree_prune(0, sp.SP_DROP, 4)
    refused(-7, lambda: st.append(0, [0], [0], [4], qr, kv))
    refused(-7, lambda: st.attention(0, [0], [0], [4], q))
    refused(-7, lambda: st.kv_load(0, 0, 0, 2))
    st.kv_compact(0)
    assert st.request_info(0) == (40, 8, 0)
    assert st.attention(0, [], [], [], q[:0]).shape == (0, 4, 256)
    assert st.append(0, [0], [3], [0], qr[:0], kv[:0]).shape == (0, 4, 32)


class _Plain:
    """A latent stage's handle where the calls of other stages take it."""

    def __init__(self, st):
        self.lib, self.handle, self.torch, self.tdtype, self.device, self._stream = st.lib, st.handle, st.torch, st.tdtype, st.device, st._stream
        self.shape = wl.ModelShape(2, 256, 4, 1, 288, 8, 1e-5, 10000.0, "bf16")


def test_calls_of_latent_stages_on_another():
    from fp4_reference import stage
    st = stage(sp, wl.ModelShape(1, 256, 4, 2, 128, 256, 1e-5, 500000.0, "bf16"), slots=128)
    st.request_init(0, 0, 64, 10)
    st.tree_insert(0, [-1])
    import ctypes as C
    one, zero = (C.c_int32 * 1)(1), (C.c_int32 * 1)(0)
    x = rnd(1, 64, 1024)
    p, lib = x.data_ptr(), st.lib
    at = C.addressof
    assert lib.sp_latent_store(st.handle, 0, 0, 0, 1, p, None) == -9 and lib.sp_latent_load(st.handle, 0, 0, 0, 1, p, None) == -9
    assert lib.sp_latent_append(st.handle, 0, 1, at(zero), at(zero), at(one), p, 0, 0, p, 0, p, 0, 0, None) == -9
    assert lib.sp_latent_attention(st.handle, 0, 1, at(zero), at(zero), at(one), p, p, None) == -9
