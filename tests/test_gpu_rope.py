"""Rotary positions against float64: rows of heads in every layout, a stage's rotation piece by piece and in forward calls.

u = 2^-8 is half a step of bf16 relative to the value, 2^-24 of float32.  On the way: the angle as a float (half a step of up to pi, 4 u of
float32), cosine and sine (two steps each), the gain, two products and a sum: 16 float32 steps of the pair's length are more."""
import numpy as np
import pytest
import torch

import workloads as wl
import paper_2504_04104_amd as sp
from fp4_reference import f64, stage
from gpu_harness import use_own_stream
from latent_reference import frequencies, pair_lengths, turn

pytestmark = pytest.mark.gpu
U, F = 2.0 ** -8, 2.0 ** -24
SCALINGS = [None, ("linear", 4.0), ("bands", 8.0, 8192.0, 1.0, 4.0), ("ramp", 16.0, 4096.0, 32.0, 1.0)]


def check(got, x, pos, rope, layout, gain, u, inverse=False):
    n = len(rope.freq)
    want = turn(x, pos, rope.freq, layout, gain, inverse)
    off = u * np.abs(want) + 16 * F * abs(gain) * pair_lengths(x, n, layout)
    passed = np.ones(x.shape[-1], bool)
    passed[:2 * n] = False
    assert np.array_equal(got[..., passed], x[..., passed])
    assert (np.abs(got - want) <= off).all(), np.max(np.abs(got - want) / (off + 1e-300))


def rows(seed, *size, dtype=torch.bfloat16):
    return torch.randn(*size, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,heads,d,dims", [(1, 1, 8, 8), (1, 32, 128, 128), (7, 3, 64, 64), (9, 5, 128, 64), (33, 2, 96, 24), (8, 1, 256, 256),
                                            (17, 4, 40, 8), (5, 8, 192, 64), (300, 1, 64, 32), (64, 128, 64, 64), (3, 7, 24, 16)])
def test_rows_of_any_shape(layout, dtype, n, heads, d, dims):
    x = rows(n + d, n, heads, d, dtype=dtype)
    pos = torch.from_numpy(np.random.default_rng(n).integers(0, 200000, n).astype(np.int32))
    rope = sp.Rope(layout, dims, 500000.0, SCALINGS[n % 4], gain=1.25)
    got = f64(sp.rotate(x, pos.cuda(), rope))
    check(got, f64(x), pos.numpy(), rope, layout, 1.25, U if dtype is torch.bfloat16 else F)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_views_in_place_and_positions_of_any_size(layout):
    big = rows(1, 40, 6, 192)
    x, keep = big[3:29, 1:5, 64:128], f64(big)
    pos = torch.tensor([0, 1, 2 ** 31 - 1, 2 ** 31 - 2, 10 ** 6, 131072] + list(range(20)), dtype=torch.int32).cuda()
    rope = sp.Rope(layout, 32, 10000.0)
    want = f64(x)
    out = torch.full((26, 4, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    sp.rotate(x, pos, rope, out=out[:, :, :64])
    check(f64(out)[:, :, :64], want, pos.cpu().numpy(), rope, layout, 1.0, U)
    assert (out[:, :, 64:] == 7).all()
    assert sp.rotate(x, pos, rope, out=x) is x
    assert torch.equal(x, out[:, :, :64])
    after = f64(big)
    after[3:29, 1:5, 64:128] = keep[3:29, 1:5, 64:128]
    assert np.array_equal(after, keep)
    head_major = torch.zeros(4, 26, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    assert torch.equal(sp.rotate(out[:, :, :64], pos, rope, out=head_major), sp.rotate(out[:, :, :64].contiguous(), pos, rope))
    one = rows(2, 1, 4, 64)
    spread = sp.rotate(one.expand(26, 4, 64), pos, rope)               # one row at many positions
    check(f64(spread), np.repeat(f64(one), 26, 0), pos.cpu().numpy(), rope, layout, 1.0, U)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_back_is_the_gradient(layout):
    """sum(w * rotate(x)) has the gradient rotate(w, back): by the formula's transpose and by differences, which are exact but for
    rounding, the rotation being linear."""
    n, heads, d, dims = 5, 3, 64, 48
    x, w = rows(1, n, heads, d, dtype=torch.float32), rows(2, n, heads, d, dtype=torch.float32)
    pos = torch.tensor([0, 3, 511, 70000, 12], dtype=torch.int32).cuda()
    rope = sp.Rope(layout, dims, 10000.0, SCALINGS[2], gain=1.5)
    back = f64(sp.rotate(w, pos, rope, inverse=True))
    check(back, f64(w), pos.cpu().numpy(), rope, layout, 1.5, F, inverse=True)
    for k in range(12):
        i = (k % n, k % heads, (k * 11) % d)
        step = torch.zeros_like(x)
        step[i] = 1.0
        diff = f64(sp.rotate(x + step, pos, rope)) - f64(sp.rotate(x - step, pos, rope))
        # x is off by two float32 steps of |x| + 1 <= 8, results by 17 of the pair's; w is at most 6
        assert abs((f64(w) * diff).sum() / 2 - back[i]) <= 2 * 6 * 2 * 20 * 8 * 1.5 * F


def test_a_captured_rotation_replays_at_the_positions_of_the_time():
    use_own_stream()
    x, pos, out = rows(1, 9, 4, 64), torch.arange(9, dtype=torch.int32).cuda(), rows(2, 9, 4, 64)
    rope = sp.Rope("half", 64, 10000.0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sp.rotate(x, pos, rope, out=out)
    for k in range(3):
        pos.add_(1000 * k + 1)
        x.mul_(0.5)
        g.replay()
        assert torch.equal(out, sp.rotate(x, pos, rope))


def test_rows_past_32_bits():
    n, heads, d = 2 ** 18 + 3, 64, 128                                  # 2^31 elements and more
    x = torch.zeros(n, heads, d, dtype=torch.bfloat16, device="cuda")
    x[-1] = rows(1, heads, d)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    rope = sp.Rope("interleaved", 128, 10000.0)
    y = sp.rotate(x, pos, rope)
    assert not y[:-1].any()
    check(f64(y[-1:]), f64(x[-1:]), [n - 1], rope, "interleaved", 1.0, U)


# ---- a stage's rotation ----------------------------------------------------------------------------------
SHAPES = {"bf16_128": ((8, 2, 128), "bf16", 0), "fp4_128": ((8, 2, 128), "bf16", sp.SP_FLAG_FP4_KV), "bf16_64": ((4, 4, 64), "bf16", 0),
          "f32_64": ((4, 2, 64), "f32", 0)}


@pytest.mark.parametrize("norms", [False, True])
@pytest.mark.parametrize("layout,part", [("half", 1), ("half", 2), ("interleaved", 1), ("interleaved", 4)])
@pytest.mark.parametrize("cache", sorted(SHAPES))
def test_appended_heads(cache, layout, part, norms):
    (nq, kv, dh), dtype, flags = SHAPES[cache]
    if flags and layout == "half" and dh // part % 64:
        pytest.skip("refused")
    sh = wl.ModelShape(1, 256, nq, kv, dh, 256, 1e-5, 500000.0, dtype)
    st = stage(sp, sh, slots=512, flags=flags, rows=64, norms=norms)
    st.request_init(0, 0, 200, 100)
    par = [-1, 0, 1, 1, 3]
    st.tree_insert(0, par)
    pos = [100, 101, 102, 102, 103]
    rope = sp.Rope(layout, dh // part, 10000.0, SCALINGS[3], gain=1.1)
    st.set_rope(rope)
    x = rows(5, 5, (nq + 2 * kv) * dh, dtype=st.tdtype)
    q = f64(st.append(0, [0], [0], [5], x)).reshape(5, nq, dh)
    h = f64(x).reshape(5, nq + 2 * kv, dh)
    hq, hk = h[:, :nq], h[:, nq:nq + kv]
    if norms:
        hq, hk = (t / np.sqrt((t * t).mean(-1, keepdims=True) + 1e-5) * f64(st.gains[0][n]) for t, n in ((hq, "q"), (hk, "k")))
    u = U if dtype == "bf16" else F
    k, v = (f64(t) for t in st.kv_load(0, 0, 100, 5))

    def near(got, t):
        want = turn(t, pos, rope.freq, layout, 1.1)
        big = np.abs(want) + 1.1 * pair_lengths(t, len(rope.freq), layout) + np.abs(t)
        return (np.abs(got - want) <= u * np.abs(want) + (32 + dh // 2) * F * big).all()
    assert near(q, hq)
    if flags:
        from fp4_reference import held
        from test_gpu_fp4 import check_held
        want = turn(hk, pos, rope.freq, layout, 1.1)
        check_held(k, want, (32 + dh // 2) * F * (np.abs(want) + 1.1 * pair_lengths(hk, len(rope.freq), layout)))
        assert np.array_equal(v, held(h[:, nq + kv:]))
    else:
        assert near(k, hk)
        assert np.array_equal(v, h[:, nq + kv:])
    st.set_rope(None)                                                   # as created
    q2 = f64(st.append(0, [0], [0], [5], x)).reshape(5, nq, dh)
    want = turn(hq, pos, frequencies(dh, 500000.0), "half")
    assert (np.abs(q2 - want) <= u * np.abs(want) + (32 + dh // 2) * F * (pair_lengths(hq, dh // 2, "half"))).all()


@pytest.mark.parametrize("dtype,n", [("bf16", 3), ("bf16", 40), ("bf16", 200), ("f32", 9)])
@pytest.mark.parametrize("kind", ["scaled", "part", "interleaved"])
def test_forward_rotates_as_the_pieces_do(dtype, n, kind):
    """One layer whose projections of the queries and keys are known: a forward call leaves the keys in the cache that an append of its
    QKV rows leaves (bf16: those rows rounded to bf16 first, the forward call's float32)."""
    use_own_stream()
    dh, nq, kv, d = (128, 4, 2, 512) if dtype == "bf16" else (64, 4, 2, 256)
    sh = wl.ModelShape(1, d, nq, kv, dh, 512, 1e-5, 500000.0, dtype)
    rope = {"scaled": sp.Rope("half", dh, 500000.0, SCALINGS[2], gain=0.9), "part": sp.Rope("half", dh // 2, 10000.0),
            "interleaved": sp.Rope("interleaved", dh, 10000.0, SCALINGS[1])}[kind]
    layout = "interleaved" if kind == "interleaved" else "half"
    st = stage(sp, sh, slots=1024, rows=256)
    st.request_init(0, 0, 900, 300)
    st.tree_insert(0, [-1] + list(range(n - 1)) if n < 50 else [-1] * n)
    pos = [300 + i if n < 50 else 300 for i in range(n)]
    w = st.plain_layers[0]
    x = rows(7, n, d, dtype=st.tdtype)
    for r in (None, rope):
        st.set_rope(r)
        st.stage_forward([0], [0], [n], x)
        k, _ = st.kv_load(0, 0, 300, n)
        xd = x.double()
        y = (xd * torch.rsqrt(xd.square().mean(-1, keepdim=True) + 1e-5) * w["norm1"].double())
        exact = f64((y @ w["wqkv"].double().T)[:, nq * dh:(nq + kv) * dh]).reshape(n, kv, dh)
        mag = f64(y.abs() @ w["wqkv"].double().abs().T)[:, nq * dh:(nq + kv) * dh].reshape(n, kv, dh)
        freq = frequencies(dh, 500000.0) if r is None else r.freq
        gain, lay = (1.0, "half") if r is None else (rope.c.gain, layout)
        want = turn(exact, pos, freq, lay, gain)
        u = U if dtype == "bf16" else F
        # the normed row rounded (a step of every product), float32 sums of d terms, the rotation, the result rounded
        off = (1.01 * u + (d + 64) * F) * (mag + 1.1 * pair_lengths(mag, len(freq), lay)) + u * np.abs(want)
        assert (np.abs(f64(k) - want) <= off).all()
        assert np.median(np.abs(f64(k) - want)) <= 4 * u * np.median(np.abs(want))


@pytest.mark.parametrize("n", [3, 40, 200])
@pytest.mark.parametrize("kind", ["part", "interleaved"])
def test_forward_into_a_cache_of_4_bits(n, kind):
    """Beside a bf16 cache's: the same float32 keys rounded to 4 bits and to bf16.  bf16's half step of 2^-9 of a value on average, and
    2^-8 at most, puts a value across a border between codes, which lie v / 4 apart or wider, for at most 2 * 2^-8 * 4 = 3.1 % of them, and a group's
    largest across a power of two for 2 * 2^-8 * 1.44 = 1.1 %."""
    from fp4_reference import held
    use_own_stream()
    sh = wl.ModelShape(1, 512, 4, 2, 128, 512, 1e-5, 500000.0, "bf16")
    rope = sp.Rope("half", 64, 10000.0) if kind == "part" else sp.Rope("interleaved", 128, 10000.0, SCALINGS[1])
    keys, layers = [], None
    for flags in (0, sp.SP_FLAG_FP4_KV):
        st = stage(sp, sh, slots=1024, rows=256, flags=flags, layers=layers)
        layers = st.plain_layers
        st.request_init(0, 0, 900, 300)
        st.tree_insert(0, [-1] * n)
        st.set_rope(rope)
        st.stage_forward([0], [0], [n], rows(7, n, 512))
        keys.append(f64(st.kv_load(0, 0, 300, n)[0]))
    assert (keys[1] == held(keys[0])).mean() >= 1 - 0.031 - 0.011


def test_replayed_forward_calls_take_a_new_rotation():
    """Layers enough that calls are replayed: a rotation that is set between them is that of the next call."""
    use_own_stream()
    sh = wl.ModelShape(6, 256, 2, 1, 128, 256, 1e-5, 500000.0, "bf16")
    layers = None
    outs = []
    ropes = [None, sp.Rope("half", 128, 500000.0, SCALINGS[1]), sp.Rope("interleaved", 64, 500000.0), None]
    x = rows(3, 20, 256)
    for fresh in (True, False):
        st = None
        got = []
        for r in ropes:
            if st is None or fresh:
                st = stage(sp, sh, slots=256, rows=64, layers=layers)
                layers = st.plain_layers
                st.kv.zero_()
                st.request_init(0, 0, 200, 50)
                st.tree_insert(0, [-1] + list(range(19)))
            st.set_rope(r)
            for _ in range(4):
                y = st.stage_forward([0], [0], [20], x)
                torch.cuda.synchronize()
            got.append(y)
        outs.append(got)
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert not torch.equal(outs[0][0], outs[0][1]) and not torch.equal(outs[0][1], outs[0][2])


def test_refusals():
    x, pos = rows(1, 4, 2, 64), torch.zeros(4, dtype=torch.int32).cuda()
    rope = sp.Rope("half", 64, 10000.0)

    def refused(status, call):
        with pytest.raises(sp.SpError) as err:
            call()
        assert err.value.status == status
    refused(-1, lambda: sp.rotate(x[..., :32].contiguous(), pos, rope))                     # more pairs than columns
    buf = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    refused(-1, lambda: sp.rotate(buf[:4], pos, rope, out=buf[1:]))
    refused(-9, lambda: sp.rotate(x, pos, rope, out=torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda").expand(4, 2, 64)))
    odd = torch.zeros(4, 2, 68, dtype=torch.bfloat16, device="cuda")
    refused(-9, lambda: sp.rotate(odd[..., :64], pos, rope))
    sh = wl.ModelShape(1, 256, 4, 2, 128, 256, 1e-5, 500000.0, "bf16")
    st = stage(sp, sh, slots=64, flags=sp.SP_FLAG_FP4_KV)
    refused(-9, lambda: st.set_rope(sp.Rope("half", 32, 10000.0)))
    refused(-1, lambda: st.set_rope(sp.Rope("half", 256, 10000.0)))
    assert sp.rotate(x[:0], pos[:0], rope).shape == (0, 2, 64)


def test_more_rows_than_a_launch_takes():
    """The rows behind the 2^23rd, in either layout and with a head of its own stride, as a call of them alone turns them."""
    n, tail = 2 ** 23 + 77, 100
    x = torch.zeros(n, 1, 16, dtype=torch.bfloat16, device="cuda")
    x[-tail:] = rows(3, tail, 1, 16)
    x[:50] = x[-50:]
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    for layout in ("half", "interleaved"):
        rope = sp.Rope(layout, 8, 10000.0)
        got = sp.rotate(x, pos, rope)
        assert torch.equal(got[-tail:], sp.rotate(x[-tail:].contiguous(), pos[-tail:].contiguous(), rope))
        assert torch.equal(got[:50], sp.rotate(x[:50].contiguous(), pos[:50].contiguous(), rope))
        assert not got[50:-tail].any()


@pytest.mark.parametrize("heads", [1, 4, 8, 31, 32, 33, 64])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_share_a_workgroup(heads, dtype):
    """Whatever the number of rows that a workgroup takes: a call of many rows has the bits of calls of one."""
    x = rows(heads, 19, heads, 128, dtype=dtype)
    pos = torch.arange(19, dtype=torch.int32, device="cuda") * 1777
    rope = sp.Rope("interleaved", 64, 10000.0)
    got = sp.rotate(x, pos, rope)
    for i in range(19):
        assert torch.equal(got[i:i + 1], sp.rotate(x[i:i + 1], pos[i:i + 1], rope))
