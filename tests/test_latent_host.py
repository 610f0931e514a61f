"""What the calls of latent stages, rotations and products per head refuse and say without touching a GPU."""
import ctypes as C

import numpy as np
import pytest

import paper_2504_04104_amd as sp
from paper_2504_04104_amd import binding
from latent_reference import frequencies

OK, INVALID, UNSUPPORTED = 0, -1, -9
P = [C.c_void_p((i + 1) << 32) for i in range(4)]                       # never read: every call below is refused first
ODD = C.c_void_p((1 << 32) + 8)


def sizes(c=512, r=64, heads=16, scale=0.1, dtype=binding.SP_BF16, flags=0, page=0, slots=2560, kv=1, d_head=None, layers=3, d_model=4096, norms=None):
    cfg = binding.sp_config(layers, d_model, heads, kv, c + r if d_head is None else d_head, 8, 1e-5, 10000.0, dtype, 2, 256, 64, slots, flags, page)
    lat = binding.sp_latent(c, r, scale, 0, norms)
    sz = binding.sp_sizes()
    return sp.load_library().sp_latent_query_sizes(C.byref(cfg), C.byref(lat), C.byref(sz)), sz


def test_sizes():
    rc, sz = sizes()
    assert rc == OK and sz.kv_row_bytes == 1152 and sz.kv_plane_bytes == 2560 * 1152 and sz.kv_bytes == 3 * 2560 * 1152
    assert sz.tables_bytes > 0 and sz.workspace_bytes > 0
    assert sizes(flags=sp.SP_FLAG_PAGED_KV, page=64)[0] == OK
    for bad in (dict(kv=2), dict(d_head=512), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(heads=0), dict(c=0),
                dict(r=0), dict(flags=sp.SP_FLAG_PAGED_KV, page=48), dict(flags=sp.SP_FLAG_PAGED_KV, page=64, slots=100), dict(dtype=7), dict(layers=0),
                dict(d_model=0), dict(slots=0), dict(norms=(C.c_void_p * 3)(4096, None, 4096)), dict(norms=(C.c_void_p * 3)(4096, 4100, 4096))):
        assert sizes(**bad)[0] == INVALID, bad
    for bad in (dict(dtype=binding.SP_F32), dict(c=260), dict(r=12), dict(c=1032), dict(r=136), dict(flags=sp.SP_FLAG_FP4_KV), dict(flags=sp.SP_FLAG_FP4_WEIGHTS),
                dict(flags=sp.SP_FLAG_PACKED_WEIGHTS), dict(d_model=12), dict(slots=1 << 31), dict(heads=1025)):
        assert sizes(**bad)[0] == UNSUPPORTED, bad
    lib = sp.load_library()
    assert lib.sp_latent_query_sizes(None, None, None) == INVALID
    assert lib.sp_latent_stage_create(None, None, None, None, None) == INVALID


@pytest.mark.parametrize("dims,theta", [(8, 10000.0), (64, 10000.0), (128, 500000.0), (256, 1000000.0), (24, 2.0)])
@pytest.mark.parametrize("scaling", [None, ("linear", 4.0), ("bands", 8.0, 8192.0, 1.0, 4.0), ("bands", 32.0, 100.0, 0.5, 0.75),
                                     ("ramp", 40.0, 4096.0, 32.0, 1.0), ("ramp", 2.0, 7.0, 4.0, 3.5)])
def test_frequencies(dims, theta, scaling):
    got = np.array(sp.Rope("half", dims, theta, scaling).freq)
    want = frequencies(dims, theta, scaling)
    # a few double roundings; a blend's weight is off by as many of the quotient it comes from, which is at most 1000 times as large
    assert np.allclose(got, want, rtol=1e-11, atol=0)
    if scaling is not None and scaling[0] != "linear":
        plain = frequencies(dims, theta)
        assert (got <= plain * (1 + 1e-12)).all() and (got >= plain / scaling[1] * (1 - 1e-12)).all()


def test_refused_frequencies():
    f = sp.load_library().sp_rope_frequencies
    out = (C.c_double * 128)()
    good = dict(dims=64, theta=1e4, scaling=2, factor=8.0, original=8192.0, first=1.0, second=4.0)
    assert f(*good.values(), out) == OK and f(*good.values(), None) == INVALID
    nan, inf = float("nan"), float("inf")
    for bad in (dict(dims=0), dict(dims=60), dict(dims=264), dict(dims=-8), dict(theta=1.0), dict(theta=nan), dict(theta=inf), dict(scaling=4), dict(scaling=-1), dict(factor=0.5),
                dict(factor=nan), dict(factor=inf), dict(original=0.0), dict(original=nan), dict(first=0.0), dict(first=4.0), dict(second=nan), dict(second=inf),
                dict(scaling=3), dict(scaling=3, first=4.0, second=4.0), dict(scaling=1, factor=0.0)):
        assert f(*{**good, **bad}.values(), out) == INVALID, bad
    assert f(*{**good, "scaling": 0, "factor": nan, "original": nan}.values(), out) == OK
    with pytest.raises(sp.SpError):
        sp.Rope("half", 64, freq=[1.0] * 31)
    with pytest.raises(ValueError):
        sp.Rope("half", 64, 1e4, ("bands", 8.0))
    with pytest.raises(KeyError):
        sp.Rope("halves", 64, 1e4)


def test_refused_rotations():
    lib = sp.load_library()
    good = dict(dtype=1, inverse=0, x=P[0], x_row=128, x_head=64, rows=4, heads=2, d=64, pos=P[1], out=P[2], out_row=128, out_head=64)

    def call(rope=None, **kw):
        r = rope or sp.Rope("half", 64, 1e4).c
        return lib.sp_rotate(C.byref(r), *{**good, **kw}.values(), None)
    for bad in (dict(dtype=2), dict(inverse=2), dict(x=None), dict(x=ODD), dict(rows=-1), dict(heads=0), dict(d=0), dict(pos=None), dict(pos=C.c_void_p(4098)), dict(out=None),
                dict(out=ODD), dict(out=P[0], out_row=256), dict(out=C.c_void_p(P[0].value + 128)), dict(pos=P[2]), dict(pos=C.c_void_p(P[2].value + 500))):
        assert call(**bad) == INVALID, bad
    for bad in (dict(d=68), dict(d=264), dict(heads=65537, x_head=0, out_head=64, out_row=65537 * 64), dict(x_row=-8), dict(x_head=4), dict(x_row=1 << 31), dict(out_row=64), dict(out_head=0), dict(out_head=32), dict(out_row=0),
                dict(out_row=100)):
        assert call(**bad) == UNSUPPORTED, bad
    assert lib.sp_rotate(None, *good.values(), None) == INVALID
    for change in (dict(layout=2), dict(layout=-1), dict(dims=72), dict(dims=4), dict(dims=0), dict(gain=float("nan")), dict(gain=float("inf"))):
        r = sp.Rope("half", 64, 1e4).c
        for k, v in change.items():
            setattr(r, k, v)
        assert call(rope=r) == INVALID, change
    r = sp.Rope("half", 64, 1e4).c
    r.freq[31] = float("inf")
    assert call(rope=r) == INVALID
    assert call(rows=0, x=None, out=None, pos=None) == OK
    assert lib.sp_stage_set_rope(None, None) == INVALID


def test_refused_products():
    lib = sp.load_library()
    good = dict(x=P[0], x_row=256, x_head=128, m=4, heads=2, w=P[1], n=512, k=128, out=P[2], out_row=1024, out_head=512)

    def call(**kw):
        return lib.sp_head_product(*{**good, **kw}.values(), None)
    for bad in (dict(x=None), dict(w=None), dict(out=None), dict(x=ODD), dict(w=ODD), dict(out=ODD), dict(m=-1), dict(heads=0), dict(n=0), dict(k=0), dict(out=P[0]), dict(out=P[1]),
                dict(out=C.c_void_p(P[0].value + 2 * (3 * 256 + 128 + 128) - 16)), dict(out=C.c_void_p(P[0].value - 2 * (3 * 1024 + 512 + 512) + 16))):
        assert call(**bad) == INVALID, bad
    for bad in (dict(n=24), dict(k=48), dict(n=4112), dict(k=4128), dict(heads=4097), dict(x_row=4), dict(x_head=-8), dict(out_row=512), dict(out_head=256), dict(out_head=0)):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(m=0, x=None, w=None, out=None) == OK


def test_calls_without_a_stage():
    lib = sp.load_library()
    one = (C.c_int32 * 1)(0)
    assert lib.sp_latent_store(None, 0, 0, 0, 1, P[0], None) == INVALID
    assert lib.sp_latent_load(None, 0, 0, 0, 1, P[0], None) == INVALID
    a = C.addressof(one)
    assert lib.sp_latent_append(None, 0, 1, a, a, a, P[0], 0, 0, P[0], 0, P[0], 0, 0, None) == INVALID
    assert lib.sp_latent_attention(None, 0, 1, a, a, a, P[0], P[0], None) == INVALID


def test_struct_layouts():
    assert C.sizeof(binding.sp_rope) == 16 + 8 * 128 and binding.sp_rope.freq.offset == 16
    assert C.sizeof(binding.sp_latent) == 24 and binding.sp_latent.norms.offset == 16


def test_stages_that_are_refused_before_the_device_is_asked():
    """Buffers too small or out of line, weights that are none: the same answers with and without a GPU."""
    lib = sp.load_library()
    out = C.c_void_p()
    cfg = binding.sp_config(1, 256, 4, 1, 576, 8, 1e-5, 10000.0, binding.SP_BF16, 1, 256, 16, 256, 0, 0)
    lat, sz = binding.sp_latent(512, 64, 0.1, 0, None), binding.sp_sizes()
    assert lib.sp_latent_query_sizes(C.byref(cfg), C.byref(lat), C.byref(sz)) == OK
    plain = binding.sp_config(1, 256, 2, 1, 128, 256, 1e-5, 10000.0, binding.SP_BF16, 1, 256, 16, 256, 0, 0)
    psz = binding.sp_sizes()
    assert lib.sp_stage_query_sizes(C.byref(plain), C.byref(psz)) == OK
    weights = (binding.sp_layer_weights * 1)()

    def create(latent, **kw):
        z = sz if latent else psz
        b = dict(kv=P[0], kv_bytes=z.kv_bytes, tables=P[1], tables_bytes=z.tables_bytes, workspace=P[2], workspace_bytes=z.workspace_bytes)
        bufs = binding.sp_buffers(*{**b, **kw}.values())
        if latent:
            return lib.sp_latent_stage_create(C.byref(cfg), C.byref(lat), C.byref(bufs), None, C.byref(out))
        return lib.sp_stage_create(C.byref(plain), weights, C.byref(bufs), None, C.byref(out))
    for latent in (True, False):
        for bad in (dict(kv=None), dict(tables=None), dict(workspace=None), dict(kv=ODD), dict(tables=ODD), dict(workspace=ODD)):
            assert create(latent, **bad) == INVALID, bad
        for bad in (dict(kv_bytes=8), dict(tables_bytes=8), dict(workspace_bytes=8)):
            assert create(latent, **bad) == -2, bad
    assert create(False) == INVALID                                     # (weights that are none)
    assert out.value is None
