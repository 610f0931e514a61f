"""What the binding of the 4-bit entry points checks before anything reaches a device."""
import contextlib
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2504_04104_amd as sp
import workloads as wl
from paper_2504_04104_amd import binding

SHAPE = wl.ModelShape(1, 256, 4, 2, 128, 512, 1e-5, 500000.0, "bf16")
SIZES = {"wqkv": (1024, 256), "wo": (256, 512), "wgu": (1024, 256), "wd": (256, 512)}


class OnDevice:
    """A host tensor that says it is on a device."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


def layer(**other):
    return {n: OnDevice(torch.zeros(other.get(n, s), dtype=torch.bfloat16)) for n, s in SIZES.items()}


@pytest.fixture
def packed(monkeypatch):
    """The calls of sp_fp4_pack_weights that would have been made."""
    lib, calls = sp.load_library(), []

    class Library:
        sp_fp4_matrix_bytes = lib.sp_fp4_matrix_bytes

        def sp_fp4_pack_weights(self, *args):
            calls.append(args)
            return 0
    monkeypatch.setattr(binding, "load_library", lambda: Library())
    monkeypatch.setattr(binding, "_raw_stream", lambda device: None)
    monkeypatch.setattr(torch.cuda, "device", lambda device: contextlib.nullcontext())
    return calls


@pytest.mark.parametrize("name", sorted(SIZES))
def test_weights_of_another_shape_than_the_models_are_not_packed(packed, name):
    rows, cols = SIZES[name]
    for size in ((rows - 16, cols), (rows + 16, cols), (rows, cols // 2), (cols, rows), (1, rows, cols), (rows * cols,)):
        if size == (rows, cols):
            continue
        with pytest.raises(AssertionError):
            sp.fp4_pack_weights(SHAPE, [layer(**{name: size})])
    assert not packed


def test_weights_of_the_models_shape_are_packed(packed):
    out = sp.fp4_pack_weights(SHAPE, [layer()])[0]
    assert len(packed) == 1
    for name, (rows, cols) in SIZES.items():
        assert (out[name].n_rows, out[name].n_cols) == (rows, cols) and out[name].data.numel() == rows * ((cols + 255) // 256) * 136


def test_a_matrix_holds_as_many_bytes_as_its_shape_takes():
    size = 3 * 2 * 2176                             # 48 x 288: strips of 16 rows, two units of 256 columns
    assert sp.Fp4Matrix(torch.zeros(size, dtype=torch.uint8), 48, 288).n_cols == 288
    for data in (torch.zeros(size - 1, dtype=torch.uint8), torch.zeros(size + 2176, dtype=torch.uint8), torch.zeros(size, dtype=torch.int8),
                 torch.zeros(2 * size, dtype=torch.uint8)[::2], torch.zeros(0, dtype=torch.uint8)):
        with pytest.raises(AssertionError):
            sp.Fp4Matrix(data, 48, 288)
    for rows, cols in ((17, 32), (0, 32), (16, 40), (1 << 18, 32)):
        with pytest.raises(sp.SpError) as err:
            sp.Fp4Matrix(torch.zeros(size, dtype=torch.uint8), rows, cols)
        assert err.value.status == -9


def test_a_call_without_requests_has_arrays_too():
    for empty in ([], (), np.zeros(0, np.int64)):
        a = binding._ids(empty)
        assert len(a) == 0 and binding._at(a) != 0


def test_host_arrays_are_cast_and_refused_as_those_of_the_forward_call():
    for given in ([3, 0, -1], (3, 0, -1), np.array([3, 0, -1], np.int64), [np.int64(3), False, -1], [3.0, 0.0, -1.0], torch.tensor([3, 0, -1]), range(3, 0, -1)):
        a, want = binding._ids(given), binding._i32(given)[0]
        assert list(a) == list(want)
        assert C.cast(binding._at(a), C.POINTER(C.c_int32))[:len(a)] == list(a)
    for refused in (b"\x00\x00\x00\x00", "ab", [None], [1 << 40], object()):
        errors = []
        for way in (binding._i32, binding._ids):
            with pytest.raises(Exception) as err:
                way(refused)
            errors.append(err.type)
        assert errors[0] is errors[1], refused
