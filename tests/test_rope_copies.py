"""A rotation that is copied or pickled, as the settings of a model are, is one of its own: calls read the copy's frequencies."""
import copy
import ctypes as C
import pickle

import pytest

import paper_2504_04104_amd as sp
from paper_2504_04104_amd import binding


@pytest.mark.parametrize("make", [copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r)), lambda r: copy.deepcopy({"rope": r})["rope"]])
def test_copies(make):
    first = sp.Rope("interleaved", 64, 10000.0, ("linear", 4.0), gain=1.5)
    want = first.freq
    other = make(first)
    assert other.at == C.addressof(other.c) and first.at == C.addressof(first.c)
    seen = binding.sp_rope.from_address(other.at)                           # what a call is handed
    assert (seen.layout, seen.dims, seen.gain) == (1, 64, 1.5) and seen.freq[:32] == want == other.freq
    first.c.freq[0] = 7.0
    assert other.freq == want and binding.sp_rope.from_address(other.at).freq[0] == want[0]
