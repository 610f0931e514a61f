"""Calls of the 4-bit operators and of stages on them that the documentation allows, in forms that test_gpu_fp4.py does not make."""
import numpy as np
import pytest
import torch

import paper_2504_04104_amd as sp
from fp4_reference import stage
from test_gpu_fp4 import rnd, shape

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
