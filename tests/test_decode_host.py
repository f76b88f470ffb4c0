"""Calls on a replica's rows, without a GPU: refusals that come before any
device is touched, and the plain implementations on cases worked by hand."""
import ctypes

import numpy as np
import pytest

import decode_ref as ref


@pytest.fixture(scope="module")
def wf():
    from paper_2609_03335_gb300 import build, wf
    build.build()
    wf.load_library()
    return wf


def test_create_refuses_sizes_out_of_range(wf):
    L, out = wf.load_library(), ctypes.c_void_p()
    for lim in ((0, 1, 0, 0), (65537, 1, 0, 0), (1, -1, 0, 0), (65536, 65536, 0, 0), (1, 0, -1, 0), (1, 0, (1 << 24) + 1, 1),
                (1, 0, 10, 65), (1, 0, 10, -1)):
        assert L.wf_decode_create(ctypes.byref(wf.wf_decode_limits(*lim)), 0, ctypes.byref(out)) == wf.WF_EINVAL, lim
        assert wf.wf_last_error() and not out
    lim = wf.wf_decode_limits(1, 1, 0, 0)
    assert L.wf_decode_create(None, 0, ctypes.byref(out)) == wf.WF_EINVAL
    assert L.wf_decode_create(ctypes.byref(lim), 0, None) == wf.WF_EINVAL
    assert L.wf_decode_create(ctypes.byref(lim), -1, ctypes.byref(out)) == wf.WF_EINVAL
    L.wf_decode_destroy(None)


def test_calls_refuse_a_null_handle(wf):
    L = wf.load_library()
    assert L.wf_kv_extend(None, None, None, None, None) == wf.WF_EINVAL
    assert L.wf_beam_select(None, None, None, None) == wf.WF_EINVAL
    assert L.wf_kv_reorder(None, None, 1, None, None, None, None, None, None) == wf.WF_EINVAL
    assert L.wf_decode_status(None, None) == wf.WF_EINVAL


def test_plain_extend_by_hand():
    # Block size 4: row 0 has 3 tokens (one block) and takes 2 (one new block); row 1 starts with 5 (two blocks); row 2
    # asks for more than its table row holds; row 3 would need a fourth free block; row 4 waits behind it.
    table = np.array([[7, -1, -1], [-1, -1, -1], [-1, -1, -1], [-1, -1, -1], [6, -1, -1]], np.int32)
    got = ref.extend(table, np.array([3, 0, 0, 0, 1], np.int32), np.array([2, 5, 13, 1, 1], np.int32),
                     np.array([9, 4, 5, 8, 1, 1, 1, 1, 1, 1], np.int32), np.array([11, 14]), 4, 9)
    assert got["table"][0].tolist() == [7, 4, -1] and got["table"][1].tolist() == [5, 8, -1]
    assert got["slot"].tolist() == [31, 16, 20, 21, 22, 23, 32, -1, -1]
    assert got["row"].tolist() == [0, 0, 1, 1, 1, 1, 1, -1, -1] and got["pos"].tolist() == [3, 4, 0, 1, 2, 3, 4, 0, 0]
    assert got["start"].tolist() == [0, 2, 7, 7, 7, 7] and got["len"].tolist() == [5, 5, 0, 0, 1]
    assert got["status"].tolist() == [0, 0, ref.LONG, ref.BLOCKS, ref.BLOCKS] and got["ends"].tolist() == [14, 14]


def test_plain_reorder_by_hand():
    # Block size 4, 6 tokens: rows share block 1; rows 1 and 2 follow old row 0, row 0 follows old row 2.
    table = np.array([[1, 2], [1, 3], [1, 4]], np.int32)
    cache = np.arange(8 * 4).reshape(1, 8, 4, 1)
    got = ref.reorder(table, np.array([6, 6, 6], np.int32), np.array([0, 5, 6, 7, 9, 9, 9, 9], np.int32), np.array([0, 4]),
                      4, 3, np.array([2, 0, 0]), table, cache)
    assert got["table"].tolist() == [[1, 4], [1, 2], [1, 3]]  # the freed block 3 takes the copy of block 2
    assert got["copies"].tolist() == [[-1, -1], [-1, -1], [2, 3]] and got["ends"].tolist() == [0, 4]
    assert got["cache"][0, 3, :, 0].tolist() == [8, 9, 14, 15]


def test_plain_sums_by_hand():
    x = np.array([[0.0, 0.0], [np.inf, np.inf], [-np.inf, 5.0], [np.nan, 1.0], [-np.inf, -np.inf]])
    c = ref.sums(x, np.array([0.0, -1.0, -2.0, 0.0, 0.0], np.float32))
    ln2 = np.log(2.0)
    assert np.allclose(c[0], -ln2) and np.allclose(c[1], -1 - ln2) and c[2].tolist() == [-np.inf, -2.0]
    assert c[3].tolist() == [-np.inf, 0.0] and (c[4] == -np.inf).all()
    assert ref.select(x[:2], np.zeros(2, np.float32), 2, 3) == [[(-ln2, 0, 0), (-ln2, 0, 1), (-ln2, 1, 0)]]
