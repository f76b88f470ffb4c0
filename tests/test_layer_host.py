"""Calls on a layer's tensors, without a GPU: refusals that come before any
device is touched, rates of rotary positions, and the plain implementations on cases
worked by hand."""
import ctypes
import math

import numpy as np
import pytest

import layer_ref as ref


@pytest.fixture(scope="module")
def wf():
    from paper_2609_03335_gb300 import build, wf
    build.build()
    wf.load_library()
    return wf


def test_calls_refuse_a_null_handle(wf):
    L = wf.load_library()
    assert L.wf_kv_write(None, None, None, None, None, None, None) == wf.WF_EINVAL
    assert L.wf_kv_copy_scales(None, None, None, None, 1, 0, 1, None) == wf.WF_EINVAL
    assert L.wf_attend(None, None, None, None, None, None) == wf.WF_EINVAL
    assert L.wf_attn_status(None, None) == wf.WF_EINVAL
    L.wf_attn_destroy(None)


def test_attn_create_refuses_sizes_out_of_range(wf):
    L, out = wf.load_library(), ctypes.c_void_p()
    for bad in ((0, 4, 64, 0), (65537, 4, 64, 0), (1, 0, 64, 0), (1, 1025, 64, 0), (1, 4, 96, 0), (1, 4, 64, 1)):
        assert L.wf_attn_create(ctypes.byref(wf.wf_attn_limits(*bad)), 0, ctypes.byref(out)) == wf.WF_EINVAL, bad
        assert wf.wf_last_error() and not out
    lim = wf.wf_attn_limits(1, 1, 64, 0)
    assert L.wf_attn_create(None, 0, ctypes.byref(out)) == wf.WF_EINVAL
    assert L.wf_attn_create(ctypes.byref(lim), 0, None) == wf.WF_EINVAL
    assert L.wf_attn_create(ctypes.byref(lim), -1, ctypes.byref(out)) == wf.WF_EINVAL


def test_turns_are_rates_in_whole_numbers(wf):
    """turn = f / 2 pi * 2^64 to one part in 2^64; scaled rates by their definition."""
    rp = wf.Rope(64, device="cpu")
    for i, (f, t) in enumerate(zip(rp.freq, rp.turn.tolist())):
        assert f == pytest.approx(10000.0 ** (-2 * i / 64), rel=1e-15)
        assert (t % 2 ** 64) / 2 ** 64 == pytest.approx(f / (2 * math.pi), rel=1e-15)
    assert wf.Rope(4, freq=[2 * math.pi * 0.75, -0.5], device="cpu").turn.tolist()[0] % 2 ** 64 == pytest.approx(0.75 * 2 ** 64, rel=1e-15)
    plain, far = wf.Rope(128, device="cpu"), wf.Rope(128, factor=8.0, context=4096, device="cpu")
    for f, g in zip(plain.freq, far.freq):
        turns = 4096 * f / (2 * math.pi)
        part = min(1.0, max(0.0, (turns - 1) / 31))
        assert g == pytest.approx(f * part + f / 8 * (1 - part), rel=1e-14)
    assert wf.Rope(8, factor=4.0, device="cpu").freq == [f / 4 for f in wf.Rope(8, device="cpu").freq]
    assert wf.Rope(0, device="cpu").freq == []


@pytest.mark.parametrize("args", [dict(dim=3), dict(dim=-2), dict(dim=130), dict(dim=4, base=0.0), dict(dim=4, factor=0.0), dict(dim=4, slow=5.0, fast=5.0),
                                  dict(dim=4, magnitude=math.inf), dict(dim=4, freq=[1.0]), dict(dim=4, freq=[1.0, math.nan]),
                                  dict(dim=4, context=-1)])
def test_rope_refuses(wf, args):
    with pytest.raises(wf.WfError):
        wf.Rope(device="cpu", **args)


def test_layer_refuses_what_is_not_on_the_device(wf):
    import torch
    with pytest.raises(wf.WfError):
        wf.KvLayer(torch.zeros((2, 4, 1, 64), dtype=torch.float16), torch.zeros((2, 4, 1, 64), dtype=torch.float16))
    with pytest.raises(wf.WfError):
        wf.KvLayer(None, None)


def test_plain_eight_bits_by_hand():
    x = [0.0, 1.0, 1.0625, 1.1875, 448.0, 449.0, 1e9, -np.inf, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11, 17.0, 19.0]
    assert ref.eight(x).tolist() == [0.0, 1.0, 1.0, 1.25, 448.0, 448.0, 448.0, -448.0, 2.0 ** -9, 0.0, 2.0 ** -8, 0.0, 16.0, 20.0]
    assert np.isnan(ref.eight(np.nan))
    assert ref.need([0.0]) == 2.0 ** -64 and ref.need([448.0, -1.0]) == 1.0 and ref.need([448.1, np.inf]) == 2.0 and ref.need([3e38]) == 2.0 ** 63


def test_plain_write_by_hand():
    # Blocks of 2: token 0 is appended to block 1, which holds one token at scale 1; tokens 1, 2 fill block 0.
    cache, scale = np.full((3, 2, 1, 1), 8.0), np.ones((3, 1))
    ref.write8(cache, scale, np.array([3, 0, 1, -1]), 2, np.array([448 * 16.0, 2.0, 1.0, 9.0])[:, None, None])
    assert scale[:, 0].tolist() == [2.0 ** -7, 16.0, 1.0]
    assert cache[:, :, 0, 0].tolist() == [[256.0, 128.0], [0.5, 448.0], [8.0, 8.0]]


def test_plain_rotation_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    half = ref.rotate(x, [1], [math.pi / 2, math.pi], False, 2.0)
    assert np.allclose(half, [[[-6.0, -4.0, 2.0, -8.0, 5.0]]])
    pairs = ref.rotate(x, [1], [math.pi / 2, math.pi], True, 1.0)
    assert np.allclose(pairs, [[[-2.0, 1.0, -3.0, -4.0, 5.0]]])


def test_plain_attention_by_hand():
    k = np.zeros((2, 2, 1, 1))
    v = np.array([[1.0, 2.0], [3.0, 5.0]]).reshape(2, 2, 1, 1)
    out = ref.attend(np.ones((3, 1, 1)), k, v, np.array([[1, 0], [0, 1]]), [0, 2, 2], [3, 0], 2, 1.0, np.full((3, 1, 1), 9.0))[0]
    assert np.allclose(out[:, 0, 0], [4.0, 3.0, 9.0])  # positions 0..1, then 0..2 of blocks 1, 0; the rest stays
