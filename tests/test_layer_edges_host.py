"""Refusals of the calls on a layer's tensors that come before any device is touched."""
import pytest


@pytest.fixture(scope="module")
def wf():
    from paper_2609_03335_gb300 import build, wf
    build.build()
    wf.load_library()
    return wf


def test_limits_of_waits_refuse_a_null_handle(wf):
    assert wf.load_library().wf_attn_limit_waits(None, 0) == wf.WF_EINVAL
