"""The example that goes from a plan to decoded tokens runs, and the cache holds what was decoded."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("window,beams,steps", [("tiny", 3, 20), ("mix", 4, 9)])
def test_decode_window(window, beams, steps):
    from gpu_util import lib
    lib()
    import decode_window as ex
    import wfgen
    prob = wfgen.config(window).problem
    device, batch = ex.first_batch(prob, n_plans=64)
    got = ex.decode(prob, device, batch, beams, steps)
    assert got["admitted"].any() and got["left"] == got["n_blocks"]
    # Sums of up to 4,096 + steps normal values in 32 bits, in two orders.
    assert got["error"] < 1e-4
    for ok, text in zip(got["admitted"], got["texts"]):
        assert len(text) == (steps if ok else 0) and all(0 < t < ex.VOCAB for t in text)
