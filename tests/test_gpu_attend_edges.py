"""wf_attend where scores, weights and values are extreme, and where a row's positions are shared among the GPU's blocks."""
import numpy as np
import pytest

from gpu_util import lib
from test_gpu_attend import attend, check
from test_gpu_write import HALF_STEP, TYPES, Step, cache_of, f64, tensor

pytestmark = pytest.mark.gpu
EIGHT = pytest.mark.parametrize("eight", (False, True), ids=("16", "8"))


def layer_type(eight, dtype):
    return "float8_e4m3fn" if eight else dtype


@EIGHT
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scaling", (0.0, 2.0 ** -140, 1.0, 4.0))
@pytest.mark.parametrize("have,add", [([300, 17], [1, 1]), ([300, 17], [40, 300]), ([6000], [70])], ids=("few", "many", "split"))
def test_scales(have, add, scaling, dtype, eight):
    """Any scale >= 0; with 0 every output is the mean of the values that its token sees."""
    wf = lib()
    rng = np.random.default_rng(51)
    st = Step(wf, rng, have, add, 16, spare=3)
    cache, scale = cache_of(rng, st, 2, 64, layer_type(eight, dtype))
    q = tensor(rng, (st.room, 6, 64), dtype)
    check(st, cache, scale, q, attend(wf, st, cache, scale, q, scaling=scaling), scaling)
    check(st, cache, scale, q, attend(wf, st, cache, scale, q, scaling=scaling, new=1), scaling)


@pytest.mark.parametrize("bs,kv,dim", [(7, 2, 64), (100, 1, 128), (1, 2, 64), (30, 4, 128)])
def test_blocks_that_no_box_fits_again_and_again(bs, kv, dim):
    """Prompts over blocks whose positions are copied one by one (no multiple of 8): many tiles under way, every call the same."""
    import torch
    wf = lib()
    rng = np.random.default_rng(55)
    st = Step(wf, rng, [900, 0, 40], [200, 700, 65], bs)
    cache, _ = cache_of(rng, st, kv, dim, "bfloat16")
    q = tensor(rng, (st.room, 2 * kv, dim), "bfloat16")
    attn = wf.Attn(max_rows=3, heads=2 * kv, dim=dim)
    first = attend(wf, st, cache, None, q, attn=attn)
    check(st, cache, None, q, first)
    for _ in range(30):
        assert torch.equal(first, attend(wf, st, cache, None, q, attn=attn))
