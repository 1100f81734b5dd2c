"""vp_append and vp_append4 of many tokens at once in both types, and positions on
several axes for heads of 128: bit for bit, as in test_append_gpu."""

import pytest
import torch

from tests.test_append_gpu import BOTH, TYPES, Append

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vp(lib):
    assert torch.cuda.is_available()
    return lib


@BOTH
@TYPES
@pytest.mark.parametrize("heads,dim,rot", [((28, 4), 128, 128), ((32, 8), 128, 64), ((8, 2), 64, 32), ((5, 5), 64, 64)])
@pytest.mark.parametrize("page", [0, 16])
def test_prompts(vp, four, dtype, heads, dim, rot, page):
    """More tokens than warps that are launched at once, and fewer; a sequence that had tokens before."""
    Append(vp, heads, dim, dtype, lens=(1027, 1500, 0), n_new=1027, new_len=(1027, 333, 0), rot=rot, page=page,
           interleaved=rot < dim, four=four).run()


@BOTH
@TYPES
@pytest.mark.parametrize("batch,n_new", [(1, 2433), (3, 811), (1, 1217), (1, 609), (2433, 1)])
def test_edges_of_the_warps_share(vp, four, dtype, batch, n_new):
    """One token more than a warp, two or four of each SM's sixteen take."""
    Append(vp, (8, 2), 64, dtype, lens=(n_new,) * batch, n_new=n_new, four=four).run()


@BOTH
@TYPES
@pytest.mark.parametrize("axes,sections", [(2, [10, 54]), (3, [16, 24, 24]), (3, [17, 23, 24]), (3, [0, 63, 1]), (3, [1, 0, 63])])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "pairs"])
def test_positions_on_axes_of_wide_heads(vp, four, dtype, axes, sections, interleaved):
    Append(vp, (28, 4), 128, dtype, lens=(50, 61), n_new=7, axes=axes, sections=sections, interleaved=interleaved,
           four=four).run()
