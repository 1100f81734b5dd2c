"""Caches whose rows lie further apart than 32 bits reach: over sequences, pages,
heads and tokens.  vp_append, vp_append4 and vp_attend4 on them do what they do on
dense ones, bit for bit."""

import pytest
import torch

from tests.test_append_gpu import Append
from tests.test_attend4_gpu import Case

pytestmark = pytest.mark.gpu
FAR = 5 << 30  # bytes between the first and the last index of the axis


@pytest.fixture(scope="module")
def vp(lib):
    assert torch.cuda.is_available()
    return lib


def _far(x, axis):
    """x with its axis spread over more than 2^32 bytes."""
    step = -(-FAR // x.element_size() // max(1, x.shape[axis] - 1)) // 1024 * 1024 + 1024
    strides, size = [0] * 4, 1
    for a in (3, 2, 1, 0):
        if a != axis:
            strides[a] = size
            size *= x.shape[a]
    assert size <= step
    strides[axis] = step
    y = torch.empty(step * (x.shape[axis] - 1) + size, dtype=x.dtype, device="cuda").as_strided(x.shape, strides)
    y.copy_(x)
    return y


@pytest.mark.parametrize("page,axis", [(0, 0), (0, 1), (0, 2), (16, 0), (16, 1), (16, 2)])
@pytest.mark.parametrize("n_new", [1, 40])
def test_attention(vp, page, axis, n_new):
    a = Case(vp, (8, 2), 64, "bf16", lens=(200, 129), n_new=n_new, page=page)
    a.call()
    torch.cuda.synchronize()
    out, lse = a.out.clone(), a.lse.clone()
    far = [_far(t, axis) for t in a.tensors]
    make = (lambda c, s: vp.kv4_paged(c, s, a.table)) if page else vp.kv4_contiguous
    a.kc, a.vc = make(*far[:2]), make(*far[2:])
    a.out.fill_(float("nan"))
    a.call()
    torch.cuda.synchronize()
    assert torch.equal(a.out, out) and torch.equal(a.lse, lse)
    a.check()
    vp.vp_free(a.ctx)


@pytest.mark.parametrize("four", [False, True], ids=["plain", "four"])
@pytest.mark.parametrize("page,axis", [(0, 0), (0, 1), (0, 2), (16, 0), (16, 2)])
def test_appending(vp, four, page, axis):
    a = Append(vp, (4, 2), 64, "bf16", lens=(200, 129), n_new=3, page=page, four=four)
    far = [tuple(_far(t, axis) for t in c) for c in a.caches]
    if four:
        make = (lambda c: vp.kv4_paged(*c, a.table_of_pages)) if page else (lambda c: vp.kv4_contiguous(*c))
    else:
        make = (lambda c: vp.kv_paged(*c, a.table_of_pages)) if page else (lambda c: vp.kv_contiguous(*c))
    a.caches = far
    a.kc, a.vc = (make(c) for c in far)
    a.run()


@pytest.mark.parametrize("n_new", [1, 5, 40])
def test_tables_of_their_own(vp, n_new):
    """Values on other pages than their keys, and a table that is wider than the sequences need."""
    a = Case(vp, (8, 2), 64, "bf16", lens=(200, 129), n_new=n_new, page=16)
    a.call()
    torch.cuda.synchronize()
    out = a.out.clone()
    pages = a.tensors[2].shape[0]
    to = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).cuda()
    codes, scales = torch.empty_like(a.tensors[2]), torch.empty_like(a.tensors[3])
    codes[to], scales[to] = a.tensors[2], a.tensors[3]
    table = torch.where(a.table >= 0, to[a.table.clamp(min=0).long()].int(), -1)
    table = torch.cat([table, torch.full_like(table, 10 ** 6)], 1).contiguous()
    a.vc = vp.kv4_paged(codes, scales, table)
    a.out.fill_(float("nan"))
    a.call()
    torch.cuda.synchronize()
    assert torch.equal(a.out, out)
    a.check()
    vp.vp_free(a.ctx)
