"""Caches with one kv-head or one sequence whose stride along that axis is any
number (a [B, T, 1, D] or [T, Hkv, D] tensor seen as [B, Hkv, T, D]): the axis has
one element, so its stride says nothing about the room of the others."""

import pytest

from oracle import vp_oracle as O
from paper_2605_31457_gb300 import workloads as W
from tests import test_anchor_gpu as A
from tests import vp_harness as Hn
from tests.test_new_tokens_gpu import Case

pytestmark = pytest.mark.gpu


def _set(caches, stride_b=None, stride_h=None):
    """The strides of a cache's one-element axes, in rows of its token axis."""
    for x in caches:
        if stride_b is not None:
            x.stride_b = stride_b * x.stride_t
        if stride_h is not None:
            x.stride_h = stride_h * x.stride_t


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,dim,lens,strides", [
    ((8, 1), 128, (300, 129, 0, 1), dict(stride_h=1)),     # a [B, T, 1, D] tensor
    ((8, 1), 128, (300, 129, 0, 1), dict(stride_h=0)),
    ((4, 1), 64, (300, 250), dict(stride_h=3)),            # the sequences bound the tokens' room
    ((8, 2), 128, (513,), dict(stride_b=2)),               # the kv-heads do
    ((8, 2), 64, (513,), dict(stride_b=0)),
    ((4, 1), 64, (700,), dict(stride_b=1, stride_h=1)),    # nothing does
    ((4, 1), 64, (700,), dict(stride_b=0, stride_h=700)),
    ((4, 1), 128, (700,), dict(stride_b=700, stride_h=1))])
@pytest.mark.parametrize("n_new", [1, 12, 100])
def test_new_tokens(lib, dtype, heads, dim, lens, strides, n_new):
    c = Case(lib, heads, dim, dtype, lens=lens, n_new=n_new, new_len=tuple(min(n_new, x) for x in lens), window=90,
             sinks=2, seed=41)
    _set((c.kc, c.vc), **strides)
    c.run()


@pytest.mark.parametrize("n_new", [1, 100])
def test_new_tokens_token_outermost(lib, n_new):
    """One sequence in a [T, Hkv, D] tensor."""
    Case(lib, (8, 2), 128, "bf16", lens=(513,), n_new=n_new, layout="outer", seed=42).run()


@pytest.mark.parametrize("dtype,D", [(W.BF16, 128), (W.BF16, 64), (W.FP32, 128)])
@pytest.mark.parametrize("kv_heads,batch,layout,strides", [
    (1, 3, "bhtd", dict(stride_h=1)), (1, 2, "padded", dict(stride_h=0)), (4, 1, "tbhd", {}),
    (4, 1, "bhtd", dict(stride_b=1)), (1, 1, "bhtd", dict(stride_b=1, stride_h=1))])
def test_decode_step(lib, dtype, D, kv_heads, batch, layout, strides):
    r = A.small(dtype=dtype, head_dim=D, heads=7 * kv_heads, kv_heads=kv_heads, batch=batch, vis_len=(300, 577, 64)[:batch],
                vis_start=(0, 13, 40)[:batch], text_len=(517, 70, 129)[:batch])
    inp = Hn.make_inputs(r)
    dev = Hn.Device(lib, inp, r.budget, layout=layout)
    _set((dev.kc, dev.vc), **strides)
    try:
        gpu = dev.run()
    finally:
        dev.close()
    for b in range(batch):
        Hn.compare_seq(inp, gpu, b, r.budget)


@pytest.mark.parametrize("batch", [2, 3])
def test_decode_gather(lib, batch, monkeypatch):
    r = A.small(heads=7, kv_heads=1, batch=batch, vis_len=(300, 577, 64)[:batch], vis_start=(0, 13, 40)[:batch],
                text_len=(517, 70, 129)[:batch])
    device = Hn.Device

    def one_head(*a, **kw):
        dev = device(*a, **kw)
        _set((dev.kc, dev.vc), stride_h=1)
        return dev

    monkeypatch.setattr(Hn, "Device", one_head)
    inp, out, sets = A._run(lib, r, dict(mode=O.FIXED_RATIO, tau=0.1, ratio_ppm=200_000))
    A._check(inp, out, sets)
