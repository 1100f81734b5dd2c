"""vp_reserve_new, vp_attend_new and vp_evict on a context of another device than
the current one."""

import ctypes

import pytest
import torch

from tests.test_new_tokens_gpu import Case

pytestmark = pytest.mark.gpu


def test_calls_need_the_contexts_device(lib):
    c = Case(lib, (8, 2), 64, "bf16", lens=(64,), n_new=2, weigh=True, seed=81)
    kept, new = (torch.full((2, 64), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    w = lib.token_weights(c.w_in)

    def calls():
        return [lambda: lib.vp_reserve_new(c.ctx, 2, 2), c.call,
                lambda: lib.vp_evict(c.ctx, 1, c.kc, c.vc, c.seq, lib.make_evict(32), c.kc, c.vc, w, w, kept, 32, new)]

    # The context's device number follows its configuration; with one GPU, another
    # number there stands for another current device.
    device = ctypes.c_int.from_address(c.ctx.value + ctypes.sizeof(lib.vp_config))
    here, device.value = device.value, device.value + 1
    assert here == torch.cuda.current_device()
    for call in calls():
        with pytest.raises(lib.VPError, match="device") as e:
            call()
        assert e.value.status == lib.VP_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert c.out.isnan().all() and (kept == -9).all()  # nothing was enqueued
    device.value = here
    for call in calls()[:2]:
        call()
    torch.cuda.synchronize()
    c.check()
    calls()[2]()
    lib.vp_check_errors(c.ctx)
    lib.vp_free(c.ctx)
