"""What vp_reserve_new, vp_attend_new and vp_evict accept and refuse, beyond
test_new_tokens_gpu.py."""

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_evict_in_place_needs_the_weights_in_place(lib):
    """In place, weights that go elsewhere are refused whatever their strides: a
    compact [B, Hkv, keep] array has no room for the entries that are cleared."""
    B, Hkv, T, keep = 2, 2, 64, 16
    k = torch.zeros(B, Hkv, T, 64, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    w = torch.rand(B, Hkv, T, device="cuda")
    seq = torch.tensor([64, 10], dtype=torch.int32, device="cuda")
    kept = torch.full((B, Hkv, keep), -9, dtype=torch.int32, device="cuda")
    ctx = lib.vp_init(lib.make_config(B, 8, Hkv, 64, 0, T, lib.VP_BF16))
    kc, vc, ws = lib.kv_contiguous(k), lib.kv_contiguous(v), lib.token_weights(w)

    def call(kd, vd, wd):
        return lib.vp_evict(ctx, B, kc, vc, seq, lib.make_evict(keep, 2, 4), kd, vd, ws, wd, kept, keep, seq.clone(),
                            check=False), lib.vp_last_error(ctx)

    compact = torch.full((B, Hkv, keep), -3.0, device="cuda")
    roomy = torch.full((B, Hkv, T), -3.0, device="cuda")
    shifted = lib.token_weights(w)
    shifted.stride_b = 0
    for wd in (lib.token_weights(compact), lib.token_weights(roomy), shifted):
        st, why = call(kc, vc, wd)
        assert st == lib.VP_ERR_INVALID_ARG and "weight_dst" in why
    # Out of place: the source's own array is refused, with its strides or others.
    kd, vd = torch.zeros_like(k[:, :, :keep]), torch.zeros_like(v[:, :, :keep])
    for wd in (ws, shifted):
        st, why = call(lib.kv_contiguous(kd), lib.kv_contiguous(vd), wd)
        assert st == lib.VP_ERR_INVALID_ARG and "weight_dst" in why
    torch.cuda.synchronize()
    assert (kept == -9).all() and (compact == -3.0).all() and (roomy == -3.0).all()  # nothing was enqueued
    assert call(lib.kv_contiguous(kd), lib.kv_contiguous(vd), lib.token_weights(compact))[0] == lib.VP_OK
    assert call(kc, vc, ws)[0] == lib.VP_OK and call(kc, vc, None)[0] == lib.VP_OK
    lib.vp_check_errors(ctx)
    lib.vp_free(ctx)
