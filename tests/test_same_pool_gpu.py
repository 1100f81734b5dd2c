"""vp_evict from some pages of a pool into others of the same pool."""

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,granularity", [(1, 1), (16, 0), (64, 1)])
def test_evict_into_fresh_pages_of_the_pool(lib, dtype, page, granularity):
    B, Hkv, T, D, keep, sinks, recent = 3, 2, 500, 64, 130, 3, 20
    lens = (500, 130, 257)
    rng = np.random.default_rng(51)
    src_pages, dst_pages = -(-T // page), -(-keep // page)
    ids = torch.from_numpy(rng.permutation(B * (src_pages + dst_pages)).astype(np.int32)).cuda()
    src, dst = (x.contiguous() for x in (ids[: B * src_pages].view(B, src_pages), ids[B * src_pages:].view(B, dst_pages)))
    kp, vp_ = (torch.from_numpy(rng.standard_normal((ids.numel(), Hkv, page, D))).to(dtype).cuda() for _ in range(2))
    k0, v0 = kp.clone(), vp_.clone()
    w = torch.from_numpy(rng.integers(0, 9, (B, Hkv, T)).astype(np.float32)).cuda()
    wd = torch.full((B, Hkv, keep), -3.0, device="cuda")
    kept = torch.full((B, Hkv if granularity else 1, keep), -9, dtype=torch.int32, device="cuda")
    seq, new = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    ctx = lib.vp_init(lib.make_config(B, 4, Hkv, D, 0, T, lib.VP_BF16 if dtype == torch.bfloat16 else lib.VP_FP32, 1, page))
    st = lib.vp_evict(ctx, B, lib.kv_paged(kp, src), lib.kv_paged(vp_, src), seq, lib.make_evict(keep, sinks, recent, granularity),
                      lib.kv_paged(kp, dst), lib.kv_paged(vp_, dst), lib.token_weights(w), lib.token_weights(wd), kept, keep,
                      new, check=False)
    assert st == lib.VP_OK, lib.vp_last_error(ctx)
    lib.vp_check_errors(ctx)

    def rows(pool, table, b, g, j):
        j = torch.from_numpy(np.asarray(j)).cuda()
        return pool[table[b].long()[j // page], g, j % page]

    for b, length in enumerate(lens):
        for g in range(Hkv):
            wsel = w[b, g] if granularity else w[b].sum(0)
            want = O.evict(wsel.cpu().numpy(), length, keep, sinks, recent)
            np.testing.assert_array_equal(kept[b, g if granularity else 0, : want.size].cpu().numpy(), want)
            at = np.arange(want.size)
            assert torch.equal(rows(kp, dst, b, g, at), rows(k0, src, b, g, want))
            assert torch.equal(rows(vp_, dst, b, g, at), rows(v0, src, b, g, want))
            assert torch.equal(wd[b, g, : want.size], w[b, g, torch.from_numpy(want).cuda()])
    assert torch.equal(kp[src.view(-1).long()], k0[src.view(-1).long()])  # the source pages are as they were
    assert torch.equal(vp_[src.view(-1).long()], v0[src.view(-1).long()])
    # One table for both, read another way, is no disjoint set of pages; nor is a contiguous cache inside the pool.
    half = lib.kv_paged(kp, src)
    half.max_pages -= 1
    flat = lib.kv_paged(kp, src)
    flat.block_table = None
    for kd in (half, flat):
        assert lib.vp_evict(ctx, B, lib.kv_paged(kp, src), lib.kv_paged(vp_, src), seq, lib.make_evict(keep, sinks, recent),
                            kd, lib.kv_paged(vp_, dst), lib.token_weights(w), lib.token_weights(wd), kept, keep, new,
                            check=False) == lib.VP_ERR_INVALID_ARG
    lib.vp_free(ctx)
