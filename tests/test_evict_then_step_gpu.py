"""Calls of one stream behind each other with no synchronisation between them."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("page", [0, 16])
def test_evict_then_decode_step(lib, in_place, page):
    """vp_decode_step reads its caches, lengths and page table before it waits for
    the call in front of it; vp_evict has completed by then.  Bits as with a
    synchronisation between the two."""
    B, H, Hkv, D, T, keep, nv = 8, 28, 4, 128, 6000, 3000, 256
    gen = torch.Generator("cuda").manual_seed(71)
    k0, v0 = (torch.randn(B, Hkv, T, D, device="cuda", generator=gen).bfloat16() for _ in range(2))
    q = torch.randn(B, H, D, device="cuda", generator=gen).bfloat16()
    w0 = torch.rand(B, Hkv, T, device="cuda", generator=gen)
    w0[:, :, :nv] = 2.0  # the visual tokens at the front stay
    lens = torch.full((B,), T, dtype=torch.int32, device="cuda")
    vs, vl = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), nv, dtype=torch.int32, device="cuda")
    text = torch.full((B,), keep - nv, dtype=torch.int32, device="cuda")
    ctx = lib.vp_init(lib.make_config(B, H, Hkv, D, nv, T, lib.VP_BF16, 1 if page else 0, page or 16))
    budget = lib.make_budget(lib.VP_ADAPTIVE, tau=0.1)
    cap = lib.vp_max_kept(budget, nv)

    def cache(x, rows):
        if not page:
            return x, None
        pages = -(-rows // page)
        y = x.view(B, Hkv, pages, page, D).transpose(1, 2).reshape(B * pages, Hkv, page, D).contiguous()
        return y, torch.arange(B * pages, dtype=torch.int32, device="cuda").view(B, pages).flip(1).contiguous()

    def kv(x):
        return lib.kv_paged(*x) if page else lib.kv_contiguous(x[0])

    results = []
    rows = T if in_place else -(-keep // 16) * 16
    for sync in (True, False, False, False):
        k, v = cache(k0.clone(), T), cache(v0.clone(), T)
        dst = (k, v) if in_place else tuple(cache(torch.zeros(B, Hkv, rows, D, dtype=k0.dtype, device="cuda"), rows)
                                            for _ in range(2))
        w = w0.clone()
        out = torch.full((B, H, D), float("nan"), dtype=q.dtype, device="cuda")
        kept = torch.full((B, Hkv, keep), -7, dtype=torch.int32, device="cuda")
        kept2 = torch.full((B, cap), -7, dtype=torch.int32, device="cuda")
        count, new = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
        mass = torch.zeros(B, H, device="cuda")
        span = lib.span(vs, vl)
        step_cfg = kv(dst[0]), kv(dst[1])
        torch.cuda.synchronize()
        lib.vp_evict(ctx, B, kv(k), kv(v), lens, lib.make_evict(keep, 4, 64), *step_cfg, lib.token_weights(w),
                     lib.token_weights(w) if in_place else None, kept, keep, new)
        if sync:
            torch.cuda.synchronize()
        lib.vp_decode_step(ctx, B, q, *step_cfg, span, text, budget, out, kept2, cap, count, mass)
        torch.cuda.synchronize()
        lib.vp_check_errors(ctx)
        assert new.tolist() == [keep] * B
        results.append((out.view(torch.int16), kept2, count, mass))
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, results[0]))
    lib.vp_free(ctx)
