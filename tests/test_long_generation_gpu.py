"""The operators together: examples/long_generation.py's layers against the
float64 definitions, and prompts long enough for one-term probabilities.

Tolerances (u = 2^-24): as in test_new_tokens_gpu.py for fp32.  bf16 prompt rows:
a probability and an output are each rounded to 8 bits, a relative 2^-8 at most,
so an output element errs by at most
  2^-8 sum_j p_j |v_j| + 2^-8 |out|   (+ the float32 terms, below 2^-14 of the first),
and, the roundings being independent and of mean zero, by no more in the root
mean square over all elements than
  2^-8 sqrt(mean(sum_j p_j^2 v_j^2) + mean(out^2)).
"""

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("heads,dim,n_new,length,window", [
    ((4, 2), 64, 2600, 2600, -1),     # rows that see few tokens and rows that see many
    ((4, 1), 128, 700, 5000, -1),     # a chunk behind a long cache
    ((2, 1), 128, 1000, 6001, 2500),  # a window wider than the bound
    ((2, 2), 64, 3100, 3100, 2048)])  # the bound itself
def test_long_prompts(lib, heads, dim, n_new, length, window):
    H, Hkv = heads
    gen = torch.Generator("cuda").manual_seed(21)
    q = torch.randn(1, n_new, H, dim, device="cuda", generator=gen).bfloat16()
    k, v = (torch.randn(1, Hkv, length, dim, device="cuda", generator=gen).bfloat16() for _ in range(2))
    out = torch.full_like(q, float("nan"))
    lse = torch.empty(1, n_new, H, device="cuda")
    seq = torch.tensor([length], dtype=torch.int32, device="cuda")
    ctx = lib.vp_init(lib.make_config(1, H, Hkv, dim, 0, length, lib.VP_BF16))
    lib.vp_reserve_new(ctx, n_new)
    lib.vp_attend_new(ctx, 1, n_new, lib.rows(q), lib.kv_contiguous(k), lib.kv_contiguous(v), seq,
                      lib.make_visible(window, 3), lib.rows(out), lse=lse)
    lib.vp_check_errors(ctx)
    lib.vp_free(ctx)
    mask = torch.from_numpy(O.seen_mask(length, n_new, window, 3)).cuda()
    err2 = noise2 = 0.0
    for h in range(H):
        kk, vv = k[0, h * Hkv // H].double(), v[0, h * Hkv // H].double()
        z = (q[0, :, h].double() @ kk.T / dim ** 0.5).masked_fill(~mask, -float("inf"))
        want_lse = torch.logsumexp(z, 1)
        p = (z - want_lse[:, None]).exp()
        want, most = p @ vv, p @ vv.abs()
        got = out[0, :, h].double()
        assert (got - want).abs().le(2.0 ** -8 * (1 + 2.0 ** -6) * (most + want.abs())).all()
        zmag = (q[0, :, h].double().abs() @ kk.abs().T).masked_fill(~mask, 0).amax(1) / dim ** 0.5
        assert (lse[0, :, h].double() - want_lse).abs().le(dim * U * zmag + 2.0 ** -21 * (1 + want_lse.abs())).all()
        err2 += float((got - want).square().sum())
        noise2 += float(((p * p) @ (vv * vv)).sum() + want.square().sum())
    assert err2 <= 2.0 ** -16 * noise2


def _close(got, q, k, v, length, n):
    r = O.attend_new(q.double().cpu().numpy(), k.double().cpu().numpy(), v.double().cpu().numpy(), length, n)
    ze = q.shape[2] * U * r["zmag"]
    rel = 2 * ze + 2.0 ** -21 * (1 + np.abs(r["lse"])) + 2.0 ** -19
    bad = np.abs(got.double().cpu().numpy() - r["out"]) > rel[..., None] * r["absout"]
    assert not bad.any()
    return r["weight"], float(rel.max())


@pytest.mark.parametrize("heads,dim", [((8, 2), 64), ((4, 1), 128)])
def test_full_layer_of_the_example(lib, heads, dim):
    """Prompt, observation window, steps and evictions, with every call's inputs
    read back; the kept sets from the library's own weights."""
    from examples.long_generation import FullLayer
    H, Hkv = heads
    B, prompt, high, keep, observe = 2, 50, 60, 40, 4
    gen = torch.Generator("cuda").manual_seed(22)

    def tokens(n):
        return (torch.randn(B, n, H, dim, device="cuda", generator=gen),
                torch.randn(B, Hkv, n, dim, device="cuda", generator=gen),
                torch.randn(B, Hkv, n, dim, device="cuda", generator=gen))

    layer = FullLayer(B, H, Hkv, dim, high + 1, torch.float32, prompt, high, keep, 2, 8, observe)
    t = tokens(prompt)
    out = layer.prompt(*t)
    weight = layer.weight.cpu().numpy()
    for b in range(B):
        _close(out[b], t[0][b], t[1][b], t[2][b], prompt, prompt)
        w, rel = _close(layer.attend(t[0][:, -observe:].contiguous())[b], t[0][b, -observe:], t[1][b], t[2][b], prompt,
                        observe)
        assert (np.abs(weight[b, :, :prompt] - w) <= (rel + 64 * U) * w + 1e-30).all()
        assert not weight[b, :, prompt:].any()
    evictions = 0
    for _ in range(45):
        q, k1, v1 = tokens(1)
        k, v, w = layer.k.clone(), layer.v.clone(), layer.weight.cpu().numpy()
        length = layer.longest
        out, evicted = layer.step(q, k1, v1)
        if evicted:
            evictions += 1
            kept = layer.kept.cpu().numpy()
            for b in range(B):
                for g in range(Hkv):
                    want = O.evict(w[b, g], length, keep, 2, 8)
                    np.testing.assert_array_equal(kept[b, g], want)
                    at = torch.from_numpy(want).cuda()
                    k[b, g, :keep], v[b, g, :keep] = k[b, g, at].clone(), v[b, g, at].clone()
                    w[b, g, :keep], w[b, g, keep:] = w[b, g, want].copy(), 0.0
            length = keep
        k[:, :, length], v[:, :, length] = k1[:, :, 0], v1[:, :, 0]
        assert torch.equal(k[:, :, :length + 1], layer.k[:, :, :length + 1])
        assert torch.equal(v[:, :, :length + 1], layer.v[:, :, :length + 1])
        assert layer.seq.tolist() == [length + 1] * B
        new = layer.weight.cpu().numpy()
        for b in range(B):
            add, rel = _close(out[b], q[b], k[b], v[b], length + 1, 1)
            want = w[b, :, :length + 1] + add
            assert (np.abs(new[b, :, :length + 1] - want) <= (rel + 64 * U) * add + 2 * U * want + 1e-30).all()
            assert not new[b, :, length + 1:].any()
    assert evictions >= 2
    layer.close()


def test_pruned_layer_of_the_example(lib):
    """The pruned step next to the full prompt: with a budget of every visual token
    it is the full attention of vp_attend_new."""
    from examples.long_generation import PrunedLayer
    B, H, Hkv, D, n_vis, prompt = 2, 8, 2, 64, 30, 45
    gen = torch.Generator("cuda").manual_seed(23)
    layer = PrunedLayer(B, H, Hkv, D, prompt + 3, torch.float32, prompt, n_vis)
    layer.budget = lib.make_budget(lib.VP_FIXED_RATIO, ratio_ppm=1_000_000)
    layer.cap = lib.vp_max_kept(layer.budget, n_vis)
    layer.kept = torch.empty(B, layer.cap, dtype=torch.int32, device="cuda")

    def tokens(n):
        return (torch.randn(B, n, H, D, device="cuda", generator=gen),
                torch.randn(B, Hkv, n, D, device="cuda", generator=gen),
                torch.randn(B, Hkv, n, D, device="cuda", generator=gen))

    t = tokens(prompt)
    out = layer.prompt(*t)
    for b in range(B):
        _close(out[b], t[0][b], t[1][b], t[2][b], prompt, prompt)
    for i in range(3):
        q, k, v = tokens(1)
        out = layer.step(q, k, v)
        assert layer.count.tolist() == [n_vis] * B
        full = layer.attend(q)
        for b in range(B):
            _close(full[b], q[b], layer.k[b], layer.v[b], prompt + 1 + i, 1)
        # two float32 results of the same sums: the step's tolerance is 1e-4 of them
        torch.testing.assert_close(out, full, rtol=0, atol=1e-4 * float(layer.v.abs().max()))
    layer.close()
