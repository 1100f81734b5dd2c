"""bf16 prompts are as exact as their output's rounding, whether a row spreads its
weight or one token has nearly all of it.

Tolerance per element, from the arithmetic (u = 2^-24): logits and the exponential
a relative 2 D u max_j scale sum_d |q_d k_jd| + 2^-21 (1 + |lse|) + 2^-19 of sum_j
p_j |v_j|, probabilities as two bf16 terms 2^-16 of it, and the output's rounding
2^-8 |out|.  (Probabilities as one bf16 term would add 2^-8 of sum_j p_j |v_j|.)"""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("peaked", [False, True])
@pytest.mark.parametrize("heads,dim", [((8, 2), 128), ((2, 2), 64)])
@pytest.mark.parametrize("length,n_new,window", [(700, 300, -1), (2500, 512, -1), (6000, 700, -1), (9001, 300, 4096)])
def test_prompt_is_as_exact_as_its_rounding(lib, peaked, heads, dim, length, n_new, window):
    H, Hkv = heads
    gen = torch.Generator("cuda").manual_seed(91)
    q = torch.randn(1, n_new, H, dim, device="cuda", generator=gen)
    k, v = (torch.randn(1, Hkv, length, dim, device="cuda", generator=gen).bfloat16() for _ in range(2))
    if peaked:   # every query looks at one key that it sees
        lo = length - n_new if window < 0 else min(window, length) - 1
        at = torch.arange(length - n_new, length, device="cuda")[:, None] - torch.randint(
            0, lo, (n_new, H), device="cuda", generator=gen)
        for h in range(H):
            q[0, :, h] = 0.3 * q[0, :, h] + 2.2 * k[0, h * Hkv // H][at[:, h]].float()
    q = q.bfloat16()
    out = torch.full_like(q, float("nan"))
    lse = torch.empty(1, n_new, H, device="cuda")
    seq = torch.tensor([length], dtype=torch.int32, device="cuda")
    ctx = lib.vp_init(lib.make_config(1, H, Hkv, dim, 0, length, lib.VP_BF16))
    lib.vp_reserve_new(ctx, n_new)
    lib.vp_attend_new(ctx, 1, n_new, lib.rows(q), lib.kv_contiguous(k), lib.kv_contiguous(v), seq,
                      lib.make_visible(window), lib.rows(out), lse=lse)
    lib.vp_check_errors(ctx)
    lib.vp_free(ctx)
    pos, t = torch.arange(length, device="cuda"), torch.arange(length - n_new, length, device="cuda")[:, None]
    seen = (pos <= t) & ((pos > t - window) | (window < 0))
    top = 0.0
    for h in range(H):
        kk, vv = k[0, h * Hkv // H].double(), v[0, h * Hkv // H].double()
        qq = q[0, :, h].double()
        z = (qq @ kk.T / dim ** 0.5).masked_fill(~seen, -float("inf"))
        want_lse = torch.logsumexp(z, 1, keepdim=True)
        p = (z - want_lse).exp()
        top += float(p.amax(1).mean()) / H
        zmag = (qq.abs() @ kk.abs().T / dim ** 0.5).masked_fill(~seen, 0).amax(1, keepdim=True)
        rel = 2 * dim * 2.0 ** -24 * zmag + 2.0 ** -21 * (1 + want_lse.abs()) + 2.0 ** -19 + 2.0 ** -16
        want, most = p @ vv, p @ vv.abs()
        err = (out[0, :, h].double() - want).abs()
        assert (err <= rel * most + 2.0 ** -8 * want.abs()).all(), float((err - 2.0 ** -8 * want.abs()).div(most).max())
    assert (top > 0.9) == peaked
