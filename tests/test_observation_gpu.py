"""vp_attend_new with 65 to 128 query rows per kv-head (an observation window, a
short chunk) and more (sequence, kv-head) items than CTAs, so that a CTA does
several of them: against the float64 definition, repeated bit for bit, and with
other calls on the same context after it.  Inputs, checks and tolerances are those
of test_new_tokens_gpu.py."""

import pytest
import torch

from tests.test_new_tokens_gpu import Case

pytestmark = pytest.mark.gpu


def _lengths(count, tiles):
    """Ragged lengths of the given tiles of 128 tokens, empty sequences last."""
    return tuple(128 * (tiles[i % len(tiles)] - 1) + 1 + 37 * i % 128 for i in range(count)) + (0, 0, 0)


@pytest.mark.parametrize("heads,dim,n_new", [((28, 4), 128, 16), ((16, 1), 128, 5), ((8, 2), 64, 32), ((6, 3), 64, 41)])
@pytest.mark.parametrize("count,tiles", [(90, (1,)), (90, (1, 2, 1, 3)), (45, (2, 1, 9, 1, 1)), (12, (1, 30))])
@pytest.mark.parametrize("weigh", [True, False])
def test_many_items_per_cta(lib, heads, dim, n_new, count, tiles, weigh):
    lens = _lengths(count * 4 // heads[1], tiles)
    c = Case(lib, heads, dim, "bf16", lens=lens, n_new=n_new, new_len=tuple(min(n_new, x) for x in lens), weigh=weigh,
             seed=31)
    c.call()
    torch.cuda.synchronize()
    c.check()
    first = c.out.clone(), c.lse.clone(), c.w_out.clone() if weigh else c.lse
    for _ in range(20):
        c.out.fill_(float("nan"))
        c.lse.fill_(float("nan"))
        c.call()
        assert torch.equal(c.out.view(torch.int16), first[0].view(torch.int16)) and torch.equal(c.lse, first[1])
        assert not weigh or torch.equal(c.w_out, first[2])
    # Other shapes on the same context find its tickets at 0: one token, and the
    # first three sequences alone (few items: CTAs of their own).
    one = torch.full_like(c.out[:, -1:], float("nan"))
    last = c.q[torch.arange(c.B), [max(n, 1) - 1 for n in c.ns]].unsqueeze(1).contiguous()
    for _ in range(2):
        lib.vp_attend_new(c.ctx, c.B, 1, lib.rows(last), c.kc, c.vc, c.seq, c.vis, lib.rows(one))
    c.out.fill_(float("nan"))
    lib.vp_attend_new(c.ctx, 3, n_new, lib.rows(c.q), c.kc, c.vc, c.seq, c.vis, lib.rows(c.out), new_len=c.new)
    torch.cuda.synchronize()
    lib.vp_check_errors(c.ctx)
    for b in range(c.B):
        n = c.ns[b]
        want = first[0][b, n - 1].float() if n else torch.zeros_like(one[b, 0], dtype=torch.float32)
        # The same sums in another order: one bf16 rounding of the output each way,
        # and well under 1e-3 from the two-term probabilities (2^-16 of |v| < 5).
        assert (one[b, 0].float() - want).abs().le(2.0 ** -7 * want.abs() + 1e-3).all()
        if b < 3:
            assert (c.out[b].float() - first[0][b].float()).abs().le(2.0 ** -7 * first[0][b].float().abs() + 1e-3).all()
    lib.vp_free(c.ctx)
