"""A logit that is not a number makes its row's log-sum-exp, output and weights
not a number; it must not look like a row that sees nothing (lse = -infinity)."""

import pytest
import torch

from tests.test_new_tokens_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,n_new", [((8, 2), 1), ((8, 2), 6), ((8, 2), 20), ((8, 2), 90)])
@pytest.mark.parametrize("length", [40, 1500])
def test_nan_in_a_query_and_in_a_key(lib, dtype, heads, n_new, length):
    n_new = min(n_new, length - 5)
    weigh = n_new * 4 <= 128
    for what in ("query", "key"):
        c = Case(lib, heads, 64, dtype, lens=(length, length), n_new=n_new, weigh=weigh, seed=61)
        # Sequence 0 has the NaN, in the last token: only its row (query) or that token's own position (key) sees it.
        if what == "query":
            c.q[0, -1, 5] = float("nan")
        else:
            c.kt[0, 1, length - 1] = float("nan")
        c.call()
        torch.cuda.synchronize()
        hit = torch.zeros(2, n_new, heads[0], dtype=torch.bool)
        if what == "query":
            hit[0, -1, 5] = True
        else:
            hit[0, -1, 4:] = True
        assert torch.equal(c.lse.isnan().cpu(), hit)
        assert torch.equal(c.out.isnan().all(-1).cpu(), hit) and torch.equal(c.out.isnan().any(-1).cpu(), hit)
        if weigh:
            assert c.w_out[0, 1, :length].isnan().all() and not c.w_out[0, 0].isnan().any()
            assert not c.w_out[1].isnan().any()
        lib.vp_check_errors(c.ctx)
        lib.vp_free(c.ctx)
