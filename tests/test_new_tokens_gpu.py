"""vp_attend_new and vp_evict against the float64 definitions.

Tolerances, per element, from the arithmetic (u = 2^-24, float32):
  logits   z_err = D u max_j scale sum_d |q_d k_jd|: the bound of a D-term
           float32 sum, plus 2^-21 (1 + |lse|) for the scaled exponent;
  lse      z_err + 2^-21 (1 + |lse|);
  weights  a relative 2 z_err + 2^-19 of the received weight (logit and lse
           errors, the exponential), plus u of the sum with the old value;
  out      a relative 2 z_err + 2^-19 of sum_j p_j |v_j|; bf16: also 2^-9 of it
           for the probabilities' rounding and 2^-9 |out| for the output's.
Whole numbers and moved rows are equal bit for bit.
"""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _lay(x, layout):
    """x [B, n, H, D] or [B, Hkv, T, D] on the device in another memory order."""
    if layout == "dense":
        return x.contiguous()
    if layout == "swapped":   # axes 1 and 2 exchanged in memory
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "outer":     # axis 2 outermost in memory
        return x.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    pad = 16 // x.element_size()   # rows padded by 16 bytes
    y = torch.full((*x.shape[:3], x.shape[3] + pad), float("nan"), dtype=x.dtype, device=x.device)
    y[..., : x.shape[3]] = x
    return y[..., : x.shape[3]]


class Case:
    def __init__(self, vp, heads=(8, 2), dim=64, dtype="fp32", lens=(33,), n_new=1, new_len=None, window=-1, sinks=0,
                 scale=0.0, page=0, layout="dense", weigh=False, w_in=True, max_seq=None, seed=0, poison=True,
                 spread=1.0):
        rng = np.random.default_rng(seed)
        self.vp, self.lens, self.n_new = vp, lens, n_new
        H, Hkv = heads
        B, T = len(lens), max(max(lens), 1)
        T = max_seq or T
        dt = torch.float32 if dtype == "fp32" else torch.bfloat16
        dev = "cuda"
        self.ns = [min(n_new, L) if new_len is None else new_len[b] for b, L in enumerate(lens)]
        q = torch.from_numpy(rng.standard_normal((B, n_new, H, dim)) * spread).to(dt)
        k = torch.from_numpy(rng.standard_normal((B, Hkv, T, dim))).to(dt)
        v = torch.from_numpy(rng.standard_normal((B, Hkv, T, dim))).to(dt)
        win = torch.from_numpy(rng.random((B, Hkv, T)).astype(np.float32))
        self.ref = [O.attend_new(q[b].double().numpy(), k[b].double().numpy(), v[b].double().numpy(), lens[b],
                                 self.ns[b], window, sinks, scale or None) for b in range(B)]
        seen = np.zeros((B, T), bool)
        for b in range(B):
            if self.ns[b]:
                seen[b, : lens[b]] = self.ref[b]["mask"].any(0)
        if poison:  # rows that no new token sees, and padding queries, hold NaN
            k[torch.from_numpy(~seen)[:, None, :, None].expand_as(k)] = float("nan")
            v[torch.from_numpy(~seen)[:, None, :, None].expand_as(v)] = float("nan")
            for b in range(B):
                q[b, self.ns[b]:] = float("nan")
        self.w_old = win.numpy() if w_in else np.zeros_like(win.numpy())
        self.q = _lay(q.to(dev), layout if layout != "outer" else "dense")
        self.out = _lay(torch.full((B, n_new, H, dim), float("nan"), dtype=dt, device=dev),
                        layout if layout != "outer" else "dense")
        self.lse = torch.full((B, n_new, H), float("nan"), device=dev)
        self.w_out = torch.full((B, Hkv, T), -7.0, device=dev) if weigh else None
        self.w_in = win.to(dev) if weigh and w_in else None
        self.seq = torch.tensor(lens, dtype=torch.int32, device=dev)
        self.new = None if new_len is None else torch.tensor(new_len, dtype=torch.int32, device=dev)
        if page:
            pages = -(-T // page)
            n_pages = B * pages + 2
            table = rng.permutation(n_pages)[: B * pages].reshape(B, pages).astype(np.int32)
            def pool(x):
                xp = torch.full((B, Hkv, pages * page, dim), float("nan"), dtype=dt)
                xp[:, :, :T] = x
                y = torch.full((n_pages, Hkv, page, dim), float("nan"), dtype=dt)
                y[torch.from_numpy(table.reshape(-1)).long()] = (
                    xp.view(B, Hkv, pages, page, dim).transpose(1, 2).reshape(-1, Hkv, page, dim))
                return y
            kp, vpool = pool(k), pool(v)
            live = np.zeros((B, pages * page), bool)
            live[:, :T] = seen
            table[~live.reshape(B, pages, page).any(2)] = -1   # pages nobody sees are not mapped
            self.kt, self.vt = _lay(kp.to(dev), layout), _lay(vpool.to(dev), layout)
            self.table = torch.from_numpy(table).to(dev)
            self.kc, self.vc = vp.kv_paged(self.kt, self.table), vp.kv_paged(self.vt, self.table)
        else:
            self.kt, self.vt = _lay(k.to(dev), layout), _lay(v.to(dev), layout)
            self.kc, self.vc = vp.kv_contiguous(self.kt), vp.kv_contiguous(self.vt)
        self.ctx = vp.vp_init(vp.make_config(B, H, Hkv, dim, 0, T, vp.VP_FP32 if dtype == "fp32" else vp.VP_BF16,
                                             1 if page else 0, page or 16))
        vp.vp_reserve_new(self.ctx, n_new, n_new if weigh else 0)
        self.vis = vp.make_visible(window, sinks, scale)
        self.B, self.D, self.T, self.bf16 = B, dim, T, dtype == "bf16"

    def call(self, stream=None):
        tw = self.vp.token_weights
        self.vp.vp_attend_new(self.ctx, self.B, self.n_new, self.vp.rows(self.q), self.kc, self.vc, self.seq, self.vis,
                              self.vp.rows(self.out), new_len=self.new, lse=self.lse,
                              weight_in=None if self.w_in is None else tw(self.w_in),
                              weight_out=None if self.w_out is None else tw(self.w_out), stream=stream)

    def check(self):
        self.vp.vp_check_errors(self.ctx)
        for b, r in enumerate(self.ref):
            out, lse = self.out[b].double().cpu().numpy(), self.lse[b].double().cpu().numpy()
            n = self.ns[b]
            finite = np.isfinite(r["lse"])
            np.testing.assert_array_equal(np.isneginf(lse), ~finite)
            ze = self.D * U * r["zmag"]
            big = np.where(finite, np.abs(r["lse"]), 0.0)
            np.testing.assert_array_less(np.abs(lse[finite] - r["lse"][finite]),
                                         (ze + 2.0 ** -21 * (1 + big) + 1e-30)[finite])
            assert not out[~finite].any(), "a row that sees nothing must come out as 0"
            rel = 2 * ze + 2.0 ** -21 * (1 + big) + 2.0 ** -19
            tol = rel[..., None] * r["absout"]
            if self.bf16:
                tol = tol + 2.0 ** -9 * r["absout"] + 2.0 ** -9 * np.abs(r["out"]) * (1 + 2.0 ** -6)
            bad = np.abs(out - r["out"]) > tol
            assert not bad.any(), (b, np.argwhere(bad)[:5], np.abs(out - r["out"])[bad][:5], tol[bad][:5])
            if self.w_out is not None:
                L = self.lens[b]
                w = self.w_out[b].double().cpu().numpy()
                assert (w[:, L:] == -7.0).all(), "entries past the sequence must not be touched"
                wrel = float(rel.max()) if rel.size else 0.0
                old = self.w_old[b][:, :L].astype(np.float64)
                want = old + r["weight"]
                tol = wrel * r["weight"] + U * (n * 16 + 2) * r["weight"] + 2 * U * np.abs(want) + 1e-30
                bad = np.abs(w[:, :L] - want) > tol
                assert not bad.any(), (b, np.argwhere(bad)[:5])

    def run(self):
        try:
            self.call()
            torch.cuda.synchronize()
            self.check()
        finally:
            self.vp.vp_free(self.ctx)


HEADS = [((8, 2), 64), ((28, 4), 128), ((16, 1), 128), ((4, 4), 64)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,dim", HEADS)
@pytest.mark.parametrize("page", [0, 16])
def test_one_token_ragged_lengths(lib, dtype, heads, dim, page):
    Case(lib, heads, dim, dtype, lens=(1, 2, 127, 128, 129, 0, 700, 1025), page=page, weigh=True, seed=1).run()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 3), (1, 0), (1, 4), (100, 4), (128, 0), (129, 130), (300, 1),
                                          (5000, 4), (2**31 - 1, 2**31 - 1), (40, 2000)])
def test_one_token_window_and_sinks(lib, dtype, window, sinks):
    Case(lib, (28, 4), 128, dtype, lens=(1, 5, 128, 301, 1000, 0), window=window, sinks=sinks, weigh=True, page=8,
         seed=2).run()
    Case(lib, (8, 2), 64, dtype, lens=(1, 5, 128, 301, 1000, 0), window=window, sinks=sinks, seed=3).run()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,dim", HEADS)
@pytest.mark.parametrize("n_new,window,sinks", [(2, -1, 0), (5, 64, 4), (8, 3, 0), (8, 0, 2)])
def test_few_tokens(lib, dtype, heads, dim, n_new, window, sinks):
    Case(lib, heads, dim, dtype, lens=(n_new, 9, 257, 640, 0), n_new=n_new, window=window, sinks=sinks, page=16,
         weigh=True, seed=4).run()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,dim", HEADS)
@pytest.mark.parametrize("n_new,lens,window,sinks", [
    (33, (33, 70), -1, 0), (150, (150, 300, 411), -1, 0), (300, (300, 1), 64, 4), (129, (600, 129), 0, 1),
    (257, (257, 900), 128, 0), (257, (513, 257), 1, 0)])
def test_prompts(lib, dtype, heads, dim, n_new, lens, window, sinks):
    Case(lib, heads, dim, dtype, lens=lens, n_new=n_new, new_len=tuple(min(n_new, x) for x in lens), window=window,
         sinks=sinks, page=0, seed=5).run()
    Case(lib, heads, dim, dtype, lens=lens, n_new=n_new, new_len=tuple(min(n_new, x) for x in lens), window=window,
         sinks=sinks, page=64, seed=6).run()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n_new", [6, 200])
def test_new_lengths_differ(lib, dtype, n_new):
    """Sequences with fewer new tokens than rows, none at all, and their padding rows."""
    lens = (n_new, 300, 0, 260, 1)
    new = (n_new, n_new // 2, 0, 0, 1)
    for window in (-1, 70):
        Case(lib, (28, 4), 128, dtype, lens=lens, n_new=n_new, new_len=new, window=window, sinks=2,
             weigh=n_new * 7 <= 128, seed=7).run()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["dense", "swapped", "outer", "padded"])
@pytest.mark.parametrize("page", [0, 2, 8, 256])
@pytest.mark.parametrize("n_new", [1, 90])
def test_layouts(lib, dtype, layout, page, n_new):
    Case(lib, (8, 2), 128, dtype, lens=(90, 333, 130), n_new=n_new, page=page, layout=layout, window=100, sinks=3,
         max_seq=340, seed=8).run()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("spread", [0.0, 8.0])
def test_flat_and_peaked_logits(lib, dtype, spread):
    """Equal logits (q = 0) and logits that leave one token all the weight."""
    for n_new in (1, 80):
        Case(lib, (28, 4), 128, dtype, lens=(1500, 400), n_new=n_new, spread=spread, weigh=n_new == 1, seed=9).run()


def test_scale_and_missing_outputs(lib):
    c = Case(lib, (8, 2), 64, "bf16", lens=(200, 90), scale=0.3, weigh=True, w_in=False, seed=10)
    c.run()
    c = Case(lib, (8, 2), 64, "bf16", lens=(200, 90), seed=11)
    c.vp.vp_attend_new(c.ctx, 2, 1, lib.rows(c.q), c.kc, c.vc, c.seq, c.vis, lib.rows(c.out))
    c.lse.copy_(torch.from_numpy(np.stack([r["lse"] for r in c.ref])))
    torch.cuda.synchronize()
    c.check()
    lib.vp_free(c.ctx)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_weights_accumulate_in_place_over_steps(lib, dtype):
    """weight_in and weight_out as one array, three calls in a row on a side stream."""
    c = Case(lib, (8, 2), 64, dtype, lens=(500, 77), weigh=True, seed=12)
    c.w_out = c.w_in = torch.from_numpy(c.w_old).cuda().contiguous()
    c.w_out[0, :, 500:] = c.w_out[1, :, 77:] = -7.0
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        c.call(stream=s)
    s.synchronize()
    for r in c.ref:
        r["weight"] = 3 * r["weight"]
    c.check()
    lib.vp_free(c.ctx)


@pytest.mark.parametrize("n_new", [1, 40])
def test_calls_follow_each_other_and_graphs(lib, n_new):
    """Different shapes on one context back to back, and a captured graph, give
    what single calls give; repeated calls agree bit for bit."""
    c = Case(lib, (28, 4), 128, "bf16", lens=(3000, 200, 1), n_new=n_new, new_len=(n_new, n_new, 1), page=16, seed=13)
    c.call()
    torch.cuda.synchronize()
    first, lse = c.out.clone(), c.lse.clone()
    c.check()
    for _ in range(4):
        c.call()
        lib.vp_attend_new(c.ctx, 1, 1, lib.rows(c.q[:1, -1:]), c.kc, c.vc, c.seq, c.vis, lib.rows(c.out.clone()))
    torch.cuda.synchronize()
    assert torch.equal(c.out.view(torch.int16), first.view(torch.int16)) and torch.equal(c.lse, lse)
    c.out.fill_(float("nan"))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.call()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.out.view(torch.int16), first.view(torch.int16))
    lib.vp_free(c.ctx)


def test_device_side_values_are_checked(lib):
    c = Case(lib, (8, 2), 64, "bf16", lens=(100, 60), n_new=2, seed=14)
    for seq, new, word in [((101, 60), None, "seq_len"), ((-1, 60), None, "seq_len"), ((100, 60), (3, 1), "new_len"),
                           ((100, 1), None, "new_len"), ((100, 60), (-1, 1), "new_len")]:
        c.seq = torch.tensor(seq, dtype=torch.int32, device="cuda")
        c.new = None if new is None else torch.tensor(new, dtype=torch.int32, device="cuda")
        c.call()
        with pytest.raises(lib.VPError, match=word):
            lib.vp_check_errors(c.ctx)
        lib.vp_check_errors(c.ctx)
    lib.vp_free(c.ctx)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n_new", [1, 150])
@pytest.mark.parametrize("where", ["k", "v"])
def test_an_unmapped_visible_page_is_left_out(lib, dtype, n_new, where):
    c = Case(lib, (8, 2), 64, dtype, lens=(400, 250), n_new=n_new, page=16, poison=False, seed=15)
    hole = c.table.clone()
    hole[0, 3] = -1
    hole[1, 0] = c.kt.shape[0]
    if where == "k":
        c.kc = lib.kv_paged(c.kt, hole)
    else:
        c.vc = lib.kv_paged(c.vt, hole)
    c.call()
    with pytest.raises(lib.VPError, match="block table"):
        lib.vp_check_errors(c.ctx)
    # The same attention with those tokens' logits gone: compare against float64 over the rest.
    for b, lo in ((0, 48), (1, 0)):
        q = c.q[b].double().cpu().numpy()
        kk, vv = (x[c.table[b].long()].transpose(0, 1).reshape(2, -1, 64).double().cpu().numpy() for x in (c.kt, c.vt))
        L = c.lens[b]
        js = np.array([j for j in range(L) if not lo <= j < lo + 16])
        for i in (0, n_new - 1):
            t = L - n_new + i
            jj = js[js <= t]
            for h in range(8):
                z = kk[h // 4, jj] @ q[i, h] / 8.0
                p = np.exp(z - z.max())
                want = (p / p.sum()) @ vv[h // 4, jj]
                got = c.out[b, i, h].double().cpu().numpy()
                assert np.abs(got - want).max() < (2e-5 if dtype == "fp32" else 2e-2)
    lib.vp_free(c.ctx)


def test_refusals_of_attend_new(lib):
    c = Case(lib, (8, 2), 64, "bf16", lens=(100, 60), n_new=3, weigh=True, seed=16)
    V = lib

    def call(batch=2, n_new=3, q=None, kc=None, seq=c.seq, vis=None, out=None, w_in=None, w_out=None):
        st = V.vp_attend_new(c.ctx, batch, n_new, q or V.rows(c.q), kc or c.kc, c.vc, seq, vis or c.vis,
                             out or V.rows(c.out), weight_in=w_in, weight_out=w_out, check=False)
        return st, V.vp_last_error(c.ctx)

    w = V.token_weights(c.w_out)
    assert call()[0] == V.VP_OK
    assert call(batch=0)[0] == V.VP_OK and call(n_new=0)[0] == V.VP_OK
    assert call(batch=3)[0] == V.VP_ERR_CAPACITY
    assert call(batch=-1)[0] == V.VP_ERR_INVALID_ARG and call(n_new=-1)[0] == V.VP_ERR_INVALID_ARG
    assert call(n_new=4) == (V.VP_ERR_CAPACITY, "vp_attend_new: vp_reserve_new has not reserved for 4 new tokens")
    assert call(n_new=33, w_out=w)[0] == V.VP_ERR_UNSUPPORTED
    assert call(w_in=w)[0] == V.VP_ERR_INVALID_ARG
    assert call(seq=None)[0] == V.VP_ERR_INVALID_ARG
    for vis in (V.make_visible(-2), V.make_visible(1, -1), V.make_visible(1, 0, -1.0), V.make_visible(1, 0, math.inf)):
        assert call(vis=vis)[0] == V.VP_ERR_INVALID_ARG
    odd = V.rows(c.q)
    odd.stride_h = 65
    assert call(q=odd) == (V.VP_ERR_INVALID_ARG, "vp_attend_new: q: strides must be >= 0 and multiples of 16 bytes")
    odd = V.rows(c.out)
    odd.data += 2
    assert call(out=odd)[0] == V.VP_ERR_INVALID_ARG
    bad = V.vp_kv(c.kc.data, c.kc.stride_b, c.kc.stride_h, 65, None, 0, 0)
    assert call(kc=bad)[0] == V.VP_ERR_INVALID_ARG
    off = V.token_weights(c.w_out)
    off.data += 2
    assert call(w_out=off)[0] == V.VP_ERR_INVALID_ARG
    for new, weighed in ((0, 0), (101, 0), (3, 4), (3, -1)):
        with pytest.raises(V.VPError) as e:
            V.vp_reserve_new(c.ctx, new, weighed)
        assert e.value.status == V.VP_ERR_INVALID_ARG
    with pytest.raises(V.VPError) as e:
        V.vp_reserve_new(c.ctx, 60, 33)
    assert e.value.status == V.VP_ERR_UNSUPPORTED
    assert call()[0] == V.VP_OK   # a refused reservation leaves the old one
    V.vp_reserve_new(c.ctx, 3, 0)
    assert call(w_out=w)[0] == V.VP_ERR_CAPACITY
    torch.cuda.synchronize()
    V.vp_free(c.ctx)


# ------------------------------------------------------------------ eviction

def _evict(vp, heads=(8, 2), dim=64, dtype="bf16", lens=(100,), keep=40, sinks=2, recent=8, granularity=1, page=0,
           in_place=False, layout="dense", weights="random", dst_page=None, cap=None, alias_len=False, w_dst=True):
    rng = np.random.default_rng(5)
    H, Hkv = heads
    B, T = len(lens), max(max(lens), 1)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    k = torch.from_numpy(rng.standard_normal((B, Hkv, T, dim))).to(dt)
    v = torch.from_numpy(rng.standard_normal((B, Hkv, T, dim))).to(dt)
    w = rng.random((B, Hkv, T)).astype(np.float32)
    if weights == "ties":      # few distinct values, signed zeros among them
        w = rng.choice(np.array([0.0, -0.0, 0.25, -1.0, 3.0], np.float32), size=w.shape)
    elif weights == "special":
        w = rng.choice(np.array([0.0, np.inf, -np.inf, np.nan, 1e-42, 1.0, np.float32(1) + np.float32(2) ** -23],
                                np.float32), size=w.shape)
    elif weights == "equal":
        w[:] = 0.5
    elif weights == "whole":   # sums over the kv-heads are exact
        w = rng.integers(0, 50, size=w.shape).astype(np.float32)
    wt = torch.from_numpy(w).cuda()
    rows = min(keep, T)

    def paged(x, t, page):
        pages = -(-t // page)
        n = B * pages + 1
        table = torch.from_numpy(rng.permutation(n)[: B * pages].reshape(B, pages).astype(np.int32))
        pool = torch.zeros(n, Hkv, page, dim, dtype=dt)
        xp = torch.zeros(B, Hkv, pages * page, dim, dtype=dt)
        xp[:, :, :t] = x
        pool[table.view(-1).long()] = xp.view(B, Hkv, pages, page, dim).transpose(1, 2).reshape(-1, Hkv, page, dim)
        return _lay(pool.cuda(), layout), table

    def logical(x, table, t):
        if table is None:
            return x.cpu()[:, :, :t]
        y = x.cpu()[table.long()]
        return y.transpose(1, 2).reshape(B, Hkv, -1, dim)[:, :, :t]

    if page:
        kt, tb = paged(k, T, page)
        vt = torch.zeros_like(kt)
        y = torch.zeros(B, Hkv, tb.shape[1] * page, dim, dtype=dt)
        y[:, :, :T] = v
        vt[tb.view(-1).long().cuda()] = y.view(B, Hkv, -1, page, dim).transpose(1, 2).reshape(-1, Hkv, page, dim).cuda()
        tbd = tb.cuda()
        ks, vs = vp.kv_paged(kt, tbd), vp.kv_paged(vt, tbd)
    else:
        kt, vt, tb = _lay(k.cuda(), layout), _lay(v.cuda(), layout), None
        ks, vs = vp.kv_contiguous(kt), vp.kv_contiguous(vt)
    if in_place:
        kd_t, vd_t, td = kt, vt, tb
        kd, vd, wd_t = ks, vs, wt
    else:
        z = torch.zeros(B, Hkv, rows, dim, dtype=dt)
        if page and dst_page != 0:
            kd_t, td = paged(z, rows, page)
            vd_t = torch.zeros_like(kd_t)
            tdd = td.cuda()
            kd, vd = vp.kv_paged(kd_t, tdd), vp.kv_paged(vd_t, tdd)
        else:
            kd_t, vd_t, td = z.cuda(), z.clone().cuda(), None
            kd, vd = vp.kv_contiguous(kd_t), vp.kv_contiguous(vd_t)
        wd_t = torch.full((B, Hkv, rows), -3.0, device="cuda")
    cap = cap or keep
    nsel = Hkv if granularity else 1
    kept = torch.full((B, nsel, cap), -9, dtype=torch.int32, device="cuda")
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    new = seq if alias_len else torch.full((B,), -9, dtype=torch.int32, device="cuda")
    ctx = vp.vp_init(vp.make_config(B, H, Hkv, dim, 0, T, vp.VP_FP32 if dtype == "fp32" else vp.VP_BF16,
                                    1 if page else 0, page or 16))
    vp.vp_evict(ctx, B, ks, vs, seq, vp.make_evict(keep, sinks, recent, granularity), kd, vd, vp.token_weights(wt),
                vp.token_weights(wd_t) if w_dst else None, kept, cap, new)
    torch.cuda.synchronize()
    vp.vp_check_errors(ctx)
    vp.vp_free(ctx)
    assert new.cpu().tolist() == [min(x, keep) for x in lens]
    gk, gv = logical(kd_t, td, T if in_place else rows), logical(vd_t, td, T if in_place else rows)
    gw, gi = wd_t.cpu().numpy(), kept.cpu().numpy()
    for b, L in enumerate(lens):
        for g in range(Hkv):
            if granularity:
                wsel = w[b, g]
            else:
                wsel = w[b, 0].copy()
                for x in range(1, Hkv):
                    wsel = wsel + w[b, x]
            idx = O.evict(wsel, L, keep, sinks, recent)
            n = idx.size
            got = gi[b, g if granularity else 0]
            np.testing.assert_array_equal(got[:n], idx)
            assert (got[n:] == -1).all()
            assert torch.equal(gk[b, g, :n], k[b, g, torch.from_numpy(idx)])
            assert torch.equal(gv[b, g, :n], v[b, g, torch.from_numpy(idx)])
            if w_dst:
                np.testing.assert_array_equal(gw[b, g, :n], w[b, g, idx])
                if in_place:
                    assert not gw[b, g, n:L].any()
                    np.testing.assert_array_equal(gw[b, g, L:], w[b, g, L:])
                else:
                    assert (gw[b, g, n:] == -3.0).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("page", [0, 1, 16])
@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 128)])
def test_evict_ragged(lib, dtype, dim, page, in_place):
    _evict(lib, (8, 2), dim, dtype, lens=(0, 1, 39, 40, 41, 100, 2111, 64), page=page, in_place=in_place)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("weights", ["ties", "special", "equal", "whole"])
@pytest.mark.parametrize("granularity", [0, 1])
def test_evict_orders_weights(lib, weights, granularity, in_place):
    if granularity == 0 and weights == "special":
        pytest.skip("sums of infinities of both signs are NaN in either order")
    _evict(lib, (16, 4), 64, lens=(300, 1200, 80, 5000), keep=77, sinks=3, recent=20, granularity=granularity,
           weights=weights, in_place=in_place)


@pytest.mark.parametrize("keep,sinks,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (50, 25, 25), (50, 0, 50), (50, 50, 0),
                                               (50, 0, 0), (199, 0, 0), (200, 4, 4), (5000, 4, 4)])
def test_evict_policies(lib, keep, sinks, recent):
    for in_place in (False, True):
        _evict(lib, (4, 4), 64, lens=(200, 57), keep=keep, sinks=sinks, recent=recent, in_place=in_place)


def test_evict_other_forms(lib):
    _evict(lib, lens=(500, 90), layout="swapped")
    _evict(lib, lens=(500, 90), layout="outer", in_place=True)
    _evict(lib, lens=(500, 90), layout="padded", in_place=True, granularity=0)
    _evict(lib, lens=(500, 90), page=16, dst_page=0)
    _evict(lib, lens=(500, 90), cap=64, w_dst=False)
    _evict(lib, lens=(500, 20), in_place=True, alias_len=True)
    _evict(lib, lens=(500, 20), in_place=True, alias_len=True, granularity=0, page=16)
    _evict(lib, (28, 4), 128, lens=(20480,) * 3, keep=4097, sinks=4, recent=1000, in_place=True)
    _evict(lib, (28, 4), 128, lens=(20480, 17), keep=4097, sinks=4, recent=1000)


def test_refusals_of_evict(lib):
    V = lib
    k = torch.zeros(1, 2, 64, 64, dtype=torch.bfloat16, device="cuda")
    v, kd, vd = k.clone(), k.clone(), k.clone()
    w = torch.zeros(1, 2, 64, device="cuda")
    wd = w.clone()
    seq = torch.tensor([64], dtype=torch.int32, device="cuda")
    new = seq.clone()
    kept = torch.zeros(1, 2, 32, dtype=torch.int32, device="cuda")
    ctx = V.vp_init(V.make_config(1, 8, 2, 64, 0, 64, V.VP_BF16))
    c = V.kv_contiguous

    def call(batch=1, pol=None, a=None, b=None, x=None, y=None, wt=None, wo=None, cap=32, kp=kept):
        return V.vp_evict(ctx, batch, a or c(k), b or c(v), seq, pol or V.make_evict(32, 2, 4), x or c(kd), y or c(vd),
                          wt or V.token_weights(w), wo or V.token_weights(wd), kp, cap, new, check=False)

    assert call() == V.VP_OK and call(batch=0) == V.VP_OK
    assert call(batch=2) == V.VP_ERR_CAPACITY and call(batch=-1) == V.VP_ERR_INVALID_ARG
    assert call(cap=31) == V.VP_ERR_CAPACITY
    for pol in ((0, 0, 0, 1), (32, -1, 0, 1), (32, 0, -1, 1), (32, 20, 13, 1), (32, 0, 0, 2), (32, 0, 0, -1)):
        assert call(pol=V.vp_evict_policy(*pol)) == V.VP_ERR_INVALID_ARG
    assert call(kp=None) == V.VP_ERR_INVALID_ARG
    assert call(x=c(k)) == V.VP_ERR_INVALID_ARG              # K in place, V not
    assert call(x=c(k), y=c(v)) == V.VP_ERR_INVALID_ARG       # in place, weights elsewhere
    assert call(wo=V.token_weights(w)) == V.VP_ERR_INVALID_ARG  # weights in place, caches not
    half = c(k)
    half.stride_t = 128
    assert call(x=half) == V.VP_ERR_INVALID_ARG
    odd = c(kd)
    odd.stride_t = 65
    assert call(x=odd) == V.VP_ERR_INVALID_ARG
    odd = c(kd)
    odd.block_table = seq.data_ptr()
    assert call(x=odd) == V.VP_ERR_INVALID_ARG
    off = V.token_weights(w)
    off.data += 1
    assert call(wt=off) == V.VP_ERR_INVALID_ARG
    seq.fill_(65)
    assert call() == V.VP_OK
    with pytest.raises(V.VPError, match="seq_len"):
        V.vp_check_errors(ctx)
    V.vp_free(ctx)


def test_null_contexts(lib):
    assert lib.lib.vp_reserve_new(None, 1, 0) == lib.VP_ERR_NOT_INITIALIZED
    assert lib.lib.vp_attend_new(None, 1, 1, *([None] * 11)) == lib.VP_ERR_NOT_INITIALIZED
    assert lib.lib.vp_evict(None, 1, *([None] * 9), 0, None, None) == lib.VP_ERR_NOT_INITIALIZED
    assert ctypes.sizeof(lib.vp_visible) == 12 and ctypes.sizeof(lib.vp_rows) == 32


def test_prompt_blocks_with_few_rows_in_a_row(lib):
    """Many short prompts whose last row block is small, several per CTA, over
    and over: every call must give the first call's bits."""
    n, B = 45, 40
    lens = tuple(n + 13 * i for i in range(B))
    c = Case(lib, (28, 4), 128, "bf16", lens=lens, n_new=n, seed=17)
    c.call()
    torch.cuda.synchronize()
    c.check()
    first = c.out.clone()
    for _ in range(30):
        c.out.fill_(float("nan"))
        c.call()
        assert torch.equal(c.out.view(torch.int16), first.view(torch.int16))
    lib.vp_check_errors(c.ctx)
    lib.vp_free(c.ctx)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n_new,heads", [(1, (28, 4)), (4, (28, 4)), (10, (28, 4)), (90, (8, 2))])
def test_logits_that_jump_far(lib, dtype, n_new, heads):
    """Logits that rise by hundreds along the cache: the running reference has to
    follow, and what was summed before it has to vanish without a trace."""
    c = Case(lib, heads, 128, dtype, lens=(700, 333), n_new=n_new, spread=30.0, seed=18, poison=False,
             weigh=n_new * heads[0] // heads[1] <= 128)
    ramp = torch.linspace(-3.0, 3.0, 700, device="cuda")[None, None, :, None]
    k = (c.kt.float() * 0.05 + ramp * c.q[:, -1:, ::heads[0] // heads[1]].float().transpose(1, 2) / 30.0).to(c.kt.dtype)
    c.kt.copy_(k)
    c.ref = [O.attend_new(c.q[b].double().cpu().numpy(), c.kt[b].double().cpu().numpy(), c.vt[b].double().cpu().numpy(),
                          c.lens[b], c.ns[b]) for b in range(2)]
    assert max(r["lse"].max() for r in c.ref) > 200
    c.run()


@pytest.mark.parametrize("longest", [4096, 4097, 8192, 8193, 32768, 32769])
@pytest.mark.parametrize("granularity,in_place", [(1, False), (1, True), (0, True)])
def test_evict_cache_lengths(lib, longest, granularity, in_place):
    """Either side of every length at which the selection changes its form."""
    _evict(lib, (4, 2), 64, lens=(longest, 3000, 31), keep=2500, sinks=4, recent=100, granularity=granularity,
           in_place=in_place, weights="whole" if granularity == 0 else "ties")
