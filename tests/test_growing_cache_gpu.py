"""vp_append, vp_append4 and vp_attend4 as they are used: a layer that takes a
prompt, drafted tokens and single tokens, with its caches growing on the device;
and their neighbours in the library behind them without anything in between.

Outputs are compared with the float64 definition over what the caches hold; the
tolerances are those of test_attend4_gpu (4 bits) and test_new_tokens_gpu."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import cache4_oracle as O4
from oracle import cache_oracle as O
from tests.test_attend4_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vp(lib):
    assert torch.cuda.is_available()
    return lib


class Layer:
    """A layer on a paged 4-bit cache; the host keeps the projections of every token."""

    def __init__(self, vp, B, H, Hkv, D, T, max_new, page=16):
        self.vp, self.B, self.H, self.Hkv, self.D = vp, B, H, Hkv, D
        gen = torch.Generator().manual_seed(3)
        pages = -(-T // page)
        self.table = torch.randperm(B * pages, generator=gen).view(B, pages).int().cuda()
        self.pools = [(torch.full((B * pages, Hkv, page, D // 2), 255, dtype=torch.uint8, device="cuda"),
                       torch.full((B * pages, Hkv, page, D // 32), float("nan"), dtype=torch.half, device="cuda"))
                      for _ in range(2)]
        self.kc, self.vc = (vp.kv4_paged(*x, self.table) for x in self.pools)
        self.ctx = vp.vp_init(vp.make_config(B, H, Hkv, D, 0, T, vp.VP_BF16, 1, page))
        vp.vp_reserve4(self.ctx, max_new)
        angle = np.arange(T)[:, None] * (100.0 ** (-np.arange(D // 2) / (D // 2)))
        self.cos_sin = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)).cuda()
        self.rotation = vp.make_rotation(self.cos_sin)
        self.seq = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.page = page

    def step(self, qkv, new_len=None):
        """qkv [B, n, H + 2 Hkv, D]; the queries are rotated in place."""
        vp, n = self.vp, qkv.shape[1]
        q, k, v = qkv[:, :, : self.H], qkv[:, :, self.H: self.H + self.Hkv], qkv[:, :, self.H + self.Hkv:]
        self.seq += n if new_len is None else new_len
        rq = vp.rows(q)
        vp.vp_append4(self.ctx, self.B, n, rq, vp.rows(k), vp.rows(v), self.seq, self.rotation, rq, self.kc, self.vc,
                      new_len=new_len)
        out = torch.full((self.B, n, self.H, self.D), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.B, n, self.H), float("nan"), device="cuda")
        vp.vp_attend4(self.ctx, self.B, n, rq, self.kc, self.vc, self.seq, vp.make_visible(), vp.rows(out),
                      new_len=new_len, lse=lse)
        return q, out, lse

    def held(self, pool, b, length):
        at = torch.arange(length)
        page, row = self.table[b].cpu().long()[at // self.page], at % self.page
        codes, scale = pool[0].cpu()[page, :, row], pool[1].cpu()[page, :, row]
        return O4.values(O4.unpack(codes.numpy()), scale.double().numpy()).transpose(1, 0, 2)


def _near(q, out, lse, k, v, n):
    """One sequence's rows against the definition."""
    r = O.attend_new(q.double().cpu().numpy(), k, v, k.shape[1], n)
    got = out.double().cpu().numpy()
    z = 2.0 ** -20 * 16 * r["zmag"] + 2.0 ** -21 * (1 + np.abs(np.where(np.isfinite(r["lse"]), r["lse"], 0)))
    assert (np.abs(lse.double().cpu().numpy()[:n] - r["lse"][:n]) <= z[:n] + 1e-30).all()
    tol = (2 * z[..., None] + 2.0 ** -9) * r["absout"] + 2.0 ** -8 * np.abs(r["out"]) * (1 + 2.0 ** -6) + 1e-30
    assert (np.abs(got - r["out"]) <= tol).all()
    assert not got[n:].any()


@pytest.mark.parametrize("heads,dim", [((8, 2), 64), ((7, 1), 128)])
def test_prompt_drafted_tokens_and_steps(vp, heads, dim):
    B, (H, Hkv), D = 3, heads, dim
    layer = Layer(vp, B, H, Hkv, D, 300, 60)
    gen = torch.Generator().manual_seed(1)
    lengths = [0] * B
    plan = [(60, (60, 17, 41)), (5, (5, 1, 3)), (1, None), (4, (0, 4, 2)), (1, None), (33, (33, 30, 1)), (1, None)]
    for n, new in plan:
        qkv = torch.randn(B, n, H + 2 * Hkv, D, generator=gen).bfloat16()
        dev = qkv.cuda()
        new_len = None if new is None else torch.tensor(new, dtype=torch.int32, device="cuda")
        q, out, lse = layer.step(dev, new_len)
        vp.vp_check_errors(layer.ctx)
        ns = [n] * B if new is None else list(new)
        for b in range(B):
            start, lengths[b] = lengths[b], lengths[b] + ns[b]
            k, v = (layer.held(x, b, lengths[b]) for x in layer.pools)
            _near(q[b], out[b], lse[b], k, v, ns[b])
            # what was held for the new tokens: within half a step of the rotated key
            cs = layer.cos_sin.cpu().numpy()[start: lengths[b]]
            turned = O4.rotate(qkv[b, : ns[b], H: H + Hkv].float().numpy(), cs[:, None, : D // 2], cs[:, None, D // 2:], False,
                               np.float32)
            codes, steps = O4.quantise(torch.from_numpy(turned).bfloat16().float().numpy())
            np.testing.assert_array_equal(k[:, start:].transpose(1, 0, 2), O4.values(codes, steps))


def test_a_captured_step_follows_the_lengths(vp):
    """One graph of the length's increment, the append and the attention, replayed."""
    B, H, Hkv, D = 4, 8, 2, 64
    layer = Layer(vp, B, H, Hkv, D, 200, 40)
    gen = torch.Generator().manual_seed(2)
    prompt = torch.randn(B, 40, H + 2 * Hkv, D, generator=gen).bfloat16().cuda()
    layer.step(prompt, torch.tensor([40, 7, 0, 16], dtype=torch.int32, device="cuda"))
    static = torch.zeros(B, 1, H + 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    lengths = [40, 7, 0, 16]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            q, out, lse = layer.step(static)
        for _ in range(5):
            static.copy_(torch.randn(static.shape, generator=gen).bfloat16())
            g.replay()
            s.synchronize()
            lengths = [x + 1 for x in lengths]
            assert layer.seq.tolist() == lengths
            for b in range(B):
                k, v = (layer.held(x, b, lengths[b]) for x in layer.pools)
                _near(q[b], out[b], lse[b], k, v, 1)
    vp.vp_check_errors(layer.ctx)


def test_a_captured_prompt(vp):
    """Calls by way of the staged rows, captured and replayed between others on the same workspace."""
    a = Case(vp, (8, 2), 64, "bf16", lens=(90, 200, 64), n_new=40, page=16)
    a.call()
    torch.cuda.synchronize()
    out = a.out.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            a.call()
        a.out.fill_(float("nan"))
        a.seq[0] -= 30              # another call in between, over other lengths
        a.call()
        a.seq[0] += 30
        a.out.fill_(float("nan"))
        g.replay()
        s.synchronize()
    assert torch.equal(a.out, out)
    a.check()


@pytest.mark.parametrize("paged", [0, 16])
def test_append_directly_before_its_neighbours(vp, paged):
    """vp_decode_step reads the caches before it waits; what vp_append wrote is there, time after time."""
    B, H, Hkv, D, n_vis, T = 8, 28, 4, 128, 512, 1500
    gen = torch.Generator("cuda").manual_seed(5)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    if paged:
        pages = -(-T // paged)
        table = torch.randperm(B * pages, generator=torch.Generator().manual_seed(1)).view(B, pages).int().cuda()
        k, v = (randn(B * pages, Hkv, paged, D) for _ in range(2))
        kc, vc = vp.kv_paged(k, table), vp.kv_paged(v, table)
    else:
        k, v = (randn(B, Hkv, T, D) for _ in range(2))
        kc, vc = vp.kv_contiguous(k), vp.kv_contiguous(v)
    ctx = vp.vp_init(vp.make_config(B, H, Hkv, D, n_vis, T, vp.VP_BF16, 1 if paged else 0, paged or 16))
    vp.vp_reserve_new(ctx, 1)
    seq = torch.tensor([700 + 90 * b for b in range(B)], dtype=torch.int32, device="cuda")
    vis = vp.span(torch.zeros_like(seq), torch.full_like(seq, n_vis))
    start, length = torch.zeros_like(seq), torch.full_like(seq, n_vis)
    vis = vp.span(start, length)
    text = seq - n_vis
    budget = vp.make_budget(vp.VP_DENSE)
    qkv = randn(12, B, 1, H + 2 * Hkv, D)
    angle = torch.arange(T, device="cuda", dtype=torch.float64)[:, None] * torch.rand(D // 2, device="cuda", generator=gen).double()
    table_cs = torch.cat([angle.cos(), angle.sin()], 1).float()
    rotation = vp.make_rotation(table_cs)
    kept = torch.empty(B, n_vis, dtype=torch.int32, device="cuda")
    count, mass = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, H, device="cuda")

    def pass_over(wait):
        outs = []
        for x in qkv:
            q, kk, vv = x[:, :, :H], x[:, :, H: H + Hkv], x[:, :, H + Hkv:]
            turned = torch.empty(B, 1, H, D, dtype=torch.bfloat16, device="cuda")
            one, two = torch.empty(B, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty_like(turned)
            torch.cuda.synchronize()
            vp.vp_append(ctx, B, 1, vp.rows(q), vp.rows(kk), vp.rows(vv), seq, rotation, vp.rows(turned), kc, vc)
            if wait:
                torch.cuda.synchronize()
            vp.vp_decode_step(ctx, B, turned, kc, vc, vis, text, budget, one, kept, n_vis, count, mass)
            vp.vp_append(ctx, B, 1, vp.rows(q), vp.rows(kk), vp.rows(vv), seq, rotation, vp.rows(turned), kc, vc)
            vp.vp_attend_new(ctx, B, 1, vp.rows(turned), kc, vc, seq, vp.make_visible(), vp.rows(two))
            outs += [one, two]
        torch.cuda.synchronize()
        vp.vp_check_errors(ctx)
        return outs

    want = pass_over(True)
    for _ in range(3):
        for x, y in zip(pass_over(False), want):
            assert torch.equal(x, y)


def test_calls_need_the_contexts_device(vp):
    a = Case(vp, (8, 2), 64, "bf16", lens=(64,), n_new=2)
    kv = vp.vp_kv4.from_buffer_copy(a.kc)
    before = [t.clone() for t in a.tensors]
    x = torch.randn(1, 2, 2, 64, device="cuda").bfloat16()
    k = torch.zeros(1, 2, 64, 64, device="cuda").bfloat16()
    plain = vp.kv_contiguous(k)
    calls = [lambda: vp.vp_reserve4(a.ctx, 2), a.call,
             lambda: vp.vp_append4(a.ctx, 1, 2, None, vp.rows(x), vp.rows(x), a.seq, None, None, kv, a.vc),
             lambda: vp.vp_append(a.ctx, 1, 2, None, vp.rows(x), vp.rows(x), a.seq, None, None, plain, plain)]
    # The context's device number follows its configuration; with one GPU, another
    # number there stands for another current device.
    device = ctypes.c_int.from_address(a.ctx.value + ctypes.sizeof(vp.vp_config))
    here, device.value = device.value, device.value + 1
    assert here == torch.cuda.current_device()
    for call in calls:
        with pytest.raises(vp.VPError, match="device") as e:
            call()
        assert e.value.status == vp.VP_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert a.out.isnan().all() and not k.any()
    assert all(torch.equal(t.view(torch.uint8), b.view(torch.uint8)) for t, b in zip(a.tensors, before))
    device.value = here
    for call in calls[:2]:
        call()
    torch.cuda.synchronize()
    a.check()
    vp.vp_free(a.ctx)


def test_a_call_of_too_many_tiles_is_refused(vp):
    """2^20 tokens of room, fp32, 4096 rows: over 2^31 units of work in the worst case."""
    ctx = vp.vp_init(vp.make_config(512, 16, 16, 64, 0, 1 << 20, vp.VP_FP32, 1, 16))
    vp.vp_reserve4(ctx, 4096)
    x = torch.zeros(16, device="cuda")
    kv = vp.vp_kv4(x.data_ptr(), x.data_ptr(), 512, 512, 32, 32, 32, 2, x.data_ptr(), 1, 1)
    rows = vp.vp_rows(x.data_ptr(), 64, 64, 64)
    assert vp.vp_attend4(ctx, 512, 4096, rows, kv, kv, x, vp.make_visible(), rows, check=False) == vp.VP_ERR_UNSUPPORTED
    assert "too large" in vp.vp_last_error(ctx)
    vp.vp_free(ctx)
