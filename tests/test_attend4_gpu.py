"""vp_attend4 against the float64 definition over the values that the cache holds.

Tolerances, per element, from the arithmetic (u = 2^-24, float32):
  logits   codes less 8 are whole numbers, so a group's terms are at most
           M = scale * sum_d |q_d| 8 |step_d| in sum; two products of 16 terms each
           round at 2^-22 of that at worst (twice float's step, for tensor cores that
           truncate), the scaled sums at u: z_err = 2^-20 M; fp32 queries in two
           fp16 terms: 2^-22 M more;
  lse      z_err + 2^-21 (1 + |lse|);
  out      a relative 2 z_err + 2^-21 (1 + |lse|) + 2^-19 of sum_j p_j |v_j|;
           bf16: P and its product with the scale are rounded to fp16, 2^-11 each
           of sum_j p_j |v_j|, and the output 2^-8 of it; fp32: two fp16 terms
           each, 2^-21 together;
           the sum of the products, one for every 128 tokens of a warp, and of 8 warps and the CTAs' records
           is rounded (tokens / 128 + 40) times at 2^-22 of sum_j p_j |v_j|;
           P, whose largest is 2^10 or more, is rounded at 2^-25 below 2^-14, and so is
           its product with the scale (of two terms the second); a code less 8 is at
           most 8: tokens * 2^-35 * 8 (max step + 1); bf16 with a scale of 2 or more:
           the largest is 2^-5, tokens * 2^-20 * 8 max step."""

import numpy as np
import pytest
import torch

from oracle import cache4_oracle as O4
from oracle import cache_oracle as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def vp(lib):
    assert torch.cuda.is_available()
    return lib


def _layout(x, how):
    x = x.cuda()
    if how == "swapped":
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    if how == "outer":
        return x.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    if how == "padded":
        pad = max(16 // x.element_size(), x.shape[3]) if x.dtype != torch.half else x.shape[3]
        y = torch.zeros(*x.shape[:3], x.shape[3] + pad, dtype=x.dtype, device=x.device)
        y[..., : x.shape[3]] = x
        return y[..., : x.shape[3]]
    return x.contiguous()


class Case:
    def __init__(self, vp, heads=(8, 2), dim=64, dtype="bf16", lens=(33,), n_new=1, new_len=None, window=-1, sinks=0,
                 scale=0.0, page=0, layout="dense", max_seq=None, seed=0, spread=1.0, k_size=1.0, v_size=1.0, steps=None, q=None, rounded=False):
        rng = np.random.default_rng(seed)
        self.vp, self.lens, self.n_new = vp, lens, n_new
        H, Hkv = heads
        B, T = len(lens), max_seq or max(max(lens), 1)
        dt = torch.float32 if dtype == "fp32" else torch.bfloat16
        self.ns = [min(n_new, L) if new_len is None else new_len[b] for b, L in enumerate(lens)]
        q_drawn = torch.from_numpy(rng.standard_normal((B, n_new, H, dim)) * spread).to(dt)
        q = q_drawn if q is None else q
        self.held = []
        for size in (k_size, v_size):
            x = torch.from_numpy(rng.standard_normal((B, Hkv, T, dim)) * size).to(dt).float().numpy()
            self.held.append(O4.quantise(x))
        if steps is not None:
            steps(self.held, rng)
        (kcode, kstep), (vcode, vstep) = self.held
        k, v = O4.values(kcode, kstep), O4.values(vcode, vstep)
        if rounded:  # calls of many rows round values that are not bf16 numbers
            k, v = (torch.from_numpy(x).bfloat16().double().numpy() for x in (k, v))
        self.ref = [O.attend_new(q[b].double().numpy(), k[b], v[b], lens[b], self.ns[b], window, sinks, scale or None)
                    for b in range(B)]
        sc = scale or dim ** -0.5
        self.bounds = []
        with np.errstate(invalid="ignore"):
            for b in range(B):
                js = slice(0, max(lens[b], 1))
                qa = np.abs(q[b].double().numpy()).reshape(n_new, Hkv, H // Hkv, dim // 32, 32).sum(-1)
                M = np.zeros((n_new, H))
                for g in range(Hkv):
                    m = (qa[:, g] * np.abs(kstep[b, g, js]).max(0)).sum(-1) * 8 * sc
                    M[:, g * (H // Hkv): (g + 1) * (H // Hkv)] = m
                vs = np.abs(vstep[b, :, js]).max(1).repeat(32, -1)          # [Hkv, D]: largest scale of a dimension
                self.bounds.append((M, vs.repeat(H // Hkv, 0)))
        seen = np.zeros((B, T), bool)
        for b in range(B):
            if self.ns[b]:
                seen[b, : lens[b]] = self.ref[b]["mask"].any(0)
            q[b, self.ns[b]:] = float("nan")
        # Tokens that nobody sees: any codes, scales that are not numbers.
        kp, vp_ = (torch.from_numpy(O4.pack(x[0])) for x in self.held)
        ks, vs = (torch.from_numpy(x[1]).half() for x in self.held)
        for y in (ks, vs):
            y[torch.from_numpy(~seen)[:, None, :, None].expand_as(y)] = float("nan")
        self.q = _layout(q, layout if layout != "outer" else "dense")
        self.out = _layout(torch.full((B, n_new, H, dim), float("nan"), dtype=dt), layout if layout != "outer" else "dense")
        if layout == "padded":
            self.out.fill_(float("nan"))
        self.lse = torch.full((B, n_new, H), float("nan"), device="cuda")
        self.seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.new = None if new_len is None else torch.tensor(new_len, dtype=torch.int32, device="cuda")
        if page:
            pages = -(-T // page)
            n_pages = B * pages + 2
            table = rng.permutation(n_pages)[: B * pages].reshape(B, pages).astype(np.int32)

            def pool(x, fill):
                xp = torch.full((B, Hkv, pages * page, x.shape[3]), fill, dtype=x.dtype)
                xp[:, :, :T] = x
                y = torch.full((n_pages, Hkv, page, x.shape[3]), fill, dtype=x.dtype)
                y[torch.from_numpy(table.reshape(-1)).long()] = (
                    xp.view(B, Hkv, pages, page, x.shape[3]).transpose(1, 2).reshape(-1, Hkv, page, x.shape[3]))
                return y

            kp, vp_, ks, vs = pool(kp, 255), pool(vp_, 255), pool(ks, float("nan")), pool(vs, float("nan"))
            live = np.zeros((B, pages * page), bool)
            live[:, :T] = seen
            table[~live.reshape(B, pages, page).any(2)] = -1
            self.table = torch.from_numpy(table).cuda()
        self.tensors = [_layout(x, layout) for x in (kp, ks, vp_, vs)]
        if page:
            self.kc, self.vc = vp.kv4_paged(*self.tensors[:2], self.table), vp.kv4_paged(*self.tensors[2:], self.table)
        else:
            self.kc, self.vc = vp.kv4_contiguous(*self.tensors[:2]), vp.kv4_contiguous(*self.tensors[2:])
        self.ctx = vp.vp_init(vp.make_config(B, H, Hkv, dim, 0, T, vp.VP_FP32 if dtype == "fp32" else vp.VP_BF16,
                                             1 if page else 0, page or 16))
        vp.vp_reserve4(self.ctx, n_new)
        self.vis = vp.make_visible(window, sinks, scale)
        self.B, self.D, self.bf16 = B, dim, dtype == "bf16"

    def call(self, stream=None):
        vp = self.vp
        vp.vp_attend4(self.ctx, self.B, self.n_new, vp.rows(self.q), self.kc, self.vc, self.seq, self.vis,
                      vp.rows(self.out), new_len=self.new, lse=self.lse, stream=stream)

    def check(self):
        self.vp.vp_check_errors(self.ctx)
        for b, ref in enumerate(self.ref):
            out, lse = self.out[b].double().cpu().numpy(), self.lse[b].double().cpu().numpy()
            M, vstep = self.bounds[b]
            finite = np.isfinite(ref["lse"])
            np.testing.assert_array_equal(np.isneginf(lse), ~finite)
            ze = 2.0 ** -20 * M * (1 if self.bf16 else 1.25)
            big = np.where(finite, np.abs(ref["lse"]), 0.0)
            assert (np.abs(lse[finite] - ref["lse"][finite]) <= (ze + 2.0 ** -21 * (1 + big) + 1e-30)[finite]).all(), (
                b, np.abs(lse[finite] - ref["lse"][finite]).max())
            assert not out[~finite].any(), "a row that sees nothing must come out as 0"
            rel = 2 * ze + 2.0 ** -21 * (1 + big) + 2.0 ** -19 + (2.0 ** -10 if self.bf16 else 2.0 ** -21)
            L = self.lens[b]
            tol = (rel[..., None] + 2.0 ** -22 * (L / 128 + 40)) * ref["absout"]
            tol = tol + L * 2.0 ** -32 * (vstep + 1)
            if self.bf16:
                tol = tol + L * 2.0 ** -17 * vstep * (vstep >= 2).any()
                tol = tol + 2.0 ** -8 * np.abs(ref["out"]) * (1 + 2.0 ** -6)
            bad = ~(np.abs(out - ref["out"]) <= tol)
            assert not bad.any(), (b, np.argwhere(bad)[:5], np.abs(out - ref["out"])[bad][:5], tol[bad][:5])

    def run(self):
        self.call()
        torch.cuda.synchronize()
        self.check()
        self.vp.vp_free(self.ctx)


TYPES = pytest.mark.parametrize("dtype", ["bf16", "fp32"])
HEADS = pytest.mark.parametrize("heads,dim", [((8, 2), 64), ((28, 4), 128), ((8, 1), 128), ((5, 5), 64), ((16, 1), 64), ((32, 2), 128)])


@TYPES
@HEADS
@pytest.mark.parametrize("page", [0, 16])
def test_one_token(vp, dtype, heads, dim, page):
    Case(vp, heads, dim, dtype, lens=(1, 15, 16, 17, 128, 129, 300, 0, 1025), page=page).run()


@TYPES
@pytest.mark.parametrize("heads,dim", [((8, 2), 64), ((28, 4), 128), ((8, 1), 128)])
@pytest.mark.parametrize("n_new", [2, 3, 5, 8])
def test_a_few_tokens(vp, dtype, heads, dim, n_new):
    Case(vp, heads, dim, dtype, lens=(n_new, 130, 257, 64), n_new=n_new, page=16).run()


@TYPES
@pytest.mark.parametrize("n_new", [33, 128, 200])
@pytest.mark.parametrize("heads,dim", [((4, 2), 64), ((7, 1), 128)])
def test_prompts(vp, dtype, n_new, heads, dim):
    Case(vp, heads, dim, dtype, lens=(n_new, n_new + 77), n_new=n_new).run()


@TYPES
@pytest.mark.parametrize("page", [1, 8, 16, 256])
@pytest.mark.parametrize("window,sinks", [(-1, 0), (0, 0), (0, 3), (37, 5), (200, 0)])
def test_prompts_of_paged_caches(vp, dtype, page, window, sinks):
    Case(vp, (7, 1), 64, dtype, lens=(90, 400, 0, 70), n_new=70, new_len=(70, 33, 0, 1), page=page, window=window,
         sinks=sinks).run()


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("layout", ["dense", "swapped", "outer", "padded"])
def test_prompts_in_other_layouts(vp, page, layout):
    Case(vp, (4, 2), 128, "bf16", lens=(150, 300, 77), n_new=77, page=page, layout=layout).run()


def test_prompts_of_more_sequences_than_are_staged_at_once(vp):
    """Room of 2^20 tokens per sequence: the workspace holds two sequences."""
    for lens in ((90, 400, 130, 77, 65), (65, 65)):
        a = Case(vp, (8, 2), 64, "bf16", lens=lens, n_new=40, page=64, new_len=(40, 33, 40, 1, 0)[: len(lens)])
        a.ctx = vp.vp_init(vp.make_config(len(lens), 8, 2, 64, 0, 1 << 20, vp.VP_BF16, 1, 64))
        vp.vp_reserve4(a.ctx, 40)
        for _ in range(2):
            a.out.fill_(float("nan"))
            a.call()
            torch.cuda.synchronize()
            a.check()
        vp.vp_free(a.ctx)


def test_unmapped_page_is_left_out_of_a_prompt(vp):
    a = Case(vp, (8, 2), 64, "bf16", lens=(200, 90), n_new=40, page=16)
    a.call()
    torch.cuda.synchronize()
    want = [x.clone() for x in (a.out, a.lse)]
    page = int(a.table[0, 3])
    a.table[0, 3] = -1
    a.call()
    with pytest.raises(vp.VPError, match="block table"):
        vp.vp_check_errors(a.ctx)
    keep = [j for j in range(200) if j // 16 != 3]
    (kc, ks), (vc, vs) = a.held
    r = O.attend_new(a.q[0].double().cpu().numpy(), O4.values(kc, ks)[0][:, keep], O4.values(vc, vs)[0][:, keep], 184, 40)
    assert np.abs(a.lse[0].cpu().numpy() - r["lse"]).max() < 1e-4
    assert torch.equal(a.out[1], want[0][1])
    a.table[0, 3] = page                       # mapped again: nothing of that is left in the workspace
    a.call()
    torch.cuda.synchronize()
    vp.vp_check_errors(a.ctx)
    assert torch.equal(a.out, want[0]) and torch.equal(a.lse, want[1])


@TYPES
@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 3), (1, 0), (5, 0), (40, 4), (128, 1), (1000, 2), (200, 300), (16, 16)])
@pytest.mark.parametrize("n_new", [1, 6])
def test_windows_and_sinks(vp, dtype, window, sinks, n_new):
    Case(vp, (6, 2), 64, dtype, lens=(n_new, 50, 260, 513), n_new=n_new, window=window, sinks=sinks, page=8).run()


@pytest.mark.parametrize("new_len", [(5, 0, 1, 3), (0, 0, 0, 0), (1, 2, 3, 4)])
@TYPES
def test_ragged_new_tokens(vp, dtype, new_len):
    Case(vp, (28, 4), 128, dtype, lens=(5, 40, 300, 129), n_new=5, new_len=new_len, window=64, sinks=2).run()


@TYPES
@pytest.mark.parametrize("layout", ["dense", "swapped", "outer", "padded"])
@pytest.mark.parametrize("page", [0, 1, 2, 8, 64, 256])
@pytest.mark.parametrize("dim", [64, 128])
def test_layouts(vp, dtype, layout, page, dim):
    Case(vp, (4, 2), dim, dtype, lens=(70, 129, 300), n_new=2, page=page, layout=layout).run()


@TYPES
def test_long_sequences_are_split(vp, dtype):
    Case(vp, (8, 2), 128, dtype, lens=(20000, 7, 4097)).run()
    Case(vp, (4, 1), 64, dtype, lens=(9001,), n_new=3, page=64).run()


@TYPES
def test_even_rows_over_a_long_range(vp, dtype):
    """Every token has nearly the same weight: the output is far smaller than its terms."""
    Case(vp, (4, 1), 64, dtype, lens=(20000, 3000), spread=0.01).run()


@TYPES
def test_queries_with_one_large_dimension(vp, dtype):
    """The others' products are small beside one of them, and are not lost."""
    a = Case(vp, (8, 2), 128, dtype, lens=(700, 65), n_new=2, spread=1.0, seed=4)
    q = a.q.clone()
    q[..., 37] = 300.0
    b = Case(vp, (8, 2), 128, dtype, lens=(700, 65), n_new=2, spread=1.0, seed=4, q=q.cpu())
    b.run()


@TYPES
def test_many_sequences(vp, dtype):
    rng = np.random.default_rng(3)
    Case(vp, (4, 2), 64, dtype, lens=tuple(int(x) for x in rng.integers(0, 400, 300))).run()


@TYPES
@pytest.mark.parametrize("spread,k_size,v_size", [(8.0, 2.0, 1.0), (1e-4, 1.0, 1.0), (1.0, 1.0, 3e-4), (1.0, 1e-3, 1.0),
                                                  (0.02, 300.0, 1.0), (1.0, 1.0, 2000.0), (1e20, 1e-4, 1.0), (1e-30, 1.0, 1.0)])
def test_sizes_of_values(vp, dtype, spread, k_size, v_size):
    """Peaked and even rows, values near the least scales and far above the usual ones."""
    Case(vp, (8, 2), 64, dtype, lens=(700, 129), n_new=2, spread=spread, k_size=k_size, v_size=v_size,
         scale=1e-17 if spread == 1e20 else 0.0).run()


@TYPES
@pytest.mark.parametrize("at", [0, 100, 600])
def test_one_large_value_scale(vp, dtype, at):
    """A token whose values' scales are far above the others': before, among and
    behind those, the fp16 form of the probabilities has to change."""
    def steps(held, rng):
        held[1][1][:, :, at] = 4096.0
        held[1][1][:, :, 650] = 61440.0
        held[1][0][:, :, 650] = 8 + (rng.random(held[1][0][:, :, 650].shape) < 0.5)

    Case(vp, (8, 2), 64, dtype, lens=(700,), n_new=2, steps=steps).run()


def test_any_fp16_scale(vp):
    """Scales of eleven significant bits, negative and zero ones: not vp_append4's, but served."""
    def steps(held, rng):
        for _, step in held:
            step[:] = (rng.standard_normal(step.shape) * 0.3).astype(np.float16)
            step[:, :, ::9] = 0

    Case(vp, (8, 2), 128, "bf16", lens=(300, 77), n_new=2, steps=steps).run()
    Case(vp, (8, 2), 128, "fp32", lens=(300, 77), n_new=40, steps=steps).run()
    Case(vp, (8, 2), 128, "bf16", lens=(300, 77), n_new=70, steps=steps, rounded=True).run()


@TYPES
@pytest.mark.parametrize("n_new", [1, 40])
def test_scales_that_are_not_numbers(vp, dtype, n_new):
    """A key that is not a number: every row that sees it is that, others are as without it."""
    a = Case(vp, (4, 2), 64, dtype, lens=(300, 200), n_new=n_new)
    a.tensors[1][0, 1, 60 if n_new == 1 else 299] = float("nan")
    a.call()
    torch.cuda.synchronize()
    out, lse = a.out.float().cpu(), a.lse.cpu()
    sees = slice(n_new - 1, n_new)
    assert torch.isnan(lse[0, sees, 2:]).all() and torch.isnan(out[0, sees, 2:]).all()
    lse[0, sees, 2:] = torch.from_numpy(a.ref[0]["lse"]).float()[sees, 2:]
    out[0, sees, 2:] = torch.from_numpy(a.ref[0]["out"]).float()[sees, 2:]
    a.lse.copy_(lse)
    a.out.copy_(out)
    a.check()


def test_unmapped_page_is_left_out(vp):
    a = Case(vp, (8, 2), 64, "bf16", lens=(200,), page=16)
    b = Case(vp, (8, 2), 64, "bf16", lens=(200,), page=16)
    a.table[0, 3] = -1
    b.table[0, 3] = 1000
    for x in (a, b):
        x.call()
        with pytest.raises(vp.VPError, match="block table"):
            vp.vp_check_errors(x.ctx)
    assert torch.equal(a.out, b.out) and torch.isfinite(a.out).all()
    keep = [j for j in range(200) if j // 16 != 3]
    (kc, ks), (vc, vs) = a.held
    q = a.q[0].double().cpu().numpy()
    k, v = O4.values(kc, ks)[0], O4.values(vc, vs)[0]
    r = O.attend_new(q, k[:, keep], v[:, keep], len(keep), 1)
    assert np.abs(a.lse[0].cpu().numpy() - r["lse"]).max() < 1e-4


def test_equal_calls_give_equal_bits_and_streams_and_graphs(vp):
    a = Case(vp, (28, 4), 128, "bf16", lens=(5000, 129, 3000), n_new=2, page=16)
    a.call()
    torch.cuda.synchronize()
    out, lse = a.out.clone(), a.lse.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(5):
            a.out.zero_()
            a.call()
        s.synchronize()
        assert torch.equal(a.out, out) and torch.equal(a.lse, lse)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            a.call()
            a.call()
    a.out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.out, out) and torch.equal(a.lse, lse)
    a.check()


def test_refusals(vp):
    a = Case(vp, (8, 2), 64, "bf16", lens=(200, 10), n_new=2, page=16)
    good = dict(batch=2, n_new=2, q=vp.rows(a.q), k_cache=a.kc, v_cache=a.vc, seq_len=a.seq, visible=a.vis,
                out=vp.rows(a.out))

    def status(**change):
        return vp.vp_attend4(a.ctx, **{**good, **change}, check=False)

    def but(struct, **fields):
        copy = type(struct).from_buffer_copy(struct)
        for name, value in fields.items():
            setattr(copy, name, value)
        return copy

    bad = vp.VP_ERR_INVALID_ARG
    assert status(batch=-1) == bad and status(n_new=-1) == bad and status(batch=3) == vp.VP_ERR_CAPACITY
    assert status(n_new=3) == vp.VP_ERR_CAPACITY
    assert status(q=None) == bad and status(out=None) == bad and status(k_cache=None) == bad and status(v_cache=None) == bad
    assert status(seq_len=None) == bad and status(visible=None) == bad
    assert status(visible=vp.make_visible(-2)) == bad and status(visible=vp.make_visible(3, -1)) == bad
    assert status(visible=vp.make_visible(scale=-1.0)) == bad and status(visible=vp.make_visible(scale=float("inf"))) == bad
    assert status(out=but(good["out"], stride_n=0)) == bad
    assert status(k_cache=but(a.kc, code_stride_h=8)) == bad and status(v_cache=but(a.vc, max_pages=0)) == bad
    assert status(k_cache=but(a.kc, code_stride_t=1 << 31)) == vp.VP_ERR_UNSUPPORTED
    assert status(v_cache=but(a.vc, scale_stride_b=1 << 31)) == vp.VP_ERR_UNSUPPORTED
    assert torch.isnan(a.out).all()
    other = vp.vp_init(vp.make_config(1, 8, 2, 64, 0, 64))
    with pytest.raises(vp.VPError) as e:
        vp.vp_reserve4(other, 65)
    assert e.value.status == bad
    assert vp.vp_attend4(other, 1, 1, *[None] * 6, check=False) == bad
    assert vp.vp_attend4(other, 1, 1, good["q"], a.kc, a.vc, a.seq, a.vis, good["out"], check=False) == vp.VP_ERR_CAPACITY
    assert status(batch=0) == vp.VP_OK and status(n_new=0) == vp.VP_OK
    vp.vp_check_errors(a.ctx)


def test_lengths_out_of_range_are_clamped(vp):
    a = Case(vp, (8, 2), 64, "bf16", lens=(64, 50, 20), n_new=2, max_seq=64)
    a.seq = torch.tensor([65, 50, -3], dtype=torch.int32, device="cuda")
    a.call()
    with pytest.raises(vp.VPError, match="seq_len"):
        vp.vp_check_errors(a.ctx)
    assert torch.isfinite(a.out[:2]).all() and not a.out[2].any()
