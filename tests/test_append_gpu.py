"""vp_append and vp_append4 against their definitions.

The rotation's operations are rounded one by one, so the rotated rows, the codes
and the scales equal the float32 restatement's bit for bit.  Against float64:
|x c| + |y s| are rounded three times (2^-24 each, relative), and the result once
to its type, 2^-8 of it for bf16 (eight significant bits: half a step of 2^-7)."""

import numpy as np
import pytest
import torch

from oracle import cache4_oracle as O4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vp(lib):
    assert torch.cuda.is_available()
    return lib


def _layout(x, how):
    """x [A, B, C, D] on the device in another memory order."""
    x = x.cuda()
    if how == "swapped":
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    if how == "outer":
        return x.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    if how == "padded":
        pad = max(16 // x.element_size(), x.shape[3])
        y = torch.zeros(*x.shape[:3], x.shape[3] + pad, dtype=x.dtype, device=x.device)
        y[..., : x.shape[3]] = x
        return y[..., : x.shape[3]]
    return x.contiguous()


class Append:
    def __init__(self, vp, heads=(8, 2), dim=64, dtype="bf16", lens=(33,), n_new=1, new_len=None, page=0, rot=None,
                 interleaved=False, axes=0, sections=None, layout="dense", four=False, queries=True, in_place=False,
                 seed=0, max_seq=None, x=None, unmapped=(), max_pos=None):
        rng = np.random.default_rng(seed)
        self.vp, self.lens, self.n_new, self.four, self.page = vp, lens, n_new, four, page
        H, Hkv = heads
        B, T = len(lens), max_seq or max(max(lens), 1)
        rot = dim if rot is None else rot
        dt = torch.float32 if dtype == "fp32" else torch.bfloat16
        self.ns = [min(n_new, L) if new_len is None else new_len[b] for b, L in enumerate(lens)]
        qkv = torch.from_numpy(rng.standard_normal((B, n_new, H + 2 * Hkv, dim)) * 3).to(dt)
        if x is not None:
            qkv[:, :, H:] = x.to(dt)
        self.qkv = qkv.cuda()
        self.q_in = self.qkv[:, :, :H] if queries else None
        self.k_in, self.v_in = self.qkv[:, :, H: H + Hkv], self.qkv[:, :, H + Hkv:]
        self.q_out = None
        if queries:
            self.q_out = self.q_in if in_place else torch.full((B, n_new, H, dim), -5.0, dtype=dt, device="cuda")
        places = np.stack([np.arange(n_new) + L - n for L, n in zip(lens, self.ns)])
        max_pos = max_pos or T + 7
        self.rotation = None
        pairs = rot // 2
        pos = None
        if rot:
            angle = np.arange(max_pos)[:, None] * (1000.0 ** (-np.arange(pairs) / pairs))
            table = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
            self.table = torch.from_numpy(table).cuda()
            if axes:
                pos = rng.integers(0, max_pos, (axes, B, n_new)).astype(np.int32)
                self.pos = torch.from_numpy(pos).cuda()
            parts = sections or ([pairs] if not axes else [pairs - (pairs // 3) * (axes - 1)] + [pairs // 3] * (axes - 1))
            self.rotation = vp.make_rotation(self.table, interleaved, self.pos if axes else None, parts)
            axis = np.repeat(np.arange(len(parts)), parts)
            at = np.broadcast_to(places[..., None], (B, n_new, pairs)) if pos is None else pos[axis].transpose(1, 2, 0)
            at = np.clip(at, 0, max_pos - 1)
            cos, sin = table[at, np.arange(pairs)][:, :, None], table[at, np.arange(pairs) + pairs][:, :, None]
        f = qkv.float().numpy()
        turn = (lambda y, t: O4.rotate(y, cos, sin, interleaved, t)) if rot else (lambda y, t: y.astype(t))
        q32, k32 = turn(f[:, :, :H], np.float32), turn(f[:, :, H: H + Hkv], np.float32)
        self.q64, self.k64 = turn(f[:, :, :H], np.float64), turn(f[:, :, H: H + Hkv], np.float64)
        if rot:
            self.k_mag = O4.rotate(np.abs(f[:, :, H: H + Hkv]), np.abs(cos), -np.abs(sin), interleaved, np.float64)
            self.k_mag = np.maximum(np.abs(self.k_mag), np.abs(O4.rotate(np.abs(f[:, :, H: H + Hkv]), np.abs(cos),
                                                                         np.abs(sin), interleaved, np.float64)))
        else:
            self.k_mag = np.zeros_like(self.k64)
        self.want_q = torch.from_numpy(q32).to(dt)
        self.want_k, self.want_v = torch.from_numpy(k32).to(dt), qkv[:, :, H + Hkv:]
        for b, n in enumerate(self.ns):  # rows that are no new tokens
            self.want_q[b, n:] = qkv[b, n:, :H] if in_place else -5.0
        self.bf16 = dtype == "bf16"
        # caches: whatever they hold must stay there outside the new tokens' places
        P = -(-T // page) if page else 0
        lead, rows = (B * P + 2, page) if page else (B, T)
        self.table_of_pages = None
        if page:
            table = rng.permutation(lead)[: B * P].reshape(B, P).astype(np.int32)
            for b, p in unmapped:
                table[b, p] = -1 if (b + p) % 2 else lead + 3
            self.tab = table
            self.table_of_pages = torch.from_numpy(table).cuda()
        if four:
            make = lambda: (torch.from_numpy(rng.integers(0, 256, (lead, Hkv, rows, dim // 2)).astype(np.uint8)),  # noqa: E731
                            torch.from_numpy(rng.random((lead, Hkv, rows, dim // 32))).half())
        else:
            make = lambda: (torch.from_numpy(rng.standard_normal((lead, Hkv, rows, dim))).to(dt),)  # noqa: E731
        self.before = [make(), make()]
        self.caches = [tuple(_layout(y, layout) for y in c) for c in self.before]
        if four:
            kv = (lambda c: vp.kv4_paged(*c, self.table_of_pages)) if page else (lambda c: vp.kv4_contiguous(*c))
            self.held = [torch.full((B, n_new, Hkv, dim), -5.0, dtype=dt, device="cuda") for _ in range(2)]
        else:
            kv = (lambda c: vp.kv_paged(*c, self.table_of_pages)) if page else (lambda c: vp.kv_contiguous(*c))
        self.kc, self.vc = (kv(c) for c in self.caches)
        self.seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.new = None if new_len is None else torch.tensor(new_len, dtype=torch.int32, device="cuda")
        self.ctx = vp.vp_init(vp.make_config(B, H, Hkv, dim, 0, T, vp.VP_FP32 if dtype == "fp32" else vp.VP_BF16,
                                             1 if page else 0, page or 16))
        self.B = B

    def call(self, stream=None):
        vp = self.vp
        rq = None if self.q_in is None else vp.rows(self.q_in)
        ro = None if self.q_in is None else vp.rows(self.q_out)
        args = (self.ctx, self.B, self.n_new, rq, vp.rows(self.k_in), vp.rows(self.v_in), self.seq, self.rotation, ro,
                self.kc, self.vc)
        if self.four:
            vp.vp_append4(*args, new_len=self.new, k_held=vp.rows(self.held[0]), v_held=vp.rows(self.held[1]), stream=stream)
        else:
            vp.vp_append(*args, new_len=self.new, stream=stream)

    def place(self, b, i):
        at = self.lens[b] - self.ns[b] + i
        if not self.page:
            return b, at
        page = int(self.tab[b, at // self.page])
        return (page, at % self.page) if 0 <= page < self.before[0][0].shape[0] else None

    def check(self, errors=False):
        if not errors:
            self.vp.vp_check_errors(self.ctx)
        if self.q_out is not None:
            assert torch.equal(self.q_out.cpu().view(torch.uint8), self.want_q.contiguous().view(torch.uint8))
        for want64, want, before, cache, held in zip((self.k64, None), (self.want_k, self.want_v), self.before, self.caches,
                                                     self.held if self.four else (None, None)):
            expect = [y.clone() for y in before]
            if self.four:
                codes, scale = O4.quantise(want.float().numpy())
                vals = torch.from_numpy(O4.values(codes, scale)).to(want.dtype)
                parts = (torch.from_numpy(O4.pack(codes)), torch.from_numpy(scale).half())
                for b, n in enumerate(self.ns):
                    vals[b, n:] = -5.0
                got = held.cpu()
                assert torch.equal(torch.isnan(got), torch.isnan(vals))
                assert torch.equal(got[~torch.isnan(got)], vals[~torch.isnan(vals)])
            else:
                parts = (want,)
            for b, n in enumerate(self.ns):
                for i in range(n):
                    at = self.place(b, i)
                    if at is not None:
                        for e, y in zip(expect, parts):
                            e[at[0], :, at[1]] = y[b, i]
            for e, got in zip(expect, cache):
                got = got.cpu()
                if got.dtype == torch.half:
                    assert torch.equal(torch.isnan(got), torch.isnan(e))
                    assert torch.equal(got[~torch.isnan(got)], e[~torch.isnan(e)])
                elif got.dtype == torch.uint8:
                    nan = torch.isnan(expect[1]).repeat_interleave(16, -1)  # codes of such groups are not defined
                    assert torch.equal(got[~nan], e[~nan])
                else:
                    assert torch.equal(got.contiguous().view(torch.uint8), e.contiguous().view(torch.uint8))
            if want64 is not None and not self.four:
                err = np.abs(want.double().numpy() - want64)
                tol = 3 * 2.0 ** -24 * self.k_mag + (2.0 ** -8 * np.abs(want64) * (1 + 2.0 ** -20) if self.bf16 else 0)
                assert (err <= tol + 1e-30).all()

    def run(self, errors=False):
        self.call()
        torch.cuda.synchronize()
        self.check(errors)
        self.vp.vp_free(self.ctx)


BOTH = pytest.mark.parametrize("four", [False, True], ids=["plain", "four"])
TYPES = pytest.mark.parametrize("dtype", ["bf16", "fp32"])


@BOTH
@TYPES
@pytest.mark.parametrize("heads,dim", [((8, 2), 64), ((28, 4), 128), ((8, 1), 128), ((5, 5), 64), ((1, 1), 128), ((16, 1), 64)])
@pytest.mark.parametrize("page", [0, 16])
def test_heads_and_types(vp, four, dtype, heads, dim, page):
    Append(vp, heads, dim, dtype, lens=(37, 1, 16, 300), page=page, four=four).run()


@BOTH
@TYPES
@pytest.mark.parametrize("dim,rot", [(64, 0), (64, 16), (64, 32), (64, 48), (128, 64), (128, 96), (128, 112), (128, 16)])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "pairs"])
def test_part_of_a_row_is_rotated(vp, four, dtype, dim, rot, interleaved):
    Append(vp, (6, 3), dim, dtype, lens=(9, 40), n_new=5, rot=rot, interleaved=interleaved, four=four).run()


@BOTH
@pytest.mark.parametrize("axes,sections", [(1, None), (2, [5, 27]), (3, [8, 12, 12]), (3, [7, 13, 12]), (3, [0, 32, 0]), (3, [32, 0, 0])])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "pairs"])
def test_positions_on_axes(vp, four, axes, sections, interleaved):
    Append(vp, (4, 2), 64, "bf16", lens=(50, 61), n_new=7, axes=axes, sections=sections, interleaved=interleaved,
           four=four).run()


@BOTH
@TYPES
@pytest.mark.parametrize("layout", ["dense", "swapped", "outer", "padded"])
@pytest.mark.parametrize("page", [0, 1, 8, 64])
def test_layouts(vp, four, dtype, layout, page):
    Append(vp, (4, 2), 64, dtype, lens=(70, 129, 3), n_new=6, new_len=(6, 2, 3), page=page, layout=layout, four=four).run()


@BOTH
@pytest.mark.parametrize("page", [0, 16])
def test_ragged_new_tokens(vp, four, page):
    Append(vp, (8, 2), 128, "bf16", lens=(20, 1, 0, 64, 33), n_new=9, new_len=(9, 1, 0, 0, 5), page=page, four=four).run()


@BOTH
def test_prompt(vp, four):
    Append(vp, (28, 4), 128, "bf16", lens=(1027, 640), n_new=1027, new_len=(1027, 333), four=four).run()


@BOTH
def test_room_behind_the_sequences(vp, four):
    Append(vp, (4, 2), 64, "bf16", lens=(5, 17), n_new=4, max_seq=40, page=16, four=four).run()


@BOTH
@TYPES
def test_queries_in_place_and_none(vp, four, dtype):
    Append(vp, (8, 2), 64, dtype, lens=(30, 12), n_new=3, new_len=(3, 1), in_place=True, four=four).run()
    Append(vp, (8, 2), 64, dtype, lens=(30, 12), n_new=3, queries=False, four=four).run()


@BOTH
def test_pages_that_are_not_mapped(vp, four):
    a = Append(vp, (4, 2), 64, "bf16", lens=(40, 33), n_new=20, page=8, unmapped=((0, 3), (1, 2)), four=four)
    a.call()
    with pytest.raises(vp.VPError) as e:
        vp.vp_check_errors(a.ctx)
    assert e.value.status == vp.VP_ERR_DEVICE_PRECOND and "block table" in str(e.value)
    a.check()


@BOTH
def test_lengths_out_of_range_append_nothing(vp, four):
    a = Append(vp, (4, 2), 64, "bf16", lens=(40, 33, 12), n_new=2, four=four, max_seq=40)
    a.seq = torch.tensor([41, 33, -1], dtype=torch.int32, device="cuda")
    a.want_q[0] = a.want_q[2] = -5.0
    a.ns = [0, 2, 0]
    a.call()
    with pytest.raises(vp.VPError, match="seq_len"):
        vp.vp_check_errors(a.ctx)
    a.check()
    b = Append(vp, (4, 2), 64, "bf16", lens=(40, 33, 1), n_new=2, four=four, new_len=(2, 1, 1))
    b.new = torch.tensor([3, 1, 2], dtype=torch.int32, device="cuda")
    b.want_q[0] = b.want_q[2] = -5.0
    b.ns = [0, 1, 0]
    b.call()
    with pytest.raises(vp.VPError, match="new_len"):
        vp.vp_check_errors(b.ctx)
    b.check()


def test_positions_outside_the_table_are_clamped(vp):
    a = Append(vp, (4, 2), 64, "bf16", lens=(40, 33), n_new=2, max_pos=39)
    a.call()
    with pytest.raises(vp.VPError, match="rotation table"):
        vp.vp_check_errors(a.ctx)
    a.check()


@TYPES
def test_values_at_the_edges_of_four_bits(vp, dtype):
    """Zeros, one large value, the least and the largest scales, halves between two
    codes, infinities and NaN; the values are not rotated."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((2, 3, 8, 64)).astype(np.float32)
    x[0, 0, 0] = 0
    x[0, 0, 1, :32] = 2.0 ** -20
    x[0, 0, 2, 5] = 1e9
    x[0, 0, 3, 40] = 3e38
    x[0, 1, 0] = np.tile(np.arange(32) / 2 - 7.5, 2)          # steps of exactly 1: every half is a tie
    x[0, 1, 1] = np.tile(7.5 - np.arange(32) / 2, 2) * 2.0 ** -9
    x[0, 1, 2, 3] = np.inf
    x[0, 1, 3, 33] = -np.inf
    x[0, 2, 0, 0] = np.nan
    x[0, 2, 1, 63] = np.nan
    x[0, 2, 2] = 2.0 ** -130
    x[1, 0] *= 2.0 ** -15
    x[1, 1] *= 40000.0
    a = Append(vp, (4, 4), 64, dtype, lens=(9, 3), n_new=3, rot=0, four=True, x=torch.from_numpy(x))
    a.run()


def test_another_stream_and_a_captured_call(vp):
    a = Append(vp, (8, 2), 64, "bf16", lens=(30, 12), n_new=3, page=16, four=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            a.call()
    for c, b in zip(a.caches, a.before):
        for y, z in zip(c, b):
            y.copy_(z)
    a.seq.copy_(torch.tensor([29, 11]))     # the lengths of a replay are what the array holds then
    g.replay()
    a.seq.copy_(torch.tensor([30, 12]))
    g.replay()
    torch.cuda.synchronize()
    vp.vp_check_errors(a.ctx)
    assert torch.equal(a.held[0].cpu(), torch.from_numpy(O4.values(*O4.quantise(a.want_k.float().numpy()))).to(torch.bfloat16))


@BOTH
def test_refusals(vp, four):
    a = Append(vp, (8, 2), 64, "bf16", lens=(30, 12), n_new=2, four=four, page=16)
    call = vp.vp_append4 if four else vp.vp_append
    good = dict(batch=2, n_new=2, q=vp.rows(a.q_in), k=vp.rows(a.k_in), v=vp.rows(a.v_in), seq_len=a.seq,
                rotation=a.rotation, q_out=vp.rows(a.q_out), k_cache=a.kc, v_cache=a.vc)
    before = [y.clone() for c in a.caches for y in c]

    def status(**change):
        return call(a.ctx, **{**good, **change}, check=False)

    def but(struct, **fields):
        copy = type(struct).from_buffer_copy(struct)
        for name, value in fields.items():
            setattr(copy, name, value)
        return copy

    bad = vp.VP_ERR_INVALID_ARG
    assert status(batch=-1) == bad and status(n_new=-1) == bad
    assert status(batch=3) == vp.VP_ERR_CAPACITY and status(n_new=31) == vp.VP_ERR_CAPACITY
    assert status(q=None) == bad and status(q_out=None) == bad
    assert status(k=None) == bad and status(v=None) == bad and status(seq_len=None) == bad
    assert status(k_cache=None) == bad and status(v_cache=None) == bad
    assert status(k=but(good["k"], data=a.k_in.data_ptr() + 2)) == bad
    assert status(v=but(good["v"], stride_n=3)) == bad
    assert status(q_out=but(good["q_out"], stride_h=0)) == bad
    assert status(q_out=but(good["q"], stride_n=1024)) == bad                   # over q, in another order
    r = a.rotation
    for change in (dict(cos_sin=None), dict(max_pos=0), dict(rot_dim=24), dict(rot_dim=0), dict(rot_dim=80),
                   dict(interleaved=2), dict(axes=0), dict(axes=4), dict(axes=2)):
        assert status(rotation=but(r, **change)) == bad, change
    three = but(r, pos=a.seq.data_ptr(), axes=3)
    three.sections[:] = [16, 15, 0]
    assert status(rotation=three) == bad
    three.sections[:] = [40, -8, 0]
    assert status(rotation=three) == bad
    assert status(k_cache=but(a.kc, block_table=None)) == bad and status(v_cache=but(a.vc, num_pages=0)) == bad
    if four:
        assert status(k_cache=but(a.kc, codes=None)) == bad and status(k_cache=but(a.kc, scales=None)) == bad
        assert status(k_cache=but(a.kc, code_stride_t=24)) == bad and status(v_cache=but(a.vc, scale_stride_t=1)) == bad
        assert status(v_cache=but(a.vc, scales=a.vc.scales + 2)) == bad
        assert status(k_held=but(vp.rows(a.held[0]), stride_b=0)) == bad
    else:
        assert status(k_cache=but(a.kc, stride_t=-8)) == bad
    assert vp.vp_last_error(a.ctx)
    torch.cuda.synchronize()
    for y, z in zip([y for c in a.caches for y in c], before):
        assert torch.equal(y, z)
    assert status(batch=0) == vp.VP_OK and status(n_new=0) == vp.VP_OK
    vp.vp_check_errors(a.ctx)
