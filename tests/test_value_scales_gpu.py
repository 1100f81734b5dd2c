"""vp_attend4 with scales of V that lie far apart: over the groups of a token, over
the tokens of a group, and beside tokens whose weight or value is nothing.

Each element is held to a bound of its own terms, S = sum_j p_j |v_j| of its
dimension: a large scale in another group, or at a token that is worth nothing,
gives it no room.  From the arithmetic, as in test_attend4_gpu:
  logits   z_err = 2^-20 M (fp32: 2^-22 M more), M what a group's terms can sum to;
           of S: 2 z_err + 2^-21 (1 + |lse|) + 2^-19;
  bf16     P and its product with the scale are rounded to fp16: 2^-11 S each, and
           the output to bf16, 2^-8 of it;
  fp32     two fp16 terms each, 2^-21 S together;
  sums     rounded (tokens / 128 + 40) times at 2^-22 S;
  floor    below 2^-14 a term's rounding is 2^-25.  The row's largest P is 2^10 or
           more where a token's is taken, and a scale at least 2^-7 in the unit that
           its group has then (the least unit is 2^-15: scales below 2^-22 as that):
           2^-25 / 2^-7 / 2^10 = 2^-28 of the largest p, times 8 steps of the token's
           own scale; P's own floor, 2^-35, and what the tensor cores cut of such
           terms, 2^-41, are within a factor of two.  fp32: the second term is 2^11
           times larger, 2^-39.
A result of zeros must not pass."""

import numpy as np
import pytest
import torch

from tests.test_attend4_gpu import Case

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", ["bf16", "fp32"])
# Query rows per kv-head from 4 to 32: the kernel's four sizes, and two of fp32.
ROWS = pytest.mark.parametrize("heads,dim,n_new", [((8, 2), 64, 1), ((28, 4), 128, 2), ((8, 2), 64, 5), ((16, 2), 128, 4)])


@pytest.fixture(scope="module")
def vp(lib):
    assert torch.cuda.is_available()
    return lib


def check(a, nothing=0.9, lost=None):
    """Runs the case; of the elements, at least the share `nothing` must tell a zero from the result.
    lost: dimensions of sequence 0 that must not come out finite."""
    a.call()
    torch.cuda.synchronize()
    a.vp.vp_check_errors(a.ctx)
    if lost is not None:
        assert not torch.isfinite(a.out[0, :, :, lost]).any()
        a.out[0, :, :, lost] = torch.from_numpy(a.ref[0]["out"]).to(a.out)[:, :, lost]
    vstep = a.held[1][1].astype(np.float64)                          # [B, Hkv, T, groups]
    told = total = 0
    for b, ref in enumerate(a.ref):
        out, lse = a.out[b].double().cpu().numpy(), a.lse[b].double().cpu().numpy()
        n, L = a.ns[b], a.lens[b]
        H, Hkv = out.shape[1], vstep.shape[1]
        M, _ = a.bounds[b]
        ze = 2.0 ** -20 * M * (1 if a.bf16 else 1.25)
        near = np.abs(lse - ref["lse"])[:n]
        assert (near <= (ze + 2.0 ** -21 * (1 + np.abs(ref["lse"])))[:n] + 1e-30).all(), (b, near.max())
        rel = 2 * ze + 2.0 ** -21 * (1 + np.abs(ref["lse"])) + 2.0 ** -19 + (2.0 ** -10 if a.bf16 else 2.0 ** -21)
        tol = (rel[..., None] + 2.0 ** -22 * (L / 128 + 40)) * ref["absout"]
        # The floor: 8 steps of every token that the row sees (codes of 0 add nothing), p at most 1.
        steps = np.maximum(np.abs(vstep[b]), 2.0 ** -22).repeat(32, -1).repeat(H // Hkv, 0)  # [H, T, D]
        floor = 8 * (2.0 ** -27 if a.bf16 else 2.0 ** -38)
        for i in range(n):
            js = ref["mask"][i] if a.weightless is None else ref["mask"][i] & ~a.weightless
            tol[i] += floor * steps[:, :L][:, js].sum(1)
        if a.bf16:
            tol += 2.0 ** -8 * np.abs(ref["out"]) * (1 + 2.0 ** -6)
        err = np.abs(out - ref["out"])[:n]
        bad = ~(err <= tol[:n])
        assert not bad.any(), (b, bad.mean(), np.argwhere(bad)[:3], (err / np.maximum(ref["absout"][:n], 1e-300)).max())
        told += (np.abs(ref["out"])[:n] > tol[:n]).sum()
        total += err.size
    assert told >= nothing * total
    a.vp.vp_free(a.ctx)


def case(vp, *args, weightless=None, **kw):
    a = Case(vp, *args, **kw)
    a.weightless = weightless
    return a


def fit_bits(x):
    """Scales as vp_append4 makes them: four significant bits."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 16) / 16, e)


@TYPES
@ROWS
@pytest.mark.parametrize("big", [2.5, 4096.0, 61440.0])
@pytest.mark.parametrize("small", [0.03, 0.001])
def test_one_group_of_one_token(vp, dtype, heads, dim, n_new, big, small):
    """The others' scales are small, in that token and everywhere else."""
    def steps(held, rng):
        step = held[1][1]
        step[:] = fit_bits(small * rng.uniform(0.5, 1.0, step.shape))
        step[:, :, 90, 0] = big
        step[:, :, 601, 1] = big

    check(case(vp, heads, dim, dtype, lens=(700, 92), n_new=n_new, steps=steps))


@TYPES
@ROWS
@pytest.mark.parametrize("small", [0.35, 0.03, 0.003])
def test_one_dimension_is_large_everywhere(vp, dtype, heads, dim, n_new, small):
    def steps(held, rng):
        step = held[1][1]
        step[:] = fit_bits(small * rng.uniform(0.5, 1.0, step.shape))
        step[..., 0] = fit_bits(2.7 * rng.uniform(0.9, 1.2, step[..., 0].shape))

    check(case(vp, heads, dim, dtype, lens=(1500, 300), n_new=n_new, steps=steps))


@TYPES
@ROWS
@pytest.mark.parametrize("big", [None, 2.7, 1000.0])
def test_behind_a_token_of_large_weight_and_no_value(vp, dtype, heads, dim, n_new, big):
    """The first token's logit is 8 above the others': it takes most of the weight and adds nothing."""
    H, L = heads[0], 2048
    q = torch.from_numpy(np.random.default_rng(1).standard_normal((1, n_new, H, dim)))
    q[..., 5] = 8 * dim ** 0.5 / 7

    def steps(held, rng):
        (kcode, kstep), (vcode, vstep) = held
        kcode[..., 5] = 8
        kcode[:, :, 0] = 8
        kcode[:, :, 0, 5] = 15
        kstep[:, :, 0] = 1.0
        vstep[:] = fit_bits(0.03 * rng.uniform(0.5, 1.0, vstep.shape))
        vcode[:, :, 0] = 8
        if big is not None:
            vstep[..., 0] = fit_bits(big * rng.uniform(0.9, 1.2, vstep[..., 0].shape))

    none = np.zeros(L, bool)
    none[0] = True
    check(case(vp, heads, dim, dtype, lens=(L,), n_new=n_new, steps=steps, weightless=none,
               q=q.to(torch.float32 if dtype == "fp32" else torch.bfloat16)), nothing=0.8)


@TYPES
@ROWS
@pytest.mark.parametrize("big", [None, 2.7, 1000.0])
def test_every_warp_behind_such_a_token(vp, dtype, heads, dim, n_new, big):
    """More sequences than there are CTAs, so that one goes through most of a sequence,
    and such a token in front of each of its warps' parts."""
    B, H, L = 512 // heads[1], heads[0], 384
    q = torch.from_numpy(np.random.default_rng(1).standard_normal((B, n_new, H, dim)))
    q[..., 5] = 8 * dim ** 0.5 / 7
    none = np.arange(L) % 32 == 0
    none[128:] = False

    def steps(held, rng):
        (kcode, kstep), (vcode, vstep) = held
        kcode[..., 5] = 8
        kcode[:, :, none] = 8
        kcode[:, :, none, 5] = 15
        kstep[:, :, none] = 1.0
        vstep[:] = fit_bits(0.03 * rng.uniform(0.5, 1.0, vstep.shape))
        vcode[:, :, none] = 8
        if big is not None:
            vstep[..., 0] = fit_bits(big * rng.uniform(0.9, 1.2, vstep[..., 0].shape))

    check(case(vp, heads, dim, dtype, lens=(L,) * B, n_new=n_new, steps=steps, weightless=none,
               q=q.to(torch.float32 if dtype == "fp32" else torch.bfloat16)), nothing=0.8)


@TYPES
@ROWS
@pytest.mark.parametrize("small", [0.3, 0.004])
def test_large_scales_of_no_value_in_the_same_group(vp, dtype, heads, dim, n_new, small):
    """Scales from 2 to 61440 at one token in five, their codes those of 0."""
    L = 700
    none = np.random.default_rng(3).random(L) < 0.2

    def steps(held, rng):
        vcode, vstep = held[1]
        vstep[:] = fit_bits(small * rng.uniform(0.5, 1.0, vstep.shape))
        large = np.minimum(fit_bits(2.0 ** rng.uniform(1, 16, vstep.shape)), 61440.0)
        vstep[:, :, none] = large[:, :, none]
        vcode[:, :, none] = 8

    check(case(vp, heads, dim, dtype, lens=(L,), n_new=n_new, steps=steps, weightless=none))


@TYPES
@ROWS
def test_scales_of_every_size(vp, dtype, heads, dim, n_new):
    """From the least that vp_append4 makes to the largest, token by token and group by group."""
    def steps(held, rng):
        vstep = held[1][1]
        vstep[:] = np.clip(fit_bits(2.0 ** rng.uniform(-14, 16, vstep.shape)), 2.0 ** -14, 61440.0)

    check(case(vp, heads, dim, dtype, lens=(333, 40), n_new=n_new, steps=steps))


@TYPES
@ROWS
def test_scales_of_other_producers(vp, dtype, heads, dim, n_new):
    """Eleven bits, either sign, zeros, and the least fp16 numbers beside the largest; the latter's value is 0."""
    L = 300
    none = np.arange(L) % 3 == 1

    def steps(held, rng):
        vcode, vstep = held[1]
        vstep[:] = (2.0 ** -24 * rng.integers(-5, 6, vstep.shape)).astype(np.float16)
        vstep[:, :, ::7] = (rng.standard_normal(vstep[:, :, ::7].shape) * 2.0 ** -22).astype(np.float16)
        vstep[:, :, none] = (65504.0 * rng.choice([-1, 1, 0.001], vstep[:, :, none].shape)).astype(np.float16)
        vcode[:, :, none] = 8

    check(case(vp, heads, dim, dtype, lens=(L,), n_new=n_new, steps=steps, weightless=none), nothing=0.6)


@TYPES
@pytest.mark.parametrize("page", [0, 1, 16])
@pytest.mark.parametrize("window,sinks", [(-1, 0), (37, 5), (200, 0)])
def test_windows_and_pages(vp, dtype, page, window, sinks):
    def steps(held, rng):
        vstep = held[1][1]
        vstep[:] = fit_bits(0.01 * rng.uniform(0.5, 1.0, vstep.shape))
        vstep[:, :, ::50, 1] = 300.0

    check(case(vp, (8, 2), 64, dtype, lens=(400, 77, 130), n_new=2, page=page, window=window, sinks=sinks, steps=steps))


@TYPES
@pytest.mark.parametrize("heads,dim", [((8, 2), 64), ((28, 4), 128), ((32, 2), 128)])
@pytest.mark.parametrize("scale", [float("inf"), float("-inf"), float("nan")])
def test_a_scale_that_is_not_finite_stays_in_its_group(vp, dtype, heads, dim, scale):
    """Among scales of every size, which take several passes; the other groups and sequences are as without it."""
    def steps(held, rng):
        vstep = held[1][1]
        vstep[:] = np.clip(fit_bits(2.0 ** rng.uniform(-14, 16, vstep.shape)), 2.0 ** -14, 61440.0)

    a = case(vp, heads, dim, dtype, lens=(300, 77), steps=steps)
    a.tensors[3][0, :, 130, 1] = scale
    a.tensors[3][0, :, 131, 1] = float("inf")
    check(a, lost=slice(32, 64))


@TYPES
def test_prompts(vp, dtype):
    """bf16: by way of staged rows, which round 300 times a code; fp32: sixteen rows at a time."""
    def steps(held, rng):
        vstep = held[1][1]
        vstep[:] = fit_bits(0.01 * rng.uniform(0.5, 1.0, vstep.shape))
        vstep[:, :, ::50, 1] = 300.0

    check(case(vp, (8, 2), 64, dtype, lens=(150, 90), n_new=70, steps=steps, rounded=dtype == "bf16"))


def test_equal_bits_in_a_graph(vp):
    """Turns that are done in several passes, captured and replayed."""
    def steps(held, rng):
        vstep = held[1][1]
        vstep[:] = np.clip(fit_bits(2.0 ** rng.uniform(-14, 16, vstep.shape)), 2.0 ** -14, 61440.0)

    a = case(vp, (28, 4), 128, "bf16", lens=(900, 129), n_new=2, page=16, steps=steps)
    a.call()
    torch.cuda.synchronize()
    out, lse = a.out.clone(), a.lse.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            a.call()
        for _ in range(2):
            a.out.fill_(float("nan"))
            g.replay()
            s.synchronize()
            assert torch.equal(a.out, out) and torch.equal(a.lse, lse)
    check(a)
