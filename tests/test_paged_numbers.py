"""Numbers of the paged attention at their limits, against 64 bits with errors that are relative to the scores."""
import math

import pytest
import torch

from paged_plain import UNIT, ceil_div
from paged_wide import widen
from test_paged_cache import BF16, FP16, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    return g


def exact(c, score_error):
    """(out, lse, out_tolerance, lse_tolerance) in 64 bits of a Case whose values are finite.  With the 32-bit sums of D products, a
    score is off by D * 2^-23 * scale * sum|q||k| and by score_error(its size before the bias, its size); a weight by twice
    that and by its rounding to the cache's type (relative: its unit); the result rounds once more."""
    o = c.opts
    t, heads, d = c.q.shape
    group, page, scale, u = heads // c.kp.shape[1], c.kp.shape[2], 1.0 / math.sqrt(d), UNIT[c.q.dtype]
    out = torch.zeros((t, heads, d), dtype=torch.float64, device="cuda")
    lse = torch.full((t, heads), -math.inf, dtype=torch.float64, device="cuda")
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    starts = c.starts.tolist()
    for r, length in enumerate(c.lens):
        rows = slice(starts[r], starts[r + 1])
        p = torch.arange(length - c.new[r], length, device="cuda")[:, None]
        j = torch.arange(length, device="cuda")[None]
        sees = j >= 0
        if o["causal"]:
            sees = sees & (j <= p)
        if o["window"]:
            sees = sees & (j > p - o["window"])
        sees = sees.expand(c.new[r], length)
        ids = c.tables[r, : ceil_div(length, page)].long()
        for h in range(heads):
            k = c.kp[ids, h // group].reshape(-1, d)[:length].double()
            v = c.vp[ids, h // group].reshape(-1, d)[:length].double()
            q = c.q[rows, h].double()
            x = q @ k.T * scale
            if o["softcap"]:
                x = o["softcap"] * torch.tanh(x / o["softcap"])
            before = x
            if o["slopes"] is not None:
                x = x + o["slopes"][h].double() * (j - p)
            e = d * 2.0 ** -23 * scale * (q.abs() @ k.abs().T) + score_error(before.abs(), x.abs())
            eb = torch.where(sees, e, 0.0).amax(1, keepdim=True)
            x = torch.where(sees, x, -math.inf)
            lse[rows, h] = torch.logsumexp(x, 1)
            w = torch.exp(x - lse[rows, h][:, None])
            out[rows, h] = w @ v
            out_tol[rows, h] = u * out[rows, h].abs() + (u + 2 * eb + 2.0 ** -18) * (w @ v.abs())
            lse_tol[rows, h] = eb[:, 0] + 2.0 ** -18 + 2.0 ** -21 * lse[rows, h].abs()
    return out, lse, out_tol, lse_tol


def check(gorio, c, score_error):
    bounds = exact(c, score_error)
    got = within(c.run(gorio), *bounds)
    c.tables = widen(c.tables, c.kp.shape[2])                 # the chunk kernel, unless one token's rows are few
    within(c.run(gorio), *bounds)
    return got


def within(got, out, lse, out_tol, lse_tol):
    off = (got["out"].double() - out).abs() / out_tol
    assert (off <= 1).all(), f"out is off by {off.max().item():.3g} of the tolerance"
    off = (got["lse"].double() - lse).abs() / lse_tol
    assert (off <= 1).all(), f"lse is off by {off.max().item():.3g} of the tolerance"
    return got


# Above a quarter of the cap its arithmetic is that of 1 - 2 / (1 + e^2u), three roundings and two approximations of a unit each:
# 2^-22 of the cap, 2^-20 of the score; below it is a series that is good to 2^-21, and the bias adds a rounding of its size.
CAP_ERROR = lambda capped, biased: 2.0 ** -19 * capped + 2.0 ** -21 * biased          # noqa: E731


@pytest.mark.parametrize("new,lens", [([1, 1], [300, 129]), ([250, 3], [430, 200])])
@pytest.mark.parametrize("cap", [1e2, 1e3, 1e4, 1e6, 1e9, 1e30, 3e38])
@pytest.mark.parametrize("dtype,dim,slopes", [(BF16, 128, False), (FP16, 64, True), (FP16, 96, False)])
def test_attention_caps_far_above_the_scores(gorio, new, lens, cap, dtype, dim, slopes):
    """A score that is small beside the cap stays what it is, however large the cap."""
    check(gorio, Case(new, lens, dim=dim, dtype=dtype, softcap=cap, slopes=slopes, seed=3), CAP_ERROR)


@pytest.mark.parametrize("new,lens", [([1, 1], [300, 129]), ([250, 3], [430, 200])])
@pytest.mark.parametrize("cap", [2.0, 20.0, 100.0, 1000.0])
@pytest.mark.parametrize("dtype,dim", [(BF16, 128), (FP16, 64)])
def test_attention_caps_across_the_scores(gorio, new, lens, cap, dtype, dim):
    """Scores of some hundreds, from far below the cap to far above it, in one row."""
    check(gorio, Case(new, lens, dim=dim, dtype=dtype, softcap=cap, sharp=30.0, seed=4), CAP_ERROR)


@pytest.mark.parametrize("new", [1, 250])
def test_attention_float16_weights_far_below_the_largest(gorio, new):
    """Forty thousand keys of a weight 2^-25.6 each beside one of 1: together they are the whole result."""
    c = Case([new], [40000], heads=4, kv_heads=2, dim=64, page=64, dtype=FP16)
    c.kp.zero_(), c.vp.fill_(1.0), c.q.fill_(1.0)
    first = c.tables[0, 0].item()
    c.kp[first, :, 0], c.vp[first, :, 0] = 2.21875, 0.0
    got = check(gorio, c, lambda capped, biased: 2.0 ** -21 * biased)
    assert (got["out"] > 7e-4).all()


@pytest.mark.parametrize("new,lens", [([1, 1], [300, 129]), ([250, 3], [430, 200]), ([250], [9000])])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_attention_of_even_and_of_rising_scores(gorio, new, lens, dtype):
    """The largest weights the types hold: all keys alike, and keys whose scores rise along the axis, in steps that do not and that do move
    the reference of the weights."""
    for step in (0.0, 0.01, 0.07):
        c = Case(new, lens, heads=4, kv_heads=2, dim=64, dtype=dtype, seed=9)
        c.q.fill_(1.0), c.kp.zero_()
        for r, n in enumerate(lens):
            for i in range(ceil_div(n, 16)):
                c.kp[c.tables[r, i].item(), :, :, 0] = 8.0 * step * (16.0 * i + torch.arange(16, device="cuda"))
        check(gorio, c, lambda capped, biased: 2.0 ** -21 * biased)
