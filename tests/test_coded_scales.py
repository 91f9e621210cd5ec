"""Attention over codes whose scales differ by many powers of two, with tolerances that count from what each row sees."""
import math

import pytest
import torch

from more_plain import UNIT
from paged_plain import ceil_div
from paged_wide import widen
from test_quantized import E4M3, INT8, Coded, encode

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    return g


def keys_of(c, r, j):
    """Pages and places of the keys j of request r."""
    return c.tables[r, j // c.page].long(), j % c.page


def check(c, got, rows=slice(None)):
    """One request's rows against 64 bits.  A weight times its value's scale is rounded to float16 where the row's largest one is 2^3 or more (2^7, or 2^4
    less where the tile's scales lie within 2^4): by 2^-11 of itself or, below the normal numbers, by 2^-25, which is 2^-28 of the largest.  The other errors are those of more_plain.attend: e of a score,
    2e + 2^-18 of a weight, the result's own rounding; and, as weights count from a maximum that holds the logarithm of a scale (`far`, at most 80), four
    roundings of numbers of that size, 2^-24 each: score minus maximum, maximum minus 15, times ln 2, logarithm of the sum."""
    n, length = c.new[0], c.lens[0]
    ids = c.tables[0, :ceil_div(length, c.page)]
    k, v = c._rows(c.kp, c.ks, ids, length), c._rows(c.vp, c.vs, ids, length)
    d, heads = k.shape[2], c.q.shape[1]
    size = c.vs[ids.clamp(0, c.vs.shape[0] - 1).long()].transpose(0, 1).flatten(1)[:, :length].abs().double()
    far = size.log2().clamp(-80.0, 80.0).abs().max().item() * 2.0 ** -22
    at, j = torch.arange(length - n, length, device="cuda")[rows], torch.arange(length, device="cuda")
    for h in range(heads):
        q = c.q[rows, h].double()
        kh, vh = k[h // (heads // k.shape[0])], v[h // (heads // k.shape[0])]
        x = q @ kh.T / math.sqrt(d)
        e = (d * 2.0 ** -23 / math.sqrt(d) * (q.abs() @ kh.abs().T) + 2.0 ** -21 * x.abs()).where(j <= at[:, None], 0.0).amax(1, keepdim=True)
        x = x.masked_fill(j > at[:, None], -math.inf)
        lse = torch.logsumexp(x, 1, keepdim=True)
        w = torch.exp(x - lse)
        out, sums = w @ vh, w @ vh.abs()
        largest = (w * vh.abs().amax(1)).amax(1, keepdim=True)
        tol = UNIT[c.q.dtype] * out.abs() + (2.0 ** -11 + 2 * e + 2.0 ** -18 + far) * sums + length * 2.0 ** -28 * largest
        off = (got["out"][rows, h].double() - out).abs()
        assert (off <= tol).all(), f"head {h}: out is off by {(off / tol).max().item():.3g} of the tolerance"
        off, tol = (got["lse"][rows, h].double() - lse[:, 0]).abs(), e[:, 0] + 2.0 ** -18 + far + 2.0 ** -21 * lse[:, 0].abs()
        assert (off <= tol).all(), f"head {h}: lse is off by {(off / tol).max().item():.3g} of the tolerance"




@pytest.mark.parametrize("form", [E4M3, INT8])
@pytest.mark.parametrize("new", [1, 100])
def test_thousands_of_values_that_are_zero(gorio, form, new):
    """Scores rise by eight octaves behind the first tile; the values there have scale 0, but for the last ones.  Alone, in parts, and as one of many
    requests over the same keys, which a block takes whole."""
    n = 20000
    c = Coded([new], [n], heads=8, kv_heads=4, dim=64, form=form, page=64, seed=1)
    c.q.fill_(1.0)
    codes, scales = encode(torch.full((4, 64), 0.6875, device="cuda"), form)   # 0.6875 * 64 / 8 = 5.5
    pages, places = keys_of(c, 0, torch.arange(n, device="cuda"))
    c.kp.view(torch.uint8)[pages, :, places], c.ks[pages, :, places] = codes.view(torch.uint8), scales
    c.ks[pages[:128], :, places[:128]] = 0.0
    c.vs[pages[:n - 200], :, places[:n - 200]] = 0.0
    c.tables = widen(c.tables, c.page)
    check(c, c.run(gorio))
    many = 80
    starts = torch.arange(many + 1, dtype=torch.int32, device="cuda") * new
    got = gorio.paged_attention_quantized(c.q.repeat(many, 1, 1), c.kp, c.vp, c.ks, c.vs, c.tables.expand(many, -1), c.lengths.repeat(many), starts, new,
                                          want_lse=True)
    for r in range(0, many, 13):
        check(c, {k: got[k][r * new:(r + 1) * new] for k in ("out", "lse")})


@pytest.mark.parametrize("form", [E4M3, INT8])
@pytest.mark.parametrize("new", [1, 5, 150])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("down", [10, 24, 32, 40, None])
def test_the_heaviest_key_has_the_smallest_value(gorio, form, new, wide, down):
    """One key's score lies some 39 octaves above the others', and its value's scale `down` powers of two below theirs, or is 0."""
    c = Coded([new], [300], heads=4, kv_heads=2, dim=64, form=form, uneven=0.5, seed=3)
    c.q.fill_(1.0)
    page, place = keys_of(c, 0, torch.tensor(70, device="cuda"))
    c.ks.mul_(0.25)
    codes, scales = encode(torch.full((2, 64), 3.5, device="cuda"), form)      # 3.5 * 64 / 8 = 28
    c.kp.view(torch.uint8)[page, :, place], c.ks[page, :, place] = codes.view(torch.uint8), scales
    c.vs[page, :, place] *= 0.0 if down is None else 2.0 ** -down
    if wide:                                                                   # the chunk kernel, for more than 16 rows a key head
        c.tables = widen(c.tables, c.page)
    check(c, c.run(gorio))


@pytest.mark.parametrize("form", [E4M3, INT8])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("up", [2.0 ** 5, 2.0 ** 23, 2.0 ** 40, 0.0])
def test_a_later_value_of_any_size_changes_nothing(gorio, form, wide, up):
    c = Coded([150], [300], heads=4, kv_heads=2, dim=64, form=form, uneven=0.5)
    if wide:
        c.tables = widen(c.tables, c.page)
    want = c.run(gorio)
    page, place = keys_of(c, 0, torch.tensor(299, device="cuda"))
    c.vs[page, :, place] *= up
    got = c.run(gorio)
    assert torch.equal(got["out"][:149], want["out"][:149]) and torch.equal(got["lse"][:149], want["lse"][:149])
    check(c, got)


@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("opts", [dict(softcap=30.0), dict(softcap=100.0, slopes=True), dict(slopes=True, window=90), dict(window=140)])
def test_a_later_value_changes_no_score_of_any_kind(gorio, dim, opts):
    """The last two keys' scales, seen by the last two rows alone, of a size that the other keys' have, and far from it."""
    c = Coded([250], [400], heads=4, kv_heads=2, dim=dim, uneven=0.5, seed=dim, **opts)
    c.tables = widen(c.tables, c.page)
    want = c.run(gorio)
    page, place = keys_of(c, 0, torch.tensor([398, 399], device="cuda"))
    old = c.vs[page, :, place].clone()
    for up in (1.7, 2.0 ** 6, 2.0 ** -6, 2.0 ** 60, 0.0, math.inf):
        c.vs[page, :, place] = old * up
        got = c.run(gorio)
        assert torch.equal(got["out"][:248], want["out"][:248]) and torch.equal(got["lse"][:248], want["lse"][:248])


@pytest.mark.parametrize("form", [E4M3, INT8])
@pytest.mark.parametrize("new", [1, 5, 100])
@pytest.mark.parametrize("length", [400, 9000])
@pytest.mark.parametrize("first,then", [(2.0 ** -75, 2.0 ** 65), (2.0 ** 65, 2.0 ** -75), (0.0, 2.0 ** 65)])
def test_scales_from_one_end_of_the_range_to_the_other(gorio, form, new, length, first, then):
    """The first keys' scales and the others' lie 140 powers of two apart: weights of both count in the sums."""
    c = Coded([new], [length], heads=4, kv_heads=1, dim=64, form=form, uneven=0.5, sharp=0.5)
    pages, places = keys_of(c, 0, torch.arange(length, device="cuda"))
    c.vs[pages, :, places] *= torch.where(torch.arange(length, device="cuda") < length // 3, first, then)[:, None]
    c.tables = widen(c.tables, c.page)
    check(c, c.run(gorio))


@pytest.mark.parametrize("form", [E4M3, INT8])
@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("first,then", [(1.0, 2.0 ** 96), (2.0 ** 96, 1.0), (2.0 ** 96, 2.0 ** 96), (2.0 ** -66, 2.0 ** 96)])
def test_scales_near_the_largest_that_count(gorio, form, new, first, then):
    c = Coded([new], [500], heads=4, kv_heads=1, dim=64, form=form, uneven=0.5, sharp=0.5)
    pages, places = keys_of(c, 0, torch.arange(500, device="cuda"))
    c.vs[pages, :, places] *= torch.where(torch.arange(500, device="cuda") < 200, first, then)[:, None]
    c.tables = widen(c.tables, c.page)
    check(c, c.run(gorio))
