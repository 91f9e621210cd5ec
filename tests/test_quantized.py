"""The quantised cache on the GPU: store and load against the format's rules, bit by bit; attention against 64 bits over the values that codes and
scales stand for."""
import math
import random

import pytest
import torch

from more_plain import assert_near, attend
from paged_plain import ceil_div

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16
E4M3, INT8 = torch.float8_e4m3fn, torch.int8
LARGEST = {E4M3: 448.0, INT8: 127.0}


@pytest.fixture(scope="module")
def gorio():
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as g
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _bytes(x):
    return x.view(torch.uint8)


def same(a, b):
    """Equal, where not-a-number equals itself (a row with an infinity is stored as one)."""
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(1.0), b.nan_to_num(1.0))


def encode(x, form):
    """The format's rules in torch's 32-bit arithmetic."""
    x = x.float()
    top = x.abs().amax(-1)
    top = torch.where(torch.isfinite(x).all(-1), top, math.nan)
    largest = torch.full_like(top, LARGEST[form])
    some = top >= 2.0 ** -100
    scale = torch.where(some, top / largest, torch.where(torch.isnan(top), math.nan, 0.0))
    y = torch.where(some[..., None], x * torch.where(some, largest / top, 0.0)[..., None], 0.0)
    return (y.round() if form == INT8 else y).to(form), scale


# ---------------------------------------------------------------- store and load

@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("form", [E4M3, INT8])
@pytest.mark.parametrize("tokens,heads,dim,page", [(1, 1, 64, 8), (1, 8, 128, 16), (63, 3, 96, 24), (1000, 2, 128, 16), (257, 5, 16, 1), (33, 2, 256, 16), (9, 1, 208, 8),
                                                   (20011, 8, 128, 16)])
@pytest.mark.parametrize("layout", ["heads", "tokens", "joint"])
def test_store_and_load(gorio, dtype, form, tokens, heads, dim, page, layout):
    g = torch.Generator(device="cuda").manual_seed(tokens)
    pages = ceil_div(tokens, page) + 3
    kv = torch.randn((tokens, 2, heads, dim), generator=g, device="cuda").mul_(torch.randn((tokens, 2, heads, 1), generator=g, device="cuda").mul_(3).exp()).to(dtype)
    k, v = (kv[:, 0], kv[:, 1]) if layout == "joint" else (kv[:, 0].contiguous(), kv[:, 1].contiguous())

    def cache():
        codes = torch.randint(0, 255, (pages, heads, page, dim), generator=g, device="cuda", dtype=torch.uint8)
        scales = torch.randn((pages, heads, page), generator=g, device="cuda")
        if layout == "tokens":
            return codes.transpose(1, 2).contiguous().view(form).transpose(1, 2), scales.transpose(1, 2).contiguous().transpose(1, 2)
        if layout == "joint":
            wide = torch.zeros((pages, heads, page, dim + 32), dtype=torch.uint8, device="cuda")
            wide[..., 16:16 + dim] = codes
            return wide.view(form)[..., 16:16 + dim], scales
        return codes.view(form), scales
    (kp, ks), (vp, vs) = cache(), cache()
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:tokens]
    if tokens > 5:
        slots[2::5] = -1
    taken = slots >= 0
    to = slots[taken]
    want = []
    for x, p, s in ((k, kp, ks), (v, vp, vs)):
        codes, scales = encode(x[taken], form)
        p, s = _bytes(p).clone(), s.clone()
        p[to // page, :, to % page] = _bytes(codes)
        s[to // page, :, to % page] = scales
        want.append((p, s))
    gorio.cache_store_quantized(k, v, kp, vp, ks, vs, slots)
    for p, s, w in ((kp, ks, want[0]), (vp, vs, want[1])):
        assert torch.equal(_bytes(p), w[0]) and same(s, w[1])
    # slots outside the cache are skipped
    gorio.cache_store_quantized(k, v, kp, vp, ks, vs, torch.full((tokens,), pages * page, device="cuda"))
    gorio.cache_store_quantized(k[:0], v[:0], kp, vp, ks, vs, slots[:0])
    for p, s, w in ((kp, ks, want[0]), (vp, vs, want[1])):
        assert torch.equal(_bytes(p), w[0]) and same(s, w[1])
    # and read as zeros; the rest as what codes and scales stand for, within half a step of what was stored
    for t in (BF16, FP16):
        got = gorio.cache_load_quantized(kp, vp, ks, vs, slots, dtype=t)
        for x, y, p, s in ((k, got[0], kp, ks), (v, got[1], vp, vs)):
            codes = p.contiguous().view(form).permute(0, 2, 1, 3).float()
            value = torch.zeros((tokens, heads, dim), device="cuda")
            value[taken] = (codes * s.permute(0, 2, 1)[..., None])[to // page, to % page]
            assert y.dtype is t and same(y, value.to(t))
            far = (value[taken].double() - x[taken].double()).abs()
            top = x[taken].double().abs().amax(-1, keepdim=True)
            # int8: half a step of M / 127; e4m3: 2^-4 of the number, or half its least step, 2^-10 * M / 448; scale and product round by 2^-24
            most = top / 254 if form == INT8 else torch.maximum(x[taken].double().abs() * 2.0 ** -4, top * 2.0 ** -10 / 448)
            fine = torch.isfinite(x[taken]).all(-1, keepdim=True)      # a row with an infinity reads as not a number
            assert ((far <= most * (1 + 2.0 ** -10) + top * 2.0 ** -22) | ~fine).all() and (torch.isnan(value[taken]) | fine).all()
    out = torch.full((tokens, 2, heads, dim), 7.0, dtype=dtype, device="cuda")
    got = gorio.cache_load_quantized(kp, vp, ks, vs, slots, dtype=dtype, out=(out[:, 1], out[:, 0]))
    again = gorio.cache_load_quantized(kp, vp, ks, vs, slots, dtype=dtype)
    assert got[0].data_ptr() == out[:, 1].data_ptr() and same(out[:, 1], again[0]) and same(out[:, 0], again[1])


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("form", [E4M3, INT8])
def test_store_of_rows_at_the_format_s_ends(gorio, dtype, form):
    """Zeros, the smallest and largest numbers, ties, one number far above the others, infinities and NaN: each row by itself."""
    info = torch.finfo(dtype)
    d = 64
    rows = torch.zeros((12, d), dtype=torch.float64)
    rows[1, 3] = info.smallest_normal * 2.0 ** (-7 if dtype == BF16 else -10)       # the least number above 0
    rows[2] = info.max
    rows[3] = -info.max
    rows[4] = torch.arange(d) - 32.0
    rows[5, 0], rows[5, 1:] = LARGEST[form], torch.arange(1, d) / 2.0               # scale 1: ties to even
    rows[6], rows[6, 9] = 1e-4, 6e4
    rows[7], rows[7, 5] = 1.0, math.inf
    rows[8], rows[8, 6] = 1.0, -math.inf
    rows[9], rows[9, 63] = 1.0, math.nan
    rows[10] = -1.0
    rows[11] = torch.linspace(-1, 1, d) * 2.0 ** -12
    if dtype == BF16:
        rows = torch.cat([rows, torch.full((1, d), 2.0 ** -100, dtype=torch.float64), torch.full((1, d), 2.0 ** -101, dtype=torch.float64),
                          torch.full((1, d), 2.0 ** 127, dtype=torch.float64)])
    x = rows.to(dtype).cuda()[:, None]
    t = x.shape[0]
    kp, vp = [torch.zeros((2, 1, 16, d), dtype=torch.uint8, device="cuda").view(form) for _ in range(2)]
    ks, vs = [torch.zeros((2, 1, 16), device="cuda") for _ in range(2)]
    slots = torch.arange(t, device="cuda")
    gorio.cache_store_quantized(x, -x, kp, vp, ks, vs, slots)
    for y, p, s in ((x, kp, ks), (-x, vp, vs)):
        codes, scales = encode(y, form)
        got, scale = p.transpose(1, 2).reshape(32, 1, d)[:t], s.transpose(1, 2).reshape(32, 1)[:t]
        assert torch.equal(got.float(), codes.float())
        assert same(scale, scales)
        assert torch.isnan(scale[7:10]).all() and scale[0] == 0
        if form == E4M3:
            assert ((_bytes(got) & 0x7f) != 0x7f).all()
    back, _ = gorio.cache_load_quantized(kp, vp, ks, vs, slots, dtype=dtype)
    assert torch.isnan(back[7:10]).all() and torch.isfinite(back[:7]).all() and (back[0] == 0).all() and torch.equal(back[10], x[10])


def test_load_of_every_code(gorio):
    """All 256 codes, the two of e4m3 that are no numbers among them."""
    every = torch.arange(256, dtype=torch.uint8, device="cuda").view(1, 1, 1, 256)
    scale = torch.full((1, 1, 1), 1.5, device="cuda")
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    for form in (E4M3, INT8):
        got, _ = gorio.cache_load_quantized(every.view(form), every.view(form), scale, scale, slots, dtype=FP16)
        want = every.view(form).float().view(-1)
        assert torch.isnan(want).sum() == (2 if form == E4M3 else 0)
        assert same(got, (want * 1.5).half().expand(3, 1, 256))


# ---------------------------------------------------------------- attention

class Coded:
    """A quantised cache with the given requests in scattered pages; what no query sees has codes of any kind and a scale that is not a number."""

    def __init__(self, new, lens, heads=8, kv_heads=4, dim=64, page=16, dtype=BF16, form=E4M3, seed=0, layout="heads", causal=True, window=0, softcap=0.0,
                 slopes=False, spare=0, sharp=2.0, freed=False, uneven=1.0, scale_of=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        width = max(1, max(ceil_div(n, page) for n in lens)) + 1
        held = sum(ceil_div(n, page) for n in lens)
        shape = (held + 4 + spare, kv_heads, page, dim)

        def cache():
            if layout == "tokens":
                codes = torch.randint(0, 256, (shape[0], page, kv_heads, dim), generator=g, device="cuda", dtype=torch.uint8).view(form).transpose(1, 2)
                return codes, torch.full((shape[0], page, kv_heads), math.nan, device="cuda").transpose(1, 2)
            if spare:
                codes = torch.zeros(shape, dtype=torch.uint8, device="cuda").view(form)
            else:
                codes = torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8).view(form)
            return codes, torch.full(shape[:3], math.nan, device="cuda")
        (self.kp, self.ks), (self.vp, self.vs) = cache(), cache()
        order = (torch.randperm(held + 4, generator=g, device="cuda") + spare).tolist()
        tables = [[-1] * width for _ in lens]
        self.lens, self.new, self.page = lens, new, page
        for r, n in enumerate(lens):
            for i in range(ceil_div(n, page)):
                tables[r][i] = order.pop()
                rows = min(page, n - i * page)
                for p, s in ((self.kp, self.ks), (self.vp, self.vs)):
                    x = torch.randn((kv_heads, rows, dim), generator=g, device="cuda") * torch.randn((kv_heads, rows, 1), generator=g, device="cuda").mul_(uneven).exp_()
                    codes, scales = encode(x.to(BF16), form)
                    if scale_of is not None:
                        scales = scale_of(scales)
                    _bytes(p)[tables[r][i], :, :rows] = _bytes(codes)
                    s[tables[r][i], :, :rows] = scales
        if freed:                                              # pages that lie before every query's window are given back
            for r, n in enumerate(lens):
                for i in range(max(0, n - new[r] - window + 1) // page):
                    tables[r][i] = -1 if (i + r) % 2 else (1 << 30)
        self.tables, self.lengths = _i32(tables), _i32(lens)
        self.starts = _i32([sum(new[:i]) for i in range(len(new) + 1)])
        self.q = torch.randn((sum(new), heads, dim), generator=g, device="cuda").mul_(sharp).to(dtype)
        if layout == "tokens":                                 # a projection's columns
            wide = torch.zeros((sum(new), heads + 3, dim), dtype=dtype, device="cuda")
            wide[:, 1:1 + heads] = self.q
            self.q = wide[:, 1:1 + heads]
        self.max_new = max(new) if new else 0
        self.opts = dict(causal=causal, window=window, softcap=softcap,
                         slopes=torch.exp2(-torch.arange(1, heads + 1, device="cuda") / 2).float() if slopes else None)

    def run(self, gorio, **more):
        return gorio.paged_attention_quantized(self.q, self.kp, self.vp, self.ks, self.vs, self.tables, self.lengths, self.starts,
                                               more.pop("max_new", self.max_new), want_lse=True, **{**self.opts, **more})

    def _rows(self, pages, scales, ids, n):
        there = (ids >= 0) & (ids < pages.shape[0])
        ids = torch.where(there, ids, 0).long()
        codes = _bytes(pages)[ids].contiguous().view(pages.dtype).float().double()
        if pages.dtype == E4M3:
            codes = torch.where(torch.isnan(codes), 480.0, codes)
        x = torch.where(there[:, None, None, None], codes * scales[ids].double()[..., None], 0.0)
        return x.transpose(0, 1).reshape(pages.shape[1], -1, pages.shape[3])[:, :n]

    def want(self, **more):
        parts = []
        for r, (n, length) in enumerate(zip(self.new, self.lens)):
            ids = self.tables[r, :ceil_div(length, self.page)]
            k, v = self._rows(self.kp, self.ks, ids, length), self._rows(self.vp, self.vs, ids, length)
            at = torch.arange(length - n, length, device="cuda")
            j = torch.arange(length, device="cuda")
            sees = torch.ones((n, length), dtype=torch.bool, device="cuda")
            if self.opts["causal"]:
                sees &= j[None] <= at[:, None]
            if self.opts["window"]:
                sees &= j[None] > at[:, None] - self.opts["window"]
            # weights times scales are rounded to float16's 11 bits, 2^-11 of themselves at most; codes are exact
            parts.append(attend(self.q[self.starts[r]:self.starts[r + 1]], k, v, sees, j[None] - at[:, None], self.opts["softcap"], self.opts["slopes"],
                                weights=2.0 ** -11, **more))
        return [torch.cat(x) for x in zip(*parts)]

    def check(self, gorio, **more):
        got = self.run(gorio, **more)
        assert_near(got, self.want())
        return got


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("form", [E4M3, INT8])
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("new,lens", [([1], [1]), ([1], [65]), ([1, 1, 1], [16, 17, 1000]), ([2, 1, 5], [2, 300, 64]), ([130], [130]), ([33, 1, 300], [500, 129, 300])])
def test_coded_types_and_lengths(gorio, dtype, form, dim, new, lens):
    c = Coded(new, lens, dim=dim, dtype=dtype, form=form, seed=dim)
    c.check(gorio)
    c.check(gorio, max_new=1)                                  # the single-token kernel, whatever the sizes


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 1), (3, 3), (10, 2), (14, 2), (32, 2), (40, 1), (9, 3)])
@pytest.mark.parametrize("new", [1, 3, 70, 900])
def test_coded_head_layouts(gorio, heads, kv_heads, new):
    Coded([new, 1], [max(new, 211), 90], heads=heads, kv_heads=kv_heads, dim=128, seed=heads, form=INT8 if new % 2 else E4M3).check(gorio)


@pytest.mark.parametrize("page", [8, 16, 24, 32, 48, 64, 128, 256])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("new", [1, 150])
def test_coded_pages_and_strides(gorio, page, layout, new):
    for dim in (64, 96, 128):
        Coded([new, 1], [777, 40], page=page, layout=layout, dim=dim, seed=page, form=INT8 if page % 32 else E4M3).check(gorio)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 5, 64, 200])
@pytest.mark.parametrize("softcap,slopes", [(0.0, False), (5.0, False), (0.0, True), (30.0, True), (100.0, True)])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 260]])
def test_coded_masks_and_scores(gorio, causal, window, softcap, slopes, new):
    Coded(new, [300, 150, 430], dim=128 if softcap else 64, causal=causal, window=window, softcap=softcap, slopes=slopes, seed=window, freed=window > 0,
          form=E4M3 if softcap else INT8).check(gorio)


def test_coded_rows_without_keys(gorio):
    for causal in (True, False):
        for new in ([1, 2, 1], [5, 9, 3], [40, 300, 7]):
            got = Coded(new, [0, 2, 0], causal=causal).check(gorio)
            assert (got["out"][:new[0]] == 0).all() and (got["lse"][:new[0]] == -math.inf).all()
    Coded([1, 0, 1], [40, 30, 20]).check(gorio)
    Coded([0, 0, 70], [40, 30, 100]).check(gorio)
    assert Coded([0, 0], [4, 5]).run(gorio)["out"].shape == (0, 8, 64)


@pytest.mark.parametrize("form", [E4M3, INT8])
@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("scale_of", ["large", "small", "mixed", "zero"])
def test_coded_scales_of_any_size(gorio, form, new, scale_of):
    """Scales from 2^-40 to 2^9 (values stay within bfloat16's and the result's range), alike or from key to key; scales of 0."""
    if scale_of == "mixed":
        change = lambda s: s * torch.exp2(torch.randint(-30, 1, s.shape, device=s.device).float())      # noqa: E731
    elif scale_of == "zero":
        change = lambda s: torch.where(torch.rand(s.shape, device=s.device) < 0.5, 0.0, s)              # noqa: E731
    else:
        change = lambda s: s * (2.0 ** 6 if scale_of == "large" else 2.0 ** -40)                        # noqa: E731
    torch.manual_seed(5)
    Coded([new, new], [300, 500], form=form, dim=128, scale_of=change, uneven=0.5, sharp=0.05 if scale_of == "large" else 2.0).check(gorio)


@pytest.mark.parametrize("new", [[4], [1], [150]])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("what", ["ks", "vs"])
def test_coded_scales_that_are_not_finite_reach_only_who_sees_them(gorio, new, bad, what):
    c = Coded(new, [200], dim=64, heads=8, kv_heads=2)
    want = c.run(gorio)
    getattr(c, what)[c.tables[0, 198 // 16].item(), :, 198 % 16] = bad       # all but the last two tokens' queries do not see it
    got = c.run(gorio)
    before = max(0, new[0] - 2)
    assert torch.equal(got["out"][:before], want["out"][:before]) and torch.equal(got["lse"][:before], want["lse"][:before])
    broken = ~torch.isfinite(got["out"][before:]).all(-1)
    if what == "ks" and bad == math.inf:
        # the score is the infinity of the dot product's sign: below zero the key's weight is 0, and the result one without it
        codes = _bytes(c.kp)[c.tables[0, 198 // 16].item(), :, 198 % 16].contiguous().view(c.kp.dtype).double()
        dot = torch.einsum("nhd,hd->nh", c.q[before:].double(), codes.repeat_interleave(4, 0))
        assert torch.equal(broken, dot > 0)
    else:
        assert broken.all()


@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_coded_extreme_scores(gorio, new, dtype):
    # weights that all but vanish beside one key's, and scores far from 0
    Coded([new], [500], sharp=60.0, dim=128, heads=16, kv_heads=4, dtype=dtype).check(gorio)
    c = Coded([new], [500], dim=128, heads=16, kv_heads=4, dtype=dtype)
    c.q.zero_()                                                # even weights: the mean of the values
    c.check(gorio)
    c = Coded([new], [500], dim=128, heads=16, kv_heads=4, dtype=dtype, sharp=1e-6)
    c.check(gorio)
    if dtype == BF16:                                          # queries far outside float16's range
        c = Coded([new], [500], dim=128, heads=16, kv_heads=4, sharp=1e30)
        got = c.run(gorio, scale=1e-30 / math.sqrt(128))
        assert_near(got, c.want(scale=1e-30 / math.sqrt(128)))


def test_coded_long_cache_in_parts(gorio):
    Coded([1], [40000], dim=128, heads=8, kv_heads=2, page=64).check(gorio)
    Coded([1, 1], [9000, 3], dim=64, heads=5, kv_heads=1).check(gorio)
    Coded([60], [20000], dim=64, heads=8, kv_heads=1, page=64, form=INT8).check(gorio)
    Coded([150], [20000], dim=64, heads=8, kv_heads=1, page=64).check(gorio)
    Coded([150], [9000], dim=128, heads=6, kv_heads=1, form=INT8).check(gorio)
    Coded([30] * 7, [9000, 100, 300, 5, 2000, 700, 30], dim=128, heads=6, kv_heads=2).check(gorio)
    Coded([300, 40, 7], [4000, 900, 2500], dim=96, heads=4, kv_heads=2).check(gorio)
    rng = random.Random(5)
    Coded([1] * 1500, [rng.randint(0, 40) for _ in range(1500)], dim=64, heads=2, kv_heads=1).check(gorio)
    Coded([rng.randint(0, 20) for _ in range(300)], [rng.randint(0, 150) for _ in range(300)], dim=64, heads=2, kv_heads=1, page=8).check(gorio)


def test_coded_offsets_past_32_bits(gorio):
    """The pages in use lie behind the 2^32nd byte of the cache."""
    spare = (1 << 32) // (2 * 64 * 128) + 8
    for new in (1, 250):
        Coded([new, 1], [500, 300], dim=128, heads=4, kv_heads=2, page=64, spare=spare).check(gorio)
        torch.cuda.empty_cache()
    pages = torch.zeros((spare + 2, 2, 64, 128), dtype=torch.uint8, device="cuda").view(INT8)
    scales = torch.zeros((spare + 2, 2, 64), device="cuda")
    x = torch.randn((3, 2, 128), device="cuda").half()
    slots = torch.tensor([(spare + 1) * 64 + 5, -1, spare * 64], device="cuda")
    gorio.cache_store_quantized(x, x, pages, pages.clone(), scales, scales.clone(), slots)
    codes, s = encode(x, INT8)
    assert torch.equal(pages[spare + 1, :, 5], codes[0]) and torch.equal(pages[spare, :, 0], codes[2]) and torch.equal(scales[spare + 1, :, 5], s[0])
    back, _ = gorio.cache_load_quantized(pages, pages, scales, scales, slots, dtype=FP16)
    assert torch.equal(back[0], (codes[0].float() * s[0][:, None]).half()) and (back[1] == 0).all()


@pytest.mark.parametrize("new", [1, 40, 140])
def test_coded_table_entries_outside_the_cache_read_as_zeros(gorio, new):
    c = Coded([1, new], [100, 200])
    for bad in (-1, 1 << 30):
        c.tables[0, 2] = bad
        c.tables[1, 3] = bad
        c.check(gorio)
    none = torch.empty((0, 4, 16, 64), dtype=E4M3, device="cuda")
    got = gorio.paged_attention_quantized(c.q, none, none, torch.empty((0, 4, 16), device="cuda"), torch.empty((0, 4, 16), device="cuda"), c.tables, c.lengths,
                                          c.starts, new)
    assert (got["out"] == 0).all()
    back, _ = gorio.cache_load_quantized(none, none, torch.empty((0, 4, 16), device="cuda"), torch.empty((0, 4, 16), device="cuda"),
                                         torch.zeros(5, dtype=torch.int64, device="cuda"))
    assert back.shape == (5, 4, 64) and (back == 0).all()


def test_coded_bad_lengths_stay_in_bounds(gorio):
    c = Coded([1, 2, 30], [50, 60, 70])
    want = c.run(gorio)
    big = (1 << 31) - 1
    for lens in ([50, 60, -9], [50, 60, big], [50, 60, -big]):
        c.lengths.copy_(_i32(lens))
        assert torch.equal(c.run(gorio)["out"][:3], want["out"][:3])
    c.lengths.copy_(_i32([50, 60, 70]))
    for starts in ([0, 1, 3, big], [-5, 1, 3, 33]):
        c.starts.copy_(_i32(starts))
        c.run(gorio)
    torch.cuda.synchronize()


@pytest.mark.parametrize("new", [1, 150])
def test_coded_step_in_a_graph_and_on_streams(gorio, new):
    """Pages, store and attention of a step, captured, replayed and beside eager calls on the stream of the capture."""
    c = Coded([new, 1], [777, 300], dim=128, heads=8, kv_heads=2, form=INT8)
    x = torch.randn((new + 1, 2, 2, 128), device="cuda").to(BF16)
    slots = []
    for r, (n, length) in enumerate(zip(c.new, c.lens)):
        slots += [c.tables[r, p // 16].item() * 16 + p % 16 for p in range(length - n, length)]
    slots = torch.tensor(slots, device="cuda")

    def step():
        gorio.cache_store_quantized(x[:, 0], x[:, 1], c.kp, c.vp, c.ks, c.vs, slots)
        return c.run(gorio)
    want = step()
    assert_near(want, c.want())
    keys, values = gorio.cache_load_quantized(c.kp, c.vp, c.ks, c.vs, slots)
    codes, scales = encode(x, INT8)
    assert torch.equal(torch.stack([keys, values], 1), (codes.float() * scales[..., None]).to(BF16))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    for _ in range(20):
        graph.replay()
        with torch.cuda.stream(side):
            more = c.run(gorio)
    torch.cuda.synchronize()
    assert torch.equal(got["out"], want["out"]) and torch.equal(more["out"], want["out"])
    there = c.run(gorio, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(there["out"], want["out"])
    gorio.attention_check()


def test_quantized_refusals(gorio):
    c = Coded([1, 2], [50, 60])
    good = dict(q=c.q, key_pages=c.kp, value_pages=c.vp, key_scales=c.ks, value_scales=c.vs, tables=c.tables, lengths=c.lengths, starts=c.starts, max_new=2)
    for name, bad in (("q", c.q.float()), ("q", c.q[:, :3]), ("q", c.q[..., :32]), ("key_pages", _bytes(c.kp)), ("key_pages", c.kp.to(BF16)), ("key_pages", c.kp[:3]),
                      ("value_pages", c.vp.view(INT8)), ("key_scales", c.ks.half()), ("key_scales", c.ks[:, :1]), ("value_scales", c.vs.cpu()),
                      ("lengths", c.lengths[:1]), ("tables", c.tables.long()), ("max_new", -1), ("key_pages", c.kp[..., ::2])):
        with pytest.raises(gorio.GorioError) as e:
            gorio.paged_attention_quantized(**{**good, name: bad})
        assert e.value.status == 1
    wide = torch.zeros((c.kp.shape[0], 4, 16, 72), dtype=torch.uint8, device="cuda").view(E4M3)[..., :64]
    with pytest.raises(gorio.GorioError):                        # rows 72 bytes apart
        gorio.paged_attention_quantized(**{**good, "key_pages": wide})
    x = torch.randn((3, 4, 64), device="cuda").to(BF16)
    slots = torch.arange(3, device="cuda")
    store = dict(keys=x, values=x, key_pages=c.kp, value_pages=c.vp, key_scales=c.ks, value_scales=c.vs, slots=slots)
    for name, bad in (("keys", x.float()), ("keys", x.half()), ("keys", x[:, :3]), ("slots", slots.int()), ("slots", slots[:2]), ("key_pages", wide),
                      ("key_scales", c.ks[:, :, :8]), ("values", None)):
        with pytest.raises(gorio.GorioError):
            gorio.cache_store_quantized(**{**store, name: bad})
    load = {k: v for k, v in store.items() if k not in ("keys", "values")}
    for more in (dict(dtype=torch.float32), dict(out=(x, x.half())), dict(out=(x[:2], x[:2])), dict(slots=slots.int()), dict(out=(x.half(), x.half()))):
        with pytest.raises(gorio.GorioError):
            gorio.cache_load_quantized(**{**load, **more})
    q = c.q.clone().requires_grad_()
    with pytest.raises(gorio.GorioError):
        gorio.paged_attention_quantized(**{**good, "q": q})["out"].sum().backward()
