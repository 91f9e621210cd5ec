"""The operators of shared prefixes and of the quantised cache together, as the example uses them behind a search."""
import importlib.util
import os

import pytest
import torch

from more_plain import assert_near, attend
from paged_plain import ceil_div

pytestmark = pytest.mark.gpu


def _rows(pages, ids, n, scales=None):
    x = pages[ids.long()].float().double() if scales is None else pages.view(torch.uint8)[ids.long()].view(pages.dtype).float().double() * scales[ids.long()].double()[..., None]
    return x.transpose(0, 1).reshape(pages.shape[1], -1, pages.shape[3])[:, :n]


@pytest.mark.parametrize("codes", [torch.float8_e4m3fn, torch.int8])
def test_sample_and_keep(codes):
    from paper_2607_04415_b200 import build
    build.build()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "sample_and_keep.py")
    spec = importlib.util.spec_from_file_location("sample_and_keep", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.main(questions=5, answers=6, found=3, passage_tokens=16, steps=18, heads=8, kv_heads=2, scale=0.02, codes=codes)
    s = r["shared"]
    parts = []
    for a in range(30):
        g, own, ahead = int(s["group_of"][a]), int(s["lengths"][a]), int(s["prefix_lengths"][0])
        k, v = [torch.cat([_rows(p, s["prefix_tables"][g], ahead), _rows(p, s["tables"][a, :ceil_div(own, 16)], own)], 1) for p in (s["key_pages"], s["value_pages"])]
        n = ahead + own
        sees = torch.ones((1, n), dtype=torch.bool, device="cuda")
        parts.append(attend(s["q"][a:a + 1], k, v, sees, torch.arange(1 - n, 1, device="cuda")[None]))
    assert_near(s, [torch.cat(x) for x in zip(*parts)])
    # what was kept is within half a step of what was stored: int8 M / 254; e4m3 2^-4 of a number or the least step's half; and bfloat16's rounding, 2^-8
    for x, y in zip((r["keys"], r["values"]), r["back"]):
        top = x.float().abs().amax(-1, keepdim=True)
        most = top / 254 if codes == torch.int8 else torch.maximum(x.float().abs() / 16, top * 2.0 ** -10 / 448)
        assert ((x.float() - y.float()).abs() <= most * (1 + 2.0 ** -10) + 2.0 ** -8 * (x.float().abs() + most) + top * 2.0 ** -22).all()
    c = r["kept"]
    assert c["served"].tolist() == [1] * 5
    parts = []
    for i in range(5):
        n, length = 7, int(c["lengths"][i])
        ids = c["tables"][i, :ceil_div(length, 16)]
        k, v = _rows(c["key_codes"], ids, length, c["key_scales"]), _rows(c["value_codes"], ids, length, c["value_scales"])
        at, j = torch.arange(length - n, length, device="cuda"), torch.arange(length, device="cuda")
        rows = slice(int(c["starts"][i]), int(c["starts"][i + 1]))
        # the rounding to 11 bits of weights times scales
        parts.append(attend(c["q"][rows], k, v, j[None] <= at[:, None], j[None] - at[:, None], weights=2.0 ** -11))
    assert_near(c, [torch.cat(x) for x in zip(*parts)])
