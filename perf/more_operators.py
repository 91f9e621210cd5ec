"""The operators of a quantised key/value cache and of shared prefixes, as cases to measure: the store of new keys and values
in 8 bits, their reading back, attention of new tokens over such a cache, and attention of a batch whose requests share
prefixes.

`run` computes a case in its plain form (elementary torch operations in 32 bits) or, with `own` set, by the package's
kernels.  A cache's page tensors are [pages, key heads, page size, head size]; a quantised one holds float8_e4m3fn or int8
numbers, each row of a token and a key head with a scale in [pages, key heads, page size] (float32): number times scale is
the value.  A row's scale is its largest magnitude over 448 or 127, rounded to 32 bits."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
FORMATS = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
LARGEST = {"e4m3": 448.0, "int8": 127.0}


def listed():
    plain = dict(causal=True, window=0, softcap=0.0, slopes=False)
    return [
        # the new keys and values of one decode step
        dict(name="quantize_decode", op="store", tokens=64, kv_heads=8, dim=128, page=16, pages=1024, dtype="bf16", format="e4m3", skipped=0),
        # those of a long prompt, an odd number of tokens, some of them not admitted
        dict(name="quantize_prompt", op="store", tokens=16383, kv_heads=8, dim=128, page=16, pages=1100, dtype="fp16", format="int8", skipped=7),
        # a short passage of the cache is handed to a layer that wants 16 bits
        dict(name="load_passage", op="load", tokens=301, kv_heads=4, dim=96, page=24, pages=200, dtype="fp16", format="int8", skipped=0),
        # a long request moves to another server: all its tokens, in order, from pages all over the cache
        dict(name="load_request", op="load", tokens=30001, kv_heads=8, dim=128, page=16, pages=2100, dtype="bf16", format="e4m3", skipped=11),
        # one user, one token: latency counts
        dict(name="coded_one", op="attention", requests=1, new_lo=1, new_hi=1, len_lo=4097, len_hi=4097, heads=32, kv_heads=8, dim=128, page=16,
             dtype="bf16", format="int8", spread=21, **plain),
        # a server's decode step, ragged lengths
        dict(name="coded_batch", op="attention", requests=64, new_lo=1, new_hi=1, len_lo=100, len_hi=16384, heads=32, kv_heads=8, dim=128, page=16,
             dtype="bf16", format="e4m3", spread=22, **plain),
        # questions over retrieved passages beside single tokens: a bias by distance and capped scores, every second head its own keys
        dict(name="coded_mixed", op="attention", requests=12, new_lo=1, new_hi=300, len_lo=300, len_hi=4096, heads=16, kv_heads=8, dim=64, page=16,
             dtype="fp16", format="int8", causal=True, window=0, softcap=30.0, slopes=True, spread=23),
        # a piece of one long prompt over what is cached of it: the largest
        dict(name="coded_prompt", op="attention", requests=1, new_lo=2048, new_hi=2048, len_lo=18432, len_hi=18432, heads=32, kv_heads=8, dim=128, page=16,
             dtype="bf16", format="e4m3", spread=24, **plain),
        # a few answers sampled for one prompt: latency counts
        dict(name="prefix_few", op="prefix", groups=1, members_lo=4, members_hi=4, prefix_lo=2000, prefix_hi=2000, new_lo=1, new_hi=1, len_lo=1, len_hi=40,
             heads=32, kv_heads=8, dim=128, page=16, dtype="bf16", spread=25, **plain),
        # a server's decode step: one system prompt, each request with a conversation of its own
        dict(name="prefix_batch", op="prefix", groups=1, members_lo=64, members_hi=64, prefix_lo=16391, prefix_hi=16391, new_lo=1, new_hi=1, len_lo=1,
             len_hi=1024, heads=32, kv_heads=8, dim=128, page=16, dtype="bf16", spread=26, **plain),
        # questions of several tokens over retrieved passages, some passages asked about once, some often; a window and a bias by distance
        dict(name="prefix_passages", op="prefix", groups=9, members_lo=0, members_hi=14, prefix_lo=300, prefix_hi=5000, new_lo=1, new_hi=33, len_lo=0,
             len_hi=200, heads=14, kv_heads=2, dim=64, page=24, dtype="fp16", causal=True, window=2500, softcap=0.0, slopes=True, spread=27),
        # many answers sampled over one very long document
        dict(name="prefix_document", op="prefix", groups=1, members_lo=128, members_hi=128, prefix_lo=100003, prefix_hi=100003, new_lo=1, new_hi=1,
             len_lo=100, len_hi=500, heads=32, kv_heads=4, dim=128, page=64, dtype="bf16", spread=28, **plain),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _scores(rng, reach):
    extra = rng.random()
    return dict(causal=rng.random() < 0.75, window=_log(rng, 1, reach) if extra < 0.2 else 0, softcap=rng.choice([20.0, 50.0]) if 0.1 < extra < 0.3 else 0.0,
                slopes=0.2 < extra < 0.4)


def draw(rng):
    op = rng.choice(["store", "load", "attention", "attention", "prefix", "prefix"])
    spread = rng.randrange(1000, 1 << 30)
    common = dict(op=op, dtype=rng.choice(["bf16", "fp16"]))
    if op in ("store", "load"):
        t = _log(rng, 1, 16383 if op == "store" else 30001)
        page = rng.choice([8, 16, 24, 32, 64])
        return dict(common, tokens=t, kv_heads=rng.choice([1, 2, 3, 4, 8]), dim=rng.choice([64, 96, 128]), page=page, pages=t // page + rng.randint(2, 60),
                    format=rng.choice(["e4m3", "int8"]), skipped=rng.choice([0, 0, 5]))
    kv_heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 5, 7, 8])
    dim = rng.choice([64, 96, 128])
    if kv_heads * group * dim > 4096:
        group = 4
    if kv_heads * group == 32 and dim == 96:
        dim = 128
    common.update(heads=kv_heads * group, kv_heads=kv_heads, dim=dim, page=rng.choice([8, 16, 16, 32, 48, 64, 128]), spread=spread)
    new_hi = 1 if rng.random() < 0.5 else _log(rng, 2, 2048 if op == "attention" else 100)
    if op == "attention":
        b = _log(rng, 1, 64 if new_hi == 1 else 16)
        if new_hi == 1:
            most = min(131072, 500000 // b)                           # keys of a request, so that all of them stay below coded_batch's
        else:
            most = min(18432, 400000 // b, 30000000 // (b * new_hi))  # and the scores below coded_prompt's
        len_hi = _log(rng, min(new_hi + 1, most), most)
        return dict(common, requests=b, new_lo=rng.choice([1, new_hi]), new_hi=new_hi, len_lo=rng.choice([1, max(1, len_hi // 2), len_hi]), len_hi=len_hi,
                    format=rng.choice(["e4m3", "int8"]), **_scores(rng, len_hi))
    groups = rng.choice([1, 1, 2, 5, 11])
    members = _log(rng, 2, 128 // groups if new_hi == 1 else max(2, 24 // groups))
    most = min(100003, 12000000 // (groups * members * new_hi))       # the scores below prefix_document's
    prefix = _log(rng, 1, most)
    return dict(common, groups=groups, members_lo=rng.choice([0, members]) if groups > 1 else members, members_hi=members, prefix_lo=rng.choice([0, prefix, prefix]),
                prefix_hi=prefix, new_lo=1, new_hi=new_hi, len_lo=rng.choice([0, 1, 30]), len_hi=_log(rng, 31, 1000), **_scores(rng, prefix + 100))


def _numbers(case, count, lo, hi, salt):
    """`count` whole numbers of [lo, hi], by the case alone: its lengths are part of the case."""
    rng = random.Random(case["spread"] * 10 + salt)
    return [rng.randint(lo, hi) for _ in range(count)]


def _groups(case):
    """Requests and prefix tokens of each group of a prefix case."""
    members = _numbers(case, case["groups"], case["members_lo"], case["members_hi"], 3)
    if not sum(members):
        members[0] = 1
    return members, _numbers(case, case["groups"], case["prefix_lo"], case["prefix_hi"], 4)


def _lens(case):
    """New tokens and keys (of its own, where prefixes are shared) of each request: where causal, the keys hold the new tokens' own."""
    b = sum(_groups(case)[0]) if case["op"] == "prefix" else case["requests"]
    new = _numbers(case, b, case["new_lo"], case["new_hi"], 1)
    keys = _numbers(case, b, case["len_lo"], case["len_hi"], 2)
    if case["causal"]:
        keys = [max(k, n) for k, n in zip(keys, new)]
    return new, keys


def _pages_of(tokens, page):
    return -(-tokens // page)


def _codes(x, form):
    """Rows in 8 bits, and their scales."""
    top = x.float().abs().amax(-1)
    largest = torch.full_like(top, LARGEST[form])          # a tensor: divisions by or of a number are products with an inverse
    scaled = x.float() * (largest / top)[..., None]
    return (scaled.round() if form == "int8" else scaled).to(FORMATS[form]), top / largest


def _tables(lens, page, order):
    """Page tables of requests of so many tokens, with the pages in `order`."""
    pages = torch.tensor([_pages_of(n, page) for n in lens], dtype=torch.int32, device="cuda")
    width = max(1, max(_pages_of(n, page) for n in lens))
    tables = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    valid = torch.arange(width, dtype=torch.int32, device="cuda")[None, :] < pages[:, None]
    held = sum(_pages_of(n, page) for n in lens)
    tables[valid] = order[:held]
    return tables, held


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    i32 = dict(dtype=torch.int32, device="cuda")
    dtype, page, d, kv = DTYPES[case["dtype"]], case["page"], case["dim"], case["kv_heads"]

    def coded_pages(pages, form, lean=None):
        """Quantised pages as the store leaves them: of rows of uneven size."""
        codes = torch.empty((pages, kv, page, d), dtype=FORMATS[form], device="cuda")
        scales = torch.empty((pages, kv, page), dtype=torch.float32, device="cuda")
        step = max(1, (1 << 27) // (kv * page * d))
        for i in range(0, pages, step):
            n = min(step, pages - i)
            x = torch.randn((n, kv, page, d), generator=g, device="cuda")
            if lean is not None:
                x.add_(lean)
            x.mul_(torch.randn((n, kv, page, 1), generator=g, device="cuda").mul_(0.3).exp_())
            codes[i:i + n], scales[i:i + n] = _codes(x.to(torch.bfloat16), form)
        return codes, scales

    if case["op"] in ("store", "load"):
        t, pages, form = case["tokens"], case["pages"], case["format"]
        slots = torch.randperm(pages * page, generator=g, device="cuda")[:t]
        if case["op"] == "load":          # tokens of a request follow each other in pages that do not
            order = torch.randperm(pages, generator=g, device="cuda")
            at = torch.arange(t, device="cuda")
            slots = order[at // page] * page + at % page
        if case["skipped"]:
            slots[:: case["skipped"]] = -1
        state = dict(case=case, slots=slots)
        state["key_pages"], state["key_scales"] = coded_pages(pages, form)
        state["value_pages"], state["value_scales"] = coded_pages(pages, form)
        if case["op"] == "store":
            # keys and values as they leave a layer's joint projection: neighbouring columns of one row
            x = torch.randn((t, 2, kv, d), generator=g, device="cuda").mul_(torch.randn((t, 2, kv, 1), generator=g, device="cuda").exp_()).to(dtype)
            state.update(keys=x[:, 0], values=x[:, 1])
        return state
    new, keys = _lens(case)
    held = sum(_pages_of(k, page) for k in keys)
    members, prefixes = _groups(case) if case["op"] == "prefix" else ([], [])
    shared = sum(_pages_of(k, page) for k in prefixes)
    order = torch.randperm(held + shared + 5, generator=g, device="cuda").to(torch.int32)
    state = dict(case=case, lengths=torch.tensor(keys, **i32), tables=_tables(keys, page, order)[0])
    state["starts"] = torch.zeros(len(new) + 1, **i32)
    state["starts"][1:] = torch.tensor(new, **i32).cumsum(0)
    # keys lean to a common direction and queries are long, so that the weights are far from even
    lean = torch.randn((kv, 1, d), generator=g, device="cuda").mul_(0.5)
    if case["op"] == "attention":
        state["key_pages"], state["key_scales"] = coded_pages(held + 5, case["format"], lean)
        state["value_pages"], state["value_scales"] = coded_pages(held + 5, case["format"])
    else:
        shape = (held + shared + 5, kv, page, d)
        state["key_pages"] = torch.randn(shape, generator=g, device="cuda").add_(lean).to(dtype)
        state["value_pages"] = torch.randn(shape, generator=g, device="cuda").to(dtype)
        state["prefix_tables"] = _tables(prefixes, page, order[held:])[0]
        state["prefix_lengths"] = torch.tensor(prefixes, **i32)
        state["group_starts"] = torch.zeros(len(members) + 1, **i32)
        state["group_starts"][1:] = torch.tensor(members, **i32).cumsum(0)
    state["q"] = torch.randn((sum(new), case["heads"], d), generator=g, device="cuda").mul_(2.0).to(dtype)
    state["slopes"] = torch.exp2(-8.0 * torch.arange(1, case["heads"] + 1, device="cuda") / case["heads"]).float() if case["slopes"] else None
    return state


def _plain_store(s):
    case, page = s["case"], s["case"]["page"]
    taken = s["slots"] >= 0
    to = s["slots"][taken]
    for name in ("key", "value"):
        codes, scales = _codes(s[name + "s"][taken], case["format"])
        s[name + "_pages"].view(torch.uint8)[to // page, :, to % page] = codes.view(torch.uint8)
        s[name + "_scales"][to // page, :, to % page] = scales
    return {name: s[name] for name in ("key_pages", "value_pages", "key_scales", "value_scales")}


def _plain_load(s):
    page, dtype = s["case"]["page"], DTYPES[s["case"]["dtype"]]
    taken = s["slots"] >= 0
    to = s["slots"].clamp(min=0)
    out = []
    for name in ("key", "value"):
        codes = s[name + "_pages"].view(torch.uint8)[to // page, :, to % page].view(s[name + "_pages"].dtype)
        x = codes.float() * s[name + "_scales"][to // page, :, to % page][..., None]
        out.append(torch.where(taken[:, None, None], x, 0.0).to(dtype))
    return dict(keys=out[0], values=out[1])


def _gathered(s, name, tables):
    """The keys or values of a table's pages in 32 bits, [requests, key heads, places, head size]."""
    at = tables.long().clamp(min=0)
    pages = s[name + "_pages"]
    b, width = tables.shape
    if name + "_scales" in s:
        x = pages.view(torch.uint8)[at].view(pages.dtype).float() * s[name + "_scales"][at][..., None]
    else:
        x = pages[at].float()
    return x.transpose(1, 2).reshape(b, pages.shape[1], width * pages.shape[2], pages.shape[3])


def _weighted(s, rows, positions, tables, lengths, first, causal):
    """Weights' maxima and sums, and the weighted sums of values, of `rows` [b, n, heads, d] that stand at positions [b, n], over
    the keys of the tables, the first of which stands at `first` [b]."""
    case = s["case"]
    b, n, heads, d = rows.shape
    kv = case["kv_heads"]
    k, v = _gathered(s, "key", tables), _gathered(s, "value", tables)
    places = k.shape[2]
    q = rows.float().view(b, n, kv, heads // kv, d).permute(0, 2, 3, 1, 4).reshape(b, kv, -1, d)
    x = (q @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(b, kv, heads // kv, n, places)
    j = torch.arange(places, device=q.device)
    far = first[:, None, None] + j - positions[:, :, None]
    if case["softcap"]:
        x = torch.tanh(x / case["softcap"]) * case["softcap"]
    if s["slopes"] is not None:
        x = x + s["slopes"].view(1, kv, -1, 1, 1) * far[:, None, None]
    hidden = (j >= lengths[:, None])[:, None]
    if causal:
        hidden = hidden | (far > 0)
    if case["window"]:
        hidden = hidden | (far <= -case["window"])
    x = x.masked_fill_(hidden[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    w = x.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    out = (w.view(b, kv, -1, places) @ v).view(b, kv, heads // kv, n, d)
    return [t.permute(0, 3, 1, 2, 4).reshape(b, n, heads, -1) for t in (top, total, out)]


def _plain_attention(s):
    q, starts, lengths = s["q"], s["starts"].long(), s["lengths"].long()
    b, t, most = lengths.shape[0], q.shape[0], s["case"]["new_hi"]
    n = starts[1:] - starts[:-1]
    r = torch.repeat_interleave(torch.arange(b, device=q.device), n, output_size=t)
    i = torch.arange(t, device=q.device) - starts[r]
    rows = torch.zeros((b, most) + q.shape[1:], dtype=q.dtype, device=q.device)
    rows[r, i] = q
    position = (lengths - n)[:, None] + torch.arange(most, device=q.device)
    top, total, out = [x[r, i] for x in _weighted(s, rows, position, s["tables"], lengths, torch.zeros_like(lengths), s["case"]["causal"])]
    if s["case"]["op"] == "prefix":
        groups = s["group_starts"].long()
        members = groups[1:] - groups[:-1]
        g = torch.repeat_interleave(torch.arange(members.shape[0], device=q.device), members, output_size=b)[r]
        at = torch.arange(t, device=q.device) - starts[groups[g]]
        widest = max(1, _group_tokens(s["case"]))
        rows = torch.zeros((members.shape[0], widest) + q.shape[1:], dtype=q.dtype, device=q.device)
        rows[g, at] = q
        position = torch.zeros((members.shape[0], widest), dtype=torch.int64, device=q.device)
        ahead = s["prefix_lengths"].long()
        position[g, at] = ahead[g] + (lengths - n)[r] + i
        top2, total2, out2 = [x[g, at] for x in _weighted(s, rows, position, s["prefix_tables"], ahead, torch.zeros_like(ahead), False)]
        both = torch.maximum(top, top2)
        f, f2 = torch.exp(top - both), torch.exp(top2 - both)
        top, total, out = both, f * total + f2 * total2, f * out + f2 * out2
    out = out / total.clamp(min=1e-30)
    lse = torch.where(total > 0, top + total.log(), -math.inf)[..., 0]
    return dict(out=out.to(q.dtype), lse=lse)


def _group_tokens(case):
    """The most new tokens of a group."""
    members, _ = _groups(case)
    new, _ = _lens(case)
    ends = [sum(members[:i + 1]) for i in range(len(members))]
    return max(sum(new[e - m:e]) for e, m in zip(ends, members))


def run(state):
    case = state["case"]
    if not own:
        return {"store": _plain_store, "load": _plain_load, "attention": _plain_attention, "prefix": _plain_attention}[case["op"]](state)
    import paper_2607_04415_b200 as gorio
    if case["op"] == "store":
        names = ("key_pages", "value_pages", "key_scales", "value_scales")
        gorio.cache_store_quantized(state["keys"], state["values"], *[state[x] for x in names], state["slots"])
        return {name: state[name] for name in names}
    if case["op"] == "load":
        keys, values = gorio.cache_load_quantized(state["key_pages"], state["value_pages"], state["key_scales"], state["value_scales"], state["slots"],
                                                  dtype=DTYPES[case["dtype"]])
        return dict(keys=keys, values=values)
    scores = dict(causal=case["causal"], window=case["window"], softcap=case["softcap"], slopes=state["slopes"], want_lse=True)
    if case["op"] == "attention":
        return gorio.paged_attention_quantized(state["q"], state["key_pages"], state["value_pages"], state["key_scales"], state["value_scales"],
                                               state["tables"], state["lengths"], state["starts"], case["new_hi"], **scores)
    return gorio.prefix_attention(state["q"], state["key_pages"], state["value_pages"], state["prefix_tables"], state["prefix_lengths"],
                                  state["group_starts"], state["tables"], state["lengths"], state["starts"], case["new_hi"], **scores)


def _seen(case, n, keys, ahead):
    """Pairs of a new token and a key that it sees, and the first and last such key, of a request with `keys` keys behind `ahead` shared ones; of its
    own keys and of the shared ones."""
    found = []
    for lo_all, hi_all, causal in ((0, keys, case["causal"]), (-ahead, 0, False)):
        pairs, lo_key, hi_key = 0, 1 << 60, -1 << 60
        for i in range(n):
            p = keys - n + i
            hi = min(hi_all, p + 1) if causal else hi_all
            lo = max(lo_all, p - case["window"] + 1) if case["window"] else lo_all
            if hi > lo:
                pairs, lo_key, hi_key = pairs + hi - lo, min(lo_key, lo), max(hi_key, hi)
        found.append((pairs, lo_key, hi_key))
    return found


def work(case):
    page, kv, d = case["page"], case["kv_heads"], case["dim"]
    if case["op"] in ("store", "load"):
        t = case["tokens"]
        taken = t - (_pages_of(t, case["skipped"]) if case["skipped"] else 0)
        rows = taken * kv
        # slots; 16-bit rows on one side (what is loaded from no slot is zeros), 8-bit rows and their scales on the other; keys and values
        whole = taken if case["op"] == "store" else t
        return dict(bytes=8 * t + 2 * (2 * d * whole * kv + (d + 4) * rows), flops=0)
    new, keys = _lens(case)
    members, prefixes = _groups(case) if case["op"] == "prefix" else ([len(new)], [0])
    element = 1 + 4 / d if case["op"] == "attention" else 2          # bytes of one; a row's scale is shared by its elements
    pairs = seen = r = 0
    for count, ahead in zip(members, prefixes):
        first = ahead
        for n, k in zip(new[r:r + count], keys[r:r + count]):
            (p, lo, hi), (shared, from_, _) = _seen(case, n, k, ahead)
            pairs += p + shared
            seen += max(0, hi - lo)
            if shared:
                first = min(first, ahead + from_)
        seen += ahead - first
        r += count
    rows = sum(new) * case["heads"]
    return dict(bytes=2 * 2 * rows * d + 4 * rows + 2 * element * seen * kv * d + 4 * _pages_of(seen, page), flops=4 * pairs * case["heads"] * d)


def exact(case, seed):
    s = prepare(case, seed)
    page, kv, d = case["page"], case["kv_heads"], case["dim"]
    if case["op"] == "store":
        got = {}
        taken = (s["slots"] >= 0).nonzero()[:, 0]
        to = s["slots"][taken]
        for name in ("key", "value"):
            x = s[name + "s"].double()[taken]
            top = x.abs().amax(-1)
            # the format's own roundings: scale and its inverse are numbers of 32 bits, and so is what is rounded to 8
            inverse = (LARGEST[case["format"]] / top).float().double()
            codes = (x * inverse[..., None]).float()
            pages = s[name + "_pages"].double()
            scales = s[name + "_scales"].double()
            pages[to // page, :, to % page] = (codes.round().clamp(-127, 127) if case["format"] == "int8" else _e4m3(codes)).double()
            scales[to // page, :, to % page] = top / LARGEST[case["format"]]
            got[name + "_pages"], got[name + "_scales"] = pages, scales
        return got
    if case["op"] == "load":
        got = {}
        taken = (s["slots"] >= 0).nonzero()[:, 0]
        to = s["slots"][taken]
        for name in ("key", "value"):
            out = torch.zeros((case["tokens"], kv, d), dtype=torch.float64, device="cuda")
            out[taken] = s[name + "_pages"].double()[to // page, :, to % page] * s[name + "_scales"].double()[to // page, :, to % page][..., None]
            got[name + "s"] = out
        return got
    q = s["q"]
    new, keys = _lens(case)
    group = case["heads"] // kv
    prefix_of = []
    if case["op"] == "prefix":
        members, prefixes = _groups(case)
        for i, m in enumerate(members):
            prefix_of += [(i, prefixes[i])] * m
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")

    def rows(name, ids, head):
        x = s[name + "_pages"][ids, head].double()
        if name + "_scales" in s:
            x = x * s[name + "_scales"][ids, head].double()[..., None]
        return x.reshape(-1, d)

    begin = 0
    for r, (n, length) in enumerate(zip(new, keys)):
        which, ahead = prefix_of[r] if prefix_of else (0, 0)
        if n == 0 or length + ahead == 0:
            begin += n
            continue
        ids = s["tables"][r, : _pages_of(length, page)].long()
        shared = s["prefix_tables"][which, : _pages_of(ahead, page)].long() if ahead else ids[:0]
        p = torch.arange(ahead + length - n, ahead + length, device="cuda")
        j = torch.arange(ahead + length, device="cuda")
        sees = torch.ones((n, ahead + length), dtype=torch.bool, device="cuda")
        if case["causal"]:
            sees &= (j[None, :] <= p[:, None]) | (j[None, :] < ahead)
        if case["window"]:
            sees &= j[None, :] > p[:, None] - case["window"]
        some = sees.any(1)
        for h in range(kv):
            k = torch.cat([rows("key", shared, h)[:ahead], rows("key", ids, h)[:length]])
            v = torch.cat([rows("value", shared, h)[:ahead], rows("value", ids, h)[:length]])
            at = slice(h * group, h * group + group)
            z = q[begin:begin + n, at].double() @ k.T / math.sqrt(d)          # [n, group, keys]
            if case["softcap"]:
                z = case["softcap"] * torch.tanh(z / case["softcap"])
            if s["slopes"] is not None:
                z = z + s["slopes"][at].double()[None, :, None] * (j[None, :] - p[:, None])[:, None, :]
            z = torch.where(sees[:, None, :], z, -math.inf)
            total = torch.logsumexp(z, 2)
            weight = torch.where(some[:, None, None], torch.exp(z - torch.where(some[:, None], total, 0.0)[:, :, None]), 0.0)
            out[begin:begin + n, at] = weight @ v
            lse[begin:begin + n, at] = total
        begin += n
    return dict(out=out, lse=lse)


def _e4m3(x):
    """To the nearest number of 4 bits of mantissa, the least 2^-9 apart, ties to even."""
    x = x.double().clamp(-448.0, 448.0)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step
