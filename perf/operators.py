"""The operators of the paged key/value cache, as cases to measure: page tables and slot maps built from request
lengths, the store of new keys and values, and attention of new tokens over the cached pages.

`run` computes a case in its plain form (elementary torch operations in 32 bits) or, with `own` set, by the
package's kernels.  A cache's page tensors are [pages, key heads, page size, head size]."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one decode step of a small server: 32 requests, one new token each
        dict(name="tables_decode", op="tables", requests=32, new_lo=1, new_hi=1, cached_lo=0, cached_hi=4096, page=16, spread=1),
        # a mixed step: some requests wait (0 new), others bring a piece of a prompt; pages of an odd size
        dict(name="tables_mixed", op="tables", requests=1000, new_lo=0, new_hi=130, cached_lo=0, cached_hi=9000, page=24, spread=2),
        # an offline job admits many prompts at once
        dict(name="tables_admit", op="tables", requests=8192, new_lo=1, new_hi=64, cached_lo=0, cached_hi=512, page=16, spread=3),
        # the new keys and values of one decode step
        dict(name="store_decode", op="store", tokens=64, kv_heads=8, dim=128, page=16, pages=1024, dtype="bf16", skipped=0),
        # those of a long prompt, an odd number of tokens, some of them not admitted
        dict(name="store_prompt", op="store", tokens=16383, kv_heads=8, dim=128, page=16, pages=1100, dtype="bf16", skipped=7),
        # one user, one token: latency counts
        dict(name="decode_one", op="attention", requests=1, new_lo=1, new_hi=1, len_lo=4097, len_hi=4097, heads=32, kv_heads=8,
             dim=128, page=16, dtype="bf16", causal=True, window=0, softcap=0.0, slopes=False, spread=4),
        # a server's decode step, ragged lengths
        dict(name="decode_batch", op="attention", requests=64, new_lo=1, new_hi=1, len_lo=100, len_hi=8192, heads=32, kv_heads=8,
             dim=128, page=16, dtype="bf16", causal=True, window=0, softcap=0.0, slopes=False, spread=5),
        # few requests over very long caches
        dict(name="decode_long", op="attention", requests=3, new_lo=1, new_hi=1, len_lo=65537, len_hi=131072, heads=32, kv_heads=8,
             dim=128, page=64, dtype="bf16", causal=True, window=0, softcap=0.0, slopes=False, spread=6),
        # a mixed step: single tokens beside pieces of prompts; every head has its own keys
        dict(name="chunk_mixed", op="attention", requests=12, new_lo=1, new_hi=512, len_lo=512, len_hi=4096, heads=16, kv_heads=16,
             dim=64, page=16, dtype="fp16", causal=True, window=0, softcap=0.0, slopes=False, spread=7),
        # layers that cap their scores, add a bias by distance and see a window
        dict(name="chunk_scored", op="attention", requests=4, new_lo=100, new_hi=700, len_lo=1000, len_hi=8192, heads=16, kv_heads=4,
             dim=128, page=32, dtype="bf16", causal=True, window=1500, softcap=30.0, slopes=True, spread=8),
        # questions over retrieved passages, which all of a question's tokens see; some questions have none
        dict(name="chunk_passages", op="attention", requests=31, new_lo=5, new_hi=77, len_lo=0, len_hi=2001, heads=14, kv_heads=2,
             dim=96, page=16, dtype="fp16", causal=False, window=0, softcap=0.0, slopes=False, spread=9),
        # a piece of one long prompt over what is cached of it: the largest
        dict(name="chunk_prompt", op="attention", requests=1, new_lo=2048, new_hi=2048, len_lo=18432, len_hi=18432, heads=32, kv_heads=8,
             dim=128, page=16, dtype="bf16", causal=True, window=0, softcap=0.0, slopes=False, spread=10),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tables", "store", "attention", "attention", "attention"])
    spread = rng.randrange(1000, 1 << 30)
    if op == "tables":
        b = _log(rng, 1, 8192)
        hi = _log(rng, 1, max(1, min(4096, 250000 // b)))
        return dict(op=op, requests=b, new_lo=rng.randint(0, 1), new_hi=hi, cached_lo=0, cached_hi=_log(rng, 1, max(16, min(65536, 4000000 // b))),
                    page=rng.choice([8, 16, 24, 32, 64, 128]), spread=spread)
    if op == "store":
        t = _log(rng, 1, 16383)
        page = rng.choice([8, 16, 24, 32, 64])
        return dict(op=op, tokens=t, kv_heads=rng.choice([1, 2, 3, 4, 8]), dim=rng.choice([64, 96, 128]), page=page,
                    pages=t // page + rng.randint(2, 60), dtype=rng.choice(["bf16", "fp16"]), skipped=rng.choice([0, 0, 5]))
    kv_heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 5, 7, 8])
    dim = rng.choice([64, 96, 128])
    if kv_heads * group * dim > 4096:
        group = 4
    if kv_heads * group == 32 and dim == 96:
        dim = 128
    new_hi = 1 if rng.random() < 0.5 else _log(rng, 2, 2048)
    b = _log(rng, 1, 64 if new_hi == 1 else 16)
    if new_hi == 1:
        most = min(131072, 250000 // b)                           # keys of a request, so that all of them stay below decode_long's
    else:
        most = min(18432, 400000 // b, 30000000 // (b * new_hi))  # and the scores below chunk_prompt's
    len_hi = _log(rng, min(new_hi + 1, most), most)
    extra = rng.random()
    return dict(op=op, requests=b, new_lo=rng.choice([1, new_hi]), new_hi=new_hi, len_lo=rng.choice([1, max(1, len_hi // 2), len_hi]), len_hi=len_hi,
                heads=kv_heads * group, kv_heads=kv_heads, dim=dim, page=rng.choice([8, 16, 16, 32, 48, 64, 128]), dtype=rng.choice(["bf16", "fp16"]),
                causal=rng.random() < 0.75, window=_log(rng, 1, len_hi) if extra < 0.2 else 0, softcap=rng.choice([20.0, 50.0]) if 0.1 < extra < 0.3 else 0.0,
                slopes=0.2 < extra < 0.4, spread=spread)


def _numbers(case, count, lo, hi, salt):
    """`count` whole numbers of [lo, hi], by the case alone: its lengths are part of the case."""
    rng = random.Random(case["spread"] * 10 + salt)
    return [rng.randint(lo, hi) for _ in range(count)]


def _lens(case):
    """New tokens and keys of each request of an attention case: where causal, the keys hold the new tokens' own."""
    new = _numbers(case, case["requests"], case["new_lo"], case["new_hi"], 1)
    keys = _numbers(case, case["requests"], case["len_lo"], case["len_hi"], 2)
    if case["causal"]:
        keys = [max(k, n) for k, n in zip(keys, new)]
    return new, keys


def _pages_of(tokens, page):
    return -(-tokens // page)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    i32 = dict(dtype=torch.int32, device="cuda")
    page = case["page"]
    if case["op"] == "tables":
        b = case["requests"]
        new = _numbers(case, b, case["new_lo"], case["new_hi"], 1)
        cached = _numbers(case, b, case["cached_lo"], case["cached_hi"], 2)
        width = max(_pages_of(c + n, page) for c, n in zip(cached, new))
        width += width == 0
        held = sum(_pages_of(c, page) for c in cached)
        need = sum(_pages_of(c + n, page) - _pages_of(c, page) for c, n in zip(cached, new))
        order = torch.randperm(held + need + 100, generator=g, device="cuda").to(torch.int32)
        cached_t = torch.tensor(cached, **i32)
        col = torch.arange(width, **i32)
        valid = col[None, :] < ((cached_t + page - 1) // page)[:, None]
        tables = torch.full((b, width), -1, **i32)
        tables[valid] = order[:held]
        return dict(case=case, lengths=cached_t, new_lens=torch.tensor(new, **i32), tables=tables, free_pages=order[held:].clone(),
                    free_count=torch.tensor([need + 100], **i32), tokens=sum(new))
    dtype = DTYPES[case["dtype"]]
    d = case["dim"]
    if case["op"] == "store":
        t, pages = case["tokens"], case["pages"]
        shape = (pages, case["kv_heads"], page, d)
        slots = torch.randperm(pages * page, generator=g, device="cuda")[:t]
        if case["skipped"]:
            slots[:: case["skipped"]] = -1
        # keys and values as they leave a layer's joint projection: neighbouring columns of one row
        kv = torch.randn((t, 2, case["kv_heads"], d), generator=g, device="cuda").to(dtype)
        return dict(case=case, keys=kv[:, 0], values=kv[:, 1], slots=slots, key_pages=torch.randn(shape, generator=g, device="cuda").to(dtype),
                    value_pages=torch.randn(shape, generator=g, device="cuda").to(dtype))
    new, keys = _lens(case)
    width = max(1, max(_pages_of(k, page) for k in keys))
    held = sum(_pages_of(k, page) for k in keys)
    order = torch.randperm(held + 5, generator=g, device="cuda").to(torch.int32)
    lengths = torch.tensor(keys, **i32)
    valid = torch.arange(width, **i32)[None, :] < ((lengths + page - 1) // page)[:, None]
    tables = torch.full((len(new), width), -1, **i32)
    tables[valid] = order[:held]
    starts = torch.zeros(len(new) + 1, **i32)
    starts[1:] = torch.tensor(new, **i32).cumsum(0)
    shape = (held + 5, case["kv_heads"], page, d)
    # keys lean to a common direction and queries are long, so that the weights are far from even
    lean = torch.randn((case["kv_heads"], 1, d), generator=g, device="cuda").mul_(0.5)
    key_pages = torch.empty(shape, dtype=dtype, device="cuda")
    value_pages = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 28) // (case["kv_heads"] * page * d))
    for i in range(0, held + 5, step):
        n = min(step, held + 5 - i)
        key_pages[i:i + n] = torch.randn((n,) + shape[1:], generator=g, device="cuda").add_(lean)
        value_pages[i:i + n] = torch.randn((n,) + shape[1:], generator=g, device="cuda")
    q = torch.randn((sum(new), case["heads"], d), generator=g, device="cuda").mul_(2.0).to(dtype)
    slopes = torch.exp2(-8.0 * torch.arange(1, case["heads"] + 1, device="cuda") / case["heads"]).float() if case["slopes"] else None
    return dict(case=case, q=q, key_pages=key_pages, value_pages=value_pages, tables=tables, lengths=lengths, starts=starts, slopes=slopes)


def _plain_tables(s):
    case, page = s["case"], s["case"]["page"]
    c, n, tables, free, f = s["lengths"].long(), s["new_lens"].long(), s["tables"], s["free_pages"], s["free_count"].long()
    b, width = tables.shape
    held, after = (c + page - 1) // page, (c + n + page - 1) // page
    ok = (c >= 0) & (n >= 0) & (after <= width)
    need = torch.where(ok, after - held, 0)
    upto = need.cumsum(0)
    served = ok & (upto <= f)
    brought = n.clamp(min=0)
    starts = torch.zeros(b + 1, dtype=torch.int64, device=c.device)
    starts[1:] = brought.cumsum(0)
    r = torch.repeat_interleave(torch.arange(b, device=c.device), brought, output_size=s["tokens"])
    position = c[r] + torch.arange(s["tokens"], device=c.device) - starts[r]
    at = position // page
    old = tables[r, at.clamp(max=width - 1)].long()
    fresh = free[(f - 1 - (upto[r] - need[r] + at - held[r])).clamp(0, free.numel() - 1)].long()
    in_page = torch.where(served[r] & (at >= held[r]), fresh, old)
    tables[r, at.clamp(max=width - 1)] = in_page.int()
    slots = torch.where(served[r], in_page * page + position % page, -1)
    return dict(tables=tables, slots=slots, positions=position.int(), requests=r.int(), starts=starts.int(), lengths=torch.where(served, c + n, c).int(),
                served=served.int(), free_count=(f - torch.where(served, need, 0).sum()).int())


def _plain_store(s):
    page = s["case"]["page"]
    taken = s["slots"] >= 0
    to = s["slots"][taken]
    s["key_pages"][to // page, :, to % page] = s["keys"][taken]
    s["value_pages"][to // page, :, to % page] = s["values"][taken]
    return dict(key_pages=s["key_pages"], value_pages=s["value_pages"])


def _plain_attention(s):
    case = s["case"]
    q, starts, lengths = s["q"], s["starts"].long(), s["lengths"].long()
    b, width = s["tables"].shape
    t, heads, d = q.shape
    kv, page = case["kv_heads"], case["page"]
    most = case["new_hi"]
    n = starts[1:] - starts[:-1]
    r = torch.repeat_interleave(torch.arange(b, device=q.device), n, output_size=t)
    i = torch.arange(t, device=q.device) - starts[r]
    rows = torch.zeros((b, most, heads, d), device=q.device)
    rows[r, i] = q.float()
    at = s["tables"].long().clamp(min=0)
    k = s["key_pages"][at].transpose(1, 2).reshape(b, kv, width * page, d).float()
    v = s["value_pages"][at].transpose(1, 2).reshape(b, kv, width * page, d).float()
    rows = rows.view(b, most, kv, heads // kv, d).permute(0, 2, 3, 1, 4).reshape(b, kv, -1, d)
    x = (rows @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(b, kv, heads // kv, most, width * page)
    j = torch.arange(width * page, device=q.device)
    p = (lengths - n)[:, None] + torch.arange(most, device=q.device)
    far = j - p[:, :, None]
    if case["softcap"]:
        x = torch.tanh(x / case["softcap"]) * case["softcap"]
    if s["slopes"] is not None:
        x = x + s["slopes"].view(1, kv, -1, 1, 1) * far[:, None, None]
    hidden = (j >= lengths[:, None])[:, None]
    if case["causal"]:
        hidden = hidden | (far > 0)
    if case["window"]:
        hidden = hidden | (far <= -case["window"])
    x = x.masked_fill_(hidden[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    w = x.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    out = (w.view(b, kv, -1, width * page) @ v).view(b, kv, heads // kv, most, d) / total.clamp(min=1e-30)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    out = out.permute(0, 3, 1, 2, 4).reshape(b, most, heads, d)[r, i]
    lse = lse.permute(0, 3, 1, 2, 4).reshape(b, most, heads)[r, i]
    return dict(out=out.to(q.dtype), lse=lse)


def run(state):
    case = state["case"]
    if not own:
        return {"tables": _plain_tables, "store": _plain_store, "attention": _plain_attention}[case["op"]](state)
    import paper_2607_04415_b200 as gorio
    if case["op"] == "tables":
        return gorio.page_tables(state["lengths"], state["new_lens"], state["tables"], state["free_pages"], state["free_count"], case["page"], state["tokens"])
    if case["op"] == "store":
        gorio.cache_store(state["keys"], state["values"], state["key_pages"], state["value_pages"], state["slots"])
        return dict(key_pages=state["key_pages"], value_pages=state["value_pages"])
    return gorio.paged_attention(state["q"], state["key_pages"], state["value_pages"], state["tables"], state["lengths"], state["starts"], case["new_hi"],
                                 causal=case["causal"], window=case["window"], softcap=case["softcap"], slopes=state["slopes"], want_lse=True)


def work(case):
    page = case["page"]
    if case["op"] == "tables":
        new = _numbers(case, case["requests"], case["new_lo"], case["new_hi"], 1)
        cached = _numbers(case, case["requests"], case["cached_lo"], case["cached_hi"], 2)
        fresh = sum(_pages_of(c + n, page) - _pages_of(c, page) for c, n in zip(cached, new))
        # in: two numbers a request, the open page's entry, the free pages taken; out: 16 bytes a token, three numbers a request, the new entries
        open_pages = sum(1 for c, n in zip(cached, new) if n and c % page)
        return dict(bytes=8 * len(new) + 4 * open_pages + 4 * fresh + 16 * sum(new) + 12 * len(new) + 4 * fresh, flops=0)
    if case["op"] == "store":
        t = case["tokens"]
        taken = t - (_pages_of(t, case["skipped"]) if case["skipped"] else 0)
        return dict(bytes=8 * t + 2 * 2 * 2 * taken * case["kv_heads"] * case["dim"], flops=0)
    new, keys = _lens(case)
    pairs = seen = 0                                   # pairs of a query and a key it sees; keys that some query sees
    for n, k in zip(new, keys):
        reach = []
        for i in range(n):
            p = k - n + i
            hi = min(k, p + 1) if case["causal"] else k
            lo = max(0, p - case["window"] + 1) if case["window"] else 0
            if hi > lo:
                pairs += hi - lo
                reach.append((lo, hi))
        seen += max(h for _, h in reach) - min(l for l, _ in reach) if reach else 0
    rows = sum(new) * case["heads"]
    return dict(bytes=2 * 2 * rows * case["dim"] + 4 * rows + 2 * 2 * seen * case["kv_heads"] * case["dim"] + 4 * _pages_of(seen, page),
                flops=4 * pairs * case["heads"] * case["dim"])


def exact(case, seed):
    if case["op"] == "tables":
        return None                                    # whole numbers
    s = prepare(case, seed)
    page = case["page"]
    if case["op"] == "store":
        got = {}
        for name in ("key", "value"):
            flat = s[name + "_pages"].double().permute(0, 2, 1, 3).reshape(-1, case["kv_heads"], case["dim"])
            taken = (s["slots"] >= 0).nonzero()[:, 0]
            flat[s["slots"][taken]] = s[name + "s"].double()[taken]
            got[name + "_pages"] = flat.view(-1, page, case["kv_heads"], case["dim"]).permute(0, 2, 1, 3).contiguous()
        return got
    q = s["q"]
    new, keys = _lens(case)
    d, group = case["dim"], case["heads"] // case["kv_heads"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    begin = 0
    for r, (n, length) in enumerate(zip(new, keys)):
        if n == 0 or length == 0:
            begin += n
            continue
        ids = s["tables"][r, : _pages_of(length, page)].long()
        p = torch.arange(length - n, length, device="cuda")
        j = torch.arange(length, device="cuda")
        sees = torch.ones((n, length), dtype=torch.bool, device="cuda")
        if case["causal"]:
            sees &= j[None, :] <= p[:, None]
        if case["window"]:
            sees &= j[None, :] > p[:, None] - case["window"]
        some = sees.any(1)
        for h in range(case["heads"]):
            k = s["key_pages"][ids, h // group].reshape(-1, d)[:length].double()
            v = s["value_pages"][ids, h // group].reshape(-1, d)[:length].double()
            z = q[begin:begin + n, h].double() @ k.T / math.sqrt(d)
            if case["softcap"]:
                z = case["softcap"] * torch.tanh(z / case["softcap"])
            if s["slopes"] is not None:
                z = z + s["slopes"][h].double() * (j[None, :] - p[:, None])
            z = torch.where(sees, z, -math.inf)
            total = torch.logsumexp(z, 1)
            weight = torch.where(some[:, None], torch.exp(z - torch.where(some, total, 0.0)[:, None]), 0.0)
            out[begin:begin + n, h] = weight @ v
            lse[begin:begin + n, h] = total
        begin += n
    return dict(out=out, lse=lse)
