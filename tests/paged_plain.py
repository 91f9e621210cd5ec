"""Plain forms of the paged-cache operators for the tests: page tables by a loop over requests, attention in
64 bits by a loop over queries' heads, with the error that the formulas allow a kernel."""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # largest relative error of one rounding


def ceil_div(a, b):
    return -(-a // b)


def plain_tables(lengths, new_lens, tables, free_pages, free_count, page_size, n_tokens):
    """Lists in, lists out, by the rules of include/gorio.h."""
    tables = [list(r) for r in tables]
    width = len(tables[0]) if tables else 1
    free = min(max(free_count, 0), len(free_pages))
    slots, positions, requests, starts, out_len, served = [], [], [], [0], [], []
    wanted = tokens = taken = 0
    for r, (c, n) in enumerate(zip(lengths, new_lens)):
        ok = c >= 0 and n >= 0 and c + n <= width * page_size
        need = ceil_div(c + n, page_size) - ceil_div(c, page_size) if ok else 0
        first = wanted
        wanted += need
        tokens += max(n, 0)
        yes = ok and wanted <= free and tokens <= n_tokens
        if yes:
            taken = wanted
            held = ceil_div(c, page_size)
            for i in range(need):
                tables[r][held + i] = free_pages[free - 1 - (first + i)]
        for j in range(min(max(n, 0), n_tokens - starts[-1])):
            p = c + j
            requests.append(r)
            positions.append(p)
            slots.append(tables[r][p // page_size] * page_size + p % page_size if yes else -1)
        starts.append(min(tokens, n_tokens))
        out_len.append(c + n if yes else c)
        served.append(int(yes))
    pad = [-1] * (n_tokens - len(slots))
    return dict(tables=tables, slots=slots + pad, positions=positions + pad, requests=requests + pad, starts=starts, lengths=out_len,
                served=served, free_count=[free - taken])


def plain_attention(q, key_pages, value_pages, tables, lengths, starts, causal=True, window=0, softcap=0.0, slopes=None, scale=None):
    """(out, lse, out_tolerance, lse_tolerance) in float64.

    Tolerances, for weights w, the type's unit u and sums of D products in 32 bits: a score is off by at
    most e = D * 2^-23 * scale * sum|q||k| (each of D additions rounds or cuts one unit) plus a few 2^-22 of its own
    size for scale, cap, bias and the change to log2, so a weight by 2e relative to their sum, and by u for its
    rounding (plus, in float16, 2^-25 of the largest weight below the normal numbers); the result rounds once more."""
    t, heads, d = q.shape
    kv = key_pages.shape[1]
    page = key_pages.shape[2]
    group = heads // kv
    dev = q.device
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = torch.zeros((t, heads, d), dtype=torch.float64, device=dev)
    lse = torch.full((t, heads), -math.inf, dtype=torch.float64, device=dev)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    u = UNIT[q.dtype]
    tiny = 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    starts, lengths = starts.tolist(), lengths.tolist()
    for r, length in enumerate(lengths):
        n = starts[r + 1] - starts[r]
        if n <= 0 or length <= 0:
            continue
        ids = tables[r, : ceil_div(length, page)].long()
        p = torch.arange(length - n, length, device=dev)
        j = torch.arange(length, device=dev)
        sees = torch.ones((n, length), dtype=torch.bool, device=dev)
        if causal:
            sees &= j[None] <= p[:, None]
        if window:
            sees &= j[None] > p[:, None] - window
        used = sees.any(0)
        ids = torch.where((ids < 0) | (ids >= key_pages.shape[0]), 0, ids)     # a page given back: no query may see it
        for h in range(heads):
            k = key_pages[ids, h // group].reshape(-1, d)[:length].double()
            v = value_pages[ids, h // group].reshape(-1, d)[:length].double()
            k[~used] = 0
            v[~used] = 0
            qh = q[starts[r]:starts[r + 1], h].double()
            x = qh @ k.T * scale
            e = d * 2.0 ** -23 * scale * (qh.abs() @ k.abs().T)
            if softcap:
                x = softcap * torch.tanh(x / softcap)
                e = e + softcap * 2.0 ** -20
            if slopes is not None:
                x = x + slopes[h].double() * (j[None] - p[:, None])
            e = e + 2.0 ** -21 * x.abs()
            x = torch.where(sees, x, -math.inf)
            top = x.amax(1, keepdim=True)
            w = torch.where(sees, torch.exp(x - torch.where(torch.isfinite(top), top, 0.0)), 0.0)
            total = w.sum(1, keepdim=True)
            w = torch.where(total > 0, w / total, 0.0)
            rows = slice(starts[r], starts[r + 1])
            bad = ~torch.isfinite(v).all(1)
            if bad.any():                                      # 0 * inf: only the queries that see such a value have it
                clean = torch.where(torch.isfinite(v), v, 0.0)
                o = w @ clean
                for key in bad.nonzero()[:, 0].tolist():
                    o = torch.where(sees[:, key:key + 1], o + w[:, key:key + 1] * torch.where(torch.isfinite(v[key]), 0.0, v[key]), o)
            else:
                clean, o = v, w @ v
            eb = torch.where(sees, e, 0.0).amax(1, keepdim=True)
            a = w @ clean.abs()
            out[rows, h] = o
            out_tol[rows, h] = u * o.abs() + (u + 2 * eb + 2.0 ** -18) * a + tiny * length * clean.abs().amax()
            lse[rows, h] = (torch.where(torch.isfinite(top), top, 0.0) + total.log())[:, 0]
            lse_tol[rows, h] = eb[:, 0] + 2.0 ** -18 + 2.0 ** -21 * torch.where(torch.isfinite(lse[rows, h]), lse[rows, h].abs(), 0.0)
    return out, lse, out_tol, lse_tol
