"""Several answers to each question over the passages that a search found, and a cache in 8 bits for what is kept, on one GPU.

Each node of the index stands for a passage whose keys and values (of one attention layer) lie in pages of a cache.  A batch of
questions is searched; a question's passages are the prefix that its answers share, so that each is read once a step for
all of them, and every answer has pages of its own for the tokens it adds (prefix_attention).  What has been answered is then
kept in 8 bits (cache_store_quantized) for a conversation to go on over it (paged_attention_quantized), and can be
read back (cache_load_quantized).

    python examples/sample_and_keep.py            # prints what it did; needs the GPU and the built library
"""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2607_04415_b200 as gorio  # noqa: E402
from workloads import make_config  # noqa: E402


def main(questions=16, answers=8, found=5, passage_tokens=32, steps=20, heads=32, kv_heads=8, dim=128, page_size=16, scale=0.05, seed=0,
         codes=torch.float8_e4m3fn):
    """Returns what the last step of each part read and gave."""
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev).manual_seed(seed)
    i32 = dict(dtype=torch.int32, device=dev)
    w = make_config(1, scale=scale, nq=questions)

    # 1. search: the ids of the passages each question gets
    ix = gorio.Index.from_workload(w)
    try:
        ix.cache_config(w.n_pages, preload=True)
        ids = ix.search(torch.as_tensor(w.queries).to(dev), K=found, L=w.L, W=w.W)["ids"].long()
    finally:
        ix.close()

    # 2. the cache: passage i owns pages [i * per_passage, (i + 1) * per_passage); the pages behind them are free
    per_passage = passage_tokens // page_size
    requests = questions * answers
    width = steps // page_size + 1
    n_pages = w.N * per_passage + requests * width
    shape = (n_pages, kv_heads, page_size, dim)
    key_pages = torch.empty(shape, dtype=torch.bfloat16, device=dev)
    value_pages = torch.empty(shape, dtype=torch.bfloat16, device=dev)
    for pages in (key_pages, value_pages):
        pages[: w.N * per_passage] = torch.randn((w.N * per_passage,) + shape[1:], generator=g, device=dev)
    free_pages = torch.arange(w.N * per_passage, n_pages, **i32)
    free_count = torch.tensor([requests * width], **i32)

    # 3. a question is a group: its passages are the prefix of all its answers, whose own tables are empty
    pages_of = ids[:, :, None] * per_passage + torch.arange(per_passage, device=dev)
    prefix_tables = pages_of.reshape(questions, -1).int()
    prefix_lengths = torch.full((questions,), found * passage_tokens, **i32)
    group_starts = torch.arange(0, requests + 1, answers, **i32)
    tables = torch.full((requests, width), -1, **i32)
    lengths = torch.zeros(requests, **i32)
    ones = torch.ones(requests, **i32)
    shared = None
    for _ in range(steps):
        plan = gorio.page_tables(lengths, ones, tables, free_pages, free_count, page_size, requests)
        lengths, free_count = plan["lengths"], plan["free_count"]
        # what a layer's projections give for the new tokens: queries, and keys and values side by side
        q = torch.randn((requests, heads, dim), generator=g, device=dev).bfloat16()
        kv = torch.randn((requests, 2, kv_heads, dim), generator=g, device=dev).bfloat16()
        gorio.cache_store(kv[:, 0], kv[:, 1], key_pages, value_pages, plan["slots"])
        out = gorio.prefix_attention(q, key_pages, value_pages, prefix_tables, prefix_lengths, group_starts, tables, lengths, plan["starts"], 1, want_lse=True)
        shared = dict(q=q, key_pages=key_pages, value_pages=value_pages, prefix_tables=prefix_tables, prefix_lengths=prefix_lengths, tables=tables,
                      lengths=lengths, group_of=torch.arange(requests, device=dev) // answers, **out)

    # 4. one answer of each question is kept: passages and answer, in 8 bits and pages of another cache
    kept = torch.arange(0, requests, answers, device=dev)
    tokens = found * passage_tokens + steps
    per_question = tokens // page_size + 1
    place = torch.arange(tokens, device=dev)
    own = (place - found * passage_tokens).clamp(min=0)
    page = torch.where(place < found * passage_tokens, prefix_tables[:, (place // page_size).clamp(max=prefix_tables.shape[1] - 1)].long(),
                       tables[kept][:, own // page_size].long())
    at = torch.where(place < found * passage_tokens, place, own) % page_size
    keys, values = key_pages[page, :, at.expand(questions, -1)], value_pages[page, :, at.expand(questions, -1)]
    coded = (questions * (per_question + 1), kv_heads, page_size, dim)
    key_codes, value_codes = (torch.zeros(coded, dtype=torch.uint8, device=dev).view(codes) for _ in range(2))
    key_scales, value_scales = (torch.zeros(coded[:3], device=dev) for _ in range(2))
    coded_tables = torch.full((questions, per_question + 1), -1, **i32)
    coded_lengths, coded_free = torch.zeros(questions, **i32), torch.tensor([coded[0]], **i32)
    stack = torch.arange(coded[0], **i32)
    plan = gorio.page_tables(coded_lengths, torch.full((questions,), tokens, **i32), coded_tables, stack, coded_free, page_size, questions * tokens)
    gorio.cache_store_quantized(keys.reshape(-1, kv_heads, dim), values.reshape(-1, kv_heads, dim), key_codes, value_codes, key_scales, value_scales, plan["slots"])
    back = gorio.cache_load_quantized(key_codes, value_codes, key_scales, value_scales, plan["slots"])

    # 5. the next question of the conversation: a chunk of new tokens over what was kept
    new = 7
    plan = gorio.page_tables(plan["lengths"], torch.full((questions,), new, **i32), coded_tables, stack, plan["free_count"], page_size, questions * new)
    q = torch.randn((questions * new, heads, dim), generator=g, device=dev).bfloat16()
    kv = torch.randn((questions * new, 2, kv_heads, dim), generator=g, device=dev).bfloat16()
    gorio.cache_store_quantized(kv[:, 0], kv[:, 1], key_codes, value_codes, key_scales, value_scales, plan["slots"])
    out = gorio.paged_attention_quantized(q, key_codes, value_codes, key_scales, value_scales, coded_tables, plan["lengths"], plan["starts"], new, want_lse=True)
    gorio.attention_check()
    return dict(shared=shared, keys=keys.reshape(-1, kv_heads, dim), values=values.reshape(-1, kv_heads, dim), back=back,
                kept=dict(q=q, key_codes=key_codes, value_codes=value_codes, key_scales=key_scales, value_scales=value_scales, tables=coded_tables,
                          lengths=plan["lengths"], starts=plan["starts"], served=plan["served"], **out))


if __name__ == "__main__":
    r = main()
    s, k = r["shared"], r["kept"]
    off = ((r["back"][0].float() - r["keys"].float()).norm() / r["keys"].float().norm()).item()
    print(f"{s['lengths'].numel()} answers of {int(s['lengths'][0])} tokens over {int(s['prefix_lengths'][0])} shared ones; "
          f"kept in 8 bits ({100 * off:.1f} % off), {int(k['served'].sum())} conversations of {int(k['lengths'][0])} keys went on; "
          f"output norm {k['out'].float().norm():.3f}")
