"""From a search to the tokens that attend over what it found, on one GPU.

Each node of the index stands for a passage of `passage_tokens` tokens whose keys and values (of one attention layer)
lie in pages of a cache.  A batch of questions is searched; the passages found become the first pages of each
question's table row, shared between the questions that found the same ones; the question's own tokens get
pages from the free ones, attend over passages and themselves, and then answer tokens follow one at a time.

    python examples/retrieve_and_attend.py            # prints what it did; needs the GPU and the built library
"""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2607_04415_b200 as gorio  # noqa: E402
from workloads import make_config  # noqa: E402


def main(questions=64, found=5, passage_tokens=32, steps=4, heads=32, kv_heads=8, dim=128, page_size=16, scale=0.05, seed=0):
    """Returns the last step's tensors: everything that the attention read, and its result."""
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev).manual_seed(seed)
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
    own_pages = questions * 8
    n_pages = w.N * per_passage + own_pages
    shape = (n_pages, kv_heads, page_size, dim)
    key_pages = torch.empty(shape, dtype=torch.bfloat16, device=dev)
    value_pages = torch.empty(shape, dtype=torch.bfloat16, device=dev)
    for pages in (key_pages, value_pages):
        pages[: w.N * per_passage] = torch.randn((w.N * per_passage,) + shape[1:], generator=g, device=dev)
    free_pages = torch.arange(w.N * per_passage, n_pages, dtype=torch.int32, device=dev)
    free_count = torch.tensor([own_pages], dtype=torch.int32, device=dev)

    # 3. each question's table row begins with the pages of its passages
    tables = torch.full((questions, found * per_passage + 8), -1, dtype=torch.int32, device=dev)
    pages_of = ids[:, :, None] * per_passage + torch.arange(per_passage, device=dev)
    tables[:, : found * per_passage] = pages_of.reshape(questions, -1).int()
    lengths = torch.full((questions,), found * passage_tokens, dtype=torch.int32, device=dev)

    # 4. the question's tokens in one chunk, then answer tokens one by one
    new = [3 + (7 * i) % 20 for i in range(questions)]
    last = None
    for step in range(1 + steps):
        total, most = (sum(new), max(new)) if step == 0 else (questions, 1)
        new_lens = torch.tensor(new, dtype=torch.int32, device=dev) if step == 0 else torch.ones(questions, dtype=torch.int32, device=dev)
        plan = gorio.page_tables(lengths, new_lens, tables, free_pages, free_count, page_size, total)
        lengths, free_count = plan["lengths"], plan["free_count"]
        # what a layer's projections give for the new tokens: queries, and keys and values side by side
        q = torch.randn((total, heads, dim), generator=g, device=dev).bfloat16()
        kv = torch.randn((total, 2, kv_heads, dim), generator=g, device=dev).bfloat16()
        gorio.cache_store(kv[:, 0], kv[:, 1], key_pages, value_pages, plan["slots"])
        out = gorio.paged_attention(q, key_pages, value_pages, tables, lengths, plan["starts"], most, want_lse=True)
        last = dict(q=q, key_pages=key_pages, value_pages=value_pages, tables=tables, lengths=lengths, starts=plan["starts"], served=plan["served"],
                    free_count=free_count, **out)
    gorio.attention_check()
    return last


if __name__ == "__main__":
    r = main()
    print(f"{r['lengths'].numel()} questions, {int(r['lengths'].min())} to {int(r['lengths'].max())} keys each, "
          f"{int(r['served'].sum())} served in the last step, {int(r['free_count'])} pages left; output norm {r['out'].float().norm():.3f}")
