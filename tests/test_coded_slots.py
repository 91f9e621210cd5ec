"""The slots through which the chunk kernel over codes hands a tile's scales to its two softmax warpgroups: a wait by parity may pass only
when that tile's scales are there.  On the CPU all orders in which the warps can run are walked through, with the numbers of slots and of told parts that
the kernel has; on the GPU batches with runs of short requests, which bring one warpgroup ahead of the other."""
import os
import random
import re

import pytest
import torch

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_04415_b200", "csrc", "paged")


def _constant(file, name):
    with open(os.path.join(CSRC, file)) as f:
        return int(re.search(rf"constexpr int {name} = (\d+);", f.read()).group(1))


def _early_pass(parts, slots, told):
    """`parts`: (tiles, one row tile?) of a block's parts in their order; all are whole units, so that of a part of one row tile and one key tile the second
    warpgroup has nothing, and waits for nothing.  Returns (tiles filled, warpgroup, tile) where a tile is read whose scales are not there, or None.

    A state is the tiles filled so far and, for each warpgroup, its part and the steps that it has made in it.  A fill takes a slot whose last tile
    has been read, of a part that has been told: parts are told `told` ahead of the last one that everybody is done with.  A warpgroup waits for a tile's
    scales (the slot's barrier is not in the phase of the parity it waits for), then for its scores: they come after all products of the parts before and after
    that of the tile before on its row tile.  Where parts are worked on by both, they meet at the end."""
    first = [0]
    for n, _ in parts:
        first.append(first[-1] + n)
    where = [(p, i) for p, (n, _) in enumerate(parts) for i in range(n)]
    steps = []                                     # of each warpgroup, of each part
    for t in range(2):
        steps.append([[(what, first[p] + i) for i in (range(t, n, 2) if one else range(n)) for what in ("scales", "scores")] +
                      ([("meet", p)] if n > 1 or not one else []) for p, (n, one) in enumerate(parts)])

    def made(state, t, p, step):
        at, s = state[1 + t]
        return at > p or (at == p and step in steps[t][p][:s])

    def read(state, tile):                         # by all that read it
        p, i = where[tile]
        return all(made(state, t, p, ("scores", tile)) for t in ([i & 1] if parts[p][1] else [0, 1]))

    def moves(state):
        filled = state[0]
        done = min(state[1][0], state[2][0])
        if filled < first[-1] and where[filled][0] < done + told and (filled < slots or read(state, filled - slots)):
            yield (filled + 1,) + state[1:], None
        for t in range(2):
            p, s = state[1 + t]
            if p == len(parts) or p >= done + told:
                continue
            bad = None
            if steps[t][p]:
                what, of = steps[t][p][s]
                if what == "meet":
                    other, at = state[2 - t]
                    if other < p or (other == p and steps[1 - t][p][at][0] != "meet"):
                        continue
                elif what == "scales":
                    times = (filled - of % slots + slots - 1) // slots      # the slot has been filled so often
                    if times % 2 == (of // slots) % 2:
                        continue
                else:
                    if not all(read(state, i) for i in range(first[p])) or not all(made(state, t, p, x) for x in steps[t][p][:s]):
                        continue
                    bad = (filled, t, of) if filled <= of else None
            then = list(state)
            then[1 + t] = (p, s + 1) if s + 1 < len(steps[t][p]) else (p + 1, 0)
            yield tuple(then), bad
    start = (0, (0, 0), (0, 0))
    seen, todo = {start}, [start]
    while todo:
        state = todo.pop()
        ways = list(moves(state))
        assert ways or state[1][0] == state[2][0] == len(parts), f"nobody can go on: {state}"
        for then, bad in ways:
            if bad is not None:
                return bad
            if then not in seen:
                seen.add(then)
                todo.append(then)
    return None


def test_no_wait_for_scales_passes_before_they_are_there():
    slots, told = _constant("coded_chunk.cuh", "kScaleSlots"), _constant("chunk.cuh", "kParts")
    runs = [[(1, True)] * n + [(m, one)] + [(3, True)] for n in range(1, 7) for m in (1, 2, 3, 5) for one in (True, False)]
    rng = random.Random(1)
    runs += [[(rng.choice([1, 1, 1, 2, 3, 4]), rng.random() < 0.8) for _ in range(9)] for _ in range(60)]
    for run in runs:
        assert _early_pass(run, slots, told) is None, run
    assert _early_pass([(1, True)] * 3 + [(2, True)], 4, 4) is not None     # four slots are too few for four parts


@pytest.mark.gpu
@pytest.mark.parametrize("form", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_runs_of_short_requests_before_longer_ones(form, dim):
    """More units than blocks, at most 128 rows each; runs of three and more requests of at most 128 keys, then ones of several tiles."""
    from paper_2607_04415_b200 import build
    build.build()
    import paper_2607_04415_b200 as gorio
    from more_plain import assert_near
    from paged_wide import widen
    from test_quantized import Coded
    rng = random.Random(dim)
    for heads, kv_heads, longest in ((8, 4, 700), (32, 8, 300)):
        new, lens = [], []
        for i in range(160):
            n = rng.randint(1, 128 // (heads // kv_heads) // 2)
            new.append(n)
            lens.append(rng.randint(n, 128) if i % 5 else rng.randint(max(n, 129), longest))
        c = Coded(new, lens, heads=heads, kv_heads=kv_heads, dim=dim, form=form, seed=dim)
        c.tables = widen(c.tables, c.page)
        want = c.check(gorio)
        for _ in range(40):
            got = c.run(gorio)
            assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    gorio.attention_check()
