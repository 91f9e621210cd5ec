"""Tables that could hold very long caches: with them the chunk kernel takes every call of more than 16 rows a key head, where it would
leave those over short caches to the single-token kernel."""
import torch


def widen(tables, page, places=1 << 22):
    """The same rows, with room for `places` tokens; entries past a request's own pages belong to other rows."""
    b, w = tables.shape
    flat = torch.full((b * w + places // page,), -1, dtype=torch.int32, device=tables.device)
    flat[: b * w] = tables.reshape(-1)
    return flat.as_strided((b, places // page), (w, 1))
