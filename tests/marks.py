"""Values that show every key tile in the result: tile t (128 keys) has ones in dim t % d and zeros in the others, so that a
tile that is lost, read twice or taken from another row changes a dim by a good part of it, however long the row is."""

import torch


def marked(n, d, dtype, device, first=0, part=0, parts=1):
    """[n][d]; the first tile marks dim `first` % d. parts: of very long rows one d tiles in so many are marked, those of
    `part` (a tile is then a larger share of its dim)."""
    v = torch.zeros((n, d), dtype=dtype, device=device)
    if n:
        t = torch.arange(n, device=device) // 128
        v.scatter_(1, ((t + first) % d)[:, None], (t // d % parts == part).to(dtype)[:, None])
    return v
