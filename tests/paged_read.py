"""Shapes of kv_paged_read that reach each form of its kernel: 8 KB a wavefront, or 2 KB where there
would be few wavefronts."""
import os
import re

from paper_2603_08739_amd import build as B

# name: block, head size, key/value heads, requests, most tokens of one, whether there are few wavefronts
SHAPES = {
    "16x64": (16, 64, 3, 400, 70, False),
    "16x128": (16, 128, 8, 200, 150, False),
    "32x64": (32, 64, 5, 300, 200, False),
    "64x128": (64, 128, 2, 110, 700, False),
    "128x256": (128, 256, 4, 30, 600, False),
    "256x256": (256, 256, 1, 40, 2000, False),
    "one request": (16, 128, 8, 1, 20000, False),
    "32x128, few": (32, 128, 2, 30, 200, True),
    "256x64, few": (256, 64, 2, 10, 600, True),
}


def few_wavefronts(n_req, rows, block, heads, dim, bytes_each):
    """Which form a call takes, by the rules of k_block.hip."""
    found = rows // block + 2 * n_req
    one = 1 if rows <= 1 else (rows - 1) // block + 2
    runs = one * n_req if one * n_req <= 2 * found else found
    each = -(-heads * block * dim * bytes_each // 8192)
    return 2 * runs * each < int(re.search(r"kFewTasks = (\d+);", open(os.path.join(B.CSRC, "k_block.hip")).read()).group(1))


def lengths(n_req, most, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(most // 2, most + 1, (n_req,), generator=g).tolist()
    if n_req > 4:
        lens[1], lens[n_req // 2], lens[-1] = 0, 1, 0
    return lens
