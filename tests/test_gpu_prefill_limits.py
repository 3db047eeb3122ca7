"""The measured prefill cost on the card at its limits: document-sized requests, and many
steps in the memory of a few."""
import numpy as np
import pytest

import tracegen as tg

pytestmark = pytest.mark.gpu


def test_document_sized_requests_are_served():
    from paper_2603_08739_amd import prefill_cost as P
    n, blocks = 12, 1000
    t = tg.from_blocks(np.arange(n * blocks))
    t.req, t.tokens_per_granule = np.repeat(np.arange(n), blocks).astype(np.uint32), 64
    done = P.measure(t, 20_000, batch=16, q_heads=2, kv_heads=1, head_dim=64)
    assert done["steps"] == 2 and done["requests"] == n and done["new_tokens"] == 64 * n * blocks


def test_memory_does_not_grow_with_the_steps():
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from paper_2603_08739_amd import prefill_cost as P
    work = K.Plan(1, 512, 16, 64, 32, 8, 128, max_new=512).work.numel()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    done = P.measure(tg.tiny(n_req=80), 2000, batch=1)
    assert done["steps"] == 80
    cache = 2 * 2000 * 8 * 16 * 128 * 2
    # at most two plans at a time, and as much again for a step's heads
    assert torch.cuda.max_memory_allocated() - before < cache + 4 * work < 80 * work
