"""The block pool and the steps of the measured prefill cost at their limits, without a
GPU: what a request that does not fit leaves behind, and how large a step may be."""
import numpy as np
import pytest

import tracegen as tg


def test_a_request_that_does_not_fit_gives_nothing_away():
    from paper_2603_08739_amd.prefill_cost import BlockPool
    p = BlockPool(4)
    for h, block in enumerate(p.take(3, set())):
        p.keep(h, block)
    assert p.take(5, set()) is None and p.take(3, {1, 2}) is None
    assert list(p.held) == [0, 1, 2] and list(p.free) == [3]
    assert p.prefix([0, 1, 2]) == [0, 1, 2]
    assert p.take(2, {1, 2, 77}) == [3, 0] and list(p.held) == [1, 2] and not p.free    # what fits is still given


def test_prefixes_survive_a_request_that_is_too_long():
    """A request longer than the cache is skipped; the ones around it reuse what they
    would have without it."""
    from paper_2603_08739_amd.prefill_cost import batches

    def trace(requests):
        t = tg.from_blocks([b for r in requests for b in r])
        t.req = np.repeat(np.arange(len(requests)), [len(r) for r in requests]).astype(np.uint32)
        return t
    short, long = [list(range(8)), list(range(8)) + [20], list(range(8)) + [21]], list(range(100, 140))
    for batch in (1, 2, 3):
        with_it = [step for step in batches(trace(short[:1] + [long] + short[1:]), 20, batch)]
        lens = [(len(run), len(got)) for step in with_it for run, got in step]
        assert lens[0] == (0, 8) and lens[1] == (8, 1)
