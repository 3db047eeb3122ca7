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


def documents(lengths, tokens=64):
    """A trace of one request for each length (in blocks), no block shared."""
    t = tg.from_blocks(np.arange(sum(lengths)))
    t.req = np.repeat(np.arange(len(lengths)), lengths).astype(np.uint32)
    t.tokens_per_granule = tokens
    return t


def test_a_step_brings_no_more_tokens_than_the_plan_takes():
    """Document-sized requests: a batch ends before its new tokens pass what a step may
    bring; a request that passes it alone is skipped."""
    from paper_2603_08739_amd.kvpaged import KV_PAGED_MAX_TOKENS
    from paper_2603_08739_amd.prefill_cost import batches
    lengths = [2047] * 9 + [8192, 8193, 2000, 2000, 2000, 2192, 1]
    t = documents(lengths)
    steps = [[len(got) for _, got in step] for step in batches(t, 100_000, 16)]
    assert all(64 * sum(s) <= KV_PAGED_MAX_TOKENS for s in steps)
    assert steps == [[2047] * 4, [2047] * 4, [2047], [8192], [2000, 2000, 2000, 2192], [1]]


def test_long_documents_of_the_workloads_fit():
    from paper_2603_08739_amd.kvpaged import KV_PAGED_MAX_TOKENS
    from paper_2603_08739_amd.prefill_cost import batches
    t = tg.longctx(n_req=300, n_docs=40)
    served = 0
    for step in batches(t, 40_000, 16):
        assert sum(len(got) for _, got in step) * t.tokens_per_granule <= KV_PAGED_MAX_TOKENS
        served += len(step)
    assert served == 300


def test_steps_of_weighted_blocks():
    """Blocks of four granules hold four times the tokens."""
    from paper_2603_08739_amd.prefill_cost import batches
    t = documents([5000, 3000, 3000], tokens=16)
    t.weight[:] = 4
    assert [[len(got) for _, got in s] for s in batches(t, 100_000, 16)] == [[5000, 3000], [3000]]
