"""The block pool behind the measured prefill cost, without a GPU: what a step
reuses, takes and gives away."""
import numpy as np
import pytest

import tracegen as tg


def test_pool_reuses_prefixes_and_gives_away_the_oldest():
    from paper_2603_08739_amd.prefill_cost import BlockPool
    p = BlockPool(4)
    assert p.prefix([1, 2]) == [] and p.take(2, set()) == [0, 1]
    p.keep(1, 0)
    p.keep(2, 1)
    assert p.take(2, set()) == [2, 3]
    p.keep(3, 2)
    p.keep(1, 3)               # held already: the block is free again
    assert p.prefix([1, 2, 9]) == [0, 1] and list(p.free) == [3]
    assert p.take(2, {1, 2}) == [3, 2] and list(p.held) == [1, 2]   # 3's block, the only unpinned one
    assert p.take(1, {1, 2}) is None and p.take(1, {2}) == [0]


@pytest.mark.parametrize("n_blocks, batch", [(64, 1), (200, 4), (100_000, 16)])
def test_steps_write_on_no_block_that_they_read(n_blocks, batch):
    from paper_2603_08739_amd.prefill_cost import batches, requests_of
    t = tg.tiny(n_req=120)
    sizes = [len(h) for h in requests_of(t)]
    assert sum(sizes) == t.n
    served = 0
    for step in batches(t, n_blocks, batch):
        assert 1 <= len(step) <= batch
        read = {b for run, _ in step for b in run}
        wrote = [b for _, got in step for b in got]
        assert len(set(wrote)) == len(wrote) and not read & set(wrote)
        assert all(0 <= b < n_blocks for b in list(read) + wrote) and all(got for _, got in step)
        served += len(step)
    assert served == sum(n <= n_blocks for n in sizes)


def test_unbounded_cache_recomputes_only_new_blocks():
    from paper_2603_08739_amd.prefill_cost import batches, requests_of
    t = tg.tiny(n_req=60)
    seen, want = set(), 0
    for hashes in requests_of(t):
        n = 0
        while n < len(hashes) - 1 and hashes[n] in seen:
            n += 1
        want += len(hashes) - n
        seen |= set(hashes)
    assert sum(len(got) for step in batches(t, 1_000_000, 1) for _, got in step) == want


def test_mixed_block_sizes_are_refused():
    from paper_2603_08739_amd import prefill_cost
    t = tg.random_trace(1, 100, 20, n_groups=1, weight_choices=(1, 4))
    assert len(np.unique(t.weight)) == 2
    with pytest.raises(ValueError):
        prefill_cost.measure(t, 10)
    with pytest.raises(ValueError):
        prefill_cost.seconds_per_token(dict(new_tokens=0), 1)
