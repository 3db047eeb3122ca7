"""Block tables, slots, positions and the free list against the oracle's walk, whole
numbers; data the device alone knows to be wrong; repeated calls and graphs."""
import random

import pytest

pytestmark = pytest.mark.gpu


def run(K, ctx, new, table, free, block, max_tokens, max_new=None, heads=(8, 2)):
    import torch
    i32 = dict(dtype=torch.int32, device="cuda")
    p = K.Plan(len(ctx), max_tokens, block, len(table[0]), heads[0], heads[1], 64, max_new=max_new)
    t = torch.tensor(table, **i32)
    args = (torch.tensor(ctx, **i32), torch.tensor(new, **i32), t, None if free is None else torch.tensor(free, **i32))
    K.kv_paged_plan(p, *args)
    got = [x.cpu().tolist() for x in (t, p.q_start, p.kv_len, p.slot, p.pos, p.result)]
    K.kv_paged_plan(p, *args)  # the same again
    assert got == [x.cpu().tolist() for x in (t, p.q_start, p.kv_len, p.slot, p.pos, p.result)]
    return got


@pytest.mark.parametrize("reqs, block, most_new, most_ctx", [(1, 16, 1, 0), (1, 16, 700, 40), (3, 64, 200, 300), (64, 16, 1, 900),
                                                             (257, 32, 9, 70), (1000, 16, 40, 200), (4096, 256, 3, 600)])
def test_against_the_walk(reqs, block, most_new, most_ctx):
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    rng = random.Random(reqs * block)
    ctx, new = [rng.randint(0, most_ctx) for _ in range(reqs)], [rng.randint(0, most_new) for _ in range(reqs)]
    new[-1] = most_new
    cols = -(-(most_ctx + most_new) // block)
    table = [[rng.randint(0, 999) if c * block < ctx[r] else -1 for c in range(cols)] for r in range(reqs)]
    free = rng.sample(range(1000, 200_000), sum(-(-(c + n) // block) - -(-c // block) for c, n in zip(ctx, new)) + 2)
    for max_tokens in (sum(new), sum(new) + 77):
        want = O.plan(ctx, new, table, free, block, max_tokens, cols, most_new)
        got = run(K, ctx, new, table, free, block, max_tokens, max_new=most_new)
        assert got == list(want) and got[5][3] == 0
    # without a free list the table's entries are taken as they stand
    filled = [[rng.randint(-1, 999) for _ in range(cols)] for _ in range(reqs)]
    assert run(K, ctx, new, filled, None, block, sum(new)) == list(O.plan(ctx, new, filled, None, block, sum(new), cols, sum(new)))


def test_wrong_lengths_are_flagged():
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    ctx, new = [5, -1, 10, 60, 3, 2 ** 31 - 1, 0], [3, 2, -4, 9, 8, 2 ** 31 - 1, 0]   # 1, 2, 3 (past the table), 4 (> max_new), 5
    table = [[i * 10 + j for j in range(4)] for i in range(7)]
    want = O.plan(ctx, new, table, [100], 16, 20, 4, 7)
    got = run(K, ctx, new, table, [100], 16, 20, max_new=7)
    assert got == list(want) and got[5] == [3, 0, 0, 1]


@pytest.mark.parametrize("max_tokens", [1, 9, 10, 24, 25, 26, 40])
def test_too_many_tokens(max_tokens):
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    ctx, new = [16, 0, 30, 5, 7], [9, 1, 15, 0, 6]
    table = [[3, -1, -1]] * 5
    free = list(range(50, 60))
    want = O.plan(ctx, new, table, free, 16, max_tokens, 3, max_tokens)
    got = run(K, ctx, new, table, free, 16, max_tokens)
    assert got == list(want)
    assert run(K, [0] * 300, [2] * 300, [[1]] * 300, None, 16, max_tokens) == list(
        O.plan([0] * 300, [2] * 300, [[1]] * 300, None, 16, max_tokens, 1, max_tokens))


@pytest.mark.parametrize("have", [0, 1, 5])
def test_too_few_blocks(have):
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    ctx, new, table = [0, 17, 4], [33, 20, 30], [[-1] * 4, [7, 8, -1, -1], [9, -1, -1, -1]]
    free = list(range(20, 20 + have))
    want = O.plan(ctx, new, table, free, 16, 90, 4, 90)
    got = run(K, ctx, new, table, free, 16, 90)
    assert got == list(want) and got[5] == [83, 6, have, 4]


def test_graph_replays_follow_the_lengths():
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    R, cols = 5, 6
    p = K.Plan(R, 40, 16, cols, 8, 2, 64)
    ctx, new = torch.zeros(R, **i32), torch.ones(R, **i32)
    table, free = torch.full((R, cols), -1, **i32), torch.arange(100, 130, **i32)
    K.kv_paged_plan(p, ctx, new, table, free)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        K.kv_paged_plan(p, ctx, new, table, free)
    for i in range(4):
        a, b = [7 * i, 3, 0, 16, 31 + i], [i, 1, 5 - i, 0, 2 * i + 1]
        rows = [[r * 7 + c for c in range(cols)] for r in range(R)]
        ctx.copy_(torch.tensor(a, **i32))
        new.copy_(torch.tensor(b, **i32))
        table.copy_(torch.tensor(rows, **i32))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = O.plan(a, b, rows, list(range(100, 130)), 16, 40, cols, 40)
        assert [x.cpu().tolist() for x in (table, p.q_start, p.kv_len, p.slot, p.pos, p.result)] == list(want)


def test_refusals():
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    p = K.Plan(3, 8, 16, 4, 8, 2, 64)
    good = [torch.zeros(3, **i32), torch.zeros(3, **i32), torch.zeros(3, 4, **i32), torch.zeros(2, **i32)]
    for i, bad in ((0, torch.zeros(2, **i32)), (1, torch.zeros(3, dtype=torch.int64, device="cuda")), (2, torch.zeros(3, 5, **i32)),
                   (2, torch.zeros(2, 4, **i32)), (2, torch.zeros(4, 3, **i32).t()), (3, torch.zeros(4, **i32)[::2]), (0, torch.zeros(3, dtype=torch.int32))):
        args = list(good)
        args[i] = bad
        with pytest.raises(ValueError):
            K.kv_paged_plan(p, *args)
    for bad in (dict(n_req=0), dict(block_size=24), dict(head_dim=80), dict(q_heads=9)):
        with pytest.raises(K.KvError):
            K.Plan(**{**dict(n_req=3, max_tokens=8, block_size=16, max_blocks=4, q_heads=8, kv_heads=2, head_dim=64), **bad})
