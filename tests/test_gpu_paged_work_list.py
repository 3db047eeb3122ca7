"""The plan's work list itself, read back from the work memory: every tile's keys covered
once, partial results and cut tiles numbered without gaps or collisions, the longest
pieces first.  Sizes reach every rule by which pieces are made; where these change the
arithmetic, attention over such a list is compared with matrix products in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

UNIT = 64  # keys


def up(x):
    return -(-x // 256) * 256


def layout(b):
    """Sizes and places in the work memory, by the rules of its header."""
    group = b.q_heads // b.kv_heads
    most = (min(b.max_new, b.max_tokens) if b.max_new else b.max_tokens) * group
    few = 16 if most <= 16 else 32 if most <= 32 else 64
    rows = few if most <= 64 and few * b.head_dim <= 4096 else 128
    busy = min(b.n_req, b.max_tokens)
    tiles = busy if rows < 128 else b.max_tokens * group // 128 + busy
    per_head = lambda n: -(-n // b.kv_heads)  # noqa: E731
    pieces = per_head(1024 if rows < 128 or b.head_dim == 64 else 512)
    items = 256
    split = up(items + 48 * (tiles + pieces))
    return dict(group=group, rows=rows, pieces=pieces, few_pieces=pieces if rows < 128 else per_head(512), max_items=tiles + pieces,
                max_parts=2 * pieces, max_split=pieces, items=items, split=split, done=up(split + 32 * pieces))


def check_list(plan, ctx, new, reach=None):
    """Checks the list against the lengths; `reach`: what the case is there for."""
    import numpy as np
    b, w = plan.batch, layout(plan.batch)
    raw = plan.work.cpu().numpy()
    ints = lambda at, n: raw[at:at + 4 * n].view(np.int32)  # noqa: E731
    n_items, n_split = ints(0, 2).tolist()
    start = np.concatenate([[0], np.cumsum(new)])
    tiles, units = {}, 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        for row0 in range(0, n * w["group"], w["rows"]):
            t0, t1 = row0 // w["group"], (min(row0 + w["rows"], n * w["group"]) - 1) // w["group"]
            begin = max(0, c + t0 + 1 - b.window) // UNIT * UNIT if b.window else 0
            tiles[r, row0] = (begin, c + t1 + 1)
            units += -(-(c + t1 + 1 - begin) // UNIT)
    assert n_items <= w["max_items"] and n_split <= w["max_split"]
    items = ints(w["items"], 12 * n_items).reshape(n_items, 12).tolist()
    cut = ints(w["split"], 8 * n_split).reshape(n_split, 8).tolist()
    of = {}
    for it in items:
        of.setdefault((it[0], it[4]), []).append(it)
    assert set(of) == set(tiles)
    parts, splits = set(), set()
    for (r, row0), pieces in of.items():
        pieces.sort(key=lambda it: it[5])
        at, end = tiles[r, row0]
        for i, (req, q_start, c, row_end, _, begin, stop, part, split, first, n, _) in enumerate(pieces):
            assert (q_start, c, row_end) == (start[r], ctx[r], new[r] * w["group"])
            assert begin == at and begin % UNIT == 0 and stop > begin and (stop % UNIT == 0 or stop == end)
            at = stop
            assert n == len(pieces) <= 32
            if n == 1:
                assert part == -1
            else:  # joined in this order
                assert part == first + i and 0 <= part < w["max_parts"] and part not in parts
                parts.add(part)
                assert cut[split][:5] == [q_start, row_end, row0, first, n]
        assert at == end
        if len(pieces) > 1:
            assert pieces[0][8] not in splits and all(it[8] == pieces[0][8] for it in pieces)
            splits.add(pieces[0][8])
            lengths = [-(-(it[6] - it[5]) // UNIT) for it in pieces]
            assert max(lengths) - min(lengths) <= 1
    assert splits == set(range(n_split)) and parts == set(range(len(parts)))
    assert not ints(w["done"], n_split * b.kv_heads).any()
    # the rules: how long a piece may be, and classes of length in order
    least = 2 if w["rows"] < 128 and units * b.kv_heads <= 256 else 4
    longest = -(-units // w["few_pieces"])
    long = longest >= 64
    longest = max(least, -(-units // w["pieces"]) if long else longest)
    most = max([-(-(e - a) // UNIT) for a, e in tiles.values()], default=0)
    for key, pieces in of.items():
        u = -(-(tiles[key][1] - tiles[key][0]) // UNIT)
        assert len(pieces) == min(-(-u // longest), 32)
    shift = 0
    while max(longest, most // 32 + 1) >> shift >= 64:
        shift += 1
    classes = [min(-(-(it[6] - it[5]) // UNIT) >> shift, 63) for it in items]
    assert classes == sorted(classes, reverse=True)
    if reach:
        facts = dict(long=long, shift=shift, tiles=len(tiles), longest=longest, cut=n_split, rows=w["rows"], capped=max((len(p) for p in of.values()), default=0) == 32)
        assert reach(facts), facts


def planned(ctx, new, block, heads, dim, max_new=None, window=0, pad=0):
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    columns = max(1, max(-(-(c + n) // block) for c, n in zip(ctx, new)))
    plan = K.Plan(len(ctx), max(1, sum(new) + pad), block, columns, heads[0], heads[1], dim, max_new=max_new, window=window)
    plan.work.fill_(0x5a)
    K.kv_paged_plan(plan, torch.tensor(ctx, **i32), torch.tensor(new, **i32), torch.zeros(len(ctx), columns, **i32))
    assert plan.result.tolist() == [sum(new), 0, 0, 0]
    return plan


def ragged(n, most_ctx, most_new, seed, idle=0):
    import random
    rng = random.Random(seed)
    return ([rng.randint(0, most_ctx) for _ in range(n)],
            [0 if idle and rng.random() < idle else rng.randint(1, most_new) for _ in range(n)])


LISTS = {
    "a short context": (([500], [1], 16, (32, 8), 128), dict(max_new=1), lambda f: f["longest"] == 2 and f["cut"] == 1),
    "contexts of 1,000": (([1000] * 16, [1] * 16, 16, (32, 8), 128), dict(max_new=1), lambda f: f["longest"] == 4),
    "chats": ((*ragged(64, 16000, 1, 1), 16, (32, 8), 128), dict(max_new=1), lambda f: f["longest"] > 4 and f["cut"] > 10),
    "a long document, pieces by total": (([131071], [1], 64, (8, 8), 128), dict(max_new=1), lambda f: f["capped"] and f["shift"] == 1),
    "a long document, one head": (([131071], [1], 64, (8, 1), 128), dict(max_new=1), lambda f: f["capped"] and f["shift"] == 1),
    "long documents": (([131000, 90000, 8192, 5], [1] * 4, 64, (64, 8), 128), dict(max_new=1), lambda f: f["capped"]),
    "chunk over a long context, heads of 64": (([60000], [300], 64, (24, 4), 64), {}, lambda f: f["long"] and f["rows"] == 128),
    "the same, heads of 128": (([60000], [300], 64, (24, 4), 128), {}, lambda f: f["long"]),
    "one head, heads of 64": (([100000, 3], [40, 40], 64, (1, 1), 64), {}, lambda f: f["capped"] and f["cut"] > 0),
    "chunks of 512": (([4096] * 4, [512] * 4, 16, (32, 8), 64), {}, lambda f: f["long"] and f["cut"] == 64),
    "shorter chunks": (([1500] * 4, [512] * 4, 16, (32, 8), 64), {}, lambda f: 4 < f["longest"] and not f["long"] and f["cut"] > 0),
    "a prompt": (([256], [8111], 16, (32, 8), 128), {}, lambda f: f["longest"] > 4),
    "a prompt, heads of 256": (([0], [1500], 16, (8, 2), 256), {}, lambda f: f["rows"] == 128),
    "thousands of requests": ((*ragged(3000, 2000, 3, 2, idle=0.1), 16, (8, 2), 64), {}, lambda f: f["tiles"] > 2048 and f["rows"] == 128),
    "thousands of requests of single tokens": ((*ragged(4096, 700, 1, 3), 16, (8, 2), 64), dict(max_new=1), lambda f: f["tiles"] == 4096),
    "thousands of long ones": ((*ragged(2500, 9000, 2, 4), 16, (16, 2), 128), {}, lambda f: f["tiles"] > 2048 and f["shift"] == 4),
    "thousands and a long one": (([20] * 2400 + [100000], [1] * 2400 + [30], 16, (16, 2), 128), {}, lambda f: f["tiles"] > 2048 and f["cut"] > 0),
    "a window": ((*ragged(12, 12000, 1300, 5, idle=0.2), 16, (24, 4), 64), dict(window=4096, pad=7), lambda f: f["cut"] > 0),
    "a short window": ((*ragged(12, 12000, 1300, 6), 16, (32, 4), 128), dict(window=272), lambda f: f["cut"] == 0 and f["tiles"] > 512),
    "a window of one": (([1000, 63, 64], [200, 1, 70], 16, (4, 4), 256), dict(window=1), lambda f: f["cut"] == 0),
    "65 heads to one": ((*ragged(20, 3000, 9, 7), 32, (65, 1), 64), {}, lambda f: f["rows"] == 128),
    "nothing new": (([5, 0, 900], [0, 0, 0], 16, (8, 2), 64), {}, lambda f: f["tiles"] == 0 and f["cut"] == 0),
}


@pytest.mark.parametrize("name", LISTS)
def test_every_tile_is_covered_once(name):
    args, more, reach = LISTS[name]
    plan = planned(*args, **more)
    check_list(plan, args[0], args[1], reach)


def test_a_plan_filled_again():
    """Other lengths in the same work memory, longer and shorter lists in turn."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    plan = K.Plan(6, 900, 16, 800, 16, 2, 128)
    for seed in range(6):
        ctx, new = ragged(6, 11000, 150 if seed % 2 else 3, seed, idle=0.3)
        K.kv_paged_plan(plan, torch.tensor(ctx, **i32), torch.tensor(new, **i32), torch.zeros(6, 800, **i32))
        check_list(plan, ctx, new)


def by_products(q, kc, vc, table, ctx, new, scale, window, ks, vs):
    """The oracle's (out, lse, spread, reach) with matrix products, one head at a time."""
    import torch
    H, J, D = q.shape[1], kc.shape[1], q.shape[2]
    f64 = dict(dtype=torch.float64, device="cuda")
    out, spread = torch.zeros(q.shape, **f64), torch.zeros(q.shape, **f64)
    lse, reach = torch.zeros(q.shape[:2], **f64), torch.zeros(q.shape[:2], **f64)
    at = 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        pages = table[r, :-(-(c + n) // kc.shape[2])].long()
        key, own = torch.arange(c + n, device="cuda"), torch.arange(c, c + n, device="cuda")[:, None]
        hidden = (key > own) | (key <= own - window) if window else key > own
        for j in range(J):
            k = kc[pages, j].double().reshape(-1, D)[:c + n]
            v = vc[pages, j].double().transpose(1, 2).reshape(-1, D)[:c + n].contiguous()
            if ks is not None:
                k, v = k * ks[j].double(), v * vs[j].double()
            kt = k.T.contiguous()
            for h in range(j * H // J, (j + 1) * H // J):
                x = q[at:at + n, h].double()
                s = (x @ kt * scale).masked_fill(hidden, -math.inf)
                w = torch.softmax(s, -1)
                out[at:at + n, h], lse[at:at + n, h], spread[at:at + n, h] = w @ v, torch.logsumexp(s, -1), w @ v.abs()
                reach[at:at + n, h] = (x.abs() @ kt.abs() * scale).masked_fill(hidden, 0.0).amax(-1)
        at += n
    return out, lse, spread, reach


@pytest.mark.parametrize("ctx, new, block, heads, dim, dtype, kept, more", [
    ([60000], [300], 64, (6, 1), 64, "f16", "f16", {}),                       # twice the pieces: heads of 64, long pieces
    ([50000, 9], [150, 33], 64, (8, 2), 64, "bf16", "fp8", {}),
    ([131071], [1], 64, (8, 8), 128, "bf16", "bf16", dict(max_new=1)),        # classes of two lengths
    ([131071, 70001], [1, 1], 64, (8, 2), 128, "bf16", "fp8", dict(max_new=1)),
    ([40000], [100], 64, (4, 1), 128, "bf16", "bf16", {}),
    ([30000, 64], [64, 200], 16, (8, 1), 256, "bf16", "bf16", {}),
    ([20000, 500], [700, 90], 16, (4, 2), 128, "bf16", "bf16", dict(window=9000))])
def test_attention_over_long_lists(ctx, new, block, heads, dim, dtype, kept, more):
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import TYPES, blocks_of, check_attention
    i32 = dict(dtype=torch.int32, device="cuda")
    table, n_blocks = blocks_of(ctx, new, block, torch.Generator().manual_seed(sum(ctx)))
    g = torch.Generator(device="cuda").manual_seed(sum(new))
    H, J = heads
    k, v = torch.randn(n_blocks, J, block, dim, device="cuda", generator=g), torch.randn(n_blocks, J, dim, block, device="cuda", generator=g)
    ks = vs = None
    if kept == "fp8":
        ks, vs = torch.rand(J, device="cuda", generator=g) * 0.02 + 0.02, torch.rand(J, device="cuda", generator=g) * 0.02 + 0.02
        k, v = (k / ks[:, None, None]).clamp(-448, 448), (v / vs[:, None, None]).clamp(-448, 448)
    k, v = k.to(TYPES[kept]), v.to(TYPES[kept])
    q = (torch.randn(sum(new), H, dim, device="cuda", generator=g) * 1.5).to(TYPES[dtype])
    plan = K.Plan(len(ctx), sum(new), block, table.shape[1], H, J, dim, **more)
    K.kv_paged_plan(plan, torch.tensor(ctx, **i32), torch.tensor(new, **i32), table)
    check_list(plan, ctx, new)
    lse = torch.empty(sum(new), H, device="cuda")
    out = K.kv_paged_attention(plan, K.Cache(k, v, ks, vs), q, lse=lse)
    check_attention(out, lse, by_products(q, k, v, table, ctx, new, dim ** -0.5, plan.batch.window, ks, vs), q)


def test_attention_of_thousands_of_requests():
    """More tiles than the plan's threads keep: both kernels."""
    from tests.test_gpu_paged_attention import case
    ctx, new = ragged(2300, 60, 2, 8, idle=0.05)
    case(ctx, new, 16, (4, 2), 64, "bf16", "bf16")
    case(ctx, new, 16, (4, 2), 64, "bf16", "bf16", max_new=2)
