"""Attention over a cache of 8 bits with a scale for each block and head against its
definition in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

KINDS = [("bf16", "i8"), ("f16", "i8"), ("bf16", "fp8"), ("f16", "fp8")]


def case(ctx, new, block, heads, dim, dtype, kept, window=0, drop=(), max_new=None, pad=0, edit=None, edit_q=None, scale=None, spread=0, seed=0):
    """Runs one batch and checks it; drop: (request, column) entries set to -1; edit(kc, vc,
    ks, vs, table) and edit_q(q) change the inputs; values' scales are apart by up to 2^spread."""
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import ROUND, TYPES, blocks_of, check_attention, held_cache
    gen = torch.Generator().manual_seed(seed + 13 * sum(ctx) + sum(new))
    H, J = heads
    table, n_blocks = blocks_of(ctx, new, block, gen)
    for r, col in drop:
        table[r, col] = -1
    kc, vc, ks, vs = held_cache(n_blocks, J, block, dim, kept, gen)
    vs *= torch.exp2((torch.rand(n_blocks, J, generator=gen) - 1) * spread).cuda()
    if edit:
        edit(kc, vc, ks, vs, table)
    total = sum(new)
    T = total + pad
    q = (torch.randn(T, H, dim, generator=gen) * (1 + torch.rand(H, 1, generator=gen))).to(TYPES[dtype]).cuda()
    if edit_q:
        edit_q(q)
    p = K.Plan(len(ctx), T, block, table.shape[1], H, J, dim, max_new=max_new, window=window)
    i32 = dict(dtype=torch.int32, device="cuda")
    K.kv_paged_plan(p, torch.tensor(ctx, **i32), torch.tensor(new, **i32), table)
    assert p.result.tolist() == [total, 0, 0, 0]
    out, lse = torch.full((T, H, dim), 5.0, dtype=q.dtype, device="cuda"), torch.full((T, H), 5.0, device="cuda")
    cache = K.Cache(kc, vc, ks, vs, block_scales=True)
    K.kv_paged_attention(p, cache, q, out=out, lse=lse, scale=scale)
    assert bool((out[total:] == 5.0).all()) and bool((lse[total:] == 5.0).all())
    # (a block's scale that is not a number belongs to blocks that nothing sees)
    k64, v64 = (x.double() * torch.nan_to_num(s.double(), nan=0.0, posinf=0.0)[:, :, None, None] for x, s in ((kc, ks), (vc, vs)))
    want = list(O.attention(q[:total], k64, v64, table.tolist(), p.q_start.tolist(), ctx, block, n_blocks, dim ** -0.5 if scale is None else scale, window))
    # Beside the roundings that check_attention counts: a weight's scale is the exponential of a
    # logarithm of at most `spread` + 8 in 32 bits, which is off by 2^-24 of that (and its result by
    # 0.7 of it); and the exponent is rounded where its two parts meet, 2^-24 of their size (1.45 reach
    # + the logarithm).  Both together are less than 2^-22 (spread + 8 + reach) of the weight:
    # given to `reach` in units of its own bound, 2 (D + 8) 2^-24 reach.
    want[3] = want[3] + 4 * (spread + 8 + want[3]) / (2 * (dim + 8))
    # A weight, in float16 whatever the queries' type, that is below its normal numbers loses up to
    # 2^-25, with weights of 2^6 where 1 is meant: 2^-31 of the largest scale for every key and number
    # (one key's where the scales are near each other: such weights are small beside the largest).
    most = {"i8": 127.0, "fp8": 448.0}[kept]
    keys = max(c + n for c, n in zip(ctx, new)) if spread > 12 else 1
    want[2] = want[2] + 2.0 ** -31 / ROUND[q.dtype] * most * float(torch.nan_to_num(vs, nan=0.0, posinf=0.0).max()) * keys
    check_attention(out[:total], lse[:total], want, q)
    again = torch.empty_like(out)
    K.kv_paged_attention(p, cache, q, out=again, scale=scale)   # no lse, and bit for bit the same
    assert torch.equal(again[:total].view(torch.int16), out[:total].view(torch.int16))
    return out[:total], lse[:total]


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("block", [16, 64])
def test_single_tokens(dtype, kept, dim, block):
    """One new token a request, contexts around every edge."""
    ctx = [0, 1, 7, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 255, 256, 300]
    case(ctx, [1] * len(ctx), block, (8, 2), dim, dtype, kept, max_new=1)


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads", [(4, 4), (6, 1), (16, 2)])
def test_chunks(dtype, kept, dim, heads):
    """Chunks of prompts, idle requests and single tokens together: tiles of 128 rows."""
    case([0, 100, 17, 0, 63, 5], [33, 1, 0, 130, 64, 65], 16, heads, dim, dtype, kept, pad=3)


@pytest.mark.parametrize("heads, new", [((16, 1), 1), ((17, 1), 1), ((32, 1), 1), ((8, 2), 4), ((8, 2), 9), ((64, 1), 1), ((65, 1), 1),
                                        ((12, 4), 5), ((1, 1), 64), ((1, 1), 65), ((5, 5), 3)])
def test_few_rows(heads, new):
    """Every width of the kernel for few rows, and the step past the last."""
    for kept in ("i8", "fp8"):
        case([0, 70, 129, 3], [new, 1, max(1, new - 1), new], 32, heads, 64, "bf16", kept, max_new=new)
        case([200, 64], [new, new], 16, heads, 128, "f16", kept, max_new=new)


@pytest.mark.parametrize("block", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window", [1, 5, 64, 100])
def test_window(block, window):
    case([0, 300, 65, 1], [40, 37, 1, 3], block, (4, 2), 64, "f16", "i8", window=window)
    case([0, 300, 65, 1], [1, 1, 1, 1], block, (4, 2), 128, "bf16", "fp8", window=window, max_new=1)
    case([0, 300, 65, 1], [40, 37, 1, 3], block, (4, 2), 128, "bf16", "i8", window=window)


@pytest.mark.parametrize("max_new", [1, None])
@pytest.mark.parametrize("dtype, kept", KINDS)
def test_missing_blocks(max_new, dtype, kept):
    """Blocks that are gone, the block a context ends in among them, and rows that see
    nothing at all."""
    new = [1, 1, 1, 1] if max_new else [20, 1, 50, 16]
    ctx = [40, 70, 30, 0]
    drop = [(0, 0), (0, 2), (0, 3), (1, 1), (1, 4)] + [(2, c) for c in range(-(-(ctx[2] + new[2]) // 16))] + [(3, 0)]
    out, lse = case(ctx, new, 16, (4, 2), 64, dtype, kept, drop=[d for d in drop if d[1] * 16 < ctx[d[0]] + new[d[0]]], max_new=max_new)
    t = new[0] + new[1]
    assert bool((out[t:].float() == 0).all()) and bool((lse[t:] == -math.inf).all())
    case([100, 90], [1, 1] if max_new else [3, 40], 16, (4, 2), 64, dtype, kept, window=8, drop=[(0, 5), (0, 6)], max_new=max_new)


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("max_new", [1, 4, None])
@pytest.mark.parametrize("dim", [64, 128])
def test_blocks_of_zeros_and_scales_that_nobody_sees(dtype, kept, max_new, dim):
    """Scales of 0 (blocks that hold zeros); blocks outside every window and blocks of nobody
    with scales that are no numbers, or huge ones."""
    import torch
    new = [min(max_new, n) if max_new else n for n in (1, 4, 30, 70)]
    ctx = [137, 110, 200, 90]

    def zeros(kc, vc, ks, vs, table):
        t = table.tolist()
        for r, col in ((0, 0), (0, 2), (1, 1), (2, 5), (3, 0), (3, 1)):
            kc.view(torch.int8)[t[r][col], 0] = 0
            ks[t[r][col], 0] = 0
            vc.view(torch.int8)[t[r][col], 1] = 0
            vs[t[r][col], 1] = 0

    def unseen(kc, vc, ks, vs, table):
        zeros(kc, vc, ks, vs, table)
        t = table.tolist()
        seen = set()
        for r in range(4):
            seen |= {t[r][p // 16] for p in range(max(0, ctx[r] + 1 - 40), ctx[r] + new[r])}
        for page in set(range(kc.shape[0])) - seen:
            ks[page] = (float("nan"), float("inf"), 1e38)[page % 3]
            vs[page] = (1e38, float("nan"), float("inf"))[page % 3]

    case(ctx, new, 16, (4, 2), dim, dtype, kept, max_new=max_new, edit=zeros)
    case(ctx, new, 16, (4, 2), dim, dtype, kept, max_new=max_new, edit=unseen, window=40)

    def everything(kc, vc, ks, vs, table):
        kc.view(torch.int8).zero_()
        vc.view(torch.int8).zero_()
        ks.zero_()
        vs.zero_()

    out, _ = case(ctx, new, 16, (4, 2), dim, dtype, kept, max_new=max_new, edit=everything)
    assert not out.any()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("max_new", [1, 4, None])
def test_not_finite_in_masked_places(dtype, max_new):
    """e4m3 has NaN: where no query looks it changes nothing; where some do, it reaches those
    and no other."""
    import torch
    new = [min(max_new, n) if max_new else n for n in (1, 4, 30, 70)]
    ctx = [37, 10, 100, 0]

    def edit(kc, vc, ks, vs, table):
        bits, nan, t = (lambda x: x.view(torch.int8)), 0x7f, table.tolist()
        for r in range(4):
            for j in range(ctx[r] + new[r], len(t[r]) * 16):   # past the request's last token
                if t[r][j // 16] >= 0:
                    bits(kc)[t[r][j // 16], :, j % 16] = nan
                    bits(vc)[t[r][j // 16], :, :, j % 16] = nan
        for p in set(range(kc.shape[0])) - {p for row in t for p in row}:
            bits(kc)[p] = nan
            bits(vc)[p] = nan
        j = ctx[3] + new[3] - 1
        bits(vc)[t[3][j // 16], 0, 1, j % 16] = nan
        j = ctx[2] + new[2] // 2
        bits(vc)[t[2][j // 16], 1, 5, j % 16] = nan

    for dim in (64, 128):
        case(ctx, new, 16, (4, 2), dim, dtype, "fp8", max_new=max_new, edit=edit)
        case(ctx, new, 16, (4, 2), dim, dtype, "fp8", max_new=max_new, edit=edit, window=6)


@pytest.mark.parametrize("kept", ["i8", "fp8"])
@pytest.mark.parametrize("max_new", [1, None])
def test_not_finite_queries(kept, max_new):
    """A query that is not finite spoils its own rows only."""
    import torch

    def edit_q(q):
        q[0, 0, 3] = float("nan")
        q[1, 1] = float("inf")

    new = [1, 1] if max_new else [5, 20]
    out, lse = case([20, 60], new, 16, (4, 2), 128, "bf16", kept, max_new=max_new, edit_q=edit_q)
    assert bool(torch.isnan(lse[0, 0])) and not bool(torch.isnan(lse[0, 1:]).any())


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("spread", [10, 40, 100])
def test_scales_far_apart(dtype, kept, spread):
    """Values' scales from block to block apart by up to 2^spread: the unit of the sums rises as
    larger ones come."""
    case([300, 500, 700, 0], [1, 1, 1, 1], 16, (8, 2), 128, dtype, kept, max_new=1, spread=spread)
    case([300, 500, 0], [40, 140, 200], 16, (4, 2), 64, dtype, kept, spread=spread)
    case([300, 90], [100, 33], 32, (4, 2), 128, dtype, kept, spread=spread)


@pytest.mark.parametrize("dtype, kept", KINDS)
def test_large_and_small_scales(dtype, kept):
    """Scores and values near the ends of their ranges."""
    def small(kc, vc, ks, vs, table):
        ks *= 2.0 ** -100
        vs *= 2.0 ** -90

    def large(kc, vc, ks, vs, table):
        ks *= 2.0 ** 40
        vs *= 2.0 ** (8 if dtype == "f16" else 60)

    for new, max_new in (([1, 1], 1), ([40, 3], None)):
        if dtype == "bf16":
            case([100, 30], new, 16, (4, 2), 64, dtype, kept, max_new=max_new, edit=small)
        case([100, 30], new, 16, (4, 2), 64, dtype, kept, max_new=max_new, edit=large, scale=2.0 ** -43)
    case([100, 300], [40, 1], 16, (4, 2), 128, dtype, kept, scale=3.0)
    case([100, 300], [1, 1], 16, (4, 2), 128, dtype, kept, scale=3.0, max_new=1)


@pytest.mark.parametrize("dtype, kept", KINDS)
def test_cut_and_joined(dtype, kept):
    """Long contexts: pieces of a request's keys, each with a unit of its own, are joined."""
    case([3000, 1], [1, 1], 16, (8, 1), 128, dtype, kept, max_new=1, spread=8)
    case([3000], [40], 64, (4, 1), 64, dtype, kept, spread=8)
    case([2000, 900], [3, 150], 16, (4, 2), 128, dtype, kept, spread=8)


def test_another_stream():
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import held_cache
    gen = torch.Generator().manual_seed(9)
    i32 = dict(dtype=torch.int32, device="cuda")
    kc, vc, ks, vs = held_cache(9, 2, 16, 64, "i8", gen)
    cache = K.Cache(kc, vc, ks, vs, block_scales=True)
    p = K.Plan(1, 20, 16, 8, 4, 2, 64)
    table = torch.arange(8, **i32)[None].contiguous()
    q = torch.randn(20, 4, 64, generator=gen).cuda().half()
    K.kv_paged_plan(p, torch.tensor([100], **i32), torch.tensor([20], **i32), table)
    want, rows = K.kv_paged_attention(p, cache, q), K.kv_paged_read(p, cache, torch.tensor([0, 120], **i32), rows=120)
    start = torch.tensor([0, 120], **i32)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        out = K.kv_paged_attention(p, cache, q, stream=stream)
        k, v = K.kv_paged_read(p, cache, start, rows=120, stream=stream)
        s.synchronize()
        assert torch.equal(out, want) and torch.equal(k, rows[0]) and torch.equal(v, rows[1])
