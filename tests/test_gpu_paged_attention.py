"""Attention over a paged cache against its definition in 64 bits: row tiles and
their edges, head groups, types, windows, missing blocks, values that are not finite
in masked places, cut and joined keys, strides, far offsets, streams and graphs."""
import math

import pytest

pytestmark = pytest.mark.gpu


def case(ctx, new, block, heads, dim, dtype, kept, window=0, drop=(), max_new=None, pad=0, spare=3, edit=None, edit_q=None, scale=None, seed=0):
    """Runs one batch and checks it; drop: (request, column) entries set to -1; edit(kc,
    vc, table) and edit_q(q) change the inputs before the call."""
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import TYPES, blocks_of, cache_values, check_attention
    gen = torch.Generator().manual_seed(seed + 13 * sum(ctx) + sum(new))
    H, J = heads
    table, n_blocks = blocks_of(ctx, new, block, gen, spare=spare)
    for r, col in drop:
        table[r, col] = -1
    kc, vc, ks, vs = cache_values(n_blocks, J, block, dim, kept, gen)
    if edit:
        edit(kc, vc, table)
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
    cache = K.Cache(kc, vc, ks, vs)
    K.kv_paged_attention(p, cache, q, out=out, lse=lse, scale=scale)
    assert bool((out[total:] == 5.0).all()) and bool((lse[total:] == 5.0).all())
    want = O.attention(q[:total], kc, vc, table.tolist(), p.q_start.tolist(), ctx, block, n_blocks,
                       dim ** -0.5 if scale is None else scale, window, ks, vs)
    check_attention(out[:total], lse[:total], want, q)
    again = torch.empty_like(out)
    K.kv_paged_attention(p, cache, q, out=again, scale=scale)   # no lse, and bit for bit the same
    assert torch.equal(again[:total].view(torch.int16), out[:total].view(torch.int16))
    return out[:total], lse[:total]


KINDS = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "fp8"), ("f16", "fp8")]


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


@pytest.mark.parametrize("heads, new", [((16, 1), 1), ((17, 1), 1), ((32, 1), 1), ((8, 2), 4), ((8, 2), 8), ((8, 2), 9), ((64, 1), 1), ((65, 1), 1),
                                        ((12, 4), 5), ((1, 1), 16), ((1, 1), 64), ((1, 1), 65), ((5, 5), 3)])
def test_few_rows(heads, new):
    """Every width of the kernel for few rows, and the step past the last."""
    for kept in ("bf16", "fp8"):
        case([0, 70, 129, 3], [new, 1, max(1, new - 1), new], 32, heads, 64, "bf16", kept, max_new=new)
        case([200, 64], [new, new], 16, heads, 128, "bf16", kept, max_new=new)


@pytest.mark.parametrize("block", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window", [1, 5, 64, 100])
def test_window(block, window):
    case([0, 300, 65, 1], [40, 37, 1, 3], block, (4, 2), 64, "f16", "f16", window=window)
    case([0, 300, 65, 1], [1, 1, 1, 1], block, (4, 2), 128, "bf16", "fp8", window=window, max_new=1)


@pytest.mark.parametrize("max_new", [1, None])
def test_missing_blocks(max_new):
    """Blocks that are gone, the block a context ends in among them, and rows that see
    nothing at all."""
    new = [1, 1, 1, 1] if max_new else [20, 1, 50, 16]
    ctx = [40, 70, 30, 0]
    drop = [(0, 0), (0, 2), (0, 3), (1, 1), (1, 4)] + [(2, c) for c in range(-(-(ctx[2] + new[2]) // 16))] + [(3, 0)]
    for kept in ("bf16", "fp8"):
        out, lse = case(ctx, new, 16, (4, 2), 64, "bf16", kept, drop=[d for d in drop if d[1] * 16 < ctx[d[0]] + new[d[0]]], max_new=max_new)
        t = new[0] + new[1]
        assert bool((out[t:].float() == 0).all()) and bool((lse[t:] == -math.inf).all())
    # a window that holds only missing blocks
    case([100, 90], [1, 1] if max_new else [3, 40], 16, (4, 2), 64, "f16", "f16", window=8, drop=[(0, 5), (0, 6)], max_new=max_new)


@pytest.mark.parametrize("kept", ["f16", "bf16", "fp8"])
@pytest.mark.parametrize("max_new", [1, 4, None])
def test_not_finite_in_masked_places(kept, max_new):
    """NaN and infinities where no query looks change nothing; where some queries look,
    they reach those and no other."""
    import torch
    new = [min(max_new, n) if max_new else n for n in (1, 4, 30, 70)]
    ctx = [37, 10, 100, 0]

    def edit(kc, vc, table):
        bits = (lambda x: x.view(torch.int8)) if kept == "fp8" else (lambda x: x)
        nan, inf = (0x7f, 0x7f) if kept == "fp8" else (float("nan"), float("inf"))
        t = table.tolist()
        for r in range(4):
            end = ctx[r] + new[r]
            for j in range(end, len(t[r]) * 16):   # past the request's last token
                if t[r][j // 16] >= 0:
                    bits(kc)[t[r][j // 16], :, j % 16] = nan
                    bits(vc)[t[r][j // 16], :, :, j % 16] = nan
                    bits(vc)[t[r][j // 16], :, 3, j % 16] = inf
        spare = set(range(kc.shape[0])) - {p for row in t for p in row}
        for p in spare:
            bits(kc)[p] = nan
            bits(vc)[p] = nan
        # values of tokens that only the later queries of the chunk see
        j = ctx[3] + new[3] - 1
        bits(vc)[t[3][j // 16], 0, 1, j % 16] = nan
        j = ctx[2] + new[2] // 2
        bits(vc)[t[2][j // 16], 1, 5, j % 16] = -inf if kept != "fp8" else nan
        if new[2] // 2 + 1 < new[2]:
            bits(vc)[t[2][(j + 1) // 16], 1, 5, (j + 1) % 16] = inf
            bits(vc)[t[2][(j + 1) // 16], 1, 9, (j + 1) % 16] = inf

    dtype = "f16" if kept == "f16" else "bf16"
    for dim in (64, 128):
        case(ctx, new, 16, (4, 2), dim, dtype, kept, max_new=max_new, edit=edit)
        case(ctx, new, 16, (4, 2), dim, dtype, kept, max_new=max_new, edit=edit, window=6)


def test_large_scores():
    """Scores far apart: weights that vanish, one that takes all, and a scale that is not
    the default."""
    def edit(kc, vc, table):
        kc.mul_(40)
    case([200, 0, 64], [1, 1, 1], 16, (8, 2), 128, "bf16", "bf16", edit=edit, max_new=1)
    case([200, 0, 64], [70, 3, 20], 16, (8, 2), 128, "bf16", "bf16", edit=edit)
    case([200, 0, 64], [70, 3, 20], 16, (8, 2), 64, "f16", "f16", scale=0.01)


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("step", [0.02, 0.3, 4.0])
def test_rising_scores(dtype, kept, dim, step):
    """Every key's score is above that of the one before it, by little or by so much
    that weights taken from an earlier maximum would overflow."""
    import torch

    def edit(kc, vc, table):
        k = torch.zeros(kc.shape, device="cuda")
        for row in table.tolist():
            for i, page in enumerate(row):
                if page >= 0:  # element 0 carries the score: q[0] is 8 below
                    k[page, :, :, 0] = (step * torch.arange(16 * i, 16 * i + 16, device="cuda")).clamp(max=440.0)
        kc.copy_(k.to(kc.dtype))

    def queries(q):
        q.mul_(0.25)[..., 0] = 8.0

    case([150, 0, 3], [90, 200, 1], 16, (4, 2), dim, dtype, kept, edit=edit, edit_q=queries, scale=0.25)
    case([150, 0, 300], [1, 1, 1], 16, (4, 2), dim, dtype, kept, edit=edit, edit_q=queries, scale=0.25, max_new=1)


@pytest.mark.parametrize("ctx, new, heads, dim, kept, max_new", [
    ([9000], [1], (4, 1), 64, "bf16", 1),
    ([5001, 1, 700, 12345], [1, 1, 1, 1], (8, 2), 128, "fp8", 1),
    ([4100, 80], [3, 2], (8, 1), 256, "bf16", 3),
    ([3000, 900], [33, 40], (2, 1), 64, "bf16", None),
    ([2500], [17], (8, 1), 128, "fp8", None)])
def test_cut_keys(ctx, new, heads, dim, kept, max_new):
    """Long contexts with few rows: the keys are cut into pieces and joined."""
    case(ctx, new, 64, heads, dim, "bf16", kept, max_new=max_new)
    case(ctx, new, 16, heads, dim, "bf16", kept, max_new=max_new, window=1500)


def test_many_requests():
    import random
    rng = random.Random(4)
    ctx, new = [rng.randint(0, 90) for _ in range(300)], [rng.choice([0, 1, 1, 2]) for _ in range(300)]
    case(ctx, new, 16, (4, 2), 64, "bf16", "bf16", max_new=2)
    case(ctx, new, 16, (4, 2), 64, "bf16", "bf16")


def test_long_chunk_against_products():
    """A chunk of some thousand tokens, checked in 64 bits with matrix products."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import blocks_of, check_attention
    i32 = dict(dtype=torch.int32, device="cuda")
    for (H, J), dim, c, n, dtype in (((4, 1), 128, 77, 2100, torch.bfloat16), ((2, 2), 64, 500, 1333, torch.float16), ((2, 1), 256, 0, 700, torch.bfloat16)):
        gen = torch.Generator().manual_seed(n)
        table, nb = blocks_of([c], [n], 16, gen)
        kc, vc = torch.randn(nb, J, 16, dim, generator=gen).to(dtype).cuda(), torch.randn(nb, J, dim, 16, generator=gen).to(dtype).cuda()
        q = torch.randn(n, H, dim, generator=gen).to(dtype).cuda()
        p = K.Plan(1, n, 16, table.shape[1], H, J, dim)
        K.kv_paged_plan(p, torch.tensor([c], **i32), torch.tensor([n], **i32), table)
        out, lse = torch.empty_like(q), torch.empty(n, H, device="cuda")
        K.kv_paged_attention(p, K.Cache(kc, vc), q, out=out, lse=lse)
        pages = table[0].long()
        hidden = torch.arange(c + n, device="cuda") > torch.arange(c, c + n, device="cuda")[:, None]
        want = [torch.zeros(n, H, dim, dtype=torch.float64, device="cuda"), torch.zeros(n, H, dtype=torch.float64, device="cuda"),
                torch.zeros(n, H, dim, dtype=torch.float64, device="cuda"), torch.zeros(n, H, dtype=torch.float64, device="cuda")]
        for h in range(H):
            j = h // (H // J)
            k = kc[pages, j].double().reshape(-1, dim)[:c + n]
            v = vc[pages, j].double().transpose(1, 2).reshape(-1, dim)[:c + n]
            kt = k.T.contiguous()
            s = (q[:, h].double() @ kt * dim ** -0.5).masked_fill(hidden, -math.inf)
            w = torch.softmax(s, -1)
            want[0][:, h], want[1][:, h], want[2][:, h] = w @ v, torch.logsumexp(s, -1), w @ v.abs()
            want[3][:, h] = (q[:, h].double().abs() @ kt.abs() * dim ** -0.5).masked_fill(hidden, 0.0).amax(-1)
        check_attention(out, lse, want, q)


def test_strides_and_far_offsets():
    """Queries inside a fused projection, outputs with heads outermost, K and V of a block
    side by side in a cache whose offsets pass 32 bits."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    g = torch.Generator(device="cuda").manual_seed(5)
    i32 = dict(dtype=torch.int32, device="cuda")
    n_blocks, J, block, dim, H = 90_000, 8, 16, 128, 16
    both = torch.zeros(n_blocks, 2, J * block * dim, device="cuda", dtype=torch.bfloat16)
    for new, max_new in ((1, 1), (90, None)):
        ctx = 200
        cols = -(-(ctx + new) // block)
        pages = torch.randint(60_000, n_blocks, (cols,), device="cuda", generator=g).unique()[:cols]
        pages = torch.cat([pages, torch.arange(cols - len(pages), device="cuda")]).flip(0)
        both[pages] = torch.randn(cols, 2, J * block * dim, device="cuda", generator=g).bfloat16()
        kc, vc = both[:, 0].view(n_blocks, J, block, dim), both[:, 1].view(n_blocks, J, dim, block)
        fused = torch.randn(new, H + 2 * J, dim, device="cuda", generator=g).bfloat16()
        out = torch.empty(H, new, dim, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
        p = K.Plan(1, new, block, cols, H, J, dim, max_new=max_new)
        lens = torch.tensor([ctx], **i32), torch.tensor([new], **i32)
        K.kv_paged_plan(p, *lens, pages.to(torch.int32)[None].contiguous())
        K.kv_paged_attention(p, K.Cache(kc, vc), fused[:, :H], out=out)
        # the same blocks in a small cache of their own
        near = K.Plan(1, new, block, cols, H, J, dim, max_new=max_new)
        K.kv_paged_plan(near, *lens, torch.arange(cols, **i32)[None].contiguous())
        want = K.kv_paged_attention(near, K.Cache(kc[pages].contiguous(), vc[pages].contiguous()), fused[:, :H].contiguous())
        assert torch.equal(out, want)


def test_other_streams_and_graph():
    import torch
    from paper_2603_08739_amd import kvpaged as K
    g = torch.Generator(device="cuda").manual_seed(6)
    i32 = dict(dtype=torch.int32, device="cuda")
    kc, vc = torch.randn(80, 2, 16, 64, device="cuda", generator=g).half(), torch.randn(80, 2, 64, 16, device="cuda", generator=g).half()
    cache = K.Cache(kc, vc)
    table = torch.randperm(80, device="cuda", generator=g).to(torch.int32).view(2, 40).contiguous()
    ctx, new = torch.tensor([600, 30], **i32), torch.tensor([1, 1], **i32)
    q = torch.randn(2, 8, 64, device="cuda", generator=g).half()
    p = K.Plan(2, 2, 16, 40, 8, 2, 64, max_new=1)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    K.kv_paged_plan(p, ctx, new, table, stream=side)
    K.kv_paged_attention(p, cache, q, out=out, stream=side)
    side.synchronize()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            K.kv_paged_plan(p, ctx, new, table)
            K.kv_paged_attention(p, cache, q, out=out)
    side.synchronize()
    for i in range(5):
        ctx.copy_(torch.tensor([600 - 113 * i, 30 + 120 * i], **i32))
        q.normal_(generator=g)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        fresh = K.Plan(2, 2, 16, 40, 8, 2, 64, max_new=1)
        K.kv_paged_plan(fresh, ctx, new, table)
        assert torch.equal(out, K.kv_paged_attention(fresh, cache, q))


def test_refusals():
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    kc, vc = torch.zeros(4, 2, 16, 64, device="cuda").half(), torch.zeros(4, 2, 64, 16, device="cuda").half()
    cache, q = K.Cache(kc, vc), torch.zeros(3, 4, 64, device="cuda").half()
    p = K.Plan(1, 3, 16, 2, 4, 2, 64)
    with pytest.raises(ValueError):
        K.kv_paged_attention(p, cache, q)
    K.kv_paged_plan(p, torch.zeros(1, **i32), torch.full((1,), 3, **i32), torch.zeros(1, 2, **i32))
    for bad in (lambda: K.kv_paged_attention(p, cache, q[:2]), lambda: K.kv_paged_attention(p, cache, q[:, :2]), lambda: K.kv_paged_attention(p, cache, q.float()),
                lambda: K.kv_paged_attention(p, cache, q, out=q.bfloat16()), lambda: K.kv_paged_attention(p, cache, q, lse=torch.zeros(3, 4, device="cuda").half()),
                lambda: K.kv_paged_attention(p, cache, q, lse=torch.zeros(3, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(K.KvError):
        K.kv_paged_attention(p, cache, q.bfloat16())
    with pytest.raises(K.KvError):
        K.kv_paged_attention(p, cache, q, scale=-1.0)


def test_a_work_list_for_other_sizes_is_not_followed():
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    kc, vc = torch.zeros(4, 2, 16, 64, device="cuda").half(), torch.zeros(4, 2, 64, 16, device="cuda").half()
    for max_new in (1, None):
        p = K.Plan(2, 2, 16, 2, 4, 2, 64, max_new=max_new)
        q, out = torch.ones(2, 4, 64, device="cuda").half(), torch.full((2, 4, 64), 3.0, device="cuda").half()
        K.kv_paged_plan(p, torch.zeros(2, **i32), torch.ones(2, **i32), torch.zeros(2, 2, **i32))
        p.batch.window = 7
        K.kv_paged_attention(p, K.Cache(kc, vc), q, out=out)
        assert bool((out == 3.0).all())
        p.batch.window = 0
        K.kv_paged_attention(p, K.Cache(kc, vc), q, out=out)
        assert bool((out == 0.0).all())


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new, kept", [(1, "f16"), (1, "fp8"), (150, "f16"), (150, "fp8")])
def test_many_small_weights(dim, new, kept):
    """One key outweighs the others, and its value is zero: what remains is a sum of
    weights near 2^-17, whose rounding has to be relative (as multiples of float16's
    smallest number they would be off by 2^-8; the scores are chosen for that)."""
    score = 11.8515625 if kept == "f16" else 11.0    # exact in the cache's type; of 8 bits, times 32 and the head's scale

    def edit(kc, vc, table):
        kc.zero_()
        vc.fill_(1.0)
        first = int(table[0, 0])
        kc[first, :, 0, 0] = score
        vc[first, :, :, 0] = 0.0

    def edit_q(q):
        q.zero_()
        q[..., 0] = 1.0
    out, _ = case([700], [new], 64, (8, 2), dim, "f16", kept, max_new=1 if new == 1 else None, edit=edit, edit_q=edit_q, scale=1.0 if kept == "f16" else 32.0)
    assert bool((out > 0).all())


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 150])
def test_large_values_while_scores_rise(dim, new):
    """Scores rise by 2^30 in weight from one run of keys to the next, over values of
    10^30: nothing on the way to their average passes the 32-bit range."""
    def edit(kc, vc, table):
        kc.zero_()
        vc.fill_(1.0e30)
        for col in range(table.shape[1]):
            kc[int(table[0, col]), :, :, 0] = 20.75 * col

    def edit_q(q):
        q.zero_()
        q[..., 0] = 1.0
    out, _ = case([700], [new], 64, (8, 2), dim, "bf16", "bf16", max_new=1 if new == 1 else None, edit=edit, edit_q=edit_q, scale=1.0)
    assert bool((out > 9.0e29).all())


@pytest.mark.parametrize("new", [1, 150])
def test_infinite_scores(new):
    """A score of -inf weighs nothing, where there is no other the query sees nothing;
    one of +inf leaves NaN, in the log-sum-exp as well."""
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    gen = torch.Generator().manual_seed(4)
    kc, vc = torch.randn(8, 1, 64, 64, generator=gen).bfloat16().cuda(), torch.randn(8, 1, 64, 64, generator=gen).bfloat16().cuda()
    q = torch.randn(new, 3, 64, generator=gen).bfloat16().cuda()
    table = torch.arange(8, **i32).view(1, 8)
    q[:, 0, 5], q[:, 1, 5], q[:, 2, 5] = -1.0, 1.0, -1.0
    q[:, 2, 6] = -1.0
    kc[3, 0, 7, 5] = float("inf")                     # heads 0, 2: -inf; head 1: +inf
    kc[:, 0, :, 6] = torch.where(torch.isinf(kc[:, 0, :, 5]), 0.0, 1.0).to(kc.dtype)
    p = K.Plan(1, new, 64, 8, 3, 1, 64, max_new=1 if new == 1 else None)
    K.kv_paged_plan(p, torch.full((1,), 300, **i32), torch.full((1,), new, **i32), table)
    lse = torch.empty(new, 3, device="cuda")
    out = K.kv_paged_attention(p, K.Cache(kc, vc), q, lse=lse)
    assert bool(torch.isnan(out[:, 1]).all()) and bool(torch.isnan(lse[:, 1]).all())
    want, want_lse, spread, _ = O.attention(q, kc, vc, table.tolist(), p.q_start.tolist(), [300], 64, 8, 64 ** -0.5, 0)
    for h in (0, 2):   # scores of less than 2^7: 64 products are off by less than 2^-10
        err = (out[:, h].double() - want[:, h]).abs()
        assert bool((err <= (2.0 ** -8 + 2.0 ** -9) * spread[:, h] + 2.0 ** -8 * want[:, h].abs()).all())
        assert bool(((lse[:, h].double() - want_lse[:, h]).abs() <= 2.0 ** -10).all())
    kc[:, :, :, 5] = float("inf")                     # heads 0 and 2: nothing but -inf
    K.kv_paged_attention(p, K.Cache(kc, vc), q, out=out, lse=lse)
    assert bool((out[:, 0] == 0).all()) and bool((out[:, 2] == 0).all()) and bool((lse[:, 0] == -math.inf).all())
