"""The write into a cache of 8 bits with a scale for each block and head, and the read
of caches into rows, against their definitions in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

KINDS = [("bf16", "i8"), ("f16", "i8"), ("bf16", "fp8"), ("f16", "fp8")]


def by_token(x):
    """[blocks, heads, dim, block] as [blocks, heads, block, dim]."""
    return x.transpose(2, 3)


def check_held(got, scale, want, x, kind, slack):
    """Held numbers (float64) against the oracle's, and the values against x: half a unit of
    the held type off, plus `slack` (how far x itself may be off, in units of the scale); a
    number may be its neighbour's where x lies between the two."""
    import torch
    near = torch.isfinite(x)
    off = (got * scale - x).abs()
    unit = torch.full_like(x, 0.5) if kind == "i8" else torch.clamp((x / scale.clamp(min=1e-300)).abs() * 2.0 ** -4, min=2.0 ** -10)
    bound = (unit * (1 + 2.0 ** -20) + slack) * scale
    assert bool((off <= bound)[near].all()), float((off / bound.clamp(min=1e-300))[near].max())
    assert int((got != want)[near].sum()) <= max(2, 1e-3 * int(near.sum()))
    rest = ~near
    assert torch.equal(torch.nan_to_num(got[rest], nan=1e9), torch.nan_to_num(want[rest], nan=1e9))


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("ctx, new, block, heads, dim, rot, interleaved", [
    ([0], [1], 16, (1, 1), 64, 64, 0),
    ([15, 16, 17, 0], [1, 1, 1, 1], 16, (8, 2), 128, 128, 0),
    ([3, 0, 40, 8, 100], [30, 0, 17, 8, 5], 16, (6, 3), 64, 32, 1),
    ([60, 1], [70, 200], 64, (4, 4), 256, 256, 0),
    ([250, 255], [20, 2], 256, (16, 1), 256, 64, 1),
    ([7, 500, 30, 0], [1, 900, 2, 16], 32, (40, 8), 128, 128, 0)])
def test_write(dtype, kept, ctx, new, block, heads, dim, rot, interleaved):
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import ROUND, TYPES, blocks_of, held_cache
    gen = torch.Generator().manual_seed(sum(ctx) + 7 * block)
    H, J = heads
    table, n_blocks = blocks_of(ctx, new, block, gen)
    total = sum(new)
    T = total + 5  # a padded step: the last rows are nobody's
    fused = (torch.randn(T, H + 2 * J, dim, generator=gen) * 3 * (1 + torch.arange(T)[:, None, None] % 3)).to(TYPES[dtype]).cuda()
    q, k, v = fused[:, :H], fused[:, H:H + J], fused[:, H + J:]
    if dim > 64:
        v[0, 0, :3] = torch.tensor([float("inf"), -float("inf"), float("nan")])
    kc, vc, ks, vs = held_cache(n_blocks, J, block, dim, kept, gen)
    kw = dict(base=500000.0, scaling=2, factor=16.0, original_len=4096)
    rope = K.Rope(rot, layout=interleaved, magnitude=1.2, **kw)
    freq = O.frequencies(rot, **kw)
    p = K.Plan(len(ctx), T, block, table.shape[1], H, J, dim)
    i32 = dict(dtype=torch.int32, device="cuda")
    K.kv_paged_plan(p, torch.tensor(ctx, **i32), torch.tensor(new, **i32), table)
    q_out = torch.full((T, H, dim), 9.0, dtype=q.dtype, device="cuda")
    before = [t.clone() for t in (kc, vc, ks, vs)]
    cache = K.Cache(kc, vc, ks, vs, block_scales=True)
    K.kv_paged_append(p, cache, k, v, q=q, q_out=q_out, rope=rope)
    pos = p.pos[:total]
    want_q = O.rope(q[:total], pos, freq, interleaved, 1.2)
    size = 1.2 * q[:total].double().abs().amax(-1, keepdim=True) * 2
    assert bool(((q_out[:total].double() - want_q).abs() <= ROUND[q.dtype] * want_q.abs() + 2.0 ** -20 * size).all())
    assert bool((q_out[total:] == 9.0).all())
    for x, got, scales, old, old_scales in (
            (O.rope(k[:total], pos, freq, interleaved, 1.2), kc, ks, before[0], before[2]),
            (v[:total].double(), by_token(vc), vs, by_token(before[1]), before[3])):
        x, numbers, want_scale = x.cpu(), old.double().cpu(), old_scales.double().cpu()
        places = O.write_blocks(x, numbers, want_scale, table.tolist(), p.q_start.tolist(), ctx, block, n_blocks, kept)
        # scales: the turned keys are off by 2^-20 of 2.4 times the largest element
        assert bool(((scales.double().cpu() - want_scale).abs() <= 2.0 ** -18 * want_scale).all())
        page, at = torch.tensor([a for a, _ in places]), torch.tensor([b for _, b in places])
        got, exact = got.double().cpu(), scales.double().cpu()
        slack = 2.0 ** -18 * O.MOST[kept]
        check_held(got[page, :, at], exact[page][:, :, None], numbers[page, :, at], x, kept, slack)
        # earlier numbers in the new unit exactly, everything else as it was
        rest = torch.ones(n_blocks, block, dtype=torch.bool)
        rest[page, at] = False
        same = lambda a, b: torch.equal(torch.nan_to_num(a, nan=1e9), torch.nan_to_num(b, nan=1e9))  # noqa: E731
        assert same(got.transpose(1, 2)[rest], numbers.transpose(1, 2)[rest])
        untouched = torch.ones(n_blocks, dtype=torch.bool)
        untouched[page] = False
        assert torch.equal(scales.cpu()[untouched], old_scales.cpu()[untouched])
    # again: nothing rises a second time
    after = [t.clone() for t in (kc, vc, ks, vs)]
    K.kv_paged_append(p, cache, k, v, q=q, q_out=q_out, rope=rope)
    assert all(torch.equal(a.view(torch.int8), b.view(torch.int8)) for a, b in zip(after, (kc, vc, ks, vs)))


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("block", [16, 64])
def test_token_by_token(dtype, kept, block):
    """A sequence that grows by single tokens, larger and smaller ones, zeros, infinities and
    NaN among them: numbers and scales after every step are those of 32-bit arithmetic."""
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import TYPES, held_cache
    gen = torch.Generator().manual_seed(block)
    i32 = dict(dtype=torch.int32, device="cuda")
    J, D, N = 2, 64, block + 9
    kc, vc, ks, vs = held_cache(4, J, block, D, kept, gen)
    cache = K.Cache(kc, vc, ks, vs, block_scales=True)
    table = torch.tensor([[2, 0]], **i32)
    plan = K.Plan(1, 1, block, 2, J, J, D, max_new=1)
    x = torch.randn(N, 2 * J, D, generator=gen)
    x *= torch.exp2(torch.randint(-6, 7, (N, 1, 1), generator=gen).float())
    x[0] = 0
    x[3, :, 5] = float("nan")
    x[4, :, 6:8] = torch.tensor([float("inf"), -float("inf")])
    x[6, 1] = 0
    x = x.to(TYPES[dtype])
    sides = [(x[:, :J], kc.double().cpu(), ks.double().cpu()), (x[:, J:], by_token(vc).double().cpu(), vs.double().cpu())]
    for t in range(N):
        K.kv_paged_plan(plan, torch.tensor([t], **i32), torch.tensor([1], **i32), table)
        step = x[t:t + 1].cuda()
        K.kv_paged_append(plan, cache, step[:, :J], step[:, J:])
        for (values, numbers, scale), got, scales in zip(sides, (kc, by_token(vc)), (ks, vs)):
            page, at = (2, 0)[t // block], t % block
            for j in range(J):
                # the definition, scales and reciprocals in 32 bits
                new = values[t, j].float()
                size = new[torch.isfinite(new)].abs().max()
                need = size / torch.tensor(O.MOST[kept])
                old = scale[page, j].float() if at else torch.tensor(0.0)
                if old > 0:
                    m = O.rises(float(need), float(old))
                    numbers[page, j, :at] = O.held(numbers[page, j, :at] * 2.0 ** -m, kept) if m else numbers[page, j, :at]
                    s = old * 2.0 ** m
                else:
                    s = need
                    if at and need > 0:
                        numbers[page, j, :at] = O.held(numbers[page, j, :at] * 0.0, kept)
                scale[page, j] = s.double()
                inverse = 1.0 / s if s > 0 else torch.tensor(2.0 ** -126)
                numbers[page, j, at] = O.held((new * inverse).double(), kept)
            assert torch.equal(scales.cpu().double(), scale), t
            assert torch.equal(torch.nan_to_num(got.double().cpu(), nan=1e9), torch.nan_to_num(numbers, nan=1e9)), t


@pytest.mark.parametrize("kept", ["i8", "fp8"])
def test_scales_that_no_write_left(kept):
    """A block that goes on with something that is no scale begins anew; its earlier numbers
    are then zeros."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import held_cache
    gen = torch.Generator().manual_seed(1)
    i32 = dict(dtype=torch.int32, device="cuda")
    kc, vc, ks, vs = held_cache(6, 1, 16, 64, kept, gen)
    bad = torch.tensor([float("nan"), float("inf"), -1.0, 0.0, 1e-40, -float("inf")], device="cuda")
    ks[:, 0], vs[:, 0] = bad, bad.flip(0)
    plan = K.Plan(6, 6, 16, 1, 1, 1, 64, max_new=1)
    K.kv_paged_plan(plan, torch.full((6,), 5, **i32), torch.ones(6, **i32), torch.arange(6, **i32)[:, None].contiguous())
    x = torch.randn(6, 2, 64, generator=gen).half().cuda()
    K.kv_paged_append(plan, K.Cache(kc, vc, ks, vs, block_scales=True), x[:, :1], x[:, 1:])
    most = torch.tensor(127.0 if kept == "i8" else 448.0, device="cuda")
    assert torch.equal(ks[:, 0], x[:, 0].float().abs().amax(-1) / most) and torch.equal(vs[:, 0], x[:, 1].float().abs().amax(-1) / most)
    assert bool((kc[:, :, :5].float() == 0).all()) and bool((vc[:, :, :, :5].float() == 0).all())
    assert bool((kc[:, 0, 5].float() != 0).any())


@pytest.mark.parametrize("kept", ["i8", "fp8"])
def test_tokens_without_a_place(kept):
    """No block, a block past the cache's end, and an idle request: nothing else changes."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import held_cache
    gen = torch.Generator().manual_seed(2)
    i32 = dict(dtype=torch.int32, device="cuda")
    x = torch.randn(60, 4, 64, generator=gen).bfloat16().cuda()
    p = K.Plan(4, 60, 16, 2, 2, 2, 64)
    table = torch.tensor([[0, -1], [-1, 1], [2, 2000], [3, -1]], **i32)
    K.kv_paged_plan(p, torch.tensor([4, 0, 0, 16], **i32), torch.tensor([20, 20, 20, 0], **i32), table)
    kc, vc, ks, vs = held_cache(5, 2, 16, 64, kept, gen)
    before = [t.clone() for t in (kc, vc, ks, vs)]
    K.kv_paged_append(p, K.Cache(kc[:4], vc[:4], ks[:4], vs[:4], block_scales=True), x[:, :2], x[:, 2:])
    wrote = torch.zeros(5, 16, dtype=torch.bool, device="cuda")
    wrote[0, :16] = wrote[1, :4] = wrote[2] = True  # (block 0's earlier tokens may be in a new unit)
    bits = lambda t: t.view(torch.int8)  # noqa: E731
    assert torch.equal(bits(kc).transpose(1, 2)[~wrote], bits(before[0]).transpose(1, 2)[~wrote])
    assert torch.equal(bits(vc).permute(0, 3, 1, 2)[~wrote], bits(before[1]).permute(0, 3, 1, 2)[~wrote])
    assert torch.equal(ks[3:], before[2][3:]) and torch.equal(vs[3:], before[3][3:])
    k, v = K.kv_paged_read(p, K.Cache(kc[:4], vc[:4], ks[:4], vs[:4], block_scales=True), torch.tensor([0, 0, 20, 40, 40], **i32), rows=40)
    assert bool((k[:16] == 0).all()) and bool((v[:16] == 0).all()) and bool((k[36:] == 0).all())
    top = x[36:40, :2].float().abs().amax((0, 2)) if kept == "i8" else None
    if top is not None:
        assert bool(((k[16:20].float() - x[36:40, :2].float()).abs() <= top[None, :, None] * (0.5 / 127 + 2.0 ** -8)).all())


def test_far_offsets():
    """Blocks whose offsets pass 32 bits, keys and values of a block side by side."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    g = torch.Generator(device="cuda").manual_seed(3)
    i32 = dict(dtype=torch.int32, device="cuda")
    n_blocks, J, block, dim = 180_000, 8, 16, 128  # 2 x 16 KiB a block: 5.9 GB
    both = torch.zeros(n_blocks, 2, J * block * dim, device="cuda", dtype=torch.int8)
    kc, vc = both[:, 0].view(n_blocks, J, block, dim), both[:, 1].view(n_blocks, J, dim, block)
    ks, vs = torch.zeros(n_blocks, J, device="cuda"), torch.zeros(n_blocks, J, device="cuda")
    cache = K.Cache(kc, vc, ks, vs, block_scales=True)
    x = torch.randn(35, 2 * J, dim, device="cuda", generator=g).bfloat16()
    p = K.Plan(1, 35, block, 4, J, J, dim)
    table = torch.tensor([[179_999, 5, 170_000, 1]], **i32)
    K.kv_paged_plan(p, torch.tensor([3], **i32), torch.tensor([35], **i32), table)
    K.kv_paged_append(p, cache, x[:, :J], x[:, J:])
    k, v = K.kv_paged_read(p, cache, torch.tensor([0, 35], **i32), first=torch.tensor([3], **i32), rows=35)
    page = p.slot // block
    for got, want, s in ((k, x[:, :J], ks), (v, x[:, J:], vs)):
        assert bool(((got.float() - want.float()).abs() <= s[page][:, :, None] * 0.5001 + got.float().abs() * 2.0 ** -8).all())
    assert int((both != 0).flatten(1).any(1).sum()) == 3 and int((ks != 0).any(1).sum()) == 3
    q = torch.randn(35, J, dim, device="cuda", generator=g).bfloat16()
    near = K.Plan(1, 35, block, 4, J, J, dim)
    pages = table[0, :3].long()
    K.kv_paged_plan(near, torch.tensor([3], **i32), torch.tensor([35], **i32), torch.tensor([[0, 1, 2, 3]], **i32))
    small = K.Cache(kc[pages].contiguous(), vc[pages].contiguous(), ks[pages], vs[pages], block_scales=True)
    assert torch.equal(K.kv_paged_attention(p, cache, q), K.kv_paged_attention(near, small, q))


@pytest.mark.parametrize("kept, dtype", [("bf16", "bf16"), ("f16", "f16"), ("head", "bf16"), ("i8", "bf16"), ("i8", "f16"), ("fp8", "f16"), ("fp8", "bf16")])
@pytest.mark.parametrize("block, dim, heads", [(16, 64, 3), (16, 128, 8), (64, 128, 2), (256, 256, 1), (32, 64, 5)])
def test_read(kept, dtype, block, dim, heads):
    """Every kind of cache; rows that are not there; parts, and rows past the last."""
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import ROUND, TYPES, blocks_of, cache_values, held_cache
    gen = torch.Generator().manual_seed(block + dim)
    lens = [1, 0, 2 * block + 5, 17, block, 3]
    table, n_blocks = blocks_of(lens, [0] * 6, block, gen)
    table[2, 1] = -1
    table[3, 0] = n_blocks + 4
    if kept in ("i8", "fp8"):
        kc, vc, ks, vs = held_cache(n_blocks, heads, block, dim, kept, gen)
        cache, scales = K.Cache(kc, vc, ks, vs, block_scales=True), (ks, vs)
    else:
        kc, vc, ks, vs = cache_values(n_blocks, heads, block, dim, "fp8" if kept == "head" else kept, gen)
        cache = K.Cache(kc, vc, ks, vs)
        scales = [torch.ones(n_blocks, heads) if s is None else s.expand(n_blocks, heads) for s in (ks, vs)]
    i32 = dict(dtype=torch.int32, device="cuda")
    p = K.Plan(6, 1, block, table.shape[1], heads, heads, dim)
    K.kv_paged_plan(p, torch.tensor(lens, **i32), torch.zeros(6, **i32), table)
    for first in (None, [0, 5, block - 3, 2, -4, 1]):
        counts = [2, 4, 2 * block, 17, block + 9, 0]
        starts = [0]
        for n in counts:
            starts.append(starts[-1] + n)
        rows = starts[-1]
        at = torch.tensor(starts, **i32)
        outs = [torch.full((rows + 6, heads + 2, dim), 7.0, dtype=TYPES[dtype], device="cuda") for _ in range(2)]
        k, v = (o[:, 1:1 + heads] for o in outs)
        K.kv_paged_read(p, cache, at, first=None if first is None else torch.tensor(first, **i32), k=k, v=v)
        for got, numbers, s, whole in ((k, kc, scales[0], outs[0]), (v, by_token(vc), scales[1], outs[1])):
            want = O.read_rows(numbers.double().cpu(), s.double().cpu(), table.tolist(), lens, block, n_blocks, starts, first or [0] * 6)
            # one rounding of the product in 32 bits, one to 16 (float16: 2^-25 below its normal numbers)
            bound = want.abs() * (ROUND[TYPES[dtype]] * (1 + 2.0 ** -20) + 2.0 ** -24) + 2.0 ** -25
            if kept in ("bf16", "f16"):
                bound = 0 * want
            assert bool(((got[:rows].double().cpu() - want).abs() <= bound).all())
            assert bool((whole[rows:] == 7.0).all()) and bool((whole[:, 0] == 7.0).all()) and bool((whole[:, -1] == 7.0).all())
        # fewer rows than row_start says: the first ones
        part = rows - 20
        k2, v2 = K.kv_paged_read(p, cache, at, first=None if first is None else torch.tensor(first, **i32), rows=part, dtype=TYPES[dtype])
        assert k2.shape == (part, heads, dim) and torch.equal(k2, k[:part]) and torch.equal(v2, v[:part])


@pytest.mark.parametrize("kept", ["i8", "fp8"])
@pytest.mark.parametrize("block", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_every_block_and_head_size(kept, block, dim):
    """Parts of blocks, whole blocks and single tokens, written without rotation: numbers are those
    of 32-bit arithmetic, and come back as such."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import blocks_of, held_cache
    gen = torch.Generator().manual_seed(block + dim)
    i32 = dict(dtype=torch.int32, device="cuda")
    J, ctx, new = 3, [0, 5, block - 1, block, 2 * block - 3, 7], [2 * block + 3, block - 5, 1, block, 2, 0]
    table, n_blocks = blocks_of(ctx, new, block, gen)
    kc, vc, ks, vs = held_cache(n_blocks, J, block, dim, kept, gen)
    old = [t.clone() for t in (ks, vs)]
    total = sum(new)
    x = (torch.randn(total, 2 * J, dim, generator=gen) * 2).bfloat16().cuda()
    p = K.Plan(len(ctx), total, block, table.shape[1], J, J, dim)
    K.kv_paged_plan(p, torch.tensor(ctx, **i32), torch.tensor(new, **i32), table)
    cache = K.Cache(kc, vc, ks, vs, block_scales=True)
    K.kv_paged_append(p, cache, x[:, :J], x[:, J:])
    most = 127.0 if kept == "i8" else 448.0
    page, at = p.slot // block, p.slot % block
    for numbers, s, before, want in ((kc, ks, old[0], x[:, :J]), (by_token(vc), vs, old[1], x[:, J:])):
        top = torch.zeros_like(s).scatter_reduce(0, page[:, None].expand(-1, J), want.float().abs().amax(-1), "amax")
        need = top / torch.full_like(top, most)
        begins = torch.zeros(n_blocks, dtype=torch.bool, device="cuda")
        begins[page[at == 0]] = True
        touched = torch.zeros_like(begins)
        touched[page] = True
        rise = torch.where(need > before, torch.ceil(torch.log2(need.double() / before.double())), 0.0)
        expect = torch.where(begins[:, None], need, torch.where(touched[:, None], (before.double() * torch.exp2(rise)).float(), before))
        assert torch.equal(s, expect)
        y = want.float() * (1.0 / s)[page][:, :, None]
        y = y.clamp(-most, most)
        y = y.round() if kept == "i8" else y.to(torch.float8_e4m3fn).float()
        assert torch.equal(numbers.float()[page, :, at], y)
    starts, firsts = [0], []
    for c, n in zip(ctx, new):
        starts.append(starts[-1] + n)
        firsts.append(c)
    k, v = K.kv_paged_read(p, cache, torch.tensor(starts, **i32), first=torch.tensor(firsts, **i32), rows=total)
    assert torch.equal(k, (kc.float()[page, :, at] * ks[page][:, :, None]).bfloat16())
    assert torch.equal(v, (vc.float()[page, :, :, at] * vs[page][:, :, None]).bfloat16())


def test_read_of_many_requests():
    """Requests by the thousand, ragged and empty ones, rows that do not begin at 0."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import blocks_of, held_cache
    gen = torch.Generator().manual_seed(5)
    i32 = dict(dtype=torch.int32, device="cuda")
    for n_req, most in ((4096, 40), (1000, 90), (65, 700), (64, 3), (2, 3000)):
        lens = torch.randint(0, most, (n_req,), generator=gen).tolist()
        lens[n_req // 2] = 0
        table, n_blocks = blocks_of(lens, [0] * n_req, 16, gen)
        kc, vc, ks, vs = held_cache(n_blocks, 2, 16, 64, "i8", gen)
        cache = K.Cache(kc, vc, ks, vs, block_scales=True)
        p = K.Plan(n_req, 1, 16, table.shape[1], 2, 2, 64)
        K.kv_paged_plan(p, torch.tensor(lens, **i32), torch.zeros(n_req, **i32), table)
        for skip in (0, 100):
            start = torch.cumsum(torch.tensor([skip] + lens), 0).to(torch.int32).cuda()
            k, v = torch.full((skip + sum(lens), 2, 64), 7.0, device="cuda", dtype=torch.bfloat16), torch.full((skip + sum(lens), 2, 64), 7.0, device="cuda", dtype=torch.bfloat16)
            K.kv_paged_read(p, cache, start, k=k, v=v)
            row = torch.arange(sum(lens), device="cuda")
            req = torch.searchsorted(start[1:] - skip, row.to(torch.int32), right=True)
            pos = row - (start[req] - skip)
            page, at = table[req, pos // 16].long(), pos % 16
            assert torch.equal(k[skip:], (kc[page, :, at].float() * ks[page][:, :, None]).bfloat16())
            assert torch.equal(v[skip:], (vc[page, :, :, at].float() * vs[page][:, :, None]).bfloat16())
            assert bool((k[:skip] == 7.0).all()) and bool((v[:skip] == 7.0).all())


def test_write_of_many_requests():
    """The same for the write: a thousand ragged prompts over cached prefixes."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import blocks_of, held_cache
    gen = torch.Generator().manual_seed(6)
    i32 = dict(dtype=torch.int32, device="cuda")
    for n_req, most, max_new in ((1000, 70, None), (4096, 2, 1), (300, 5, 4)):
        ctx = torch.randint(0, 50, (n_req,), generator=gen).tolist()
        new = torch.randint(0, most, (n_req,), generator=gen).tolist()
        table, n_blocks = blocks_of(ctx, new, 16, gen)
        kc, vc, ks, vs = held_cache(n_blocks, 2, 16, 64, "i8", gen)
        total = sum(new)
        x = torch.randn(total, 4, 64, generator=gen).half().cuda()
        p = K.Plan(n_req, total, 16, table.shape[1], 2, 2, 64, max_new=max_new)
        K.kv_paged_plan(p, torch.tensor(ctx, **i32), torch.tensor(new, **i32), table)
        assert p.result.tolist() == [total, 0, 0, 0]
        K.kv_paged_append(p, K.Cache(kc, vc, ks, vs, block_scales=True), x[:, :2], x[:, 2:])
        page, at = p.slot // 16, p.slot % 16
        for got, want, s in ((kc[page, :, at], x[:, :2], ks[page]), (vc[page, :, :, at], x[:, 2:], vs[page])):
            assert bool(((got.float() - want.float() / s[:, :, None]).abs() <= 0.5001).all())


def test_a_step_end_to_end_in_a_graph():
    """Plan, write, attention and read together, captured and replayed as the requests grow;
    each replay against the same calls made eagerly."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import held_cache
    gen = torch.Generator().manual_seed(7)
    i32 = dict(dtype=torch.int32, device="cuda")
    R, H, J, D, B, W = 5, 8, 2, 128, 16, 6
    table = torch.randperm(R * W, generator=gen).to(torch.int32).reshape(R, W).cuda()
    first = held_cache(R * W, J, B, D, "i8", gen)
    ctx0 = torch.tensor([0, 14, 15, 16, 40], **i32)
    x = torch.empty(R, H + 2 * J, D, device="cuda", dtype=torch.bfloat16)
    steps = [torch.randn(R, H + 2 * J, D, generator=gen).cuda().bfloat16() * (1 + i) for i in range(6)]
    rope = K.Rope(D)

    def make():
        tensors = [t.clone() for t in first]
        plan = K.Plan(R, R, B, W, H, J, D, max_new=1)
        return dict(cache=K.Cache(*tensors, block_scales=True), tensors=tensors, plan=plan, ctx=ctx0.clone(), new=torch.ones(R, **i32),
                    rows=torch.arange(0, 17 * R, 16, **i32)[:R + 1].contiguous(), k=torch.zeros(16 * R, J, D, device="cuda", dtype=torch.bfloat16),
                    v=torch.zeros(16 * R, J, D, device="cuda", dtype=torch.bfloat16), q=torch.empty(R, H, D, device="cuda", dtype=torch.bfloat16),
                    out=torch.empty(R, H, D, device="cuda", dtype=torch.bfloat16))

    def step(s):
        K.kv_paged_plan(s["plan"], s["ctx"], s["new"], table)
        K.kv_paged_append(s["plan"], s["cache"], x[:, H:H + J], x[:, H + J:], q=x[:, :H], q_out=s["q"], rope=rope)
        K.kv_paged_attention(s["plan"], s["cache"], s["q"], out=s["out"])
        K.kv_paged_read(s["plan"], s["cache"], s["rows"], k=s["k"], v=s["v"])

    eager, held = make(), make()
    x.copy_(steps[0])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(held)
    torch.cuda.synchronize()
    for i, values in enumerate(steps):
        x.copy_(values)
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        for a, b in zip(eager["tensors"] + [eager["out"], eager["k"], eager["v"]], held["tensors"] + [held["out"], held["k"], held["v"]]):
            assert torch.equal(a.view(torch.int8), b.view(torch.int8)), i
        eager["ctx"] += 1
        held["ctx"] += 1


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("window", [0, 20])
def test_what_a_new_cache_holds_does_not_matter(dtype, kept, window):
    """Prompts and single tokens over memory that holds anything, scales that are no numbers
    among it, give what they give over a cleared cache, bit for bit."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import TYPES
    gen = torch.Generator().manual_seed(8)
    i32 = dict(dtype=torch.int32, device="cuda")
    R, H, J, D, B, W = 3, 8, 2, 128, 16, 8
    held = TYPES.get(kept, torch.int8)
    pool = torch.randperm(R * W + 5, generator=gen).to(torch.int32).cuda()
    steps = [[33, 5, 60], [1, 1, 1], [0, 30, 1], [1, 1, 1]]
    inputs = [(torch.randn(sum(n), H + 2 * J, D, generator=gen)).to(TYPES[dtype]).cuda() for n in steps]
    results = []
    for dirty in (False, True):
        kc, vc = torch.zeros(R * W + 5, J, B, D, dtype=torch.int8), torch.zeros(R * W + 5, J, D, B, dtype=torch.int8)
        ks, vs = torch.zeros(R * W + 5, J), torch.zeros(R * W + 5, J)
        if dirty:
            kc, vc = (torch.randint(-128, 128, t.shape, generator=gen).to(torch.int8) for t in (kc, vc))
            bad = torch.tensor([float("nan"), float("inf"), 1e38, -1.0, 0.0, 1e-42])
            ks, vs = (bad[torch.randint(0, 6, t.shape, generator=gen)] for t in (ks, vs))
        cache = K.Cache(*[t.cuda().view(held) for t in (kc, vc)], ks.cuda(), vs.cuda(), block_scales=True)
        rope = K.Rope(D)
        table, taken, ctx, outs = torch.full((R, W), -1, **i32), 0, [0] * R, []
        for new, x in zip(steps, inputs):
            n = sum(new)
            p = K.Plan(R, n, B, W, H, J, D, max_new=max(new), window=window)
            K.kv_paged_plan(p, torch.tensor(ctx, **i32), torch.tensor(new, **i32), table, pool[taken:].contiguous())
            q = torch.empty(n, H, D, device="cuda", dtype=x.dtype)
            K.kv_paged_append(p, cache, x[:, H:H + J], x[:, H + J:], q=x[:, :H], q_out=q, rope=rope)
            outs.append(K.kv_paged_attention(p, cache, q))
            starts = torch.zeros(R + 1, **i32)
            starts[1:] = torch.cumsum(p.kv_len, 0)
            outs += K.kv_paged_read(p, cache, starts, rows=int(starts[-1]), dtype=x.dtype)
            taken += int(p.result[2])
            ctx = p.kv_len.tolist()
        results.append(outs)
    for a, b in zip(*results):
        assert bool(torch.isfinite(a.float()).all()) and torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_refusals():
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    f32 = dict(dtype=torch.float32, device="cuda")
    x = torch.zeros(8, 2, 64, device="cuda", dtype=torch.bfloat16)
    kc, vc = torch.zeros(4, 2, 16, 64, device="cuda", dtype=torch.int8), torch.zeros(4, 2, 64, 16, device="cuda", dtype=torch.int8)
    s = torch.ones(4, 2, **f32)
    cache = K.Cache(kc, vc, s, s.clone(), block_scales=True)
    p = K.Plan(1, 8, 16, 2, 4, 2, 64)
    start = torch.tensor([0, 8], **i32)
    with pytest.raises(ValueError):
        K.kv_paged_read(p, cache, start, rows=8)  # not planned yet
    K.kv_paged_plan(p, torch.zeros(1, **i32), torch.full((1,), 8, **i32), torch.zeros(1, 2, **i32))
    for bad in (lambda: K.Cache(kc, vc, s, s), lambda: K.Cache(kc, vc, block_scales=True), lambda: K.Cache(kc, vc, s, block_scales=True),
                lambda: K.Cache(kc, vc, s[:3], s, block_scales=True), lambda: K.Cache(kc, vc, s.double(), s.double(), block_scales=True),
                lambda: K.Cache(kc, vc, s.cpu(), s.cpu(), block_scales=True), lambda: K.Cache(kc, vc, s[:, 0], s[:, 0], block_scales=True),
                lambda: K.Cache(kc.bfloat16(), vc.bfloat16(), s, s, block_scales=True), lambda: K.Cache(kc.view(torch.uint8), vc.view(torch.uint8), s, s, block_scales=True),
                lambda: K.Cache(kc, vc, s.t().contiguous().t(), s, block_scales=True),
                lambda: K.kv_paged_read(p, cache, start), lambda: K.kv_paged_read(p, cache, start[:1], rows=8), lambda: K.kv_paged_read(p, cache, start.long(), rows=8),
                lambda: K.kv_paged_read(p, cache, start, k=x), lambda: K.kv_paged_read(p, cache, start, k=x, v=x[:7]), lambda: K.kv_paged_read(p, cache, start, k=x, v=x.half()),
                lambda: K.kv_paged_read(p, cache, start, k=x.float(), v=x.float()), lambda: K.kv_paged_read(p, cache, start, k=x, v=x, rows=9),
                lambda: K.kv_paged_read(p, cache, start, rows=8, dtype=torch.float32), lambda: K.kv_paged_read(p, cache, start, k=x, v=x, dtype=torch.float16),
                lambda: K.kv_paged_read(p, cache, start, first=start.float(), rows=8)):
        with pytest.raises(ValueError):
            bad()
    plain = K.Cache(kc.bfloat16(), vc.bfloat16())
    with pytest.raises(K.KvError):
        K.kv_paged_read(p, plain, start, rows=8, dtype=torch.float16)
    with pytest.raises(K.KvError):
        K.kv_paged_read(p, cache, start, k=x, v=x)
    k, v = K.kv_paged_read(p, cache, start, rows=0)
    assert k.shape == (0, 2, 64) and v.shape == (0, 2, 64)
    assert math.isfinite(float(K.kv_paged_attention(p, cache, torch.ones(8, 4, 64, device="cuda", dtype=torch.bfloat16)).float().sum()))
