"""Reads large enough for 8 KB a wavefront, and small ones, of every kind of cache into both types
of rows: missing blocks, first positions that are not 0, rows cut off, rows at strides."""
import pytest

from tests import paged_read as R

pytestmark = pytest.mark.gpu

KINDS = [("bf16", "bf16"), ("f16", "f16"), ("head", "bf16"), ("head", "f16"), ("i8", "bf16"), ("i8", "f16"), ("fp8", "f16"), ("fp8", "bf16")]


def make(kept, block, dim, heads, lens, gen):
    """A cache, its table, and its numbers by token with their scales."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import blocks_of, cache_values, held_cache
    table, n_blocks = blocks_of(lens, [0] * len(lens), block, gen)
    if kept in ("i8", "fp8"):
        kc, vc, ks, vs = held_cache(n_blocks, heads, block, dim, kept, gen)
        cache, scales = K.Cache(kc, vc, ks, vs, block_scales=True), (ks, vs)
    else:
        kc, vc, ks, vs = cache_values(n_blocks, heads, block, dim, "fp8" if kept == "head" else kept, gen)
        cache = K.Cache(kc, vc, ks, vs)
        scales = [None if s is None else s.expand(n_blocks, heads) for s in (ks, vs)]
    return cache, table, n_blocks, ((kc, scales[0]), (vc.transpose(2, 3), scales[1]))


def rows_of(numbers, scale, table, n_blocks, kv_len, starts, first, block, dtype):
    """The rows by indexing: products in 32 bits, rounded once."""
    import torch
    row = torch.arange(starts[-1], device="cuda")
    start = torch.tensor(starts, device="cuda")
    req = torch.searchsorted(start[1:], row, right=True)
    pos = torch.tensor(first, device="cuda")[req] + row - start[req]
    column = torch.div(pos, block, rounding_mode="floor")
    inside = (pos >= 0) & (pos < torch.tensor(kv_len, device="cuda")[req])
    page = torch.where(inside, table.long()[req, column.clamp(0, table.shape[1] - 1)], -1)
    inside = (page >= 0) & (page < n_blocks)
    page = torch.where(inside, page, 0)
    x = numbers.view(torch.int8 if numbers.element_size() == 1 else torch.int16)[page, :, pos % block].view(numbers.dtype)
    if scale is not None:
        x = (x.float() * scale[page][:, :, None]).to(dtype)
    return torch.where(inside[:, None, None], x, torch.zeros_like(x))


def check(kept, dtype, block, dim, heads, n_req, lens, firsts, edit=True):
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import TYPES
    gen = torch.Generator().manual_seed(block + dim)
    cache, table, n_blocks, sides = make(kept, block, dim, heads, lens, gen)
    if edit:  # some blocks are gone, some are past the cache
        lost = torch.rand(table.shape, generator=gen).cuda()
        table[(lost < 0.05) & (table >= 0)] = -1
        table[(lost > 0.95) & (table >= 0)] = n_blocks + 3
    i32 = dict(dtype=torch.int32, device="cuda")
    p = K.Plan(n_req, 1, block, table.shape[1], heads, heads, dim)
    K.kv_paged_plan(p, torch.tensor(lens, **i32), torch.zeros(n_req, **i32), table)
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    rows, kind, at = starts[-1], TYPES[dtype], torch.tensor(starts, **i32)
    for first in firsts:
        given = None if first is None else torch.tensor(first, **i32)
        outs = [torch.full((rows + 6, heads + 2, dim), 7.0, dtype=kind, device="cuda") for _ in range(2)]
        K.kv_paged_read(p, cache, at, first=given, k=outs[0][:, 1:1 + heads], v=outs[1][:, 1:1 + heads])
        wants = [rows_of(x, s, table, n_blocks, lens, starts, first or [0] * n_req, block, kind) for x, s in sides]
        for whole, want in zip(outs, wants):
            assert torch.equal(whole[:rows, 1:1 + heads].contiguous().view(torch.int16), want.view(torch.int16))
            assert bool((whole[rows:] == 7.0).all()) and bool((whole[:, 0] == 7.0).all()) and bool((whole[:, -1] == 7.0).all())
        part = rows - 20
        for whole in outs:
            whole.fill_(7.0)
        K.kv_paged_read(p, cache, at, first=given, k=outs[0][:, 1:1 + heads], v=outs[1][:, 1:1 + heads], rows=part)
        for whole, want in zip(outs, wants):
            assert torch.equal(whole[:part, 1:1 + heads].contiguous().view(torch.int16), want[:part].view(torch.int16))
            assert bool((whole[part:] == 7.0).all())


@pytest.mark.parametrize("kept, dtype", KINDS)
@pytest.mark.parametrize("name", R.SHAPES)
def test_read(kept, dtype, name):
    import torch
    block, dim, heads, n_req, most, few = R.SHAPES[name]
    lens = R.lengths(n_req, most, 0)
    rows, wide = sum(lens), 1 if kept in ("i8", "fp8", "head") else 2
    assert all(R.few_wavefronts(n_req, n, block, heads, dim, wide) == few for n in (rows + 6, rows - 20))
    shift = torch.randint(-block - 3, 2 * block, (n_req,), generator=torch.Generator().manual_seed(3)).tolist()
    check(kept, dtype, block, dim, heads, n_req, lens, (None, shift))


@pytest.mark.parametrize("rows", [16352, 16353])
@pytest.mark.parametrize("kept, dtype", [("i8", "f16"), ("fp8", "bf16")])
def test_both_sides_of_the_border(kept, dtype, rows):
    """(The six rows past the last that check() adds do not count where `rows` is given.)"""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import TYPES
    assert R.few_wavefronts(1, rows, 16, 2, 64, 1) == (rows == 16352)
    cache, table, n_blocks, sides = make(kept, 16, 64, 2, [rows], torch.Generator().manual_seed(1))
    i32 = dict(dtype=torch.int32, device="cuda")
    p = K.Plan(1, 1, 16, table.shape[1], 2, 2, 64)
    K.kv_paged_plan(p, torch.tensor([rows], **i32), torch.zeros(1, **i32), table)
    for first in (0, 5):
        got = K.kv_paged_read(p, cache, torch.tensor([0, rows], **i32), first=torch.tensor([first], **i32), rows=rows, dtype=TYPES[dtype])
        for x, (numbers, scale) in zip(got, sides):
            want = rows_of(numbers, scale, table, n_blocks, [rows], [0, rows], [first], 16, TYPES[dtype])
            assert torch.equal(x.view(torch.int16), want.view(torch.int16))
