"""Rows read back in float16 near the end of its range: a held number times its scale may be
more than the value that was written, and more than float16 holds."""
import pytest

pytestmark = pytest.mark.gpu

MOST16 = 65504.0


def rows(cache, table, length):
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    J, block, D = cache.shape
    p = K.Plan(1, 1, block, table.shape[1], J, J, D)
    K.kv_paged_plan(p, torch.tensor([length], **i32), torch.zeros(1, **i32), table)
    return K.kv_paged_read(p, cache, torch.tensor([0, length], **i32), rows=length, dtype=torch.float16)


# A first token of this size, then one of 65,504: the scale is doubled, and 65,504 is 100.53 units
# (held as 101: 65,811) or, in e4m3, 377.1 (held as 384: 66,706).
@pytest.mark.parametrize("kept, before, held", [("i8", 41376.0, 101.0), ("fp8", 38912.0, 384.0)])
def test_finite_values_come_back_finite(kept, before, held):
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    kind = torch.int8 if kept == "i8" else torch.float8_e4m3fn
    kc, vc = torch.zeros(1, 1, 16, 64, device="cuda", dtype=kind), torch.zeros(1, 1, 64, 16, device="cuda", dtype=kind)
    cache = K.Cache(kc, vc, torch.zeros(1, 1, device="cuda"), torch.zeros(1, 1, device="cuda"), block_scales=True)
    table = torch.zeros(1, 1, **i32)
    p = K.Plan(1, 1, 16, 1, 1, 1, 64, max_new=1)
    for t, size in enumerate((before, MOST16)):
        x = torch.zeros(1, 2, 64, device="cuda", dtype=torch.float16)
        x[0, :, 3], x[0, :, 5], x[0, :, 6] = size, -size, size / 2
        K.kv_paged_plan(p, torch.tensor([t], **i32), torch.ones(1, **i32), table)
        K.kv_paged_append(p, cache, x[:, :1], x[:, 1:])
    assert kc[0, 0, 1, 3].float() == held and vc[0, 0, 5, 1].float() == -held
    assert float(cache.k_scale) * held > 65520.0  # what float16 rounds to infinity
    for got in rows(cache, table, 2):
        assert got[1, 0, 3] == MOST16 and got[1, 0, 5] == -MOST16
        assert bool(((got[:, 0, 6].float() - torch.tensor([before, MOST16], device="cuda") / 2).abs() <= 2.0 ** -4 * MOST16).all())


def test_finite_values_come_back_finite_with_scales_by_head():
    """65,504 is 436.7 of these units, held as 448."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    kc, vc = (torch.zeros(*s, device="cuda", dtype=torch.float8_e4m3fn) for s in ((1, 2, 16, 64), (1, 2, 64, 16)))
    scale = torch.full((2,), 150.0, device="cuda")
    cache, table = K.Cache(kc, vc, scale, scale), torch.zeros(1, 1, **i32)
    p = K.Plan(1, 1, 16, 1, 2, 2, 64, max_new=1)
    K.kv_paged_plan(p, torch.zeros(1, **i32), torch.ones(1, **i32), table)
    x = torch.full((1, 4, 64), MOST16, device="cuda", dtype=torch.float16)
    x[:, :, ::2] *= -1
    K.kv_paged_append(p, cache, x[:, :2], x[:, 2:])
    for got in rows(cache, table, 1):
        assert torch.equal(got, x[:, :2])


@pytest.mark.parametrize("blocks", [3, 1100])   # few wavefronts and many
@pytest.mark.parametrize("kept", ["i8", "fp8", "head"])
def test_the_ends_of_the_range(kept, blocks):
    """Every held number under scales around the range's end: float16 rows are the products in 32
    bits rounded, or +-65,504; NaN is NaN; bfloat16 rows hold them all."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    gen = torch.Generator().manual_seed(blocks)
    J, block, D, n = 2, 32, 128, blocks * 32 - 5
    codes = torch.randint(-127 if kept == "i8" else -128, 128, (blocks, J, block, D), generator=gen).to(torch.int8).cuda()
    turned = codes.flip(0).transpose(2, 3).contiguous()
    kind = torch.int8 if kept == "i8" else torch.float8_e4m3fn
    if kept == "head":
        scales = [torch.tensor([100.0, 700.0], device="cuda"), torch.tensor([146.3, 1e30], device="cuda")]
    else:
        scales = [torch.exp2(torch.rand(blocks, J, generator=gen) * 12 + 3).cuda() for _ in range(2)]
    cache = K.Cache(codes.view(kind), turned.view(kind), *scales, block_scales=kept != "head")
    table = torch.randperm(blocks, generator=gen).to(torch.int32).cuda()[None].contiguous()
    i32 = dict(dtype=torch.int32, device="cuda")
    p = K.Plan(1, 1, block, blocks, J, J, D)
    K.kv_paged_plan(p, torch.tensor([n], **i32), torch.zeros(1, **i32), table)
    page, at = table[0].long().repeat_interleave(block)[:n], torch.arange(n, device="cuda") % block
    for dtype in (torch.float16, torch.bfloat16):
        k, v = K.kv_paged_read(p, cache, torch.tensor([0, n], **i32), rows=n, dtype=dtype)
        for got, numbers, s in ((k, codes.view(kind).float()[page, :, at], scales[0]), (v, turned.view(kind).float()[page, :, :, at], scales[1])):
            want = numbers * (s[page] if kept != "head" else s[None])[:, :, None]
            assert bool((want.abs() > 65520.0).any()) and bool((want.abs() < 60000.0).any())
            if dtype == torch.float16:
                want = want.clamp(-MOST16, MOST16)
            assert torch.equal(torch.isnan(got), torch.isnan(want)) and bool(torch.isnan(want).any()) == (kept != "i8")
            number = ~torch.isnan(want)
            assert torch.equal(got[number], want[number].to(dtype))


# In units of 2^120, bfloat16's largest number is 255.  A first token of 254, then one of 255: the scale is doubled to 4, and 255
# is held as 64 units, 2^128.  In e4m3, after 240: 238 units, held as 240, 257 x 2^120.
@pytest.mark.parametrize("kept, before, held", [("i8", 254.0, 64.0), ("fp8", 240.0, 240.0)])
def test_finite_values_come_back_finite_in_bfloat16(kept, before, held):
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    kind, most = torch.int8 if kept == "i8" else torch.float8_e4m3fn, 255.0 * 2.0 ** 120
    kc, vc = torch.zeros(1, 1, 16, 64, device="cuda", dtype=kind), torch.zeros(1, 1, 64, 16, device="cuda", dtype=kind)
    cache = K.Cache(kc, vc, torch.zeros(1, 1, device="cuda"), torch.zeros(1, 1, device="cuda"), block_scales=True)
    table = torch.zeros(1, 1, **i32)
    p = K.Plan(1, 1, 16, 1, 1, 1, 64, max_new=1)
    for t, size in enumerate((before * 2.0 ** 120, most)):
        x = torch.zeros(1, 2, 64, device="cuda", dtype=torch.bfloat16)
        x[0, :, 3], x[0, :, 5] = size, -size
        K.kv_paged_plan(p, torch.tensor([t], **i32), torch.ones(1, **i32), table)
        K.kv_paged_append(p, cache, x[:, :1], x[:, 1:])
    assert kc[0, 0, 1, 3].float() == held and vc[0, 0, 5, 1].float() == -held
    # the last step's plan, one token in the cache and one new
    for got in K.kv_paged_read(p, cache, torch.tensor([0, 2], **i32), rows=2):
        assert got[1, 0, 3] == most and got[1, 0, 5] == -most and not got[1, 0, 6]
        assert bool(torch.isfinite(got).all())


def test_nan_and_large_scales_by_head_in_bfloat16():
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    codes = torch.arange(-128, 128, dtype=torch.int32).to(torch.int8).reshape(1, 1, 16, 16).repeat(1, 2, 1, 4).cuda()  # every e4m3 number
    kc, vc = codes.view(torch.float8_e4m3fn), codes.transpose(2, 3).contiguous().view(torch.float8_e4m3fn)
    scale = torch.tensor([1.0, 2.0 ** 121], device="cuda")
    p = K.Plan(1, 1, 16, 1, 2, 2, 64)
    K.kv_paged_plan(p, torch.tensor([16], **i32), torch.zeros(1, **i32), torch.zeros(1, 1, **i32))
    k, v = K.kv_paged_read(p, K.Cache(kc, vc, scale, scale), torch.tensor([0, 16], **i32), rows=16)
    want = (kc[0].float() * scale[:, None, None]).clamp(-255.0 * 2.0 ** 120, 255.0 * 2.0 ** 120).bfloat16().transpose(0, 1)
    for got in (k, v):
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and int(torch.isnan(got).sum()) == 2 * 2 * 4
        number = ~torch.isnan(want)
        assert torch.equal(got[number], want[number])
