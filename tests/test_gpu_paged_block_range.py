"""Attention with float16 queries over a cache with scales by block, near the end of the
type's range: what is held may be more than the values that were written, and more than
float16 holds."""
import pytest

pytestmark = pytest.mark.gpu

MOST16 = 65504.0


def answer(kept, code, scale, ctx, new, dim, edit=None, dtype="f16"):
    """Every value is the held number `code` (negative for odd elements) times `scale`."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import TYPES, blocks_of
    gen = torch.Generator().manual_seed(sum(ctx))
    H, J, block = 4, 2, 16
    table, n_blocks = blocks_of(ctx, new, block, gen)
    kind = torch.int8 if kept == "i8" else torch.float8_e4m3fn
    kc = torch.randint(-60, 60, (n_blocks, J, block, dim), generator=gen).float().cuda().to(kind)
    values = torch.full((n_blocks, J, dim, block), float(code), device="cuda")
    values[:, :, 1::2] *= -1
    ks, vs = torch.full((n_blocks, J), 0.02, device="cuda"), torch.full((n_blocks, J), scale, device="cuda")
    vc = values.to(kind)
    if edit:
        edit(vc, table)
    T = sum(new)
    p = K.Plan(len(ctx), T, block, table.shape[1], H, J, dim, max_new=max(new))
    i32 = dict(dtype=torch.int32, device="cuda")
    K.kv_paged_plan(p, torch.tensor(ctx, **i32), torch.tensor(new, **i32), table)
    q = torch.randn(T, H, dim, generator=gen).to(TYPES[dtype]).cuda()
    lse = torch.empty(T, H, device="cuda")
    out = K.kv_paged_attention(p, K.Cache(kc, vc, ks, vs, block_scales=True), q, lse=lse)
    assert bool(torch.isfinite(lse).all())
    return out


@pytest.mark.parametrize("kept, code, scale", [("i8", 101, 651.59), ("fp8", 384.0, 173.71), ("i8", 127, 3000.0)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("ctx, new", [([0, 40, 300], [1, 1, 1]), ([5000], [1]), ([0, 40], [70, 3]), ([3000], [40])])  # the last of each are cut and joined
def test_finite_values_give_finite_answers(kept, code, scale, dim, ctx, new):
    import torch
    out = answer(kept, code, scale, ctx, new, dim)
    want = torch.full_like(out, MOST16)
    want[..., 1::2] *= -1
    assert torch.equal(out, want)
    # bfloat16 holds it: off by its rounding and by that of the weights to float16
    out = answer(kept, code, scale, ctx, new, dim, dtype="bf16").float()
    assert bool((out.abs() - code * scale).abs().max() <= code * scale * (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -16))


@pytest.mark.parametrize("ctx, new", [([20], [1]), ([5000], [1]), ([0], [70]), ([3000], [40])])
def test_nan_stays(ctx, new):
    import torch

    def edit(vc, table):
        vc.view(torch.int8)[table[0, 0].item(), 0, 3, 0] = 0x7f

    out = answer("fp8", 384.0, 173.71, ctx, new, 64, edit=edit)
    assert bool(torch.isnan(out[:, :2, 3]).all()) and int(torch.isnan(out).sum()) == 2 * out.shape[0]
