"""Attention over caches with scales by block: weights are rounded to float16 whatever the
queries' type, which is closer than bfloat16 queries' own type would be."""
import pytest

from tests import paged_block as B

pytestmark = pytest.mark.gpu

KINDS = [("bf16", "i8"), ("f16", "i8"), ("bf16", "fp8"), ("f16", "fp8")]


def case(ctx, new, block, heads, dim, dtype, kept, window=0, max_new=None):
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import TYPES, blocks_of, held_cache
    gen = torch.Generator().manual_seed(dim + sum(ctx))
    H, J = heads
    table, n_blocks = blocks_of(ctx, new, block, gen)
    kc, vc, ks, vs = held_cache(n_blocks, J, block, dim, kept, gen)
    total = sum(new)
    q = (torch.randn(total, H, dim, generator=gen) * (1 + torch.rand(H, 1, generator=gen))).to(TYPES[dtype]).cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    p = K.Plan(len(ctx), total, block, table.shape[1], H, J, dim, max_new=max_new, window=window)
    K.kv_paged_plan(p, torch.tensor(ctx, **i32), torch.tensor(new, **i32), table)
    out, lse = torch.empty_like(q), torch.empty(total, H, device="cuda")
    K.kv_paged_attention(p, K.Cache(kc, vc, ks, vs, block_scales=True), q, out=out, lse=lse)
    t, starts = table.tolist(), p.q_start.tolist()
    want = O.attention(q, kc.double() * ks.double()[:, :, None, None], vc.double() * vs.double()[:, :, None, None], t, starts, ctx, block, n_blocks, dim ** -0.5, window)
    keys = min(window or 1 << 30, max(c + n for c, n in zip(ctx, new)))
    worst = B.off_by(out, lse, want, B.bound(want, q.dtype, dim, kept, B.largest_seen(vs, t, starts, ctx, block, window, H), keys))
    assert worst <= 1.0, worst


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads", [(8, 2), (32, 1), (64, 1)])
def test_few_rows(dtype, kept, dim, heads):
    case([0, 1, 15, 16, 33, 64, 127, 300], [1] * 8, 16, heads, dim, dtype, kept, max_new=1)


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_tiles(dtype, kept, dim):
    case([0, 100, 17, 63], [130, 33, 1, 64], 16, (8, 2), dim, dtype, kept)
    case([200, 5], [70, 140], 64, (6, 3), dim, dtype, kept, window=50)


@pytest.mark.parametrize("dtype, kept", KINDS)
def test_joined_pieces(dtype, kept):
    case([3000, 1], [1, 1], 16, (8, 1), 128, dtype, kept, max_new=1)
    case([3000], [40], 64, (4, 1), 64, dtype, kept)
