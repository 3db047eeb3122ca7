"""Scales of blocks that no query of a request sees change nothing, whatever they hold."""
import pytest

from tests import paged_block as B

pytestmark = pytest.mark.gpu

KINDS = [("bf16", "i8"), ("f16", "i8"), ("bf16", "fp8"), ("f16", "fp8")]
INF, NAN = float("inf"), float("nan")


def compare(ctx, new, block, heads, dim, dtype, kept, window, max_new=None, drop=()):
    """Once with ordinary scales everywhere, then with huge ones, infinities and NaN where nobody looks: the same
    bits, within the bound that the seen scales alone give."""
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import TYPES, blocks_of, held_cache
    gen = torch.Generator().manual_seed(sum(ctx) + 3 * sum(new) + window)
    H, J = heads
    table, n_blocks = blocks_of(ctx, new, block, gen)
    if drop:  # block 0, whose scale is read in a missing one's place, is nobody's
        table[table == 0] = table[drop[0]].clone()
    for r, col in drop:
        table[r, col] = -1
    kc, vc, ks, vs = held_cache(n_blocks, J, block, dim, kept, gen)
    t, seen = table.tolist(), set()
    for r, (c, n) in enumerate(zip(ctx, new)):
        seen |= {t[r][p // block] for p in range(max(0, c + 1 - window) if window else 0, c + n)}
    unseen = sorted(set(range(n_blocks)) - seen)
    assert unseen
    total = sum(new)
    q = (torch.randn(total, H, dim, generator=gen) * (1 + torch.rand(H, 1, generator=gen))).to(TYPES[dtype]).cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    p = K.Plan(len(ctx), total, block, table.shape[1], H, J, dim, max_new=max_new, window=window)
    K.kv_paged_plan(p, torch.tensor(ctx, **i32), torch.tensor(new, **i32), table)
    starts = p.q_start.tolist()
    want = O.attention(q, kc.double() * ks.double()[:, :, None, None], vc.double() * vs.double()[:, :, None, None], t, starts, ctx, block, n_blocks, dim ** -0.5, window)
    limits = B.bound(want, q.dtype, dim, kept, B.largest_seen(vs, t, starts, ctx, block, window, H), min(window or 1 << 30, max(c + n for c, n in zip(ctx, new))))
    results = []
    for strange in (None, (1e38, 1e38), (NAN, 1e38), (1e38, NAN), (INF, INF)):
        k_scale, v_scale = ks.clone(), vs.clone()
        if strange:
            k_scale[unseen], v_scale[unseen] = strange
        out, lse = torch.empty_like(q), torch.empty(total, H, device="cuda")
        K.kv_paged_attention(p, K.Cache(kc, vc, k_scale, v_scale, block_scales=True), q, out=out, lse=lse)
        results.append((out, lse))
    worst = B.off_by(*results[0], want, limits)
    assert worst <= 1.0, worst
    for out, lse in results[1:]:
        assert torch.equal(out.view(torch.int16), results[0][0].view(torch.int16)) and torch.equal(lse.view(torch.int32), results[0][1].view(torch.int32))


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("max_new", [1, 4, None])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_outside_every_window(dtype, kept, max_new, dim):
    new = [min(max_new, n) if max_new else n for n in (1, 4, 30, 70)]
    compare([137, 110, 200, 90], new, 16, (4, 2), dim, dtype, kept, 40, max_new=max_new)


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("max_new", [1, None])
@pytest.mark.parametrize("block", [16, 64, 256])
def test_blocks_of_nobody_and_missing_ones(dtype, kept, max_new, block):
    new = [1, 1, 1] if max_new else [20, 140, 1]
    compare([5 * block, 3 * block + 7, 9], new, block, (8, 2), 64, dtype, kept, 0, max_new=max_new, drop=[(0, 0), (0, 3), (1, 1)])


@pytest.mark.parametrize("dtype, kept", KINDS)
def test_long_contexts_cut_in_pieces(dtype, kept):
    compare([4000], [1], 16, (4, 1), 128, dtype, kept, 1500, max_new=1)
    compare([4000], [40], 64, (4, 1), 64, dtype, kept, 1500)
