"""The bounds of attention over caches with scales by block have to fail wrong answers: tried
on the definition itself, without a device."""
import pytest
import torch

from oracle import paged as O
from tests import paged_block as B

KINDS = [("bf16", "i8"), ("f16", "i8"), ("bf16", "fp8"), ("f16", "fp8")]


def attention(dtype, kept, round_weights=None, huge=True, window=40):
    """A step over a cache whose unseen blocks have scales of 1e38: (out, lse) as a kernel would round them, the
    oracle's answer and the bounds.  round_weights: what the weights are rounded to on their way into the second product,
    relative to the largest at 2^6."""
    gen = torch.Generator().manual_seed(4)
    block, J, H, D, ctx, new = 16, 2, 4, 64, [137, 110], [1, 30]
    need = [-(-(c + n) // block) for c, n in zip(ctx, new)]
    n_blocks = sum(need) + 3
    pool = torch.randperm(n_blocks, generator=gen).tolist()
    table = [pool[:need[0]] + [-1] * (max(need) - need[0]), pool[need[0]:sum(need)] + [-1] * (max(need) - need[1])]
    most = B.MOST[kept]
    numbers = [O.held(torch.randn(*s, generator=gen).double() * most / 4, kept) for s in ((n_blocks, J, block, D), (n_blocks, J, D, block))]
    ks, vs = (((torch.rand(n_blocks, J, generator=gen) * 3 + 1) / most).double() for _ in range(2))
    seen = {table[r][p // block] for r in range(2) for p in range(max(0, ctx[r] + 1 - window), ctx[r] + new[r])}
    if huge:
        vs[[p for p in range(n_blocks) if p not in seen]] = 1e38
    starts = [0, 1, 31]
    q = torch.randn(31, H, D, generator=gen).to({"bf16": torch.bfloat16, "f16": torch.float16}[dtype])
    k, v = (x * s[:, :, None, None] for x, s in zip(numbers, (ks, vs)))
    want = O.attention(q, k, v, table, starts, ctx, block, n_blocks, D ** -0.5, window)
    out = want[0].clone()
    if round_weights:
        for r in range(2):
            for t in range(starts[r], starts[r + 1]):
                p = ctx[r] + t - starts[r]
                keys = list(range(max(0, p - window + 1), p + 1))
                page, at = torch.tensor([table[r][j // block] for j in keys]), torch.tensor([j % block for j in keys])
                unit = 2.0 ** torch.floor(torch.log2(vs[list(seen)].amax(0)))
                for h in range(H):
                    j = h // (H // J)
                    w = torch.exp(D ** -0.5 * k[page, j, at] @ q[t, h].double())
                    w = 64.0 * w / w.max()
                    rounded = (w * vs[page, j] / unit[j]).to(round_weights).double() * unit[j]
                    out[t, h] = rounded @ numbers[1][page, j, :, at] / w.sum()
    limits = B.bound(want, q.dtype, D, kept, B.largest_seen(vs, table, starts, ctx, block, window, H), window)
    return out.to(q.dtype), want[1].float(), want, limits


@pytest.mark.parametrize("dtype, kept", KINDS)
def test_wrong_answers_fail(dtype, kept):
    out, lse, want, limits = attention(dtype, kept)
    assert B.off_by(out, lse, want, limits) <= 1.0
    for wrong in (torch.zeros_like(out), -out, torch.full_like(out, 1e4), out * 1.01, torch.full_like(out, float("nan"))):
        assert B.off_by(wrong, lse, want, limits) > 1.0
    for wrong in (lse + 1e-3, lse * 1.001, torch.full_like(lse, float("nan"))):
        assert B.off_by(out, wrong, want, limits) > 1.0
