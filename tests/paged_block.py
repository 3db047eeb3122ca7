"""Bounds for attention over caches with scales by block, for the GPU tests and for the CPU test
that tries them on wrong answers."""
import torch

from tests.paged import ROUND

MOST = {"i8": 127.0, "fp8": 448.0}


def largest_seen(vs, table, q_start, ctx, block, window, heads):
    """[T, heads]: the largest value scale in the blocks that the queries of a token's request see; lists
    but for vs [n_blocks, kv_heads]."""
    n_blocks, J = vs.shape
    out = torch.zeros(q_start[-1], heads, dtype=torch.float64, device=vs.device)
    for r in range(len(ctx)):
        first, end = q_start[r], q_start[r + 1]
        if first == end:
            continue
        low = max(0, ctx[r] + 1 - window) if window else 0
        pages = [table[r][c] for c in range(low // block, (ctx[r] + end - first - 1) // block + 1) if 0 <= table[r][c] < n_blocks]
        if pages:
            out[first:end] = vs[pages].double().amax(0).repeat_interleave(heads // J)
    return out


def bound(want, dtype, dim, kept, seen, keys, spread=0):
    """How far (out, lse) may be from the oracle's (out, lse, spread, reach): `seen` as largest_seen() gives
    it, `keys` the most that a query sees, values' scales apart by up to 2^spread.

    A score is a sum of dim products with 32-bit sums, off by at most (dim + 8) 2^-24 reach; weights and their
    sum are both off by that, and by 2^-20 for exponentials and sums.  A weight's scale is the exponential
    of a logarithm of at most spread + 8 in 32 bits, and the exponent is rounded where its parts meet: 2^-22 of
    spread + 8 + reach.  A weight is rounded to float16, whatever the queries' type: 2^-11 of it, or, where it is below
    the normal numbers, 2^-25 where 2^6 is the largest's: 2^-31 of the largest seen scale, for every key.
    The result is rounded once, to the queries' type (float16: 2^-25 below its normal numbers)."""
    out, lse, size, reach = want
    e = 2 * (dim + 8) * 2.0 ** -24 * reach + 2.0 ** -20 + 2.0 ** -22 * (spread + 8 + reach)
    small = 2.0 ** -31 * MOST[kept] * seen * keys
    return (2.0 ** -11 + e[..., None]) * size + small[..., None] + ROUND[dtype] * out.abs() + 2.0 ** -25, e + 2.0 ** -21 * lse.abs()


def off_by(got, lse, want, bounds):
    """The largest error in units of its bound; everything finite, but for rows that see nothing."""
    nothing = torch.isinf(want[1])
    assert torch.equal(lse.double()[nothing], want[1][nothing]) and not got[nothing].any()
    a = ((got.double() - want[0]).abs() / bounds[0])[~nothing]
    b = ((lse.double() - want[1]).abs() / bounds[1])[~nothing]
    return max(float(torch.nan_to_num(x, nan=float("inf")).max()) if x.numel() else 0.0 for x in (a, b))
