"""Inputs and bounds shared by the GPU tests of the paged-cache operators."""
import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}
# unit roundoff: half the spacing of the type's numbers relative to the number
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def blocks_of(ctx, new, block, gen, spare=3, max_blocks=None):
    """Every request's blocks from a shuffled pool: (table [R, max_blocks] int32 on the
    GPU with -1 elsewhere, number of blocks of the cache)."""
    need = [-(-(c + n) // block) for c, n in zip(ctx, new)]
    total = sum(need) + spare
    pool = torch.randperm(total, generator=gen).to(torch.int32)
    table = torch.full((len(ctx), max_blocks or max(max(need), 1)), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = pool[at:at + n]
        at += n
    return table.cuda(), total


def cache_values(n_blocks, heads, block, dim, kind, gen):
    """k, v and their scales (8-bit caches)."""
    shape = (n_blocks, heads, block, dim)
    k, v = torch.randn(*shape, generator=gen), torch.randn(n_blocks, heads, dim, block, generator=gen)
    if kind != "fp8":
        return k.to(TYPES[kind]).cuda(), v.to(TYPES[kind]).cuda(), None, None
    ks, vs = torch.rand(heads, generator=gen) * 0.02 + 0.02, torch.rand(heads, generator=gen) * 0.02 + 0.02
    to8 = lambda x, s: (x / s[:, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).cuda()  # noqa: E731
    return to8(k, ks), to8(v, vs), ks.cuda(), vs.cuda()


def check_attention(got, lse, want, q):
    """got, lse against the oracle's (out, lse, spread, reach).

    Bounds.  A score is a sum of D products with 32-bit sums, so it is off by at most
    (D + 8) 2^-24 reach (the 8 covers the scale's product, the subtraction of the
    maximum and the exponential); weights and their sum are both off by that much
    relatively, and by 2^-20 for exponentials and sums of weights.  A weight is
    rounded to q's type on its way into the second product: at most u of the weight.
    The result is rounded once more."""
    out, ref_lse, spread, reach = want
    u = ROUND[q.dtype]
    e = 2 * (q.shape[-1] + 8) * 2.0 ** -24 * reach + 2.0 ** -20
    got64 = got.double()
    fine = torch.isfinite(out)
    assert torch.equal(torch.isnan(got64), torch.isnan(out))
    rest = ~fine & ~torch.isnan(out)
    assert torch.equal(got64[rest], out[rest])
    bound = (u + e[..., None]) * spread + u * out.abs() + 2.0 ** -24
    worst = ((got64 - out).abs() / bound)[fine]
    assert worst.numel() == 0 or float(worst.max()) <= 1.0, float(worst.max())
    if lse is not None:
        l64 = lse.double()
        fine = torch.isfinite(ref_lse)
        assert torch.equal(torch.isnan(l64), torch.isnan(ref_lse))
        rest = ~fine & ~torch.isnan(ref_lse)
        assert torch.equal(l64[rest], ref_lse[rest])
        bad = ((l64 - ref_lse).abs() > e + 2.0 ** -21 * ref_lse.abs())[fine]
        assert not bool(bad.any())


def held_cache(n_blocks, heads, block, dim, kind, gen):
    """k, v of 8 bits and their scales [n_blocks, heads], as a cache that was written to has
    them: the whole range of numbers, blocks of different sizes."""
    most = {"i8": 127.0, "fp8": 448.0}[kind]

    def numbers(*shape):
        x = (torch.randn(*shape, generator=gen) * (most / 4)).clamp(-most, most)
        return (x.round().to(torch.int8) if kind == "i8" else x.to(torch.float8_e4m3fn)).cuda()

    scales = [(torch.rand(n_blocks, heads, generator=gen) * 3 + 1) / most for _ in range(2)]
    return numbers(n_blocks, heads, block, dim), numbers(n_blocks, heads, dim, block), scales[0].cuda(), scales[1].cuda()
