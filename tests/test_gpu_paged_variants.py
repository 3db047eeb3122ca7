"""Variants of the attention kernels with layouts of their own: windows with heads of 256,
8-bit tiles in every block size, masked values that are not finite with heads of 256."""
import pytest

from tests.test_gpu_paged_attention import KINDS, case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, kept", KINDS)
@pytest.mark.parametrize("window", [1, 33, 64, 200])
def test_windows_with_heads_of_256(dtype, kept, window):
    case([0, 300, 65, 1], [40, 137, 1, 3], 16, (4, 2), 256, dtype, kept, window=window)
    case([0, 300, 65, 1], [1, 1, 1, 1], 16, (4, 2), 256, dtype, kept, window=window, max_new=1)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("block", [16, 32, 64, 128, 256])
def test_8_bit_tiles_in_every_block_size(dtype, dim, block):
    ctx, new = [0, 300, 17, 255, 256], [140, 33, 64, 2, 1]
    case(ctx, new, block, (4, 2), dim, dtype, "fp8")
    case(ctx, new, block, (4, 2), dim, dtype, "fp8", window=70)
    case(ctx, [1] * 5, block, (4, 2), dim, dtype, "fp8", max_new=1)


@pytest.mark.parametrize("kept", ["f16", "bf16", "fp8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("block", [16, 64])
@pytest.mark.parametrize("max_new", [1, 2, None])
def test_not_finite_in_masked_places(kept, dim, block, max_new):
    """Past the requests' ends, in blocks that nobody has, and in values that some queries
    of a request see and others do not."""
    import torch
    new = [min(max_new, n) if max_new else n for n in (1, 2, 40, 150)]
    ctx = [37, 70, 100, 0]
    nan, inf = (0x7f, 0x7f) if kept == "fp8" else (float("nan"), float("inf"))

    def edit(kc, vc, table):
        bits = (lambda x: x.view(torch.int8)) if kept == "fp8" else (lambda x: x)
        t = table.tolist()
        for r in range(4):
            for j in range(ctx[r] + new[r], len(t[r]) * block):
                if t[r][j // block] >= 0:
                    bits(kc)[t[r][j // block], :, j % block] = nan
                    bits(vc)[t[r][j // block], :, :, j % block] = inf if j % 2 else nan
        for p in set(range(kc.shape[0])) - {p for row in t for p in row}:
            bits(kc)[p] = nan
            bits(vc)[p] = nan
        for r, head, element, what in ((3, 0, dim - 1, nan), (2, 1, 5, inf), (2, 1, dim // 2 + 1, nan), (3, 1, 40, inf)):
            j = ctx[r] + new[r] // 2
            bits(vc)[t[r][j // block], head, element, j % block] = what

    dtype = "f16" if kept == "f16" else "bf16"
    case(ctx, new, block, (4, 2), dim, dtype, kept, max_new=max_new, edit=edit)
    case(ctx, new, block, (4, 2), dim, dtype, kept, max_new=max_new, edit=edit, window=6)
