"""The bounds of attention over caches with scales by block hold weights to float16's rounding:
tried on the definition itself, without a device."""
import pytest
import torch

from tests import paged_block as B
from tests.test_paged_block_bounds_host import KINDS, attention


@pytest.mark.parametrize("dtype, kept", KINDS)
def test_weights_of_8_bits_fail(dtype, kept):
    """The weights are rounded to float16 whatever the queries' type; rounded to bfloat16 they are outside."""
    out, lse, want, limits = attention(dtype, kept, torch.float16)
    assert B.off_by(out, lse, want, limits) <= 1.0
    out, lse, want, limits = attention(dtype, kept, torch.bfloat16)
    assert B.off_by(out, lse, want, limits) > 1.0
