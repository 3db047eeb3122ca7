"""The read's tested shapes reach the form of the kernel that they are there for, for caches of
either width."""
import pytest

from tests import paged_read as R


@pytest.mark.parametrize("name", R.SHAPES)
@pytest.mark.parametrize("bytes_each", [1, 2])
def test_shapes_reach_their_form(name, bytes_each):
    block, dim, heads, n_req, most, few = R.SHAPES[name]
    rows = sum(R.lengths(n_req, most, 0))
    for n in (rows, rows - 20, rows + 6):
        assert R.few_wavefronts(n_req, n, block, heads, dim, bytes_each) == few


def test_both_sides_of_the_border():
    assert R.few_wavefronts(1, 16352, 16, 2, 64, 1) and not R.few_wavefronts(1, 16353, 16, 2, 64, 1)
