"""Values that the paged-cache library cannot hold are refused before any device work."""
import pytest


@pytest.mark.parametrize("magnitude", [1e300, -1e39, 3.5e38, 1e-60, -1e-46])
def test_magnitudes_past_32_bits_are_refused(magnitude):
    """The kernels multiply in 32 bits: such a magnitude would be infinite or zero there."""
    from paper_2603_08739_amd import kvpaged as K
    with pytest.raises(K.KvError) as e:
        K.Rope(64, magnitude=magnitude)
    assert e.value.status == K.KV_ERR_INVALID and "magnitude" in str(e.value)
