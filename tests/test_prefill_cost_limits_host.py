"""Arguments that the measured prefill cost refuses, without a device."""
import pytest

import tracegen as tg


@pytest.mark.parametrize("n", [0, -1])
def test_no_requests_are_refused(n):
    from paper_2603_08739_amd import prefill_cost as P
    with pytest.raises(ValueError, match="max_requests"):
        P.measure(tg.tiny(n_req=3), 100, max_requests=n)
