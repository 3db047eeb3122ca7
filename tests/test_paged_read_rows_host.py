"""The number of rows that a read is asked for, without a device: none that the row tensors do not
have reaches the library, whose field for it has 32 bits."""
import pytest
import torch

from tests.test_paged_binding_host import binding, on_gpu, plan_for, step  # noqa: F401


@pytest.mark.parametrize("rows", [-1, -(1 << 31), 4 - (1 << 32), 9 - (1 << 33), 9, (1 << 32) + 2])
def test_rows_that_are_not_there_are_refused(binding, rows):  # noqa: F811
    K, lib = binding
    f16, i32 = dict(dtype=torch.float16), dict(dtype=torch.int32)
    p = plan_for(K)
    K.kv_paged_plan(p, *step())
    cache = K.Cache(on_gpu(torch.zeros(3, 2, 16, 64, **f16)), on_gpu(torch.zeros(3, 2, 64, 16, **f16)))
    k, v = (on_gpu(torch.zeros(8, 2, 64, **f16)) for _ in range(2))
    start, n = on_gpu(torch.zeros(3, **i32)), len(lib.calls)
    with pytest.raises(ValueError, match="rows|shape"):
        K.kv_paged_read(p, cache, start, k=k, v=v, rows=rows)
    if rows < 0:
        with pytest.raises(ValueError, match="rows"):
            K.kv_paged_read(p, cache, start, rows=rows)
    assert len(lib.calls) == n
    for good in (0, 3, 8, None):
        K.kv_paged_read(p, cache, start, k=k, v=v, rows=good)
        assert lib.calls[-1][1][5] == (8 if good is None else good)
