"""Scale arrays of a cache with scales by block that overlap are not written: the workgroups of
keys and of values would race for what they share.  Without a device."""
import ctypes

import pytest

from tests.test_paged_host import batch, cache, refused, view

BYTES = 4 * 4 * 2  # [n_blocks 4][kv_heads 2] float32


def append(K, **more):
    b, w = batch(K), view(K)
    c = cache(K, **more)
    # (keys that are not there, so that no call gets past the checks)
    return K.LIB.kv_paged_append(ctypes.byref(b), ctypes.byref(c), None, 0, w, w, view(K, ptr=None), w, None)


@pytest.mark.parametrize("dtype", ["KV_DT_FP8_BLOCK", "KV_DT_I8_BLOCK"])
@pytest.mark.parametrize("apart", [0, 4, -4, BYTES - 4, 4 - BYTES])
def test_overlapping_scale_arrays_are_refused(dtype, apart):
    from paper_2603_08739_amd import kvpaged as K
    refused(K, append(K, dtype=getattr(K, dtype), k_scale=0x100000, v_scale=0x100000 + apart), "scale", "overlap")


@pytest.mark.parametrize("dtype", ["KV_DT_FP8_BLOCK", "KV_DT_I8_BLOCK"])
@pytest.mark.parametrize("apart", [BYTES, -BYTES, 1 << 20])
def test_arrays_side_by_side_are_not(dtype, apart):
    """They pass: the call is refused for what is looked at next, keys that are not there."""
    from paper_2603_08739_amd import kvpaged as K
    refused(K, append(K, dtype=getattr(K, dtype), k_scale=0x100000, v_scale=0x100000 + apart), "view", "NULL")


def test_scales_by_head_may_be_one():
    from paper_2603_08739_amd import kvpaged as K
    refused(K, append(K, dtype=K.KV_DT_FP8, k_scale=0x100000, v_scale=0x100000), "view", "NULL")
