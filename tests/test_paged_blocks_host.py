"""Caches of 8 bits with scales by block, and the read into rows, without a device: what
is refused before any device work, and the oracle by hand."""
import ctypes

import pytest

from tests.test_paged_host import batch, cache, refused, view


@pytest.mark.parametrize("dtype", ["KV_DT_FP8_BLOCK", "KV_DT_I8_BLOCK"])
@pytest.mark.parametrize("more, word", [
    (dict(k_scale=None), "scale arrays"), (dict(v_scale=None), "scale arrays"), (dict(k_scale=0x1002), "misaligned"), (dict(v=None), "NULL"),
    (dict(k_block_stride=2 * 16 * 64 + 8), "stride"), (dict(n_blocks=0), "n_blocks")])
def test_caches_are_refused(dtype, more, word):
    from paper_2603_08739_amd import kvpaged as K
    b, w = batch(K), view(K)
    c = cache(K, **{**dict(dtype=getattr(K, dtype), k_scale=0x1000, v_scale=0x1000), **more})
    refused(K, K.LIB.kv_paged_append(ctypes.byref(b), ctypes.byref(c), None, 0, w, w, w, w, None), word)
    refused(K, K.LIB.kv_paged_attention(ctypes.byref(b), ctypes.byref(c), 0, w, w, None, 1.0, None), word)
    refused(K, K.LIB.kv_paged_read(ctypes.byref(b), ctypes.byref(c), 0, 0x1000, None, 4, w, w, None), word)


@pytest.mark.parametrize("dtype", ["KV_DT_FP8_BLOCK", "KV_DT_I8_BLOCK"])
def test_one_scale_array_for_both_is_not_written(dtype):
    from paper_2603_08739_amd import kvpaged as K
    b, w = batch(K), view(K)
    c = cache(K, dtype=getattr(K, dtype), k_scale=0x1000, v_scale=0x1000)
    refused(K, K.LIB.kv_paged_append(ctypes.byref(b), ctypes.byref(c), None, 0, w, w, w, w, None), "same")


@pytest.mark.parametrize("kept", [-1, 3, 6, 1 << 31])
def test_unknown_types_are_refused(kept):
    from paper_2603_08739_amd import kvpaged as K
    b, c, w = batch(K), cache(K, dtype=kept & 0xffffffff, k_scale=0x1000, v_scale=0x1000), view(K)
    refused(K, K.LIB.kv_paged_read(ctypes.byref(b), ctypes.byref(c), 0, 0x1000, None, 4, w, w, None), "dtype")


def test_reads_are_refused():
    from paper_2603_08739_amd import kvpaged as K
    b, c, w = batch(K), cache(K), view(K)
    other = view(K, ptr=0x2000)

    def read(b=b, c=c, dtype=0, row_start=0x1000, first=None, rows=4, k=w, v=other):
        return K.LIB.kv_paged_read(b and ctypes.byref(b), c and ctypes.byref(c), dtype, row_start, first, rows, k, v, None)

    refused(K, read(b=None), "NULL")
    refused(K, read(c=None), "NULL")
    refused(K, read(b=batch(K, kv_len=None)), "NULL")
    refused(K, read(dtype=2), "dtype")
    refused(K, read(dtype=1), "dtype")
    refused(K, read(dtype=4), "dtype")
    refused(K, read(row_start=None), "row_start")
    refused(K, read(row_start=0x1002), "row_start")
    refused(K, read(first=0x1001), "first")
    refused(K, read(rows=1 << 31), "max_rows")
    refused(K, read(k=view(K, ptr=None)), "NULL")
    refused(K, read(v=view(K, ptr=0x1008)), "16-byte")
    refused(K, read(k=view(K, token=12)), "strides")
    refused(K, read(v=w), "same")
    assert read(rows=0) == K.KV_OK


def test_oracle_write_by_hand():
    import torch
    from oracle import paged as O
    # one head of one element; a block of 16 whose context ends at place 1
    numbers, scale = torch.zeros(2, 1, 16, 1, dtype=torch.float64), torch.zeros(2, 1, dtype=torch.float64)
    numbers[1, 0, 0], scale[1, 0] = 101.0, 0.5
    x = torch.tensor([[[127.0]], [[-3.0]]], dtype=torch.float64)
    assert O.write_blocks(x, numbers, scale, [[1]], [0, 2], [1], 16, 2, "i8") == [(1, 1), (1, 2)]
    # need 1 = 2 * 0.5: one rise; 101 / 2 is a tie and goes to the even 50
    assert scale[1, 0] == 1.0 and numbers[1, 0, :3, 0].tolist() == [50.0, 127.0, -3.0] and not numbers[0].any()
    rows = O.read_rows(numbers, scale, [[1]], [3], 16, 2, [0, 4], [0])
    assert rows[:, 0, 0].tolist() == [50.0, 127.0, -3.0, 0.0]


def test_oracle_rounding_is_the_held_types():
    import torch
    from oracle import paged as O
    x = torch.randn(4000, dtype=torch.float64, generator=torch.Generator().manual_seed(0)) * torch.exp2(torch.linspace(-14, 9, 4000, dtype=torch.float64))
    assert torch.equal(O.held(x, "fp8"), x.float().clamp(-448, 448).to(torch.float8_e4m3fn).double())
    assert torch.equal(O.held(x, "i8"), x.clamp(-127, 127).round().to(torch.int8).double())
    assert O.rises(1.0, 1.0) == 0 and O.rises(1.0000001, 1.0) == 1 and O.rises(16.0, 1.0) == 4 and O.rises(0.0, 1.0) == 0
