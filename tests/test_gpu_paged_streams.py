"""Paged-cache calls on a stream that is not the current one, outputs made by the call."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("as_handle", [False, True])
def test_outputs_do_not_take_memory_of_the_current_stream(as_handle):
    """Memory freed on the current stream, which may still be at work on it, is not what
    a call on another stream writes; the results are those of the current stream."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    kc, vc = torch.randn(64, 2, 16, 128, device="cuda", generator=g).bfloat16(), torch.randn(64, 2, 128, 16, device="cuda", generator=g).bfloat16()
    cache, rope = K.Cache(kc, vc), K.Rope(128)
    x = torch.randn(700, 8, 128, device="cuda", generator=g).bfloat16()
    pos = torch.arange(700, **i32)
    p = K.Plan(1, 700, 16, 64, 8, 2, 128)
    K.kv_paged_plan(p, torch.full((1,), 300, **i32), torch.full((1,), 700, **i32), torch.randperm(64, device="cuda", generator=g).to(torch.int32)[None])
    calls = [lambda **kw: K.kv_rope_apply(rope, x, pos, **kw), lambda **kw: K.kv_paged_attention(p, cache, x, **kw)]
    want = [call() for call in calls]
    side = torch.cuda.Stream()
    stream = side.cuda_stream if as_handle else side
    side.wait_stream(torch.cuda.current_stream())
    for call, ref in zip(calls, want):
        torch.cuda.synchronize()
        freed = [torch.empty_like(x) for _ in range(4)]
        addresses = {t.data_ptr() for t in freed}
        del freed
        out = call(stream=stream)
        assert out.data_ptr() not in addresses
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, ref)
        again = call(out=torch.empty_like(x))
        assert torch.equal(again, ref)
    rope.free()
