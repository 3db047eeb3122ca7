"""The rotation in automatic differentiation on the card, against the formula's gradient
in 64 bits.  A gradient is a rotation: products and their sum in 32 bits (2^-20 of the
pair's size, sines and cosines included) and one rounding to the type."""
import pytest

pytestmark = pytest.mark.gpu


def near(got, grad, pos, freq, interleaved, magnitude, backward):
    from oracle import paged as O
    from tests.paged import ROUND
    want = O.rope(grad, pos, freq, interleaved, magnitude, backward=backward)
    size = 2 * abs(magnitude) * grad.double().abs().amax(-1, keepdim=True)
    assert got.dtype == grad.dtype
    assert bool(((got.double() - want).abs() <= ROUND[got.dtype] * want.abs() + 2.0 ** -20 * size + 2.0 ** -24).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens, heads, dim, rot, interleaved", [(1, 1, 64, 64, 0), (37, 6, 128, 64, 1), (300, 8, 256, 256, 0), (5, 3, 80, 16, 1)])
def test_backward_pass(dtype, tokens, heads, dim, rot, interleaved):
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import TYPES
    g = torch.Generator(device="cuda").manual_seed(tokens)
    rope, freq = K.Rope(rot, base=500000.0, layout=interleaved, magnitude=1.25), O.frequencies(rot, 500000.0)
    fused = torch.randn(tokens, heads + 2, dim, device="cuda", generator=g).to(TYPES[dtype]).requires_grad_()
    pos = torch.randint(0, 131072, (tokens,), device="cuda", generator=g, dtype=torch.int32)
    w = torch.randn(tokens, heads, dim, device="cuda", generator=g).to(TYPES[dtype])
    for backward in (False, True):
        for how in ("made", "given", "in place", "inside"):
            fused.grad = None
            x = fused[:, 1:1 + heads]
            if how == "made":
                y = K.kv_rope_apply(rope, x, pos, backward=backward)
            elif how == "given":
                y = K.kv_rope_apply(rope, x, pos, out=torch.empty(tokens, heads, dim, device="cuda", dtype=x.dtype), backward=backward)
            elif how == "in place":
                y = x.clone()
                assert K.kv_rope_apply(rope, y, pos, out=y, backward=backward) is y
            else:  # its gradient comes at an odd address
                y = torch.cat([x.new_zeros(3), K.kv_rope_apply(rope, x, pos, backward=backward).flatten()])[3:].view(x.shape)
            near(y.detach(), x.detach(), pos, freq, interleaved, 1.25, backward)
            (y * w).sum().backward()
            near(fused.grad[:, 1:1 + heads], w, pos, freq, interleaved, 1.25, not backward)
            assert not bool(fused.grad[:, 0].any()) and not bool(fused.grad[:, 1 + heads:].any())
    rope.free()


def test_on_another_stream():
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    g = torch.Generator(device="cuda").manual_seed(2)
    rope, freq = K.Rope(64), O.frequencies(64, 10000.0)
    x = torch.randn(50, 4, 64, device="cuda", generator=g).half().requires_grad_()
    pos = torch.arange(50, device="cuda", dtype=torch.int32)
    w = torch.randn(50, 4, 64, device="cuda", generator=g).half()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        for given in (False, True):
            x.grad = None
            side.wait_stream(torch.cuda.current_stream())
            y = K.kv_rope_apply(rope, x, pos, out=torch.empty_like(w) if given else None, stream=stream)
            torch.cuda.synchronize()
            (y * w).sum().backward()
            torch.cuda.synchronize()
            near(y.detach(), x.detach(), pos, freq, 0, 1.0, False)
            near(x.grad, w, pos, freq, 0, 1.0, True)
    rope.free()
