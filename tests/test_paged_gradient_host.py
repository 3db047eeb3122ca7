"""The rotation in automatic differentiation, without a device: the library's call is
played by the formula on host memory, at the addresses and strides it is given."""
import ctypes

import pytest
import torch

from tests.test_paged_binding_host import Recorder, on_gpu

ROT, TURNS = 16, 0.37


def formula(x, pos, backward):
    a, b = x[..., :ROT // 2].float(), x[..., ROT // 2:ROT].float()
    angle = pos[:, None, None].float() * TURNS * (-1.0 if backward else 1.0)
    c, s = torch.cos(angle), torch.sin(angle)
    return torch.cat([a * c - b * s, a * s + b * c, x[..., ROT:].float()], -1).to(x.dtype)


class Library(Recorder):
    def kv_rope_apply(self, handle, dtype, vx, vy, pos, n, heads, dim, backward, stream):
        if handle is None:
            return -1
        assert vx.ptr % 16 == 0 and vy.ptr % 16 == 0 and not (vx.token_stride | vx.head_stride | vy.token_stride | vy.head_stride) % 8

        def at(v):
            many = (n - 1) * v.token_stride + (heads - 1) * v.head_stride + dim
            raw = torch.frombuffer((ctypes.c_uint16 * many).from_address(v.ptr), dtype=torch.float16)
            return raw.as_strided((n, heads, dim), (v.token_stride, v.head_stride, 1))
        p = torch.frombuffer((ctypes.c_int32 * n).from_address(pos), dtype=torch.int32)
        at(vy).copy_(formula(at(vx).clone(), p, backward))
        self.calls.append(("kv_rope_apply", (backward, stream)))
        return 0


@pytest.fixture
def binding(monkeypatch):
    from paper_2603_08739_amd import kvpaged as K
    lib = Library(K)
    monkeypatch.setattr(K, "LIB", lib)
    monkeypatch.setattr(K, "_device", lambda: 0)
    monkeypatch.setattr(K, "_raw_stream", lambda dev: 70)
    # host tensors pass for device ones wherever autograd makes them
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    rope = K.Rope.__new__(K.Rope)
    rope.handle = 5
    yield K, lib, rope
    rope.handle = None


def data(n=6, heads=2, dim=32, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(n, heads, dim, generator=g).half(), torch.randint(0, 50, (n,), generator=g, dtype=torch.int32), torch.randn(n, heads, dim, generator=g).half()


def test_an_input_that_needs_a_gradient_gets_one(binding):
    K, lib, rope = binding
    for turned_back in (False, True):
        x, pos, w = data()
        x.requires_grad_()
        y = K.kv_rope_apply(rope, x, pos, backward=turned_back)
        assert y.requires_grad and torch.equal(y.detach(), formula(x.detach(), pos, turned_back))
        (y * w).sum().backward()
        assert torch.equal(x.grad, formula(w, pos, not turned_back))
        assert [c[1][0] for c in lib.calls[-2:]] == [int(turned_back), int(not turned_back)]


def test_gradients_at_any_stride_and_address(binding):
    K, lib, rope = binding
    x, pos, w = data()
    x.requires_grad_()
    K.kv_rope_apply(rope, x, pos).sum().backward()                       # one number, expanded
    assert torch.equal(x.grad, formula(torch.ones_like(w), pos, True))
    x.grad = None
    y = K.kv_rope_apply(rope, x, pos)
    (torch.cat([torch.zeros(3).half(), y.flatten()])[3:] * w.flatten()).sum().backward()   # inside another tensor
    assert torch.equal(x.grad, formula(w, pos, True))
    x.grad = None
    (K.kv_rope_apply(rope, x, pos).permute(2, 1, 0) * w.permute(2, 1, 0)).sum().backward()
    assert torch.equal(x.grad, formula(w, pos, True))


def test_heads_of_a_fused_projection(binding):
    """The gradient of a strided view goes where the view lies."""
    K, lib, rope = binding
    g = torch.Generator().manual_seed(5)
    fused = torch.randn(6, 5, 32, generator=g).half().requires_grad_()
    _, pos, w = data()
    (K.kv_rope_apply(rope, fused[:, 1:3], pos) * w).sum().backward()
    want = torch.zeros_like(fused)
    want[:, 1:3] = formula(w, pos, True)
    assert torch.equal(fused.grad, want)


def test_given_outputs_carry_the_gradient(binding):
    K, lib, rope = binding
    x, pos, w = data()
    x.requires_grad_()
    out = torch.full((8, 2, 32), 3.0).half()      # two rows more than tokens
    assert K.kv_rope_apply(rope, x, pos, out=out) is out
    assert torch.equal(out.detach()[:6], formula(x.detach(), pos, False)) and bool((out.detach()[6:] == 3.0).all())
    (out[:6] * w).sum().backward()
    assert torch.equal(x.grad, formula(w, pos, True))
    x.grad = None
    q = x * 2
    assert K.kv_rope_apply(rope, q, pos, out=q) is q                     # in place
    assert torch.equal(q.detach(), formula(2 * x.detach(), pos, False))
    (q * w).sum().backward()
    assert torch.equal(x.grad, 2 * formula(w, pos, True))


def test_nothing_is_recorded_without_a_need(binding):
    K, lib, rope = binding
    x, pos, w = data()
    out = torch.empty_like(x)
    assert not K.kv_rope_apply(rope, x, pos).requires_grad and K.kv_rope_apply(rope, x, pos, out=out) is out and not out.requires_grad
    x.requires_grad_()
    with torch.no_grad():
        assert not K.kv_rope_apply(rope, x, pos).requires_grad and not K.kv_rope_apply(rope, x, pos, out=out).requires_grad
        K.kv_rope_apply(rope, x, pos, out=x)
    assert len(lib.calls) == 5


def test_a_gradient_of_the_gradient(binding):
    K, lib, rope = binding
    x, pos, w = data()
    x.requires_grad_()
    w.requires_grad_()
    grad, = torch.autograd.grad((K.kv_rope_apply(rope, x, pos) * w).sum(), x, create_graph=True)
    (grad * x.detach()).sum().backward()
    assert torch.equal(w.grad, formula(x.detach(), pos, False))


def test_a_rotation_freed_too_early_is_refused(binding):
    K, lib, rope = binding
    x, pos, w = data()
    y = K.kv_rope_apply(rope, x.requires_grad_(), pos)
    rope.handle, kept = None, rope.handle
    with pytest.raises(K.KvError):
        y.sum().backward()
    rope.handle = kept
