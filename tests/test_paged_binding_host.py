"""The paged-cache binding without a device: what a refused call leaves behind, what it
checks and where it allocates.  Tensors lie on the host and say that they are on a GPU;
the library is a recorder that refuses when told to."""
import pytest
import torch


class OnGpu(torch.Tensor):
    """A host tensor that passes for one on GPU `dev`."""
    dev = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.dev


def on_gpu(t, dev=0):
    x = torch.Tensor._make_subclass(OnGpu, t)
    x.dev = dev
    return x


class Recorder:
    """Stands in for the library: keeps the calls, answers with `status`."""

    def __init__(self, K):
        self.calls, self.status, self.real = [], K.KV_OK, K.LIB

    def __getattr__(self, name):
        if name in ("kv_paged_work_bytes", "kv_last_error"):
            return getattr(self.real, name)

        def call(*args):
            self.calls.append((name, args))
            return self.status
        return call


@pytest.fixture
def binding(monkeypatch):
    from paper_2603_08739_amd import kvpaged as K
    lib = Recorder(K)
    monkeypatch.setattr(K, "LIB", lib)
    monkeypatch.setattr(K, "_device", lambda: 0)
    monkeypatch.setattr(K, "_raw_stream", lambda dev: 70 + dev)
    return K, lib


def step(n_free=3):
    i32 = dict(dtype=torch.int32)
    return [on_gpu(torch.zeros(*s, **i32)) for s in ((2,), (2,), (2, 4), (n_free,))]


def plan_for(K):
    p = K.Plan(2, 8, 16, 4, 4, 2, 64, device="cpu")
    for name in ("q_start", "kv_len", "slot", "pos", "result", "work"):
        setattr(p, name, on_gpu(getattr(p, name)))
    p.dev = 0
    return p


def aim(p):
    b = p.batch
    return b.ctx_len, b.new_len, b.table, b.n_free, b.free_list


@pytest.mark.parametrize("at, bad", [
    (0, lambda t: t.long()), (1, lambda t: t[:1]), (2, lambda t: t[:1]), (2, lambda t: t[:, :3].contiguous()), (2, lambda t: t.T),
    (3, lambda t: t.long()), (3, lambda t: torch.zeros(6, dtype=torch.int32)[::2])])
def test_a_refused_plan_leaves_the_earlier_one(binding, at, bad):
    """The batch goes on pointing at the step that was planned, whose tensors are kept
    alive; never at a refused one's, which nobody keeps."""
    K, lib = binding
    p, first = plan_for(K), step()
    K.kv_paged_plan(p, *first)
    before = aim(p)
    assert before[:3] == tuple(t.data_ptr() for t in first[:3]) and before[3:] == (3, first[3].data_ptr())
    second = step(5)
    second[at] = on_gpu(bad(second[at]))
    with pytest.raises(ValueError):
        K.kv_paged_plan(p, *second)
    assert aim(p) == before and len(lib.calls) == 1
    assert all(a is b for a, b in zip(p.inputs, first))


def test_a_plan_that_the_library_refuses_leaves_the_earlier_one(binding):
    K, lib = binding
    p, first = plan_for(K), step()
    lib.status = K.KV_ERR_INVALID
    with pytest.raises(K.KvError):
        K.kv_paged_plan(p, *first)
    assert aim(p) == (None, None, None, 0, None) and p.inputs is None
    lib.status = K.KV_OK
    K.kv_paged_plan(p, *first)
    before = aim(p)
    lib.status = K.KV_ERR_INVALID
    with pytest.raises(K.KvError):
        K.kv_paged_plan(p, *step(5))
    assert aim(p) == before and all(a is b for a, b in zip(p.inputs, first))


class Side:
    cuda_stream, device_index = 1234, 0


@pytest.fixture
def places(monkeypatch):
    """The handles of the streams that tensors are made under (None: the current one)."""
    made, under = [], []
    real = torch.empty

    class Under:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            under.append(self.s.cuda_stream)

        def __exit__(self, *_):
            under.pop()

    class External:
        def __init__(self, handle, device=None):
            self.cuda_stream, self.device_index = handle, 0

    def empty(*a, device=None, **kw):
        made.append(under[-1] if under else None)
        return on_gpu(real(*a, **kw))
    monkeypatch.setattr(torch.cuda, "stream", Under)
    monkeypatch.setattr(torch.cuda, "ExternalStream", External)
    monkeypatch.setattr(torch, "empty", empty)
    return made


@pytest.mark.parametrize("stream, where, handle", [(None, None, 70), (70, None, 70), (Side, 1234, 1234), (1234, 1234, 1234), (0, 0, 0)])
def test_outputs_are_made_under_the_stream_that_writes_them(binding, places, stream, where, handle):
    """Memory that the current stream still works on is not given to another stream's
    call, nor back to the current stream while the other one writes."""
    K, lib = binding
    p = plan_for(K)
    K.kv_paged_plan(p, *step())
    f16 = dict(dtype=torch.float16)
    x = on_gpu(torch.zeros(8, 4, 64, **f16))
    cache = K.Cache(on_gpu(torch.zeros(3, 2, 16, 64, **f16)), on_gpu(torch.zeros(3, 2, 64, 16, **f16)))
    rope = K.Rope.__new__(K.Rope)
    rope.handle = 5
    places.clear()
    out = K.kv_paged_attention(p, cache, x, stream=stream)
    assert out.shape == x.shape and out.dtype == x.dtype and places == [where] and lib.calls[-1][1][-1] == handle
    out = K.kv_rope_apply(rope, x, on_gpu(torch.zeros(8, dtype=torch.int32)), stream=stream)
    assert out.shape == x.shape and out.dtype == x.dtype and places == [where] * 2 and lib.calls[-1][1][-1] == handle
    rope.handle = None


def test_tensors_of_another_device_are_refused(binding):
    """Every tensor has to be on the current device, where the kernels run; so have the
    plan, the cache and the stream."""
    K, lib = binding
    f16, i32 = dict(dtype=torch.float16), dict(dtype=torch.int32)
    p = plan_for(K)
    for at in range(4):
        tensors = step()
        tensors[at] = on_gpu(torch.Tensor(tensors[at]).to(torch.int32), 1)
        with pytest.raises(ValueError, match="current device"):
            K.kv_paged_plan(p, *tensors)
    K.kv_paged_plan(p, *step())
    x, kc, vc = torch.zeros(8, 4, 64, **f16), torch.zeros(3, 2, 16, 64, **f16), torch.zeros(3, 2, 64, 16, **f16)
    cache = K.Cache(on_gpu(kc), on_gpu(vc))
    rope = K.Rope.__new__(K.Rope)
    rope.handle = 5
    here, there, pos = on_gpu(x), on_gpu(x, 1), on_gpu(torch.zeros(8, **i32))
    kv, kv_there = here[:, :2], on_gpu(x[:, :2], 1)
    n = len(lib.calls)
    elsewhere = plan_for(K)
    K.kv_paged_plan(elsewhere, *step())
    elsewhere.dev = 1
    for bad in (lambda: K.kv_rope_apply(rope, there, pos, out=here), lambda: K.kv_rope_apply(rope, here, pos, out=there),
                lambda: K.kv_rope_apply(rope, here, on_gpu(torch.zeros(8, **i32), 1), out=here),
                lambda: K.kv_paged_append(p, cache, kv_there, kv), lambda: K.kv_paged_append(p, cache, kv, kv_there),
                lambda: K.kv_paged_append(p, cache, kv, kv, q=there, q_out=here), lambda: K.kv_paged_append(p, cache, kv, kv, q=here, q_out=there),
                lambda: K.kv_paged_attention(p, cache, there, out=here), lambda: K.kv_paged_attention(p, cache, here, out=there),
                lambda: K.kv_paged_attention(p, cache, here, out=here, lse=on_gpu(torch.zeros(8, 4), 1)),
                lambda: K.kv_paged_attention(p, K.Cache(on_gpu(kc, 1), on_gpu(vc, 1)), here, out=here),
                lambda: K.Cache(on_gpu(kc), on_gpu(vc, 1)),
                lambda: K.Cache(on_gpu(kc.to(torch.float8_e4m3fn)), on_gpu(vc.to(torch.float8_e4m3fn)), k_scale=on_gpu(torch.ones(2), 1)),
                lambda: K.kv_paged_attention(elsewhere, cache, here, out=here),
                lambda: K.kv_paged_plan(elsewhere, *step())):
        with pytest.raises(ValueError, match="device"):
            bad()
    other = type("S", (), dict(cuda_stream=9, device_index=1))
    for bad in (lambda: K.kv_paged_plan(p, *step(), stream=other), lambda: K.kv_paged_append(p, cache, kv, kv, stream=other),
                lambda: K.kv_rope_apply(rope, here, pos, out=here, stream=other), lambda: K.kv_paged_attention(p, cache, here, out=here, stream=other)):
        with pytest.raises(ValueError, match="device"):
            bad()
    assert len(lib.calls) == n + 1
    rope.handle = None


def test_the_stride_of_one_element_says_nothing(binding):
    """One token at an odd stride, and a cache of one key/value head whose blocks were
    made token by token: each lies as the library needs it."""
    K, lib = binding
    f16, i32 = dict(dtype=torch.float16), dict(dtype=torch.int32)
    rope = K.Rope.__new__(K.Rope)
    rope.handle = 5
    one = on_gpu(torch.zeros(400, **f16).as_strided((1, 4, 64), (259, 64, 1)))
    assert one.stride(0) % 8
    out = on_gpu(torch.zeros(1, 4, 64, **f16))
    K.kv_rope_apply(rope, one, on_gpu(torch.zeros(1, **i32)), out=out)
    vx, vy = lib.calls[-1][1][2:4]
    assert vx.token_stride % 8 == 0 and vx.head_stride == 64 and vy.head_stride == 64
    head = on_gpu(torch.zeros(400, **f16).as_strided((4, 1, 64), (64, 3, 1)))
    K.kv_rope_apply(rope, head, on_gpu(torch.zeros(4, **i32)), out=on_gpu(torch.zeros(4, 1, 64, **f16)))
    vx = lib.calls[-1][1][2]
    assert vx.token_stride == 64 and vx.head_stride % 8 == 0
    kc = on_gpu(torch.zeros(3, 16, 1, 64, **f16).transpose(1, 2))
    vc = on_gpu(torch.zeros(3, 64, 1, 16, **f16).transpose(1, 2))
    assert kc.stride(1) == 64 and vc.stride(1) == 16
    c = K.Cache(kc, vc).c
    assert (c.k_block_stride, c.v_block_stride, c.n_blocks) == (1024, 1024, 3)
    for k, v in ((torch.zeros(3, 16, 2, 64, **f16).transpose(1, 2), torch.zeros(3, 2, 64, 16, **f16)),
                 (torch.zeros(3, 2, 16, 64, **f16), torch.zeros(3, 2, 16, 64, **f16).transpose(2, 3))):
        with pytest.raises(ValueError, match="contiguous"):
            K.Cache(on_gpu(k), on_gpu(v))
    rope.handle = None
