"""ctypes binding of the paged-cache operators (include/kvpaged.h).

As in :mod:`.kvcfg`, every computation runs in the HIP library: this module
checks tensors, holds the arrays of a step's batch and passes pointers.  One
serving step is

    plan = Plan(n_req, max_tokens, block_size, max_blocks, q_heads, kv_heads, head_dim, max_new=...)
    kv_paged_plan(plan, ctx_len, new_len, table, free_list)          # once a step
    kv_paged_append(plan, cache, k, v, q=q, q_out=q, rope=rope)      # every layer
    kv_paged_attention(plan, cache, q, out=out)

and kv_paged_read(plan, cache, row_start, ...) gives tokens of the cache back as rows.

Tensors, plan, cache and rotation are on the current device.  Calls go to the current
stream, or to `stream`: a torch.cuda.Stream or a stream's handle.  With a stream that
is not the current one the rules are torch's: inputs, plan and cache have to be ready
on it, their memory must not be given away before it is done with them, and an output
that the call makes (out=None) belongs to it: the current stream waits for it before a
use, and such a use is recorded (Tensor.record_stream) if the output may be dropped
before it ends.

kv_rope_apply takes part in automatic differentiation.  The other calls do not: what
they write carries no gradient.
"""
from __future__ import annotations

import ctypes

import torch

from .kvcfg import KV_ERR_INVALID, KV_ERR_UNSUPPORTED, KV_OK, LIB, KvError, _check, kv_last_error  # noqa: F401

KV_DT_BF16, KV_DT_F16, KV_DT_FP8, KV_DT_FP8_BLOCK, KV_DT_I8_BLOCK = 0, 1, 2, 4, 5
KV_ROPE_HALF, KV_ROPE_INTERLEAVED = 0, 1
KV_ROPE_PLAIN, KV_ROPE_LINEAR, KV_ROPE_BY_PARTS = 0, 1, 2
KV_PLAN_BAD_LENGTH, KV_PLAN_TOKENS, KV_PLAN_BLOCKS = 1, 2, 4
KV_PAGED_MAX_REQ, KV_PAGED_MAX_TOKENS = 4096, 524288

_u64, _u32, _i64, _f64, _vp = (ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int64, ctypes.c_double,
                               ctypes.c_void_p)


class kv_rope_desc(ctypes.Structure):
    _fields_ = [("rot_dim", _u32), ("layout", _u32), ("scaling", _u32), ("original_len", _u32),
                ("base", _f64), ("factor", _f64), ("fast", _f64), ("slow", _f64),
                ("magnitude", _f64)]


class kv_heads_view(ctypes.Structure):
    _fields_ = [("ptr", _vp), ("token_stride", _i64), ("head_stride", _i64)]


class kv_paged_batch(ctypes.Structure):
    _fields_ = [("n_req", _u32), ("max_tokens", _u32), ("max_new", _u32), ("block_size", _u32),
                ("max_blocks", _u32), ("q_heads", _u32), ("kv_heads", _u32), ("head_dim", _u32),
                ("window", _u32), ("n_free", _u32), ("ctx_len", _vp), ("new_len", _vp),
                ("table", _vp), ("free_list", _vp), ("q_start", _vp), ("kv_len", _vp),
                ("slot", _vp), ("pos", _vp), ("result", _vp), ("work", _vp), ("work_bytes", _u64)]


class kv_paged_cache(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_block_stride", _i64), ("v_block_stride", _i64),
                ("n_blocks", _u32), ("dtype", _u32), ("k_scale", _vp), ("v_scale", _vp)]


EXPORTS = ("kv_rope_create", "kv_rope_free", "kv_rope_apply", "kv_paged_work_bytes",
           "kv_paged_plan", "kv_paged_append", "kv_paged_read", "kv_paged_attention")

_P = ctypes.POINTER
LIB.kv_rope_create.argtypes = [_P(kv_rope_desc), _P(_vp)]
LIB.kv_rope_free.argtypes = [_vp]
LIB.kv_rope_apply.argtypes = [_vp, _u32, kv_heads_view, kv_heads_view, _vp, _u32, _u32, _u32,
                              ctypes.c_int, _vp]
LIB.kv_paged_work_bytes.argtypes = [_P(kv_paged_batch), _P(_u64)]
LIB.kv_paged_plan.argtypes = [_P(kv_paged_batch), _vp]
LIB.kv_paged_append.argtypes = [_P(kv_paged_batch), _P(kv_paged_cache), _vp, _u32, kv_heads_view,
                                kv_heads_view, kv_heads_view, kv_heads_view, _vp]
LIB.kv_paged_read.argtypes = [_P(kv_paged_batch), _P(kv_paged_cache), _u32, _vp, _vp, _u32, kv_heads_view,
                              kv_heads_view, _vp]
LIB.kv_paged_attention.argtypes = [_P(kv_paged_batch), _P(kv_paged_cache), _u32, kv_heads_view,
                                   kv_heads_view, _vp, ctypes.c_float, _vp]
for _name in EXPORTS:
    getattr(LIB, _name).restype = ctypes.c_int


_TYPES = {torch.bfloat16: KV_DT_BF16, torch.float16: KV_DT_F16, torch.float8_e4m3fn: KV_DT_FP8}
_BLOCK_TYPES = {torch.float8_e4m3fn: KV_DT_FP8_BLOCK, torch.int8: KV_DT_I8_BLOCK}
_NO_VIEW = kv_heads_view()
_raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _stream(stream, dev):
    """The handle of a stream of the current device `dev`.  The current stream's is
    _raw_stream(dev): these calls take a few microseconds on the device, and
    torch.cuda.current_stream() would take three more."""
    if isinstance(stream, int):
        return stream
    if getattr(stream, "device_index", dev) != dev:
        raise ValueError(f"the stream is on device {stream.device_index}; the current device is {dev}")
    return stream.cuda_stream


def _output(like, shape, stream, dev, dtype=None):
    """An output of `like`'s type (or `dtype`), made under the stream that will write it: the memory
    is then none that another stream may still be working on, and is not given to
    another stream while this one writes."""
    if stream is None or _stream(stream, dev) == _raw_stream(dev):
        return torch.empty(shape, dtype=dtype or like.dtype, device=like.device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=like.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype or like.dtype, device=like.device)


_HEAD_TYPES = {torch.bfloat16: KV_DT_BF16, torch.float16: KV_DT_F16}


def _dtype(dtype, name):
    d = _HEAD_TYPES.get(dtype)
    if d is None:
        raise ValueError(f"{name} has dtype {dtype}; expected bfloat16 or float16")
    return d


def _view(t, name, dev, tokens, heads, dim, dtype):
    """[tokens, heads, dim] of this dtype on device `dev`, with contiguous elements and at
    least `tokens` rows."""
    if t.get_device() != dev:
        raise ValueError(f"{name} must be a CUDA tensor of the current device")
    s = t.shape
    if len(s) != 3 or s[0] < tokens or s[1] != heads or s[2] != dim:
        raise ValueError(f"{name} has shape {tuple(s)}; the call needs [>={tokens}, {heads}, {dim}]")
    if t.dtype is not dtype:
        raise ValueError(f"{name} has dtype {t.dtype}; expected {dtype}")
    by_token, by_head, by_element = t.stride()
    if by_element != 1:
        raise ValueError(f"{name}: a head's elements must be contiguous")
    if (by_token | by_head) & 7:  # refused by the library, but not for a dimension of one element
        by_token, by_head = 0 if s[0] == 1 else by_token, 0 if s[1] == 1 else by_head
    return kv_heads_view(t.data_ptr(), by_token, by_head)


def _array(t, name, dev, dtype, numel):
    """A contiguous tensor of this dtype on device `dev` with at least `numel` elements."""
    if t.get_device() != dev or t.dtype is not dtype or not t.is_contiguous() or t.numel() < numel:
        raise ValueError(f"{name} must be a contiguous CUDA {dtype} tensor of the current device, of at least {numel} elements")
    return t.data_ptr()


class Rope:
    """Rotary positions over the first `rot_dim` elements of a head (owns the
    kv_rope handle, on the current device)."""

    def __init__(self, rot_dim, base=10000.0, layout=KV_ROPE_HALF, scaling=KV_ROPE_PLAIN,
                 factor=1.0, original_len=0, fast=32.0, slow=1.0, magnitude=1.0):
        self.handle = None
        d = kv_rope_desc(rot_dim, layout, scaling, original_len, base, factor, fast, slow, magnitude)
        h = _vp()
        _check(LIB.kv_rope_create(ctypes.byref(d), ctypes.byref(h)))
        self.handle = h

    def free(self):
        if self.handle is not None:
            h, self.handle = self.handle, None
            _check(LIB.kv_rope_free(h))

    def __del__(self):
        try:
            if self.handle is not None:
                LIB.kv_rope_free(self.handle)
        except Exception:
            pass


class _Rotation(torch.autograd.Function):
    """y = rotation of x; the gradient of x is that of y turned the other way."""

    @staticmethod
    def forward(ctx, x, rope, pos, backward, stream):
        ctx.save_for_backward(pos)
        ctx.rope, ctx.turned_back = rope, backward
        return kv_rope_apply(rope, x, pos, backward=backward, stream=stream)  # recording is off in here

    @staticmethod
    def backward(ctx, grad):
        pos, = ctx.saved_tensors
        # gradients come expanded, transposed or from the inside of other tensors
        if grad.data_ptr() % 16 or not grad.is_contiguous():
            grad = grad.clone(memory_format=torch.contiguous_format)
        return kv_rope_apply(ctx.rope, grad, pos, backward=not ctx.turned_back), None, None, None, None


def _recorded_rotation(rope, x, pos, out, backward, stream):
    turned = _Rotation.apply(x, rope, pos, backward, stream)
    if out is None:
        return turned
    _view(out, "out", _device(), *x.shape, x.dtype)
    if stream is None:
        out[:x.shape[0]].copy_(turned)
    else:
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=x.device) if isinstance(stream, int) else stream):
            out[:x.shape[0]].copy_(turned)
    return out


def kv_rope_apply(rope: Rope, x, pos, out=None, backward=False, stream=None):
    """x: [tokens, heads, dim] bfloat16 / float16 at any token and head stride;
    pos: int32 [tokens]; out: like x (may be x), made when None.  Returns out.

    An x that requires a gradient gets one (rope and the values in pos are to be kept
    until the backward pass); a given out then takes part as by out.copy_()."""
    if x.requires_grad and torch.is_grad_enabled():
        return _recorded_rotation(rope, x, pos, out, backward, stream)
    dev, dtype = _device(), x.dtype
    n, heads, dim = x.shape
    kind, vx = _dtype(dtype, "x"), _view(x, "x", dev, n, heads, dim, dtype)
    if out is None:
        out = _output(x, (n, heads, dim), stream, dev)
    vy = vx if out is x else _view(out, "out", dev, n, heads, dim, dtype)
    _check(LIB.kv_rope_apply(rope.handle, kind, vx, vy, _array(pos, "pos", dev, torch.int32, n), n, heads, dim,
                             1 if backward else 0, _raw_stream(dev) if stream is None else _stream(stream, dev)))
    return out


class Plan:
    """The arrays of one step's batch.  Sizes are fixed, so a plan can be filled
    again for every step, also inside a captured graph; the device arrays
    q_start, kv_len, slot, pos and result are valid once the stream has
    completed kv_paged_plan.  It serves one stream at a time."""

    def __init__(self, n_req, max_tokens, block_size, max_blocks, q_heads, kv_heads, head_dim,
                 max_new=None, window=0, device="cuda"):
        b = self.batch = kv_paged_batch()
        b.n_req, b.max_tokens, b.max_new = int(n_req), int(max_tokens), int(max_new or 0)
        b.block_size, b.max_blocks = int(block_size), int(max_blocks)
        b.q_heads, b.kv_heads, b.head_dim, b.window = int(q_heads), int(kv_heads), int(head_dim), int(window)
        size = _u64()
        _check(LIB.kv_paged_work_bytes(ctypes.byref(b), ctypes.byref(size)))
        self.q_start = torch.empty(b.n_req + 1, dtype=torch.int32, device=device)
        self.dev = self.q_start.get_device()
        self.kv_len = torch.empty(b.n_req, dtype=torch.int32, device=device)
        self.slot = torch.empty(b.max_tokens, dtype=torch.int64, device=device)
        self.pos = torch.empty(b.max_tokens, dtype=torch.int32, device=device)
        self.result = torch.empty(4, dtype=torch.int32, device=device)
        self.work = torch.empty(size.value, dtype=torch.uint8, device=device)
        b.q_start, b.kv_len = self.q_start.data_ptr(), self.kv_len.data_ptr()
        b.slot, b.pos, b.result = self.slot.data_ptr(), self.pos.data_ptr(), self.result.data_ptr()
        b.work, b.work_bytes = self.work.data_ptr(), size.value
        self.ref = ctypes.byref(b)
        # the planned step's tensors, kept alive as the later calls of the step read the
        # table, and what the batch says of them
        self.inputs, self.step = None, (None, None, None, 0, None)


def kv_paged_plan(plan: Plan, ctx_len, new_len, table, free_list=None, stream=None):
    """ctx_len, new_len: int32 [n_req]; table: int32 [n_req, max_blocks], written
    where a request takes new blocks from free_list (int32), read otherwise."""
    b, dev = plan.batch, _device()
    if plan.dev != dev:
        raise ValueError(f"the plan is on device {plan.dev}; the current device is {dev}")
    n, columns, shape = b.n_req, b.max_blocks, table.shape
    if len(shape) != 2 or shape[1] != columns:
        raise ValueError(f"table has shape {tuple(shape)}; the plan's rows have {columns} blocks")
    i32 = torch.int32
    # all of it is checked before the batch points at any of it: after a refusal the
    # batch is that of the step planned before, whose tensors are kept
    step = (_array(ctx_len, "ctx_len", dev, i32, n), _array(new_len, "new_len", dev, i32, n),
            _array(table, "table", dev, i32, n * columns), 0 if free_list is None else free_list.numel(),
            # an empty tensor has no address, and NULL would mean that table names every block
            None if free_list is None else _array(free_list, "free_list", dev, i32, 0) or b.result)
    stream = _raw_stream(dev) if stream is None else _stream(stream, dev)
    b.ctx_len, b.new_len, b.table, b.n_free, b.free_list = step
    try:
        _check(LIB.kv_paged_plan(plan.ref, stream))
    except KvError:
        b.ctx_len, b.new_len, b.table, b.n_free, b.free_list = plan.step
        raise
    plan.inputs, plan.step = (ctx_len, new_len, table, free_list), step


class Cache:
    """A layer's cache: k [n_blocks, kv_heads, block_size, head_dim], v [n_blocks,
    kv_heads, head_dim, block_size]; blocks may lie at any stride, each block is
    contiguous.  float8_e4m3fn caches take k_scale, v_scale: float32 [kv_heads].

    With block_scales, k_scale and v_scale are float32 [n_blocks, kv_heads], a scale for
    each block and head, and kv_paged_append writes them; k and v are int8 or
    float8_e4m3fn.  The contents of a new cache do not matter."""

    def __init__(self, k, v, k_scale=None, v_scale=None, block_scales=False):
        if k.dim() != 4 or v.dim() != 4 or not k.is_cuda or not v.is_cuda:
            raise ValueError("k and v must be CUDA tensors of four dimensions")
        dev = self.dev = k.get_device()
        if v.get_device() != dev:
            raise ValueError("k and v must be on one device")
        n, heads, block, dim = k.shape
        types = _BLOCK_TYPES if block_scales else _TYPES
        if tuple(v.shape) != (n, heads, dim, block) or v.dtype != k.dtype or k.dtype not in types:
            raise ValueError(f"v has shape {tuple(v.shape)} and dtype {v.dtype}, k {tuple(k.shape)} and {k.dtype}")
        # (by the first block: a dimension of one element may have any stride)
        if not k[:1].is_contiguous() or not v[:1].is_contiguous():
            raise ValueError("a block of the cache must be contiguous")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.shape = (heads, block, dim)
        one = heads * block * dim  # the stride of a cache of one block says nothing
        c = self.c = kv_paged_cache()
        c.k, c.v = k.data_ptr(), v.data_ptr()
        c.k_block_stride = k.stride(0) if n > 1 else one
        c.v_block_stride = v.stride(0) if n > 1 else one
        c.n_blocks, c.dtype = n, types[k.dtype]
        if block_scales:
            for name, s in (("k_scale", k_scale), ("v_scale", v_scale)):
                if s is None or tuple(s.shape) != (n, heads):
                    raise ValueError(f"{name} must have shape {(n, heads)}: a scale for each block and head")
            heads *= n
        c.k_scale = None if k_scale is None else _array(k_scale, "k_scale", dev, torch.float32, heads)
        c.v_scale = None if v_scale is None else _array(v_scale, "v_scale", dev, torch.float32, heads)
        self.ref = ctypes.byref(c)


def _fits(plan, cache, dev):
    """The batch and its number of tokens; the cache has the plan's shape."""
    b = plan.batch
    if plan.dev != dev or cache.dev != dev:
        raise ValueError(f"the plan is on device {plan.dev}, the cache on {cache.dev}; the current device is {dev}")
    if cache.shape != (b.kv_heads, b.block_size, b.head_dim):
        raise ValueError(f"the cache's heads, block and head size are {cache.shape}; "
                         f"the plan's {(b.kv_heads, b.block_size, b.head_dim)}")
    if plan.inputs is None:
        raise ValueError("the plan is empty: call kv_paged_plan first")
    return b, b.max_tokens


def kv_paged_append(plan: Plan, cache: Cache, k, v, q=None, q_out=None, rope: Rope | None = None,
                    stream=None):
    """k, v: [>=max_tokens, kv_heads, dim]; q, q_out: [>=max_tokens, q_heads, dim]
    (q_out may be q) or None."""
    dev = _device()
    b, n = _fits(plan, cache, dev)
    heads, _, dim = cache.shape
    dtype = k.dtype
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    if rope is not None and rope.handle is None:  # NULL would mean that nothing turns
        raise ValueError("the rotation has been freed")
    kind, vk, vv = _dtype(dtype, "k"), _view(k, "k", dev, n, heads, dim, dtype), _view(v, "v", dev, n, heads, dim, dtype)
    if q is None:
        vq = vo = _NO_VIEW
    else:
        heads = b.q_heads
        vq = _view(q, "q", dev, n, heads, dim, dtype)
        vo = vq if q_out is q else _view(q_out, "q_out", dev, n, heads, dim, dtype)
    _check(LIB.kv_paged_append(plan.ref, cache.ref, None if rope is None else rope.handle, kind, vq, vo, vk, vv,
                               _raw_stream(dev) if stream is None else _stream(stream, dev)))


def kv_paged_read(plan: Plan, cache: Cache, row_start, first=None, k=None, v=None, rows=None, dtype=None,
                  stream=None):
    """Keys and values of every request from position first[r] on (int32 [n_req]; None: 0)
    as rows row_start[r] .. row_start[r+1] - 1 (int32 [n_req+1]) of k and v: [rows,
    kv_heads, dim] bfloat16 / float16.  k and v go together; where they are None they are
    made, with `rows` rows (rows that nothing is read into hold anything) of `dtype`,
    the cache's own or bfloat16.  Rows of a cache of 8 bits end at dtype's largest
    number.  Returns (k, v)."""
    dev = _device()
    b, _ = _fits(plan, cache, dev)
    heads, _, dim = cache.shape
    if (k is None) != (v is None):
        raise ValueError("k and v go together")
    if rows is not None and rows < 0:  # (the library would take its lowest 32 bits)
        raise ValueError(f"rows is {rows}; expected none or more")
    if k is None:
        if rows is None:
            raise ValueError("either k and v or the number of rows has to be given")
        like = cache.k
        if dtype is None:
            dtype = like.dtype if like.dtype in _HEAD_TYPES else torch.bfloat16
        k, v = (_output(like, (int(rows), heads, dim), stream, dev, dtype) for _ in range(2))
    elif dtype is not None and dtype is not k.dtype:
        raise ValueError(f"k has dtype {k.dtype}; expected {dtype}")
    n = k.shape[0] if rows is None else int(rows)
    dtype = k.dtype
    kind, vk, vv = _dtype(dtype, "k"), _view(k, "k", dev, n, heads, dim, dtype), _view(v, "v", dev, n, heads, dim, dtype)
    _check(LIB.kv_paged_read(plan.ref, cache.ref, kind, _array(row_start, "row_start", dev, torch.int32, b.n_req + 1),
                             None if first is None else _array(first, "first", dev, torch.int32, b.n_req), n, vk, vv,
                             _raw_stream(dev) if stream is None else _stream(stream, dev)))
    return k, v


def kv_paged_attention(plan: Plan, cache: Cache, q, out=None, lse=None, scale=None, stream=None):
    """q, out: [>=max_tokens, q_heads, dim]; lse: float32 [>=max_tokens, q_heads] or
    None; scale: dim ** -0.5 when None.  Returns out."""
    dev = _device()
    b, n = _fits(plan, cache, dev)
    heads, dim, dtype = b.q_heads, cache.shape[2], q.dtype
    kind, vq = _dtype(dtype, "q"), _view(q, "q", dev, n, heads, dim, dtype)
    if out is None:
        out = _output(q, (n, heads, dim), stream, dev)
    vo = _view(out, "out", dev, n, heads, dim, dtype)
    pl = None if lse is None else _array(lse, "lse", dev, torch.float32, n * heads)
    _check(LIB.kv_paged_attention(plan.ref, cache.ref, kind, vq, vo, pl, dim ** -0.5 if scale is None else scale,
                                  _raw_stream(dev) if stream is None else _stream(stream, dev)))
    return out
