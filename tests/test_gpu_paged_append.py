"""The write of keys and values into the cache against the definition in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu


def near(got, want, tol, what):
    import torch
    g = got.double()
    assert torch.equal(torch.isnan(g), torch.isnan(want)), what
    ok = ((g - want).abs() <= tol) | torch.isnan(want)
    assert bool(ok.all()), (what, float((g - want).abs().max()))


@pytest.mark.parametrize("dtype, kept", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("ctx, new, block, heads, dim, rot, interleaved", [
    ([0], [1], 16, (1, 1), 64, 64, 0),
    ([15, 16, 17, 0], [1, 1, 1, 1], 16, (8, 2), 128, 128, 0),
    ([3, 0, 40, 8, 100], [30, 0, 17, 8, 5], 16, (6, 3), 64, 32, 1),
    ([60, 1], [70, 200], 64, (4, 4), 256, 256, 0),
    ([250], [20], 256, (16, 1), 128, 64, 1),
    ([7, 500], [1, 900], 32, (40, 8), 128, 128, 0)])
def test_append(dtype, kept, ctx, new, block, heads, dim, rot, interleaved):
    import torch
    from oracle import paged as O
    from paper_2603_08739_amd import kvpaged as K
    from tests.paged import ROUND, TYPES, blocks_of
    gen = torch.Generator().manual_seed(sum(ctx) + 7 * block)
    H, J = heads
    table, n_blocks = blocks_of(ctx, new, block, gen)
    total = sum(new)
    T = total + 5  # a padded step: the last rows are nobody's
    fused = (torch.randn(T, H + 2 * J, dim, generator=gen) * 3).to(TYPES[dtype]).cuda()
    q, k, v = fused[:, :H], fused[:, H:H + J], fused[:, H + J:]
    if dim > 64:
        v[0, 0, :3] = torch.tensor([float("inf"), -float("inf"), float("nan")])
    kc = torch.zeros(n_blocks, J, block, dim).to(TYPES[kept]).cuda()
    vc = torch.zeros(n_blocks, J, dim, block).to(TYPES[kept]).cuda()
    ks = vs = None
    if kept == "fp8":
        ks, vs = (torch.rand(J, generator=gen) * 0.02 + 0.005).cuda(), (torch.rand(J, generator=gen) * 0.02 + 0.005).cuda()
    kw = dict(base=500000.0, scaling=2, factor=16.0, original_len=4096)
    rope = K.Rope(rot, layout=interleaved, magnitude=1.2, **kw)
    freq = O.frequencies(rot, **kw)
    p = K.Plan(len(ctx), T, block, table.shape[1], H, J, dim)
    i32 = dict(dtype=torch.int32, device="cuda")
    K.kv_paged_plan(p, torch.tensor(ctx, **i32), torch.tensor(new, **i32), table)
    q_out = torch.full((T, H, dim), 9.0, dtype=q.dtype, device="cuda")
    K.kv_paged_append(p, K.Cache(kc, vc, ks, vs), k, v, q=q, q_out=q_out, rope=rope)
    pos, slot = p.pos[:total], p.slot[:total]
    want_q = O.rope(q[:total], pos, freq, interleaved, 1.2)
    size = 1.2 * q[:total].double().abs().amax(-1, keepdim=True) * 2
    near(q_out[:total], want_q, ROUND[q.dtype] * want_q.abs() + 2.0 ** -20 * size, "q")
    assert bool((q_out[total:] == 9.0).all())
    want_k, want_v = O.rope(k[:total], pos, freq, interleaved, 1.2), v[:total].double()
    page, off = slot // block, slot % block
    got_k, got_v = kc.to(torch.float32)[page, :, off], vc.to(torch.float32)[page, :, :, off]
    size = 1.2 * k[:total].double().abs().amax(-1, keepdim=True) * 2
    if kept == "fp8":
        # 4 significant bits: half a spacing is 2^-4 of the number, or 2^-10 below 2^-6
        want_k = (want_k / ks.double()[:, None]).clamp(-448, 448)
        want_v = (want_v / vs.double()[:, None]).clamp(-448, 448)
        near(got_k, want_k, 2.0 ** -4 * want_k.abs() + 2.0 ** -10 + 2.0 ** -19 * size / ks.double()[:, None], "k")
        near(got_v, want_v, 2.0 ** -4 * want_v.abs() + 2.0 ** -10, "v")
        exact = (v[:total].float() / vs[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).float()
        assert torch.equal(torch.nan_to_num(got_v, 1e9), torch.nan_to_num(exact, 1e9))
    else:
        near(got_k, want_k, ROUND[q.dtype] * want_k.abs() + 2.0 ** -20 * size, "k")
        assert torch.equal(torch.nan_to_num(got_v, 7.5, 8.5, 9.5), torch.nan_to_num(v[:total].float(), 7.5, 8.5, 9.5))
    # nothing else was touched
    mask = torch.ones(n_blocks, block, dtype=torch.bool, device="cuda")
    mask[page, off] = False
    assert bool((kc.float().transpose(1, 2)[mask] == 0).all()) and bool((vc.float().permute(0, 3, 1, 2)[mask] == 0).all())


def test_without_rotation_or_queries_and_in_place():
    import torch
    from paper_2603_08739_amd import kvpaged as K
    g = torch.Generator(device="cuda").manual_seed(1)
    i32 = dict(dtype=torch.int32, device="cuda")
    x = torch.randn(40, 6, 64, device="cuda", generator=g).half()
    q, k, v = x[:, :4], x[:, 4:5], x[:, 5:]
    p = K.Plan(2, 40, 16, 4, 4, 1, 64)
    table = torch.tensor([[2, 0, -1, -1], [4, 1, 3, -1]], **i32)
    K.kv_paged_plan(p, torch.tensor([0, 20], **i32), torch.tensor([15, 25], **i32), table)
    kc, vc = torch.zeros(5, 1, 16, 64, device="cuda").half(), torch.zeros(5, 1, 64, 16, device="cuda").half()
    cache = K.Cache(kc, vc)
    K.kv_paged_append(p, cache, k, v)
    page, off = p.slot // 16, p.slot % 16
    assert torch.equal(kc[page, :, off], k) and torch.equal(vc[page, :, :, off], v)
    out = torch.empty(40, 4, 64, device="cuda").half()
    K.kv_paged_append(p, cache, k, v, q=q, q_out=out)
    assert torch.equal(out, q)
    rope = K.Rope(64)
    K.kv_paged_append(p, cache, k, v, q=q, q_out=out, rope=rope)
    assert torch.equal(out, K.kv_rope_apply(rope, q, p.pos)) and torch.equal(kc[page, :, off], K.kv_rope_apply(rope, k, p.pos))
    keep = k.clone()
    K.kv_paged_append(p, cache, k, v, q=q, q_out=q, rope=rope)
    assert torch.equal(q, out) and torch.equal(k, keep)


def test_tokens_without_a_place():
    """No block, a block past the cache's end, and an idle request."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    g = torch.Generator(device="cuda").manual_seed(2)
    i32 = dict(dtype=torch.int32, device="cuda")
    k, v = torch.randn(60, 2, 64, device="cuda", generator=g).bfloat16(), torch.randn(60, 2, 64, device="cuda", generator=g).bfloat16()
    p = K.Plan(4, 60, 16, 2, 2, 2, 64)
    table = torch.tensor([[0, -1], [-1, 1], [2, 2000], [3, -1]], **i32)
    K.kv_paged_plan(p, torch.tensor([4, 0, 0, 16], **i32), torch.tensor([20, 20, 20, 0], **i32), table)
    kc, vc = torch.zeros(5, 2, 16, 64, device="cuda").bfloat16(), torch.zeros(5, 2, 64, 16, device="cuda").bfloat16()
    K.kv_paged_append(p, K.Cache(kc[:4], vc[:4]), k, v)
    want_k, want_v = torch.zeros_like(kc), torch.zeros_like(vc)
    for b, off, t, n in ((0, 4, 0, 12), (1, 0, 36, 4), (2, 0, 40, 16)):
        want_k[b, :, off:off + n] = k[t:t + n].transpose(0, 1)
        want_v[b, :, :, off:off + n] = v[t:t + n].permute(1, 2, 0)
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


def test_blocks_at_a_stride_and_far_offsets():
    """K and V of one block side by side, in a cache whose offsets pass 32 bits."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    g = torch.Generator(device="cuda").manual_seed(3)
    i32 = dict(dtype=torch.int32, device="cuda")
    n_blocks, J, block, dim = 90_000, 8, 16, 128  # 2 x 32 KiB a block: 5.9 GB
    both = torch.zeros(n_blocks, 2, J * block * dim, device="cuda", dtype=torch.bfloat16)
    kc, vc = both[:, 0].view(n_blocks, J, block, dim), both[:, 1].view(n_blocks, J, dim, block)
    k, v = torch.randn(35, J, dim, device="cuda", generator=g).bfloat16(), torch.randn(35, J, dim, device="cuda", generator=g).bfloat16()
    p = K.Plan(1, 35, block, 4, 8, J, dim)
    table = torch.tensor([[89_999, 5, 70_000, 1]], **i32)
    K.kv_paged_plan(p, torch.tensor([3], **i32), torch.tensor([35], **i32), table)
    K.kv_paged_append(p, K.Cache(kc, vc), k, v)
    page, off = p.slot // block, p.slot % block
    assert torch.equal(kc[page, :, off], k) and torch.equal(vc[page, :, :, off], v)
    assert int((both != 0).sum()) == int((k != 0).sum()) + int((v != 0).sum())


def test_refusals():
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    x = torch.zeros(8, 2, 64, device="cuda", dtype=torch.bfloat16)
    kc, vc = torch.zeros(4, 2, 16, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(4, 2, 64, 16, device="cuda", dtype=torch.bfloat16)
    p = K.Plan(1, 8, 16, 2, 4, 2, 64)
    cache = K.Cache(kc, vc)
    with pytest.raises(ValueError):
        K.kv_paged_append(p, cache, x, x)  # not planned yet
    K.kv_paged_plan(p, torch.zeros(1, **i32), torch.full((1,), 8, **i32), torch.zeros(1, 2, **i32))
    for bad in (lambda: K.kv_paged_append(p, cache, x[:7], x), lambda: K.kv_paged_append(p, cache, x, x[:, :1]),
                lambda: K.kv_paged_append(p, cache, x.float(), x.float()), lambda: K.kv_paged_append(p, cache, x, x.half()),
                lambda: K.kv_paged_append(p, cache, x, x, q=x), lambda: K.kv_paged_append(p, cache, x, x, q=x, q_out=x),
                lambda: K.kv_paged_append(p, K.Cache(kc[:, :1], vc[:, :1]), x, x), lambda: K.Cache(kc, kc), lambda: K.Cache(kc.cpu(), vc.cpu()),
                lambda: K.Cache(kc, vc.half()), lambda: K.Cache(kc.transpose(0, 1), vc.transpose(0, 1))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(K.KvError):
        K.kv_paged_append(p, cache, x.half(), x.half())
    with pytest.raises(K.KvError):
        K.kv_paged_append(p, cache, x, x, rope=K.Rope(128))
    with pytest.raises(K.KvError):
        K.kv_paged_append(p, K.Cache(kc, vc, k_scale=torch.ones(2, device="cuda")), x, x)


def test_a_freed_rotation_is_refused():
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    x = torch.ones(8, 2, 64, device="cuda", dtype=torch.bfloat16)
    kc, vc = torch.zeros(4, 2, 16, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(4, 2, 64, 16, device="cuda", dtype=torch.bfloat16)
    p = K.Plan(1, 8, 16, 2, 4, 2, 64)
    K.kv_paged_plan(p, torch.zeros(1, **i32), torch.full((1,), 8, **i32), torch.zeros(1, 2, **i32))
    rope = K.Rope(64)
    rope.free()
    with pytest.raises(ValueError):
        K.kv_paged_append(p, K.Cache(kc, vc), x, x, rope=rope)
    with pytest.raises(K.KvError):
        K.kv_rope_apply(rope, x, p.pos)
    assert not kc.any()
