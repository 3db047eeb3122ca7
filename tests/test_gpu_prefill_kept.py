"""The measured prefill cost over a quantised cache on the card."""
import pytest

import tracegen as tg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kept", ["fp8", "i8"])
def test_a_trace_is_served_from_a_quantised_cache(kept):
    from paper_2603_08739_amd import prefill_cost as P
    t = tg.tiny(n_req=20)
    done = P.measure(t, 2048, batch=8, q_heads=8, kv_heads=2, head_dim=64, kept=kept)
    assert done["requests"] == 20 and done["new_tokens"] > 0 and min(done["plan_s"], done["append_s"], done["attention_s"]) > 0


def test_command():
    from paper_2603_08739_amd import prefill_cost as P
    done, t, obj, flags = P.main(["--requests", "24", "--blocks", "2048", "--layers", "2", "--cache", "i8"])
    assert done["requests"] == 24 and t > 0 and obj.shape == (64, 3) and flags.sum() >= 1


def test_reused_blocks_give_the_same_answers():
    """A request served in steps that end inside blocks gets what it gets when all of it is
    computed at once, up to the units of its blocks."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)
    H, J, D, bs, n = 8, 2, 128, 16, 170
    fused = torch.randn(n, H + 2 * J, D, device="cuda", generator=g).bfloat16()
    rope, rows, units = K.Rope(D), [], []
    for parts in ((n,), (90, 80), (96, 73, 1), (5,) * 34):
        kc, vc = torch.zeros(20, J, bs, D, device="cuda", dtype=torch.int8), torch.zeros(20, J, D, bs, device="cuda", dtype=torch.int8)
        ks, vs = torch.zeros(20, J, device="cuda"), torch.zeros(20, J, device="cuda")
        cache, table = K.Cache(kc, vc, ks, vs, block_scales=True), torch.randperm(20, device="cuda", generator=g).to(torch.int32)[None, :12].contiguous()
        at = 0
        for m in parts:
            p = K.Plan(1, m, bs, 12, H, J, D, max_new=m)
            K.kv_paged_plan(p, torch.tensor([at], **i32), torch.tensor([m], **i32), table)
            x = fused[at:at + m]
            K.kv_paged_append(p, cache, x[:, H:H + J], x[:, H + J:], q=x[:, :H], q_out=torch.empty(m, H, D, device="cuda", dtype=x.dtype), rope=rope)
            at += m
        rows.append(K.kv_paged_read(p, cache, torch.tensor([0, n], **i32), rows=n))
        page = table[0].long().repeat_interleave(bs)[:n]
        units.append((ks[page], vs[page]))
    for other, unit in zip(rows[1:], units[1:]):
        for a, b, u, first in zip(other, rows[0], unit, units[0]):
            # a doubled scale is below twice the largest; a number is at most half a unit off, and
            # less than one whole unit after its rises; read back in 8 significant bits
            assert bool((u < 2 * first * (1 + 2.0 ** -20)).all()) and bool((u >= first * (1 - 2.0 ** -20)).all())
            assert bool(((a.float() - b.float()).abs() <= (u + 0.5 * first)[:, :, None] * 1.001 + 2.0 ** -8 * (a.float().abs() + b.float().abs())).all())
