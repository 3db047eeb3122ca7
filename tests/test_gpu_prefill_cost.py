"""The measured prefill cost on the card: the operators run together over a trace."""
import pytest

import tracegen as tg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_blocks, batch", [(400, 3), (8192, 16)])
def test_a_trace_is_served(n_blocks, batch):
    from paper_2603_08739_amd import prefill_cost as P
    t = tg.tiny(n_req=40)
    steps = list(P.batches(t, n_blocks, batch))
    done = P.measure(t, n_blocks, batch=batch, q_heads=8, kv_heads=2, head_dim=64)
    block = t.tokens_per_granule
    assert done["steps"] == len(steps) and done["requests"] == sum(map(len, steps))
    assert done["cached_tokens"] == block * sum(len(run) for s in steps for run, _ in s)
    assert done["new_tokens"] == block * sum(len(got) for s in steps for _, got in s)
    assert min(done["plan_s"], done["append_s"], done["attention_s"]) > 0
    one, two = P.seconds_per_token(done, 1), P.seconds_per_token(done, 2, other=1e-6)
    assert 0 < one < two - 1e-6


def test_reused_blocks_give_the_same_answers():
    """A request served in two steps, its prefix from the cache, gets what it gets when
    all of it is computed at once."""
    import torch
    from paper_2603_08739_amd import kvpaged as K
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)
    H, J, D, bs, n, cut = 8, 2, 128, 16, 170, 96
    fused = torch.randn(n, H + 2 * J, D, device="cuda", generator=g).bfloat16()
    rope = K.Rope(D)
    outs = []
    for parts in ((n,), (cut, n - cut), (cut, n - cut - 1, 1)):
        kc, vc = torch.zeros(20, J, bs, D, device="cuda").bfloat16(), torch.zeros(20, J, D, bs, device="cuda").bfloat16()
        cache, table = K.Cache(kc, vc), torch.full((1, 12), -1, **i32)
        free, taken, at, out = torch.randperm(20, device="cuda", generator=g).to(torch.int32), 0, 0, []
        for m in parts:
            p = K.Plan(1, m, bs, 12, H, J, D, max_new=m)
            K.kv_paged_plan(p, torch.tensor([at], **i32), torch.tensor([m], **i32), table, free[taken:].contiguous())
            x = fused[at:at + m]
            q = torch.empty(m, H, D, device="cuda", dtype=x.dtype)
            K.kv_paged_append(p, cache, x[:, H:H + J], x[:, H + J:], q=x[:, :H], q_out=q, rope=rope)
            out.append(K.kv_paged_attention(p, cache, q))
            taken += int(p.result[2])
            at += m
        outs.append(torch.cat(out).float())
    # the kernels' weights are rounded from other maxima: two roundings of 2^-8 each of
    # the sum of weighted values, which is at most the largest value
    tol = 2 * 2.0 ** -8 * float(fused[:, H + J:].float().abs().max())
    assert float((outs[0] - outs[1]).abs().max()) <= tol and float((outs[0] - outs[2]).abs().max()) <= tol


def test_command():
    from paper_2603_08739_amd import prefill_cost as P
    done, t, obj, flags = P.main(["--requests", "24", "--blocks", "2048", "--layers", "2"])
    assert done["requests"] == 24 and t > 0 and obj.shape == (64, 3) and flags.sum() >= 1
