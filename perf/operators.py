"""Performance cases of the paged-cache operators: one serving step over a KV cache of fixed-size blocks.

  rope    rotary positions applied to a tensor of heads, forward or backward
  plan    block tables, slots, positions and the attention's pieces from request lengths
  append  rotary positions on queries and keys, keys and values written into the cache
  attn    attention of the new tokens of every request over its cached blocks

Block sizes and lengths are those of the traces the framework evaluates: 16-token blocks for prompts and chats, 64-token
blocks and contexts of 8,192 to 131,072 tokens for documents.  Head counts are generic.  Lengths follow from the case
(`lens` seeds them), every value in the tensors from prepare()'s seed.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}
HALF, INTERLEAVED = 0, 1
PLAIN, LINEAR, BY_PARTS = 0, 1, 2
BASE, ORIGINAL, FAST, SLOW = 500_000.0, 8192, 32.0, 1.0


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # queries of one decoding step of 64 requests: latency
        dict(name="rope_step", op="rope", tokens=64, heads=32, dim=128, rot=128, layout=HALF, scaling=PLAIN, dtype="bf16", backward=False, fused=False),
        # gradient of a long chunk's queries inside a fused projection's output, half of the head turned
        dict(name="rope_back", op="rope", tokens=8191, heads=40, dim=128, rot=64, layout=INTERLEAVED, scaling=BY_PARTS, dtype="f16", backward=True, fused=True),
        # one decoding step of 64 chats: the smallest plan
        dict(name="plan_step", op="plan", reqs=64, new_lo=1, new_hi=1, ctx_lo=100, ctx_hi=8000, block=16, idle=0, lens=1),
        # a thousand prompts arrive over cached prefixes, ragged, some of them idle
        dict(name="plan_prompts", op="plan", reqs=1000, new_lo=1, new_hi=800, ctx_lo=1, ctx_hi=8192, block=16, idle=9, lens=2),
        # one decoding step of 64 chats
        dict(name="append_step", op="append", reqs=64, new_lo=1, new_hi=1, ctx_lo=100, ctx_hi=8000, block=16, idle=0, q_heads=32, kv_heads=8, dim=128,
             rot=128, layout=HALF, scaling=PLAIN, dtype="bf16", cache="bf16", lens=3),
        # prompts of a long-context service, 64-token blocks
        dict(name="append_chunk", op="append", reqs=24, new_lo=20, new_hi=1500, ctx_lo=1, ctx_hi=131072, block=64, idle=0, q_heads=32, kv_heads=8, dim=128,
             rot=128, layout=HALF, scaling=BY_PARTS, dtype="bf16", cache="bf16", lens=4),
        # ragged prompts into an 8-bit cache, interleaved layout, part of the head
        dict(name="append_fp8", op="append", reqs=37, new_lo=1, new_hi=400, ctx_lo=1, ctx_hi=8192, block=16, idle=8, q_heads=24, kv_heads=4, dim=128,
             rot=64, layout=INTERLEAVED, scaling=LINEAR, dtype="f16", cache="fp8", lens=5),
        # a single chat generates: the smallest attention
        dict(name="attn_single", op="attn", reqs=1, new_lo=1, new_hi=1, ctx_lo=500, ctx_hi=500, block=16, idle=0, q_heads=32, kv_heads=8, dim=128,
             window=0, dtype="bf16", cache="bf16", lens=6),
        # one decoding step of 64 chats of very different lengths
        dict(name="attn_step", op="attn", reqs=64, new_lo=1, new_hi=1, ctx_lo=100, ctx_hi=16000, block=16, idle=0, q_heads=32, kv_heads=8, dim=128,
             window=0, dtype="bf16", cache="bf16", lens=7),
        # eight long documents are answered from an 8-bit cache
        dict(name="attn_long_fp8", op="attn", reqs=8, new_lo=1, new_hi=1, ctx_lo=8192, ctx_hi=131071, block=64, idle=0, q_heads=64, kv_heads=8, dim=128,
             window=0, dtype="bf16", cache="fp8", lens=8),
        # chunks of prompts and single tokens together, over cached prefixes, sliding window whose older blocks are gone
        dict(name="attn_mixed", op="attn", reqs=12, new_lo=1, new_hi=1300, ctx_lo=50, ctx_hi=12000, block=16, idle=5, q_heads=24, kv_heads=4, dim=64,
             window=4096, dtype="f16", cache="f16", lens=423),
        # a long prompt after a short cached prefix: bound by the matrix cores
        dict(name="attn_prompt", op="attn", reqs=1, new_lo=8111, new_hi=8111, ctx_lo=256, ctx_hi=256, block=16, idle=0, q_heads=32, kv_heads=8, dim=128,
             window=0, dtype="bf16", cache="bf16", lens=10),
    ]


def _size(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    while True:
        op = rng.choice(["rope", "plan", "append", "attn", "attn"])
        c = dict(op=op)
        if op == "rope":
            dim = rng.choice([64, 128, 256])
            c |= dict(tokens=_size(rng, 1, 16384), heads=_size(rng, 1, 64), dim=dim, rot=rng.choice([dim, dim // 2, dim // 4]),
                      layout=rng.choice([HALF, INTERLEAVED]), scaling=rng.choice([PLAIN, LINEAR, BY_PARTS]), dtype=rng.choice(["bf16", "f16"]),
                      backward=rng.random() < 0.5, fused=rng.random() < 0.5)
        else:
            decode = rng.random() < 0.5
            reqs = _size(rng, 1, 64 if decode else 16) if op == "attn" else _size(rng, 1, 1000)
            new_hi = 1 if decode else _size(rng, 2, 4096 if op == "attn" else 1500)
            ctx_hi = _size(rng, 16, 131071 if decode else 16000)
            c |= dict(reqs=reqs, new_lo=1, new_hi=new_hi, ctx_lo=rng.randint(1, ctx_hi), ctx_hi=ctx_hi, block=rng.choice([16, 32, 64]),
                      idle=rng.choice([0, 0, 5]) if reqs > 5 else 0)
            if op != "plan":
                kv_heads = rng.choice([1, 2, 4, 8])
                dtype = rng.choice(["bf16", "f16"])
                c |= dict(q_heads=kv_heads * rng.choice([1, 4, 6, 8]), kv_heads=kv_heads, dim=rng.choice([64, 128, 256]), dtype=dtype,
                          cache=rng.choice([dtype, "fp8"]))
                if op == "append":
                    c |= dict(rot=rng.choice([c["dim"], c["dim"] // 2]), layout=rng.choice([HALF, INTERLEAVED]), scaling=rng.choice([PLAIN, LINEAR, BY_PARTS]))
                else:
                    c |= dict(window=rng.choice([0, 0, _size(rng, 32, 8192)]))
            c["lens"] = rng.randint(100, 1 << 30)
        if _fits(c):
            return c


def _fits(c):
    if c["op"] == "rope":
        return c["tokens"] * c["heads"] * c["dim"] <= 8191 * 40 * 128
    ctx, new = _lengths(c)
    if sum(new) > 140_000 or sum(new) < 1:
        return False
    if c["op"] == "plan":
        return True
    blocks = sum((a + b + c["block"] - 1) // c["block"] for a, b in zip(ctx, new))
    if c["op"] == "append":
        return work(c)["bytes"] <= 2.5e8 and c["reqs"] * max(a + b for a, b in zip(ctx, new)) < 5e7
    longest = max(a + b for a, b in zip(ctx, new))
    return (c["reqs"] * c["q_heads"] * max(new) * longest <= 2.2e9 and c["reqs"] * c["kv_heads"] * longest * c["dim"] <= 1.3e9
            and blocks * c["block"] * c["kv_heads"] * c["dim"] <= 1.3e9)


def _lengths(c):
    """Cached and new tokens of every request: spread over the logarithm; every idle-th request has nothing new."""
    rng = random.Random(c["lens"])
    ctx = [_size(rng, c["ctx_lo"], c["ctx_hi"]) if c["ctx_hi"] > c["ctx_lo"] else c["ctx_lo"] for _ in range(c["reqs"])]
    new = [_size(rng, c["new_lo"], c["new_hi"]) if c["new_hi"] > c["new_lo"] else c["new_lo"] for _ in range(c["reqs"])]
    if c["idle"]:
        new = [0 if i % c["idle"] == c["idle"] - 1 else n for i, n in enumerate(new)]
    return [min(x, c["ctx_hi"]) for x in ctx], [min(x, c["new_hi"]) for x in new]


def _ceil(a, b):
    return -(-a // b)


# ---------------------------------------------------------------- inputs

def _frequencies(c):
    """Radians a token for every pair, in double."""
    rot = c["rot"]
    f = [BASE ** (-2.0 * i / rot) for i in range(rot // 2)]
    if c["scaling"] == LINEAR:
        return [x / 4.0 for x in f]
    if c["scaling"] == BY_PARTS:
        g = [min(1.0, max(0.0, (ORIGINAL * x / (2 * math.pi) - SLOW) / (FAST - SLOW))) for x in f]
        return [a * x + (1 - a) * x / 16.0 for a, x in zip(g, f)]
    return f


def _magnitude(c):
    return 1.0 + 0.1 * math.log(16.0) if c["scaling"] == BY_PARTS else 1.0


def _rope(c):
    from paper_2603_08739_amd import kvpaged
    factor = {PLAIN: 1.0, LINEAR: 4.0, BY_PARTS: 16.0}[c["scaling"]]
    return kvpaged.Rope(c["rot"], base=BASE, layout=c["layout"], scaling=c["scaling"], factor=factor, original_len=ORIGINAL, fast=FAST, slow=SLOW,
                        magnitude=_magnitude(c))


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, dtype):
        return torch.randn(*shape, device="cuda", generator=g).to(dtype)

    s = {"c": c}
    if c["op"] in ("rope", "append"):
        # 45 bits of every pair's frequency in turns a token: exact over any position of a context
        s["turns"] = torch.tensor([round(f / (2 * math.pi) * 2 ** 45) for f in _frequencies(c)], dtype=torch.int64, device="cuda")
        s["rope"] = _rope(c) if own else None
    if c["op"] == "rope":
        wide = normal(c["tokens"], c["heads"] + (16 if c["fused"] else 0), c["dim"], dtype=TYPES[c["dtype"]])
        s["x"] = wide[:, :c["heads"]]
        s["pos"] = torch.randint(0, 131072, (c["tokens"],), device="cuda", generator=g, dtype=torch.int32)
        s["out"] = torch.empty(c["tokens"], c["heads"], c["dim"], device="cuda", dtype=TYPES[c["dtype"]])
        return s

    ctx, new = _lengths(c)
    block, reqs = c["block"], c["reqs"]
    total = sum(new)
    width = max(_ceil(a + b, block) for a, b in zip(ctx, new))
    s |= dict(ctx=torch.tensor(ctx, dtype=torch.int32, device="cuda"), new=torch.tensor(new, dtype=torch.int32, device="cuda"), tokens=total, width=width,
              longest_new=max(new))
    have = (s["ctx"] + block - 1) // block
    want = (s["ctx"] + s["new"] + block - 1) // block
    column = torch.arange(width, device="cuda", dtype=torch.int32)[None]
    if c["op"] == "attn":
        # every block of a request is its own; the pool is in no order
        blocks = sum(_ceil(a + b, block) for a, b in zip(ctx, new))
        pool = torch.randperm(blocks, device="cuda", generator=g, dtype=torch.int32)
        at = torch.cumsum(want, 0) - want
        table = torch.where(column < want[:, None], pool[(at[:, None] + column).clamp(max=blocks - 1)], -1).to(torch.int32)
        if c["window"]:  # the blocks that no new token can see any more were given back
            table = torch.where((column + 1) * block <= (s["ctx"] - c["window"] + 1)[:, None], -1, table).to(torch.int32)
    else:
        # requests share their prefix (blocks 0 .. 63 in some order); the last cached block and all new ones are their own
        need = int((want - have).sum())
        blocks = 64 + reqs + need
        pool = 64 + torch.randperm(blocks - 64, device="cuda", generator=g, dtype=torch.int32)
        s["free"] = pool[reqs:reqs + need].contiguous()
        shared = torch.randint(0, 64, (reqs, width), device="cuda", generator=g, dtype=torch.int32)
        table = torch.where(column < have[:, None], torch.where(column == have[:, None] - 1, pool[:reqs, None], shared), -1).to(torch.int32)
        if need == 0:
            s["free"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        if c["op"] == "append":
            s["table"] = table
            table = _plain_plan(s)["table"]
    s["table"] = table.contiguous()

    heads = c.get("q_heads", 8), c.get("kv_heads", 8)
    if own:
        from paper_2603_08739_amd import kvpaged
        s["plan"] = kvpaged.Plan(reqs, total, block, width, heads[0], heads[1], c.get("dim", 128), max_new=s["longest_new"], window=c.get("window", 0))
    if c["op"] == "plan":
        return s

    q_heads, kv_heads = heads
    dim, dtype, kept = c["dim"], TYPES[c["dtype"]], TYPES[c["cache"]]
    done = _plain_plan(s)
    s |= dict(q_start=done["q_start"], slot=done["slot"], pos=done["pos"], kv_len=done["kv_len"])
    scale = kept == torch.float8_e4m3fn
    s["k_scale"] = torch.rand(kv_heads, device="cuda", generator=g) * 0.02 + 0.02 if scale else None
    s["v_scale"] = torch.rand(kv_heads, device="cuda", generator=g) * 0.02 + 0.02 if scale else None

    def kept_values(blocks, *shape, by):
        # in slices: a long context's values in 32 bits would be four times the cache
        whole = torch.empty(blocks, *shape, device="cuda", dtype=kept)
        step = max(1, (1 << 28) // math.prod(shape))
        for i in range(0, blocks, step):
            x = torch.randn(min(step, blocks - i), *shape, device="cuda", generator=g)
            whole[i:i + step] = ((x / by[:, None, None]).clamp(-448.0, 448.0) if by is not None else x).to(kept)
        return whole

    if c["op"] == "append":
        s["k_cache"] = torch.zeros(blocks, kv_heads, block, dim, device="cuda").to(kept)
        s["v_cache"] = torch.zeros(blocks, kv_heads, dim, block, device="cuda").to(kept)
        fused = normal(total, q_heads + 2 * kv_heads, dim, dtype=dtype)
        s["q"], s["k"], s["v"] = fused[:, :q_heads], fused[:, q_heads:q_heads + kv_heads], fused[:, q_heads + kv_heads:]
        s["q_out"] = torch.empty(total, q_heads, dim, device="cuda", dtype=dtype)
    else:
        s["k_cache"] = kept_values(blocks, kv_heads, block, dim, by=s["k_scale"])
        s["v_cache"] = kept_values(blocks, kv_heads, dim, block, by=s["v_scale"])
        # queries of trained heads are larger than their keys: some rows look at few keys
        s["q"] = (torch.randn(total, q_heads, dim, device="cuda", generator=g) * (1.0 + torch.rand(q_heads, 1, device="cuda", generator=g))).to(dtype)
        s["out"] = torch.empty(total, q_heads, dim, device="cuda", dtype=dtype)
        s["lse"] = torch.empty(total, q_heads, device="cuda", dtype=torch.float32)
    if own:
        s["cache"] = kvpaged.Cache(s["k_cache"], s["v_cache"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        kvpaged.kv_paged_plan(s["plan"], s["ctx"], s["new"], s["table"])
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    s, op = state, state["c"]["op"]
    if not own:
        return {"rope": _plain_rope_case, "plan": _plain_plan, "append": _plain_append, "attn": _plain_attention}[op](s)
    from paper_2603_08739_amd import kvpaged
    if op == "rope":
        return kvpaged.kv_rope_apply(s["rope"], s["x"], s["pos"], out=s["out"], backward=s["c"]["backward"])
    p = s["plan"]
    if op == "plan":
        kvpaged.kv_paged_plan(p, s["ctx"], s["new"], s["table"], free_list=s["free"])
        return dict(table=s["table"], q_start=p.q_start, kv_len=p.kv_len, slot=p.slot, pos=p.pos, result=p.result)
    if op == "append":
        kvpaged.kv_paged_append(p, s["cache"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rope=s["rope"])
        return dict(q=s["q_out"], k_cache=s["k_cache"], v_cache=s["v_cache"])
    kvpaged.kv_paged_attention(p, s["cache"], s["q"], out=s["out"], lse=s["lse"])
    return dict(out=s["out"], lse=s["lse"])


# ---------------------------------------------------------------- the plain forms

def _plain_rope(c, turns, x, pos, backward=False):
    """x [tokens, heads, dim] in 32 bits."""
    x = x.float()
    part = ((pos.long()[:, None] * turns) & (2 ** 45 - 1)).float() * 2.0 ** -45
    angle = part * (2 * math.pi)
    cos, sin = (torch.cos(angle) * _magnitude(c))[:, None], (torch.sin(angle) * _magnitude(c))[:, None]
    if backward:
        sin = -sin
    rot = c["rot"]
    if c["layout"] == HALF:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_rope_case(s):
    return _plain_rope(s["c"], s["turns"], s["x"], s["pos"], s["c"]["backward"]).to(s["x"].dtype)


def _plain_plan(s):
    c, ctx, new, table, block, total = s["c"], s["ctx"], s["new"], s["table"], s["c"]["block"], s["tokens"]
    ends = torch.cumsum(new, 0)
    q_start = torch.cat([torch.zeros_like(ends[:1]), ends]).to(torch.int32)
    kv_len = ctx + new
    if "free" in s:
        have, want = (ctx + block - 1) // block, (kv_len + block - 1) // block
        need = want - have
        first = torch.cumsum(need, 0) - need
        column = torch.arange(s["width"], device=ctx.device, dtype=torch.int32)[None]
        place = first[:, None] + column - have[:, None]
        fresh = torch.where(place < s["free"].numel(), s["free"][place.clamp(0, s["free"].numel() - 1)], -1)
        table = torch.where((column >= have[:, None]) & (column < want[:, None]), fresh, table)
        needed = need.sum()
    else:
        needed = torch.zeros_like(ends[0])
    token = torch.arange(total, device=ctx.device)
    req = torch.searchsorted(ends, token, right=True)
    pos = (ctx[req] + token - q_start[req]).to(torch.int32)
    entry = table[req, (pos // block).long()].long()
    slot = torch.where(entry >= 0, entry * block + pos % block, -1)
    result = torch.stack([ends[-1], needed, needed, torch.zeros_like(needed)]).to(torch.int32)
    return dict(table=table, q_start=q_start, kv_len=kv_len, slot=slot, pos=pos, result=result)


def _plain_append(s):
    c, block = s["c"], s["c"]["block"]
    q = _plain_rope(c, s["turns"], s["q"], s["pos"])
    k = _plain_rope(c, s["turns"], s["k"], s["pos"])
    v = s["v"].float()
    if s["k_scale"] is not None:
        k = (k / s["k_scale"][:, None]).clamp(-448.0, 448.0)
        v = (v / s["v_scale"][:, None]).clamp(-448.0, 448.0)
    page, offset = s["slot"] // block, s["slot"] % block
    bits = (lambda x: x.view(torch.int8)) if s["k_scale"] is not None else (lambda x: x)
    bits(s["k_cache"])[page, :, offset] = bits(k.to(s["k_cache"].dtype))
    bits(s["v_cache"])[page, :, :, offset] = bits(v.to(s["v_cache"].dtype))
    return dict(q=q.to(s["q"].dtype), k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_attention(s):
    c, table, block = s["c"], s["table"], s["c"]["block"]
    reqs, kv_heads, dim = c["reqs"], c["kv_heads"], c["dim"]
    group, n, keys = c["q_heads"] // kv_heads, s["longest_new"], s["width"] * block
    pages = table.clamp(min=0).long()
    k = s["k_cache"][pages].float().permute(0, 2, 1, 3, 4).reshape(reqs, kv_heads, keys, dim)
    v = s["v_cache"][pages].float().permute(0, 2, 1, 4, 3).reshape(reqs, kv_heads, keys, dim)
    if s["k_scale"] is not None:
        k = k * s["k_scale"][:, None, None]
        v = v * s["v_scale"][:, None, None]
    step = torch.arange(n, device=table.device)
    row = (s["q_start"][:-1, None] + step).clamp(max=s["tokens"] - 1).long()  # rows past a request's last one are dropped below
    q = s["q"][row].float().reshape(reqs, n, kv_heads, group, dim).permute(0, 2, 3, 1, 4).reshape(reqs, kv_heads, group * n, dim)
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()).reshape(reqs, kv_heads, group, n, keys) * dim ** -0.5
    key = torch.arange(keys, device=table.device)
    at = s["ctx"][:, None] + step
    seen = (key <= at[..., None]) & (key < s["kv_len"][:, None, None]) & (table >= 0).repeat_interleave(block, 1)[:, None]
    if c["window"]:
        seen = seen & (key > at[..., None] - c["window"])
    scores = scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    weights = scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = weights.sum(-1, keepdim=True)
    lse = (top + total.log())[..., 0]
    out = torch.matmul(weights.reshape(reqs, kv_heads, group * n, keys), v).reshape(reqs, kv_heads, group, n, dim) / total.clamp(min=1e-38)
    token = torch.arange(s["tokens"], device=table.device)
    req = torch.searchsorted(s["q_start"][1:], token, right=True)
    place = token - s["q_start"][req]
    out = out.permute(0, 3, 1, 2, 4).reshape(reqs, n, c["q_heads"], dim)[req, place]
    lse = lse.permute(0, 3, 1, 2).reshape(reqs, n, c["q_heads"])[req, place]
    return dict(out=out.to(s["q"].dtype), lse=lse)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "rope":
        size = c["tokens"] * c["heads"] * c["dim"]
        return {"bytes": 4 * size + 4 * c["tokens"], "flops": 3 * c["tokens"] * c["heads"] * c["rot"]}
    ctx, new = _lengths(c)
    block, total = c["block"], sum(new)
    fresh = sum(_ceil(a + b, block) - _ceil(a, block) for a, b in zip(ctx, new))
    if c["op"] == "plan":
        # slots, positions; new table entries and what they are taken from; lengths, starts and ends
        return {"bytes": 12 * total + 8 * fresh + 16 * c["reqs"], "flops": 0}
    kept = 1 if c["cache"] == "fp8" else 2
    q, kv = total * c["q_heads"] * c["dim"], total * c["kv_heads"] * c["dim"]
    if c["op"] == "append":
        return {"bytes": 4 * q + 2 * kv * (2 + kept) + 12 * total, "flops": 3 * total * (c["q_heads"] + c["kv_heads"]) * c["rot"]}
    window = c["window"] or 1 << 40
    pairs = keys = 0
    for a, b in zip(ctx, new):
        if b:
            short = min(b, max(0, window - a - 1))  # tokens that see everything before them
            pairs += short * a + short * (short + 1) // 2 + (b - short) * (window if b > short else 0)
            keys += a + b - max(0, a + 1 - window)
    return {"bytes": 4 * q + 4 * total * c["q_heads"] + 2 * keys * c["kv_heads"] * c["dim"] * kept, "flops": 4 * pairs * c["q_heads"] * c["dim"]}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rope":
        return _exact_rope(c, s["x"], s["pos"], c["backward"])
    ctx, new = _lengths(c)
    if c["op"] == "plan":
        return None
    starts = [sum(new[:r]) for r in range(len(new))]
    if c["op"] == "append":
        k, v = _exact_rope(c, s["k"], s["pos"], False), s["v"].double()
        if s["k_scale"] is not None:
            k, v = (k / s["k_scale"].double()[:, None]).clamp(-448, 448), (v / s["v_scale"].double()[:, None]).clamp(-448, 448)
        k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
        table = s["table"].cpu().tolist()
        for r, (a, b) in enumerate(zip(ctx, new)):
            done = 0
            while done < b:  # block by block
                at = a + done
                many = min(c["block"] - at % c["block"], b - done)
                page, i, t = table[r][at // c["block"]], at % c["block"], starts[r] + done
                k_cache[page, :, i:i + many] = k[t:t + many].transpose(0, 1)
                v_cache[page, :, :, i:i + many] = v[t:t + many].permute(1, 2, 0)
                done += many
        return dict(q=_exact_rope(c, s["q"], s["pos"], False), k_cache=k_cache, v_cache=v_cache)
    group = c["q_heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    for r, (a, b) in enumerate(zip(ctx, new)):
        if not b:
            continue
        low = max(0, a + 1 - c["window"]) if c["window"] else 0
        first = low // c["block"]
        pages = s["table"][r, first:_ceil(a + b, c["block"])].long()
        key = torch.arange(first * c["block"], a + b, device="cuda")
        at = torch.arange(a, a + b, device="cuda")[:, None]
        hidden = (key > at) | (key <= at - c["window"]) if c["window"] else key > at
        for j in range(c["kv_heads"]):
            k = s["k_cache"][pages, j].double().reshape(-1, c["dim"])[:len(key)]
            v = s["v_cache"][pages, j].double().transpose(1, 2).reshape(-1, c["dim"])[:len(key)]
            if s["k_scale"] is not None:
                k, v = k * s["k_scale"][j].double(), v * s["v_scale"][j].double()
            for h in range(j * group, (j + 1) * group):
                logit = (s["q"][starts[r]:starts[r] + b, h].double() @ k.T / math.sqrt(c["dim"])).masked_fill_(hidden, -math.inf)
                lse[starts[r]:starts[r] + b, h] = torch.logsumexp(logit, -1)
                out[starts[r]:starts[r] + b, h] = torch.softmax(logit, -1) @ v
    return dict(out=out, lse=lse)


def _exact_rope(c, x, pos, backward):
    f = torch.tensor(_frequencies(c), dtype=torch.float64, device=x.device)
    # multiplication by a complex number of the pair's angle
    turn = torch.polar(torch.full_like(f, _magnitude(c)) + 0 * pos[:, None], (-1.0 if backward else 1.0) * pos.double()[:, None] * f)
    x = x.double()
    rot = c["rot"]
    pairs = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) if c["layout"] == HALF else torch.complex(x[..., 0:rot:2], x[..., 1:rot:2])
    pairs = pairs * turn[:, None]
    done = torch.cat([pairs.real, pairs.imag], -1) if c["layout"] == HALF else torch.stack([pairs.real, pairs.imag], -1).flatten(-2)
    return torch.cat([done, x[..., rot:]], -1)
