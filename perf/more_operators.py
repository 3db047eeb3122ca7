"""Performance cases of a paged KV cache held in 8 bits with a scale for each block and head.

  write  one step's queries and keys turned, keys and values quantised as they are written, a block's scale found from what goes into it (and raised,
         with its earlier tokens, where new ones are larger); the blocks that the step touched are read back
  read   the tokens of every request read back from the cache into contiguous rows of 16 bits
  attn   attention of the new tokens of every request over its cached blocks

Held numbers are e4m3 ("fp8") or whole numbers of -127 .. 127 ("i8"); a held number stands for itself times the scale of its block and head.  Block
sizes and lengths are those of the traces the framework evaluates: 16-token blocks for prompts and chats, 64-token blocks and contexts of 8,192 to
131,072 tokens for documents.  Head counts are generic.  Lengths follow from the case (`lens` seeds them), every value in the tensors from
prepare()'s seed.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn, "i8": torch.int8}
MOST = {"fp8": 448.0, "i8": 127.0}
HALF, INTERLEAVED = 0, 1
BASE = 500_000.0


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # one decoding step of 64 chats: latency, and blocks whose scale has to rise
        dict(name="write_step", op="write", reqs=64, new_lo=1, new_hi=1, ctx_lo=100, ctx_hi=8000, block=16, idle=0, q_heads=32, kv_heads=8, dim=128,
             rot=128, layout=HALF, dtype="bf16", cache="i8", lens=1),
        # prompts of a long-context service, 64-token blocks
        dict(name="write_chunk", op="write", reqs=24, new_lo=20, new_hi=1500, ctx_lo=1, ctx_hi=131072, block=64, idle=0, q_heads=32, kv_heads=8, dim=128,
             rot=128, layout=HALF, dtype="bf16", cache="i8", lens=2),
        # ragged prompts in blocks of 16 tokens, some requests idle, interleaved layout, part of the head turned
        dict(name="write_ragged_fp8", op="write", reqs=37, new_lo=1, new_hi=400, ctx_lo=1, ctx_hi=8192, block=16, idle=8, q_heads=24, kv_heads=4, dim=128,
             rot=64, layout=INTERLEAVED, dtype="f16", cache="fp8", lens=3),
        # three short chats leave the cache: the smallest read
        dict(name="read_chats", op="read", reqs=3, ctx_lo=20, ctx_hi=700, block=16, kv_heads=8, dim=128, dtype="bf16", cache="i8", lens=4),
        # prefixes of many prompts, to go on in another cache
        dict(name="read_prompts", op="read", reqs=64, ctx_lo=100, ctx_hi=8192, block=16, kv_heads=8, dim=64, dtype="f16", cache="i8", lens=5),
        # long documents
        dict(name="read_documents_fp8", op="read", reqs=4, ctx_lo=8192, ctx_hi=131071, block=64, kv_heads=8, dim=128, dtype="bf16", cache="fp8", lens=6),
        # a single chat generates: the smallest attention
        dict(name="attn_single", op="attn", reqs=1, new_lo=1, new_hi=1, ctx_lo=500, ctx_hi=500, block=16, idle=0, q_heads=32, kv_heads=8, dim=128,
             window=0, dtype="bf16", cache="i8", lens=7),
        # one decoding step of 64 chats of very different lengths
        dict(name="attn_step", op="attn", reqs=64, new_lo=1, new_hi=1, ctx_lo=100, ctx_hi=16000, block=16, idle=0, q_heads=32, kv_heads=8, dim=128,
             window=0, dtype="bf16", cache="i8", lens=8),
        # eight long documents are answered
        dict(name="attn_long_fp8", op="attn", reqs=8, new_lo=1, new_hi=1, ctx_lo=8192, ctx_hi=131071, block=64, idle=0, q_heads=64, kv_heads=8, dim=128,
             window=0, dtype="bf16", cache="fp8", lens=9),
        # chunks of prompts and single tokens together, over cached prefixes, sliding window whose older blocks are gone
        dict(name="attn_mixed", op="attn", reqs=12, new_lo=1, new_hi=1300, ctx_lo=50, ctx_hi=12000, block=16, idle=5, q_heads=24, kv_heads=4, dim=64,
             window=4096, dtype="f16", cache="i8", lens=21),
        # a long prompt after a short cached prefix: bound by the matrix cores
        dict(name="attn_prompt", op="attn", reqs=1, new_lo=7777, new_hi=7777, ctx_lo=300, ctx_hi=300, block=16, idle=0, q_heads=32, kv_heads=8, dim=128,
             window=0, dtype="bf16", cache="i8", lens=11),
        # the same from an e4m3 cache in blocks of 64
        dict(name="attn_prompt_fp8", op="attn", reqs=1, new_lo=5003, new_hi=5003, ctx_lo=2000, ctx_hi=2000, block=64, idle=0, q_heads=32, kv_heads=8, dim=128,
             window=0, dtype="f16", cache="fp8", lens=12),
    ]


def _size(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    while True:
        op = rng.choice(["write", "read", "attn", "attn"])
        decode = rng.random() < 0.5
        kv_heads, dim, dtype = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 256]), rng.choice(["bf16", "f16"])
        c = dict(op=op, block=rng.choice([16, 32, 64]), kv_heads=kv_heads, dim=dim, dtype=dtype, cache=rng.choice(["i8", "fp8"]), lens=rng.randint(100, 1 << 30))
        if op == "read":
            ctx_hi = _size(rng, 16, 131071)
            c |= dict(reqs=_size(rng, 1, 128), ctx_lo=rng.randint(1, ctx_hi), ctx_hi=ctx_hi)
        else:
            reqs = _size(rng, 1, 64 if decode else 16) if op == "attn" else _size(rng, 1, 1000)
            new_hi = 1 if decode else _size(rng, 2, 4096 if op == "attn" else 1500)
            ctx_hi = _size(rng, 16, 131071 if decode else 16000)
            c |= dict(reqs=reqs, new_lo=1, new_hi=new_hi, ctx_lo=rng.randint(1, ctx_hi), ctx_hi=ctx_hi, idle=rng.choice([0, 0, 5]) if reqs > 5 else 0,
                      q_heads=kv_heads * rng.choice([1, 4, 6, 8]))
            if op == "write":
                c |= dict(rot=rng.choice([dim, dim // 2]), layout=rng.choice([HALF, INTERLEAVED]))
            else:
                c |= dict(window=rng.choice([0, 0, _size(rng, 32, 8192)]))
        if _fits(c):
            return c


def _fits(c):
    """No more than the largest listed cases of its kind, and a plain form that a card holds three times over."""
    ctx, new = _lengths(c)
    blocks = sum(_ceil(a + b, c["block"]) for a, b in zip(ctx, new))
    longest = max(a + b for a, b in zip(ctx, new))
    if c["op"] == "read":
        return work(c)["bytes"] <= 1.6e9
    if sum(new) > 140_000 or sum(new) < 1:
        return False
    if c["op"] == "write":
        return work(c)["bytes"] <= 3.5e8 and c["reqs"] * longest < 5e7
    return (c["reqs"] * c["q_heads"] * max(new) * longest <= 2.2e9 and c["reqs"] * c["kv_heads"] * longest * c["dim"] <= 1.3e9
            and blocks * c["block"] * c["kv_heads"] * c["dim"] <= 1.3e9)


def _lengths(c):
    """Cached and new tokens of every request: spread over the logarithm; every idle-th request has nothing new."""
    rng = random.Random(c["lens"])
    ctx = [_size(rng, c["ctx_lo"], c["ctx_hi"]) if c["ctx_hi"] > c["ctx_lo"] else c["ctx_lo"] for _ in range(c["reqs"])]
    ctx = [min(x, c["ctx_hi"]) for x in ctx]
    if c["op"] == "read":
        return ctx, [0] * c["reqs"]
    new = [_size(rng, c["new_lo"], c["new_hi"]) if c["new_hi"] > c["new_lo"] else c["new_lo"] for _ in range(c["reqs"])]
    if c["idle"]:
        new = [0 if i % c["idle"] == c["idle"] - 1 else n for i, n in enumerate(new)]
    return ctx, [min(x, c["new_hi"]) for x in new]


def _ceil(a, b):
    return -(-a // b)


def _rows(c, ctx, new):
    """What is read back of every request: first position and number of tokens.  A write's: the blocks that it touched."""
    if c["op"] == "read":
        return [0] * len(ctx), ctx
    return [a // c["block"] * c["block"] for a in ctx], [a % c["block"] + b if b else 0 for a, b in zip(ctx, new)]


# ---------------------------------------------------------------- inputs

def _frequencies(c):
    """Radians a token for every pair, in double."""
    return [BASE ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)]


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    i32 = dict(dtype=torch.int32, device="cuda")
    ctx, new = _lengths(c)
    block, reqs, kv_heads, dim, dtype, kept = c["block"], c["reqs"], c["kv_heads"], c["dim"], TYPES[c["dtype"]], TYPES[c["cache"]]
    q_heads = c.get("q_heads", kv_heads)
    total = sum(new)
    width = max(_ceil(a + b, block) for a, b in zip(ctx, new))
    starts = [sum(new[:r]) for r in range(reqs + 1)]
    s = dict(c=c, ctx=torch.tensor(ctx, **i32), new=torch.tensor(new, **i32), tokens=total, width=width, longest_new=max(new),
             q_start=torch.tensor(starts, **i32))
    s["kv_len"] = s["ctx"] + s["new"]
    want = (s["kv_len"] + block - 1) // block
    column = torch.arange(width, **i32)[None]
    if c["op"] == "write":
        # requests share their prefix (blocks 0 .. 63 in some order); the block that a context ends in and the new ones are their own
        kept_whole = s["ctx"] // block
        mine = want - kept_whole
        blocks = 64 + sum(_ceil(a + b, block) - a // block for a, b in zip(ctx, new))
        pool = 64 + torch.randperm(blocks - 64, generator=g, **i32)
        at = (torch.cumsum(mine, 0) - mine)[:, None] + column - kept_whole[:, None]
        shared = torch.randint(0, 64, (reqs, width), generator=g, **i32)
        table = torch.where(column < kept_whole[:, None], shared, torch.where(column < want[:, None], pool[at.clamp(0, blocks - 65)], -1))
    else:
        # every block of a request is its own; the pool is in no order
        blocks = sum(_ceil(a + b, block) for a, b in zip(ctx, new))
        pool = torch.randperm(blocks, generator=g, **i32)
        at = torch.cumsum(want, 0) - want
        table = torch.where(column < want[:, None], pool[(at[:, None] + column).clamp(max=blocks - 1)], -1)
        if c.get("window"):  # the blocks that no new token can see any more were given back
            table = torch.where((column + 1) * block <= (s["ctx"] - c["window"] + 1)[:, None], -1, table)
    s["table"] = table.to(torch.int32).contiguous()

    # held numbers as a quantised cache has them: normal values whose largest is the type's, blocks of different sizes
    def held(*shape):
        whole = torch.empty(blocks, *shape, device="cuda", dtype=kept)
        step = max(1, (1 << 28) // math.prod(shape))
        for i in range(0, blocks, step):
            x = torch.randn(min(step, blocks - i), *shape, device="cuda", generator=g) * (MOST[c["cache"]] / 4)
            x = x.clamp(-MOST[c["cache"]], MOST[c["cache"]])
            whole[i:i + step] = (x.round() if c["cache"] == "i8" else x).to(kept)
        return whole

    s["k_cache"], s["v_cache"] = held(kv_heads, block, dim), held(kv_heads, dim, block)
    scales = lambda: (torch.rand(blocks, kv_heads, device="cuda", generator=g) * 3.0 + 1.5) / MOST[c["cache"]]  # noqa: E731
    s["k_scale"], s["v_scale"] = scales(), scales()

    if c["op"] != "attn":
        first, rows = _rows(c, ctx, new)
        s["first"], s["rows"] = torch.tensor(first, **i32), sum(rows)
        s["row_start"] = torch.tensor([sum(rows[:r]) for r in range(reqs + 1)], **i32)
        s["k_out"], s["v_out"] = (torch.empty(s["rows"], kv_heads, dim, device="cuda", dtype=dtype) for _ in range(2))
    if c["op"] == "write":
        # 45 bits of every pair's frequency in turns a token: exact over any position of a context
        s["turns"] = torch.tensor([round(f / (2 * math.pi) * 2 ** 45) for f in _frequencies(c)], dtype=torch.int64, device="cuda")
        fused = torch.randn(total, q_heads + 2 * kv_heads, dim, device="cuda", generator=g).to(dtype)
        s["q"], s["k"], s["v"] = fused[:, :q_heads], fused[:, q_heads:q_heads + kv_heads], fused[:, q_heads + kv_heads:]
        s["q_out"] = torch.empty(total, q_heads, dim, device="cuda", dtype=dtype)
    if c["op"] == "attn":
        # queries of trained heads are larger than their keys: some rows look at few keys
        s["q"] = (torch.randn(total, q_heads, dim, device="cuda", generator=g) * (1.0 + torch.rand(q_heads, 1, device="cuda", generator=g))).to(dtype)
        s["out"] = torch.empty(total, q_heads, dim, device="cuda", dtype=dtype)
        s["lse"] = torch.empty(total, q_heads, device="cuda", dtype=torch.float32)
    if own:
        from paper_2603_08739_amd import kvpaged
        s["plan"] = kvpaged.Plan(reqs, max(total, 1), block, width, q_heads, kv_heads, dim, max_new=max(s["longest_new"], 1), window=c.get("window", 0))
        s["cache"] = kvpaged.Cache(s["k_cache"], s["v_cache"], k_scale=s["k_scale"], v_scale=s["v_scale"], block_scales=True)
        s["rope"] = kvpaged.Rope(c["rot"], base=BASE, layout=c["layout"]) if c["op"] == "write" else None
        kvpaged.kv_paged_plan(s["plan"], s["ctx"], s["new"], s["table"])
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    s, op = state, state["c"]["op"]
    if not own:
        return {"write": _plain_write, "read": _plain_read, "attn": _plain_attention}[op](s)
    from paper_2603_08739_amd import kvpaged
    if op == "attn":
        kvpaged.kv_paged_attention(s["plan"], s["cache"], s["q"], out=s["out"], lse=s["lse"])
        return dict(out=s["out"], lse=s["lse"])
    if op == "write":
        kvpaged.kv_paged_append(s["plan"], s["cache"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rope=s["rope"])
    kvpaged.kv_paged_read(s["plan"], s["cache"], s["row_start"], first=s["first"], k=s["k_out"], v=s["v_out"])
    if op == "read":
        return dict(k=s["k_out"], v=s["v_out"])
    return dict(q=s["q_out"], k_scale=s["k_scale"], v_scale=s["v_scale"], k=s["k_out"], v=s["v_out"])


# ---------------------------------------------------------------- the plain forms

def _plain_rope(c, turns, x, pos):
    """x [tokens, heads, dim] in 32 bits."""
    x = x.float()
    part = ((pos.long()[:, None] * turns) & (2 ** 45 - 1)).float() * 2.0 ** -45
    angle = part * (2 * math.pi)
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    rot = c["rot"]
    if c["layout"] == HALF:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _to_held(c, x):
    """Numbers in units of their scale to the held type, to nearest even."""
    x = x.clamp(-MOST[c["cache"]], MOST[c["cache"]])
    return (x.round() if c["cache"] == "i8" else x).to(TYPES[c["cache"]])


def _bits(x):
    return x.view(torch.int8)


def _plain_quantised(s, x, cache, scale, by_token):
    """Writes x [tokens, heads, dim] (32 bits) into its slots; `by_token` puts a cache's tokens before its elements."""
    c, block = s["c"], s["c"]["block"]
    token = torch.arange(s["tokens"], device=x.device)
    req = torch.searchsorted(s["q_start"][1:], token, right=True)
    pos = (s["ctx"][req] + token - s["q_start"][req]).long()
    page, offset = s["table"][req, pos // block].long(), pos % block
    # the largest magnitude that goes into each block
    most = torch.zeros_like(scale).scatter_reduce(0, page[:, None].expand(-1, scale.shape[1]), x.abs().amax(-1), "amax")
    need = most / torch.full_like(most, MOST[c["cache"]])
    # the block that a request's context ends in keeps its scale, doubled until the new tokens fit
    edge = s["table"].gather(1, (s["ctx"] // block).clamp(max=s["width"] - 1).long()[:, None])[:, 0].clamp(min=0).long()
    open_ = (s["ctx"] % block > 0) & (s["new"] > 0)
    old, want = scale[edge], need[edge]
    (m, e), (m_want, e_want) = torch.frexp(old), torch.frexp(want)
    rise = torch.where(want > old, e_want - e + (m_want > m), torch.zeros_like(e))
    grown = torch.ldexp(old, rise)
    touched = torch.zeros(scale.shape[0], dtype=torch.bool, device=x.device).index_fill(0, page, True)
    fresh = torch.where(touched[:, None], need, scale)
    fresh[edge] = torch.where(open_[:, None], grown, fresh[edge])
    # its earlier tokens in the new unit
    factor = torch.where(open_[:, None], torch.ldexp(torch.ones_like(old), -rise), 1.0)
    _bits(cache)[edge] = _bits(_to_held(c, cache[edge].float() * factor[:, :, None, None]))
    scale.copy_(fresh)
    inverse = torch.where(scale > 0, torch.reciprocal(scale), 2.0 ** -126)
    _bits(by_token(cache))[page, :, offset] = _bits(_to_held(c, x * inverse[page][:, :, None]))


def _plain_write(s):
    c = s["c"]
    token = torch.arange(s["tokens"], device="cuda")
    req = torch.searchsorted(s["q_start"][1:], token, right=True)
    pos = s["ctx"][req] + token - s["q_start"][req]
    q = _plain_rope(c, s["turns"], s["q"], pos)
    _plain_quantised(s, _plain_rope(c, s["turns"], s["k"], pos), s["k_cache"], s["k_scale"], lambda x: x)
    _plain_quantised(s, s["v"].float(), s["v_cache"], s["v_scale"], lambda x: x.transpose(2, 3))
    return dict(q=q.to(s["q"].dtype), k_scale=s["k_scale"], v_scale=s["v_scale"], **_plain_read(s))


def _plain_read(s):
    block = s["c"]["block"]
    row = torch.arange(s["rows"], device="cuda")
    req = torch.searchsorted(s["row_start"][1:], row, right=True)
    pos = (s["first"][req] + row - s["row_start"][req]).long()
    page, offset = s["table"][req, pos // block].long(), pos % block
    k = _bits(s["k_cache"])[page, :, offset].view(s["k_cache"].dtype).float() * s["k_scale"][page][:, :, None]
    v = _bits(s["v_cache"])[page, :, :, offset].view(s["v_cache"].dtype).float() * s["v_scale"][page][:, :, None]
    return dict(k=k.to(s["k_out"].dtype), v=v.to(s["v_out"].dtype))


def _plain_attention(s):
    c, table, block = s["c"], s["table"], s["c"]["block"]
    reqs, kv_heads, dim = c["reqs"], c["kv_heads"], c["dim"]
    group, n, keys = c["q_heads"] // kv_heads, s["longest_new"], s["width"] * block
    pages = table.clamp(min=0).long()
    k = (s["k_cache"][pages].float() * s["k_scale"][pages][..., None, None]).permute(0, 2, 1, 3, 4).reshape(reqs, kv_heads, keys, dim)
    v = (s["v_cache"][pages].float() * s["v_scale"][pages][..., None, None]).permute(0, 2, 1, 4, 3).reshape(reqs, kv_heads, keys, dim)
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
    ctx, new = _lengths(c)
    block, width = c["block"], c["kv_heads"] * c["dim"]
    if c["op"] != "attn":
        first, rows = _rows(c, ctx, new)
        parts = sum(_ceil(a + n, block) - a // block for a, n in zip(first, rows))
        # held numbers, scales, 16-bit rows
        b = 2 * (3 * sum(rows) * width + 4 * parts * c["kv_heads"]) + 4 * parts
        if c["op"] == "read":
            return {"bytes": b, "flops": 2 * sum(rows) * width}
        total, touched = sum(new), sum(_ceil(a + n, block) - a // block for a, n in zip(ctx, new) if n)
        q = total * c["q_heads"] * c["dim"]
        b += 4 * q + 2 * (3 * total * width + 4 * touched * c["kv_heads"]) + 12 * total
        return {"bytes": b, "flops": 3 * total * (c["q_heads"] + c["kv_heads"]) * c["rot"] + 6 * total * width}
    window = c["window"] or 1 << 40
    pairs = keys = 0
    for a, b in zip(ctx, new):
        if b:
            short = min(b, max(0, window - a - 1))  # tokens that see everything before them
            pairs += short * a + short * (short + 1) // 2 + (b - short) * (window if b > short else 0)
            keys += a + b - max(0, a + 1 - window)
    q = sum(new) * c["q_heads"]
    return {"bytes": 4 * q * c["dim"] + 4 * q + 2 * keys * width + 8 * c["kv_heads"] * keys // block, "flops": 4 * pairs * c["q_heads"] * c["dim"]}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    c, s = case, prepare(case, seed)
    ctx, new = _lengths(c)
    block, dim = c["block"], c["dim"]
    k_scale, v_scale = s["k_scale"].double(), s["v_scale"].double()
    if c["op"] != "attn":
        k_held, v_held = s["k_cache"].double(), s["v_cache"].double()
        table = s["table"].cpu().tolist()
        starts = s["q_start"].tolist()
        if c["op"] == "write":
            pos = torch.cat([torch.arange(a, a + b, device="cuda") for a, b in zip(ctx, new)])
            q, k, v = _exact_rope(c, s["q"], pos), _exact_rope(c, s["k"], pos), s["v"].double()
            for r, (a, b) in enumerate(zip(ctx, new)):
                done = 0
                while done < b:  # block by block
                    i = (a + done) % block
                    many = min(block - i, b - done)
                    page, t = table[r][(a + done) // block], starts[r] + done
                    _exact_block(c, k_held[page], k_scale[page], k[t:t + many].transpose(0, 1), i)
                    _exact_block(c, v_held[page].transpose(1, 2), v_scale[page], v[t:t + many].transpose(0, 1), i)
                    done += many
        ks, vs = [], []
        for r, (a, n) in enumerate(zip(*_rows(c, ctx, new))):
            if n:
                pages = torch.tensor(table[r][a // block:_ceil(a + n, block)], device="cuda")
                ks.append((k_held[pages] * k_scale[pages][..., None, None]).transpose(1, 2).flatten(0, 1)[:n])
                vs.append((v_held[pages] * v_scale[pages][..., None, None]).permute(0, 3, 1, 2).flatten(0, 1)[:n])
        back = dict(k=torch.cat(ks), v=torch.cat(vs))
        return back if c["op"] == "read" else dict(q=q, k_scale=k_scale, v_scale=v_scale, **back)
    group = c["q_heads"] // c["kv_heads"]
    starts = s["q_start"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    for r, (a, b) in enumerate(zip(ctx, new)):
        if not b:
            continue
        low = max(0, a + 1 - c["window"]) if c["window"] else 0
        first = low // block
        pages = s["table"][r, first:_ceil(a + b, block)].long()
        key = torch.arange(first * block, a + b, device="cuda")
        at = torch.arange(a, a + b, device="cuda")[:, None]
        hidden = (key > at) | (key <= at - c["window"]) if c["window"] else key > at
        for j in range(c["kv_heads"]):
            k = (s["k_cache"][pages, j].double() * k_scale[pages, j][:, None, None]).reshape(-1, dim)[:len(key)]
            v = (s["v_cache"][pages, j].double() * v_scale[pages, j][:, None, None]).transpose(1, 2).reshape(-1, dim)[:len(key)]
            for h in range(j * group, (j + 1) * group):
                logit = (s["q"][starts[r]:starts[r] + b, h].double() @ k.T / math.sqrt(dim)).masked_fill_(hidden, -math.inf)
                lse[starts[r]:starts[r] + b, h] = torch.logsumexp(logit, -1)
                out[starts[r]:starts[r] + b, h] = torch.softmax(logit, -1) @ v
    return dict(out=out, lse=lse)


def _exact_block(c, held, scale, x, at):
    """x [heads, n, dim] into places at .. at + n - 1 of a block: held [heads, block, dim] and scale [heads] are changed."""
    most = MOST[c["cache"]]
    need = x.abs().amax((1, 2)) / most
    if at:
        rise = torch.ceil(torch.log2(need / scale)).clamp(min=0)
        held[:, :at] = _exact_round(c, held[:, :at] * torch.exp2(-rise)[:, None, None])
        scale *= torch.exp2(rise)
    else:
        scale.copy_(need)
    held[:, at:at + x.shape[1]] = _exact_round(c, x / scale[:, None, None])


def _exact_round(c, x):
    x = x.clamp(-MOST[c["cache"]], MOST[c["cache"]])
    if c["cache"] == "i8":
        return x.round()
    # e4m3: spacing 2^-3 of the power of two below, 2^-9 at the least
    spacing = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return (x / spacing).round() * spacing


def _exact_rope(c, x, pos):
    f = torch.tensor(_frequencies(c), dtype=torch.float64, device=x.device)
    # multiplication by a complex number of the pair's angle
    turn = torch.polar(torch.ones_like(f) + 0 * pos[:, None], pos.double()[:, None] * f)
    x = x.double()
    rot = c["rot"]
    pairs = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) if c["layout"] == HALF else torch.complex(x[..., 0:rot:2], x[..., 1:rot:2])
    pairs = pairs * turn[:, None]
    done = torch.cat([pairs.real, pairs.imag], -1) if c["layout"] == HALF else torch.stack([pairs.real, pairs.imag], -1).flatten(-2)
    return torch.cat([done, x[..., rot:]], -1)
