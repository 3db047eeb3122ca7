"""The paged-cache operators by their definitions: one request, one token, one key
at a time where that is bearable, in 64 bits.  Test infrastructure only; shares
nothing with the HIP library.  Tensors may live on either device."""
from __future__ import annotations

import math

import torch


def plan(ctx, new, table, free, block, max_tokens, max_blocks, max_new):
    """Lists in, lists out: table, q_start, kv_len, slot, pos, result."""
    table = [list(r) for r in table]
    flags, start, needed, taken = 0, [0], 0, 0
    kv_len, slot, pos = [], [], []
    dropped = False
    for r, (c, n) in enumerate(zip(ctx, new)):
        if c < 0 or n < 0 or n > max_new or c + n > max_blocks * block:
            c = n = 0
            flags |= 1
        if dropped or start[-1] + n > max_tokens:
            dropped, n = True, 0
            flags |= 2
        kv_len.append(c + n)
        if free is not None:
            for col in range(-(-c // block), -(-(c + n) // block)):
                if needed < len(free):
                    table[r][col] = free[needed]
                    taken += 1
                else:
                    table[r][col] = -1
                    flags |= 4
                needed += 1
        for p in range(c, c + n):
            page = table[r][p // block]
            pos.append(p)
            slot.append(page * block + p % block if page >= 0 else -1)
        start.append(start[-1] + n)
    slot += [-1] * (max_tokens - len(slot))
    pos += [0] * (max_tokens - len(pos))
    return table, start, kv_len, slot, pos, [start[-1], needed, taken, flags]


def frequencies(rot, base, scaling=0, factor=1.0, original_len=0, fast=32.0, slow=1.0):
    f = []
    for i in range(rot // 2):
        x = base ** (-2.0 * i / rot)
        if scaling == 1:
            x /= factor
        if scaling == 2:
            g = (original_len * x / (2 * math.pi) - slow) / (fast - slow)
            g = min(1.0, max(0.0, g))
            x = g * x + (1 - g) * x / factor
        f.append(x)
    return f


def rope(x, pos, freq, interleaved, magnitude=1.0, backward=False):
    """x [tokens, heads, dim] -> float64."""
    y = x.double().clone()
    half = len(freq)
    for i, f in enumerate(freq):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = pos.double() * f * (-1.0 if backward else 1.0)
        c, s = magnitude * torch.cos(angle)[:, None], magnitude * torch.sin(angle)[:, None]
        y[..., a] = x[..., a].double() * c - x[..., b].double() * s
        y[..., b] = x[..., a].double() * s + x[..., b].double() * c
    return y


def attention(q, k_cache, v_cache, table, q_start, ctx, block, n_blocks, scale, window, k_scale=None, v_scale=None):
    """out [T, H, D], lse [T, H], spread [T, H, D] = sum_j w_j |V_j|, reach [T, H] =
    the largest scale * sum_i |q_i K_ji| over the keys seen; all float64.  ctx and
    q_start are lists; `table` a list of lists."""
    T, H, D = q.shape
    J = k_cache.shape[1]
    out = torch.zeros(T, H, D, dtype=torch.float64, device=q.device)
    spread = torch.zeros_like(out)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=q.device)
    reach = torch.zeros(T, H, dtype=torch.float64, device=q.device)
    for r in range(len(ctx)):
        for t in range(q_start[r], q_start[r + 1]):
            p = ctx[r] + t - q_start[r]
            low = max(0, p - window + 1) if window else 0
            keys = [j for j in range(low, p + 1) if 0 <= table[r][j // block] < n_blocks]
            if not keys:
                continue
            page = torch.tensor([table[r][j // block] for j in keys], device=q.device)
            off = torch.tensor([j % block for j in keys], device=q.device)
            k, v = k_cache[page, :, off].double(), v_cache[page, :, :, off].double()   # [keys, J, D]
            if k_scale is not None:
                k = k * k_scale.double()[:, None]
            if v_scale is not None:
                v = v * v_scale.double()[:, None]
            x = q[t].double().reshape(J, H // J, D)
            kj = k.permute(1, 2, 0).contiguous()
            s = scale * (x @ kj)                                                       # [J, G, keys]
            w = torch.softmax(s, -1)
            vj = v.transpose(0, 1).contiguous()
            out[t] = (w @ vj).reshape(H, D)
            spread[t] = (w @ vj.abs()).reshape(H, D)
            lse[t] = torch.logsumexp(s, -1).reshape(H)
            reach[t] = (scale * (x.abs() @ kj.abs())).amax(-1).reshape(H)
    return out, lse, spread, reach


# ---- a cache of 8 bits with a scale for each block and head ----

MOST = {"fp8": 448.0, "i8": 127.0}


def held(x, kind):
    """The held numbers nearest to x (float64, in units of the scale), ties to even."""
    y = torch.nan_to_num(x, nan=math.nan, posinf=MOST[kind], neginf=-MOST[kind]).clamp(-MOST[kind], MOST[kind])
    if kind == "i8":
        return torch.nan_to_num(y, nan=0.0).round()
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)   # 3 bits below the first, 2^-9 at the least
    return (y / step).round() * step


def rises(need, old):
    """The least n >= 0 with need <= old * 2^n."""
    n = 0
    while need > old * 2.0 ** n:
        n += 1
    return n


def write_blocks(x, numbers, scale, table, q_start, ctx, block, n_blocks, kind):
    """A step's values x [T, J, D] float64 into numbers [n_blocks, J, block, D] and scale
    [n_blocks, J], float64, both changed; lists elsewhere.  Returns the (block, place) of
    every token, or None for one that is not written."""
    places = [None] * q_start[-1]
    for r in range(len(ctx)):
        t, end = q_start[r], q_start[r + 1]
        while t < end:
            at = (ctx[r] + t - q_start[r]) % block
            n = min(block - at, end - t)
            page = table[r][(ctx[r] + t - q_start[r]) // block]
            if 0 <= page < n_blocks:
                for j in range(x.shape[1]):
                    new = x[t:t + n, j]
                    size = new[torch.isfinite(new)].abs()
                    need = float(size.max()) / MOST[kind] if size.numel() else 0.0
                    old = float(scale[page, j]) if at else 0.0
                    if not (0.0 < old < math.inf):
                        if at and need > 0:
                            numbers[page, j, :at] = held(numbers[page, j, :at] * 0.0, kind)
                        scale[page, j] = need
                    else:
                        m = rises(need, old)
                        numbers[page, j, :at] = held(numbers[page, j, :at] * 2.0 ** -m, kind) if m else numbers[page, j, :at]
                        scale[page, j] = old * 2.0 ** m
                    s = float(scale[page, j])
                    numbers[page, j, at:at + n] = held(new / s if s else torch.where(torch.isinf(new), new, new * 0.0), kind)
                for i in range(n):
                    places[t + i] = (page, at + i)
            t += n
    return places


def read_rows(numbers, scale, table, kv_len, block, n_blocks, starts, first):
    """Rows [starts[-1], J, D] float64 of numbers [n_blocks, J, block, D] times scale
    [n_blocks, J]."""
    rows = torch.zeros(starts[-1], numbers.shape[1], numbers.shape[3], dtype=torch.float64)
    for r in range(len(kv_len)):
        for i in range(starts[r], starts[r + 1]):
            p = first[r] + i - starts[r]
            page = table[r][p // block] if 0 <= p < kv_len[r] else -1
            if 0 <= page < n_blocks:
                rows[i] = numbers[page, :, p % block] * scale[page][:, None]
    return rows
