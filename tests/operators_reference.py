"""The operators around the paged cache in plain form, 64 bits wide, from their definitions; shares no code with the library."""
import math

import torch


def assign_blocks(lengths, held, tables, stack, count, block):
    """Lists in, lists out: (tables, held, stack, count, denied)."""
    tables, held, stack = [list(t) for t in tables], list(held), list(stack)
    width = len(tables[0]) if tables else 0
    need = [-(-max(n, 0) // block) for n in lengths]
    need = [h if n > width else n for n, h in zip(need, held)]
    for r in range(len(lengths)):
        for b in tables[r][need[r]:held[r]]:
            if count < len(stack):
                stack[count] = b
                count += 1
        held[r] = min(held[r], need[r])
    wanted, avail, denied = 0, count, False
    for r in range(len(lengths)):
        wanted += need[r] - held[r]
        if need[r] > held[r] and wanted > avail:
            denied = True
            continue
        for j in range(held[r], need[r]):
            count -= 1
            tables[r][j] = stack[count]
        held[r] = need[r]
    return tables, held, stack, count, denied


def map_slots(lengths, done, tables, block, unit=1, min_new=0):
    """(offsets, slots, positions) of all new tokens."""
    offsets, slots, positions = [0], [], []
    for r, n in enumerate(lengths):
        n = max(n, 0)
        for p in range(max(0, min((done[r] if done else 0) * unit, n - min_new)), n):
            b = tables[r][p // block] if p // block < len(tables[r]) else -1
            slots.append(b * block + p % block if b >= 0 else -1)
            positions.append(p)
        offsets.append(len(slots))
    return offsets, slots, positions


E4M3 = sorted({(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)) for e in range(16) for m in range(8) if (e, m) != (15, 7)})


def e4m3_nearest(x):
    """float64 tensor x >= 0 -> nearest e4m3 value (ties to the even code), at most 448."""
    grid = torch.tensor(E4M3, dtype=torch.float64, device=x.device)
    x = x.clamp(max=448.0)
    hi = torch.searchsorted(grid, x).clamp(1, len(E4M3) - 1)
    lo = hi - 1
    below, above = x - grid[lo], grid[hi] - x
    take_hi = (above < below) | ((above == below) & (hi % 2 == 0))      # a code is its index: values ascend with it
    return torch.where(take_hi, grid[hi], grid[lo])


def quantised(x, t):
    """The values the 4-bit cache holds for rows x [..., D] with tensor scale t, float64."""
    g = x.double().unflatten(-1, (-1, 16))
    a = g.abs().amax(-1, keepdim=True)
    s = torch.where(a.isnan(), a, e4m3_nearest(torch.nan_to_num(a, nan=0.0) / (7 * t))) * t
    q = torch.where(s > 0, (g / s).round(), torch.zeros_like(g)).nan_to_num(nan=0.0).clamp(-8, 7)
    return (q * s).flatten(-2)


def gather(values, table_row, n, block):
    """values [blocks, B, H, D]; the first n tokens of a request: rows [n, H, D] and which of them have a valid block."""
    tok = torch.arange(n, device=values.device)
    ok = tok // block < table_row.numel()
    ids = torch.where(ok, table_row.long()[(tok // block).clamp(max=table_row.numel() - 1)], -1)
    ok = ok & (ids >= 0) & (ids < values.shape[0])
    return values[ids.clamp(0, values.shape[0] - 1), tok % block], ok


def attend(q, offsets, lengths, tables, k_values, v_values, block, scale):
    """q [T, Hq, D]; k_values, v_values float64 [blocks, B, H, D] -> (out, sum p |v|, largest sum |q k| scale, rows that belong to a request)."""
    T, Hq, D = q.shape
    H = k_values.shape[2]
    G = Hq // H
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    spread, scores = torch.zeros_like(out), torch.zeros(q.shape[:2] + (1,), dtype=torch.float64, device=q.device)
    owned = torch.zeros(T, dtype=torch.bool, device=q.device)
    for r, n in enumerate(lengths):
        a, b = offsets[r], offsets[r + 1]
        owned[a:b] = True
        if n <= 0 or a >= b:
            continue
        k, ok = gather(k_values, tables[r], n, block)
        v, _ = gather(v_values, tables[r], n, block)
        for i in range(a, b):
            pos = n - (b - a) + (i - a)
            see = ok.clone()
            see[max(pos + 1, 0):] = False
            if not bool(see.any()):
                continue
            ks, vs = k[see].repeat_interleave(G, dim=1), v[see].repeat_interleave(G, dim=1)
            s = torch.einsum("hd,nhd->hn", q[i].double(), ks) * scale
            p = torch.softmax(s, dim=1)
            out[i] = torch.einsum("hn,nhd->hd", p, vs)
            spread[i] = torch.einsum("hn,nhd->hd", p, vs.abs())
            scores[i, :, 0] = torch.einsum("hd,nhd->hn", q[i].double().abs(), ks.abs()).amax(1) * abs(scale)
    return out, spread, scores, owned


def attend_tolerance(q, out, spread, scores, keys, v_max, fmt_packed, k_sum):
    """How far a result may be off, element by element.

    Products of 16-bit operands are exact, their sums 32 bits wide (and may be truncated, one step of 2^-23 of the running sum per
    addend): a score is off by at most D 2^-23 sum|q k| scale, the scale factor and exp2 add a few 2^-22 relative; a weight is off by
    twice that relative to the sum of weights.  Weights are rounded to 16 bits: half a step of the type, and below fp16's normal range half of 2^-24.
    The 4-bit cache takes bf16 queries as fp16: at most 2^-25 of the row's largest element each.  The result is rounded once."""
    D = q.shape[-1]
    half = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
    fp16_weights = fmt_packed or q.dtype == torch.float16
    e_score = (D + 8) * 2.0 ** -23 * scores + 2.0 ** -20
    if fmt_packed and q.dtype == torch.bfloat16:
        e_score = e_score + 2.0 ** -25 * q.double().abs().amax(-1, keepdim=True) * k_sum
    e_weight = (2.0 ** -11 if fp16_weights else 2.0 ** -8) + 2 * e_score
    tol = spread * e_weight + half[q.dtype] * out.abs()
    if fp16_weights:
        tol = tol + keys * 2.0 ** -25 * v_max
    if q.dtype == torch.float16:
        tol = tol + 2.0 ** -25
    return tol
