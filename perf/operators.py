"""The operators around the paged cache as calls to time: block bookkeeping, the 4-bit cache's writer and reader, attention over the cache.

Each case is one call (or one pair of calls) a serving step makes on one GPU.  `run` computes them in elementary torch operations, or
with `own` set through the framework's binding.  `exact` computes the same from the definitions in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

GROUP = 16      # elements that share a scale in the 4-bit cache
TILE = 16       # tokens of a tile of the 4-bit cache
K_SCALE, V_SCALE = 2.0 ** -4, 2.0 ** -6       # tensor scales of the 4-bit cache, powers of two
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---- cases ------------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the bookkeeping of one decode step of 64 requests, a few of which have ended (tables as wide as a 6256-token prompt): latency only
        {"name": "plan_decode_64", "op": "plan", "requests": 64, "lo": 2000, "hi": 6256, "new_lo": 1, "new_hi": 1, "gone": 0.05, "block": 16, "width": 392, "lay": 1},
        # a very large batch of short requests whose prefixes were found in the store
        {"name": "plan_many_16384", "op": "plan", "requests": 16384, "lo": 64, "hi": 1024, "new_lo": 0, "new_hi": 64, "gone": 0.1, "block": 16, "width": 64, "lay": 2},
        # one decode step's K/V of 64 requests written into the 4-bit cache and read back
        {"name": "packed_write_64", "op": "write", "tokens": 64, "kv_heads": 8, "dim": 128, "block": 16, "dtype": "bf16", "lay": 3},
        # the K/V of 16384 prompt tokens
        {"name": "packed_write_16384", "op": "write", "tokens": 16384, "kv_heads": 8, "dim": 128, "block": 16, "dtype": "bf16", "lay": 4},
        # one chat answering over a 4k document, 4-bit cache: latency
        {"name": "packed_decode_1", "op": "attend", "packed": True, "requests": 1, "lo": 4160, "hi": 4160, "new_lo": 1, "new_hi": 1,
         "heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "dtype": "bf16", "lay": 5},
        # a decode step of 64 requests over long documents, ragged, 4-bit cache
        {"name": "packed_decode_64", "op": "attend", "packed": True, "requests": 64, "lo": 2064, "hi": 6256, "new_lo": 1, "new_hi": 1,
         "heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "dtype": "bf16", "lay": 6},
        # 8 requests over 16k documents with 64 query heads and 32-token blocks, 4-bit cache
        {"name": "packed_decode_8x16k", "op": "attend", "packed": True, "requests": 8, "lo": 16384, "hi": 16640, "new_lo": 1, "new_hi": 1,
         "heads": 64, "kv_heads": 8, "dim": 128, "block": 32, "dtype": "fp16", "lay": 7},
        # 16 prompts whose 4k document was found in the store: 64 fresh tokens each attend over the 4-bit cache
        {"name": "packed_suffix_16", "op": "attend", "packed": True, "requests": 16, "lo": 4160, "hi": 4160, "new_lo": 64, "new_hi": 64,
         "heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "dtype": "bf16", "lay": 8},
        # the decode step of 64 ragged requests over a 16-bit cache
        {"name": "decode_64", "op": "attend", "packed": False, "requests": 64, "lo": 2064, "hi": 6256, "new_lo": 1, "new_hi": 1,
         "heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "dtype": "bf16", "lay": 9},
        # 16 prompts with a stored 4k prefix and ragged questions, 16-bit cache
        {"name": "suffix_16", "op": "attend", "packed": False, "requests": 16, "lo": 4160, "hi": 4351, "new_lo": 64, "new_hi": 255,
         "heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "dtype": "bf16", "lay": 10},
        # a packed batch of 8 whole prompts of different lengths, nothing found in the store
        {"name": "prompts_8", "op": "attend", "packed": False, "requests": 8, "lo": 2064, "hi": 6256, "new_lo": -1, "new_hi": -1,
         "heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "dtype": "bf16", "lay": 11},
        # one whole 16k prompt with 64 query heads
        {"name": "prompt_16384", "op": "attend", "packed": False, "requests": 1, "lo": 16384, "hi": 16384, "new_lo": -1, "new_hi": -1,
         "heads": 64, "kv_heads": 8, "dim": 128, "block": 32, "dtype": "fp16", "lay": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "write", "attend", "attend", "attend"])
    lay = rng.randrange(1 << 30)
    if op == "plan":
        R = _log(rng, 1, 16384)
        block = rng.choice([8, 16, 32, 64])
        hi = min(_log(rng, 32, 16384), max(32, (1 << 24) // R))
        return {"op": op, "requests": R, "lo": 1, "hi": hi, "new_lo": 0, "new_hi": min(_log(rng, 1, 512), hi, max(1, (1 << 20) // R)), "gone": rng.choice([0.0, 0.2]),
                "block": block, "width": hi // block + 1 + rng.randrange(3), "lay": lay}
    dim, dtype = rng.choice([64, 128, 128]), rng.choice(["bf16", "fp16"])
    kv_heads = rng.choice([1, 2, 4, 8])
    if op == "write":
        return {"op": op, "tokens": _log(rng, 1, 16384), "kv_heads": kv_heads, "dim": dim, "block": rng.choice([16, 32, 48, 128]), "dtype": dtype, "lay": lay}
    packed = rng.random() < 0.5
    heads = kv_heads * rng.choice([1, 2, 3, 4, 6, 8])
    block = rng.choice([16, 32, 64] if packed else [8, 16, 24, 32, 64])
    kind = rng.choice(["decode", "suffix", "prompt"])
    if kind == "decode":
        R = _log(rng, 1, 128)
        hi = min(_log(rng, 16, 32768), (1 << 19) // R)
        new = rng.choice([1, 1, 2, 4])
        return {"op": op, "packed": packed, "requests": R, "lo": max(1, hi // 4), "hi": hi, "new_lo": 1, "new_hi": new, "heads": heads,
                "kv_heads": kv_heads, "dim": dim, "block": block, "dtype": dtype, "lay": lay}
    R = _log(rng, 1, 32)
    hi = min(_log(rng, 64, 16384), (1 << 16) // R)
    if kind == "suffix":
        return {"op": op, "packed": packed, "requests": R, "lo": max(1, hi // 2), "hi": hi, "new_lo": 1, "new_hi": max(1, min(hi // 4, 1024)), "heads": heads,
                "kv_heads": kv_heads, "dim": dim, "block": block, "dtype": dtype, "lay": lay}
    hi = min(hi, int(16384 / math.sqrt(R)))
    return {"op": op, "packed": packed, "requests": R, "lo": max(1, hi // 4), "hi": hi, "new_lo": -1, "new_hi": -1, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "block": block, "dtype": dtype, "lay": lay}


def _lengths(case):
    """Context length and new tokens of every request: part of the case, not of the seed.  new < 0 means the whole prompt."""
    rng = random.Random(case["lay"])
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["requests"])]
    new = [n if case["new_lo"] < 0 else min(n, rng.randint(case["new_lo"], case["new_hi"])) for n in lens]
    return lens, new


def _plan(case):
    """lengths, tokens already in the cache and blocks held of every request; a request that has ended gives its blocks back."""
    lens, new = _lengths(case)
    done = [n - m for n, m in zip(lens, new)]
    held = [-(-d // case["block"]) for d in done]
    rng = random.Random(case["lay"] + 1)
    for r in range(len(lens)):
        if rng.random() < case["gone"]:
            lens[r] = done[r] = 0
    return lens, done, held


def work(case):
    if case["op"] == "plan":
        lens, done, held = _plan(case)
        moved = sum(abs(-(-n // case["block"]) - h) for n, h in zip(lens, held))
        # lengths, done and held read, held and offsets written; ids read and set; slots (8 bytes) and positions (4) written
        return {"bytes": len(lens) * 20 + moved * 8 + (sum(lens) - sum(done)) * 12, "flops": 0}
    if case["op"] == "write":
        n = 2 * case["tokens"] * case["kv_heads"] * case["dim"]
        return {"bytes": 2 * (2 * n + n // 2 + n // GROUP) + 8 * case["tokens"], "flops": 6 * n}
    lens, new = _lengths(case)
    row = case["dim"] * 2 if not case["packed"] else case["dim"] // 2 + case["dim"] // GROUP
    kv = sum(lens) * case["kv_heads"] * row * 2
    qo = 2 * 2 * sum(new) * case["heads"] * case["dim"]
    pairs = sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lens, new))
    return {"bytes": kv + qo + 4 * sum(-(-n // case["block"]) for n in lens), "flops": 4 * case["dim"] * case["heads"] * pairs}


# ---- the 4-bit cache's bytes ------------------------------------------------------------------------------------------------------
def _chunk_place(dim):
    """Where the 16-byte chunk c of token n's codes sits in a tile: index n * chunks + c -> place."""
    c, rho = dim // 32, 256 // dim
    return [(n // rho) * 8 + (((n % rho) * c + k) ^ (2 * (n >> 2))) for n in range(TILE) for k in range(c)]


def _pack(codes, scales, is_v):
    """codes uint8 [blocks, B, H, D] in 0..15, scales uint8 [blocks, B, H, D/16] (e4m3 bytes) -> uint8 [blocks, B * H * 9 D / 16]."""
    nb, B, H, D = codes.shape
    t = codes.view(nb, B // TILE, TILE, H, D).permute(0, 3, 1, 2, 4)
    t = (t[..., 0::2] | (t[..., 1::2] << 4)).reshape(nb, H, B // TILE, TILE * D // 32, 16)
    out = torch.empty_like(t)
    out[:, :, :, _chunk_place(D)] = t
    s = scales.view(nb, B // TILE, TILE, H, D // GROUP).permute(0, 3, 1, 2, 4)
    if is_v:
        s = s.transpose(3, 4)
    return torch.cat([out.reshape(nb, H, B // TILE, -1), s.reshape(nb, H, B // TILE, -1)], dim=3).reshape(nb, -1)


def _unpack(data, B, H, D, is_v):
    """The values the bytes of whole blocks [blocks, chunk] stand for, without the tensor scale, in 32 bits: [blocks, B, H, D]."""
    nb = data.shape[0]
    t = data.view(nb, H, B // TILE, 9 * D)
    c = t[..., :8 * D].reshape(nb, H, B // TILE, TILE * D // 32, 16)[:, :, :, _chunk_place(D)].reshape(nb, H, B // TILE, TILE, D // 2)
    c = torch.stack([c & 15, c >> 4], dim=-1).view(nb, H, B // TILE, TILE, D // GROUP, GROUP)
    s = t[..., 8 * D:].view(torch.float8_e4m3fn).to(torch.float32)
    s = s.reshape(nb, H, B // TILE, D // GROUP, TILE).transpose(3, 4) if is_v else s.reshape(nb, H, B // TILE, TILE, D // GROUP)
    v = (c.to(torch.float32) - 8.0) * s[..., None]
    return v.view(nb, H, B, D).permute(0, 2, 1, 3)


def _quantise(x, t):
    """codes and e4m3 scales of x [..., D] (groups of 16 along D, tensor scale t).  64 bits: values sit next to rounding borders."""
    g = x.to(torch.float64).unflatten(-1, (-1, GROUP))
    a = g.abs().amax(dim=-1)
    s = torch.clamp(a / (7.0 * t), max=448.0).to(torch.float32).to(torch.float8_e4m3fn)
    sv = s.to(torch.float64)[..., None] * t
    q = torch.where(sv > 0, torch.round(g / sv), torch.zeros_like(g)).clamp(-8, 7)
    return q.flatten(-2), s


# ---- inputs -----------------------------------------------------------------------------------------------------------------------
def _kv_values(gen, shape, dtype, scale):
    """K/V as a model makes them: normal, a few channels several times larger than the rest."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    loud = 1.0 + 7.0 * (torch.rand((1,) * (len(shape) - 1) + shape[-1:], generator=gen, device="cuda") < 0.05).float()
    return (x * loud * scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 17)
    dev = {"device": "cuda"}
    st = {"case": case}
    if own:
        from paper_2607_22648_b200 import binding
        st["G"] = binding
    if case["op"] == "plan":
        lens, done, held = _plan(case)
        R, B, W = case["requests"], case["block"], case["width"]
        st["lengths"] = torch.tensor(lens, dtype=torch.int32, **dev)
        st["done"] = torch.tensor(done, dtype=torch.int32, **dev)
        st["held"] = torch.tensor(held, dtype=torch.int32, **dev)
        grown = sum(max(0, -(-n // B) - h) for n, h in zip(lens, held))
        total = sum(held) + grown + 64
        perm = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((R, W), -1, dtype=torch.int32, **dev)
        cols = torch.arange(W, **dev)
        table[cols[None, :] < st["held"][:, None].long()] = perm[:sum(held)]
        st["tables"] = table
        st["free_ids"] = torch.full((total,), -1, dtype=torch.int32, **dev)
        st["free_ids"][:total - sum(held)] = perm[sum(held):]
        st["free_count"] = torch.tensor([total - sum(held)], dtype=torch.int32, **dev)
        st["held_out"], st["free_out"] = torch.empty_like(st["held"]), torch.empty_like(st["free_count"])
        st["max_tokens"] = sum(lens) - sum(done)
        return st
    H, D, B, dtype = case["kv_heads"], case["dim"], case["block"], DTYPES[case["dtype"]]
    if case["op"] == "write":
        T = case["tokens"]
        nb = -(-T // B) + 3
        st["k"], st["v"] = _kv_values(gen, (T, H, D), dtype, 1.0), _kv_values(gen, (T, H, D), dtype, 0.25)
        st["slots"] = torch.randperm(nb * B, generator=gen, device="cuda")[:T] if T <= 256 else _prompt_slots(gen, T, nb, B)
        if own:
            G = st["G"]
            st["layout"] = G.KVLayout(H, D, B, G.KV_PACKED, K_SCALE, V_SCALE)
            st["cache"] = G.PagedKV(1, nb, st["layout"].chunk_bytes)
        return st
    lens, new = _lengths(case)
    R = case["requests"]
    blocks = [-(-n // B) for n in lens]
    nb, W = sum(blocks) + 3, max(blocks)
    perm = torch.randperm(nb, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((R, W), -1, dtype=torch.int32, **dev)
    cols = torch.arange(W, **dev)
    table[cols[None, :] < torch.tensor(blocks, **dev)[:, None]] = perm[:sum(blocks)]
    st["tables"] = table
    st["lengths"] = torch.tensor(lens, dtype=torch.int32, **dev)
    st["offsets"] = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, **dev)
    st["lens"], st["new"] = lens, new       # a user's program knows its requests on the host too
    st["q"] = _kv_values(gen, (sum(new), case["heads"], D), dtype, 1.0)
    chunks = []
    for is_v, t, scale in ((False, K_SCALE, 1.0), (True, V_SCALE, 0.25)):
        x = _kv_values(gen, (nb, B, H, D), dtype, scale)
        if case["packed"]:
            parts = []
            for i in range(0, nb, 1024):      # the 64-bit quantiser's temporaries stay small
                q, s = _quantise(x[i:i + 1024], t)
                parts.append(_pack((q + 8).to(torch.uint8), s.view(torch.uint8), is_v))
            chunks.append(torch.cat(parts))
        else:
            chunks.append(x.view(nb, -1).view(torch.uint8))
    st["data"] = torch.stack(chunks)          # [K|V][blocks][chunk], one layer's cache
    if own:
        G = st["G"]
        fmt = G.KV_PACKED if case["packed"] else {"bf16": G.KV_BF16, "fp16": G.KV_FP16}[case["dtype"]]
        st["layout"] = G.KVLayout(H, D, B, fmt, K_SCALE, V_SCALE) if case["packed"] else G.KVLayout(H, D, B, fmt)
        st["cache"] = G.PagedKV(1, nb, st["layout"].chunk_bytes, tensors=[st["data"]])
        st["max_new"] = max(new)
        st["workspace"] = G.attend_workspace(st["layout"])
        st["out"] = torch.empty_like(st["q"])
    return st


def _prompt_slots(gen, T, nb, B):
    """Slots of consecutive tokens in shuffled blocks."""
    perm = torch.randperm(nb, generator=gen, device="cuda")
    t = torch.arange(T, device="cuda")
    return perm[t // B] * B + t % B


# ---- one pass ---------------------------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if case["op"] == "plan":
        return _run_plan(state)
    if case["op"] == "write":
        return _run_write(state)
    return _run_attend(state)


def _run_plan(st):
    c = st["case"]
    B = c["block"]
    if own:
        G = st["G"]
        held, free = G.assign_blocks(st["lengths"], st["held"], st["tables"], st["free_ids"], st["free_count"], B, held_out=st["held_out"],
                                     free_count_out=st["free_out"])
        offsets, slots, positions = G.map_slots(st["lengths"], st["done"], st["tables"], B, st["max_tokens"])
        return st["tables"], held, st["free_ids"], free, offsets, slots, positions
    lens, held, table, ids = st["lengths"].long(), st["held"].long(), st["tables"].clone(), st["free_ids"].clone()
    R, W = table.shape
    need = (lens + B - 1) // B
    cols = torch.arange(W, device="cuda")[None, :]
    back = (cols >= need[:, None]) & (cols < held[:, None])           # surplus blocks, in (request, block) order
    returned = table[back]
    top = st["free_count"].long()[0]
    ids = torch.where(torch.arange(ids.numel(), device="cuda") < top, ids, -1)
    ids[top + torch.arange(returned.numel(), device="cuda")] = returned
    top = top + returned.numel()
    grow = torch.clamp(need - held, min=0)
    upto = torch.cumsum(grow, 0)
    granted = (grow > 0) & (upto <= top)
    first = upto - grow
    take = granted[:, None] & (cols >= held[:, None]) & (cols < need[:, None])
    rank = (first[:, None] + cols - held[:, None])[take]
    table[take] = ids[top - 1 - rank]
    held = torch.where(granted | (need < held), need, held)
    free = (top - (grow * granted).sum()).to(torch.int32).reshape(1)
    done = torch.clamp(torch.minimum(st["done"].long(), lens), min=0)
    new = lens - done
    offsets = torch.zeros(R + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.cumsum(new, 0)
    T = st["max_tokens"]
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(offsets, t, right=True) - 1
    pos = done[r] + t - offsets[r]
    b = table[r, pos // B].long()
    slots = torch.where(b >= 0, b * B + pos % B, -1)
    return table, held.to(torch.int32), ids, free, offsets.to(torch.int32), slots, pos.to(torch.int32)


def _run_write(st):
    c = st["case"]
    if own:
        G = st["G"]
        G.kv_write(st["layout"], st["cache"], 0, st["k"], st["v"], st["slots"])
        return G.kv_read(st["layout"], st["cache"], 0, st["slots"], st["k"].dtype)
    out = []
    for x, t in ((st["k"], K_SCALE), (st["v"], V_SCALE)):
        q, s = _quantise(x, t)
        sv = (s.to(torch.float32) * t)[..., None]
        out.append((q.to(torch.float32).unflatten(-1, (-1, GROUP)) * sv).flatten(-2).to(x.dtype))
    return tuple(out)


def _run_attend(st):
    c = st["case"]
    if own:
        return st["G"].attend(st["layout"], st["cache"], 0, st["q"], st["offsets"], st["lengths"], st["tables"], st["max_new"],
                              out=st["out"], workspace=st["workspace"])
    H, D, B, heads = c["kv_heads"], c["dim"], c["block"], c["heads"]
    G = heads // H
    out = torch.zeros_like(st["q"])
    at = 0
    for r, (n, m) in enumerate(zip(st["lens"], st["new"])):
        if m == 0:
            continue
        ids = st["tables"][r, :-(-n // B)].long()
        if c["packed"]:
            k = _unpack(st["data"][0][ids], B, H, D, False).reshape(-1, H, D)[:n] * K_SCALE
            v = _unpack(st["data"][1][ids], B, H, D, True).reshape(-1, H, D)[:n] * V_SCALE
        else:
            k = st["data"][0][ids].view(st["q"].dtype).view(-1, H, D)[:n].float()
            v = st["data"][1][ids].view(st["q"].dtype).view(-1, H, D)[:n].float()
        q = st["q"][at:at + m].float()
        hidden = torch.arange(n, device="cuda")[None, :] > (n - m + torch.arange(m, device="cuda"))[:, None]
        for h in range(H):                    # one kv head at a time: the scores of a long prompt are large
            qh = q[:, h * G:(h + 1) * G].transpose(0, 1)                                  # [G, m, D]
            s = torch.matmul(qh, k[:, h].t()) * (1.0 / math.sqrt(D))
            s = s.masked_fill_(hidden, float("-inf"))
            s = torch.exp(s - s.amax(dim=-1, keepdim=True))
            s = s / s.sum(dim=-1, keepdim=True)
            out[at:at + m, h * G:(h + 1) * G] = torch.matmul(s, v[:, h]).transpose(0, 1).to(out.dtype)
        at += m
    return out


# ---- the definitions, in 64 bits ----------------------------------------------------------------------------------------------------
def _e4m3_value(byte):
    """float64 values of e4m3 bytes (numpy): 4 exponent bits of bias 7, 3 mantissa bits, subnormals, no infinities."""
    b = byte.astype(np.int64)
    e, m = (b >> 3) & 15, b & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0)) * np.where(b & 128, -1.0, 1.0)


def _e4m3_nearest(x):
    """x >= 0 (float64) to the nearest e4m3 value, ties to the even mantissa, at most 448."""
    x = np.minimum(x, 448.0)
    _, e = np.frexp(np.maximum(x, 2.0 ** -6))
    step = 2.0 ** (e - 4.0)
    return np.minimum(np.rint(x / step) * step, 448.0)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "plan":
        return _exact_plan(st)
    if case["op"] == "write":
        out = []
        for x, t in ((st["k"], K_SCALE), (st["v"], V_SCALE)):
            g = x.double().cpu().numpy().reshape(-1, GROUP)
            s = _e4m3_nearest(np.abs(g).max(axis=1) / (7.0 * t))[:, None] * t
            code = np.clip(np.rint(np.divide(g, s, out=np.zeros_like(g), where=s > 0)), -8, 7)
            out.append(torch.from_numpy((code * s).reshape(x.shape)))
        return tuple(out)
    return _exact_attend(st)


def _exact_plan(st):
    c = st["case"]
    B = c["block"]
    table, held, lens, done = (st[k].cpu().tolist() for k in ("tables", "held", "lengths", "done"))
    stack, top = st["free_ids"].cpu().tolist(), int(st["free_count"].item())
    need = [-(-n // B) for n in lens]
    for r in range(len(lens)):
        for b in table[r][need[r]:held[r]]:
            stack[top] = b
            top += 1
        held[r] = min(held[r], need[r])
    wanted, avail = 0, top
    for r in range(len(lens)):
        wanted += need[r] - held[r]
        if wanted > avail:
            continue
        for j in range(held[r], need[r]):
            top -= 1
            table[r][j] = stack[top]
        held[r] = need[r]
    offsets, slots, positions = [0], [], []
    for r, n in enumerate(lens):
        for p in range(max(0, min(done[r], n)), n):
            b = table[r][p // B]
            slots.append(b * B + p % B if b >= 0 else -1)
            positions.append(p)
        offsets.append(len(slots))
    as_t = lambda x, d: torch.tensor(x, dtype=d)
    return (as_t(table, torch.int32), as_t(held, torch.int32), as_t(stack, torch.int32), as_t([top], torch.int32), as_t(offsets, torch.int32),
            as_t(slots, torch.int64), as_t(positions, torch.int32))


def _exact_attend(st):
    c = st["case"]
    H, D, B, heads = c["kv_heads"], c["dim"], c["block"], c["heads"]
    G = heads // H
    place = torch.tensor(_chunk_place(D), device="cuda")
    decode = torch.from_numpy(_e4m3_value(np.arange(256, dtype=np.uint8))).cuda()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    first = 0
    for r, (n, m) in enumerate(zip(st["lens"], st["new"])):
        tok = torch.arange(n, device="cuda")
        blk, inb = st["tables"][r].long()[tok // B], tok % B
        for h in range(H if m else 0):
            kv = []
            for side, t in ((0, K_SCALE), (1, V_SCALE)):
                data = st["data"][side]
                if not c["packed"]:
                    kv.append(data.view(st["q"].dtype).view(-1, B, H, D)[blk, inb, h].double())
                    continue
                tiles = data.view(-1, H, B // TILE, 9 * D)[blk, h, inb // TILE]               # one tile per token: [n, 9 D]
                i = inb % TILE
                d = torch.arange(D, device="cuda")
                byte = place[i[:, None] * (D // 32) + d[None, :] // 32] * 16 + (d[None, :] % 32) // 2
                code = (tiles.gather(1, byte) >> (4 * (d % 2)).to(torch.uint8)) & 15
                g = d[None, :] // GROUP
                sb = 8 * D + (g * TILE + i[:, None] if side else i[:, None] * (D // GROUP) + g)
                kv.append((code.double() - 8.0) * decode[tiles.gather(1, sb).long()] * t)
            pos = n - m + torch.arange(m, device="cuda")
            seen = tok[None, :] <= pos[:, None]
            for gq in range(G):
                s = (st["q"][first:first + m, h * G + gq].double() @ kv[0].t()) / math.sqrt(D)
                s = torch.where(seen, s, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
                s = torch.softmax(s, dim=1)
                out[first:first + m, h * G + gq] = s @ kv[1]
        first += m
    return out
