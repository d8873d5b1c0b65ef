"""Attention over a cache of shared latent vectors, and eviction of tokens by the attention they were given, as calls to time.

Each case is one call (or the calls that follow one another) a serving step makes on one GPU.  `run` computes them in elementary torch
operations, or with `own` set through the framework's binding.  `exact` computes the same from the definitions in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

GROUP = 16      # elements that share a scale in the 4-bit cache
TILE = 16       # tokens of a tile of the 4-bit cache
ROPE = 64       # elements of a latent row's rotary part
K_SCALE, V_SCALE = 2.0 ** -4, 2.0 ** -6       # tensor scales of the 4-bit cache, powers of two
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---- cases ------------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one decode step's latent vectors of 64 requests written into the cache and read back: latency
        {"name": "latent_rows_64", "op": "rows", "tokens": 64, "latent": 512, "block": 16, "dtype": "bf16", "lay": 1},
        # those of 16384 prompt tokens, read back to be expanded
        {"name": "latent_rows_16384", "op": "rows", "tokens": 16384, "latent": 512, "block": 16, "dtype": "bf16", "lay": 2},
        # one chat answering over a 4k document, absorbed form: latency
        {"name": "latent_decode_1", "op": "latent", "requests": 1, "lo": 4160, "hi": 4160, "new_lo": 1, "new_hi": 1, "heads": 16, "latent": 512, "block": 16,
         "dtype": "bf16", "lay": 3},
        # a decode step of 64 ragged requests over long documents with 128 query heads
        {"name": "latent_decode_64", "op": "latent", "requests": 64, "lo": 2064, "hi": 6256, "new_lo": 1, "new_hi": 1, "heads": 128, "latent": 512, "block": 16,
         "dtype": "bf16", "lay": 4},
        # 16 prompts whose 4k document was found in the store: 64 fresh tokens each attend over the latent cache
        {"name": "latent_suffix_16", "op": "latent", "requests": 16, "lo": 4160, "hi": 4160, "new_lo": 64, "new_hi": 64, "heads": 16, "latent": 512, "block": 64,
         "dtype": "fp16", "lay": 5},
        # a packed batch of 8 whole prompts of different lengths, keys and values expanded
        {"name": "expanded_prompts_8", "op": "expanded", "requests": 8, "lo": 2064, "hi": 6256, "new_lo": -1, "new_hi": -1, "heads": 16, "dtype": "bf16", "lay": 6},
        # 4 prompts whose first tokens were found and expanded again: long questions behind them
        {"name": "expanded_suffix_4", "op": "expanded", "requests": 4, "lo": 6000, "hi": 8192, "new_lo": 1000, "new_hi": 2048, "heads": 32, "dtype": "fp16", "lay": 7},
        # the attention that one decode step's 64 ragged requests gave to the tokens of a 16-bit cache
        {"name": "weights_decode_64", "op": "weights", "cache": "bf16", "requests": 64, "lo": 2064, "hi": 6256, "new_lo": 1, "new_hi": 1, "heads": 32, "kv_heads": 8,
         "dim": 128, "block": 16, "dtype": "bf16", "lay": 8},
        # what the last 32 tokens of 16 prompts gave to the 4k before them, 4-bit cache: a vote on what to keep
        {"name": "weights_window_16", "op": "weights", "cache": "packed", "requests": 16, "lo": 4160, "hi": 4351, "new_lo": 32, "new_hi": 32, "heads": 32, "kv_heads": 8,
         "dim": 128, "block": 16, "dtype": "bf16", "lay": 9},
        # a decode step of 8 requests over 16k latent vectors with 64 query heads
        {"name": "weights_latent_8", "op": "weights", "cache": "latent", "requests": 8, "lo": 16000, "hi": 16640, "new_lo": 1, "new_hi": 1, "heads": 64, "kv_heads": 1,
         "dim": 576, "block": 32, "dtype": "fp16", "lay": 10},
        # one request's cache cut to 4096 tokens: latency
        {"name": "evict_1", "op": "evict", "cache": "bf16", "requests": 1, "lo": 6256, "hi": 6256, "budget": 4096, "first": 4, "recent": 512, "kv_heads": 8, "dim": 128,
         "block": 16, "dtype": "bf16", "lay": 11},
        # 64 ragged requests cut to 2048 tokens
        {"name": "evict_64", "op": "evict", "cache": "bf16", "requests": 64, "lo": 2000, "hi": 6256, "budget": 2048, "first": 4, "recent": 256, "kv_heads": 8, "dim": 128,
         "block": 16, "dtype": "bf16", "lay": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rows", "latent", "latent", "expanded", "weights", "weights", "evict"])
    lay, dtype = rng.randrange(1 << 30), rng.choice(["bf16", "fp16"])
    if op == "rows":
        return {"op": op, "tokens": _log(rng, 1, 16384), "latent": rng.choice([256, 512, 512]), "block": rng.choice([8, 16, 48, 128]), "dtype": dtype, "lay": lay}
    if op == "latent":
        heads, latent, block = rng.choice([1, 6, 16, 20, 32, 64, 128]), rng.choice([256, 512, 512]), rng.choice([8, 16, 24, 64, 128])
        if rng.random() < 0.5:
            R, new = _log(rng, 1, 128), rng.choice([1, 1, 2, 4])
            hi = min(_log(rng, 16, 32768), (1 << 25) // (R * heads * new))
            lo = max(1, hi // 4)
        else:
            R = _log(rng, 1, 32)
            hi = _log(rng, 64, 16384)
            new = max(1, min(hi // 4, (1 << 25) // (R * heads * hi)))
            lo = max(1, hi // 2)
        return {"op": op, "requests": R, "lo": lo, "hi": hi, "new_lo": 1, "new_hi": new, "heads": heads, "latent": latent, "block": block, "dtype": dtype, "lay": lay}
    if op == "expanded":
        R, heads = _log(rng, 1, 32), rng.choice([1, 2, 5, 16, 32])
        hi = min(_log(rng, 64, 16384), int(math.sqrt((1 << 30) / (R * heads))))
        if rng.random() < 0.5:
            return {"op": op, "requests": R, "lo": max(1, hi // 4), "hi": hi, "new_lo": -1, "new_hi": -1, "heads": heads, "dtype": dtype, "lay": lay}
        return {"op": op, "requests": R, "lo": max(1, hi // 2), "hi": hi, "new_lo": 1, "new_hi": max(1, hi // 2), "heads": heads, "dtype": dtype, "lay": lay}
    cache = rng.choice([dtype, dtype, "packed", "latent"]) if op == "weights" else rng.choice([dtype, dtype, "latent"])
    kv_heads = 1 if cache == "latent" else rng.choice([1, 2, 4, 8])
    dim = rng.choice([320, 576, 576]) if cache == "latent" else rng.choice([64, 128, 128])
    block = rng.choice([16, 32, 64] if cache == "packed" else [8, 16, 24, 64])
    if op == "weights":
        heads = rng.choice([8, 16, 40, 64, 128]) if cache == "latent" else kv_heads * rng.choice([1, 2, 3, 4, 8])
        R = _log(rng, 1, 128)
        hi = min(_log(rng, 16, 32768), (1 << 19) // R)
        new = rng.choice([1, 1, _log(rng, 2, 64)])
        new = max(1, min(new, hi // 2, (1 << 26) // (R * hi * heads)))
        return {"op": op, "cache": cache, "requests": R, "lo": max(1, hi // 4), "hi": hi, "new_lo": 1, "new_hi": new, "heads": heads, "kv_heads": kv_heads, "dim": dim,
                "block": block, "dtype": dtype, "lay": lay}
    R = _log(rng, 1, 128)
    hi = min(_log(rng, 32, 32768), (1 << 18) // R)
    budget = max(1, int(hi * rng.uniform(0.1, 0.9)))
    first = rng.choice([0, min(4, budget // 4)])
    return {"op": op, "cache": cache, "requests": R, "lo": max(1, hi // 3), "hi": hi, "budget": budget, "first": first, "recent": rng.randrange(0, budget // 2 + 1),
            "kv_heads": kv_heads, "dim": dim, "block": block, "dtype": dtype, "lay": lay}


def _lengths(case):
    """Context length and new tokens of every request: part of the case, not of the seed.  new < 0 means the whole prompt."""
    rng = random.Random(case["lay"])
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["requests"])]
    if case["op"] == "evict":
        return lens, [min(n, case["budget"]) for n in lens]
    new = [n if case["new_lo"] < 0 else min(n, rng.randint(case["new_lo"], case["new_hi"])) for n in lens]
    return lens, new


def _pairs(lens, new):
    return sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lens, new))


def work(case):
    if case["op"] == "rows":
        row = 2 * (case["latent"] + ROPE)
        return {"bytes": case["tokens"] * (4 * row + 8), "flops": 0}       # rows read, cache written, cache read, rows written; slots
    lens, new = _lengths(case)
    if case["op"] == "latent":
        L, heads = case["latent"], case["heads"]
        return {"bytes": 2 * sum(lens) * (L + ROPE) + 2 * sum(new) * heads * (2 * L + ROPE) + 4 * sum(-(-n // case["block"]) for n in lens),
                "flops": 2 * heads * (2 * L + ROPE) * _pairs(lens, new)}
    if case["op"] == "expanded":
        heads = case["heads"]
        return {"bytes": 2 * sum(lens) * (heads * 256 + ROPE) + 2 * sum(new) * heads * (192 + 128), "flops": 2 * heads * (192 + 128) * _pairs(lens, new)}
    H, D = case["kv_heads"], case["dim"]
    row = D // 2 + D // GROUP if case["cache"] == "packed" else 2 * D
    width = _width(case, lens)
    if case["op"] == "weights":
        return {"bytes": sum(lens) * H * row + sum(new) * case["heads"] * (2 * D + 4) + 4 * case["requests"] * H * width,
                "flops": 2 * D * case["heads"] * _pairs(lens, new)}
    # weights read, the kept tokens' rows read and written; weights and indexes of the kept ones written
    planes = 1 if case["cache"] == "latent" else 2
    return {"bytes": 4 * H * sum(lens) + 2 * planes * sum(new) * H * row + 4 * case["requests"] * H * (width + case["budget"]), "flops": 0}


def _width(case, lens):
    return -(-max(lens) // case["block"]) * case["block"]


# ---- the 4-bit cache's bytes ------------------------------------------------------------------------------------------------------
def _chunk_place(dim):
    """Where the 16-byte chunk c of token n's codes sits in a tile: index n * chunks + c -> place."""
    c, rho = dim // 32, 256 // dim
    return [(n // rho) * 8 + (((n % rho) * c + k) ^ (2 * (n >> 2))) for n in range(TILE) for k in range(c)]


def _pack(x, t):
    """K rows x [blocks, B, H, D] as 4-bit codes and e4m3 scales: uint8 [blocks, B * H * 9 D / 16]."""
    nb, B, H, D = x.shape
    g = x.double().unflatten(-1, (-1, GROUP))
    s = torch.clamp(g.abs().amax(dim=-1) / (7.0 * t), max=448.0).float().to(torch.float8_e4m3fn)
    sv = s.double()[..., None] * t
    codes = (torch.where(sv > 0, torch.round(g / sv), torch.zeros_like(g)).clamp(-8, 7) + 8).to(torch.uint8).flatten(-2)
    c = codes.view(nb, B // TILE, TILE, H, D).permute(0, 3, 1, 2, 4)
    c = (c[..., 0::2] | (c[..., 1::2] << 4)).reshape(nb, H, B // TILE, TILE * D // 32, 16)
    out = torch.empty_like(c)
    out[:, :, :, _chunk_place(D)] = c
    sc = s.view(torch.uint8).view(nb, B // TILE, TILE, H, D // GROUP).permute(0, 3, 1, 2, 4)
    return torch.cat([out.reshape(nb, H, B // TILE, -1), sc.reshape(nb, H, B // TILE, -1)], dim=3).reshape(nb, -1)


def _unpack(data, B, H, D):
    """The K values the bytes of whole blocks [blocks, chunk] stand for, without the tensor scale, in 32 bits: [blocks, B, H, D]."""
    nb = data.shape[0]
    t = data.view(nb, H, B // TILE, 9 * D)
    c = t[..., :8 * D].reshape(nb, H, B // TILE, TILE * D // 32, 16)[:, :, :, _chunk_place(D)].reshape(nb, H, B // TILE, TILE, D // 2)
    c = torch.stack([c & 15, c >> 4], dim=-1).view(nb, H, B // TILE, TILE, D // GROUP, GROUP)
    s = t[..., 8 * D:].view(torch.float8_e4m3fn).to(torch.float32).reshape(nb, H, B // TILE, TILE, D // GROUP)
    return ((c.to(torch.float32) - 8.0) * s[..., None]).view(nb, H, B, D).permute(0, 2, 1, 3)


# ---- inputs -----------------------------------------------------------------------------------------------------------------------
def _values(gen, shape, dtype, scale=1.0):
    """Activations as a model makes them: normal, a few channels several times larger than the rest."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    loud = 1.0 + 7.0 * (torch.rand((1,) * (len(shape) - 1) + shape[-1:], generator=gen, device="cuda") < 0.05).float()
    return (x * loud * scale).to(dtype)


def _shuffled_tables(gen, lens, B, first=0):
    """Block tables with shuffled ids first, first + 1, ...; (tables, ids handed out)."""
    blocks = [-(-n // B) for n in lens]
    nb = sum(blocks)
    perm = first + torch.randperm(nb, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(max(blocks), 1)), -1, dtype=torch.int32, device="cuda")
    cols = torch.arange(table.shape[1], device="cuda")
    table[cols[None, :] < torch.tensor(blocks, device="cuda")[:, None]] = perm
    return table, nb


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(n):
    return _int([0] + [int(x) for x in np.cumsum(n)])


def _format(G, case):
    name = case.get("cache", "latent")
    if name == "latent":
        return {"bf16": G.KV_LATENT_BF16, "fp16": G.KV_LATENT_FP16}[case["dtype"]]
    return {"packed": G.KV_PACKED, "bf16": G.KV_BF16, "fp16": G.KV_FP16}[name]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 29)
    st = {"case": case}
    if own:
        from paper_2607_22648_b200 import binding
        st["G"] = binding
    return {"rows": _prepare_rows, "latent": _prepare_latent, "expanded": _prepare_expanded, "weights": _prepare_weights, "evict": _prepare_evict}[case["op"]](case, gen, st)


def _prepare_rows(case, gen, st):
    T, L, B, dtype = case["tokens"], case["latent"], case["block"], DTYPES[case["dtype"]]
    nb = -(-T // B) + 3
    st["latent"], st["rope"] = _values(gen, (T, L), dtype), _values(gen, (T, ROPE), dtype)
    perm = torch.randperm(nb, generator=gen, device="cuda")
    t = torch.arange(T, device="cuda")
    st["slots"] = torch.randperm(nb * B, generator=gen, device="cuda")[:T] if T <= 256 else perm[t // B] * B + t % B
    if own:
        G = st["G"]
        st["layout"] = G.KVLayout(1, L + ROPE, B, _format(G, case))
        st["cache"] = G.PagedKV(1, nb, st["layout"].chunk_bytes)
        st["out"] = (torch.empty_like(st["latent"]), torch.empty_like(st["rope"]))
    return st


def _prepare_latent(case, gen, st):
    L, B, dtype = case["latent"], case["block"], DTYPES[case["dtype"]]
    lens, new = _lengths(case)
    st["lens"], st["new"] = lens, new       # a user's program knows its requests on the host too
    st["tables"], nb = _shuffled_tables(gen, lens, B)
    st["lengths"], st["offsets"] = _int(lens), _starts(new)
    # the two layers of a latent cache lie where K and V of one layer would
    st["data"] = torch.zeros((2, nb, B * (L + ROPE)), dtype=dtype, device="cuda")
    st["layer"] = case["lay"] & 1
    st["data"][st["layer"]] = _values(gen, (nb * B, L + ROPE), dtype).view(nb, -1)
    st["q_latent"], st["q_rope"] = _values(gen, (sum(new), case["heads"], L), dtype, 0.5), _values(gen, (sum(new), case["heads"], ROPE), dtype)
    st["scale"] = 192 ** -0.5
    if own:
        G = st["G"]
        st["layout"] = G.KVLayout(1, L + ROPE, B, _format(G, case))
        st["cache"] = G.PagedKV(1, nb, st["layout"].chunk_bytes, tensors=[st["data"]])
        st["workspace"] = G.latent_workspace(st["layout"])
        st["out"] = torch.empty_like(st["q_latent"])
        st["max_new"] = max(new)
    return st


def _prepare_expanded(case, gen, st):
    H, dtype = case["heads"], DTYPES[case["dtype"]]
    lens, new = _lengths(case)
    st["lens"], st["new"] = lens, new
    st["q"] = _values(gen, (sum(new), H, 192), dtype, 0.5)
    st["kv"] = _values(gen, (sum(lens), H, 256), dtype)         # one matrix product's output: keys without rotation, and values
    st["rope"] = _values(gen, (sum(lens), ROPE), dtype)
    st["offsets"], st["key_offsets"] = _starts(new), _starts(lens)
    if own:
        st["out"] = torch.empty((sum(new), H, 128), dtype=dtype, device="cuda")
        st["max_new"] = max(new)
    return st


def _prepare_weights(case, gen, st):
    H, D, B, heads, dtype = case["kv_heads"], case["dim"], case["block"], case["heads"], DTYPES[case["dtype"]]
    lens, new = _lengths(case)
    st["lens"], st["new"] = lens, new
    st["tables"], nb = _shuffled_tables(gen, lens, B)
    st["lengths"], st["offsets"] = _int(lens), _starts(new)
    k = _values(gen, (nb, B, H, D), dtype)
    if case["cache"] == "packed":
        plane = torch.cat([_pack(k[i:i + 1024], K_SCALE) for i in range(0, nb, 1024)])      # the 64-bit quantiser's temporaries stay small
    else:
        plane = k.view(nb, -1).view(torch.uint8)
    del k
    st["layer"] = case["lay"] & 1 if case["cache"] == "latent" else 0
    st["data"] = torch.zeros((2,) + plane.shape, dtype=torch.uint8, device="cuda")
    st["data"][st["layer"]] = plane
    st["q"] = _values(gen, (sum(new), heads, D), dtype, 0.5 if case["cache"] == "latent" else 1.0)
    st["scale"] = (192 if case["cache"] == "latent" else D) ** -0.5
    # what the attention before it left: the logarithm of every row's sum
    lse, at = torch.empty((sum(new), heads), device="cuda"), 0
    for r, (n, m) in enumerate(zip(lens, new)):
        for h in range(H):
            s = _scores(st, r, at, h, torch.float32)
            lse[at:at + m, h * (heads // H):(h + 1) * (heads // H)] = torch.logsumexp(s, dim=2).t()
        at += m
    st["lse"] = lse
    width = _width(case, lens)
    if own:
        G = st["G"]
        st["layout"] = G.KVLayout(H, D, B, _format(G, case), K_SCALE, V_SCALE) if case["cache"] == "packed" else G.KVLayout(H, D, B, _format(G, case))
        st["cache"] = G.PagedKV(1, nb, st["layout"].chunk_bytes, tensors=[st["data"]])
        st["max_new"] = max(new)
    st["weights"] = torch.zeros((len(lens), H, width), device="cuda")
    return st


def _keys(st, r, h):
    """Keys of one request and kv head [n, D], 32 bits."""
    c = st["case"]
    H, D, B, n = c["kv_heads"], c["dim"], c["block"], st["lens"][r]
    data = st["data"][st["layer"]][st["tables"][r, :-(-n // B)].long()]
    if c["cache"] == "packed":
        return _unpack(data, B, H, D)[:, :, h].reshape(-1, D)[:n] * K_SCALE
    return data.view(DTYPES[c["dtype"]]).view(-1, H, D)[:n, h].float()


def _scores(st, r, at, h, dtype):
    """Scaled scores [group, new, n] of one request and kv head, minus infinity behind a row's position."""
    c = st["case"]
    n, m, G = st["lens"][r], st["new"][r], c["heads"] // c["kv_heads"]
    q = st["q"][at:at + m, h * G:(h + 1) * G].to(dtype).transpose(0, 1)
    s = torch.matmul(q, _keys(st, r, h).to(dtype).t()) * st["scale"]
    hidden = torch.arange(n, device="cuda")[None, :] > (n - m + torch.arange(m, device="cuda"))[:, None]
    return s.masked_fill_(hidden, float("-inf"))


def _prepare_evict(case, gen, st):
    H, D, B, dtype = case["kv_heads"], case["dim"], case["block"], DTYPES[case["dtype"]]
    lens, kept = _lengths(case)
    st["lens"] = lens
    st["tables"], nb = _shuffled_tables(gen, lens, B)
    st["to_tables"], nd = _shuffled_tables(gen, kept, B, nb)       # the evicted copy gets blocks of its own, the full one stays (others share it)
    st["source"] = nb
    st["layer"] = case["lay"] & 1 if case["cache"] == "latent" else 0
    st["planes"] = [st["layer"]] if case["cache"] == "latent" else [0, 1]
    st["data"] = torch.zeros((2, nb + nd, B * H * D), dtype=dtype, device="cuda")
    for p in st["planes"]:
        st["data"][p, :nb] = _values(gen, (nb, B * H * D), dtype, 1.0 if p == 0 else 0.25)
    st["lengths"] = _int(lens)
    # accumulated attention: a few tokens have most of it; some have none
    w = torch.exp(2.0 * torch.randn((len(lens), H, _width(case, lens)), generator=gen, device="cuda"))
    w *= (torch.rand(w.shape, generator=gen, device="cuda") > 0.05).float()
    st["weights"] = w * (torch.arange(w.shape[2], device="cuda") < st["lengths"][:, None, None]).float()
    if own:
        G = st["G"]
        st["layout"] = G.KVLayout(H, D, B, _format(G, case))
        st["cache"] = G.PagedKV(1, nb + nd, st["layout"].chunk_bytes, tensors=[st["data"]])
        st["kept"] = torch.empty((len(lens), H, case["budget"]), dtype=torch.int32, device="cuda")
        st["lengths_out"], st["weights_out"] = torch.empty_like(st["lengths"]), torch.empty_like(st["weights"])
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------------------------
def run(state):
    return {"rows": _run_rows, "latent": _run_latent, "expanded": _run_expanded, "weights": _run_weights, "evict": _run_evict}[state["case"]["op"]](state)


def _run_rows(st):
    if own:
        G = st["G"]
        G.latent_write(st["layout"], st["cache"], 0, st["latent"], st["rope"], st["slots"])
        return G.latent_read(st["layout"], st["cache"], 0, st["slots"], latent=st["out"][0], rope=st["out"][1])
    c = st["case"]
    rows = torch.cat([st["latent"], st["rope"]], dim=1)
    cache = torch.empty(((-(-c["tokens"] // c["block"]) + 3) * c["block"], rows.shape[1]), dtype=rows.dtype, device="cuda")
    cache[st["slots"]] = rows
    back = cache[st["slots"]]
    return back[:, :c["latent"]].contiguous(), back[:, c["latent"]:].contiguous()


def _run_latent(st):
    c = st["case"]
    if own:
        return st["G"].latent_attend(st["layout"], st["cache"], st["layer"], st["q_latent"], st["q_rope"], st["offsets"], st["lengths"], st["tables"], st["max_new"],
                                     st["scale"], out=st["out"], workspace=st["workspace"])
    L, B = c["latent"], c["block"]
    out, at = torch.zeros_like(st["q_latent"]), 0
    for r, (n, m) in enumerate(zip(st["lens"], st["new"])):
        rows = st["data"][st["layer"]][st["tables"][r, :-(-n // B)].long()].view(-1, L + ROPE)[:n].float()
        hidden = torch.arange(n, device="cuda")[None, :] > (n - m + torch.arange(m, device="cuda"))[:, None]
        q = torch.cat([st["q_latent"][at:at + m], st["q_rope"][at:at + m]], dim=2).float()
        s = (torch.matmul(q, rows.t()) * st["scale"]).masked_fill_(hidden[:, None, :], float("-inf"))
        s = torch.exp(s - s.amax(dim=-1, keepdim=True))
        s = s / s.sum(dim=-1, keepdim=True)
        out[at:at + m] = torch.matmul(s, rows[:, :L]).to(out.dtype)
        at += m
    return out


def _run_expanded(st):
    c = st["case"]
    k, v = st["kv"][:, :, :128], st["kv"][:, :, 128:]
    if own:
        return st["G"].expanded_attend(st["q"], k, st["rope"], v, st["offsets"], st["key_offsets"], st["max_new"], out=st["out"])
    out, at, k0 = torch.zeros((sum(st["new"]), c["heads"], 128), dtype=st["q"].dtype, device="cuda"), 0, 0
    for n, m in zip(st["lens"], st["new"]):
        hidden = torch.arange(n, device="cuda")[None, :] > (n - m + torch.arange(m, device="cuda"))[:, None]
        rope = st["rope"][k0:k0 + n].float()
        for h in range(c["heads"]):           # one head at a time: the scores of a long prompt are large
            q = st["q"][at:at + m, h].float()
            s = torch.matmul(q[:, :128], k[k0:k0 + n, h].float().t()) + torch.matmul(q[:, 128:], rope.t())
            s = (s * 192 ** -0.5).masked_fill_(hidden, float("-inf"))
            s = torch.exp(s - s.amax(dim=-1, keepdim=True))
            s = s / s.sum(dim=-1, keepdim=True)
            out[at:at + m, h] = torch.matmul(s, v[k0:k0 + n, h].float()).to(out.dtype)
        at += m
        k0 += n
    return out


def _run_weights(st):
    c = st["case"]
    if own:
        return st["G"].attend_weights(st["layout"], st["cache"], st["layer"], st["q"], st["lse"], st["offsets"], st["lengths"], st["tables"], st["max_new"], st["weights"],
                                      scale=st["scale"], accumulate=False)
    out, at, G = torch.zeros_like(st["weights"]), 0, c["heads"] // c["kv_heads"]
    for r, (n, m) in enumerate(zip(st["lens"], st["new"])):
        for h in range(c["kv_heads"]):
            p = torch.exp(_scores(st, r, at, h, torch.float32) - st["lse"][at:at + m, h * G:(h + 1) * G].t()[:, :, None])
            out[r, h, :n] = p.sum(dim=(0, 1))
        at += m
    return out


def _run_evict(st):
    c = st["case"]
    budget, first, recent, B, H, D = c["budget"], c["first"], c["recent"], c["block"], c["kv_heads"], c["dim"]
    if own:
        G = st["G"]
        kept, lengths, weights = G.select_tokens(st["weights"], st["lengths"], budget, first, recent, kept=st["kept"], lengths_out=st["lengths_out"],
                                                 weights_out=st["weights_out"])
        G.kv_compact(st["layout"], st["cache"], st["layer"], kept, lengths, st["tables"], to_tables=st["to_tables"])
        return (kept, lengths, weights) + tuple(st["data"][p, st["source"]:] for p in st["planes"])
    R, _, width = st["weights"].shape
    kept = torch.full((R, H, budget), -1, dtype=torch.int32, device="cuda")
    weights = torch.zeros_like(st["weights"])
    out = [torch.zeros_like(st["data"][p, st["source"]:]).view(-1, H, D) for p in st["planes"]]
    heads = torch.arange(H, device="cuda")[:, None]
    for r, n in enumerate(st["lens"]):
        m = min(n, budget)
        if n <= budget:
            ids = torch.arange(n, device="cuda").expand(H, n)
        else:
            order = torch.sort(st["weights"][r, :, first:n - recent], dim=1, descending=True, stable=True).indices[:, :budget - first - recent] + first
            always = torch.cat([torch.arange(first, device="cuda"), torch.arange(n - recent, n, device="cuda")]).expand(H, first + recent)
            ids = torch.sort(torch.cat([order, always], dim=1), dim=1).values
        kept[r, :, :m] = ids.to(torch.int32)
        weights[r, :, :m] = st["weights"][r].gather(1, ids)
        at = torch.arange(m, device="cuda")
        to = (st["to_tables"][r, at // B].long() - st["source"]) * B + at % B
        slot = st["tables"][r, ids // B].long() * B + ids % B
        for p, o in zip(st["planes"], out):
            o[to[None, :], heads] = st["data"][p].view(-1, H, D)[slot, heads]
    lengths = torch.clamp(st["lengths"], max=budget)
    return (kept, lengths, weights) + tuple(o.view(-1, B * H * D) for o in out)


# ---- the definitions, in 64 bits ----------------------------------------------------------------------------------------------------
def _e4m3_values():
    """float64 values of the 256 e4m3 bytes: 4 exponent bits of bias 7, 3 mantissa bits, subnormals, no infinities."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    return torch.from_numpy(np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0)) * np.where(b & 128, -1.0, 1.0)).cuda()


def exact(case, seed):
    st = prepare(case, seed)
    return {"rows": _exact_rows, "latent": _exact_latent, "expanded": _exact_expanded, "weights": _exact_weights, "evict": _exact_evict}[case["op"]](st)


def _exact_rows(st):
    return st["latent"].double(), st["rope"].double()       # 16-bit values are kept as they are


def _softmax64(s):
    e = (s - s.max(dim=-1, keepdim=True).values).exp()
    return e / e.sum(dim=-1, keepdim=True)


def _exact_latent(st):
    c = st["case"]
    L, B = c["latent"], c["block"]
    rows64 = st["data"][st["layer"]].view(-1, B, L + ROPE)
    out, first = torch.zeros(st["q_latent"].shape, dtype=torch.float64, device="cuda"), 0
    for r, (n, m) in enumerate(zip(st["lens"], st["new"])):
        tok = torch.arange(n, device="cuda")
        c_j = rows64[st["tables"][r].long()[tok // B], tok % B].double()
        for i in range(m):
            seen = c_j[:n - m + i + 1]
            s = (st["q_latent"][first + i].double() @ seen[:, :L].t() + st["q_rope"][first + i].double() @ seen[:, L:].t()) * st["scale"]
            out[first + i] = _softmax64(s) @ seen[:, :L]
        first += m
    return out


def _exact_expanded(st):
    c = st["case"]
    out, at, k0 = torch.zeros((sum(st["new"]), c["heads"], 128), dtype=torch.float64, device="cuda"), 0, 0
    for n, m in zip(st["lens"], st["new"]):
        for h in range(c["heads"]):
            k = torch.cat([st["kv"][k0:k0 + n, h, :128], st["rope"][k0:k0 + n]], dim=1).double()
            v = st["kv"][k0:k0 + n, h, 128:].double()
            for i in range(0, m, 2048):
                rows = torch.arange(i, min(i + 2048, m), device="cuda")
                s = st["q"][at + rows, h].double() @ k.t() / math.sqrt(192)
                s = torch.where(torch.arange(n, device="cuda")[None, :] <= (n - m + rows)[:, None], s, -math.inf)
                out[at + rows, h] = _softmax64(s) @ v
        at += m
        k0 += n
    return out


def _exact_weights(st):
    c = st["case"]
    H, D, B, G = c["kv_heads"], c["dim"], c["block"], c["heads"] // c["kv_heads"]
    plane = st["data"][st["layer"]]
    out, first = torch.zeros(st["weights"].shape, dtype=torch.float64, device="cuda"), 0
    if c["cache"] == "packed":
        decode, place = _e4m3_values(), torch.tensor(_chunk_place(D), device="cuda")
    for r, (n, m) in enumerate(zip(st["lens"], st["new"])):
        tok = torch.arange(n, device="cuda")
        blk, inb = st["tables"][r].long()[tok // B], tok % B
        for h in range(H):
            if c["cache"] == "packed":
                tiles = plane.view(-1, H, B // TILE, 9 * D)[blk, h, inb // TILE]               # one tile per token: [n, 9 D]
                i, d = inb % TILE, torch.arange(D, device="cuda")
                byte = place[i[:, None] * (D // 32) + d[None, :] // 32] * 16 + (d[None, :] % 32) // 2
                code = (tiles.gather(1, byte) >> (4 * (d % 2)).to(torch.uint8)) & 15
                scale = tiles.gather(1, 8 * D + i[:, None] * (D // GROUP) + d[None, :] // GROUP)
                k = (code.double() - 8.0) * decode[scale.long()] * K_SCALE
            else:
                k = plane.view(DTYPES[c["dtype"]]).view(-1, B, H, D)[blk, inb, h].double()
            for i in range(m):
                end = n - m + i + 1
                s = st["q"][first + i, h * G:(h + 1) * G].double() @ k[:end].t() * st["scale"]
                out[r, h, :end] += torch.exp(s - st["lse"][first + i, h * G:(h + 1) * G].double()[:, None]).sum(dim=0)
        first += m
    return out


def _exact_evict(st):
    c = st["case"]
    B, H, D = c["block"], c["kv_heads"], c["dim"]
    w = st["weights"].double().cpu().numpy()
    R, _, width = w.shape
    kept, weights = np.full((R, H, c["budget"]), -1, dtype=np.int64), np.zeros((R, H, width))
    src, dst = st["tables"].long().cpu().numpy(), st["to_tables"].long().cpu().numpy() - st["source"]
    frm, to, hd = [], [], []
    for r, n in enumerate(st["lens"]):
        m = min(n, c["budget"])
        for h in range(H):
            if n <= c["budget"]:
                ids = np.arange(n)
            else:
                idx = np.arange(c["first"], n - c["recent"])
                best = idx[np.lexsort((idx, -w[r, h, idx]))][:c["budget"] - c["first"] - c["recent"]]
                ids = np.sort(np.concatenate([np.arange(c["first"]), best, np.arange(n - c["recent"], n)]))
            kept[r, h, :m], weights[r, h, :m] = ids, w[r, h, ids]
            i = np.arange(m)
            frm.append(src[r, ids // B] * B + ids % B)
            to.append(dst[r, i // B] * B + i % B)
            hd.append(np.full(m, h))
    frm, to, hd = (torch.from_numpy(np.concatenate(x)).cuda() for x in (frm, to, hd))
    outs = []
    for p in st["planes"]:
        o = torch.zeros((st["data"].shape[1] - st["source"]) * B, H, D, dtype=torch.float32, device="cuda")
        o[to, hd] = st["data"][p].view(-1, H, D)[frm, hd].float()
        outs.append(o.view(-1, B * H * D))
    lengths = [min(n, c["budget"]) for n in st["lens"]]
    return (torch.from_numpy(kept), torch.tensor(lengths), torch.from_numpy(weights)) + tuple(outs)
