"""Logarithms of the attention's sums, what every cached token was given, the choice of tokens to keep and their move, on the GPU against the definitions in 64 bits."""
import math
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

from tests import operators_reference as ref
from tests import test_latent_gpu as latent
from tests import test_operators_gpu as ops

dev, gen_of, rows, make = ops.dev, ops.gen_of, ops.rows, ops.make
FORMATS = ops.FORMATS


@pytest.fixture(scope="module")
def G():
    from paper_2607_22648_b200 import binding
    return binding


def scores_of(q, keys, scale, packed):
    """Scores [heads, n] in 64 bits of one row, and how far they may be off in 32: sums of exact products (one step of 2^-23 of the running sum per addend), the
    scale factor and the exponential 2^-20; bf16 rows over the 4-bit cache go as fp16, off by 2^-25 of the row's largest element."""
    q = q.double()
    D = q.shape[-1]
    s = torch.einsum("hd,nhd->hn", q, keys) * scale
    big = torch.einsum("hd,nhd->hn", q.abs(), keys.abs()) * abs(scale)
    e = (D + 8) * 2.0 ** -23 * big.amax(1, keepdim=True) + 2.0 ** -20
    if packed:
        e = e + 2.0 ** -25 * q.abs().amax(1, keepdim=True) * keys.abs().sum(-1).amax(0)[:, None] * abs(scale)
    return s, e


def expected(b, k_values, scale, block, packed, group, lse=None):
    """lse [T, heads] and weights [R, kv heads, longest] in 64 bits, and their errors' bounds.  With lse given the weights are those that follow from it."""
    T, heads = b["q"].shape[:2]
    H = heads // group
    out_lse, e_lse = torch.full((T, heads), math.nan, dtype=torch.float64, device="cuda"), torch.zeros(T, heads, dtype=torch.float64, device="cuda")
    width = max(b["lens"] + [1])
    w = torch.zeros(len(b["lens"]), H, width, dtype=torch.float64, device="cuda")
    e_w = torch.zeros_like(w)
    for r, n in enumerate(b["lens"]):
        a, e = b["offsets"][r], b["offsets"][r + 1]
        if n > 0:
            k, ok = ref.gather(k_values, b["tables"][r], n, block)
        for i in range(a, e):
            pos = n - (e - a) + (i - a)
            see = torch.zeros(max(n, 0), dtype=torch.bool, device="cuda")
            if pos >= 0:
                see[:pos + 1] = ok[:pos + 1]
            if not bool(see.any()):
                out_lse[i] = -math.inf
                continue
            s, err = scores_of(b["q"][i], k[see].repeat_interleave(group, 1), scale, packed)
            out_lse[i], e_lse[i] = torch.logsumexp(s, 1), 2 * err[:, 0] + 2.0 ** -18
            given = out_lse[i] if lse is None else lse[i].double()
            p = torch.exp(s - given[:, None]).view(H, group, -1)
            at = see.nonzero()[:, 0]
            w[r][:, at] += p.sum(1)
            # a weight is off by what its exponent is, relative; the exponent is rounded to 2^-24 of its size and lse's; sums round once per addend
            size = s.abs() + given[:, None].abs()
            e_w[r][:, at] += (p * (2 * err[:, 0, None] + 2.0 ** -22 * size + 2.0 ** -21).view(H, group, -1)).sum(1) + (e - a) * group * 2.0 ** -24 * p.sum(1)
    return out_lse, e_lse, w, e_w


def check_weights(got, want, err, lens):
    for r, n in enumerate(lens):
        n = max(n, 0)
        off = (got[r, :, :n].double() - want[r, :, :n]).abs()
        assert bool((off <= err[r, :, :n] + 1e-30).all()), (r, float((off / (err[r, :, :n] + 1e-30)).max()))
        assert bool((got[r, :, n:] == 0).all()), r


def run(G, b, accumulate=False, weights=None, scale=None, status=None):
    heads, max_new = b["q"].shape[1], max(b["new"] + [1])
    scale = b["q"].shape[2] ** -0.5 if scale is None else scale
    lse = torch.full(b["q"].shape[:2], 9.0, device="cuda")
    out = torch.full_like(b["out"], 5.0)
    plain = torch.full_like(b["out"], 5.0)
    args = (b["lay"], b["cache"], 0, b["q"], dev(b["offsets"]), dev(b["lens"]), b["tables"], max_new)
    G.attend(*args, scale=scale, out=plain)
    G.attend(*args, scale=scale, out=out, lse=lse)
    assert torch.equal(out.view(torch.int16), plain.view(torch.int16))
    if weights is None:
        weights = torch.full((len(b["lens"]), b["lay"].heads, max(b["lens"] + [1])), 3.0, device="cuda")
    G.attend_weights(b["lay"], b["cache"], 0, b["q"], lse, dev(b["offsets"]), dev(b["lens"]), b["tables"], max_new, weights, scale=scale, accumulate=accumulate, status=status)
    return lse, weights


def check(G, b, scale=None):
    lse, w = run(G, b, scale=scale)
    packed, s = b["lay"].format == G.KV_PACKED and b["q"].dtype == torch.bfloat16, b["q"].shape[2] ** -0.5 if scale is None else scale
    group = b["q"].shape[1] // b["lay"].heads
    T = b["offsets"][-1]
    want, err, _, _ = expected(b, b["values"][0], s, b["lay"].block_tokens, packed, group)
    fine = (lse[:T].double() - want[:T]).abs() <= err[:T] + 2.0 ** -21 * want[:T].abs()
    assert bool((fine | (lse[:T].double() == want[:T])).all()) and bool((lse[T:] == 9.0).all())
    _, _, ww, e = expected(b, b["values"][0], s, b["lay"].block_tokens, packed, group, lse=lse)
    check_weights(w, ww, e, b["lens"])


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("dim,heads,kv_heads", [(128, 32, 8), (64, 6, 2), (128, 5, 5), (64, 16, 1)])
def test_decode_ragged(G, fmt, dtype, dim, heads, kv_heads):
    lens = [1, 2, 15, 16, 17, 127, 128, 129, 500]
    check(G, make(G, getattr(G, fmt), dtype, heads, kv_heads, dim, 16, lens, [1] * len(lens), seed=dim + heads))


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("block", [16, 48])
def test_mixed_new_tokens_and_empty_rows(G, fmt, dtype, block):
    lens, new = [0, 5, 40, 200, 0, 33, 130, 1, 64], [1, 0, 40, 3, 0, 36, 130, 1, 64]
    check(G, make(G, getattr(G, fmt), dtype, 8, 2, 128, block, lens, new, seed=9, strided=block == 48))
    check(G, make(G, getattr(G, fmt), dtype, 8, 2, 128, block, [3000, 20], [40, 20], seed=10))            # row tiles cut into chunks and joined
    check(G, make(G, getattr(G, fmt), dtype, 8, 2, 128, block, [3000, 20], [1, 1], seed=11))


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("scale", [-0.1, 0.0, 3.0])
def test_scales(G, fmt, dtype, scale):
    check(G, make(G, getattr(G, fmt), dtype, 4, 2, 64, 16, [200, 40], [1, 20], seed=3, spread=0.5), scale=scale)


@pytest.mark.parametrize("block", [5, 24])
def test_odd_blocks_of_a_16_bit_cache(G, block):
    check(G, make(G, G.KV_BF16, torch.bfloat16, 8, 2, 128, block, [300, 7, 64], [1, 2, 20], seed=block))


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("new", [1, 30])
def test_weights_add_up(G, fmt, dtype, new):
    b = make(G, getattr(G, fmt), dtype, 8, 2, 64, 16, [200, 64, 31], [new] * 3, seed=21)
    lse, w = run(G, b)
    start = torch.rand(3, 3, 230, device="cuda")[:, 1:, :]            # strided, wider than the requests
    both = start.clone()
    wide = torch.empty(3, 4, 230, device="cuda")[:, :2]
    wide.copy_(both)
    run(G, b, accumulate=True, weights=wide)
    n = w.shape[2]
    assert torch.equal(wide[:, :, :n], torch.where(torch.arange(n, device="cuda") < dev(b["lens"])[:, None, None], both[:, :, :n] + w, both[:, :, :n]))
    assert torch.equal(wide[:, :, n:], both[:, :, n:])
    narrow = torch.full((3, 2, 50), 3.0, device="cuda")               # tokens behind the width are not counted
    run(G, b, weights=narrow)
    assert torch.equal(narrow, w[:, :, :50])
    # every row's weights add up to one for each head
    for r in range(3):
        assert float((w[r].double().sum() - min(new, b["lens"][r]) * 8).abs()) < 1e-3


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_entries_outside_the_cache(G, fmt, dtype):
    b = make(G, getattr(G, fmt), dtype, 8, 2, 128, 16, [300, 90], [3, 1], seed=5)
    t = b["tables"].clone()
    t[0, 1], t[0, 18], t[1, 0] = 1 << 20, -5, -1
    b["tables"] = t
    status = dev([0])
    run(G, b, status=status)
    assert int(status.item()) == G.S_BOUNDS
    check(G, b)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_what_is_not_finite_stays_with_its_token(G, fmt, dtype):
    b = make(G, getattr(G, fmt), dtype, 8, 2, 128, 16, [200, 40], [50, 1], seed=6)
    clean = run(G, b)[1].clone()
    slot = dev([int(b["tables"][0, 190 // 16]) * 16 + 190 % 16], torch.int64)
    bad = torch.full((1, 2, 128), math.nan, dtype=dtype, device="cuda")
    lse, _ = run(G, b)
    G.kv_write(b["lay"], b["cache"], 0, bad, bad, slot)
    w = torch.empty_like(clean)
    G.attend_weights(b["lay"], b["cache"], 0, b["q"], lse, dev(b["offsets"]), dev(b["lens"]), b["tables"], 50, w, accumulate=False)
    assert bool(w[0, :, 190].isnan().all())
    w[0, :, 190] = clean[0, :, 190]
    assert torch.equal(w, clean)


@pytest.mark.parametrize("dtype", latent.BOTH)
@pytest.mark.parametrize("L,heads,new", [(512, 64, 1), (256, 16, 1), (512, 16, 20), (512, 100, 2)])
def test_latent_cache(G, dtype, L, heads, new):
    lens = [1, 63, 64, 65, 400, 0]
    b = latent.make(G, L, dtype, heads, 16, lens, [min(new, max(n, 1)) for n in lens], seed=heads)
    latent.call(G, b)
    w = torch.full((6, 1, 410), 3.0, device="cuda")
    status = dev([0])
    G.attend_weights(b["lay"], b["cache"], b["layer"], b["q"], b["lse"], dev(b["offsets"]), dev(lens), b["tables"], max(b["new"]), w, scale=b["scale"], accumulate=False,
                     status=status)
    assert int(status.item()) == 0
    ref_b = dict(b, q=b["q"])
    _, _, want, err = expected(ref_b, b["values"].unsqueeze(2), b["scale"], 16, False, heads, lse=b["lse"])
    check_weights(w, want, err, lens)


def test_a_wait_that_runs_out_is_reported(G):
    b = make(G, G.KV_BF16, torch.bfloat16, 8, 2, 128, 16, [3000] * 8, [16] * 8, seed=30)
    lse, w = run(G, b)
    args = (b["lay"], b["cache"], 0, b["q"], lse, dev(b["offsets"]), dev(b["lens"]), b["tables"], 16)
    for _ in range(4):
        status, again = dev([0]), torch.zeros_like(w)
        G.attend_weights(*args, again, accumulate=False, status=status, wait_polls=1)
        assert int(status.item()) in (0, G.S_TIMEOUT) and (int(status.item()) or torch.equal(again, w))
    G.attend_weights(*args, again, accumulate=False)
    assert torch.equal(again, w)


# ---- the choice of tokens -----------------------------------------------------------------------------------------------------------
def choose(weights, lengths, budget, first, recent):
    """By sorting: (kept, lengths, weights) as lists."""
    kept, lens, out = [], [], []
    for r, raw in enumerate(lengths):
        width = len(weights[r][0])
        n = min(max(raw, 0), width)
        lens.append(min(n, budget))
        kept.append([])
        out.append([])
        for row in weights[r]:
            ids = list(range(n))
            if n > budget:
                inner = sorted(range(first, n - recent), key=lambda j: (-math.inf if math.isnan(row[j]) else -row[j] if row[j] != math.inf else -1e300, j))
                nan_first = [j for j in inner if math.isnan(row[j])] + [j for j in inner if not math.isnan(row[j])]
                ids = sorted(list(range(first)) + nan_first[:budget - first - recent] + list(range(n - recent, n)))
            kept[-1].append(ids + [-1] * (budget - len(ids)))
            out[-1].append([row[j] for j in ids] + [0.0] * (width - len(ids)))
    return kept, lens, out


def same(a, b):
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def check_choice(G, w, lengths, budget, first, recent):
    want = choose(w.tolist(), lengths, budget, first, recent)
    status = dev([0])
    for in_place in (False, True):
        src = w.clone()
        out = src if in_place else torch.full_like(w, 7.0)
        kept, lens, got = G.select_tokens(src, dev(lengths), budget, first, recent, weights_out=None if in_place else out, status=status)
        assert got is out and kept.tolist() == want[0] and lens.tolist() == want[1]
        assert same(got, torch.tensor(want[2], device="cuda"))
        assert in_place or same(src, w)
    clamped = any(n < 0 or n > w.shape[2] for n in lengths)
    assert int(status.item()) == (G.S_BOUNDS if clamped else 0)


@pytest.mark.parametrize("budget,first,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (16, 0, 0), (16, 4, 12), (100, 3, 30), (511, 0, 64), (512, 4, 100)])
def test_choice_over_lengths(G, budget, first, recent):
    gen = gen_of(budget)
    lengths = [0, 1, 2, budget - 1, budget, budget + 1, 513, 700, 1024, 1025, 1500, -4, 1600]
    w = torch.exp(2 * torch.randn(len(lengths), 2, 1500, generator=gen, device="cuda"))
    check_choice(G, w, lengths, budget, first, recent)


@pytest.mark.parametrize("kind", ["equal", "few", "zeros", "negative", "special", "bits"])
def test_choice_of_equal_and_special_weights(G, kind):
    gen = gen_of(7)
    w = torch.rand(2, 3, 900, generator=gen, device="cuda")
    if kind == "equal":
        w.fill_(0.25)
    elif kind == "few":
        w = (w * 4).floor()
    elif kind == "zeros":
        w = torch.where(w < 0.5, torch.zeros_like(w), -torch.zeros_like(w))
        w[:, :, 700] = 1e-40
    elif kind == "negative":
        w = w - 0.5
    elif kind == "special":
        w[w < 0.1], w[w > 0.9] = math.nan, math.inf
        w[0, 0] = math.nan
        w[1, 1, ::2] = -math.inf
    else:
        w = torch.randint(-2 ** 31, 2 ** 31 - 1, w.shape, generator=gen, device="cuda").to(torch.int32).view(torch.float32)
    for budget, first, recent in ((10, 0, 0), (300, 5, 20), (899, 0, 1)):
        check_choice(G, w, [900, 850], budget, first, recent)


@pytest.mark.parametrize("n", [8191, 8192, 8193, 20000])
def test_choice_of_long_requests(G, n):
    gen = gen_of(n)
    w = torch.exp(3 * torch.randn(1, 2, n, generator=gen, device="cuda"))
    w[0, 1] = (w[0, 1] * 8).floor()
    check_choice(G, w, [n], n // 3, 4, 128)
    check_choice(G, w, [n], n // 2, 0, 0)


@pytest.mark.parametrize("budget,first,recent", [(101, 0, 0), (150, 4, 140), (5000, 10, 100)])
def test_choice_with_a_budget_beyond_the_rows(G, budget, first, recent):
    w = torch.rand(4, 3, 100, generator=gen_of(8), device="cuda")
    check_choice(G, w, [100, 0, 37, 99], budget, first, recent)
    check_choice(G, w, [100, -1, 37, 101], budget, first, recent)
    kept = torch.full((4, 3, budget), 7, dtype=torch.int32, device="cuda")
    got = G.select_tokens(w, dev([100, 0, 37, 99]), budget, first, recent, kept=kept, weights_out=torch.empty_like(w))[0]
    assert got is kept and kept.tolist() == choose(w.tolist(), [100, 0, 37, 99], budget, first, recent)[0]
    for bad in ((budget, -1, 0), (budget, 0, -1), (budget, budget, 1)):
        with pytest.raises(G.PTStoreError):
            G.select_tokens(w, dev([1, 2, 3, 4]), *bad)


def test_choice_with_strides(G):
    gen = gen_of(3)
    big = torch.rand(5, 4, 3, 640, generator=gen, device="cuda")
    w = big[:, 1, :2, 8:608]
    before = big.clone()
    want = choose(w.tolist(), [600] * 5, 77, 2, 9)
    kept, lens, got = G.select_tokens(w, dev([600] * 5), 77, 2, 9)
    assert kept.tolist() == want[0] and got.data_ptr() == w.data_ptr() and torch.equal(w, torch.tensor(want[2], device="cuda"))
    before[:, 1, :2, 8:608] = w
    assert torch.equal(big, before)


# ---- the move -------------------------------------------------------------------------------------------------------------------------
CACHES = [("KV_PACKED", 2, 128, 16), ("KV_PACKED", 3, 64, 48), ("KV_BF16", 2, 128, 16), ("KV_FP16", 4, 64, 5), ("KV_LATENT_BF16", 1, 576, 8), ("KV_LATENT_FP16", 1, 320, 24)]


def values_at(G, lay, cache, layer, tables, r, n):
    """What the cache holds for the first n tokens of a request: a list of tensors [n, heads, ...]."""
    B = lay.block_tokens
    slots = torch.tensor([int(tables[r, p // B]) * B + p % B for p in range(n)], dtype=torch.int64, device="cuda")
    if lay.latent:
        return [torch.cat(G.latent_read(lay, cache, layer, slots), 1)[:, None].view(torch.int16)]
    dtype = torch.float16 if lay.format == G.KV_FP16 else torch.bfloat16
    return [x.view(torch.int16) for x in G.kv_read(lay, cache, layer, slots, dtype)]


@pytest.mark.parametrize("fmt,heads,dim,block", CACHES)
@pytest.mark.parametrize("in_place", [True, False])
def test_move(G, fmt, heads, dim, block, in_place):
    gen = gen_of(dim + block)
    lay = G.KVLayout(heads, dim, block, getattr(G, fmt))
    lens, budget, layer = [0, 1, 700, 699, 1400, 64, 900], 640, 1 if fmt.startswith("KV_LATENT") else 0
    blocks, to_blocks = [-(-n // block) for n in lens], [-(-min(n, budget) // block) for n in lens]
    nb = sum(blocks) + sum(to_blocks) + 1
    cache = G.PagedKV(1, nb, lay.chunk_bytes)
    cache.tensors[0].copy_(torch.randint(0, 256, cache.tensors[0].shape, generator=gen, device="cuda", dtype=torch.uint8))
    if fmt == "KV_PACKED":                                          # (scales that are not NaN, so that equal bytes are equal values and the other way round)
        cache.tensors[0].bitwise_and_(0x77)
    perm = torch.randperm(nb, generator=gen, device="cuda").int().tolist()

    def table(counts, at):
        width, t = max(counts) + 1, []
        for c in counts:
            t.append(perm[at:at + c] + [-1] * (width - c))
            at += c
        return dev(t).view(len(counts), width), at
    tables, at = table(blocks, 0)
    to, _ = table(to_blocks, at)
    w = torch.rand(len(lens), heads, max(lens), generator=gen, device="cuda")
    kept, new_lens, _ = G.select_tokens(w, dev(lens), budget, 3, 50, weights_out=torch.empty_like(w))
    before = [values_at(G, lay, cache, layer, tables, r, n) for r, n in enumerate(lens)]
    raw = cache.tensors[0].clone()
    status = dev([0])
    G.kv_compact(lay, cache, layer, kept, new_lens, tables, to_tables=None if in_place else to, status=status)
    assert int(status.item()) == 0
    for r, n in enumerate(lens):
        m = min(n, budget)
        got = values_at(G, lay, cache, layer, tables if in_place else to, r, m)
        for x, y in zip(got, before[r]):
            for h in range(heads):
                assert torch.equal(x[:, h], y[kept[r, h, :m].long(), h]), (r, h)
    # nothing else moved: the other layer, blocks of nobody, tokens behind the kept ones
    used = set(tables.flatten().tolist()) if in_place else set(to.flatten().tolist())
    others = torch.tensor([b for b in range(nb) if b not in used], device="cuda")
    assert torch.equal(cache.tensors[0][:, others], raw[:, others])
    if lay.latent:
        assert torch.equal(cache.tensors[0][1 - layer], raw[1 - layer])
    if in_place:
        for r, n in enumerate(lens):
            if n:
                for x, y in zip(values_at(G, lay, cache, layer, tables, r, n), before[r]):
                    assert torch.equal(x[min(n, budget):], y[min(n, budget):])


def test_move_skips_what_is_outside(G):
    lay = G.KVLayout(1, 64, 4, G.KV_BF16)
    cache = G.PagedKV(1, 6, lay.chunk_bytes)
    plane = cache.tensors[0].view(torch.bfloat16).view(2, 24, 64)
    plane.copy_(torch.arange(24, device="cuda")[None, :, None].expand(2, 24, 64))
    status = dev([0])
    # index 9 is outside the row, -1 too; the row's second entry is outside the cache; the target's second entry as well
    G.kv_compact(lay, cache, 0, dev([[[2, 9, -1, 5, 3, 1]]]), dev([6]), dev([[0, 99]]), to_tables=dev([[3, -2]]), status=status)
    assert int(status.item()) == G.S_BOUNDS
    assert plane[0, 12:16, 0].tolist() == [2, 13, 14, 15] and plane[1, 12:16, 5].tolist() == [2, 13, 14, 15]
    assert plane[0, :12, 0].tolist() == list(range(12)) and plane[0, 16:, 0].tolist() == list(range(16, 24))


# ---- as they are used: decode, add up, cut, go on -----------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,dtype", FORMATS + [("KV_LATENT_BF16", torch.bfloat16)])
def test_a_request_goes_on_over_its_evicted_cache(G, fmt, dtype):
    """Two requests decode behind prompts; at a limit each head keeps its heaviest tokens, the blocks behind them go back, and the next step's attention is that over the kept tokens."""
    gen = gen_of(77)
    is_latent = fmt.startswith("KV_LATENT")
    heads, kv_heads, dim, block = (8, 1, 576, 16) if is_latent else (8, 2, 128, 16)
    lay = G.KVLayout(kv_heads, dim, block, getattr(G, fmt)) if fmt != "KV_PACKED" else G.KVLayout(kv_heads, dim, block, G.KV_PACKED, 2.0 ** -4, 2.0 ** -6)
    cache = G.PagedKV(1, 64, lay.chunk_bytes)
    cache.tensors[0].fill_(0xFF)
    lens, budget, first, recent, scale = dev([300, 180]), 128, 2, 20, 0.08
    tables, held = torch.full((2, 24), -1, dtype=torch.int32, device="cuda"), None
    free_ids, count, status = torch.randperm(64, generator=gen, device="cuda").int(), dev([64]), dev([0])
    w = torch.zeros(2, kv_heads, 24 * block, device="cuda")

    def step(done):
        nonlocal held
        held, _ = G.assign_blocks(lens, held, tables, free_ids, count, block, status=status)
        off, slots, _ = G.map_slots(lens, done, tables, block, 480 if done is None else 2, status=status)
        T = slots.numel()
        max_new = 300 if done is None else 1
        q = rows(gen, (T, heads, dim), dtype)
        lse = torch.empty(T, heads, device="cuda")
        if is_latent:
            c, r = rows(gen, (T, 512), dtype), rows(gen, (T, 64), dtype)
            G.latent_write(lay, cache, 0, c, r, slots, status=status)
            out = G.latent_attend(lay, cache, 0, q[:, :, :512], q[:, :, 512:], off, lens, tables, max_new, scale, lse=lse, status=status)
        else:
            k, v = rows(gen, (T, kv_heads, dim), dtype), rows(gen, (T, kv_heads, dim), dtype)
            G.kv_write(lay, cache, 0, k, v, slots, status=status)
            out = G.attend(lay, cache, 0, q, off, lens, tables, max_new, scale=scale, lse=lse, status=status)
        G.attend_weights(lay, cache, 0, q, lse, off, lens, tables, max_new, w, scale=scale, status=status)
        return q, out, off
    q, _, _ = step(None)
    # a row's weights add up to one: each is off by what its score and the row's lse are, (D + 8) 2^-23 sum |q k| scale + 2^-20 each
    k = torch.cat([values_at(G, lay, cache, 0, tables, r, n)[0].view(torch.bfloat16 if fmt == "KV_PACKED" else dtype).double() for r, n in enumerate(lens.tolist())])
    big = float((q.double().abs().flatten(0, 1) @ k.abs().flatten(0, 1).t()).max()) * scale
    fp16_rows = 2.0 ** -25 * float(q.double().abs().max() * k.abs().sum(-1).max()) * scale if fmt == "KV_PACKED" and dtype == torch.bfloat16 else 0.0
    assert abs(float(w.double().sum()) - 480 * heads) < 480 * heads * 2 * ((dim + 8) * 2.0 ** -23 * big + 2.0 ** -20 + fp16_rows)
    full = [[x.clone() for x in values_at(G, lay, cache, 0, tables, r, n)] for r, n in enumerate(lens.tolist())]
    old = w.clone()
    kept, new_lens, _ = G.select_tokens(w, lens, budget, first, recent, status=status)
    G.kv_compact(lay, cache, 0, kept, new_lens, tables, status=status)
    lens.copy_(new_lens)
    used = 64 - int(count.item())
    held, _ = G.assign_blocks(lens, held, tables, free_ids, count, block, status=status)
    assert lens.tolist() == [128, 128] and 64 - int(count.item()) == 16 < used
    for r in range(2):
        best = choose(old[r:r + 1, :, :[300, 180][r]].tolist(), [[300, 180][r]], budget, first, recent)
        assert kept[r].tolist() == best[0][0]
    done = lens.clone()
    lens += 1
    q, out, off = step(done)
    assert int(status.item()) == 0
    held_as = torch.bfloat16 if fmt == "KV_PACKED" else dtype             # as values_at reads them (4-bit values are exact in bf16)
    for r in range(2):
        now = [x.view(held_as).double() for x in values_at(G, lay, cache, 0, tables, r, 129)]
        then = [x.view(held_as).double() for x in full[r]]
        for h in range(kv_heads):
            assert torch.equal(now[0][:128, h], then[0][kept[r, h].long(), h]) and torch.equal(now[-1][:128, h], then[-1][kept[r, h].long(), h])
        g = heads // kv_heads
        for h in range(heads):
            # weights and the output are rounded to 16 bits (of a 4-bit cache the weights are fp16), scores are off as scores_of says, weights below fp16's normal range by 2^-25
            s, err = scores_of(q[r, h:h + 1], now[0][:, h // g:h // g + 1], scale, fmt == "KV_PACKED" and dtype == torch.bfloat16)
            p, v = torch.softmax(s, 1)[0], now[0][:, 0, :512] if is_latent else now[1][:, h // g]
            want, spread = p @ v, p @ v.abs()
            tol = spread * (latent.HALF[torch.float16 if fmt == "KV_PACKED" else dtype] + 2 * err[0]) + latent.HALF[dtype] * want.abs() + 130 * 2.0 ** -25 * v.abs().max()
            assert bool(((out[r, h].double() - want).abs() <= tol).all()), (r, h)


def test_streams_and_graphs(G):
    b = make(G, G.KV_BF16, torch.bfloat16, 8, 2, 128, 16, [2000, 700], [1, 1], seed=50)
    lse, w = run(G, b)
    off, lens, out = dev(b["offsets"]), dev(b["lens"]), torch.empty_like(w)
    kept, new_lens = torch.empty(2, 2, 256, dtype=torch.int32, device="cuda"), dev([0, 0])
    compacted = torch.empty_like(w)

    def step():
        G.attend_weights(b["lay"], b["cache"], 0, b["q"], lse, off, lens, b["tables"], 1, out, accumulate=False)
        G.select_tokens(out, lens, 256, 4, 32, kept=kept, lengths_out=new_lens, weights_out=compacted)
        G.kv_compact(b["lay"], b["cache"], 0, kept, new_lens, b["tables"])
    raw = b["cache"].tensors[0].clone()
    step()
    want = [x.clone() for x in (out, kept, new_lens, compacted, b["cache"].tensors[0])]
    assert torch.equal(want[0], w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.stream(s):
        for g in graphs:
            with torch.cuda.graph(g, stream=s):
                step()
    for g in graphs:
        b["cache"].tensors[0].copy_(raw)
        for x in (out, kept, new_lens, compacted):
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip((out, kept, new_lens, compacted, b["cache"].tensors[0]), want):
            assert torch.equal(x, y)


def with_infinite_key(G, b, r, token, element, value):
    """One element of a cached token's key, for all heads."""
    B, lay = b["lay"].block_tokens, b["lay"]
    slot = dev([int(b["tables"][r, token // B]) * B + token % B], torch.int64)
    if lay.latent:
        c, p = G.latent_read(lay, b["cache"], b["layer"], slot)
        x = torch.cat([c, p], 1)
        x[:, element] = value
        G.latent_write(lay, b["cache"], b["layer"], x[:, :b["L"]].contiguous(), x[:, b["L"]:].contiguous(), slot)
    else:
        k, v = G.kv_read(lay, b["cache"], 0, slot, b["q"].dtype)
        k[:, :, element] = value
        G.kv_write(lay, b["cache"], 0, k, v, slot)


def check_infinite_scores(G, b, new, scale):
    """A token whose scores are all minus infinity was given nothing, one with an infinite score (beside a finite logarithm) infinitely much; the others what they were given before."""
    element, first = 5, -b["q"].abs()[:, :, 5] - 0.5
    b["q"][:, :, element] = first if scale > 0 else -first
    T, heads = b["q"].shape[:2]
    lse, layer = torch.empty(T, heads, device="cuda"), b.get("layer", 0)
    args = (dev(b["offsets"]), dev(b["lens"]), b["tables"], new)
    if b["lay"].latent:
        L = b["L"]
        G.latent_attend(b["lay"], b["cache"], layer, b["q"][:, :, :L], b["q"][:, :, L:], *args, scale, lse=lse)
    else:
        G.attend(b["lay"], b["cache"], 0, b["q"], *args, scale=scale, lse=lse)
    w = torch.empty(len(b["lens"]), b["lay"].heads, max(b["lens"]), device="cuda")
    G.attend_weights(b["lay"], b["cache"], layer, b["q"], lse, *args, w, scale=scale, accumulate=False)
    want = w.clone()
    assert bool(want.isfinite().all())
    for r, token, value, given in ((0, 30, math.inf, 0.0), (0, 141, -math.inf, math.inf), (1, 7, math.inf, 0.0)):
        with_infinite_key(G, b, r, token, element, value)
        want[r, :, token] = given
    G.attend_weights(b["lay"], b["cache"], layer, b["q"], lse, *args, w, scale=scale, accumulate=False)
    assert torch.equal(w, want)


SCALES = [0.08838834764, 0.1, -0.07, 0.05, 0.3, -0.125]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("fmt,dtype", FORMATS[2:])
@pytest.mark.parametrize("heads,new", [(32, 1), (8, 16), (32, 20)])
def test_infinite_scores(G, fmt, dtype, heads, new, scale):
    check_infinite_scores(G, make(G, getattr(G, fmt), dtype, heads, 2, 128, 16, [200, 40], [new] * 2, seed=6, spread=0.3), new, scale)


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("dtype", latent.BOTH)
@pytest.mark.parametrize("heads,new", [(16, 1), (64, 1), (64, 3)])
def test_infinite_scores_of_a_latent_cache(G, dtype, heads, new, scale):
    check_infinite_scores(G, latent.make(G, 512, dtype, heads, 16, [200, 40], [new] * 2, seed=6, spread=0.3), new, scale)


@pytest.mark.parametrize("fmt,dtype", FORMATS[2:])
@pytest.mark.parametrize("heads,new", [(2, 1), (8, 1), (30, 1), (8, 5), (32, 6), (8, 33), (6, 47)])
def test_infinite_scores_beside_rows_that_do_not_fill_a_chunk(G, fmt, dtype, heads, new):
    check_infinite_scores(G, make(G, getattr(G, fmt), dtype, heads, 2, 128, 16, [200, 60], [new] * 2, seed=7, spread=0.3), new, 0.09)


@pytest.mark.parametrize("dtype", latent.BOTH)
@pytest.mark.parametrize("L,heads,new", [(512, 5, 1), (256, 40, 1), (512, 20, 4)])
def test_infinite_scores_of_a_latent_cache_beside_rows_that_do_not_fill_a_chunk(G, L, dtype, heads, new):
    check_infinite_scores(G, latent.make(G, L, dtype, heads, 16, [200, 60], [new] * 2, seed=7, spread=0.3), new, 0.09)


@pytest.mark.parametrize("fmt,dtype", FORMATS + [("KV_LATENT_BF16", torch.bfloat16), ("KV_LATENT_FP16", torch.float16)])
@pytest.mark.parametrize("new", [1, 20])
def test_weights_of_large_scores_that_add_up_exactly(G, fmt, dtype, new):
    """Keys of two elements and scores near 950: sums of products are exact (at most 17 bits), so nothing is lost but in the exponent, which is the difference of two numbers of 48 bits
    (2^-40 of a score), rounded to 32 when small (2^-23 of itself), in exp2 (2^-21) and in sums of rows (2^-24 an addend); and in what scores are enlarged by, at most 2.6 parts in
    2^24."""
    is_latent = fmt.startswith("KV_LATENT")
    n, block, scale = 300, 16, 0.08838834764
    b = latent.make(G, 512, dtype, 8, block, [n], [new]) if is_latent else make(G, getattr(G, fmt), dtype, 8, 2, 128, block, [n], [new])
    heads, kv_heads, D, lay, gen = 8, b["lay"].heads, b["q"].shape[2], b["lay"], gen_of(1)
    slots = torch.tensor([int(b["tables"][0, p // block]) * block + p % block for p in range(n)], dtype=torch.int64, device="cuda")
    k = torch.zeros(n, kv_heads, D, dtype=dtype, device="cuda")
    k[:, :, 0] = 84.0
    k[:, :, 16] = 7 * torch.randint(-8, 9, (n, kv_heads), generator=gen, device="cuda").to(dtype) / 8
    if is_latent:
        G.latent_write(lay, b["cache"], b["layer"], k[:, 0, :512], k[:, 0, 512:], slots)
        assert torch.equal(torch.cat(G.latent_read(lay, b["cache"], b["layer"], slots), 1), k[:, 0])
    else:
        G.kv_write(lay, b["cache"], 0, k, k, slots)
        assert torch.equal(G.kv_read(lay, b["cache"], 0, slots, dtype)[0], k)
    q = b["q"].zero_()
    q[:, :, 0] = 128.0
    q[:, :, 16] = torch.randint(-4, 5, q.shape[:2], generator=gen, device="cuda").to(dtype)
    group = heads // kv_heads
    s = torch.einsum("ihgd,nhd->ihgn", q[:new].double().unflatten(1, (kv_heads, group)), k.double()) * float(torch.tensor(scale, dtype=torch.float32))
    s = s.masked_fill(torch.arange(n, device="cuda") > torch.arange(n - new, n, device="cuda")[:, None, None, None], -math.inf)
    lse = torch.zeros(q.shape[:2], device="cuda")
    lse[:new] = torch.logsumexp(s, 3).flatten(1).float()
    e = s - lse[:new].double().unflatten(1, (kv_heads, group))[..., None]
    p = torch.exp(e)
    size = torch.where(p > 0, e.abs() * 1.4427, 0.0)
    tol = (p * (2.0 ** -23 * size + 2.0 ** -21 + (2.0 ** -40 + 2.6 * 2.0 ** -24) * 1000)).sum((0, 2)) + new * group * 2.0 ** -24 * p.sum((0, 2))
    w = torch.empty(1, kv_heads, n, device="cuda")
    G.attend_weights(lay, b["cache"], b.get("layer", 0), q, lse, dev(b["offsets"]), dev([n]), b["tables"], new, w, scale=scale, accumulate=False)
    err = (w[0].double() - p.sum((0, 2))).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("fmt,dtype", FORMATS + [("KV_LATENT_BF16", torch.bfloat16), ("KV_LATENT_FP16", torch.float16)])
@pytest.mark.parametrize("heads,n", [(8, 400), (32, 3000)])
def test_weights_of_a_row_add_up_to_one(G, fmt, dtype, heads, n):
    """Products of small integers, whose sums lose nothing, and scores of at most 30.  A logarithm is off by the roundings of its reference and its two last steps, half a step of a number
    below 64 each (2^-19), its sum by 2^-21 of an exponential and 2^-24 of 2 addends a key block of 16 and of one a block; a weight by half a step of an exponent below 64, by 2^-21 and by
    the 2.6 parts in 2^24 of its score."""
    is_latent = fmt.startswith("KV_LATENT")
    b = latent.make(G, 512, dtype, heads, 16, [n], [1]) if is_latent else make(G, getattr(G, fmt), dtype, heads, 2, 128, 16, [n], [1])
    lay, gen, kv_heads, D = b["lay"], gen_of(5), b["lay"].heads, b["q"].shape[2]
    slots = torch.tensor([int(b["tables"][0, p // 16]) * 16 + p % 16 for p in range(n)], dtype=torch.int64, device="cuda")
    k = (7 * torch.randint(-1, 2, (n, kv_heads, D), generator=gen, device="cuda")).to(dtype) / 8
    if is_latent:
        G.latent_write(lay, b["cache"], b["layer"], k[:, 0, :512], k[:, 0, 512:], slots)
    else:
        G.kv_write(lay, b["cache"], 0, k, k, slots)
        assert torch.equal(G.kv_read(lay, b["cache"], 0, slots, dtype)[0], k)
    q = b["q"]
    q.copy_(torch.randint(-2, 3, q.shape, generator=gen, device="cuda"))
    group = heads // kv_heads
    scale = 25.0 / float((q[:1].double().unflatten(1, (kv_heads, group)) @ k.double().permute(1, 2, 0)).abs().max())
    lse, args = torch.zeros(q.shape[:2], device="cuda"), (dev(b["offsets"]), dev([n]), b["tables"], 1)
    if is_latent:
        G.latent_attend(lay, b["cache"], b["layer"], q[:, :, :512].contiguous(), q[:, :, 512:].contiguous(), *args, scale, lse=lse)
    else:
        G.attend(lay, b["cache"], 0, q, *args, scale=scale, lse=lse)
    w = torch.empty(1, kv_heads, n, device="cuda")
    G.attend_weights(lay, b["cache"], b.get("layer", 0), q, lse, *args, w, scale=scale, accumulate=False)
    tol = 3 * 2.0 ** -19 + 2.0 ** -21 + 2.0 ** -24 * (2 + n / 16) + 2.0 ** -19 + 2.0 ** -21 + 2.6 * 2.0 ** -24 * 30
    assert float((w[0].double().sum(1) / group - 1).abs().max()) < tol


# ---- batches that give a CTA several tiles -----------------------------------------------------------------------------------------------
def check_request(b, r, got, lse, k_values, scale, packed):
    """One request's weights against the definition, all its rows at once; tolerances as in `expected`."""
    n, a, e = b["lens"][r], b["offsets"][r], b["offsets"][r + 1]
    if n == 0:
        assert bool((got[r] == 0).all())
        return
    q, heads, D = b["q"][a:e].double(), b["q"].shape[1], b["q"].shape[2]
    H = b["lay"].heads
    group = heads // H
    k, ok = ref.gather(k_values, b["tables"][r], n, b["lay"].block_tokens)
    assert bool(ok.all())
    see = torch.arange(n, device="cuda") <= torch.arange(n - (e - a), n, device="cuda")[:, None, None]
    for h in range(H):
        mine, given = q[:, h * group:(h + 1) * group], lse[a:e, h * group:(h + 1) * group].double()[..., None]
        s = (mine @ k[:, h].t()) * scale
        err = (D + 8) * 2.0 ** -23 * (mine.abs() @ k[:, h].abs().t()).masked_fill(~see, 0.0).amax(2, keepdim=True) * scale + 2.0 ** -20
        if packed:
            err = err + 2.0 ** -25 * mine.abs().amax(2, keepdim=True) * k[:, h].abs().sum(1).max() * scale
        p = torch.exp(s - given).masked_fill(~see, 0.0)
        want = p.sum((0, 1))
        tol = (p * (2 * err + 2.0 ** -22 * (s.abs() + given.abs()) + 2.0 ** -21)).sum((0, 1)) + (e - a) * group * 2.0 ** -24 * want + 1e-30
        off = (got[r, h, :n].double() - want).abs()
        assert bool((off <= tol).all()), (r, h, float((off / tol).max()))
    assert bool((got[r, :, n:] == 0).all()), r


def check_batch(G, b, lse, layer, max_new, scale, k_values, packed):
    R, H, width = len(b["lens"]), b["lay"].heads, max(b["lens"])
    args = (b["lay"], b["cache"], layer, b["q"], lse, dev(b["offsets"]), dev(b["lens"]), b["tables"], max_new)
    w, status = torch.full((R, H, width), 3.0, device="cuda"), dev([0])
    G.attend_weights(*args, w, scale=scale, accumulate=False, status=status)
    for r in (0, 1, 2, 3, R // 2, R - 1):
        check_request(b, r, w, lse, k_values, scale, packed)
    start = torch.rand(R, H, width + 9, device="cuda")
    more = start.clone()
    G.attend_weights(*args, more, scale=scale, status=status)
    there = torch.arange(width, device="cuda") < dev(b["lens"])[:, None, None]
    assert torch.equal(more[:, :, :width], torch.where(there, start[:, :, :width] + w, start[:, :, :width])) and torch.equal(more[:, :, width:], start[:, :, width:])
    assert int(status.item()) == 0


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("dim,new", [(128, 1), (128, 20), (128, 40), (64, 1), (64, 50)])
def test_several_tiles(G, fmt, dtype, dim, new):
    """40 requests x 8 heads of up to 5000 tokens: runs of tiles a CTA, whose rows (4, 80, 160, 200 of a kv head) fill a chunk, several, or more than stay in shared memory."""
    rng = random.Random(new)
    lens = [5000, 0, 1000 + new, new] + [rng.randint(2000, 5000) for _ in range(36)]
    b = make(G, getattr(G, fmt), dtype, 32, 8, dim, 16, lens, [min(new, n) for n in lens], seed=new)
    lse = torch.zeros(b["q"].shape[:2], device="cuda")
    scale = dim ** -0.5
    G.attend(b["lay"], b["cache"], 0, b["q"], dev(b["offsets"]), dev(lens), b["tables"], new, scale=scale, lse=lse)
    check_batch(G, b, lse, 0, new, scale, b["values"][0], fmt == "KV_PACKED" and dtype == torch.bfloat16)


@pytest.mark.parametrize("dtype", latent.BOTH)
@pytest.mark.parametrize("L,heads,new", [(512, 16, 1), (512, 64, 1), (512, 50, 3), (256, 128, 1)])
def test_several_tiles_of_a_latent_cache(G, L, dtype, heads, new):
    rng = random.Random(heads)
    lens = [4000, 0, 1000 + new, new] + [rng.randint(1000, 4000) for _ in range(36)]
    b = latent.make(G, L, dtype, heads, 16, lens, [min(new, n) for n in lens], seed=heads)
    latent.call(G, b)
    check_batch(G, b, b["lse"], b["layer"], new, b["scale"], b["values"].unsqueeze(2), False)


# ---- the choice where there are more rows than SMs -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["spread", "ties", "special"])
def test_choice_of_more_rows_than_sms(G, kind):
    gen = gen_of(len(kind))
    lengths = [4095, 4096, 4097, 8191, 8192, 8193, 9000, 0, 1, 700, 701, 4160, 9001, -1] + [50 + 211 * i for i in range(26)]
    w = torch.exp(2 * torch.randn(len(lengths), 4, 9000, generator=gen, device="cuda"))
    if kind == "ties":
        w = (w * 2).floor()
        w[:, 1] = 0.5
    elif kind == "special":
        w[w < 0.2], w[w > 20] = math.nan, math.inf
        w[:, 2, ::3] = -math.inf
        w[:, 3] = math.nan
    check_choice(G, w, lengths, 700, 4, 64)
    check_choice(G, w, lengths, 4096, 0, 1)
