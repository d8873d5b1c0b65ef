"""The operators around the paged cache on the GPU against their definitions in 64 bits."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

from tests import operators_reference as ref


@pytest.fixture(scope="module")
def G():
    from paper_2607_22648_b200 import binding
    return binding


def dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


# ---- block tables and slots -----------------------------------------------------------------------------------------------------------
def check_plan(G, lengths, held, width, block, count, capacity, seed=0, in_place=True):
    rng = random.Random(seed)
    R = len(lengths)
    ids = list(range(sum(held) + count))
    rng.shuffle(ids)
    tables, at = [], 0
    for h in held:
        tables.append(ids[at:at + h] + [-1] * (width - h))
        at += h
    stack = ids[at:at + count] + [-7] * (capacity - count)
    want = ref.assign_blocks(lengths, held, tables, stack, count, block)
    t, hd, st, ct, status = dev(tables).view(R, width), dev(held), dev(stack), dev([count]), dev([0])
    if in_place:
        h2, c2 = G.assign_blocks(dev(lengths), hd, t, st, ct, block, status=status)
        assert h2 is hd and c2 is ct
    else:
        h2, c2 = G.assign_blocks(dev(lengths), hd, t, st, ct, block, held_out=torch.empty_like(hd), free_count_out=torch.empty_like(ct), status=status)
        assert hd.tolist() == held and ct.tolist() == [count]
    assert t.tolist() == want[0] and h2.tolist() == want[1] and st.tolist() == want[2] and c2.tolist() == [want[3]]
    too_long = any(-(-max(n, 0) // block) > width or n < 0 for n in lengths)
    lost = sum(max(0, h - (-(-max(n, 0) // block))) for n, h in zip(lengths, held)) > capacity - count
    assert int(status.item()) == (G.S_NOSPACE if want[4] else 0) | (G.S_BOUNDS if too_long or lost else 0)
    # the slots of the tokens behind a random part of every request
    done = [rng.randrange(0, max(n, 0) + 2) for n in lengths]
    for unit, min_new, d in ((1, 0, done), (block, 1, [x // block for x in done]), (1, 0, None)):
        off, slots, pos = ref.map_slots(lengths, d, want[0], block, unit, min_new)
        total = off[-1]
        room = total + 5
        go, gs, gp = G.map_slots(dev(lengths), dev(d) if d else None, t, block, room, done_unit=unit, min_new=min_new)
        assert go.tolist() == off and gs.tolist() == slots + [-1] * 5 and gp.tolist() == pos + [-1] * 5


@pytest.mark.parametrize("R", [1, 2, 31, 64, 1000, 1025])
@pytest.mark.parametrize("block", [1, 16, 24])
def test_plan_grow_shrink_end(G, R, block):
    rng = random.Random(R * 100 + block)
    width = 9
    held = [rng.randint(0, width) for _ in range(R)]
    lengths = [rng.choice([0, 0, 1, block, block + 1, rng.randint(0, width * block), width * block]) for _ in range(R)]
    check_plan(G, lengths, held, width, block, R * width, 3 * R * width, seed=R)
    check_plan(G, lengths, held, width, block, R, 3 * R * width, seed=R, in_place=False)      # some are denied
    check_plan(G, lengths, held, width, block, 0, 3 * R * width, seed=R)                       # growth lives on what others return


def test_plan_more_requests_than_one_scan_step(G):
    """More than 16,384 requests: sums are carried from step to step, pops follow all pushes."""
    rng = random.Random(5)
    R, block, width = 40000, 16, 3
    held = [rng.randint(0, width) for _ in range(R)]
    lengths = [rng.randint(0, width * block) for _ in range(R)]
    check_plan(G, lengths, held, width, block, R // 4, 3 * R)
    check_plan(G, lengths, held, width, block, R, 3 * R, in_place=False)


def test_plan_bad_values(G):
    check_plan(G, [-3, 200, 16], [0, 1, 0], 4, 16, 5, 9)                        # a negative length, one beyond the row
    check_plan(G, [0, 0, 16], [2, 3, 0], 4, 16, 1, 3)                           # a stack too small for what comes back
    # counts outside their ranges are clamped
    t, st, status = dev([[0, 1], [2, 3]]), dev([9, 8, 7, 6]), dev([0])
    h, c = G.assign_blocks(dev([32, 32]), dev([5, -2]), t, st, dev([99]), 16, status=status)
    assert h.tolist() == [2, 2] and c.tolist() == [2] and t.tolist() == [[0, 1], [6, 7]] and int(status.item()) == G.S_BOUNDS


def test_plan_new_batch_and_empty(G):
    t, st = torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), dev([4, 5, 6])
    h, c = G.assign_blocks(dev([17, 1]), None, t, st, dev([3]), 16)
    assert h.tolist() == [2, 1] and c.tolist() == [0] and t.tolist() == [[6, 5, -1, -1], [4, -1, -1, -1]]
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    h, c = G.assign_blocks(e, None, torch.empty((0, 4), dtype=torch.int32, device="cuda"), st, dev([2]), 16, free_count_out=dev([0]))
    assert c.tolist() == [2]
    off, slots, _ = G.map_slots(e, None, torch.empty((0, 4), dtype=torch.int32, device="cuda"), 16, 3)
    assert off.tolist() == [0] and slots.tolist() == [-1, -1, -1]


def test_map_slots_limits(G):
    status = dev([0])
    off, slots, pos = G.map_slots(dev([40, 10]), None, dev([[3, -1], [5, 6]]), 16, 45, status=status)
    want = ref.map_slots([40, 10], None, [[3, -1], [5, 6]], 16)
    assert off.tolist() == want[0] and slots.tolist() == want[1][:45] and pos.tolist() == want[2][:45]
    assert int(status.item()) == G.S_BOUNDS                                       # tokens beyond the row and beyond max_tokens
    big = (1 << 31) // 16 - 1                                                     # slots pass 32 bits
    off, slots, _ = G.map_slots(dev([33]), None, dev([[big, big, big]]), 48, 33)
    assert slots.tolist() == [big * 48 + p % 48 for p in range(33)]


# ---- the 4-bit cache ------------------------------------------------------------------------------------------------------------------
def layer(G, lay, blocks, fill=0xFF):
    """A one-layer cache whose unwritten bytes read as NaN."""
    c = G.PagedKV(1, blocks, lay.chunk_bytes)
    c.tensors[0].fill_(fill)
    return c


def rows(gen, shape, dtype, spread=1.0):
    x = torch.randn(shape, generator=gen, device="cuda") * spread
    x = x * (1 + 7 * (torch.rand(shape[-1:], generator=gen, device="cuda") < 0.06))
    return x.to(dtype)


def gen_of(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,block,tokens", [(1, 16, 1), (8, 16, 64), (3, 48, 101), (2, 128, 300)])
def test_packed_round_trip(G, dim, dtype, heads, block, tokens):
    gen = gen_of(dim + heads + tokens)
    lay = G.KVLayout(heads, dim, block, G.KV_PACKED, 2.0 ** -4, 2.0 ** -6)
    blocks = -(-tokens // block) + 2
    c = layer(G, lay, blocks)
    k, v = rows(gen, (tokens, heads, dim), dtype), rows(gen, (tokens, heads, dim), dtype, 0.1)
    # values on the quantiser's borders: halves of a code, ties of the scale, groups of zeros
    k[0, 0, :16] = torch.tensor([7 * 16 / 16, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, -3.5, 3.5, 6.5, -6.5, 0, 1, 2, 3, -7], device="cuda").to(dtype)
    v[0, 0, 16:32] = 0
    v[tokens - 1, heads - 1, :16] = 7 * 448 * 2.0 ** -6 * 2                        # beyond the largest scale
    slots = torch.randperm(blocks * block, generator=gen, device="cuda")[:tokens]
    status = dev([0])
    before = c.tensors[0].clone()
    G.kv_write(lay, c, 0, k, v, slots, status=status)
    k2, v2 = G.kv_read(lay, c, 0, slots, dtype, status=status)
    assert int(status.item()) == 0
    assert torch.equal(k2.double(), ref.quantised(k, lay.k_scale)) and torch.equal(v2.double(), ref.quantised(v, lay.v_scale))
    # nothing but those slots' bytes changed: the other slots still read as NaN
    other = torch.tensor(sorted(set(range(blocks * block)) - set(slots.tolist())), device="cuda")
    k3, v3 = G.kv_read(lay, c, 0, other, dtype)
    assert bool(k3.isnan().all()) and bool(v3.isnan().all())
    changed = (c.tensors[0] != before).sum().item()
    assert changed <= 2 * tokens * heads * dim * 9 // 16


def test_packed_special_values(G):
    lay = G.KVLayout(1, 64, 16, G.KV_PACKED, 1.0, 2.0 ** 20)
    c = layer(G, lay, 1)
    k = torch.randn(6, 1, 64, device="cuda").bfloat16()
    k[0, 0, 3] = float("inf")
    k[1, 0, 20] = float("-inf")
    k[2, 0, 40] = float("nan")
    k[3] = 1e-30                                      # scale rounds to zero
    k[4] = 3e38                                       # far beyond the range
    k[5, 0, :16] = 2.0 ** -9 * 7 * 0.5                # the scale's tie between zero and its smallest value: even, so zero
    v = (k.float() * 2.0 ** 20).bfloat16()
    slots = torch.arange(6, device="cuda")
    G.kv_write(lay, c, 0, k, v, slots)
    k2, v2 = G.kv_read(lay, c, 0, slots, torch.bfloat16)
    for got, x, t in ((k2, k, lay.k_scale), (v2, v, lay.v_scale)):
        want = ref.quantised(x, t)
        assert torch.equal(got.double().isnan(), want.isnan()) and bool(want[2, 0, 32:48].isnan().all()) and int(want.isnan().sum()) == 16
        assert torch.equal(got.double().nan_to_num(0), want.nan_to_num(0))
    assert float(k2[0, 0, 3]) == 7 * 448 and float(k2[1, 0, 20]) == -8 * 448 and not bool(k2[3].any())


@pytest.mark.parametrize("fmt", ["KV_BF16", "KV_FP16", "KV_PACKED"])
def test_write_strided_rows_and_skipped_slots(G, fmt):
    """K and V as slices of one projection's output; slots of -1 and outside the cache."""
    dtype = torch.float16 if fmt == "KV_FP16" else torch.bfloat16
    heads, dim, block, T = 2, 64, 16, 40
    lay = G.KVLayout(heads, dim, block, getattr(G, fmt))
    c = layer(G, lay, 4, fill=0x11)
    qkv = torch.randn(T, 6, dim, device="cuda").to(dtype)
    k, v = qkv[:, 2:4], qkv[:, 4:6]
    slots = torch.randperm(64, generator=gen_of(1), device="cuda")[:T]
    slots[3], slots[7], slots[9] = -1, 64, -5
    status = dev([0])
    G.kv_write(lay, c, 0, k, v, slots, status=status)
    assert int(status.item()) == G.S_BOUNDS
    out = torch.full((2, T, heads, dim), 9.0, device="cuda", dtype=dtype)
    status.zero_()
    G.kv_read(lay, c, 0, slots, dtype, k=out[0], v=out[1], status=status)
    assert int(status.item()) == G.S_BOUNDS
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[[3, 7, 9]] = False
    for got, x in ((out[0], k), (out[1], v)):
        want = ref.quantised(x, 1.0) if fmt == "KV_PACKED" else x.double()
        assert torch.equal(got[keep].double(), want[keep]) and bool((got[~keep] == 9.0).all())
    used = torch.zeros(64, dtype=torch.bool, device="cuda")
    used[slots[keep]] = True
    if fmt != "KV_PACKED":
        raw = c.tensors[0].view(2, 64, heads * dim * 2)
        assert bool((raw[:, ~used] == 0x11).all())


# ---- attention ------------------------------------------------------------------------------------------------------------------------
def make(G, fmt, dtype, heads, kv_heads, dim, block, lens, new, seed=0, tail_rows=3, strided=False, width=None, spread=1.0):
    """A batch over a cache whose slots behind the sequences hold NaN; returns the call's arguments and the values the cache stands for."""
    gen = gen_of(1000 + seed)
    t = (2.0 ** -4, 2.0 ** -6) if fmt == G.KV_PACKED else (1.0, 1.0)
    lay = G.KVLayout(kv_heads, dim, block, fmt, *t)
    blocks = [-(-max(n, 0) // block) for n in lens]
    nb = sum(blocks) + 2
    c = layer(G, lay, nb)
    perm = torch.randperm(nb, generator=gen, device="cuda").int().tolist()
    width = width or max(blocks + [1]) + 1
    tables, at, slots = [], 0, []
    for n, b in zip(lens, blocks):
        row = perm[at:at + b]
        at += b
        slots += [row[p // block] * block + p % block for p in range(max(n, 0))]
        tables.append(row + [-1] * (width - b))
    n = len(slots)
    k, v = rows(gen, (n, kv_heads, dim), dtype, spread), rows(gen, (n, kv_heads, dim), dtype, 0.25)
    slots = torch.tensor(slots, dtype=torch.int64, device="cuda")
    G.kv_write(lay, c, 0, k, v, slots)
    values = []
    for x, ts in ((k, t[0]), (v, t[1])):
        full = torch.full((nb * block, kv_heads, dim), float("nan"), dtype=torch.float64, device="cuda")
        full[slots] = ref.quantised(x, ts) if fmt == G.KV_PACKED else x.double()
        values.append(full.view(nb, block, kv_heads, dim))
    offsets = [0]
    for m in new:
        offsets.append(offsets[-1] + m)
    T = offsets[-1] + tail_rows
    if strided:
        q = rows(gen, (T, heads + 2 * kv_heads, dim), dtype)[:, :heads]
        out = torch.full((T, 2, heads, dim), 5.0, dtype=dtype, device="cuda")[:, 1]
    else:
        q = rows(gen, (T, heads, dim), dtype)
        out = torch.full((T, heads, dim), 5.0, dtype=dtype, device="cuda")
    return dict(lay=lay, cache=c, q=q, out=out, offsets=offsets, lens=list(lens), new=list(new), tables=dev(tables).view(len(lens), width), values=values)


def call(G, b, max_new=None, scale=None, workspace=None, status=None, out=None):
    return G.attend(b["lay"], b["cache"], 0, b["q"], dev(b["offsets"]), dev(b["lens"]), b["tables"], max(b["new"] + [1]) if max_new is None else max_new, scale=scale,
                    out=b["out"] if out is None else out, workspace=workspace, status=status)


def check(G, b, scale=None, got=None):
    dim = b["q"].shape[2]
    s = dim ** -0.5 if scale is None else scale
    want, spread, scores, owned = ref.attend(b["q"], b["offsets"], b["lens"], b["tables"], b["values"][0], b["values"][1], b["lay"].block_tokens, s)
    keys = max(b["lens"] + [0])
    v_max, k_sum = float(b["values"][1].nan_to_num(0).abs().max()), float(b["values"][0].nan_to_num(0).abs().sum(-1).max()) * abs(s)
    tol = ref.attend_tolerance(b["q"], want, spread, scores, keys, v_max, b["lay"].format == G.KV_PACKED, k_sum)
    got = b["out"] if got is None else got
    err = (got.double() - want).abs()
    bad = owned[:, None, None] & ~(err <= tol)
    assert not bool(bad.any()), "worst %.3g of the tolerance at %s" % (float((err / tol)[owned].nan_to_num(1e9).max()), bad.nonzero()[0].tolist())
    assert bool((got[~owned] == 5.0).all()), "rows of no request changed"


FORMATS = [("KV_PACKED", torch.bfloat16), ("KV_PACKED", torch.float16), ("KV_BF16", torch.bfloat16), ("KV_FP16", torch.float16)]


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2), (24, 3), (16, 1), (10, 2)])
def test_decode_ragged(G, fmt, dtype, dim, heads, kv_heads):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 200, 333, 1030]
    b = make(G, getattr(G, fmt), dtype, heads, kv_heads, dim, 16, lens, [1] * len(lens), seed=heads)
    call(G, b)
    check(G, b)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("block", [16, 32, 48, 1024])
def test_decode_block_sizes(G, fmt, dtype, block):
    b = make(G, getattr(G, fmt), dtype, 8, 2, 128, block, [5, 100, 1500, 0, 48], [1, 1, 1, 1, 1], seed=block)
    call(G, b)
    check(G, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("block", [1, 3, 8, 24, 100])
@pytest.mark.parametrize("new", [1, 3, 40])
def test_16_bit_cache_odd_block_sizes(G, dtype, block, new):
    lens = [new, new + 1, 77, 130, 290]
    b = make(G, G.KV_FP16 if dtype == torch.float16 else G.KV_BF16, dtype, 6, 2, 64 if block == 24 else 128, block, lens, [new] * 5, seed=block)
    call(G, b)
    check(G, b)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
def test_mixed_new_tokens_and_empty_rows(G, fmt, dtype, dim):
    """Whole prompts, suffixes, single tokens, requests without rows, rows before the first key, a request without keys."""
    lens = [50, 131, 300, 64, 0, 20, 7, 1, 700]
    new = [50, 70, 1, 0, 3, 33, 7, 1, 129]
    b = make(G, getattr(G, fmt), dtype, 8, 2, dim, 32, lens, new, seed=3)
    call(G, b)
    check(G, b)
    assert not bool(b["out"][b["offsets"][4]:b["offsets"][5]].any())              # no keys: zeros
    assert not bool(b["out"][b["offsets"][5]:b["offsets"][5] + 13].any())         # 33 rows over 20 keys: 13 rows see nothing


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("new", [2, 3, 4, 9, 17, 100, 260])
def test_new_token_counts(G, fmt, dtype, new):
    b = make(G, getattr(G, fmt), dtype, 12, 3, 128, 16, [new, 2 * new + 5, 411 + new], [new, new - 1, new], seed=new, strided=True)
    call(G, b)
    check(G, b)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_one_long_request_is_split_and_joined(G, fmt, dtype):
    b = make(G, getattr(G, fmt), dtype, 8, 1, 128, 16, [20011], [1], seed=9, tail_rows=0)
    call(G, b)
    check(G, b)
    first = b["out"].clone()
    for _ in range(3):                                                            # equal bits, whoever joins
        b["out"].fill_(5.0)
        call(G, b)
        assert torch.equal(first, b["out"])


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_many_requests(G, fmt, dtype):
    rng = random.Random(8)
    lens = [rng.randint(1, 90) for _ in range(700)]
    b = make(G, getattr(G, fmt), dtype, 4, 1, 64, 16, lens, [1] * 700, seed=1)
    call(G, b)
    check(G, b)


def test_workspace_is_left_ready(G):
    """One workspace through calls of different shapes: nothing of a call reaches the next."""
    ws = None
    for i, (lens, new, heads, kv) in enumerate([([5000, 3], [1, 1], 8, 2), ([17] * 40, [1] * 40, 16, 2), ([900, 2000], [4, 2], 8, 8), ([9000], [1], 64, 8), ([5000, 3], [1, 1], 8, 2)]):
        b = make(G, G.KV_PACKED, torch.bfloat16, heads, kv, 128, 16, lens, new, seed=i)
        if ws is None:
            ws = G.attend_workspace(b["lay"])
        call(G, b, workspace=ws)
        check(G, b)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("new", [1, 4, 40])
def test_table_entries_outside_the_cache_are_not_seen(G, fmt, dtype, new):
    b = make(G, getattr(G, fmt), dtype, 8, 2, 128, 16, [200, 100, 32], [new, new, new], seed=4)
    nb = b["values"][0].shape[0]
    b["tables"][0, 3] = -1
    b["tables"][0, 7] = nb
    b["tables"][1, 0] = 2 ** 31 - 1
    b["tables"][2, 0:2] = -5                                                     # nothing left to see: zeros
    status = dev([0])
    call(G, b, status=status)
    assert int(status.item()) == G.S_BOUNDS
    check(G, b)
    if new == 1:
        assert not bool(b["out"][2].any())


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("new", [1, 3, 50])
def test_lengths_beyond_the_table(G, fmt, dtype, new):
    """A length the table's row cannot hold: the tokens it lacks are not seen, positions stay."""
    b = make(G, getattr(G, fmt), dtype, 4, 2, 64, 16, [64, 90], [new, new], seed=6, width=6)
    b["lens"] = [130, 90]
    call(G, b)
    check(G, b)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("heads,kv_heads,new", [(4, 2, 3), (8, 2, 4), (4, 1, 40), (8, 1, 150)])
def test_infinities_and_nan_in_later_tokens_do_not_reach_earlier_rows(G, fmt, dtype, heads, kv_heads, new):
    """The last tokens of a prompt hold NaN (and infinities): rows before them are as without, rows that see them are NaN."""
    lens = [new, 100 + new]
    b = make(G, getattr(G, fmt), dtype, heads, kv_heads, 128, 16, lens, [new, new], seed=7)
    bad_from = [n - 1 for n in lens]
    slots = torch.tensor([int(b["tables"][r, p // 16]) * 16 + p % 16 for r, p in enumerate(bad_from)], device="cuda")
    k = torch.full((2, kv_heads, 128), float("nan"), dtype=dtype, device="cuda")
    v = torch.full((2, kv_heads, 128), float("nan"), dtype=dtype, device="cuda")
    if fmt != "KV_PACKED":
        v[0] = float("inf")
        k[1] = float("-inf")
    call(G, b)
    clean = b["out"].clone()
    G.kv_write(b["lay"], b["cache"], 0, k, v, slots)
    b["out"].fill_(5.0)
    call(G, b)
    for r in range(2):
        a, e = b["offsets"][r], b["offsets"][r + 1]
        assert torch.equal(b["out"][a:e - 1], clean[a:e - 1]), "request %d" % r
        assert not bool(torch.isfinite(b["out"][e - 1]).any())
    assert bool((b["out"][b["offsets"][2]:] == 5.0).all())


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("heads,kv_heads,dim,block", [(16, 4, 128, 16), (10, 2, 64, 48), (24, 8, 128, 128)])
def test_many_prompts(G, fmt, dtype, heads, kv_heads, dim, block):
    """More row tiles than the GPU has room for at once: steps are not cut into chunks (in the tests above they are)."""
    rng = random.Random(heads)
    lens = [rng.randint(1, 220) for _ in range(150 // kv_heads)] + [700]
    new = [rng.choice([n, n, rng.randint(0, n)]) for n in lens[:-1]] + [400]
    b = make(G, getattr(G, fmt), dtype, heads, kv_heads, dim, block, lens, new, seed=heads)
    call(G, b)
    check(G, b)
    # the last token of every whole prompt turns into NaN: nothing before it changes
    clean = b["out"].clone()
    rows_of = [(r, b["offsets"][r + 1] - 1) for r in range(len(lens)) if new[r] > 1]
    slots = torch.tensor([int(b["tables"][r, (lens[r] - 1) // block]) * block + (lens[r] - 1) % block for r, _ in rows_of], device="cuda")
    bad = torch.full((len(rows_of), kv_heads, dim), float("nan"), dtype=dtype, device="cuda")
    G.kv_write(b["lay"], b["cache"], 0, bad, bad, slots)
    b["out"].fill_(5.0)
    call(G, b)
    keep = torch.ones(b["out"].shape[0], dtype=torch.bool, device="cuda")
    keep[[i for _, i in rows_of]] = False
    assert torch.equal(b["out"][keep], clean[keep]) and not bool(torch.isfinite(b["out"][~keep]).any())


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("new", [40, 64, 300])
def test_one_prompt_behind_a_long_prefix(G, fmt, dtype, new):
    """One request's steps spread over the GPU and joined; equal bits every time; scores that grow along the prefix."""
    b = make(G, getattr(G, fmt), dtype, 8, 2, 128, 16, [4096 + new], [new], seed=new)
    ws = G.attend_workspace(b["lay"])
    call(G, b, workspace=ws)
    check(G, b)
    first = b["out"].clone()
    for _ in range(2):
        b["out"].fill_(5.0)
        call(G, b, workspace=ws)
        assert torch.equal(first, b["out"])
    # the split kernel finds its counters as it left them
    d = make(G, getattr(G, fmt), dtype, 8, 2, 128, 16, [5000, 70], [1, 1], seed=2)
    call(G, d, workspace=ws)
    check(G, d)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_large_and_equal_scores(G, fmt, dtype):
    """Scores far beyond the range of exp, equal scores, a scale of zero and a negative one."""
    for scale in (None, 0.0, -0.1, 20.0):
        b = make(G, getattr(G, fmt), dtype, 4, 2, 64, 16, [300, 40], [1, 20], seed=11)
        call(G, b, scale=scale)
        check(G, b, scale=scale)


def test_q_may_be_the_output(G):
    b = make(G, G.KV_PACKED, torch.bfloat16, 8, 2, 128, 16, [6000, 50, 300], [1, 1, 1], seed=12, tail_rows=0)
    call(G, b)
    want = b["out"].clone()
    got = call(G, b, out=b["q"])
    assert torch.equal(got, want)


def test_large_max_new_gives_the_same_answers(G):
    """max_new only chooses the kernel: a bound that is too large is as right."""
    b = make(G, G.KV_BF16, torch.bfloat16, 8, 2, 128, 16, [600, 50, 300], [1, 2, 1], seed=13)
    call(G, b, max_new=1000)
    check(G, b)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("new", [1, 3, 45])
def test_blocks_that_hold_k_and_v_side_by_side(G, fmt, dtype, new):
    """A cache laid out [blocks][K, V][chunk]: strides of the other order."""
    b = make(G, getattr(G, fmt), dtype, 8, 2, 128, 16, [100, 45, 260], [new, new, new], seed=21)
    t = b["cache"].tensors[0]
    other = t.transpose(0, 1).contiguous().transpose(0, 1)
    assert other.stride() != t.stride()
    b["cache"] = G.PagedKV(1, t.shape[1], t.shape[2], tensors=[other])
    call(G, b)
    check(G, b)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("new,block", [(1, 16), (5, 16), (60, 16), (60, 256)])
def test_a_row_of_nan_stays_alone(G, fmt, dtype, new, block):
    b = make(G, getattr(G, fmt), dtype, 6, 2, 64, block, [200, new], [new, new], seed=22)
    call(G, b)
    clean = b["out"].clone()
    b["q"][new // 2, 3] = float("nan")
    b["out"].fill_(5.0)
    call(G, b)
    assert bool(b["out"][new // 2, 3].isnan().all())
    b["out"][new // 2, 3] = clean[new // 2, 3]
    assert torch.equal(b["out"], clean)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("new", [2, 50])
def test_one_query_row_for_all_tokens(G, fmt, dtype, new):
    """q expanded over the tokens: a token stride of zero."""
    b = make(G, getattr(G, fmt), dtype, 8, 2, 128, 16, [130, new], [new, new], seed=23, tail_rows=0)
    one = b["q"][:1].clone()
    b["q"] = one.expand(2 * new, -1, -1)
    call(G, b)
    check(G, b)


@pytest.mark.parametrize("dim", [64, 128])
def test_calls_of_all_shapes_share_a_workspace(G, dim):
    """Grids of 8 and 16 rows, of 4-bit and 16-bit caches and whole prompts leave the workspace as the next call needs it."""
    lens = [333 + 97 * i for i in range(24)]
    batches = []
    for i, (fmt, dtype) in enumerate([("KV_PACKED", torch.bfloat16), ("KV_BF16", torch.bfloat16)]):
        for new in (1, 4, 40):
            batches.append(make(G, getattr(G, fmt), dtype, 8, 2, dim, 16, lens, [new] * 24, seed=30 + i))
    work = G.attend_workspace(batches[0]["lay"])
    right = []
    for b in batches:
        call(G, b)
        check(G, b)
        right.append(b["out"].clone())
    for first in range(len(batches)):
        for second in range(len(batches)):
            for i in (first, second, first):
                batches[i]["out"].fill_(5.0)
                call(G, batches[i], workspace=work)
                assert torch.equal(batches[i]["out"], right[i]), (first, second, i)


@pytest.mark.parametrize("many", [20, 300])
@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_row_tiles_that_see_nothing(G, fmt, dtype, many):
    """Whole row tiles in front of the first key, beside tiles that see some: their rows are zeros, run after run."""
    b = make(G, getattr(G, fmt), dtype, 8, 2, 128, 16, [0] * many + [40, 700], [64] * many + [300, 100], seed=25)
    for _ in range(3):
        b["out"].fill_(5.0)
        call(G, b)
        assert not bool(b["out"][:64 * many + 260].any())
    check(G, b)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_one_row_of_any_stride(G, fmt, dtype):
    """One token, one kv head: the strides of axes of one do not matter."""
    b = make(G, getattr(G, fmt), dtype, 24, 1, 64, 16, [77], [1], seed=24, tail_rows=0)
    b["q"] = b["q"].as_strided((1, 24, 64), (24 * 64 + 5, 64, 1))
    call(G, b)
    check(G, b)
    call(G, b, max_new=40)
    check(G, b)
    rows1 = torch.zeros(64, dtype=dtype, device="cuda").as_strided((1, 1, 64), (67, 65, 1))
    G.kv_write(b["lay"], b["cache"], 0, rows1, rows1, torch.zeros(1, dtype=torch.int64, device="cuda"))
    k, v = G.kv_read(b["lay"], b["cache"], 0, torch.zeros(1, dtype=torch.int64, device="cuda"), dtype)
    assert not bool(k.any()) and not bool(v.any())


def test_two_graphs_share_a_workspace(G):
    """Captured calls of different shapes over one workspace, replayed in turn; the arrival counters are zero after every call."""
    ws, graphs, want, batches = None, [], [], []
    for i, (lens, new, fmt) in enumerate([([6000, 10], [1, 1], G.KV_PACKED), ([3000], [70], G.KV_BF16), ([900, 4000], [2, 1], G.KV_BF16)]):
        b = make(G, fmt, torch.bfloat16, 8, 2, 128, 16, lens, new, seed=30 + i)
        ws = G.attend_workspace(b["lay"]) if ws is None else ws
        call(G, b, workspace=ws)
        check(G, b)
        want.append(b["out"].clone())
        args = (b["lay"], b["cache"], 0, b["q"], dev(b["offsets"]), dev(b["lens"]), b["tables"], max(new))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            G.attend(*args, out=b["out"], workspace=ws)
        graphs.append(g)
        batches.append((b, args))
    for k in (0, 1, 2, 1, 0, 0, 2):
        batches[k][0]["out"].fill_(5.0)
        graphs[k].replay()
        assert torch.equal(batches[k][0]["out"], want[k])
        assert not bool(ws[:2560].any())


def test_offsets_beyond_32_bits(G):
    """A cache larger than 4 GiB, the request in its last blocks."""
    lay = G.KVLayout(8, 128, 16, G.KV_BF16)
    nb = (5 << 30) // (2 * lay.chunk_bytes)
    c = G.PagedKV(1, nb, lay.chunk_bytes)
    gen = gen_of(3)
    n = 100
    k, v = rows(gen, (n, 8, 128), torch.bfloat16), rows(gen, (n, 8, 128), torch.bfloat16, 0.25)
    ids = [nb - 1 - i for i in range(7)]
    slots = torch.tensor([ids[p // 16] * 16 + p % 16 for p in range(n)], device="cuda")
    for j in ids:
        c.tensors[0][:, j] = 0xFF
    G.kv_write(lay, c, 0, k, v, slots)
    k2, v2 = G.kv_read(lay, c, 0, slots, torch.bfloat16)
    assert torch.equal(k, k2) and torch.equal(v, v2)
    for new in (1, 40):
        q = rows(gen, (new, 16, 128), torch.bfloat16)
        out = G.attend(lay, c, 0, q, dev([0, new]), dev([n]), dev([ids]), new)
        want, spread, scores, _ = ref.attend(q, [0, new], [n], dev([list(range(7))]), torch.cat([k, k[:12]]).double().view(7, 16, 8, 128),
                                             torch.cat([v, v[:12]]).double().view(7, 16, 8, 128), 16, 128 ** -0.5)
        tol = ref.attend_tolerance(q, want, spread, scores, n, float(v.abs().max()), False, 0.0)
        assert bool(((out.double() - want).abs() <= tol).all())


def test_streams_and_graph(G):
    """A whole step on another stream and replayed from a captured graph, with new inputs in the same tensors."""
    lay = G.KVLayout(2, 128, 16, G.KV_PACKED, 2.0 ** -4, 2.0 ** -6)
    R, width, heads = 3, 9, 8
    c = layer(G, lay, 32)
    lens, done = dev([40, 3, 100]), dev([39, 2, 99])
    tables = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    held, free_ids, free_count = dev([0, 0, 0]), torch.arange(32, dtype=torch.int32, device="cuda"), dev([32])
    offsets, slots, positions = torch.empty(R + 1, dtype=torch.int32, device="cuda"), torch.empty(8, dtype=torch.int64, device="cuda"), torch.empty(8, dtype=torch.int32, device="cuda")
    gen = gen_of(5)
    k, v, q = (rows(gen, (8, n, 128), torch.bfloat16) for n in (2, 2, heads))
    out, ws = torch.zeros(8, heads, 128, dtype=torch.bfloat16, device="cuda"), G.attend_workspace(lay)

    def step():
        G.assign_blocks(lens, held, tables, free_ids, free_count, 16)
        G.map_slots(lens, done, tables, 16, 8, token_offsets=offsets, slots=slots, positions=positions)
        G.kv_write(lay, c, 0, k, v, slots)
        G.attend(lay, c, 0, q, offsets, lens, tables, 1, out=out, workspace=ws)
    # the cache's history
    G.assign_blocks(lens, held, tables, free_ids, free_count, 16)
    _, s0, _ = G.map_slots(done, None, tables, 16, 141)
    hk, hv = rows(gen, (141, 2, 128), torch.bfloat16), rows(gen, (141, 2, 128), torch.bfloat16)
    G.kv_write(lay, c, 0, hk, hv, s0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    side_out = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    out.zero_()
    graph.replay()
    assert torch.equal(out[:3], side_out[:3])
    # the next token of every request: lengths grow by one, new rows, the same graph
    for i in range(30):
        lens += 1
        done += 1
        for t in (k, v, q):
            t.copy_(rows(gen, tuple(t.shape), torch.bfloat16))
        graph.replay()
    assert held.tolist() == [-(-n // 16) for n in lens.tolist()]
    kk, vv = G.kv_read(lay, c, 0, torch.arange(32 * 16, device="cuda"), torch.bfloat16)
    want, spread, scores, _ = ref.attend(q[:3], [0, 1, 2, 3], lens.tolist(), tables, kk.double().view(32, 16, 2, 128), vv.double().view(32, 16, 2, 128), 16, 128 ** -0.5)
    tol = ref.attend_tolerance(q[:3], want, spread, scores, 140, float(vv.nan_to_num(0).abs().max()), True, float(kk.nan_to_num(0).double().abs().sum(-1).max()) * 128 ** -0.5)
    assert bool(((out[:3].double() - want).abs() <= tol).all())


def test_a_serving_step_over_a_packed_store(G):
    """The operators together with the store, as a serving program uses them: block tables, prefix lookup and gather of 4-bit blocks, slots of
    what was not found, write, attention, insert of the new blocks."""
    import numpy as np
    B, heads, dim, layers, hq = 16, 2, 64, 2, 8
    lay = G.KVLayout(heads, dim, B, G.KV_PACKED, 2.0 ** -4, 2.0 ** -6)
    st = G.PTStore(layers=layers, heads=heads, block_tokens=B, hbm_blocks=64, max_requests=8, max_batch_blocks=8 * 16, **lay.store_args())
    assert st.chunk_bytes == lay.chunk_bytes
    rng = np.random.default_rng(4)
    doc = rng.integers(0, 1000, size=100).astype(np.int32)
    nb, width = 48, 10
    table_of = torch.randn(1000, 2 * layers, heads, dim, device="cuda").bfloat16()        # a "model": K and V depend on the token and its position
    ws = G.attend_workspace(lay)
    found = []
    for turn, prompts in enumerate([[doc], [np.concatenate([doc, doc[:9]]), doc[:48], rng.integers(0, 1000, size=33).astype(np.int32)]]):
        R = len(prompts)
        tokens = torch.from_numpy(np.concatenate(prompts)).cuda()
        cum = np.concatenate([[0], np.cumsum([len(p) for p in prompts])])
        offs = torch.from_numpy(cum.astype(np.int64)).cuda()
        lens = dev([len(p) for p in prompts])
        cache = G.PagedKV(layers, nb, lay.chunk_bytes)
        for t in cache.tensors:
            t.fill_(0xFF)
        tables = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
        G.assign_blocks(lens, None, tables, torch.randperm(nb, device="cuda").int(), dev([nb]), B)
        matched, ids = st.lookup_fetch(tokens, offs, width, cache, tables, G.PIN)
        T = int(cum[-1])
        t_off, slots, pos = G.map_slots(lens, matched, tables, B, T, done_unit=B, min_new=1)
        n_new = int(t_off[-1].item())
        found.append(matched.tolist())
        r_of = torch.searchsorted(t_off[1:].contiguous(), torch.arange(T, device="cuda", dtype=torch.int32), right=True).clamp(max=R - 1)
        tok = tokens[(offs[:-1][r_of] + pos).clamp(min=0).long()].long()
        rope = 1 + 0.01 * pos.clamp(min=0).float()[:, None, None]
        outs, q = [], torch.randn(T, hq, dim, device="cuda").bfloat16()
        for l in range(layers):
            k, v = ((table_of[tok, 2 * l + i] * rope).bfloat16() for i in range(2))
            G.kv_write(lay, cache, l, k, v, slots)
            outs.append(G.attend(lay, cache, l, q, t_off, lens, tables, T, workspace=ws, out=torch.full_like(q, 5.0)))
        # what the cache has to hold, computed from the prompts alone
        for l in range(layers):
            vals = []
            for i, ts in ((0, lay.k_scale), (1, lay.v_scale)):
                full = torch.full((nb * B, heads, dim), float("nan"), dtype=torch.float64, device="cuda")
                for r, p in enumerate(prompts):
                    ps = torch.arange(len(p), device="cuda")
                    x = (table_of[torch.from_numpy(p).cuda().long(), 2 * l + i] * (1 + 0.01 * ps.float()[:, None, None])).bfloat16()
                    full[tables[r].long()[ps // B] * B + ps % B] = ref.quantised(x, ts)
                vals.append(full.view(nb, B, heads, dim))
            check(G, dict(q=q, out=outs[l], offsets=t_off.tolist(), lens=lens.tolist(), tables=tables, values=vals, lay=lay))
        assert n_new == sum(len(p) - min(m * B, len(p) - 1) for p, m in zip(prompts, matched.tolist()))
        st.insert(tokens, offs, width, cache, tables, after_lookup=True)
        st.release(ids, matched)
    assert found == [[0], [6, 3, 0]]
    assert st.status() == 0
    st.close()


def test_the_binding_refuses(G):
    b = make(G, G.KV_PACKED, torch.bfloat16, 8, 2, 128, 16, [50], [1])
    lay, c = b["lay"], b["cache"]
    with pytest.raises(ValueError):
        G.attend(lay, c, 1, b["q"], dev([0, 1]), dev([50]), b["tables"], 1)                       # no such layer
    with pytest.raises(ValueError):
        G.attend(lay, c, 0, b["q"].float(), dev([0, 1]), dev([50]), b["tables"], 1)
    with pytest.raises(ValueError):
        G.attend(lay, c, 0, b["q"], dev([0, 1], torch.int64), dev([50]), b["tables"], 1)
    with pytest.raises(ValueError):
        G.attend(lay, c, 0, b["q"], dev([0, 1]), dev([50]), b["tables"].t(), 1)
    with pytest.raises(ValueError):
        G.attend(lay, c, 0, b["q"].transpose(1, 2), dev([0, 1]), dev([50]), b["tables"], 1)
    with pytest.raises(ValueError):
        G.attend(lay, c, 0, b["q"], dev([0, 1]).cpu(), dev([50]), b["tables"], 1)                 # pageable host memory
    with pytest.raises(ValueError):
        G.attend(G.KVLayout(2, 64, 16, G.KV_PACKED), c, 0, b["q"], dev([0, 1]), dev([50]), b["tables"], 1)
    with pytest.raises(G.PTStoreError) as e:
        G.attend(lay, c, 0, b["q"], dev([0, 1]), dev([50]), b["tables"], 1, workspace=torch.zeros(1024, dtype=torch.uint8, device="cuda"))
    assert e.value.code == G.E_NOMEM
    with pytest.raises(G.PTStoreError):
        G.attend(lay, c, 0, b["q"][:, :7], dev([0, 1]), dev([50]), b["tables"], 1)                # 7 heads over 2
    with pytest.raises(ValueError):
        G.kv_write(lay, c, 0, b["q"][:2, :2], b["q"][:2, :2].half(), torch.arange(2, device="cuda"))
    with pytest.raises(ValueError):
        G.kv_write(lay, c, 0, b["q"][:2, :2], b["q"][:3, :2], torch.arange(2, device="cuda"))
    with pytest.raises(ValueError):
        G.map_slots(dev([3]), dev([1, 2]), b["tables"], 16, 4)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,new", [(128, 1), (128, 4), (64, 1), (64, 3)])
def test_a_cta_goes_from_item_to_item_of_a_ragged_batch(G, dtype, dim, new):
    """A CTA of the split kernel works on parts of several items of a 4-bit cache one after the other: the next one's tiles arrive where the last
    one's sums were joined.  Equal bits every time, and right."""
    rng = random.Random(41)
    lens = [rng.choice([5, 70, 200, rng.randint(100, 900)]) for _ in range(96)]
    b = make(G, G.KV_PACKED, dtype, 16, 4, dim, 16, lens, [min(new, n) for n in lens], seed=41)
    work = G.attend_workspace(b["lay"])
    call(G, b, workspace=work)
    check(G, b)
    first = b["out"].clone()
    for _ in range(20):
        b["out"].fill_(5.0)
        call(G, b, workspace=work)
        assert torch.equal(first, b["out"])


def test_plan_keeps_both_complaints_of_a_large_batch(G):
    """More than one scan step: a denied row in the first, and a length beyond its row handled by the same thread in the second."""
    R, block, width = 16384 + 1024, 16, 2
    for lane in (0, 5, 1023):
        lengths, held = [0] * R, [0] * R
        lengths[lane], lengths[16384 + lane] = 32, 33
        t, st, count, status = torch.full((R, width), -1, dtype=torch.int32, device="cuda"), dev([7, 8]), dev([1]), dev([0])
        h, c = G.assign_blocks(dev(lengths), dev(held), t, st, count, block, status=status)
        assert int(status.item()) == G.S_NOSPACE | G.S_BOUNDS, lane
        assert not bool(h.any()) and c.tolist() == [1] and bool((t == -1).all())


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("lens,new,rows_in", [([40, 30, 20, 10], [1, 1, 1, 1], 2), ([50, 70, 9], [4, 4, 4], 6), ([300, 200, 100], [40, 60, 30], 71), ([333, 90], [300, 64], 290)])
def test_rows_that_do_not_fit_keep_the_positions_of_the_others(G, fmt, dtype, lens, new, rows_in):
    """Offsets reach beyond q (the outputs of map_slots with too small a max_tokens): the rows that are there are as with all of them, and see
    no key behind their own position."""
    b = make(G, getattr(G, fmt), dtype, 8, 2, 128, 16, lens, new, seed=51, tail_rows=0)
    done = dev([n - m for n, m in zip(lens, new)])
    status = dev([0])
    offsets, slots, positions = G.map_slots(dev(lens), done, b["tables"], 16, rows_in, status=status)
    assert int(status.item()) == G.S_BOUNDS and offsets.tolist() == b["offsets"]
    out = torch.full_like(b["q"][:rows_in], 5.0)
    G.attend(b["lay"], b["cache"], 0, b["q"][:rows_in], offsets, dev(lens), b["tables"], max(new), out=out)
    want, spread, scores, _ = ref.attend(b["q"], b["offsets"], lens, b["tables"], b["values"][0], b["values"][1], 16, 128 ** -0.5)
    v_max, k_sum = float(b["values"][1].nan_to_num(0).abs().max()), float(b["values"][0].nan_to_num(0).abs().sum(-1).max()) * 128 ** -0.5
    tol = ref.attend_tolerance(b["q"], want, spread, scores, max(lens), v_max, fmt == "KV_PACKED", k_sum)
    assert bool(((out.double() - want[:rows_in]).abs() <= tol[:rows_in]).all())
    # the keys behind the last row that is there do not matter, NaN included
    r = max(i for i in range(len(lens)) if b["offsets"][i] < rows_in)
    first = int(positions[rows_in - 1]) + 1
    if first < lens[r]:
        behind = torch.tensor([int(b["tables"][r, p // 16]) * 16 + p % 16 for p in range(first, lens[r])], device="cuda")
        bad = torch.full((len(behind), 2, 128), float("nan"), dtype=dtype, device="cuda")
        G.kv_write(b["lay"], b["cache"], 0, bad, bad, behind)
        again = torch.full_like(out, 5.0)
        G.attend(b["lay"], b["cache"], 0, b["q"][:rows_in], offsets, dev(lens), b["tables"], max(new), out=again)
        assert torch.equal(again, out)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("new", [2, 40])
def test_lengths_and_offsets_at_the_ends_of_their_range(G, fmt, dtype, new):
    """The largest and smallest 32-bit lengths and offsets: a row sees what its table holds, or nothing."""
    top, low = 2 ** 31 - 1, -2 ** 31
    b = make(G, getattr(G, fmt), dtype, 4, 2, 64, 16, [90, 50], [new, new], seed=52, width=6, tail_rows=0)
    b["tables"] = b["tables"][:, :3].contiguous()                 # rows hold 48 tokens
    out = torch.full_like(b["q"], 5.0)
    G.attend(b["lay"], b["cache"], 0, b["q"], dev([0, new, 2 * new]), dev([top, low]), b["tables"], new, out=out)
    b["lens"] = [48 + new, 0]
    want = torch.full_like(out, 5.0)
    G.attend(b["lay"], b["cache"], 0, b["q"], dev([0, new, 2 * new]), dev([48 + new, 0]), b["tables"], new, out=want)
    assert torch.equal(out, want) and bool(torch.isfinite(out[:new]).all()) and not bool(out[new:].any())
    # offsets of the whole range: every row there is belongs to the one request and lies in front of its first key, or behind its last
    out.fill_(5.0)
    G.attend(b["lay"], b["cache"], 0, b["q"], dev([0, top, top]), dev([48, 48]), b["tables"], new, out=out)
    assert not bool(out.any())
    out.fill_(5.0)
    G.attend(b["lay"], b["cache"], 0, b["q"], dev([low, 2 * new, 2 * new]), dev([48 + 2 * new, 0]), b["tables"], new, out=out)
    assert torch.equal(out[:new], want[:new])


@pytest.mark.parametrize("polls", [1, 2, 5])
@pytest.mark.parametrize("fmt,dtype,heads,block,lens,new", [
    ("KV_PACKED", torch.bfloat16, 8, 16, [5000, 70, 3000, 900], [1, 1, 1, 1]),          # split kernel: its tiles are awaited long after they were asked for
    ("KV_PACKED", torch.float16, 8, 32, [2000 + 11 * i for i in range(40)], [4] * 40),    # ... CTAs that go on to other items
    ("KV_PACKED", torch.bfloat16, 8, 16, [4000, 300], [70, 300]),                        # 256-row tiles cut into chunks, 4-bit
    ("KV_PACKED", torch.float16, 8, 16, [300 + i for i in range(90)], [250] * 90),        # ... uncut
    ("KV_BF16", torch.bfloat16, 8, 16, [4000, 300], [70, 300]),                          # 16-bit through tensor maps
    ("KV_FP16", torch.float16, 8, 32, [300 + i for i in range(90)], [250] * 90),
    ("KV_BF16", torch.bfloat16, 6, 24, [2000, 300], [70, 300]),                          # 16-byte copies, a group that does not divide 128
    ("KV_FP16", torch.float16, 6, 24, [300 + i for i in range(90)], [250] * 90)])
def test_a_wait_that_runs_out_is_reported_and_leaves_the_workspace_ready(G, fmt, dtype, heads, block, lens, new, polls):
    """Limits of a few polls on a healthy GPU: a wait that runs out raises S_TIMEOUT and the call returns; without one the answers are right.  The same
    workspace then serves calls with the usual limit."""
    b = make(G, getattr(G, fmt), dtype, heads, 2, 128, block, lens, new, seed=61)
    ws = G.attend_workspace(b["lay"])
    call(G, b, workspace=ws)
    if max(new) < 200:
        check(G, b)
    want = b["out"].clone()
    seen, big = 0, torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    for _ in range(8):
        status = dev([0])
        b["out"].fill_(5.0)
        big.fill_(1)                                              # the cache comes from memory, not from L2
        G.attend(b["lay"], b["cache"], 0, b["q"], dev(b["offsets"]), dev(lens), b["tables"], max(new), out=b["out"], workspace=ws, status=status, wait_polls=polls)
        assert int(status.item()) in (0, G.S_TIMEOUT)
        if int(status.item()):
            seen += 1
        else:
            assert torch.equal(b["out"], want)
        assert bool((b["out"][b["offsets"][-1]:] == 5.0).all()) and not bool(ws[:2560].any())
    if polls == 1 and max(new) > 4:                               # the first wait follows its copy at once
        assert seen > 0
    status = dev([0])
    b["out"].fill_(5.0)
    call(G, b, workspace=ws, status=status)
    assert torch.equal(b["out"], want) and int(status.item()) == 0


@pytest.mark.parametrize("dtype,new,dim", [(torch.bfloat16, 1, 128), (torch.float16, 4, 128), (torch.bfloat16, 1, 64)])
def test_a_wait_of_the_split_kernel_that_runs_out(G, dtype, new, dim):
    """As above where tiles come late: every SM asks for its first tiles at once, while another stream copies at the memory's full rate."""
    lens = [6000 + 37 * (i % 5) for i in range(64)]
    b = make(G, G.KV_PACKED, dtype, 8, 2, dim, 16, lens, [new] * 64, seed=62)
    ws = G.attend_workspace(b["lay"])
    call(G, b, workspace=ws)
    check(G, b)
    want = b["out"].clone()
    src, dst, side, seen = (*torch.zeros(2, 1 << 30, dtype=torch.uint8, device="cuda"), torch.cuda.Stream(), 0)
    offsets, lengths = dev(b["offsets"]), dev(lens)
    for _ in range(6):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(10):
                dst.copy_(src)
        for _ in range(5):
            status = dev([0])
            b["out"].fill_(5.0)
            G.attend(b["lay"], b["cache"], 0, b["q"], offsets, lengths, b["tables"], new, out=b["out"], workspace=ws, status=status, wait_polls=1)
            assert int(status.item()) in (0, G.S_TIMEOUT)
            if int(status.item()):
                seen += 1
            else:
                assert torch.equal(b["out"], want)
            assert bool((b["out"][b["offsets"][-1]:] == 5.0).all()) and not bool(ws[:2560].any())
    torch.cuda.current_stream().wait_stream(side)
    print("ran out in %d of 30 calls" % seen)
    if dim == 128:                                                # of head size 64 twice as many tiles are asked for ahead
        assert seen > 0
    status = dev([0])
    b["out"].fill_(5.0)
    call(G, b, workspace=ws, status=status)
    assert torch.equal(b["out"], want) and int(status.item()) == 0


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("heads", [8, 6])
@pytest.mark.parametrize("new,many", [(1, 3), (1, 60), (3, 3), (3, 60), (40, 3), (40, 400), (300, 3), (300, 100)])
def test_every_kernel_writes_over_its_q(G, fmt, dtype, heads, new, many):
    """out is q itself: one token, a few, whole row tiles; items and steps that are cut and joined, and ones that are not; groups that divide a row
    tile and that do not."""
    rng = random.Random(new + many)
    lens = [new + (rng.randint(0, 2000) if many == 3 else rng.randint(0, 60)) for _ in range(many)]
    b = make(G, getattr(G, fmt), dtype, heads, 2, 64, 16, lens, [new] * many, seed=71, tail_rows=2)
    q = b["q"].clone()
    call(G, b)
    if new * many < 2000:
        check(G, b)
    want = b["out"].clone()
    want[-2:] = q[-2:]
    for _ in range(2):
        b["q"].copy_(q)
        call(G, b, out=b["q"])
        assert torch.equal(b["q"], want)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("lens,new", [([1, 40, 900], [1, 1, 1]), ([5000], [1]), ([3, 70, 2000], [3, 3, 3]), ([40, 3000], [40, 40]), ([200 + i for i in range(160)], [200] * 160)])
def test_scores_that_are_all_minus_infinity(G, fmt, dtype, lens, new):
    """A row that sees keys, all of them with a score of minus infinity, has no softmax: NaN, and only it.  A row that sees nothing is zero all the same."""
    b = make(G, getattr(G, fmt), dtype, 8, 2, 64, 16, lens + [5], new + [9], seed=81)
    slots = torch.tensor([int(b["tables"][r, p // 16]) * 16 + p % 16 for r, n in enumerate(lens + [5]) for p in range(n)], device="cuda") if len(lens) < 9 else None
    if slots is None:                                              # many: the same by whole rows of the table
        t = b["tables"].long()
        tok = torch.arange(t.shape[1] * 16, device="cuda")
        at = t[:, tok // 16] * 16 + tok % 16
        slots = at[tok[None, :] < dev(lens + [5])[:, None]]
    k = rows(gen_of(82), (len(slots), 2, 64), dtype).abs() + 0.5
    v = rows(gen_of(83), (len(slots), 2, 64), dtype, 0.25)
    G.kv_write(b["lay"], b["cache"], 0, k, v, slots)
    call(G, b)
    clean = b["out"].clone()
    assert bool(torch.isfinite(clean).all())
    odd = [(0, 0), (b["offsets"][1] - 1, 5), (b["offsets"][len(lens)] - 1, 7), (b["offsets"][len(lens)], 3)]
    for i, h in odd:
        b["q"][i, h] = float("-inf")
    b["out"].fill_(5.0)
    call(G, b)
    for i, h in odd[:3]:
        assert bool(b["out"][i, h].isnan().all()), (i, h)
        b["out"][i, h] = clean[i, h]
    assert torch.equal(b["out"], clean)
    assert not bool(b["out"][b["offsets"][len(lens)]:b["offsets"][len(lens)] + 4].any())      # nine rows over five keys: four see nothing
    b["tables"][:] = -1                                            # blocks that are not there are not seen
    b["out"].fill_(5.0)
    call(G, b)
    assert not bool(b["out"][:b["offsets"][-1]].any())


def test_attend_refuses_pinned_q_and_cache(G):
    """Both are fetched by bulk copies, which serve device memory; what is read by plain loads may be pinned."""
    for fmt, dtype in FORMATS[1:3]:
        b = make(G, getattr(G, fmt), dtype, 8, 2, 64, 16, [50, 70], [20, 1], seed=91)
        q, c = b["q"], b["cache"]
        for new in (1, 20):
            b["q"] = torch.empty(q.shape, dtype=q.dtype, pin_memory=True).copy_(q)
            with pytest.raises(ValueError):
                call(G, b, max_new=new)
            b["q"] = q
            b["cache"] = G.PagedKV(1, c.num_blocks, c.tensors[0].shape[2], tensors=[torch.empty(c.tensors[0].shape, dtype=torch.uint8, pin_memory=True)])
            with pytest.raises(ValueError):
                call(G, b, max_new=new)
            b["cache"] = c
        lens, offsets = (torch.tensor(x, dtype=torch.int32).pin_memory() for x in (b["lens"], b["offsets"]))
        tables = torch.empty(b["tables"].shape, dtype=torch.int32, pin_memory=True).copy_(b["tables"])
        G.attend(b["lay"], c, 0, q, offsets, lens, tables, 20, out=b["out"])
        check(G, b)


def check_some_rows(G, b, got, picks):
    """picks: (request, row of it).  Each is compared with a request of its own: one new token behind its position."""
    lay = b["lay"]
    every = torch.arange(b["cache"].tensors[0].shape[1] * lay.block_tokens, device="cuda")
    kv = G.kv_read(lay, b["cache"], 0, every, b["q"].dtype)
    values = [x.double().view(-1, lay.block_tokens, lay.heads, lay.dim) for x in kv]
    at = [b["offsets"][r] + i for r, i in picks]
    lens = [b["lens"][r] - b["new"][r] + i + 1 for r, i in picks]
    q, tables = b["q"][at], b["tables"][[r for r, _ in picks]]
    s = lay.dim ** -0.5
    want, spread, scores, _ = ref.attend(q, list(range(len(at) + 1)), lens, tables, values[0], values[1], lay.block_tokens, s)
    v_max, k_sum = float(values[1].nan_to_num(0).abs().max()), float(values[0].nan_to_num(0).abs().sum(-1).max()) * s
    tol = ref.attend_tolerance(q, want, spread, scores, max(lens), v_max, lay.format == G.KV_PACKED, k_sum)
    err = (got[at].double() - want).abs()
    assert bool((err <= tol).all()), "worst %.3g of the tolerance" % float((err / tol).nan_to_num(1e9).max())


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,new", [([4000, 900], [1, 1]), ([4000, 900], [3, 3]), ([4000], [60]), ([4000, 2500, 3100], [4000, 2500, 3100])])
@pytest.mark.parametrize("growth", [0.02, 0.3])
def test_scores_that_grow_along_the_sequence(G, fmt, dtype, dim, lens, new, growth):
    """Every score is larger than the ones before: the running maximum moves from step to step, and what was added up so far is scaled down each time.
    One token, a few, a suffix whose steps are cut, whole prompts whose row tiles are not cut."""
    b = make(G, getattr(G, fmt), dtype, 8, 2, dim, 16, lens, new, seed=95, tail_rows=0)
    gen, lay = gen_of(96), b["lay"]
    u = torch.randn(dim, generator=gen, device="cuda").sign()
    for r, n in enumerate(lens):
        pos = torch.arange(n, device="cuda")
        slots = b["tables"][r].long()[pos // 16] * 16 + pos % 16
        k = (u * (growth * pos / dim ** 0.5)[:, None, None] + 0.1 * torch.randn(n, 2, dim, generator=gen, device="cuda")).to(dtype)
        v = rows(gen, (n, 2, dim), dtype, 0.25)
        G.kv_write(lay, b["cache"], 0, k, v, slots)
    b["q"].copy_((u + 0.1 * torch.randn(b["q"].shape, generator=gen, device="cuda")).to(dtype))
    got = call(G, b)
    picks = [(r, i) for r, m in enumerate(new) for i in sorted({0, m // 3, m // 2, max(0, m - 130), m - 1})]
    check_some_rows(G, b, got, picks)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_row_tiles_over_many_keys_that_are_not_cut(G, fmt, dtype):
    """Whole prompts of some thousand tokens, more row tiles than would be cut; rows at both ends and in the middle of their tiles."""
    rng = random.Random(97)
    lens = [3000, 2049, 5000]
    b = make(G, getattr(G, fmt), dtype, 12, 2, 128, 16, lens, [3000, 2049, 4700], seed=97, tail_rows=0)
    got = call(G, b)
    picks = [(r, i) for r, m in enumerate(b["new"]) for i in (0, 42, 43, m // 2, m - 44, m - 1, rng.randrange(m), rng.randrange(m))]
    check_some_rows(G, b, got, picks)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("lens,new", [([1, 40, 900], [1, 1, 1]), ([3000, 70], [3, 3]), ([40, 2000], [40, 40]), ([120 + i for i in range(100)], [100] * 100)])
@pytest.mark.parametrize("scale", [1e6, 3e8, -1e10, 1e14, 1e30])
def test_scores_larger_than_their_differences_can_be_resolved(G, fmt, dtype, lens, new, scale):
    """Scores of up to 1e31 times log2 e: the largest one's weight is 1 and the others' are 0, wherever 32-bit sums can tell the two largest apart."""
    b = make(G, getattr(G, fmt), dtype, 4, 2, 64, 16, lens, new, seed=99, tail_rows=0)
    got = call(G, b, scale=scale)
    told = 0
    for r, (n, m) in enumerate(zip(lens, new)):
        k, _ = ref.gather(b["values"][0], b["tables"][r], n, 16)
        v, _ = ref.gather(b["values"][1], b["tables"][r], n, 16)
        q = b["q"][b["offsets"][r]:b["offsets"][r + 1]].double()
        s = torch.einsum("ihd,jhd->ihj", q, k.repeat_interleave(2, 1)) * (1 if scale > 0 else -1)
        # a sum of 64 products is off by at most 64 steps of 2^-23 of the products' magnitudes, bf16 rows as fp16 by 2^-25 of the row's largest element each
        off = 2.0 ** -16 * torch.einsum("ihd,jhd->ihj", q.abs(), k.abs().repeat_interleave(2, 1)).amax(2) + 2.0 ** -25 * 64 * q.abs().amax(2) * float(k.abs().max())
        seen = torch.arange(n, device="cuda")[None, None, :] <= (n - m + torch.arange(m, device="cuda"))[:, None, None]
        s = s.masked_fill(~seen, float("-inf"))
        top = s.topk(min(2, n), dim=2)
        gap = top.values[..., 0] - top.values[..., 1] if n > 1 else torch.full(s.shape[:2], float("inf"), dtype=torch.float64, device="cuda")
        # beyond the sums' error the weights' exponents differ by more than any type's range
        clear = gap > 2 * off + 2.0 ** -22 * top.values[..., 0].abs() + 400.0 / abs(scale)
        want = v[top.indices[..., 0], torch.arange(4, device="cuda") // 2]
        # The one weight is rounded to 16 bits before it meets V and is not before the sum: half a step of its type; then the result once: half a step
        half = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
        tol = (half[torch.float16 if fmt == "KV_PACKED" else dtype] + half[dtype] + 2.0 ** -20) * want.abs() + 2.0 ** -25
        err = (got[b["offsets"][r]:b["offsets"][r + 1]].double() - want).abs()
        assert bool((err <= tol)[clear].all()), "request %d" % r
        told += int(clear.sum())
    assert told > 0.5 * 4 * sum(new)
    assert bool(torch.isfinite(got).all())


@pytest.mark.parametrize("lens,new", [([1, 40, 900], [1, 1, 1]), ([70, 40], [3, 3]), ([40, 2000], [40, 40]), ([30 + i for i in range(100)], [20] * 100)])
def test_the_largest_queries_over_a_cache_of_zeros(G, lens, new):
    """bf16 rows over a 4-bit cache are scaled by a power of two that goes into the softmax scale: of the largest rows the product passes the range of 32 bits,
    and scores of zero are zero all the same.  Every row is the mean of the values it sees."""
    b = make(G, G.KV_PACKED, torch.bfloat16, 8, 2, 64, 16, lens, new, seed=101, tail_rows=0)
    b["lay"] = G.KVLayout(2, 64, 16, G.KV_PACKED, 2.0 ** 20, 2.0 ** -6)
    t = b["tables"].long()
    tok = torch.arange(t.shape[1] * 16, device="cuda")
    slots = (t[:, tok // 16] * 16 + tok % 16)[tok[None, :] < dev(lens)[:, None]]
    v = rows(gen_of(102), (len(slots), 2, 64), torch.bfloat16, 0.25)
    G.kv_write(b["lay"], b["cache"], 0, torch.zeros_like(v), v, slots)
    b["q"].fill_(3e38)
    b["values"] = [x.double().view(-1, 16, 2, 64) for x in G.kv_read(b["lay"], b["cache"], 0, torch.arange(b["cache"].num_blocks * 16, device="cuda"), torch.bfloat16)]
    got = call(G, b)
    for r, n in enumerate(lens):
        vs, _ = ref.gather(b["values"][1], b["tables"][r], n, 16)
        for i in sorted({0, new[r] - 1}):
            see = vs[:n - new[r] + i + 1].repeat_interleave(4, 1)
            # every weight is 1, exactly; a sum of 32 bits and one rounding
            tol = 2.0 ** -8 * see.mean(0).abs() + 2.0 ** -22 * n * see.abs().mean(0)
            bad = ~((got[b["offsets"][r] + i].double() - see.mean(0)).abs() <= tol)
            assert not bool(bad.any()), (r, i)
