"""The cache of latent vectors and the absorbed attention over it, on the GPU, against the definitions in 64 bits."""
import math
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

from tests import operators_reference as ref

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # largest relative error of a rounding


@pytest.fixture(scope="module")
def G():
    from paper_2607_22648_b200 import binding
    return binding


def dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def gen_of(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows(gen, shape, dtype, spread=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * spread).to(dtype)


def layout(G, L, block, dtype):
    return G.KVLayout(1, L + 64, block, {torch.bfloat16: G.KV_LATENT_BF16, torch.float16: G.KV_LATENT_FP16}[dtype])


def make(G, L, dtype, heads, block, lens, new, seed=0, tail_rows=3, strided=False, layer=1, spread=1.0):
    """A batch over a cache whose bytes behind the sequences (and whose other layer) read as NaN."""
    gen = gen_of(2000 + seed)
    lay = layout(G, L, block, dtype)
    blocks = [-(-max(n, 0) // block) for n in lens]
    nb = sum(blocks) + 2
    cache = G.PagedKV(1, nb, lay.chunk_bytes)
    cache.tensors[0].fill_(0xFF)
    perm = torch.randperm(nb, generator=gen, device="cuda").int().tolist()
    width, tables, at, slots = max(blocks + [1]) + 1, [], 0, []
    for n, b in zip(lens, blocks):
        row = perm[at:at + b]
        at += b
        slots += [row[p // block] * block + p % block for p in range(max(n, 0))]
        tables.append(row + [-1] * (width - b))
    n = len(slots)
    c, r = rows(gen, (n, L), dtype, spread), rows(gen, (n, 64), dtype, spread)
    slots = torch.tensor(slots, dtype=torch.int64, device="cuda")
    G.latent_write(lay, cache, layer, c, r, slots)
    values = torch.full((nb * block, L + 64), float("nan"), dtype=torch.float64, device="cuda")
    values[slots] = torch.cat([c, r], 1).double()
    offsets = [0]
    for m in new:
        offsets.append(offsets[-1] + m)
    T = offsets[-1] + tail_rows
    q = rows(gen, (T, heads, L + 64), dtype)
    if strided:
        out = torch.full((T, 2, heads, L), 5.0, dtype=dtype, device="cuda")[:, 1]
        ql, qr = q[:, :, :L], q[:, :, L:]
    else:
        out = torch.full((T, heads, L), 5.0, dtype=dtype, device="cuda")
        ql, qr = q[:, :, :L].contiguous(), q[:, :, L:].contiguous()
    lse = torch.full((T, heads), 7.0, device="cuda")
    return dict(lay=lay, cache=cache, layer=layer, ql=ql, qr=qr, q=q, out=out, lse=lse, offsets=offsets, lens=list(lens), new=list(new),
                tables=dev(tables).view(len(lens), width), values=values.view(nb, block, L + 64), L=L, scale=192 ** -0.5)


def call(G, b, **kw):
    args = dict(out=b["out"], lse=b["lse"])
    args.update(kw)
    max_new, scale = args.pop("max_new", max(b["new"] + [1])), args.pop("scale", b["scale"])
    return G.latent_attend(b["lay"], b["cache"], b["layer"], b["ql"], b["qr"], dev(b["offsets"]), dev(b["lens"]), b["tables"], max_new, scale, **args)


def check(b, got=None, lse=None, scale=None, picks=None):
    """A score is the sum of exact products, 32 bits wide (one step of 2^-23 of the running sum per addend, at most): off by (D + 8) 2^-23 sum |q k| scale, the
    scale factor and exp2 add 2^-20 relative.  A weight is off by twice that relative to their sum, and by half a step of 16 bits (below fp16's normal
    range 2^-25).  The output is rounded once.  lse: off by what a score is, the sum's relative error and a few steps of its own size."""
    got, lse = b["out"] if got is None else got, b["lse"] if lse is None else lse
    scale, block, L = b["scale"] if scale is None else scale, b["lay"].block_tokens, b["L"]
    dtype = got.dtype
    half = HALF[dtype]
    owned = torch.zeros(got.shape[0], dtype=torch.bool, device="cuda")
    for r, n in enumerate(b["lens"]):
        a, e = b["offsets"][r], b["offsets"][r + 1]
        owned[a:e] = True
        if a == e:
            continue
        which = range(a, e) if picks is None else [i for i in range(a, e) if i in picks]
        if n > 0:
            keys, ok = ref.gather(b["values"], b["tables"][r], n, block)
        for i in which:
            pos = n - (e - a) + (i - a)
            see = torch.zeros(0, L + 64, dtype=torch.float64, device="cuda") if pos < 0 else keys[:pos + 1][ok[:pos + 1]]
            if see.shape[0] == 0:
                assert bool((got[i] == 0).all()) and bool((lse[i] == -math.inf).all()), (r, i)
                continue
            q = b["q"][i].double()
            s = q @ see.t() * scale
            p = torch.softmax(s, 1)
            want, spread = p @ see[:, :L], p @ see[:, :L].abs()
            scores = (q.abs() @ see.abs().t()).amax(1, keepdim=True) * abs(scale)
            e_score = (L + 72) * 2.0 ** -23 * scores + 2.0 ** -20
            tol = spread * (half + 2 * e_score) + half * want.abs()
            if dtype == torch.float16:
                tol = tol + see.shape[0] * 2.0 ** -25 * float(see[:, :L].abs().max()) + 2.0 ** -25
            err = (got[i].double() - want).abs()
            assert bool((err <= tol).all()), "row %d of request %d: worst %.3g of the tolerance" % (i - a, r, float((err / tol).nan_to_num(1e9).max()))
            w = torch.logsumexp(s, 1)
            err = (lse[i].double() - w).abs()
            assert bool((err <= 2 * e_score[:, 0] + 2.0 ** -21 * w.abs() + 2.0 ** -18).all()), (r, i, float(err.max()))
    assert bool((got[~owned] == 5.0).all()) and bool((lse[~owned] == 7.0).all()), "rows of no request changed"


BOTH = [torch.bfloat16, torch.float16]


# ---- rows -----------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("L,block,tokens", [(512, 16, 1), (512, 8, 64), (256, 24, 333), (512, 128, 5000)])
def test_rows_round_trip(G, L, block, tokens, dtype):
    gen = gen_of(tokens)
    lay = layout(G, L, block, dtype)
    nb = -(-tokens // block) + 2
    cache = G.PagedKV(1, nb, lay.chunk_bytes)
    for layer in (0, 1):
        cache.tensors[0].fill_(0xEE)
        c, r = rows(gen, (tokens, L + 8), dtype)[:, :L], rows(gen, (tokens, 2, 64), dtype)[:, 1]       # any token stride
        slots = torch.randperm(nb * block, generator=gen, device="cuda")[:tokens]
        skip = torch.rand(tokens, generator=gen, device="cuda") < 0.2
        slots[skip] = -1
        status = dev([0])
        G.latent_write(lay, cache, layer, c, r, slots, status=status)
        plane = cache.tensors[0][layer].view(dtype).view(nb * block, L + 64)
        keep = slots[~skip]
        assert torch.equal(plane[keep], torch.cat([c, r], 1)[~skip])
        other = torch.ones(nb * block, dtype=torch.bool, device="cuda")
        other[keep] = False
        assert bool((plane[other].view(torch.uint8) == 0xEE).all()) and bool((cache.tensors[0][1 - layer] == 0xEE).all())
        c2, r2 = torch.full((tokens, L), 3.0, dtype=dtype, device="cuda"), torch.full((tokens, 64), 3.0, dtype=dtype, device="cuda")
        G.latent_read(lay, cache, layer, slots, latent=c2, rope=r2, status=status)
        assert torch.equal(c2[~skip], c[~skip]) and torch.equal(r2[~skip], r[~skip]) and bool((c2[skip] == 3).all()) and bool((r2[skip] == 3).all())
        assert int(status.item()) == 0


def test_rows_outside_the_cache_are_reported(G):
    lay = layout(G, 512, 16, torch.bfloat16)
    cache = G.PagedKV(1, 2, lay.chunk_bytes)
    cache.tensors[0].zero_()
    one = torch.ones(4, 512, dtype=torch.bfloat16, device="cuda")
    status = dev([0])
    G.latent_write(lay, cache, 0, one, one[:, :64], dev([-2, 32, 31, 1 << 40], torch.int64), status=status)
    assert int(status.item()) == G.S_BOUNDS and float(cache.tensors[0].view(torch.bfloat16).float().sum()) == 576
    status.zero_()
    got, _ = G.latent_read(lay, cache, 0, dev([31, 99], torch.int64), latent=torch.zeros(2, 512, dtype=torch.bfloat16, device="cuda"), status=status)
    assert int(status.item()) == G.S_BOUNDS and got.float().sum(1).tolist() == [512, 0]


# ---- attention ------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("L", [512, 256])
@pytest.mark.parametrize("heads", [1, 16, 40, 64, 65, 128])
def test_decode_ragged(G, L, dtype, heads):
    lens = [1, 2, 7, 8, 9, 63, 64, 65, 127, 128, 129, 300, 1000, 77]
    b = make(G, L, dtype, heads, 16, lens, [1] * len(lens), seed=heads)
    call(G, b)
    check(b)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("block", [8, 24, 64, 128, 200])
def test_block_sizes_and_strides(G, dtype, block):
    b = make(G, 512, dtype, 12, block, [500, 3, 129, 64], [1, 3, 2, 20], seed=block, strided=True)
    call(G, b)
    check(b)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("L,heads", [(512, 16), (256, 48), (512, 100)])
def test_mixed_new_tokens_and_empty_rows(G, L, heads, dtype):
    """Requests without rows, without tokens, with more rows than tokens, and whole prompts."""
    lens, new = [0, 5, 40, 200, 0, 33, 130, 1, 64], [1, 0, 40, 3, 0, 36, 130, 1, 64]
    b = make(G, L, dtype, heads, 16, lens, new, seed=9)
    call(G, b)
    check(b)
    b["out"].fill_(5.0)
    call(G, b, max_new=100000)
    check(b)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("n,new,heads", [(20000, 1, 16), (9000, 1, 128), (5000, 4, 20), (3000, 70, 16)])
def test_one_long_request_is_split_and_joined(G, dtype, n, new, heads):
    b = make(G, 512, dtype, heads, 32, [n], [new], seed=n)
    call(G, b)
    check(b, picks={0, 1, new // 2, new - 1})
    first, lse = b["out"].clone(), b["lse"].clone()
    for _ in range(3):
        call(G, b)
        assert torch.equal(b["out"], first) and torch.equal(b["lse"], lse)


@pytest.mark.parametrize("dtype", BOTH)
def test_many_requests(G, dtype):
    rng = random.Random(4)
    lens = [rng.choice([0, 1, 16, rng.randint(1, 400)]) for _ in range(900)]
    b = make(G, 256, dtype, 8, 16, lens, [rng.choice([0, 1, 1, 2]) for _ in lens], seed=4)
    call(G, b)
    check(b)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("new", [1, 5, 40])
def test_entries_outside_the_cache_and_lengths_beyond_the_table(G, dtype, new):
    lens = [300, 90, 129, 64]
    b = make(G, 512, dtype, 16, 16, lens, [new] * 4, seed=new)
    t = b["tables"].clone()
    t[0, 1], t[0, 18], t[1, 0], t[3, :] = 1 << 20, -5, -1, -1
    b["tables"] = t
    status = dev([0])
    call(G, b, status=status)
    assert int(status.item()) == G.S_BOUNDS
    check(b)
    b = make(G, 512, dtype, 16, 16, [50, 20], [new, 1], seed=5)
    b["tables"] = b["tables"][:, :2].contiguous()
    b["lens"] = [50, 20]
    call(G, b)                                                    # keys behind the row of the table are not seen
    check(b)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("new,heads", [(64, 16), (3, 16), (20, 128)])
def test_what_is_not_finite_in_later_tokens_does_not_reach_earlier_rows(G, dtype, new, heads):
    lens = [200, new, 65]
    b = make(G, 512, dtype, heads, 16, lens, [new, new, min(new, 65)], seed=11)
    kinds = [math.inf, -math.inf, math.nan]
    bad = {0: 200 - new // 2 - 1, 1: new - 1, 2: 64}
    for r, p in bad.items():
        blk, t = int(b["tables"][r, p // 16]), p % 16
        plane = b["cache"].tensors[0][b["layer"]].view(dtype).view(-1, 16, 576)
        plane[blk, t, 5 + r] = kinds[r]
        plane[blk, t, 520] = kinds[r]
    call(G, b)
    got, lse = b["out"].clone(), b["lse"].clone()
    for r, p in bad.items():
        a, e = b["offsets"][r], b["offsets"][r + 1]
        for i in range(a, e):
            if lens[r] - (e - a) + (i - a) >= p:
                assert bool(got[i, :, 5 + r].isnan().all()), (r, i)
                got[i] = 5.0
        b["new"][r] = 0
    clean = make(G, 512, dtype, heads, 16, lens, [new, new, min(new, 65)], seed=11)
    call(G, clean)
    seen = (got == 5.0).all(-1)
    assert bool(((got == clean["out"]) | seen[..., None]).all())


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("scale", [-0.07, 0.0, 40.0])
def test_scales(G, dtype, scale):
    b = make(G, 256, dtype, 16, 16, [300, 40], [1, 20], seed=3, spread=0.3)
    call(G, b, scale=scale)
    check(b, scale=scale)


@pytest.mark.parametrize("dtype", BOTH)
def test_scores_that_grow_along_the_sequence(G, dtype):
    """The reference moves with every step: the sums before it are rescaled."""
    b = make(G, 512, dtype, 16, 16, [1500, 700], [1, 30], seed=8)
    plane = b["cache"].tensors[0][b["layer"]].view(dtype).view(-1, 16, 576)
    b["q"][:, :, 512] = 6.0
    b["qr"][:, :, 0] = 6.0
    for r, n in enumerate(b["lens"]):
        for p in range(n):
            plane[int(b["tables"][r, p // 16]), p % 16, 512] = p / 16.0
    b["values"] = plane.double()
    call(G, b)
    check(b)


@pytest.mark.parametrize("dtype", BOTH)
def test_rows_whose_scores_are_all_minus_infinity(G, dtype):
    b = make(G, 256, dtype, 4, 16, [90, 33], [1, 2], seed=6, spread=0.0)
    b["cache"].tensors[0][b["layer"]].view(dtype).view(-1, 320)[:, 300] = 1.0
    b["qr"].zero_()
    b["qr"][:, :, 300 - 256] = -math.inf
    call(G, b)
    assert bool(b["out"][:3].isnan().all()) and bool((b["lse"][:3] == -math.inf).all()) and bool((b["out"][3:] == 5.0).all())


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("new,n", [(1, 4000), (40, 300)])
def test_q_may_be_the_output(G, dtype, new, n):
    b = make(G, 512, dtype, 24, 16, [n, 70], [new, min(new, 70)], seed=12)
    call(G, b)
    want = b["out"].clone()
    again = b["ql"].clone()
    b["ql"] = again
    call(G, b, out=again)
    T = b["offsets"][-1]
    assert torch.equal(again[:T], want[:T])


@pytest.mark.parametrize("dtype", BOTH)
def test_q_of_many_short_requests_may_be_the_output(G, dtype):
    """Two CTAs share 128 rows and go through several requests each, not in step: neither may overwrite what the other has still to read."""
    lens = [64 + 37 * i % 200 for i in range(700)]
    b = make(G, 512, dtype, 128, 16, lens, [1] * 700, seed=13)
    call(G, b)
    want = b["out"].clone()
    first = b["ql"].clone()
    for _ in range(5):
        again = first.clone()
        b["ql"] = again
        call(G, b, out=again)
        assert torch.equal(again[:700], want[:700])


@pytest.mark.parametrize("dtype", BOTH)
def test_calls_of_all_shapes_share_a_workspace(G, dtype):
    """What a call leaves in the workspace does not reach the next one."""
    shapes = [([9000], [1], 16), ([100], [1], 16), ([3000, 2000], [40, 1], 16), ([5000, 64], [1, 1], 128), ([1], [1], 1)]
    batches = [make(G, 512, dtype, h, 16, lens, new, seed=20 + i) for i, (lens, new, h) in enumerate(shapes)]
    want = []
    for b in batches:
        call(G, b)
        want.append((b["out"].clone(), b["lse"].clone()))
    ws = G.latent_workspace(batches[0]["lay"])
    ws.fill_(0xFF)
    for i in (0, 1, 0, 2, 1, 3, 4, 2, 0, 3):
        b = batches[i]
        b["out"].fill_(5.0)
        call(G, b, workspace=ws)
        assert torch.equal(b["out"], want[i][0]) and torch.equal(b["lse"], want[i][1]), i


@pytest.mark.parametrize("dtype", BOTH)
def test_streams_and_graphs(G, dtype):
    b = make(G, 512, dtype, 32, 16, [4000, 500, 90], [1, 2, 1], seed=30)
    call(G, b)
    want = b["out"].clone()
    ws = G.latent_workspace(b["lay"])
    off, lens = dev(b["offsets"]), dev(b["lens"])

    def step():
        G.latent_attend(b["lay"], b["cache"], b["layer"], b["ql"], b["qr"], off, lens, b["tables"], 2, b["scale"], out=b["out"], workspace=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b["out"].fill_(5.0)
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    b["out"].fill_(5.0)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g in graphs:
        with torch.cuda.graph(g):
            step()
    lens.copy_(dev([100, 400, 90]))                              # replayed with other lengths, then with the first ones
    graphs[0].replay()
    lens.copy_(dev(b["lens"]))
    graphs[1].replay()
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(b["out"], want)


@pytest.mark.parametrize("polls", [1, 3])
@pytest.mark.parametrize("heads,lens,new", [(16, [4000] * 3, 1), (128, [3000] * 40, 1), (16, [2000, 300], 70)])
def test_a_wait_that_runs_out_is_reported_and_the_workspace_serves_on(G, heads, lens, new, polls):
    b = make(G, 512, torch.bfloat16, heads, 16, lens, [new] * len(lens), seed=40)
    ws = G.latent_workspace(b["lay"])
    call(G, b, workspace=ws)
    want = b["out"].clone()
    seen, big = 0, torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    for _ in range(4):
        status = dev([0])
        b["out"].fill_(5.0)
        big.fill_(1)
        call(G, b, workspace=ws, status=status, wait_polls=polls)
        got = int(status.item())
        assert got in (0, G.S_TIMEOUT)
        seen += got != 0
        assert got or torch.equal(b["out"], want)
        assert bool((b["out"][b["offsets"][-1]:] == 5.0).all())
    if polls == 1:
        assert seen > 0
    status = dev([0])
    call(G, b, workspace=ws, status=status)
    assert torch.equal(b["out"], want) and int(status.item()) == 0


def test_offsets_beyond_32_bits(G):
    """A cache of more than 4 GB, whose last blocks are used."""
    lay = layout(G, 512, 64, torch.bfloat16)
    nb = (5 << 30) // lay.chunk_bytes
    cache = G.PagedKV(1, nb, lay.chunk_bytes)
    gen = gen_of(50)
    n = 200
    ids = [nb - 1, 3, nb - 2, nb // 2]
    slots = torch.tensor([ids[p // 64] * 64 + p % 64 for p in range(n)], dtype=torch.int64, device="cuda")
    c, r = rows(gen, (n, 512), torch.bfloat16), rows(gen, (n, 64), torch.bfloat16)
    G.latent_write(lay, cache, 1, c, r, slots)
    c2, r2 = G.latent_read(lay, cache, 1, slots)
    assert torch.equal(c, c2) and torch.equal(r, r2)
    q = rows(gen, (1, 16, 576), torch.bfloat16)
    out = G.latent_attend(lay, cache, 1, q[:, :, :512], q[:, :, 512:], dev([0, 1]), dev([n]), dev([ids]), 1, 0.07)
    k = torch.cat([c, r], 1).double()
    want = torch.softmax(q[0].double() @ k.t() * 0.07, 1) @ c.double()
    assert float((out[0].double() - want).abs().max()) < 0.02


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("L,heads,new,max_new", [(512, 80, 1, 1), (512, 96, 1, 1), (512, 20, 1, 2), (512, 16, 9, 9), (512, 32, 3, 3), (256, 72, 1, 1)])
def test_rows_that_leave_pieces_of_a_tile_out(G, L, heads, new, max_new, dtype):
    """The output of a pair of CTAs goes out 32 rows and 128 elements at a time, through two places in turn.  Pieces without rows are left out: the turns must not follow the pieces' numbers."""
    lens = [64 + 37 * i % 200 for i in range(300)]
    b = make(G, L, dtype, heads, 16, lens, [new] * 300, seed=heads + new)
    call(G, b, max_new=max_new)
    check(b, picks={b["offsets"][r] + i for r in range(0, 300, 7) for i in (0, new - 1)})
    want, lse = b["out"].clone(), b["lse"].clone()
    for _ in range(20):
        b["out"].fill_(5.0)
        call(G, b, max_new=max_new)
        assert torch.equal(b["out"], want) and torch.equal(b["lse"], lse)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("heads,new", [(16, 1), (16, 3), (100, 1)])
def test_an_infinity_in_the_rotary_part_counts_by_its_score(G, dtype, heads, new):
    """Scores of minus infinity leave the token out; heads whose score is infinite, or not a number, have no output."""
    b = make(G, 512, dtype, heads, 16, [300, 70], [new] * 2, seed=60)
    b["qr"][:, :, 9] = -1.0
    b["qr"][:, 1, 9] = 2.0
    b["qr"][:, 2, 9] = 0.0
    b["q"][:, :, 512:] = b["qr"]
    plane = b["cache"].tensors[0][b["layer"]].view(dtype).view(-1, 16, 576)
    for r, p in ((0, 150), (1, 3)):
        plane[int(b["tables"][r, p // 16]), p % 16, 512 + 9] = math.inf
    call(G, b)
    got, lse = b["out"].clone(), b["lse"].clone()
    rows_of = slice(0, b["offsets"][-1])
    assert bool(got[rows_of, 1:3].isnan().all()) and bool(got[rows_of, 3:].isfinite().all()) and bool(got[rows_of, 0].isfinite().all())
    # the other heads as if the tokens' scores were far below the rest (powers of two of less than -150 vanish in 32 bits)
    for r, p in ((0, 150), (1, 3)):
        plane[int(b["tables"][r, p // 16]), p % 16, 512 + 9] = 60000.0
    call(G, b)
    keep = [h for h in range(heads) if h not in (1, 2)]
    assert torch.equal(got[rows_of][:, keep], b["out"][rows_of][:, keep]) and torch.equal(lse[rows_of][:, keep], b["lse"][rows_of][:, keep])


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("heads,new,max_new", [(80, 1, 1), (96, 1, 1), (20, 1, 2), (16, 9, 9)])
def test_q_may_be_the_output_of_rows_that_leave_pieces_out(G, heads, new, max_new, dtype):
    lens = [64 + 37 * i % 200 for i in range(300)]
    b = make(G, 512, dtype, heads, 16, lens, [new] * 300, seed=heads + new)
    call(G, b, max_new=max_new)
    want, first, T = b["out"].clone(), b["ql"].clone(), b["offsets"][-1]
    for _ in range(5):
        b["ql"] = first.clone()
        call(G, b, max_new=max_new, out=b["ql"])
        assert torch.equal(b["ql"][:T], want[:T]) and torch.equal(b["ql"][T:], first[T:])
