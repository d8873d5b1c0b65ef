"""Attention over expanded keys and values on the GPU against its definition in 64 bits."""
import math
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

BOTH = [torch.bfloat16, torch.float16]
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # largest relative error of a rounding


@pytest.fixture(scope="module")
def G():
    from paper_2607_22648_b200 import binding
    return binding


def dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def rows(gen, shape, dtype, spread=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * spread).to(dtype)


def make(dtype, heads, keys, new, seed=0, tail=3, spread=1.0, layout="joint"):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3000 + seed)
    T, N = sum(new) + tail, sum(keys) + tail
    q, r = rows(gen, (T, heads, 192), dtype), rows(gen, (N, 64), dtype, spread)
    kv = rows(gen, (N, heads, 256), dtype, spread)
    k, v = kv[:, :, :128], kv[:, :, 128:]
    if layout == "strided":
        q = rows(gen, (T, heads + 1, 200), dtype)[:, :heads, :192]
        k, v, r = k.transpose(0, 1).contiguous().transpose(0, 1), v.contiguous(), rows(gen, (N, 2, 64), dtype)[:, 1]
    elif layout == "shared":                                       # one key and value for all heads
        k, v = k[:, :1].expand(N, heads, 128), v[:, :1].expand(N, heads, 128)
    k[sum(keys):], v[sum(keys):], r[sum(keys):] = math.nan, math.nan, math.nan      # of no request
    out = torch.full((T, 2, heads, 128), 5.0, dtype=dtype, device="cuda")[:, 1] if layout == "strided" else torch.full((T, heads, 128), 5.0, dtype=dtype, device="cuda")
    start = lambda n: [sum(n[:i]) for i in range(len(n) + 1)]
    return dict(q=q, k=k, r=r, v=v, out=out, off=start(new), koff=start(keys), new=list(new), keys=list(keys), scale=192 ** -0.5)


def call(G, b, **kw):
    args = dict(out=b["out"], scale=b["scale"])
    args.update(kw)
    return G.expanded_attend(b["q"], b["k"], b["r"], b["v"], dev(b["off"]), dev(b["koff"]), args.pop("max_new", max(b["new"] + [1])), **args)


def check(b, got=None, scale=None, picks=None):
    """A score is off by what 32-bit sums of exact products may be (one step of 2^-23 of the running sum per addend), the scale and the exponential add 2^-20 relative; a weight by twice
    that relative to their sum and by half a step of 16 bits (below fp16's normal range 2^-25); the output is rounded once."""
    got, scale = b["out"] if got is None else got, b["scale"] if scale is None else scale
    dtype, heads = got.dtype, got.shape[1]
    owned = torch.zeros(got.shape[0], dtype=torch.bool, device="cuda")
    for x in range(len(b["new"])):
        a, e, ka, n = b["off"][x], b["off"][x + 1], b["koff"][x], b["keys"][x]
        owned[a:e] = True
        ids = torch.arange(a, e, device="cuda") if picks is None else torch.tensor(sorted({min(a + p, e - 1) for p in picks} if e > a else []), dtype=torch.int64, device="cuda")
        if ids.numel() == 0:
            continue
        see = torch.arange(n, device="cuda")[None] <= (n - (e - a) + ids - a)[:, None]
        none = ~see.any(1)
        assert bool((got[ids[none]] == 0).all()), x
        ids, see = ids[~none], see[~none]
        if ids.numel() == 0:
            continue
        for h in range(heads):
            k = torch.cat([b["k"][ka:ka + n, h], b["r"][ka:ka + n]], 1).double()
            v, q = b["v"][ka:ka + n, h].double(), b["q"][ids, h].double()
            s = torch.where(see, q @ k.t() * scale, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
            p = torch.softmax(s, 1)
            want, spread = p @ v, p @ v.abs()
            big = torch.where(see, q.abs() @ k.abs().t() * abs(scale), torch.zeros((), dtype=torch.float64, device="cuda")).amax(1, keepdim=True)
            tol = spread * (HALF[dtype] + 2 * ((192 + 8) * 2.0 ** -23 * big + 2.0 ** -20)) + HALF[dtype] * want.abs()
            if dtype == torch.float16:
                tol = tol + n * 2.0 ** -25 * float(v.abs().max()) + 2.0 ** -25
            err = (got[ids, h].double() - want).abs()
            assert bool((err <= tol).all()), "request %d head %d: worst %.3g of the tolerance" % (x, h, float((err / tol).nan_to_num(1e9).max()))
    assert bool((got[~owned] == 5.0).all()), "rows of no request changed"


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 400])
def test_one_prompt(G, dtype, n):
    b = make(dtype, 2, [n], [n], seed=n)
    call(G, b)
    check(b)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("layout,heads", [("joint", 3), ("joint", 16), ("strided", 5), ("shared", 4), ("joint", 1)])
def test_ragged_batches(G, dtype, layout, heads):
    """Whole prompts, suffixes, single tokens, requests without rows, without keys, with more rows than keys."""
    keys, new = [300, 5, 0, 700, 64, 0, 33, 1, 513], [300, 0, 0, 3, 64, 2, 40, 1, 260]
    b = make(dtype, heads, keys, new, seed=heads, layout=layout)
    call(G, b)
    check(b)
    b["out"].fill_(5.0)
    call(G, b, max_new=100000)
    check(b)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("n,new", [(3000, 3000), (5000, 300), (4096, 256)])
def test_long_prompts(G, dtype, n, new):
    b = make(dtype, 2, [n, 100], [new, 100], seed=n)
    call(G, b)
    check(b, picks={0, 1, 127, 128, 255, 256, new // 2, new - 1})
    first = b["out"].clone()
    for _ in range(3):
        call(G, b)
        assert torch.equal(b["out"], first)


@pytest.mark.parametrize("dtype", BOTH)
def test_many_requests(G, dtype):
    rng = random.Random(5)
    keys = [rng.choice([0, 1, 16, rng.randint(1, 300)]) for _ in range(700)]
    new = [rng.randint(0, min(n, 20)) for n in keys]
    b = make(dtype, 2, keys, new, seed=5)
    call(G, b)
    check(b)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("scale", [-0.1, 0.0, 30.0])
def test_scales(G, dtype, scale):
    b = make(dtype, 2, [300, 40], [300, 7], seed=6, spread=0.4)
    call(G, b, scale=scale)
    check(b, scale=scale)


@pytest.mark.parametrize("dtype", BOTH)
def test_scores_that_grow_along_the_sequence(G, dtype):
    b = make(dtype, 1, [1500], [600], seed=8)
    b["q"][:, :, 130] = 6.0
    b["r"][:1500, 2] = torch.arange(1500, device="cuda") / 16.0
    call(G, b)
    check(b)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("scale", [2.0 ** 24, -(2.0 ** 26)])
def test_scores_larger_than_their_differences_can_be_resolved(G, dtype, scale):
    """Scores of 2^24 and more, equal in groups: the largest weight is one however they are rounded."""
    b = make(dtype, 1, [300], [300], seed=9)
    b["q"].zero_()
    b["q"][:, :, 0] = 8.0
    b["k"][:300, :, 0] = (torch.arange(300, device="cuda") % 7 - 3).to(dtype)[:, None]
    call(G, b, scale=scale)
    for i in (0, 5, 6, 7, 128, 299):
        s = b["k"][:i + 1, 0, 0].double() * (1 if scale > 0 else -1)
        at = (s == s.max()).nonzero()[:, 0]
        want = b["v"][at, 0].double().mean(0)
        assert float((b["out"][i, 0].double() - want).abs().max()) <= HALF[dtype] * (float(b["v"][at, 0].double().abs().mean(0).max()) + float(want.abs().max())) + 2.0 ** -16


@pytest.mark.parametrize("dtype", BOTH)
def test_what_is_not_finite_behind_a_row_has_no_influence(G, dtype):
    keys, new = [200, 150, 300], [200, 30, 280]
    clean = make(dtype, 2, keys, new, seed=11)
    call(G, clean)
    b = make(dtype, 2, keys, new, seed=11)
    spots = [(0, 130, math.nan), (1, 140, math.inf), (2, 299, -math.inf), (2, 20, math.inf)]
    for x, p, y in spots:
        b["v"][b["koff"][x] + p, 1, 7 + x] = y
    call(G, b)
    got, want = b["out"].clone(), clean["out"].clone()
    for x, p, y in spots:
        for i in range(b["off"][x], b["off"][x + 1]):
            if keys[x] - new[x] + i - b["off"][x] >= p:
                z = b["out"][i, 1, 7 + x].item()
                assert not math.isfinite(z), (x, i)
                got[i, 1, 7 + x] = want[i, 1, 7 + x] = 0
    assert torch.equal(got, want)
    # keys that are not finite: only the rows that see them
    b = make(dtype, 2, keys, new, seed=11)
    b["k"][130, 0, 3], b["r"][b["koff"][2] + 250, 3] = math.nan, math.nan
    call(G, b)
    assert bool(b["out"][130:200, 0].isnan().all()) and bool(b["out"][b["off"][2] + 230:b["off"][3]].isnan().all())
    same = b["out"] == clean["out"]
    assert bool(same[:130].all()) and bool(same[130:200, 1].all()) and bool(same[200:b["off"][2] + 230].all())


@pytest.mark.parametrize("dtype", BOTH)
def test_rows_whose_scores_are_all_minus_infinity(G, dtype):
    b = make(dtype, 1, [90], [4], seed=12)
    b["q"].zero_()
    b["q"][:, :, 5] = -math.inf
    b["k"][:90, :, 5] = 1.0
    call(G, b)
    assert bool(b["out"][:4].isnan().all()) and bool((b["out"][4:] == 5.0).all())


@pytest.mark.parametrize("dtype", BOTH)
def test_offsets_at_the_ends_of_their_range(G, dtype):
    """Rows and keys that the offsets put behind the arrays count for the positions although they are not there."""
    b = make(dtype, 2, [300], [40], seed=13, tail=0)
    call(G, b)
    want = b["out"].clone()
    out = torch.full_like(want, 5.0)
    call(G, dict(b, off=[0, 60], koff=[0, 320]), out=out, max_new=60)
    assert torch.equal(out, want)
    out.fill_(5.0)
    call(G, dict(b, off=[-5, 10], koff=[-3, 270]), out=out)
    assert torch.equal(out[:10], want[:10]) and bool((out[10:] == 5.0).all())
    out.fill_(5.0)
    call(G, dict(b, off=[30, 20], koff=[0, 300]), out=out)
    assert bool((out == 5.0).all())


def test_streams_and_graphs(G):
    b = make(torch.bfloat16, 4, [500, 90], [200, 90], seed=14)
    call(G, b)
    want = b["out"].clone()
    off, koff = dev(b["off"]), dev(b["koff"])

    def step():
        G.expanded_attend(b["q"], b["k"], b["r"], b["v"], off, koff, 200, out=b["out"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b["out"].fill_(5.0)
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    assert torch.equal(b["out"], want)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g in graphs:
        with torch.cuda.graph(g):
            step()
    for g in graphs:
        b["out"].fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(b["out"], want)


@pytest.mark.parametrize("polls", [1, 3])
@pytest.mark.parametrize("keys,new,heads", [([3000] * 4, [300] * 4, 8), ([600] * 3, [600] * 3, 40)])
def test_a_wait_that_runs_out_is_reported(G, keys, new, heads, polls):
    b = make(torch.bfloat16, heads, keys, new, seed=15)
    call(G, b)
    want = b["out"].clone()
    seen, big = 0, torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    for _ in range(4):
        status = dev([0])
        b["out"].fill_(5.0)
        big.fill_(1)
        call(G, b, status=status, wait_polls=polls)
        got = int(status.item())
        assert got in (0, G.S_TIMEOUT)
        seen += got != 0
        assert got or torch.equal(b["out"], want)
        assert bool((b["out"][b["off"][-1]:] == 5.0).all())
    if polls == 1:
        assert seen > 0
    call(G, b)
    assert torch.equal(b["out"], want)


def test_expanded_and_absorbed_forms_agree(G):
    """A prompt whose first part was found in the store: its rows read back and expanded, against the absorbed form over the cache."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(99)
    H, n, found, block = 4, 300, 200, 16
    lay = G.KVLayout(1, 576, block, G.KV_LATENT_BF16)
    cache = G.PagedKV(1, 32, lay.chunk_bytes)
    tables = torch.randperm(32, generator=gen, device="cuda").int()[None, :24].contiguous()
    _, slots, _ = G.map_slots(dev([n]), None, tables, block, n)
    c, r = rows(gen, (n, 512), torch.bfloat16, 0.5), rows(gen, (n, 64), torch.bfloat16)
    G.latent_write(lay, cache, 0, c, r, slots)
    wk, wv = (torch.randn(H, 128, 512, generator=gen, device="cuda") * 512 ** -0.5 for _ in range(2))
    new = n - found
    qn, qr = torch.randn(new, H, 128, generator=gen, device="cuda"), rows(gen, (new, H, 64), torch.bfloat16)
    c2, r2 = G.latent_read(lay, cache, 0, slots)
    assert torch.equal(c2, c) and torch.equal(r2, r)
    kv = torch.einsum("nc,hdc->nhd", c2.float(), torch.cat([wk, wv], 1)).bfloat16()
    q = torch.cat([qn.bfloat16(), qr], 2)
    expanded = G.expanded_attend(q, kv[:, :, :128], r2, kv[:, :, 128:], dev([0, new]), dev([0, n]), new)
    ql = torch.einsum("ihd,hdc->ihc", qn, wk).bfloat16()
    absorbed = G.latent_attend(lay, cache, 0, ql, qr, dev([0, new]), dev([n]), tables, new, 192 ** -0.5)
    absorbed = torch.einsum("ihc,hdc->ihd", absorbed.float(), wv)
    assert float((expanded.float() - absorbed).abs().max()) < 0.06          # intermediate values are rounded to bf16 in different places
