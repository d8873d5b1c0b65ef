"""The operators around the paged cache refuse bad arguments on the host, before anything touches a device."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest
import torch

from paper_2607_22648_b200 import build
from tests import operators_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, E_INVAL, E_NOMEM, E_LIMIT = 0, -1, -3, -4


@pytest.fixture(scope="module")
def G():
    build.build()
    from paper_2607_22648_b200 import binding
    return binding


A = 1 << 20      # an address that is never followed


def test_structs_match_the_c_layout(G):
    prog = r'''
#include <stdio.h>
#include <stddef.h>
#include "ptstore.h"
int main(void) {
  printf("%zu %zu %zu %zu %zu %zu %zu\n", sizeof(ptstore_kv_cache_t), offsetof(ptstore_kv_cache_t, format), offsetof(ptstore_kv_cache_t, v_scale),
         sizeof(ptstore_attend_t), offsetof(ptstore_attend_t, out), offsetof(ptstore_attend_t, requests), offsetof(ptstore_attend_t, scale));
  return 0;
}
'''
    with tempfile.TemporaryDirectory() as d:
        path, exe = os.path.join(d, "t.c"), os.path.join(d, "t")
        open(path, "w").write(prog)
        subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-o", exe, path])
        got = [int(x) for x in subprocess.check_output([exe]).split()]
    assert got == [C.sizeof(G.KvCache), G.KvCache.format.offset, G.KvCache.v_scale.offset, C.sizeof(G.Attend), G.Attend.out.offset,
                   G.Attend.requests.offset, G.Attend.scale.offset]


def test_chunk_bytes(G):
    f = G.lib.ptstore_kv_chunk_bytes
    assert f(G.KV_BF16, 16, 8, 128) == 32768 and f(G.KV_FP16, 1, 1, 64) == 128
    assert f(G.KV_PACKED, 16, 8, 128) == 9216 and f(G.KV_PACKED, 48, 1, 64) == 48 * 36
    for bad in ((3, 16, 8, 128), (G.KV_PACKED, 8, 8, 128), (G.KV_PACKED, 24, 8, 128), (G.KV_BF16, 0, 8, 128), (G.KV_BF16, 16, 0, 128),
                (G.KV_BF16, 16, 8, 96), (G.KV_BF16, 16, 8, 256)):
        assert f(*bad) == 0
    with pytest.raises(G.PTStoreError):
        G.KVLayout(8, 96, 16)
    lay = G.KVLayout(8, 128, 16, G.KV_PACKED)
    a = lay.store_args()
    assert 16 * 8 * a["dim"] * a["elem_bytes"] == lay.chunk_bytes


def test_assign_blocks_refuses(G):
    f = G.lib.ptstore_assign_blocks
    good = [A, A, 4, 16, A, 8, A, 100, A, A, A, None, None]

    def call(**kw):
        names = ["lengths", "held", "R", "block", "tables", "width", "ids", "cap", "count", "held_out", "count_out", "status", "stream"]
        return f(*[kw.get(n, g) for n, g in zip(names, good)])
    for kw in ({"R": -1}, {"block": 0}, {"width": 0}, {"cap": -1}, {"lengths": None}, {"tables": None}, {"ids": None}, {"count": None},
               {"held_out": None}, {"count_out": None}):
        assert call(**kw) == E_INVAL, kw
    assert call(R=(1 << 30) + 1) == E_LIMIT
    assert call(R=16384, width=1 << 20) == E_LIMIT


def test_map_slots_refuses(G):
    f = G.lib.ptstore_map_slots
    good = [A, A, 1, 0, 4, A, 8, 16, 100, A, A, A, None, None]

    def call(**kw):
        names = ["lengths", "done", "unit", "min_new", "R", "tables", "width", "block", "tokens", "offsets", "slots", "positions", "status", "stream"]
        return f(*[kw.get(n, g) for n, g in zip(names, good)])
    for kw in ({"R": -1}, {"block": 0}, {"width": 0}, {"tokens": -1}, {"tokens": 1 << 31}, {"unit": 0}, {"min_new": -1}, {"lengths": None},
               {"tables": None}, {"offsets": None}, {"slots": None}):
        assert call(**kw) == E_INVAL, kw
    assert call(R=(1 << 30) + 1) == E_LIMIT


def cache(G, **kw):
    d = dict(base=A, kv=9216 * 10, bs=9216, nb=10, block=16, heads=8, dim=128, fmt=G.KV_PACKED, ks=0.5, vs=0.25)
    d.update(kw)
    return G.KvCache(d["base"], d["kv"], d["bs"], d["nb"], d["block"], d["heads"], d["dim"], d["fmt"], 0, d["ks"], d["vs"])


BAD_CACHES = [{"base": None}, {"base": A + 8}, {"kv": 9216 * 10 + 8}, {"bs": 9216 + 8}, {"bs": 9200}, {"nb": 0}, {"block": 8}, {"block": 0},
              {"heads": 0}, {"dim": 96}, {"fmt": 3}, {"ks": 0.0}, {"ks": -1.0}, {"ks": 0.75}, {"vs": float("nan")}, {"vs": float("inf")}, {"vs": 2.0 ** -65},
              {"ks": 2.0 ** 65}]


def test_kv_write_and_read_refuse(G):
    def write(c, k=A, ks=(1024, 128), v=A, vs=(1024, 128), n=4, dtype=0, slots=A):
        return G.lib.ptstore_kv_write(k, ks[0], ks[1], v, vs[0], vs[1], n, dtype, slots, C.byref(c), None, None)

    def read(c, k=A, ks=(1024, 128), v=A, vs=(1024, 128), n=4, dtype=0, slots=A):
        return G.lib.ptstore_kv_read(C.byref(c), slots, n, dtype, k, ks[0], ks[1], v, vs[0], vs[1], None, None)
    for f in (write, read):
        for kw in BAD_CACHES:
            assert f(cache(G, **kw)) == E_INVAL, kw
        for kw in ({"k": None}, {"v": None}, {"slots": None}, {"k": A + 8}, {"v": A + 2}, {"ks": (1020, 128)}, {"vs": (1024, 4)}, {"n": -1}, {"dtype": 2}):
            assert f(cache(G), **kw) == E_INVAL, kw
        assert f(cache(G, fmt=G.KV_FP16, bs=32768), dtype=G.KV_BF16) == E_INVAL          # a 16-bit cache keeps its own type
        assert f(cache(G), n=1 << 60) == E_LIMIT
        assert f(cache(G), n=0, k=None, v=None, slots=None) == OK                          # nothing to do
    assert G.lib.ptstore_kv_write(A, 8, 8, A, 8, 8, 1, 0, A, None, None, None) == E_INVAL


def attend_args(G, **kw):
    d = dict(size=C.sizeof(G.Attend), dtype=0, q=A, qt=4096, qh=128, out=A, ot=4096, oh=128, off=A, lens=A, tabs=A, R=2, width=8, heads=32, tokens=10,
             max_new=5, scale=0.1)
    d.update(kw)
    return G.Attend(d["size"], d["dtype"], d["q"], d["qt"], d["qh"], d["out"], d["ot"], d["oh"], d["off"], d["lens"], d["tabs"], d["R"], d["width"],
                    d["heads"], d["tokens"], d["max_new"], d["scale"])


def test_attend_refuses(G):
    need = G.lib.ptstore_attend_workspace_bytes(128)
    assert need > 0 and G.lib.ptstore_attend_workspace_bytes(96) == 0

    def call(c=None, work=A, size=need, **kw):
        return G.lib.ptstore_attend(C.byref(attend_args(G, **kw)), C.byref(c or cache(G)), work, size, None, None)
    for kw in BAD_CACHES:
        assert call(cache(G, **kw)) == E_INVAL, kw
    for kw in ({"size": 8}, {"dtype": 2}, {"q": None}, {"q": A + 8}, {"qt": 4092}, {"qh": 4}, {"out": None}, {"out": A + 4}, {"ot": 1}, {"off": None},
               {"lens": None}, {"tabs": None}, {"R": -1}, {"width": 0}, {"heads": 0}, {"heads": 12}, {"tokens": -1}, {"max_new": -1},
               {"scale": float("nan")}, {"scale": float("inf")}):
        if kw == {"size": 8}:
            a = attend_args(G, size=8)
            assert G.lib.ptstore_attend(C.byref(a), C.byref(cache(G)), A, need, None, None) == E_INVAL
            continue
        assert call(**kw) == E_INVAL, kw
    assert call(cache(G, fmt=G.KV_FP16, bs=32768)) == E_INVAL
    assert call(work=None) == E_INVAL and call(work=A + 16) == E_INVAL
    assert call(size=need - 1) == E_NOMEM
    assert call(R=(1 << 20) + 1) == E_LIMIT and call(tokens=1 << 27) == E_LIMIT
    assert call(width=(1 << 26) + 1) == E_LIMIT                                               # more than 2^30 tokens in a row of the table
    assert call(R=0) == OK and call(tokens=0) == OK and call(max_new=0) == OK
    assert G.lib.ptstore_attend(None, C.byref(cache(G)), A, need, None, None) == E_INVAL


def test_reference_bookkeeping_by_hand():
    """Two rows shrink or end, one grows, one is denied: the worked example of the definitions."""
    tables = [[5, 6, 7, -1], [8, 9, -1, -1], [1, -1, -1, -1], [-1] * 4]
    t, held, stack, count, denied = ref.assign_blocks([17, 0, 64, 33], [3, 2, 1, 0], tables, [3, 4, -1, -1, -1, -1], 2, 16)
    # pushes 7 (row 0 keeps two blocks), 8, 9 -> stack 3 4 7 8 9; row 2 pops 9 8 7; row 3 wants three of the two left
    assert stack[:5] == [3, 4, 7, 8, 9] and t[2] == [1, 9, 8, 7] and held == [2, 0, 4, 0] and count == 2 and denied
    off, slots, pos = ref.map_slots([17, 0, 64, 0], [1, 0, 4, 0], t, 16, unit=16, min_new=1)
    assert off == [0, 1, 1, 2, 2] and pos == [16, 63] and slots == [6 * 16, 7 * 16 + 15]


def test_reference_e4m3_against_torch():
    x = torch.cat([torch.linspace(0, 500, 20001, dtype=torch.float64), torch.linspace(0, 0.1, 20001, dtype=torch.float64)])
    want = x.clamp(max=448).float().to(torch.float8_e4m3fn).double()
    assert torch.equal(ref.e4m3_nearest(x.float().double()), want)


def test_attend_takes_both_sizes_of_its_struct(G):
    """A caller built without the fields behind `scale` passes the first size; any other size is refused."""
    need = G.lib.ptstore_attend_workspace_bytes(128)
    assert G.Attend.wait_polls.offset == 104 and C.sizeof(G.Attend) == 112
    for size, want in ((104, OK), (112, OK), (0, E_INVAL), (100, E_INVAL), (108, E_INVAL), (120, E_INVAL)):
        a = attend_args(G, size=size, R=0)
        assert G.lib.ptstore_attend(C.byref(a), C.byref(cache(G)), A, need, None, None) == want, size


def test_attend_refuses_a_scale_that_overflows_with_the_tensor_scale(G):
    """Scores are multiplied by scale * log2 e (and K's tensor scale and the 4-bit values' factor of 2^8): that has to be finite too."""
    need = G.lib.ptstore_attend_workspace_bytes(128)

    def call(c, **kw):
        return G.lib.ptstore_attend(C.byref(attend_args(G, **kw)), C.byref(c), A, need, None, None)
    plain = dict(fmt=G.KV_BF16, bs=32768, kv=327680)
    for scale in (3e38, -3e38):
        assert call(cache(G, **plain), scale=scale) == E_INVAL
        assert call(cache(G, ks=2.0 ** 20), scale=scale / 2.0 ** 24) == E_INVAL
    assert call(cache(G, ks=2.0 ** 64), scale=2.0 ** 56) == E_INVAL
    assert call(cache(G, ks=2.0 ** 64), scale=0.1, R=0) == OK and call(cache(G, **plain), scale=3e38, R=0) == E_INVAL
