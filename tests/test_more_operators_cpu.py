"""The operators over latent vectors and those of eviction refuse bad arguments on the host, before anything touches a device."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest

from tests.test_operators_cpu import A, E_INVAL, E_LIMIT, E_NOMEM, OK, ROOT, G, cache  # noqa: F401  (G: the fixture)


def latent_cache(G, **kw):
    d = dict(kv=0, bs=16 * 576 * 2, heads=1, dim=576, fmt=G.KV_LATENT_BF16)
    d.update(kw)
    return cache(G, **d)


def bad_latent_caches(G):
    return [{"base": None}, {"base": A + 8}, {"bs": 16 * 576 * 2 + 8}, {"bs": 16 * 576 * 2 - 16}, {"nb": 0}, {"block": 0}, {"block": 12}, {"block": 1 << 17}, {"heads": 2}, {"dim": 512},
            {"dim": 128}, {"fmt": 6}, {"fmt": G.KV_BF16, "dim": 128, "heads": 8, "bs": 32768}]


def test_structs_match_the_c_layout(G):  # noqa: F811
    want, lines = [], []
    for name, struct, fields in (("ptstore_latent_attend_t", G.LatentAttend, ("out", "lse", "requests", "scale")), ("ptstore_expanded_attend_t", G.ExpandedAttend, ("v", "out", "keys", "wait_polls")),
                                 ("ptstore_attend_weights_t", G.AttendWeights, ("lse", "weights", "width", "accumulate", "wait_polls"))):
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(C.sizeof(struct))
        for f in fields:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, f))
            want.append(getattr(struct, f).offset)
    prog = '#include <stdio.h>\n#include <stddef.h>\n#include "ptstore.h"\nint main(void) { %s return 0; }\n' % " ".join(lines)
    with tempfile.TemporaryDirectory() as d:
        path, exe = os.path.join(d, "t.c"), os.path.join(d, "t")
        open(path, "w").write(prog)
        subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-o", exe, path])
        assert [int(x) for x in subprocess.check_output([exe]).split()] == want


def test_latent_chunk_and_workspace_bytes(G):  # noqa: F811
    f = G.lib.ptstore_kv_chunk_bytes
    assert f(G.KV_LATENT_BF16, 16, 1, 576) == 16 * 1152 and f(G.KV_LATENT_FP16, 8, 1, 320) == 8 * 640
    for bad in ((G.KV_LATENT_BF16, 16, 2, 576), (G.KV_LATENT_BF16, 12, 1, 576), (G.KV_LATENT_BF16, 16, 1, 512), (6, 16, 1, 576), (G.KV_BF16, 16, 1, 576)):
        assert f(*bad) == 0
    assert G.lib.ptstore_latent_workspace_bytes(576) > G.lib.ptstore_latent_workspace_bytes(320) > 0 and G.lib.ptstore_latent_workspace_bytes(512) == 0
    with pytest.raises(G.PTStoreError):
        G.KVLayout(2, 576, 16, G.KV_LATENT_BF16)


def test_latent_rows_refuse(G):  # noqa: F811
    def write(c, l=A, ls=512, r=A, rs=64, n=4, slots=A):
        return G.lib.ptstore_latent_write(l, ls, r, rs, n, slots, C.byref(c), None, None)

    def read(c, l=A, ls=512, r=A, rs=64, n=4, slots=A):
        return G.lib.ptstore_latent_read(C.byref(c), slots, n, l, ls, r, rs, None, None)
    for f in (write, read):
        for kw in bad_latent_caches(G):
            assert f(latent_cache(G, **kw)) == E_INVAL, kw
        for kw in ({"l": None}, {"r": None}, {"slots": None}, {"l": A + 8}, {"r": A + 2}, {"ls": 516}, {"rs": 4}, {"n": -1}):
            assert f(latent_cache(G), **kw) == E_INVAL, kw
        assert f(latent_cache(G), n=1 << 60) == E_LIMIT
        assert f(latent_cache(G), n=0, l=None, r=None, slots=None) == OK
    # K and V rows do not go into a latent cache
    assert G.lib.ptstore_kv_write(A, 576, 576, A, 576, 576, 1, 0, A, C.byref(latent_cache(G)), None, None) == E_INVAL
    assert G.lib.ptstore_kv_read(C.byref(latent_cache(G)), A, 1, 0, A, 576, 576, A, 576, 576, None, None) == E_INVAL


def test_latent_attend_refuses(G):  # noqa: F811
    need = G.lib.ptstore_latent_workspace_bytes(576)
    good = dict(struct_size=C.sizeof(G.LatentAttend), q_latent=A, q_latent_token_stride=16 * 512, q_latent_head_stride=512, q_rope=A, q_rope_token_stride=16 * 64, q_rope_head_stride=64,
                out=A, out_token_stride=16 * 512, out_head_stride=512, token_offsets=A, lengths=A, block_tables=A, requests=2, max_blocks=8, num_heads=16, tokens=10, max_new=5, scale=0.1)

    def call(c=None, work=A, size=need, **kw):
        return G.lib.ptstore_latent_attend(C.byref(G.LatentAttend(**dict(good, **kw))), C.byref(c or latent_cache(G)), work, size, None, None)
    for kw in bad_latent_caches(G):
        assert call(latent_cache(G, **kw)) == E_INVAL, kw
    for kw in ({"struct_size": 8}, {"q_latent": None}, {"q_latent": A + 8}, {"q_latent_token_stride": 4}, {"q_latent_head_stride": 12}, {"q_rope": None}, {"q_rope": A + 4},
               {"q_rope_head_stride": 4}, {"out": None}, {"out": A + 2}, {"out_token_stride": 1}, {"token_offsets": None}, {"lengths": None}, {"block_tables": None}, {"requests": -1},
               {"max_blocks": 0}, {"num_heads": 0}, {"num_heads": 65536}, {"tokens": -1}, {"max_new": -1}, {"scale": float("nan")}, {"scale": 3e38}, {"work": None}, {"work": A + 16}):
        assert call(**kw) == E_INVAL, kw
    assert call(size=need - 1) == E_NOMEM
    assert call(requests=(1 << 20) + 1) == E_LIMIT and call(tokens=1 << 28) == E_LIMIT and call(max_blocks=(1 << 26) + 1) == E_LIMIT
    assert call(requests=0) == OK and call(tokens=0) == OK and call(max_new=0) == OK
    # K and V attention does not take a latent cache
    a = G.Attend(C.sizeof(G.Attend), 0, A, 4096, 128, A, 4096, 128, A, A, A, 2, 8, 32, 10, 5, 0.1)
    assert G.lib.ptstore_attend(C.byref(a), C.byref(latent_cache(G)), A, 1 << 30, None, None) == E_INVAL
    assert G.lib.ptstore_attend_lse(C.byref(a), C.byref(latent_cache(G)), A, 1 << 30, A, None, None) == E_INVAL


def test_expanded_attend_refuses(G):  # noqa: F811
    good = dict(struct_size=C.sizeof(G.ExpandedAttend), dtype=0, q=A, q_token_stride=16 * 192, q_head_stride=192, k=A, k_token_stride=16 * 256, k_head_stride=256, k_rope=A,
                k_rope_token_stride=64, v=A + 256, v_token_stride=16 * 256, v_head_stride=256, out=A, out_token_stride=16 * 128, out_head_stride=128, token_offsets=A, key_offsets=A,
                requests=2, heads=16, tokens=10, keys=20, max_new=5, scale=0.1)

    def call(**kw):
        return G.lib.ptstore_expanded_attend(C.byref(G.ExpandedAttend(**dict(good, **kw))), None, None)
    for kw in ({"struct_size": 8}, {"dtype": 2}, {"q": None}, {"q": A + 8}, {"q_token_stride": 4}, {"q_token_stride": 0}, {"q_head_stride": -192}, {"k": None}, {"k": A + 2},
               {"k_token_stride": -4096}, {"k_head_stride": 4}, {"k_rope": None}, {"k_rope_token_stride": 12}, {"v": None}, {"v": A + 4}, {"v_token_stride": 1 << 38}, {"out": None},
               {"out_head_stride": 4}, {"token_offsets": None}, {"key_offsets": None}, {"requests": -1}, {"heads": 0}, {"heads": 65536}, {"tokens": -1}, {"keys": -1}, {"max_new": -1},
               {"scale": float("inf")}, {"scale": -3e38}):
        assert call(**kw) == E_INVAL, kw
    assert call(requests=(1 << 20) + 1) == E_LIMIT and call(keys=(1 << 29) + 1) == E_LIMIT and call(tokens=(1 << 29) + 1) == E_LIMIT
    assert call(requests=0) == OK and call(tokens=0) == OK and call(max_new=0) == OK
    assert G.lib.ptstore_expanded_attend(None, None, None) == E_INVAL


def test_attend_weights_refuses(G):  # noqa: F811
    good = dict(struct_size=C.sizeof(G.AttendWeights), dtype=0, q=A, q_token_stride=4096, q_head_stride=128, lse=A, token_offsets=A, lengths=A, block_tables=A, requests=2, max_blocks=8,
                num_heads=32, tokens=10, weights=A, weights_request_stride=1024, weights_head_stride=128, width=128, max_new=5, accumulate=1, scale=0.1)

    def call(c=None, **kw):
        return G.lib.ptstore_attend_weights(C.byref(G.AttendWeights(**dict(good, **kw))), C.byref(c or cache(G)), None, None)
    for kw in ({"base": None}, {"nb": 0}, {"block": 8}, {"dim": 96}, {"fmt": 3}, {"ks": 0.75}):
        assert call(cache(G, **kw)) == E_INVAL, kw
    for kw in ({"struct_size": 8}, {"dtype": 2}, {"q": None}, {"q": A + 8}, {"q_token_stride": 4}, {"q_head_stride": 4}, {"lse": None}, {"token_offsets": None}, {"lengths": None},
               {"block_tables": None}, {"requests": -1}, {"max_blocks": 0}, {"num_heads": 0}, {"num_heads": 12}, {"tokens": -1}, {"weights": None}, {"width": -1}, {"accumulate": 2},
               {"scale": float("nan")}, {"scale": 3e38}):
        assert call(**kw) == E_INVAL, kw
    assert call(cache(G, fmt=G.KV_FP16, bs=32768)) == E_INVAL and call(latent_cache(G, fmt=G.KV_LATENT_FP16)) == E_INVAL                # the cache's own type
    assert call(requests=(1 << 20) + 1) == E_LIMIT and call(tokens=1 << 27) == E_LIMIT and call(max_blocks=(1 << 26) + 1) == E_LIMIT and call(width=(1 << 30) + 1) == E_LIMIT
    assert call(requests=0) == OK and call(width=0) == OK and call(tokens=0) == OK


def test_select_tokens_refuses(G):  # noqa: F811
    names = ["weights", "ws", "wh", "lengths", "R", "heads", "width", "budget", "first", "recent", "kept", "lengths_out", "out", "os", "oh", "status", "stream"]
    good = [A, 1024, 128, A, 4, 8, 128, 64, 4, 16, A, A + 4096, A, 1024, 128, None, None]

    def call(**kw):
        return G.lib.ptstore_select_tokens(*[kw.get(n, g) for n, g in zip(names, good)])
    for kw in ({"R": -1}, {"heads": 0}, {"width": 0}, {"budget": 0}, {"budget": 129}, {"first": -1}, {"recent": -1}, {"first": 65}, {"recent": 61}, {"weights": None}, {"lengths": None},
               {"kept": None}, {"lengths_out": None}, {"lengths_out": A}, {"out": None}, {"os": 1032}, {"oh": 64}):
        assert call(**kw) == E_INVAL, kw
    assert call(width=(1 << 30) + 1) == E_LIMIT and call(R=1 << 30, heads=2) == E_LIMIT
    assert call(R=0) == OK


def test_kv_compact_refuses(G):  # noqa: F811
    def call(c=None, kept=A, lengths=A, R=2, width=64, frm=A, fb=8, to=A + 64, tb=4):
        return G.lib.ptstore_kv_compact(C.byref(c or cache(G)), kept, lengths, R, width, frm, fb, to, tb, None, None)
    for kw in ({"base": None}, {"nb": 0}, {"block": 8}, {"dim": 96}, {"fmt": 3}):
        assert call(cache(G, **kw)) == E_INVAL, kw
    for kw in ({"kept": None}, {"lengths": None}, {"R": -1}, {"width": -1}, {"frm": None}, {"fb": 0}, {"to": None}, {"tb": 0}, {"to": A}):
        assert call(**kw) == E_INVAL, kw                     # ({"to": A}: in place with another number of blocks)
    assert call(width=(1 << 30) + 1) == E_LIMIT and call(R=(1 << 20) + 1) == E_LIMIT
    assert call(R=0) == OK and call(width=0) == OK


def test_latent_attend_refuses_q_as_output_with_other_strides(G):  # noqa: F811
    need = G.lib.ptstore_latent_workspace_bytes(576)
    same = dict(struct_size=C.sizeof(G.LatentAttend), q_latent=A, q_latent_token_stride=16 * 512, q_latent_head_stride=512, q_rope=A + 4096, q_rope_token_stride=16 * 64, q_rope_head_stride=64,
                out=A, out_token_stride=16 * 512, out_head_stride=512, token_offsets=A, lengths=A, block_tables=A, requests=2, max_blocks=8, num_heads=16, tokens=10, max_new=5, scale=0.1)

    def call(size=need - 1, **kw):                           # (a workspace that is too small is found later)
        return G.lib.ptstore_latent_attend(C.byref(G.LatentAttend(**dict(same, **kw))), C.byref(latent_cache(G)), A, size, None, None)
    assert call() == E_NOMEM
    for kw in ({"out_token_stride": 32 * 512}, {"out_head_stride": 1024}, {"q_latent_token_stride": 16 * 576}, {"tokens": 1, "out_head_stride": 1024}, {"num_heads": 1, "out_token_stride": 1024}):
        assert call(**kw) == E_INVAL, kw
    # the stride of an axis of one does not matter, and other memory may have any strides
    for kw in ({"tokens": 1, "out_token_stride": 8}, {"num_heads": 1, "out_head_stride": 8}, {"out": A + (1 << 20), "out_token_stride": 32 * 512}):
        assert call(**kw) == E_NOMEM, kw


def test_a_latent_cache_has_no_stride_from_k_to_v(G):  # noqa: F811
    """kv_stride_bytes is not used, so it may hold anything; of K and V it has to be a multiple of 16 as before."""
    def write(c):
        return G.lib.ptstore_latent_write(A, 512, A, 64, 0, A, C.byref(c), None, None)
    assert write(latent_cache(G, kv=8)) == OK and write(latent_cache(G, kv=(1 << 64) - 1)) == OK
    assert G.lib.ptstore_kv_write(A, 4096, 128, A, 4096, 128, 0, 0, A, C.byref(cache(G, kv=8)), None, None) == E_INVAL
