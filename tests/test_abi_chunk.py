"""Refusals of the chunk operators, before any launch (CPU only)."""
import ctypes

import numpy as np
import pytest

from paper_2608_02691_amd import int2kv as K

GOOD = K._Cache(16, 4, 2, 16, 128, 32)
AX = bytes(64)


def _rope(**kw):
    a = dict(q=1 << 20, hq=4, qs=512, k=2 << 20, hk=2, ks=256, pos=16, axes=1, axis=AX, n=8, cs=16, max_pos=8, qo=3 << 20, qos=512,
             ko=4 << 20, kos=256)
    a.update(kw)
    st = K.load_library().int2kv_rope_axes(a["q"], a["hq"], a["qs"], a["k"], a["hk"], a["ks"], a["pos"], a["axes"], a["axis"],
                                           a["n"], a["cs"], a["max_pos"], a["qo"], a["qos"], a["ko"], a["kos"], None)
    return st, K.load_library().int2kv_last_error()


@pytest.mark.parametrize("kw,word", [
    (dict(n=-1), b"num_tokens"), (dict(hq=-1), b"head"), (dict(axes=0), b"num_axes"), (dict(axes=9), b"num_axes"),
    (dict(axis=None), b"NULL"), (dict(axis=bytes([1] * 64)), b"pair_axis"), (dict(pos=None), b"NULL"), (dict(cs=None), b"NULL"),
    (dict(q=None), b"NULL"), (dict(qo=None), b"NULL"), (dict(k=None), b"NULL"), (dict(max_pos=0), b"max_pos"),
    (dict(qs=511), b"stride"), (dict(qs=516), b"stride"), (dict(kos=128), b"stride"), (dict(qs=1 << 40), b"stride"),
    (dict(q=(1 << 20) + 8), b"aligned"), (dict(cs=8), b"aligned"), (dict(ko=(4 << 20) + 2), b"aligned"),
    (dict(qo=(1 << 20) + 1024), b"overlap"), (dict(qo=1 << 20, qos=1024), b"overlap"), (dict(ko=3 << 20), b"overlap"),
    (dict(ko=1 << 20), b"overlap"), (dict(qo=2 << 20), b"overlap"),
])
def test_rope_axes_refusals(kw, word):
    st, msg = _rope(**kw)
    assert st == K.INT2KV_EINVAL and word in msg, msg


def test_rope_axes_with_nothing_to_do():
    assert _rope(n=0)[0] == K.INT2KV_OK
    assert _rope(hq=0, hk=0)[0] == K.INT2KV_OK
    st, msg = _rope(n=1 << 27)  # more than a launch holds
    assert st == K.INT2KV_EUNSUPPORTED and b"num_tokens" in msg


def test_axis_tables():
    assert K.rope_axis_table([64]) == bytes(64)
    assert K.rope_axis_table([16, 24, 24]) == bytes([0] * 16 + [1] * 24 + [2] * 24)
    t = K.rope_axis_table([16, 24, 24], interleaved=True)
    assert t[:6] == bytes([0, 1, 2, 0, 1, 2]) and [t.count(bytes([a])) for a in range(3)] == [16, 24, 24]
    for bad in ([63], [60, 5], [-1, 65]):
        with pytest.raises(ValueError):
            K.rope_axis_table(bad)


def _read(cache=GOOD, slots=16, n=4, R_k=None, R_v=None, mu=None, fmt=0, k=1 << 20, v=2 << 20):
    st = K.load_library().int2kv_read_rows(ctypes.byref(cache) if cache else None, slots, n, R_k, R_v, mu, fmt, k, v, None)
    return st, K.load_library().int2kv_last_error()


@pytest.mark.parametrize("kw,word", [
    (dict(cache=None), b"cache"), (dict(n=-1), b"num_tokens"), (dict(fmt=2), b"row_format"), (dict(mu=16), b"mu"),
    (dict(slots=None), b"NULL"), (dict(k=None, v=None), b"NULL"), (dict(R_k=8), b"aligned"), (dict(v=(2 << 20) + 8), b"aligned"),
    (dict(v=(1 << 20) + 512), b"overlap"),
])
def test_read_rows_refusals(kw, word):
    st, msg = _read(**kw)
    assert st == K.INT2KV_EINVAL and word in msg, msg


def test_read_rows_of_nothing_and_bad_caches():
    assert _read(n=0)[0] == K.INT2KV_OK
    st, msg = _read(n=1 << 27)  # two heads: more than a launch holds
    assert st == K.INT2KV_EUNSUPPORTED and b"num_tokens" in msg
    assert _read(cache=K._Cache(16, 4, 2, 16, 128, 64))[0] == K.INT2KV_EUNSUPPORTED
    assert _read(cache=K._Cache(16, 4, 2, 8, 128, 32))[0] == K.INT2KV_EUNSUPPORTED


def _chunk(cache=GOOD, **kw):
    a = dict(q=1 << 20, qs=512, starts=16, B=2, total=8, max_q=8, hq=4, table=16, mb=4, lens=16, max_ctx=64, R_k=16, R_v=16,
             k=2 << 20, ks=256, v=3 << 20, vs=256, mu=16, out=4 << 20, ws=1 << 24, wb=1 << 30)
    a.update(kw)
    st = K.load_library().int2kv_chunk_attention(
        ctypes.byref(cache) if cache else None, a["q"], a["qs"], a["starts"], a["B"], a["total"], a["max_q"], a["hq"], a["table"],
        a["mb"], a["lens"], a["max_ctx"], a["R_k"], a["R_v"], a["k"], a["ks"], a["v"], a["vs"], a["mu"], a["out"], a["ws"], a["wb"],
        None)
    return st, K.load_library().int2kv_last_error()


@pytest.mark.parametrize("kw,word", [
    (dict(cache=None), b"cache"), (dict(B=0), b"batch"), (dict(hq=3), b"num_q_heads"), (dict(hq=0), b"num_q_heads"),
    (dict(total=-1), b"total_q"), (dict(max_q=-1), b"total_q"), (dict(max_ctx=-1), b"max_ctx"), (dict(mb=0), b"max_blocks"),
    (dict(q=None), b"NULL"), (dict(starts=None), b"NULL"), (dict(table=None), b"NULL"), (dict(lens=None), b"NULL"),
    (dict(R_k=None), b"NULL"), (dict(R_v=None), b"NULL"), (dict(out=None), b"NULL"), (dict(k=None), b"together"),
    (dict(v=None), b"together"), (dict(mu=None), b"together"), (dict(qs=504), b"stride"), (dict(qs=516), b"stride"),
    (dict(ks=255), b"stride"), (dict(vs=0), b"stride"), (dict(q=(1 << 20) + 8), b"aligned"), (dict(R_v=24), b"aligned"),
    (dict(v=(3 << 20) + 4), b"aligned"), (dict(out=1 << 20), b"overlap"), (dict(out=(2 << 20) + 1024), b"overlap"),
    (dict(out=(3 << 20) - 1024), b"overlap"), (dict(ws=(1 << 24) + 16), b"workspace"),
])
def test_chunk_attention_refusals(kw, word):
    st, msg = _chunk(**kw)
    assert st == K.INT2KV_EINVAL and word in msg, msg


def test_chunk_attention_workspace():
    lib = K.load_library()
    need = K.int2kv_chunk_attention_workspace_bytes(2, 4, 2, 8, 8, 64)
    assert need > 0
    st, msg = _chunk(wb=need - 1)
    assert st == K.INT2KV_EWORKSPACE and b"workspace" in msg
    assert _chunk(ws=None)[0] == K.INT2KV_EWORKSPACE
    assert _chunk(total=1 << 30, max_q=1)[0] == K.INT2KV_EUNSUPPORTED
    # 2^23 sequences of a token: as many work-groups a KV head as a launch of two holds, and one more
    assert _chunk(total=(1 << 23) - 1, B=(1 << 23) - 1, max_q=1, q=1 << 40, k=2 << 40, v=3 << 40, out=4 << 40, wb=0)[0] == K.INT2KV_EWORKSPACE
    assert _chunk(total=1 << 23, B=1 << 23, max_q=1, q=1 << 40, k=2 << 40, v=3 << 40, out=4 << 40)[0] == K.INT2KV_EUNSUPPORTED
    assert _chunk(max_q=0)[0] == K.INT2KV_OK and _chunk(total=0)[0] == K.INT2KV_OK
    for bad in ((0, 4, 2, 8, 8, 64), (2, 3, 2, 8, 8, 64), (2, 4, 2, -1, 8, 64), (2, 4, 2, 8, 8, -1)):
        assert lib.int2kv_chunk_attention_workspace_bytes(*bad) == 0
    # the longest sequence is no longer than all of them; more of anything needs no less
    assert K.int2kv_chunk_attention_workspace_bytes(2, 4, 2, 8, 999, 64) == need
    grow = [K.int2kv_chunk_attention_workspace_bytes(1, 32, 8, n, n, 4096) for n in (1, 64, 2048, 16384)]
    assert grow == sorted(grow)


def test_chunk_attention_workspace_serves_every_smaller_call():
    """One workspace, sized for the largest batch, is enough for every call within its bounds."""
    rng = np.random.default_rng(0)
    for hq, h in ((32, 8), (40, 8), (8, 8), (64, 1)):
        for _ in range(400):
            big = [int(x) for x in np.exp(rng.uniform(0, [6, 9, 8, 11]))]                # batch, total_q, max_q, max_ctx
            small = [int(x * rng.uniform(0, 1) ** 0.5) for x in big]
            small[0] = max(1, small[0])
            b, t, m, c = big
            assert (K.int2kv_chunk_attention_workspace_bytes(b, hq, h, t, m, c)
                    >= K.int2kv_chunk_attention_workspace_bytes(small[0], hq, h, *small[1:])), (hq, h, big, small)
