"""Refusals of the operators for drafted trees and for eviction, before any launch (CPU only)."""
import ctypes

import numpy as np
import pytest

from paper_2608_02691_amd import int2kv as K

GOOD = K._Cache(16, 4, 2, 16, 128, 32)


def _tree(cache=GOOD, **kw):
    a = dict(q=1 << 20, qs=512, starts=16, B=2, total=8, max_q=8, hq=4, ts=16, tt=8, mt=8, par=16, k=2 << 20, ks=256, v=3 << 20, vs=256,
             mu=16, table=16, mb=4, lens=16, max_ctx=64, R_k=16, R_v=16, out=4 << 20, ws=1 << 24, wb=1 << 30)
    a.update(kw)
    st = K.load_library().int2kv_tree_attention(
        ctypes.byref(cache) if cache else None, a["q"], a["qs"], a["starts"], a["B"], a["total"], a["max_q"], a["hq"], a["ts"], a["tt"],
        a["mt"], a["par"], a["k"], a["ks"], a["v"], a["vs"], a["mu"], a["table"], a["mb"], a["lens"], a["max_ctx"], a["R_k"], a["R_v"],
        a["out"], a["ws"], a["wb"], None)
    return st, K.load_library().int2kv_last_error()


@pytest.mark.parametrize("kw,word", [
    (dict(cache=None), b"cache"), (dict(B=0), b"batch"), (dict(hq=3), b"num_q_heads"), (dict(total=-1), b"total_q"), (dict(max_q=-1), b"total_q"),
    (dict(max_ctx=-1), b"max_ctx"), (dict(mb=0), b"max_blocks"), (dict(tt=-1), b"total_tree"), (dict(mt=-1), b"max_tree"), (dict(ts=None), b"NULL"),
    (dict(par=None), b"NULL"), (dict(k=None), b"NULL"), (dict(v=None), b"NULL"), (dict(mu=None), b"NULL"), (dict(q=None), b"NULL"),
    (dict(starts=None), b"NULL"), (dict(table=None), b"NULL"), (dict(lens=None), b"NULL"), (dict(R_k=None), b"NULL"), (dict(out=None), b"NULL"),
    (dict(qs=504), b"stride"), (dict(ks=255), b"stride"), (dict(vs=0), b"stride"), (dict(q=(1 << 20) + 8), b"aligned"), (dict(R_v=24), b"aligned"),
    (dict(v=(3 << 20) + 4), b"aligned"), (dict(par=18), b"aligned"), (dict(out=1 << 20), b"overlap"), (dict(out=(2 << 20) + 1024), b"overlap"),
    (dict(ws=(1 << 24) + 16), b"workspace"),
])
def test_tree_attention_refusals(kw, word):
    st, msg = _tree(**kw)
    assert st == K.INT2KV_EINVAL and word in msg, msg


def test_tree_attention_bounds():
    need = K.int2kv_tree_attention_workspace_bytes(2, 4, 2, 8, 8, 8, 64)
    assert need > 0
    st, msg = _tree(wb=need - 1)
    assert st == K.INT2KV_EWORKSPACE and b"tree_attention_workspace" in msg
    assert _tree(mt=257)[0] == K.INT2KV_EUNSUPPORTED
    assert _tree(total=1 << 30, max_q=1)[0] == K.INT2KV_EUNSUPPORTED
    assert _tree(tt=1 << 30)[0] == K.INT2KV_EUNSUPPORTED
    assert _tree(max_q=0)[0] == K.INT2KV_OK and _tree(total=0)[0] == K.INT2KV_OK
    for bad in ((0, 4, 2, 8, 8, 8, 64), (2, 3, 2, 8, 8, 8, 64), (2, 4, 2, -1, 8, 8, 64), (2, 4, 2, 8, 8, 257, 64), (2, 4, 2, 8, 8, -1, 64),
                (2, 4, 2, 8, 8, 8, -1)):
        assert K.int2kv_tree_attention_workspace_bytes(*bad) == 0


def test_tree_attention_workspace_serves_every_smaller_call():
    rng = np.random.default_rng(0)
    for hq, h in ((32, 8), (40, 8), (8, 8), (64, 1)):
        for _ in range(300):
            big = [int(x) for x in np.exp(rng.uniform(0, [5, 9, 6, 5.5, 11]))]            # batch, total_q, max_q, max_tree, max_ctx
            small = [max(int(i == 0), int(x * rng.uniform(0, 1) ** 0.5)) for i, x in enumerate(big)]
            assert (K.int2kv_tree_attention_workspace_bytes(big[0], hq, h, *big[1:])
                    >= K.int2kv_tree_attention_workspace_bytes(small[0], hq, h, *small[1:])), (hq, h, big, small)


def _weights(cache=GOOD, **kw):
    a = dict(q=1 << 20, qs=512, starts=16, B=2, total=8, max_q=8, hq=4, table=16, mb=4, lens=16, max_ctx=64, R_k=16, wi=2 << 20, decay=1.0,
             wo=3 << 20, stride=64, ws=1 << 24, wb=1 << 30)
    a.update(kw)
    st = K.load_library().int2kv_token_weights(
        ctypes.byref(cache) if cache else None, a["q"], a["qs"], a["starts"], a["B"], a["total"], a["max_q"], a["hq"], a["table"], a["mb"],
        a["lens"], a["max_ctx"], a["R_k"], a["wi"], a["decay"], a["wo"], a["stride"], a["ws"], a["wb"], None)
    return st, K.load_library().int2kv_last_error()


@pytest.mark.parametrize("kw,word", [
    (dict(cache=None), b"cache"), (dict(B=0), b"batch"), (dict(hq=3), b"num_q_heads"), (dict(total=-1), b"total_q"), (dict(max_q=-1), b"total_q"),
    (dict(max_ctx=-1), b"max_ctx"), (dict(mb=0), b"max_blocks"), (dict(decay=float("nan")), b"decay"), (dict(decay=float("inf")), b"decay"),
    (dict(stride=63), b"weights_stride"), (dict(q=None), b"NULL"), (dict(R_k=None), b"NULL"), (dict(starts=None), b"NULL"), (dict(table=None), b"NULL"),
    (dict(lens=None), b"NULL"), (dict(wo=None), b"NULL"), (dict(qs=504), b"stride"), (dict(qs=516), b"stride"), (dict(q=(1 << 20) + 8), b"aligned"),
    (dict(R_k=24), b"aligned"), (dict(wi=(2 << 20) + 2), b"aligned"), (dict(wo=(2 << 20) + 64), b"overlap"), (dict(wi=(3 << 20) + 4), b"overlap"),
    (dict(ws=(1 << 24) + 16), b"workspace"),
])
def test_token_weights_refusals(kw, word):
    st, msg = _weights(**kw)
    assert st == K.INT2KV_EINVAL and word in msg, msg


def test_token_weights_bounds():
    need = K.int2kv_token_weights_workspace_bytes(2, 4, 2, 8, 8, 64)
    assert need > 0
    st, msg = _weights(wb=need - 1)
    assert st == K.INT2KV_EWORKSPACE and b"token_weights_workspace" in msg
    assert _weights(max_ctx=0)[0] == K.INT2KV_OK
    assert _weights(total=1 << 30)[0] == K.INT2KV_EUNSUPPORTED
    assert _weights(B=1 << 24, max_ctx=1 << 20, stride=1 << 20, wi=None)[0] == K.INT2KV_EUNSUPPORTED
    assert _weights(B=1 << 21, max_q=4, wi=None, wb=1 << 60)[0] == K.INT2KV_EUNSUPPORTED  # (1,024 threads a sequence and KV head)
    assert _weights(B=1, max_ctx=2 ** 31 - 1, stride=1 << 31, wi=None, wb=1 << 60)[0] == K.INT2KV_EUNSUPPORTED
    for bad in ((0, 4, 2, 8, 8, 64), (2, 3, 2, 8, 8, 64), (2, 4, 2, -1, 8, 64), (2, 4, 2, 8, 8, -1), (2, 4, 2, 1 << 30, 8, 64),
                (2, 4, 2, 8, 8, 2 ** 31 - 1)):
        assert K.load_library().int2kv_token_weights_workspace_bytes(*bad) == 0


def test_token_weights_workspace_serves_every_smaller_call():
    rng = np.random.default_rng(0)
    for hq, h in ((32, 8), (40, 8), (8, 8), (64, 1), (12, 1)):
        for _ in range(300):
            big = [int(x) for x in np.exp(rng.uniform(0, [6, 9, 8, 11]))]                # batch, total_q, max_q, max_ctx
            small = [max(int(i == 0), int(x * rng.uniform(0, 1) ** 0.5)) for i, x in enumerate(big)]
            assert (K.int2kv_token_weights_workspace_bytes(big[0], hq, h, *big[1:])
                    >= K.int2kv_token_weights_workspace_bytes(small[0], hq, h, *small[1:])), (hq, h, big, small)


def _select(**kw):
    a = dict(w=1 << 20, ws=64, B=2, H=2, lens=16, max_ctx=64, budget=32, sink=4, recent=8, kept=2 << 20, ks=32, kl=16)
    a.update(kw)
    st = K.load_library().int2kv_select_tokens(a["w"], a["ws"], a["B"], a["H"], a["lens"], a["max_ctx"], a["budget"], a["sink"], a["recent"],
                                               a["kept"], a["ks"], a["kl"], None)
    return st, K.load_library().int2kv_last_error()


@pytest.mark.parametrize("kw,word", [
    (dict(B=0), b"batch"), (dict(H=0), b"num_kv_heads"), (dict(max_ctx=-1), b"max_ctx"), (dict(ws=63), b"weights_stride"), (dict(budget=-1), b"budget"),
    (dict(sink=-1), b"budget"), (dict(recent=-1), b"budget"), (dict(sink=25), b"budget"), (dict(sink=1 << 30, recent=1 << 30), b"budget"),
    (dict(ks=31), b"kept_stride"), (dict(w=None), b"NULL"), (dict(lens=None), b"NULL"), (dict(kept=None), b"NULL"), (dict(kl=None), b"NULL"),
    (dict(w=(1 << 20) + 2), b"aligned"), (dict(kept=(2 << 20) + 1), b"aligned"),
])
def test_select_tokens_refusals(kw, word):
    st, msg = _select(**kw)
    assert st == K.INT2KV_EINVAL and word in msg, msg


def test_select_tokens_bounds():
    assert _select(B=1 << 22, H=2)[0] == K.INT2KV_EUNSUPPORTED
    for max_ctx in (2 ** 31 - 1, 2 ** 31 - 4097, 2 ** 31 - 2 ** 18):  # a span's step past the list has to fit 32 bits too
        assert _select(max_ctx=max_ctx, ws=1 << 31)[0] == K.INT2KV_EUNSUPPORTED


def _move(cache=GOOD, **kw):
    a = dict(table=16, mb=4, kept=16, ks=32, kl=16, B=2, mk=32, ot=64, om=2, w=1 << 20, wst=64, ow=2 << 20, ows=32, ws=None, wb=0)
    a.update(kw)
    st = K.load_library().int2kv_move_tokens(ctypes.byref(cache) if cache else None, a["table"], a["mb"], a["kept"], a["ks"], a["kl"], a["B"],
                                             a["mk"], a["ot"], a["om"], a["w"], a["wst"], a["ow"], a["ows"], a["ws"], a["wb"], None)
    return st, K.load_library().int2kv_last_error()


@pytest.mark.parametrize("kw,word", [
    (dict(cache=None), b"cache"), (dict(B=0), b"batch"), (dict(mb=0), b"max_blocks"), (dict(mk=-1), b"max_kept"), (dict(ks=31), b"kept_stride"),
    (dict(om=1), b"table"), (dict(ot=None, mb=1), b"table"), (dict(w=None), b"together"), (dict(ow=None), b"together"), (dict(wst=0), b"weights_stride"),
    (dict(ows=31), b"weights_stride"), (dict(table=None), b"NULL"), (dict(kept=None), b"NULL"), (dict(kl=None), b"NULL"), (dict(kept=18), b"aligned"),
    (dict(ow=(1 << 20) + 64), b"overlap"), (dict(ow=1 << 20), b"overlap"), (dict(ot=None, ws=(1 << 24) + 8, wb=1 << 24), b"workspace"),
])
def test_move_tokens_refusals(kw, word):
    st, msg = _move(**kw)
    assert st == K.INT2KV_EINVAL and word in msg, msg


def test_move_tokens_bounds():
    assert _move(mk=0)[0] == K.INT2KV_OK
    need = K.int2kv_move_tokens_workspace_bytes(2, 2, 32, 32)
    assert need == 2 * 2 * 2 * (1536 + 64)
    for kw in (dict(ot=None), dict(ot=16), dict(ot=None, ws=1 << 24, wb=need - 1)):
        st, msg = _move(**kw)
        assert st == K.INT2KV_EWORKSPACE and b"move_tokens_workspace" in msg
    assert _move(B=1 << 24, mk=1 << 20, ks=1 << 20, mb=1 << 16, om=1 << 16, w=None, ow=None)[0] == K.INT2KV_EUNSUPPORTED
    for bad in ((0, 2, 32, 32), (2, 0, 32, 32), (2, 2, 64, 32), (2, 2, 32, -1)):
        assert K.load_library().int2kv_move_tokens_workspace_bytes(*bad) == 0
