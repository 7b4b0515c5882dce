"""Rotary positions with several axes: bit for bit the fp64 result rounded once to bf16."""
import numpy as np
import pytest
import torch

from oracle import int2kv_oracle as O
from paper_2608_02691_amd import int2kv as K
from paper_2608_02691_amd import workloads as W

pytestmark = pytest.mark.gpu

MAX_POS = 5000


def _table():
    return W.rope_cos_sin(MAX_POS)


def _reference(x, pos, axis, cs):
    """bf16 bits [n, heads, 128] of int16-viewable rows x at positions [axes, n]."""
    bits = x.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
    rows = np.stack([cs[pos[a], i] for i, a in enumerate(axis)] + [cs[pos[a], 64 + i] for i, a in enumerate(axis)], 1)
    # a table of one row per token, each at its own position
    return O.rope(bits, np.arange(len(bits)), rows)


def _bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


AXES = {"one": K.rope_axis_table([64]), "sections": K.rope_axis_table([16, 24, 24]),
        "turns": K.rope_axis_table([16, 24, 24], interleaved=True), "odd": K.rope_axis_table([1, 0, 50, 13]),
        "eight": K.rope_axis_table([8] * 8, interleaved=True)}


@pytest.mark.parametrize("kind", AXES)
@pytest.mark.parametrize("n,hq,hk", [(1, 1, 1), (7, 4, 1), (64, 40, 8), (301, 5, 3), (9, 65, 2), (1500, 8, 0), (33, 0, 4)])
def test_matches_the_fp64_rounding(n, hq, hk, kind):
    print(f"\n[rope axes] {kind} n={n} heads {hq}/{hk}", flush=True)
    rng = np.random.default_rng(n + hq)
    axis = AXES[kind]
    axes = max(axis) + 1
    cs = _table()
    pos = rng.integers(0, MAX_POS, (axes, n)).astype(np.int32)
    pos[:, 0] = [0, MAX_POS - 1, 1, 2, 3, 4, 5, 6][:axes]
    x = [torch.from_numpy(rng.standard_normal((n, h, 128)).astype(np.float32) * np.exp(3 * rng.standard_normal((n, h, 1))).astype(np.float32)).to(torch.bfloat16)
         if h else None for h in (hq, hk)]
    q, k = (t.cuda() if t is not None else None for t in x)
    got = K.int2kv_rope_axes(torch.from_numpy(pos).cuda(), axis, torch.from_numpy(cs).cuda(), q, k)
    for g, t in zip(got, x):
        if t is None:
            assert g is None
        else:
            np.testing.assert_array_equal(_bits(g), _reference(t, pos, axis, cs))


def test_views_of_a_projection_in_place_and_apart():
    rng = np.random.default_rng(1)
    n, hq, hk, axis = 83, 8, 2, AXES["sections"]
    cs, pos = _table(), rng.integers(0, MAX_POS, (3, n)).astype(np.int32)
    qkv = torch.from_numpy(rng.standard_normal((n, hq + 2 * hk, 128)).astype(np.float32)).to(torch.bfloat16)
    want_q, want_k = _reference(qkv[:, :hq], pos, axis, cs), _reference(qkv[:, hq:hq + hk], pos, axis, cs)
    dev = (torch.from_numpy(pos).cuda(), axis, torch.from_numpy(cs).cuda())
    a = qkv.cuda()
    q, k = K.int2kv_rope_axes(*dev, a[:, :hq], a[:, hq:hq + hk])
    np.testing.assert_array_equal(_bits(q), want_q)
    np.testing.assert_array_equal(_bits(k), want_k)
    assert torch.equal(a.cpu(), qkv)
    K.int2kv_rope_axes(*dev, a[:, :hq], a[:, hq:hq + hk], q_out=a[:, :hq], k_out=a[:, hq:hq + hk])
    np.testing.assert_array_equal(_bits(a[:, :hq]), want_q)
    np.testing.assert_array_equal(_bits(a[:, hq:hq + hk]), want_k)
    assert torch.equal(a[:, hq + hk:].cpu(), qkv[:, hq + hk:])


def test_positions_outside_the_table_skip_their_token():
    rng = np.random.default_rng(2)
    n, cs, axis = 40, _table(), AXES["turns"]
    pos = rng.integers(0, MAX_POS, (3, n)).astype(np.int32)
    pos[0, 3], pos[1, 11], pos[2, 39], pos[2, 17] = -1, MAX_POS, 2 ** 31 - 1, -2 ** 31
    bad = [3, 11, 39, 17]
    q = torch.from_numpy(rng.standard_normal((n, 6, 128)).astype(np.float32)).to(torch.bfloat16).cuda()
    out = torch.full_like(q, 9.0)
    K.int2kv_rope_axes(torch.from_numpy(pos).cuda(), axis, torch.from_numpy(cs).cuda(), q, q_out=out)
    good = np.setdiff1d(np.arange(n), bad)
    assert bool((out[bad] == 9.0).all())
    np.testing.assert_array_equal(_bits(out[good]), _reference(q.cpu()[good], pos[:, good], axis, cs))


def test_one_axis_equals_the_cache_writes_keys():
    rng = np.random.default_rng(3)
    n, H = 50, 2
    cs = torch.from_numpy(_table()).cuda()
    pos = torch.from_numpy(rng.integers(0, MAX_POS, n).astype(np.int32)).cuda()
    k = torch.from_numpy(rng.standard_normal((n, H, 128)).astype(np.float32)).to(torch.bfloat16).cuda()
    cache = K.Int2KVCache(4, H)
    R = K.hadamard_rotation(H)
    k_rope = torch.empty_like(k)
    K.int2kv_quantize_append_rope(cache, k, k, torch.arange(n, dtype=torch.int32, device="cuda"), pos, cs, None, None,
                                  K.int2kv_prepare_mu_rot(R, torch.zeros((H, 128), device="cuda")),
                                  flags=K.INT2KV_HADAMARD_K | K.INT2KV_HADAMARD_V, k_rope_out=k_rope)
    _, got = K.int2kv_rope_axes(pos[None], AXES["one"], cs, k=k)
    assert torch.equal(got, k_rope)


def test_zeros_infinities_and_graphs():
    rng = np.random.default_rng(4)
    n, cs, axis = 20, _table(), AXES["sections"]
    pos = torch.from_numpy(rng.integers(1, MAX_POS, (3, n)).astype(np.int32)).cuda()
    q = torch.from_numpy(rng.standard_normal((n, 4, 128)).astype(np.float32)).to(torch.bfloat16)
    q[1] = 0
    q[2, 1, 5], q[3, 2, 70] = float("inf"), float("nan")
    q = q.cuda()
    c = torch.from_numpy(cs).cuda()
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        K.int2kv_rope_axes(pos, axis, c, q, q_out=out)
    for turn in range(3):
        pos.copy_((pos + 100 * turn) % MAX_POS)
        want, _ = K.int2kv_rope_axes(pos, axis, c, q)
        out.zero_()
        g.replay()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        assert bool((want[1] == 0).all())
        fine = torch.isfinite(want.float())
        assert not fine[2, 1, 5] and not fine[2, 1, 69] and not fine[3, 2, 70] and not fine[3, 2, 6]
        assert int((~fine).sum()) == 4
        torch.cuda.synchronize()


def test_new_outputs_are_zero_where_a_token_is_skipped():
    """The padding of a batch (position -1), in memory that held something else before."""
    rng = np.random.default_rng(5)
    cs = torch.from_numpy(_table()).cuda()
    q, k = (torch.from_numpy(rng.standard_normal((40, h, 128)).astype(np.float32)).to(torch.bfloat16).cuda() for h in (4, 2))
    pos = torch.arange(40, dtype=torch.int32, device="cuda")[None].contiguous()
    pos[0, 25:] = -1
    for _ in range(3):
        junk = [torch.full((40, h, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for h in (4, 2)]
        del junk
        for x in K.int2kv_rope_axes(pos, K.rope_axis_table([64]), cs, q, k):
            assert bool((x[25:] == 0).all()) and bool(torch.isfinite(x.float()).all())
