"""Attention of drafted trees' tokens (int2kv_tree_attention) against its definition in fp64."""
import numpy as np
import pytest
import torch

from _chunk import assert_chunk_close
from _tokens import K, TreeCall, dev, random_tree

pytestmark = pytest.mark.gpu


def check(call, what, **kw):
    ref, spread = call.reference()
    got = call.call(**kw)
    torch.cuda.synchronize()
    worst = assert_chunk_close(got, ref, spread, what)
    print(f"{what}: {worst:.3f} of the tolerance")
    return got


def tree(seed, T):
    return random_tree(np.random.default_rng(seed), T)


@pytest.mark.parametrize("heads,gq", [(1, 1), (2, 4), (2, 5), (1, 12)])
@pytest.mark.parametrize("group", [32, 128])
def test_ragged_trees(heads, gq, group):
    seqs = [(1, 1, tree(1, 1)), (7, 100, tree(2, 7)), (0, 33, tree(0, 0)), (16, 0, tree(3, 16)), (3, 515, tree(4, 3))]
    check(TreeCall(seqs, heads, gq, group, seed=gq, pad=2), f"ragged {heads} x {gq}, {group}")


@pytest.mark.parametrize("T", [31, 32, 33, 63, 64, 65, 128, 255, 256])
def test_sizes_around_tiles_and_words(T):
    check(TreeCall([(T, 65, tree(T, T))], 1, 2, seed=T), f"{T} tokens")


@pytest.mark.parametrize("n,T", [(1, 1), (1, 200), (8, 49), (5, 64), (30, 250), (64, 256)])
@pytest.mark.parametrize("gq", [1, 4])
def test_next_level(n, T, gq):
    """The queries are the last tokens of a longer tree."""
    check(TreeCall([(n, 90, tree(n + T, T)), (n, 17, tree(T, T))], 2, gq, seed=n), f"{n} of {T}", )


def test_chain_is_the_chunk():
    """A tree without branches sees what a drafted chunk sees."""
    c = TreeCall([(40, 77, np.arange(-1, 39)), (9, 300, np.arange(-1, 8))], 2, 4, seed=5)
    got = check(c, "chains")
    cache = K.Int2KVCache(c.pool.shape[0], c.H, pool=dev(c.pool), group_size=c.group)
    chunk = K.int2kv_chunk_attention(cache, c.q.cuda(), dev(c.starts), c.max_q, dev(c.table), dev(c.lens), c.max_ctx, dev(c.R_k), dev(c.R_v),
                                     c.k.cuda(), c.v.cuda(), dev(c.mu))
    assert torch.equal(got, chunk)


def test_deep_chain_and_wide_star():
    check(TreeCall([(256, 20, np.arange(-1, 255)), (256, 50, np.full(256, -1)), (256, 0, np.zeros(256) - np.eye(256)[0])], 1, 1, seed=6), "chain, star")


@pytest.mark.parametrize("bad", [-2, -(2 ** 31), 2 ** 31 - 1, 9, 8])
@pytest.mark.parametrize("n,gq", [(12, 1), (12, 8), (40, 4), (70, 4)])
def test_absent_tokens(bad, n, gq):
    """Token 8 names no token before it: it and what follows it see nothing, whatever their rows hold."""
    p = tree(7, n)
    p[8], p[9], p[10], p[11] = bad, 8, 9, 3
    p[12:] = np.minimum(p[12:], 7)
    c = TreeCall([(n, 40, p), (n, 700, tree(8, n))], 1, gq, seed=n)
    for t in (8, 9, 10):
        c.q[t] = float("nan")
        c.k[t] = float("inf")
        c.v[t] = float("nan")
    got = check(c, f"absent {bad}")
    assert torch.count_nonzero(got[8:11]) == 0


@pytest.mark.parametrize("split", [False, True])
def test_more_queries_than_tokens(split):
    """Queries in front of the tree are no tokens of it: zeros."""
    ctx = 3000 if split else 30
    c = TreeCall([(12, ctx, tree(9, 9)), (4, 20, tree(0, 0))], 1, 4, seed=9)
    got = check(c, "more queries")
    assert torch.count_nonzero(got[:3]) == 0 and torch.count_nonzero(got[12:]) == 0


def test_cut_trees():
    """max_tree cuts the tree's end: what stays keeps its place."""
    c = TreeCall([(20, 50, tree(10, 20))], 2, 2, seed=10)
    ref, spread = c.reference()
    ref[15:], spread[15:] = 0, 0
    assert_chunk_close(c.call(max_tree=15), ref, spread, "max_tree")
    c.seqs[0] = (20, 32, c.seqs[0][2])  # a table that ends early
    c.table = c.table[:, :2].copy()
    ref, spread = c.reference()
    assert_chunk_close(c.call(), ref, spread, "table")
    c = TreeCall([(20, 50, tree(10, 20))], 2, 2, seed=10)
    ref, spread = c.reference()
    got = c.call(max_q=7, out=torch.full((20, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda"))
    assert_chunk_close(got[:7], ref[:7], spread[:7], "max_q")
    assert torch.all(got[7:] == 3.0)


@pytest.mark.parametrize("n,gq,B", [(5, 4, 3), (64, 4, 2), (200, 4, 1), (30, 5, 1)])
def test_long_contexts_are_cut_into_pieces(n, gq, B):
    check(TreeCall([(n, 4000 - 371 * b, tree(n + b, n)) for b in range(B)], 1, gq, seed=n), f"{n} x {gq}, {B}")


def test_many_sequences():
    """More than a wave plans for."""
    rng = np.random.default_rng(11)
    seqs = [(int(n), int(c), random_tree(rng, int(n + g))) for n, c, g in zip(rng.integers(0, 9, 100), rng.integers(0, 200, 100), rng.integers(0, 20, 100))]
    check(TreeCall(seqs, 1, 4, seed=11), "100 sequences")


def test_views_and_padding():
    c = TreeCall([(9, 60, tree(12, 9)), (20, 5, tree(13, 20))], 2, 4, seed=12, pad=5, fused=True)
    out = torch.full((c.total, c.Hq, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    ref, spread = c.reference()
    got = c.call(out=out)
    assert_chunk_close(got[:29], ref[:29], spread[:29], "views")
    assert torch.all(got[29:] == 3.0)


@pytest.mark.parametrize("n", [6, 80])
def test_values_that_are_not_finite_reach_only_those_that_see_them(n):
    p = tree(14, n)
    p[2], p[3], p[4], p[5] = 0, 2, 0, 4
    p[6:] = np.where(p[6:] == 2, 0, p[6:])
    p[6:] = np.where(p[6:] == 3, 0, p[6:])
    c = TreeCall([(n, 100, p)], 1, 4, seed=14)
    ref, spread = c.reference()
    c.v[2, :, 7] = float("inf")
    c.v[2, :, 9] = float("nan")
    got = c.call().float().cpu()
    for t in range(n):
        if t in (2, 3):
            assert torch.all(torch.isinf(got[t, :, 7])) and torch.all(torch.isnan(got[t, :, 9]))
    rest = [t for t in range(n) if t not in (2, 3)]
    assert_chunk_close(got[rest], ref[rest], spread[rest], "others")


def test_missing_pages():
    c = TreeCall([(10, 200, tree(15, 10)), (10, 40, tree(16, 10))], 2, 4, seed=15)
    c.table[0, 3], c.table[0, 12], c.table[1, :] = -1, 1 << 30, -7
    check(c, "missing pages")


def test_streams_graphs_and_overlapping_calls():
    """Two calls at once on streams of their own, and a captured one whose tree changes between replays."""
    a = TreeCall([(30, 900, tree(17, 30))], 2, 4, seed=17)
    b = TreeCall([(30, 900, tree(18, 30))], 2, 4, seed=18)
    refs = [x.reference() for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for x, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            outs.append(x.call())
    torch.cuda.synchronize()
    for o, (ref, spread) in zip(outs, refs):
        assert_chunk_close(o, ref, spread, "streams")

    cache = K.Int2KVCache(a.pool.shape[0], a.H, pool=dev(a.pool), group_size=a.group)
    par, lens = dev(a.parents), dev(a.lens)
    fixed = (a.q.cuda(), dev(a.starts), a.max_q, par, a.k.cuda(), a.v.cuda(), dev(a.mu), dev(a.table), lens, a.max_ctx, dev(a.R_k), dev(a.R_v))
    out = torch.zeros((a.total, a.Hq, 128), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(K.int2kv_tree_attention_workspace_bytes(1, a.Hq, a.H, a.total, a.max_q, a.max_q, a.max_ctx), dtype=torch.uint8, device="cuda")
    K.int2kv_tree_attention(cache, *fixed, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.int2kv_tree_attention(cache, *fixed, out=out, workspace=ws)
    for seed, ctx in ((17, 900), (19, 555), (20, 0), (21, 899)):
        a.parents = tree(seed, 30)
        a.seqs[0], a.lens = (30, ctx, a.parents), np.array([ctx], np.int32)
        par.copy_(dev(a.parents))
        lens.copy_(dev(a.lens))
        graph.replay()
        eager = a.call(max_ctx=900)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        assert_chunk_close(out, *a.reference(), f"replay {seed}")


def test_bitwise_repeatable():
    c = TreeCall([(50, 2500, tree(22, 50)), (3, 100, tree(23, 3))], 2, 4, seed=22)
    first = c.call()
    assert all(torch.equal(first, c.call()) for _ in range(3))


def test_binding_refusals():
    c = TreeCall([(4, 20, tree(24, 4))], 1, 2, seed=24)
    with pytest.raises(RuntimeError, match="max_tree"):
        c.call(max_tree=257)
    with pytest.raises(ValueError, match="same tokens"):
        c.parents = c.parents[:3].copy()
        c.call()
