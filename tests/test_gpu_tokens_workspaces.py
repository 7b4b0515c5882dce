"""Workspaces of the operators for drafted trees and for eviction: exactly the size that their function gives, for the call itself and for
larger bounds, with NaN in every place and guard bytes behind them. A call's results do not depend on what lies there, and it writes nothing behind."""
import numpy as np
import pytest
import torch

from _tokens import K, TreeCall, WeightsCall, dev, random_tree
from test_gpu_evict import Move

pytestmark = pytest.mark.gpu

GUARD, GUARD_BYTES = 0xA5, 4096


def guarded(need, fill):
    ws = torch.full((need + GUARD_BYTES,), fill, dtype=torch.uint8, device="cuda")
    ws[need:] = GUARD
    return ws


def check(call, sizes, what):
    """call(workspace) -> tensors; the same, bit for bit, from a zeroed workspace that is larger than needed, and from each exact one."""
    want = call(torch.zeros(max(sizes) + (1 << 20), dtype=torch.uint8, device="cuda"))
    for need in sizes:
        for fill in (0xFF, 0x7F):  # NaN and negative numbers; 3.4e38 and large ones
            ws = guarded(need, fill)
            got = call(ws[:need])
            torch.cuda.synchronize()
            assert bool((ws[need:] == GUARD).all()), f"{what}: writes behind {need} bytes"
            for x, y in zip(got, want):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), f"{what}: {need} bytes of {fill:#x}"


def tree(seed, T):
    return random_tree(np.random.default_rng(seed), T)


# name: sequences (queries, cached, tokens of the tree), query heads of a KV head
TREES = {
    "few, cut": ([(5, 3000, 9), (3, 400, 3), (8, 65, 8)], 4),
    "few, whole": ([(5, 40, 5), (0, 33, 0), (3, 0, 3)], 4),
    "few, planned": ([(2 + b % 3, 17 * b % 900, 9) for b in range(70)], 4),
    "four waves, cut": ([(30, 2500, 30), (24, 10, 60)], 4),
    "four waves, planned": ([(30, 19 * b % 700, 30) for b in range(66)], 4),
    "eight waves, cut": ([(256, 3000, 256), (250, 1, 256)], 4),
}


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("name", TREES)
def test_trees(name, group):
    seqs, gq = TREES[name]
    print(f"\n[workspace] tree {name} G={group}", flush=True)
    c = TreeCall([(n, ctx, tree(n + ctx, T)) for n, ctx, T in seqs], 2, gq, group, seed=len(name), pad=3)
    for t in range(2, len(c.parents), 11):
        c.parents[t] = -2
    B, size = len(seqs), K.int2kv_tree_attention_workspace_bytes
    sizes = [size(B, c.Hq, 2, c.total, c.max_q, c.max_tree, c.max_ctx), size(B + 9, c.Hq, 2, 2 * c.total, c.max_q + 40, 256, 2 * c.max_ctx + 100)]
    assert sizes[0] <= sizes[1]
    check(lambda ws: [c.call(workspace=ws)], sizes, name)


# name: sequences (new, cached), KV heads, query heads of one, max_ctx
WEIGHTS = {
    "one launch": ([(1, 700), (0, 30), (2, 90), (0, 0)], 2, 4, None),
    "pieces": ([(1, 700), (0, 30), (2, 90), (0, 0)], 2, 4, 2600),
    "pieces, operands first": ([(1, 2300 - 31 * b) for b in range(40)], 8, 4, None),
    "many rows, one chunk": ([(20, 300), (0, 0), (3, 40), (0, 90)], 1, 4, None),
    "many rows, chunks": ([(700, 900), (0, 400), (64, 64), (1, 2), (200, 1500)], 2, 4, None),
    "prompts": ([(900, 900), (33, 33), (0, 0), (1100, 1100)], 2, 5, None),
    "no rows": ([(0, 100), (0, 300)], 2, 4, None),
}


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("name", WEIGHTS)
def test_weights(name, group):
    seqs, heads, gq, max_ctx = WEIGHTS[name]
    print(f"\n[workspace] weights {name} G={group}", flush=True)
    top = max(c for _, c in seqs)
    c = WeightsCall(seqs, heads, gq, group, seed=len(name), pad=2, wide=(max_ctx or top) - top)
    c.table[0, 2] = -1
    B, size = len(seqs), K.int2kv_token_weights_workspace_bytes
    own = dict(max_ctx=max_ctx or top)
    sizes = [size(B, c.Hq, heads, c.total, c.max_q, own["max_ctx"]), size(B + 5, c.Hq, heads, 3 * c.total, c.max_q + 70, 2 * own["max_ctx"] + 300)]
    assert sizes[0] <= sizes[1]
    check(lambda ws: [c.call(workspace=ws, out=torch.full(c.shape, -3.0, device="cuda"), **own)], [max(s, 256) for s in sizes], name)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("weights", [False, True])
def test_moves_in_place(weights, group):
    print(f"\n[workspace] move in place G={group}", flush=True)
    m = Move([300, 17, 64, 1], [130, 16, 33, 1], heads=3, group=group, seed=3)
    B, size = len(m.lens), K.int2kv_move_tokens_workspace_bytes
    w = np.random.default_rng(4).random((B, 3, 310)).astype(np.float32)

    def call(ws):
        cache = K.Int2KVCache(m.pool.shape[0], 3, pool=dev(m.pool), group_size=group)
        sums = dev(w) if weights else None
        K.int2kv_move_tokens(cache, dev(m.table), dev(m.kept), dev(m.keep), m.most, weights=sums, workspace=ws)
        return [cache.pool] + ([sums] if weights else [])

    check(call, [size(B, 3, group, m.most), size(B + 2, 3, group, 3 * m.most)], "move")
