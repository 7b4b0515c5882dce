"""The operators for drafted trees and for eviction where nothing is there: trees without a token, lists without an entry. An empty tensor has no
address, so these reach the library as NULL."""
import numpy as np
import pytest
import torch

from _tokens import K, TreeCall, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs,gq", [([(3, 40), (2, 5), (0, 7)], 4), ([(200, 3000)], 4), ([(2, 30)] * 70, 1), ([(4, 0)], 8)])
@pytest.mark.parametrize("max_tree", [0, 16])
def test_queries_without_trees(seqs, gq, max_tree):
    """Every query lies in front of its sequence's tree: zeros, and rows behind the last sequence as they were."""
    print(f"\n[empty trees] {len(seqs)} x {gq}, max_tree {max_tree}", flush=True)
    c = TreeCall([(n, ctx, np.zeros(0, np.int32)) for n, ctx in seqs], 2, gq, seed=len(seqs), pad=2)
    out = torch.full((c.total, c.Hq, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    got = c.call(out=out, max_tree=max_tree)
    torch.cuda.synchronize()
    assert bool((got[:-2] == 0).all()) and bool((got[-2:] == 3.0).all())


@pytest.mark.parametrize("in_place", [False, True])
def test_moves_of_nothing(in_place):
    """max_kept 0, with sums and without: the cache and the sums stay as they were, new sums are empty."""
    pool = dev(np.random.default_rng(0).integers(0, 256, (8, 3, 1536)).astype(np.uint8))
    cache, before = K.Int2KVCache(8, 3, pool=pool), pool.clone()
    table, other = dev(np.arange(4, dtype=np.int32).reshape(2, 2)), dev(np.arange(4, 8, dtype=np.int32).reshape(2, 2))
    kept, lens = torch.zeros((2, 3, 0), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    w = torch.rand((2, 3, 30), device="cuda")
    sums = w.clone()
    out = None if in_place else other
    assert K.int2kv_move_tokens(cache, table, kept, lens, 0, out_table=out) is None
    got = K.int2kv_move_tokens(cache, table, kept, lens, 0, out_table=out, weights=w)
    torch.cuda.synchronize()
    assert torch.equal(pool, before) and torch.equal(w, sums)
    assert got.data_ptr() == w.data_ptr() if in_place else got.shape == (2, 3, 0)
