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
