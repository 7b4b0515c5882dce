"""Keys and values that are not finite, in trees whose rows are one piece and in trees whose context is cut: the same rows come
out as NaN or infinite in both, and absent tokens as zeros."""
import numpy as np
import pytest
import torch

from _chunk import assert_chunk_close
from _tokens import TreeCall, path_of, random_tree
from test_gpu_chunk import _meta

pytestmark = pytest.mark.gpu

STRUCK = 2  # the token whose row is not finite
# tokens, query heads of the KV head: the kernel of few rows, four waves, eight
SIZES = [(12, 4), (200, 4), (256, 4)]


def struck_tree(n, ctx, seed, batch=1, absent=()):
    """A call, the rows that see STRUCK and those of absent tokens. Batches above 64 sequences take the planning launch."""
    rng = np.random.default_rng(seed)
    p = random_tree(rng, n)
    p[STRUCK], p[STRUCK + 1] = 0, STRUCK
    p[4], p[5] = 0, 4
    for t in absent:
        p[t] = -2
    tail = [(1, 20, np.array([-1]))] * (batch - 1)
    c = TreeCall([(n, ctx, p)] + tail, 1, 4, seed=seed)
    paths = [path_of(p, t) for t in range(n)]
    sees = np.array([x is not None and STRUCK in x for x in paths] + [False] * (batch - 1))
    gone = np.array([x is None for x in paths] + [False] * (batch - 1))
    assert sees.sum() >= 2 and (~sees & ~gone).sum() >= 3
    return c, sees, gone


@pytest.mark.parametrize("n,gq", SIZES)
@pytest.mark.parametrize("ctx,batch", [(0, 1), (30, 1), (3000, 1), (6000, 1), (3000, 70)])
def test_infinite_scores_are_nan_cut_or_not(n, gq, ctx, batch):
    """A key with an infinite channel whose score is +infinity: inf - inf in the softmax of the rows that see it, as in the chunk
    attention; never the zeros of an absent token."""
    print(f"\n[infinite key] {n} x {gq} after {ctx}, {batch}", flush=True)
    c, sees, gone = struck_tree(n, ctx, n + ctx, batch, absent=(7,))
    c.q[..., 7] = c.q[..., 7].abs() + 0.5
    ref, spread = c.reference()
    c.k[STRUCK, :, 7] = float("inf")
    got = c.call().float().cpu()
    assert bool(torch.isnan(got[torch.from_numpy(sees)]).all())
    assert_chunk_close(got.numpy()[~sees], ref[~sees], spread[~sees], "the others")
    assert bool((got[torch.from_numpy(gone)] == 0).all())


@pytest.mark.parametrize("n,gq", SIZES)
@pytest.mark.parametrize("ctx", [30, 3000])
def test_scores_of_minus_infinity_have_no_weight(n, gq, ctx):
    """The same key where its score is -infinity: the rows come out as with a key whose score is far below all others."""
    print(f"\n[-infinite key] {n} x {gq} after {ctx}", flush=True)
    c, sees, _ = struck_tree(n, ctx, n + ctx + 1, absent=(7,))
    c.q[..., 7] = -(c.q[..., 7].abs() + 0.5)
    c.k[STRUCK] = torch.from_numpy(c.mu).to(torch.bfloat16)
    c.k[STRUCK, :, 7] = 2.0 ** 13  # at most -0.5 * 2^13 / sqrt(128) = -362: e^-300 beside any other token of the path
    ref, spread = c.reference()
    c.k[STRUCK, :, 7] = float("inf")
    assert_chunk_close(c.call(), ref, spread, "rows with and without it")


@pytest.mark.parametrize("n,gq", SIZES)
@pytest.mark.parametrize("ctx", [30, 3000])
@pytest.mark.parametrize("what", ["key scale", "key zero", "value scale"])
def test_cached_rows_that_are_not_finite(n, gq, ctx, what):
    """A cached token that every token of the tree sees: no row is finite, and those of absent tokens are zeros."""
    print(f"\n[cached {what}] {n} x {gq} after {ctx}", flush=True)
    c, _, gone = struck_tree(n, ctx, n + ctx + 2, absent=(7, n - 1))
    k, v = _meta(c.pool, c.group)
    if what == "value scale":
        v[c.table[0, 0], :, 0, :, 11] = np.inf
    else:
        k[c.table[0, 0], :, 11, :, 0 if what == "key scale" else 1] = np.inf
    got = c.call().float().cpu().numpy()
    assert not np.isfinite(got[~gone]).all(-1).any()
    assert np.all(got[gone] == 0)


@pytest.mark.parametrize("n,gq", SIZES)
@pytest.mark.parametrize("ctx", [30, 3000, 6000])
def test_values_that_are_not_finite_in_cut_trees(n, gq, ctx):
    """Channels of a value: they reach the rows that see it in those channels, and nothing else."""
    print(f"\n[values] {n} x {gq} after {ctx}", flush=True)
    c, sees, gone = struck_tree(n, ctx, n + ctx + 3, absent=(7,))
    ref, spread = c.reference()
    c.v[STRUCK, :, 7], c.v[STRUCK, :, 9] = float("inf"), float("nan")
    got = c.call().float().cpu().numpy()
    assert np.isinf(got[sees][:, :, 7]).all() and np.isnan(got[sees][:, :, 9]).all()
    assert np.isfinite(np.delete(got[sees], (7, 9), -1)).all()
    assert_chunk_close(got[~sees], ref[~sees], spread[~sees], "the others")
    assert np.all(got[gone] == 0)
