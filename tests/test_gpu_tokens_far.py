"""Trees and eviction where offsets pass 32 bits: records, lists, sums and rows, bit for bit as near ones."""
import numpy as np
import pytest
import torch

from _tokens import K, TreeCall, WeightsCall, dev, kept_reference, moved_pool, paged, random_tree
from _chunk import random_pool

pytestmark = pytest.mark.gpu

BLOCKS = (1 << 32) // 1536 + 4000


def far_cache(c):
    """A cache of one head whose last blocks are the call's, and the table that names them."""
    pool = torch.zeros((BLOCKS, 1, 1536), dtype=torch.uint8, device="cuda")
    pool[-c.pool.shape[0]:] = dev(c.pool)
    return K.Int2KVCache(BLOCKS, 1, pool=pool), np.where(c.table >= 0, c.table + (BLOCKS - c.pool.shape[0]), -1).astype(np.int32)


def far_rows(x, step):
    """x's tokens `step` elements apart."""
    room = torch.empty((x.shape[0] - 1) * step + x[0].numel(), dtype=x.dtype, device="cuda")
    view = room.as_strided(x.shape, (step, x.shape[2], 1))
    view.copy_(x)
    return view


@pytest.mark.parametrize("n", [1, 7, 40])
def test_tree_records(n):
    rng = np.random.default_rng(n)
    c = TreeCall([(n, 700, random_tree(rng, 40)), (min(n, 9), 33, random_tree(rng, 9))], 1, 4, seed=n)
    want = c.call()
    cache, c.table = far_cache(c)
    assert torch.equal(c.call(cache=cache), want)


def test_tree_rows():
    rng = np.random.default_rng(3)
    c = TreeCall([(20, 100, random_tree(rng, 20))], 2, 4, seed=3)
    want = c.call()
    step = 1 << 27
    cache = K.Int2KVCache(c.pool.shape[0], 2, pool=dev(c.pool))
    got = K.int2kv_tree_attention(cache, far_rows(c.q, step), dev(c.starts), 20, dev(c.parents), far_rows(c.k, step), far_rows(c.v, step),
                                  dev(c.mu), dev(c.table), dev(c.lens), 100, dev(c.R_k), dev(c.R_v))
    assert torch.equal(got, want)


@pytest.mark.parametrize("n,ctx", [(1, 900), (2, 900), (30, 900)])
def test_weights_records(n, ctx):
    c = WeightsCall([(n, ctx), (n, 50)], 1, 4, seed=n)
    want = c.call()
    cache, c.table = far_cache(c)
    assert torch.equal(c.call(cache=cache), want)


@pytest.mark.parametrize("n", [1, 40])
def test_weights_rows_and_sums(n):
    """Queries 2^27 elements apart, sums of heads 2^30 numbers apart."""
    c = WeightsCall([(n, 300), (n, 80)], 1, 4, seed=n)
    want = c.call()
    q = far_rows(c.q, 1 << 27)
    cache = K.Int2KVCache(c.pool.shape[0], 1, pool=dev(c.pool))
    w = torch.empty((2, 1, (1 << 30) + 64), device="cuda")
    w[:, :, :300] = dev(c.w)
    got = K.int2kv_token_weights(cache, q, dev(c.starts), n, dev(c.table), dev(c.lens), 300, dev(c.R_k), weights=w, decay=0.75, out=w)
    for b, length in enumerate((300, 80)):
        assert torch.equal(got[b, :, :length], want[b, :, :length])


def test_select_lists():
    rng = np.random.default_rng(5)
    w = torch.empty((2, 1, (1 << 30) + 64), device="cuda")
    kept = torch.empty((2, 1, (1 << 30) + 32), dtype=torch.int32, device="cuda")
    x = rng.random((2, 1, 5000)).astype(np.float32)
    w[:, :, :5000] = dev(x)
    kept[:, :, :300] = -1
    _, n = K.int2kv_select_tokens(w, dev(np.array([5000, 4000], np.int32)), 5000, 200, 3, 20, kept=kept)
    for b, length in enumerate((5000, 4000)):
        assert np.array_equal(kept[b, 0, :200].cpu().numpy(), kept_reference(x[b, 0], length, 200, 3, 20))
        assert bool((kept[b, 0, 200:300] == -1).all())
    assert n.tolist() == [200, 200]


@pytest.mark.parametrize("in_place", [True, False])
def test_move_records_lists_and_sums(in_place):
    rng = np.random.default_rng(6)
    lens = np.array([400, 90], np.int32)
    table, blocks = paged(rng, lens)
    small = random_pool(rng, blocks, 1, 32)
    pool = torch.zeros((BLOCKS, 1, 1536), dtype=torch.uint8, device="cuda")
    pool[-blocks:] = dev(small)
    far = np.where(table >= 0, table + (BLOCKS - blocks), -1).astype(np.int32)
    kept = torch.empty((2, 1, (1 << 30) + 32), dtype=torch.int32, device="cuda")
    lists = np.stack([np.sort(rng.permutation(c)[:70]) for c in lens])[:, None].astype(np.int32)
    kept[:, :, :70] = dev(lists)
    w = torch.zeros((2, 1, (1 << 30) + 64), device="cuda")
    x = rng.random((2, 1, 400)).astype(np.float32)
    w[:, :, :400] = dev(x)
    new = np.arange(10, dtype=np.int32).reshape(2, 5)
    cache = K.Int2KVCache(BLOCKS, 1, pool=pool)
    out = None if in_place else torch.zeros((2, 1, 70), device="cuda")
    got = K.int2kv_move_tokens(cache, dev(far), kept, dev(np.array([70, 70], np.int32)), 70, None if in_place else dev(new), w, out)
    if in_place:
        assert np.array_equal(pool[-blocks:].cpu().numpy(), moved_pool(small, table, lists, [70, 70], table))
    else:
        both = np.concatenate([np.zeros((10, 1, 1536), np.uint8), small])
        ref = moved_pool(both, np.where(table >= 0, table + 10, -1), lists, [70, 70], new)
        assert np.array_equal(pool[:10].cpu().numpy(), ref[:10]) and np.array_equal(pool[-blocks:].cpu().numpy(), small)
    for b in range(2):
        assert np.array_equal(got[b, 0, :70].cpu().numpy(), x[b, 0, lists[b, 0]])
