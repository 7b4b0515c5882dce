"""The tokens that stay (int2kv_select_tokens) and their rows' move (int2kv_move_tokens): exact."""
import numpy as np
import pytest
import torch

from _chunk import random_pool
from _tokens import K, dev, kept_reference, moved_pool, paged

pytestmark = pytest.mark.gpu


def select(w, lens, budget, sink=0, recent=0, max_ctx=None, **kw):
    kept, n = K.int2kv_select_tokens(dev(w), dev(np.asarray(lens, np.int32)), w.shape[2] if max_ctx is None else max_ctx, budget, sink, recent, **kw)
    return kept.cpu().numpy(), n.cpu().numpy()


def check_select(w, lens, budget, sink=0, recent=0, max_ctx=None, what=""):
    cap = w.shape[2] if max_ctx is None else max_ctx
    kept, n = select(w, lens, budget, sink, recent, max_ctx)
    for b in range(w.shape[0]):
        length = min(max(int(lens[b]), 0), cap)
        assert n[b] == min(length, budget), what
        for h in range(w.shape[1]):
            ref = kept_reference(w[b, h], length, budget, sink, recent)
            assert np.array_equal(kept[b, h, :n[b]], ref), f"{what}: list {b}, {h}"
            assert np.all(kept[b, h, n[b]:] == -1)


@pytest.mark.parametrize("length", [1, 2, 63, 64, 65, 1023, 1024, 1025, 2047, 5000])
def test_select_sizes(length):
    rng = np.random.default_rng(length)
    w = rng.lognormal(0, 2, (2, 3, length)).astype(np.float32)
    for budget in sorted({0, 1, length // 3, length - 1, length, length + 5}):
        check_select(w, [length, max(0, length - 7)], budget, what=f"{budget} of {length}")
        check_select(w, [length, max(0, length - 7)], budget, sink=budget // 4, recent=budget // 2, what=f"{budget} of {length}, forced")


def test_select_ragged():
    rng = np.random.default_rng(0)
    w = rng.lognormal(0, 2, (9, 2, 3000)).astype(np.float32)
    check_select(w, [0, 1, 99, 100, 101, 3000, 2999, -5, 4000], 100, sink=4, recent=30)
    check_select(w, [0, 1, 99, 100, 101, 3000, 2999, -5, 4000], 100, sink=60, recent=40)   # forced ones only
    check_select(w, [0, 1, 99, 100, 101, 3000, 2999, -5, 4000], 700, sink=0, recent=700, max_ctx=1500)
    check_select(w, [0, 1, 99, 100, 101, 3000, 2999, -5, 4000], 700, sink=700, max_ctx=1500)


def test_select_ties_go_to_the_lower_index():
    rng = np.random.default_rng(1)
    for values in ([0.0], [0.0, -0.0], [1.0, 2.0], [1.0, np.nextafter(np.float32(1), 2)], [5e-45, 0.0, -5e-45]):
        w = rng.choice(np.array(values, np.float32), (2, 2, 2500))
        for budget in (1, 64, 1000, 2400):
            check_select(w, [2500, 1777], budget, sink=1 if budget > 8 else 0, recent=7 if budget > 8 else 0, what=f"{values}, {budget}")


def test_select_any_floats():
    rng = np.random.default_rng(2)
    w = rng.integers(0, 2 ** 32, (2, 2, 4000), dtype=np.uint64).astype(np.uint32).view(np.float32)
    w[0, 0, ::3] = np.inf
    w[0, 1, ::3] = -np.inf
    w[1, 0, ::2] = np.nan
    w[1, 1] = np.nan
    for budget in (10, 1500, 3990):
        check_select(w, [4000, 3900], budget, what=f"{budget}")


@pytest.mark.parametrize("length", [40000, 70001, 140000])
def test_select_long(length):
    rng = np.random.default_rng(3)
    w = np.exp(rng.standard_normal((1, 2, length))).astype(np.float32).view(np.uint32)
    w = (w & 0xFFFF0000).view(np.float32)
    kept, n = select(w, [length], 20000, 64, 256)
    for h in range(2):
        t = np.arange(64, length - 256)
        best = t[np.argsort(-w[0, h, t], kind="stable")[:20000 - 320]]
        assert np.array_equal(kept[0, h], np.sort(np.concatenate([np.arange(64), best, np.arange(length - 256, length)])))


def test_select_strides_and_untouched_entries():
    rng = np.random.default_rng(4)
    w = rng.random((2, 2, 500)).astype(np.float32)
    kept = torch.full((2, 2, 123), 7, dtype=torch.int32, device="cuda")
    got, n = K.int2kv_select_tokens(dev(w), dev(np.array([300, 20], np.int32)), 300, 100, kept=kept)
    assert got is kept and torch.all(kept[0, :, 100:] == 7) and torch.all(kept[1, :, 20:] == 7)
    for h in range(2):
        assert np.array_equal(kept[0, h, :100].cpu().numpy(), kept_reference(w[0, h], 300, 100, 0, 0))


def test_select_streams_and_graphs():
    rng = np.random.default_rng(5)
    w = dev(rng.random((2, 2, 3000)).astype(np.float32))
    lens, kept, n = dev(np.array([3000, 2000], np.int32)), torch.zeros((2, 2, 500), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    K.int2kv_select_tokens(w, lens, 3000, 500, 4, 100, kept, n)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        K.int2kv_select_tokens(w, lens, 3000, 500, 4, 100, kept, n)
    for step in range(4):
        w.copy_(dev(rng.random((2, 2, 3000)).astype(np.float32)))
        lens.copy_(dev(np.array([3000 - 600 * step, 499 + step], np.int32)))
        kept.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for b in range(2):
            for h in range(2):
                ref = kept_reference(w[b, h].cpu().numpy(), int(lens[b]), 500, 4, 100)
                assert np.array_equal(kept[b, h, :len(ref)].cpu().numpy(), ref) and int(n[b]) == len(ref)


class Move:
    def __init__(self, lens, keep, heads=2, group=32, seed=0, sort=True):
        rng = np.random.default_rng(seed)
        self.lens, self.keep = np.array(lens, np.int32), np.array(keep, np.int32)
        B = len(lens)
        self.table, blocks = paged(rng, self.lens)
        out, more = paged(rng, self.keep, spare=1)
        self.out_table = np.where(out >= 0, out + blocks, -1).astype(np.int32)
        self.group, self.most = group, max(1, int(self.keep.max()))
        self.pool = random_pool(rng, blocks + more, heads, group)
        self.kept = np.full((B, heads, self.most), -1, np.int32)
        for b in range(B):
            for h in range(heads):
                x = rng.permutation(self.lens[b])[:self.keep[b]] if self.lens[b] >= self.keep[b] else rng.integers(0, self.lens[b], self.keep[b])
                self.kept[b, h, :self.keep[b]] = np.sort(x) if sort else x
        self.w = rng.random((B, heads, max(1, int(self.lens.max())))).astype(np.float32)

    def run(self, in_place=False, weights=None, out_weights=None, max_kept=None, workspace=None):
        pool = dev(self.pool)
        cache = K.Int2KVCache(pool.shape[0], pool.shape[1], pool=pool, group_size=self.group)
        got = K.int2kv_move_tokens(cache, dev(self.table), dev(self.kept), dev(self.keep), self.most if max_kept is None else max_kept,
                                   None if in_place else dev(self.out_table), weights, out_weights, workspace)
        torch.cuda.synchronize()
        return pool.cpu().numpy(), got

    def check(self, in_place, what=""):
        pool, _ = self.run(in_place)
        ref = moved_pool(self.pool, self.table, self.kept, self.keep, self.table if in_place else self.out_table)
        assert np.array_equal(pool, ref), what
        w = dev(self.w)
        pool, got = self.run(in_place, weights=w)
        assert np.array_equal(pool, ref), what
        got = got.cpu().numpy()
        for b in range(len(self.keep)):
            for h in range(self.kept.shape[1]):
                n = self.keep[b]
                assert np.array_equal(got[b, h, :n], self.w[b, h, self.kept[b, h, :n]]), what
                rest = self.w[b, h, n:] if in_place else 0.0
                assert np.all(got[b, h, n:] == rest), what


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("heads", [1, 3, 8])
def test_move(group, in_place, heads):
    Move([100, 16, 1, 33, 300], [50, 16, 1, 0, 131], heads, group, seed=heads).check(in_place)
    Move([777], [500], heads, group, seed=heads + 1).check(in_place)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33])
def test_move_ends_inside_a_page(n):
    for in_place in (False, True):
        Move([60, 40], [n, max(0, n - 3)], 2, 32 if n % 2 else 128, seed=n).check(in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_move_in_any_order_with_repeats(in_place):
    Move([100, 64], [100, 64], seed=1, sort=False).check(in_place, "permuted")
    m = Move([100, 90], [40, 33], seed=2, sort=False)
    m.kept[:, :, 3], m.kept[:, :, 20] = m.kept[:, :, 2], m.kept[:, :, 0]
    m.check(in_place, "repeats")
    m = Move([20], [20], seed=3)
    m.kept[0, 0, :] = 19
    m.check(in_place, "one token")


@pytest.mark.parametrize("in_place", [False, True])
def test_move_of_what_is_not_there(in_place):
    """Indices outside the table and blocks outside the cache leave rows and weights as they were."""
    m = Move([100, 90, 50], [60, 48, 20], seed=4)
    m.kept[0, 0, 5], m.kept[0, 1, 17], m.kept[1, 0, 0], m.kept[1, 1, 47] = -1, 1 << 30, -(2 ** 31), m.table.shape[1] * 16
    m.table[2, 1] = -1
    m.table[0, 2] = 1 << 29
    if not in_place:
        m.out_table[1, 1] = -1
        m.out_table[0, 0] = m.pool.shape[0]
    ref = moved_pool(m.pool, m.table, m.kept, m.keep, m.table if in_place else m.out_table)
    assert np.array_equal(m.run(in_place)[0], ref)
    w = dev(m.w)
    pool, got = m.run(in_place, weights=w, out_weights=torch.full((3, 2, 60), 9.0, device="cuda"))
    assert np.array_equal(pool, ref)
    got = got.cpu().numpy()
    assert got[0, 0, 5] == 9 and got[0, 1, 17] == 9 and got[1, 0, 0] == 9 and got[1, 1, 47] == 9


def test_move_is_cut_to_max_kept():
    m = Move([100, 64], [60, 40], seed=5)
    ref = moved_pool(m.pool, m.table, m.kept, m.keep, m.out_table, max_kept=37)
    assert np.array_equal(m.run(max_kept=37)[0], ref)
    m.keep = np.array([-3, 1 << 30], np.int32)
    m.kept[1, :, 40:] = 3
    ref = moved_pool(m.pool, m.table, m.kept, np.array([0, 37]), m.out_table, max_kept=37)
    assert np.array_equal(m.run(max_kept=37)[0], ref)


def test_move_streams_and_graphs():
    """A captured move in place with its own workspace, lists changing between replays."""
    m = Move([200, 150], [64, 64], seed=6)
    pool = dev(m.pool)
    cache = K.Int2KVCache(pool.shape[0], pool.shape[1], pool=pool, group_size=m.group)
    table, kept, n, w = dev(m.table), dev(m.kept), dev(m.keep), dev(m.w)
    ws = torch.empty(K.int2kv_move_tokens_workspace_bytes(2, 2, 32, 64), dtype=torch.uint8, device="cuda")
    K.int2kv_move_tokens(cache, table, kept, n, 64, weights=w, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.int2kv_move_tokens(cache, table, kept, n, 64, weights=w, workspace=ws)
    rng = np.random.default_rng(7)
    for step in range(4):
        m.kept = np.stack([np.stack([np.sort(rng.permutation(c)[:64]) for _ in range(2)]) for c in (200, 150)]).astype(np.int32)
        m.keep = np.array([64 - step, 30 + step], np.int32)
        pool.copy_(dev(m.pool))
        kept.copy_(dev(m.kept))
        n.copy_(dev(m.keep))
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(pool.cpu().numpy(), moved_pool(m.pool, m.table, m.kept, m.keep, m.table))


def test_move_binding_refusals():
    m = Move([40], [20], seed=8)
    with pytest.raises(RuntimeError, match="workspace"):
        m.run(True, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="out_weights"):
        m.run(out_weights=torch.zeros((1, 2, 20), device="cuda"))
    with pytest.raises(ValueError, match="kept"):
        m.run(max_kept=21)
