"""Eviction and drafted trees together, as a serving loop calls them: a prompt whose last tokens vote, decode steps that add to the
sums, the cache cut to a budget, a drafted tree over what is left, its accepted path appended, and decode steps again."""
import numpy as np
import pytest
import torch

from paper_2608_02691_amd import workloads as W

from _chunk import PAGE, haar
from _helpers import assert_rows_close
from _tokens import K, dev, kept_reference, path_of

pytestmark = pytest.mark.gpu

H, GQ, BUDGET, SINK, RECENT, DECAY = 2, 4, 160, 4, 40, 0.875


def _attend(q, keys, values, gq):
    """fp64 attention of one token's q [Hq, 128] over keys, values [L, H, 128], and its spread."""
    out, spread = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape[0], dtype=torch.float64)
    for j in range(q.shape[0]):
        p = torch.softmax(keys[:, j // gq] @ q[j] / np.sqrt(128), -1)
        out[j] = p @ values[:, j // gq]
        spread[j] = ((p ** 2) @ (values[:, j // gq] ** 2).sum(-1)).sqrt()
    return out, spread


class Loop:
    """Two sequences; `lens` tokens in the cache, `pos` the next position (what was evicted keeps its place in the text)."""

    def __init__(self, group, seed):
        self.rng = rng = np.random.default_rng(seed)
        self.prompts, self.cap = [300, 213], 24 * PAGE
        self.R = haar(rng, H), haar(rng, H)
        self.R_k, self.R_v = dev(self.R[0]), dev(self.R[1])
        self.mu = dev((5 * rng.standard_normal((H, 128))).astype(np.float32))
        self.mu_rk = K.int2kv_prepare_mu_rot(self.R_k, self.mu)
        self.cs, self.axis = dev(W.rope_cos_sin(1000)), K.rope_axis_table([64])
        self.table = rng.permutation(100)[:48].reshape(2, 24).astype(np.int32)
        self.cache = K.Int2KVCache(100, H, group_size=group)
        self.lens, self.pos = np.zeros(2, np.int32), np.zeros(2, np.int32)

    def rows(self, positions):
        """q, k, v of tokens at the given positions, rotated."""
        x = torch.from_numpy(self.rng.standard_normal((len(positions), H * GQ + 2 * H, 128)).astype(np.float32)).to(torch.bfloat16).cuda()
        q, k = K.int2kv_rope_axes(dev(np.asarray(positions, np.int32)[None]), self.axis, self.cs, x[:, :H * GQ], x[:, H * GQ:H * GQ + H])
        return q, k, x[:, H * GQ + H:].contiguous()

    def slots(self, b, tokens):
        t = np.asarray(tokens)
        return self.table[b, t // PAGE] * PAGE + t % PAGE

    def append(self, k, v, slots):
        K.int2kv_quantize_append(self.cache, k, v, dev(np.asarray(slots, np.int32)), self.R_k, self.R_v, self.mu_rk)

    def held(self, b, n=None, rotated=True):
        """Centered keys and values of a sequence's cached tokens in fp64, in the model's bases (or as stored)."""
        s = dev(self.slots(b, np.arange(self.lens[b] if n is None else n)).astype(np.int32))
        k, v = K.int2kv_read_rows(self.cache, s, dtype=torch.float32)
        k, v = k.double().cpu(), v.double().cpu()
        if rotated:
            k = torch.einsum("thc,hdc->thd", k, torch.from_numpy(self.R[0]).double())
            v = torch.einsum("thc,hdc->thd", v, torch.from_numpy(self.R[1]).double())
        return k, v

    def weights(self, q, n, w):
        """Adds the votes of n tokens a sequence to w in place; w against fp64: a weight is off by 2^-18 of the terms of its
        score, which come to less than 64 for normal queries and rows."""
        want = DECAY * w.double().cpu()
        for b in range(2):
            keys, _ = self.held(b)
            for i in range(n):
                limit = self.lens[b] - n + i + 1
                for j in range(H * GQ):
                    a = keys[:limit, j // GQ] @ q[b * n + i, j].double().cpu() / np.sqrt(128)
                    want[b, j // GQ, :limit] += torch.softmax(a, -1)
        lens = dev(self.lens)
        got = K.int2kv_token_weights(self.cache, q, dev(np.array([0, n, 2 * n], np.int32)), n, dev(self.table), lens, int(self.lens.max()),
                                     self.R_k, weights=w, decay=DECAY, out=w)
        assert got is w
        for b in range(2):
            g, r = w[b, :, :self.lens[b]].double().cpu(), want[b, :, :self.lens[b]]
            assert bool(((g - r).abs() <= 2.0 ** -12 * r + 2.0 ** -100).all())
        assert bool((w[0, :, self.lens[0]:] == 0).all())

    def decode_step(self, w):
        """Append a token a sequence, attend, vote."""
        q, k, v = self.rows(self.pos)
        slots = [self.slots(b, self.lens[b]) for b in range(2)]
        self.append(k, v, slots)
        self.lens, self.pos = self.lens + 1, self.pos + 1
        out = K.int2kv_decode(self.cache, q, dev(self.table), dev(self.lens), int(self.lens.max()), self.R_k, self.R_v)
        for b in range(2):
            ref, _ = _attend(q[b].double().cpu(), *self.held(b), GQ)
            assert_rows_close(out[b:b + 1].cpu().numpy().reshape(1, -1), ref.numpy().reshape(1, -1), what="decode")
        self.weights(q, 1, w)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("in_place", [True, False])
def test_a_serving_loop(group, in_place):
    c = Loop(group, 31 + group)
    w = torch.zeros((2, H, c.cap), device="cuda")
    # the prompts, the last 32 tokens of which vote
    q = []
    for b, n in enumerate(c.prompts):
        qb, k, v = c.rows(np.arange(n))
        c.append(k, v, c.slots(b, np.arange(n)))
        q.append(qb[-32:])
    c.lens, c.pos = np.array(c.prompts, np.int32), np.array(c.prompts, np.int32)
    c.weights(torch.cat(q), 32, w)
    for _ in range(3):
        c.decode_step(w)
    # the cut
    kept, kept_lens = K.int2kv_select_tokens(w, dev(c.lens), int(c.lens.max()), BUDGET, SINK, RECENT)
    before = [c.held(b, rotated=False) for b in range(2)]
    sums = w.cpu().numpy()
    lists = kept.cpu().numpy()
    for b in range(2):
        for h in range(H):
            assert np.array_equal(lists[b, h], kept_reference(sums[b, h], int(c.lens[b]), BUDGET, SINK, RECENT))
    if in_place:
        K.int2kv_move_tokens(c.cache, dev(c.table), kept, kept_lens, BUDGET, weights=w)
        w[..., BUDGET:] = 0
    else:
        free = np.setdiff1d(np.arange(100), c.table.ravel())[:48].reshape(2, 24).astype(np.int32)
        w2 = torch.zeros_like(w)
        K.int2kv_move_tokens(c.cache, dev(c.table), kept, kept_lens, BUDGET, dev(free), w, w2)
        c.table, w = free, w2
    assert kept_lens.tolist() == [BUDGET, BUDGET]
    c.lens = np.array([BUDGET, BUDGET], np.int32)
    for b in range(2):
        for x, y in zip(before[b], c.held(b, rotated=False)):
            for h in range(H):
                assert torch.equal(y[:, h], x[torch.from_numpy(lists[b, h]).long(), h])
        for h in range(H):
            assert np.array_equal(w[b, h, :BUDGET].cpu().numpy(), sums[b, h, lists[b, h]])
    for _ in range(2):
        c.decode_step(w)
    # drafted trees, of nine tokens and of six and an empty place
    trees = [np.array([-1, -1, 0, 0, 1, 2, 2, 4, 6], np.int32), np.array([-1, 0, 0, 1, 3, 4, -2], np.int32)]
    starts = np.array([0, 9, 16], np.int32)
    depth = [[len(path_of(t, i) or [0]) - 1 for i in range(len(t))] for t in trees]
    q, k, v = c.rows(np.concatenate([c.pos[b] + np.array(depth[b]) for b in range(2)]))
    out = K.int2kv_tree_attention(c.cache, q, dev(starts), 9, dev(np.concatenate(trees)), k, v, c.mu, dev(c.table), dev(c.lens),
                                  int(c.lens.max()), c.R_k, c.R_v)
    m = c.mu.double().cpu()
    for b in range(2):
        keys, values = c.held(b)
        for i in range(len(trees[b])):
            path = path_of(trees[b], i)
            if path is None:
                assert not out[starts[b] + i].any()
                continue
            at = torch.tensor(path) + int(starts[b])
            ref, spread = _attend(q[starts[b] + i].double().cpu(), torch.cat([keys, k[at].double().cpu() - m]),
                                  torch.cat([values, v[at].double().cpu()]), GQ)
            err = (out[starts[b] + i].double().cpu() - ref).norm(dim=-1)
            assert bool((err <= 2.0 ** -7 * (ref.norm(dim=-1) + spread)).all())
    # the accepted paths join the cache, the other rows get no slot
    slots = np.full(16, -1, np.int32)
    for b, leaf in enumerate((8, 5)):
        path = path_of(trees[b], leaf)[::-1]
        slots[starts[b] + np.array(path)] = c.slots(b, c.lens[b] + np.arange(len(path)))
        c.lens[b] += len(path)
        c.pos[b] += len(path)
    c.append(k, v, slots)
    for _ in range(2):
        c.decode_step(w)
