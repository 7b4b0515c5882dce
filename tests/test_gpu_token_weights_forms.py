"""int2kv_token_weights for few rows a sequence: contexts that one work-group holds (up to 2,048 tokens by max_ctx) and the
same calls in pieces of a context, against the definition in fp64."""
import numpy as np
import pytest
import torch

from _tokens import K, WeightsCall, assert_weights_close, dev

pytestmark = pytest.mark.gpu

LONG = 2100  # max_ctx of the calls in pieces


def calls(seqs, heads, gq, group=32, **kw):
    return WeightsCall(seqs, heads, gq, group, wide=LONG - max(c for _, c in seqs), **kw)


def check(c, what, decay=0.75):
    """Both forms; entries behind a length stay as they were in each."""
    ref, tol = c.reference(decay)
    got = []
    for max_ctx in (c.max_ctx, LONG):
        out = torch.full(c.shape, -3.0, device="cuda")
        c.call(decay=decay, max_ctx=max_ctx, out=out)
        for b, (_, n) in enumerate(c.seqs):
            worst = assert_weights_close(out[b, :, :n], ref[b, :, :n], tol[b, :, :n], f"{what}, max_ctx {max_ctx}")
            assert bool((out[b, :, n:] == -3.0).all()), what
            print(f"{what}, max_ctx {max_ctx}: {worst:.3f} of the tolerance")
        got.append(out)
    return got


@pytest.mark.parametrize("length", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 511, 512, 513, 1023, 1024, 1025, 2047, 2048])
@pytest.mark.parametrize("gq,group", [(1, 32), (4, 128), (5, 32), (8, 128)])
def test_lengths(length, gq, group):
    """The longest sequence fills a work-group's waves or ends inside one; others are shorter, empty or without a token."""
    check(calls([(1, length), (0, (length + 1) // 2), (1, 1), (0, 0), (1, 0), (1, max(1, length - 17))], 2, gq, group, seed=length), f"{length} x {gq}")


@pytest.mark.parametrize("n,gq", [(8, 1), (2, 4), (4, 2), (2, 3), (3, 2)])
def test_several_tokens(n, gq):
    check(calls([(n, 700), (n, n), (1, 1500), (n, max(0, n - 2))], 3, gq, seed=n + gq), f"{n} x {gq}")


@pytest.mark.parametrize("top", [500, 1000, 2000])
def test_missing_pages(top):
    c = calls([(2, top), (1, 40), (1, 300)], 2, 4, seed=top, first=True)
    c.table[0, 3], c.table[0, 11], c.table[1, :], c.table[2, :12] = -1, 1 << 30, -7, 1 << 29
    for got in check(c, "missing pages"):
        assert torch.count_nonzero(got[1, :, :40]) == 0 and torch.count_nonzero(got[2, :, :192]) == 0
        assert torch.count_nonzero(got[0, :, 48:64]) == 0


@pytest.mark.parametrize("gq", [4, 8])
def test_the_maximum_moves_far(gq):
    """Scores that rise by hundreds along the context, and fall again; rows of very different scores."""
    c = calls([(1, 2000)], 1, gq, seed=gq, q_scale=8.0, first=True)
    c.q[0, 1] *= 0.001
    rise = np.concatenate([np.linspace(0.1, 8, 1000), np.linspace(8, 0.1, 1000)]).astype(np.float16)
    for t in range(2000):
        rec = c.pool[c.table[0, t // 16], 0]
        m = rec[1024 + 16 * (t % 16):1040 + 16 * (t % 16)].view(np.float16)
        m *= rise[t]
    check(c, "moving maximum")


@pytest.mark.parametrize("length", [37, 700, 1900])
def test_stale_slots_do_not_count(length):
    """Parameters behind a length, and those of other blocks, may hold anything."""
    c = calls([(1, length), (2, 21)], 1, 4, seed=length)
    for b, n in enumerate((length, 21)):
        rec = c.pool[c.table[b, n // 16], 0]
        for t in range(n % 16, 16):
            rec[1024 + 16 * t:1024 + 16 * t + 16] = 0xFF  # NaN
    c.pool[[x for x in range(c.pool.shape[0]) if x not in c.table], 0, 1024:] = 0xFF
    check(c, "stale slots")


@pytest.mark.parametrize("max_ctx", [500, 1000, 2000, LONG])
def test_in_place_decay_and_cut_contexts(max_ctx):
    """Sums in place; a context that max_ctx cuts keeps its entries behind the cut, and its tokens what they saw of the rest."""
    c = calls([(1, 600), (0, 480), (1, 300)], 2, 4, seed=21)
    w = dev(c.w)
    before = w.clone()
    got = c.call(weights=w, out=w, max_ctx=max_ctx, decay=-0.5)
    assert got.data_ptr() == w.data_ptr()
    cut = [min(n, max_ctx) for _, n in c.seqs]
    c.seqs = [(n, x) for (n, _), x in zip(c.seqs, cut)]  # one token a sequence: it sees all that is left
    ref, tol = c.reference(-0.5)
    for b, n in enumerate(cut):
        assert_weights_close(w[b, :, :n], ref[b, :, :n], tol[b, :, :n], "in place")
        assert torch.equal(w[b, :, n:], before[b, :, n:])


@pytest.mark.parametrize("max_ctx", [512, 2048, 2500])
def test_graphs(max_ctx):
    """A captured step replayed over contexts that grow, with eager work between the replays."""
    c = WeightsCall([(1, 400), (1, 70)], 2, 4, seed=22, wide=max_ctx - 400)
    cache = K.Int2KVCache(c.pool.shape[0], c.H, pool=dev(c.pool), group_size=c.group)
    lens, w, out = dev(c.lens), dev(c.w), torch.zeros(c.shape, dtype=torch.float32, device="cuda")
    ws = torch.empty(K.int2kv_token_weights_workspace_bytes(2, c.Hq, c.H, c.total, c.max_q, max_ctx), dtype=torch.uint8, device="cuda")
    args = (cache, c.q.cuda(), dev(c.starts), c.max_q, dev(c.table), lens, max_ctx, dev(c.R_k))
    K.int2kv_token_weights(*args, weights=w, decay=0.75, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.int2kv_token_weights(*args, weights=w, decay=0.75, out=out, workspace=ws)
    for step, ctx in enumerate(((400, 70), (333, 1), (1, 70), (399, 64))):
        c.seqs, c.lens = [(1, x) for x in ctx], np.array(ctx, np.int32)
        lens.copy_(dev(c.lens))
        out.zero_()
        graph.replay()
        eager = c.call(max_ctx=max_ctx, out=torch.zeros_like(out))
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        assert_weights_close(out, *c.reference(), f"replay {step}")


@pytest.mark.parametrize("length", [500, 1000, 2000])
def test_many_sequences_are_repeatable(length):
    """More work-groups than the chip holds at once."""
    c = WeightsCall([(1, length - 7 * (i % 13)) for i in range(150)], 8, 4, 128, seed=23)
    first = c.call()
    assert all(torch.equal(first, c.call()) for _ in range(3))
    total = (first - 0.75 * torch.where(torch.arange(length, device="cuda") < dev(c.lens)[:, None, None], dev(c.w), 0)).double().sum(-1)
    # each of the `length` differences is off by a rounding of its parts and the weight's own error: 2^-22 of sums up to a few tens
    assert torch.allclose(total, torch.full_like(total, 4.0), atol=length * 2.0 ** -18)
