"""int2kv_token_weights for few rows a sequence: contexts that one work-group holds (up to 2,048 tokens by max_ctx) and the
same calls in pieces of a context, against the definition in fp64."""
import numpy as np
import pytest
import torch

from _chunk import stored_rows
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


def typical_error(c):
    """Norms over all weights [.., tokens] of the sums and of what their error comes to in fp32, with no running sums. With s_g D_g
    and z_g Q_g the parts of a score x (base 2): each part and x are sums in which at most 8 roundings of that size count (a
    group's products come in two terms, each of which may round up to four times; fma chains over the groups). A rounding is
    uniform within half a step, at most 2^-24 of the value, thus 2^-24 / sqrt(3) in the root mean square, and the score is off
    by delta = sqrt(8 / 3) 2^-24 sqrt(sum_g (s_g D_g)^2 + (z_g Q_g)^2 + x^2). A weight is off by ln 2 of that of itself, and by as much
    again for its row's log sum, a mean of such errors; the logarithm, the exponential and the sum add 2^-22."""
    D, PAGE = 128, 16
    want, off, q, ng = 0.0, 0.0, c.q.double().numpy(), D // c.group
    for b, (n, ctx) in enumerate(c.seqs):
        if ctx == 0 or n == 0:
            continue
        kc, _ = stored_rows(c.pool, c.table[b], ctx)
        for h in range(c.H):
            z, w, e = c._zeros(b, ctx, h), np.zeros(ctx), np.zeros(ctx)
            for j in range(h * c.gq, (h + 1) * c.gq):
                qr = q[c.starts[b]:c.starts[b] + n, j] @ c.R_k[h].astype(np.float64) / np.sqrt(D) * np.log2(np.e)
                x = qr @ kc[:, h].T
                parts = x ** 2
                for g in range(ng):
                    s = slice(g * c.group, (g + 1) * c.group)
                    Q = qr[:, s].sum(1)[:, None] * z[None, :, g]
                    parts += (qr[:, s] @ kc[:, h, s].T - Q) ** 2 + Q ** 2
                x = np.where(np.arange(ctx) < ctx - n + np.arange(n)[:, None] + 1, x, -np.inf)
                p = np.exp2(x - x.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                w += p.sum(0)
                e += (p * (2 * np.log(2) * np.sqrt(8 / 3) * 2.0 ** -24 * np.sqrt(parts) + 2.0 ** -22)).sum(0)
            want, off = want + (w ** 2).sum(), off + (e ** 2).sum()
    return np.sqrt(want), np.sqrt(off)


@pytest.mark.parametrize("seqs,heads,gq,group", [
    ([(1, 31)] * 6, 2, 4, 32), ([(1, 400)] * 4, 2, 4, 128), ([(1, 900), (1, 700)], 4, 5, 32), ([(1, 2000)] * 2, 2, 8, 128),
    ([(1, 1500)] * 4, 2, 1, 32), ([(2, 600)] * 3, 2, 3, 32), ([(12, 600)] * 2, 2, 4, 32), ([(12, 600)] * 2, 2, 4, 128)])
def test_typical_errors_are_those_of_fp32(seqs, heads, gq, group):
    """The worst case above leaves room for terms that lose bits everywhere; the norm of the error does not."""
    c = calls(seqs, heads, gq, group, seed=31, first=True)
    ref, _ = c.reference()
    want, most = typical_error(c)
    for max_ctx in (c.max_ctx, LONG):
        got = c.call(max_ctx=max_ctx, out=torch.zeros(c.shape, device="cuda")).double().cpu().numpy()
        err = np.sqrt(((got - ref) ** 2).sum())
        print(f"max_ctx {max_ctx}: {err / want:.2e} of the weights, {err / most:.3f} of the bound")
        assert err <= most, (max_ctx, err / want, most / want)
