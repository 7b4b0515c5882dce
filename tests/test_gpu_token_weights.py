"""The weight that cached tokens receive (int2kv_token_weights) against its definition in fp64."""
import numpy as np
import pytest
import torch

from _tokens import K, WeightsCall, assert_weights_close, dev

pytestmark = pytest.mark.gpu


def check(call, what, **kw):
    ref, tol = call.reference()
    got = call.call(**kw)
    torch.cuda.synchronize()
    worst = assert_weights_close(got, ref, tol, what)
    print(f"{what}: {worst:.3f} of the tolerance")
    return got


@pytest.mark.parametrize("heads,gq", [(1, 1), (2, 4), (2, 5), (8, 4), (1, 8), (1, 12), (1, 16), (3, 2)])
@pytest.mark.parametrize("group", [32, 128])
def test_decode_steps(heads, gq, group):
    """One token a sequence; a sequence without one; lengths of one and around pages and ranges."""
    seqs = [(1, 1), (1, 100), (0, 33), (1, 255), (1, 256), (1, 257), (1, 16), (1, 515)]
    check(WeightsCall(seqs, heads, gq, group, seed=gq, pad=1, fused=gq == 4), f"{heads} x {gq}, {group}")


@pytest.mark.parametrize("n,ctx", [(3, 4500), (20, 3000), (64, 2500), (64, 5), (2, 2), (2, 300), (7, 40), (8, 8), (9, 500), (31, 33), (32, 32), (33, 700), (64, 64), (65, 1030), (150, 150), (200, 201)])
@pytest.mark.parametrize("gq", [1, 4, 5])
def test_several_tokens(n, ctx, gq):
    check(WeightsCall([(n, ctx), (1, 70)], 1, gq, 32 if n % 2 else 128, seed=n), f"{n} of {ctx} x {gq}")


def test_ragged_prompts():
    seqs = [(300, 300), (0, 0), (1, 1), (57, 400), (0, 90), (128, 1300), (2, 3)]
    check(WeightsCall(seqs, 2, 4, seed=3, pad=4, wide=7), "ragged")


def test_long_context():
    check(WeightsCall([(1, 9001), (3, 5000)], 2, 4, seed=4), "long")
    check(WeightsCall([(40, 9001), (3, 5000)], 1, 4, seed=5), "long, many rows")


def test_first_sums_and_decay():
    c = WeightsCall([(3, 60), (1, 300)], 2, 4, seed=6, first=True)
    check(c, "first")
    c = WeightsCall([(3, 60), (1, 300)], 2, 4, seed=6)
    for decay in (0.0, 1.0, -0.5):
        ref, tol = c.reference(decay)
        assert_weights_close(c.call(decay=decay), ref, tol, f"decay {decay}")
    # without a token the sums decay
    got = c.call(decay=0.5, max_q=0)
    for b, n in enumerate((60, 300)):
        assert torch.equal(got[b, :, :n], dev(c.w)[b, :, :n] * 0.5)


def test_in_place_and_untouched_places():
    c = WeightsCall([(2, 50), (1, 130)], 2, 4, seed=7, wide=9)
    ref, tol = c.reference()
    w = dev(c.w)
    before = w.clone()
    got = c.call(weights=w, out=w)
    assert got.data_ptr() == w.data_ptr()
    for b, n in enumerate((50, 130)):
        assert_weights_close(w[b, :, :n], ref[b, :, :n], tol[b, :, :n], "in place")
        assert torch.equal(w[b, :, n:], before[b, :, n:])


def test_tokens_in_missing_pages_receive_nothing():
    c = WeightsCall([(3, 200), (1, 40), (40, 300)], 2, 4, seed=8, first=True)
    c.table[0, 3], c.table[0, 11], c.table[1, :], c.table[2, 2] = -1, 1 << 30, -7, 1 << 29
    got = check(c, "missing pages")
    assert torch.count_nonzero(got[1]) == 0 and torch.count_nonzero(got[0, :, 48:64]) == 0


def test_stale_slots_do_not_count():
    """Parameters behind a length, and those of other blocks, may hold anything."""
    c = WeightsCall([(3, 21), (1, 40)], 1, 4, seed=9)
    ref, tol = c.reference()
    for b, n in enumerate((21, 40)):
        rec = c.pool[c.table[b, n // 16], 0]
        for t in range(n % 16, 16):
            rec[1024 + 16 * t:1024 + 16 * t + 16] = 0xFF  # NaN
    c.pool[[x for x in range(c.pool.shape[0]) if x not in c.table], 0, 1024:] = 0xFF
    assert_weights_close(c.call(), ref, tol, "stale slots")


def test_more_queries_than_cached_tokens():
    """A length that does not hold the sequence: its first tokens see nothing."""
    check(WeightsCall([(10, 4), (3, 0), (40, 33)], 1, 4, seed=10), "short lengths")


def test_cut_sequences_keep_their_place():
    """max_q, max_ctx and the table cut; a token sees what it saw of what is left."""
    c = WeightsCall([(20, 100)], 1, 4, seed=11, first=True)
    q = c.q.clone()
    c.q[6:] = 0
    full = c.seqs
    part = WeightsCall([(20, 100)], 1, 4, seed=11, first=True)
    part.q, part.seqs = q[:6], [(6, 86)]  # the first six of twenty: they see 81 .. 86 tokens
    ref, tol = part.reference()
    c.q, c.seqs = q, full
    got = c.call(max_q=6)
    assert_weights_close(got[:, :, :86], ref[:, :, :86], tol[:, :, :86], "max_q")
    assert torch.count_nonzero(got[:, :, 86:]) == 0
    # the last tokens, all beyond the cut, see all that is left
    c2 = WeightsCall([(4, 100)], 1, 4, seed=12, first=True)
    got = c2.call(max_ctx=64)
    c2.table[0, 4:] = -1
    ref, tol = c2.reference()
    assert_weights_close(got, ref[:, :, :64], tol[:, :, :64], "max_ctx")


@pytest.mark.parametrize("n", [1, 12])
@pytest.mark.parametrize("q_scale,k_scale", [(30.0, 4.0), (0.01, 1.0), (1e-4, 100.0), (200.0, 0.01)])
def test_sizes_of_scores(q_scale, k_scale, n):
    """Peaked rows, flat rows, rows of very different scores."""
    c = WeightsCall([(n, 700), (n, 90)], 1, 4, seed=13, q_scale=q_scale, k_scale=k_scale)
    c.q[0, 1] *= 0.001
    check(c, f"{q_scale}, {k_scale}")


@pytest.mark.parametrize("n,pad", [(2, 0), (12, 0), (70, 0), (70, 5)])
def test_only_late_pages_exist(n, pad):
    """Rows whose every score lies far from zero, and none over the first tokens: their weights still sum to one."""
    c = WeightsCall([(n, 900), (n, 300)], 1, 4, seed=19, q_scale=30.0, k_scale=4.0, first=True)
    c.table[0, :-4 - (n + 15) // 16] = -1  # rows see the last pages only: from one token to n
    c.table[1, :] = np.where(np.arange(c.table.shape[1]) == 12 + pad, c.table[1], -1)
    got = check(c, "late pages")
    assert abs(float(got[0].double().sum()) - 4 * n) < 1e-3 * n


@pytest.mark.parametrize("n", [1, 10])
def test_the_maximum_moves_far(n):
    """Scores that rise by hundreds along the context, and fall again."""
    c = WeightsCall([(n, 1200)], 1, 4, seed=14, q_scale=8.0, first=True)
    rise = np.concatenate([np.linspace(0.1, 8, 600), np.linspace(8, 0.1, 600)]).astype(np.float16)
    for t in range(1200):
        rec = c.pool[c.table[0, t // 16], 0]
        m = rec[1024 + 16 * (t % 16):1040 + 16 * (t % 16)].view(np.float16)
        m *= rise[t]
    check(c, "moving maximum")


def test_total_weight():
    """Each row's weights sum to one."""
    c = WeightsCall([(37, 1000)], 2, 4, seed=15, first=True)
    got = c.call().double().sum(-1).cpu()
    assert torch.allclose(got, torch.full_like(got, 37 * 4), rtol=1e-5)


@pytest.mark.parametrize("n", [1, 20])
def test_streams_and_graphs(n):
    a, b = WeightsCall([(n, 900), (n, 70)], 2, 4, seed=16), WeightsCall([(n, 900), (n, 70)], 2, 4, seed=17)
    refs = [x.reference() for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for x, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            outs.append(x.call())
    torch.cuda.synchronize()
    for o, (ref, tol) in zip(outs, refs):
        assert_weights_close(o, ref, tol, "streams")
    cache = K.Int2KVCache(a.pool.shape[0], a.H, pool=dev(a.pool), group_size=a.group)
    lens, w, out = dev(a.lens), dev(a.w), torch.zeros(a.shape, dtype=torch.float32, device="cuda")
    ws = torch.empty(K.int2kv_token_weights_workspace_bytes(2, a.Hq, a.H, a.total, a.max_q, a.max_ctx), dtype=torch.uint8, device="cuda")
    args = (cache, a.q.cuda(), dev(a.starts), a.max_q, dev(a.table), lens, a.max_ctx, dev(a.R_k))
    K.int2kv_token_weights(*args, weights=w, decay=0.75, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.int2kv_token_weights(*args, weights=w, decay=0.75, out=out, workspace=ws)
    for step, ctx in enumerate(((900, 70), (555, 1), (n, n), (899, 64))):
        a.seqs, a.lens = [(n, c) for c in ctx], np.array(ctx, np.int32)
        lens.copy_(dev(a.lens))
        out.zero_()
        graph.replay()
        eager = a.call(max_ctx=900, out=torch.zeros_like(out))
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        assert_weights_close(out, *a.reference(), f"replay {step}")


def test_bitwise_repeatable():
    for n in (1, 130):
        c = WeightsCall([(n, 2500), (n, 300)], 2, 4, seed=18)
        first = c.call()
        assert all(torch.equal(first, c.call()) for _ in range(3))
