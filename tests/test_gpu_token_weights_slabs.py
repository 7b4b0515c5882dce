"""int2kv_token_weights for prompts whose row tiles are taken in slabs: the sums are those of calls over parts of the prompt, which have
room at once."""
import numpy as np
import pytest
import torch

from _tokens import K, WeightsCall, dev

pytestmark = pytest.mark.gpu

SEQS = [(300, 500), (22001, 29000), (0, 700), (1, 20), (40, 300)]
LONG = 1
HEADS, GQ = 2, 16


@pytest.fixture(scope="module", params=[32, 128])
def prompt(request):
    return WeightsCall(SEQS, HEADS, GQ, request.param, seed=request.param)


def in_parts(c, step, decay):
    """fp64 sums from calls over `step` tokens of the long prompt at a time, and the other sequences' from a call of their own."""
    cache = K.Int2KVCache(c.pool.shape[0], HEADS, pool=dev(c.pool), group_size=c.group)
    w = torch.where(torch.arange(c.max_ctx, device="cuda") < dev(c.lens)[:, None, None], dev(c.w).double(), 0.0)
    got = decay * w
    q, R = c.q.cuda(), dev(c.R_k)
    starts = [int(x) for x in c.starts]
    for b, (n, ctx) in enumerate(SEQS):
        for a in range(0, n, step):
            m = min(step, n - a)
            lens = dev(np.array([ctx - n + a + m], np.int32))
            rows = q[starts[b] + a:starts[b] + a + m]
            assert K.int2kv_token_weights_workspace_bytes(1, c.Hq, HEADS, m, m, ctx) < 1 << 30
            x = K.int2kv_token_weights(cache, rows, dev(np.array([0, m], np.int32)), m, dev(c.table[b:b + 1]), lens, ctx, R)
            got[b, :, :ctx] += x[0].double()
    return got.cpu().numpy()


def test_slabs_are_the_sums_of_parts(prompt):
    """Both add the same numbers up: a part's row tiles are the prompt's (its first token is even, a tile has 32 rows, two tokens), and a
    row's statistics and a token's terms do not depend on the others. A sum of positive terms is off by at most its number of additions
    times 2^-24: 512 in a chunk's lane, one a chunk (344 for the prompt), three for the halves and the running sum; parts are added up
    in 64 bits. On either side: 2 (512 + 344 + 3) 2^-24."""
    c = prompt
    need = K.int2kv_token_weights_workspace_bytes(len(SEQS), c.Hq, HEADS, c.total, c.max_q, c.max_ctx)
    assert need == 1 << 30  # the bound: slabs
    print(f"\n[slabs] G={c.group}, workspace {need}", flush=True)
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN)
    out = torch.full(c.shape, -3.0, device="cuda")
    c.call(decay=0.75, out=out, workspace=ws[:need])
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0xFF).all())
    want = in_parts(c, 4000, 0.75)
    got = out.double().cpu().numpy()
    for b, (n, ctx) in enumerate(SEQS):
        assert np.all(got[b, :, ctx:] == -3.0)
        err = np.abs(got[b, :, :ctx] - want[b, :, :ctx]) / want[b, :, :ctx]
        print(f"sequence {b}: off by {err.max():.2e}")
        assert err.max() <= 2 * 859 * 2.0 ** -24
        total = got[b, :, :ctx].sum(-1) - 0.75 * c.w[b, :, :ctx].astype(np.float64).sum(-1)
        assert np.all(np.abs(total - n * GQ) <= 2 * 859 * 2.0 ** -24 * (n * GQ + ctx))


def test_slabs_repeat_and_replay(prompt):
    """In place in a captured call, replayed with other lengths and with eager work between the replays."""
    c = prompt
    cache = K.Int2KVCache(c.pool.shape[0], HEADS, pool=dev(c.pool), group_size=c.group)
    lens, out = dev(c.lens), torch.zeros(c.shape, device="cuda")
    need = K.int2kv_token_weights_workspace_bytes(len(SEQS), c.Hq, HEADS, c.total, c.max_q, c.max_ctx)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    args = (cache, c.q.cuda(), dev(c.starts), c.max_q, dev(c.table), lens, c.max_ctx, dev(c.R_k))
    K.int2kv_token_weights(*args, weights=out, decay=0.5, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.int2kv_token_weights(*args, weights=out, decay=0.5, out=out, workspace=ws)
    for step, long_ctx in enumerate((29000, 22001, 25003)):
        now = c.lens.copy()
        now[LONG] = long_ctx
        lens.copy_(dev(now))
        out.copy_(dev(c.w))
        ws.fill_(0xFF)
        graph.replay()
        eager = dev(c.w)
        K.int2kv_token_weights(*args, weights=eager, decay=0.5, out=eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), step
