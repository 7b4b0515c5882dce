"""How the attention of a chunk is laid out over the chip: every kernel of it with whole and cut tiles, all on the chip at
once and one after another, batches planned by every work-group and by a launch of their own;
workspaces to the byte, streams, strides."""
import numpy as np
import pytest
import torch

from paper_2608_02691_amd import int2kv as K

from _chunk import Chunk, assert_chunk_close
from test_gpu_chunk import _meta

pytestmark = pytest.mark.gpu


def _ragged(n, new, ctx, seed):
    rng = np.random.default_rng(seed)
    return [(int(rng.integers(*new)), int(rng.integers(*ctx))) for _ in range(n)]


# name: sequences (new, cached), KV heads, query heads per KV head
PLANS = {
    "few, cut": ([(5, 6000)], 1, 4),
    "few, a ragged batch": (_ragged(24, (2, 9), (100, 6000), 1), 8, 5),
    "few, more tiles than places": (_ragged(60, (1, 8), (1500, 5500), 2), 12, 5),
    "few, listed and cut": (_ragged(70, (1, 4), (0, 5000), 3), 1, 4),
    "few, listed, long steps": (_ragged(66, (1, 3), (4500, 5000), 4), 8, 1),
    "few, one long sequence among many": ([(3, 50)] * 70 + [(120, 3000)], 2, 4),
    "few, one prompt among single tokens": ([(1, 700)] * 30 + [(300, 0)], 2, 4),
    "narrow": (_ragged(20, (17, 33), (0, 900), 5), 8, 4),
    "narrow, cut": ([(24, 4000), (30, 10)], 2, 4),
    "narrow, listed": (_ragged(80, (12, 33), (0, 300), 6), 2, 4),
    "narrow, nothing cached": ([(700, 0), (33, 0)], 8, 4),
    "narrow, more tiles than places": (_ragged(40, (50, 130), (0, 700), 7), 8, 4),
    "narrow, nothing cached, more tiles than places": (_ragged(40, (50, 130), (0, 1), 9), 8, 4),
    "narrow, listed, ragged": (_ragged(66, (0, 140), (0, 500), 8), 2, 4),
    "wide, nothing cached": (_ragged(20, (180, 300), (0, 1), 10), 8, 4),
    "wide, cut": ([(100, 6000)], 1, 4),
    "wide, cut over the chunk's own tokens": ([(700, 100)], 1, 2),
    "wide, more tiles than places": (_ragged(20, (180, 300), (0, 700), 11), 8, 4),
    "wide, tiles by their own length": ([(250, 900), (64, 20), (130, 300), (190, 2500)], 8, 4),
    "wide, listed": (_ragged(66, (150, 250), (0, 500), 12), 1, 4),
}


@pytest.mark.parametrize("cached", [False, True])
@pytest.mark.parametrize("name", PLANS)
def test_plans(name, cached):
    seqs, heads, gq = PLANS[name]
    print(f"\n[plan] {name} cached={cached} sequences {len(seqs)} H={heads} G_q={gq}", flush=True)
    c = Chunk(seqs, heads, gq, 128 if heads == 12 else 32, cached, seed=len(name), blocks=97)
    need = K.int2kv_chunk_attention_workspace_bytes(len(seqs), c.Hq, heads, c.total, c.max_q, c.max_ctx)
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")  # (as floats: NaN)
    got = c.call(workspace=ws[:need])
    ref, spread = c.reference()
    worst = assert_chunk_close(got, ref, spread, what=name)
    assert bool((ws[need:] == 0xFF).all())
    assert torch.equal(c.call(workspace=ws[:need]), got)
    print(f"error {worst:.3f} of the tolerance", flush=True)


def test_two_streams_with_workspaces_of_their_own():
    calls = [Chunk(_ragged(9, (1, 40), (0, 2000), s), 2, 4, seed=s, blocks=50) for s in (1, 2)]
    want = [c.call() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    ws = [torch.empty(K.int2kv_chunk_attention_workspace_bytes(9, 8, 2, c.total, c.max_q, c.max_ctx), dtype=torch.uint8,
                      device="cuda") for c in calls]
    outs = [torch.zeros_like(w) for w in want]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, st, w, o in zip(calls, streams, ws, outs):
            with torch.cuda.stream(st):
                c.call(workspace=w, out=o)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert torch.equal(w, o)


def test_wide_strides_and_a_mean_at_any_word():
    """Tokens 2 MB apart; mu where a vector load is not aligned."""
    c = Chunk([(20, 100), (3, 0)], 2, 4, seed=21)
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    far = torch.full((23, 1 << 20), 5.0, dtype=torch.bfloat16, device="cuda")
    q, k, v = (far[:, o:o + n * 128].unflatten(1, (n, 128)) for o, n in ((0, 8), (4096, 2), (8192, 2)))
    q.copy_(c.q), k.copy_(c.k), v.copy_(c.v)
    mu = torch.zeros(2 * 128 + 1, device="cuda")[1:].unflatten(0, (2, 128)).copy_(dev(c.mu))
    cache = K.Int2KVCache(c.pool.shape[0], 2, pool=dev(c.pool))
    got = K.int2kv_chunk_attention(cache, q, dev(c.starts), 20, dev(c.table), dev(c.lens), 100, dev(c.R_k), dev(c.R_v), k, v, mu)
    assert mu.data_ptr() % 16 == 4
    assert_chunk_close(got, *c.reference())


@pytest.mark.parametrize("gq", [1, 4])
def test_values_beyond_fp16_reach_only_the_tokens_that_see_them(gq):
    """code * s + z past 65504 in a unit that some rows see a part of (few rows with gq 1, many with 4)."""
    n, at = 60, 41
    c = Chunk([(n, 150)], 2, gq, cached=True, seed=22)
    ref, spread = c.reference()
    tok = 150 - n + at
    _, v = _meta(c.pool, 32)
    v[c.table[0, tok // 16], :, 0, :, tok % 16] = 60000.0
    got = c.call().float().cpu().numpy()
    assert_chunk_close(got[:at], ref[:at], spread[:at])


@pytest.mark.parametrize("batch", [20, 70])
def test_a_captured_call_plans_by_the_lengths_of_its_replay(batch):
    """Lengths that change in place between replays, an eager call beside each: every work-group's own plan, and the launch's."""
    c = Chunk(_ragged(batch, (1, 30), (0, 1500), 23), 2, 4, seed=23, blocks=60)
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    cache = K.Int2KVCache(c.pool.shape[0], 2, pool=dev(c.pool))
    q, k, v, starts, lens = c.q.cuda(), c.k.cuda(), c.v.cuda(), dev(c.starts), dev(c.lens)
    rest = (dev(c.R_k), dev(c.R_v), k, v, dev(c.mu))
    table = dev(np.where(c.table >= 0, c.table, 0).astype(np.int32))
    need = K.int2kv_chunk_attention_workspace_bytes(batch, 8, 2, c.total, c.max_q, 1600)
    ws = [torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.zeros((c.total, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    call = lambda i: K.int2kv_chunk_attention(cache, q, starts, c.max_q, table, lens, 1600, *rest, out=outs[i], workspace=ws[i])  # noqa: E731
    call(1)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(0)
    rng = np.random.default_rng(24)
    room = table.shape[1] * 16
    for turn in range(5):
        new = np.minimum(rng.integers(0, 1500, batch), room) if turn % 2 else np.where(np.arange(batch) == turn, min(1500, room), 3)
        lens.copy_(dev(new.astype(np.int32)))
        outs[0].zero_()
        g.replay()
        assert torch.equal(call(1), outs[0]), turn
        torch.cuda.synchronize()
