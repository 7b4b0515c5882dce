"""Attention of a chunk of new tokens over the INT2 cache against the fp64 definition: both forms, head layouts, lengths
from nothing to several tiles and pieces, views, padding, masked and non-finite places, streams and graphs."""
import numpy as np
import pytest
import torch

from paper_2608_02691_amd import int2kv as K

from _chunk import Chunk, PAGE, assert_chunk_close

pytestmark = pytest.mark.gpu

# (new, cached) tokens: single tokens, borders of pages, units and tiles, empty sequences and contexts
SEQS = {
    "one": [(1, 1)],
    "one-fresh": [(1, 0)],
    "draft": [(5, 1011)],
    "borders": [(2, 17), (8, 64), (1, 63), (3, 65), (4, 16), (7, 128)],
    "holes": [(65, 129), (0, 30), (200, 77), (0, 0)],
    "fresh": [(300, 0), (17, 500)],
    "pieces": [(3, 5000), (1, 300), (6, 2049)],
    "tiles": [(129, 1500), (64, 64)],
}


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("heads,gq", [(2, 4), (1, 1), (3, 5), (1, 12)])
@pytest.mark.parametrize("cached", [False, True])
@pytest.mark.parametrize("name", SEQS)
def test_matches_definition(name, cached, heads, gq, group):
    print(f"\n[chunk] {name} cached={cached} H={heads} G_q={gq} G={group}", flush=True)
    c = Chunk(SEQS[name], heads, gq, group, cached, seed=len(name) + heads)
    worst = assert_chunk_close(c.call(), *c.reference(), what=name)
    print(f"error {worst:.3f} of the tolerance", flush=True)


@pytest.mark.parametrize("n", [15, 16, 17, 31, 32, 33, 63, 64, 65, 257])
def test_row_tiles(n):
    """Chunk lengths around every tile size (rows per tile 64, 128, 256; four rows a token)."""
    for cached in (False, True):
        c = Chunk([(n, 70 + n), (1, n)], 2, 4, cached=cached, seed=n)
        assert_chunk_close(c.call(), *c.reference(), what=f"{n} {cached}")


def test_more_new_than_cached_tokens():
    """The cached form with lengths that do not hold the chunk: tokens that see nothing get zeros."""
    c = Chunk([(20, 7), (3, 0), (4, 4), (90, 80)], 2, 4, cached=True, seed=3)
    ref, spread = c.reference()
    assert (spread == 0).sum() == (13 + 3 + 10) * 8
    assert_chunk_close(c.call(), ref, spread)


def test_views_and_padding():
    """Views of a fused projection; rows behind the last sequence keep what they held."""
    c = Chunk([(33, 100), (5, 0), (40, 300)], 2, 4, seed=5, pad=7, fused=True)
    out = torch.full((c.total, c.Hq, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    got = c.call(out=out)
    assert got is out and bool((out[-7:] == 3.0).all())
    ref, spread = c.reference()
    assert_chunk_close(out[:-7], ref[:-7], spread[:-7])


def test_blocks_outside_the_cache_are_skipped():
    for cached in (False, True):
        c = Chunk([(20, 200), (3, 90)], 2, 4, cached=cached, seed=6)
        c.table[0, 3], c.table[0, 7], c.table[1, 0] = -1, c.pool.shape[0], 2 ** 31 - 1
        assert_chunk_close(c.call(), *c.reference())


def test_lengths_are_clamped():
    """Context lengths beyond max_ctx and the table, sequences beyond max_q."""
    c = Chunk([(20, 200), (9, 90)], 2, 4, seed=7)
    ref, spread = c.reference()
    c.lens[:] = [2 ** 30, -5]
    c.seqs = [(20, 208), (9, 0)]
    c.table = c.table[:, :13]
    c.table[0, 12] = 0
    assert_chunk_close(c.call(max_ctx=1 << 20), *c.reference())
    d = Chunk([(20, 64)], 1, 4, seed=8)
    out = torch.full((20, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    d.call(out=out, max_q=11)
    ref, spread = d.reference()
    assert_chunk_close(out[:11], ref[:11], spread[:11])
    assert bool((out[11:] == 3.0).all())


def _meta(pool, group):
    """Views of a pool's fp16 parameters: K (s, z) [nb, H, 16, ng, 2] and V [nb, H, (s, z), ng, 16]."""
    ng = 128 // group
    nb, H, _ = pool.shape
    k = pool[..., 1024:1024 + 64 * ng].view(np.float16).reshape(nb, H, PAGE, ng, 2)
    v = pool[..., 1024 + 64 * ng:].view(np.float16).reshape(nb, H, 2, ng, PAGE)
    return k, v


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("cached", [False, True])
def test_stale_slots_hold_anything(cached, group):
    """NaN and infinities in slots behind a sequence's end and in pages that do not exist reach nobody."""
    c = Chunk([(5, 37), (70, 203)], 2, 4, group, cached, seed=9)
    c.table[1, 4] = -1
    ref, spread = c.reference()
    k, v = _meta(c.pool, group)
    for b, (_, ctx) in enumerate(c.seqs):
        page, t = c.table[b, ctx // PAGE], ctx % PAGE
        k[page, :, t:], v[page, :, :, :, t:] = np.nan, np.inf
    spare = sorted(set(range(c.pool.shape[0])) - set(c.table.reshape(-1).tolist()))
    k[spare], v[spare] = np.inf, np.nan
    if 0 in spare:
        k[0], v[0] = np.inf, np.nan
    assert_chunk_close(c.call(), ref, spread)


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("what", ["key", "value"])
@pytest.mark.parametrize("cached", [False, True])
def test_a_token_that_is_not_finite_reaches_only_those_that_see_it(cached, what, value):
    n, at = 90, 70
    c = Chunk([(n, 150 if cached else 40), (6, 100)], 2, 4, cached=cached, seed=10)
    ref, spread = c.reference()
    if cached:
        tok = 150 - n + at
        k, v = _meta(c.pool, 32)
        if what == "key":
            k[c.table[0, tok // PAGE], :, tok % PAGE] = value
        else:
            v[c.table[0, tok // PAGE], :, 1, :, tok % PAGE] = value
    else:
        (c.k if what == "key" else c.v)[at] = float(value)
    got = c.call().float().cpu().numpy()
    keep = np.r_[0:at, n:n + 6]
    assert_chunk_close(got[keep], ref[keep], spread[keep])
    if what == "value" or np.isnan(value):
        assert not np.isfinite(got[at:n]).all(axis=-1).any()


def test_large_values_and_sharp_scores():
    """Values to a few thousand, scores of some hundreds: the running maximum moves often."""
    c = Chunk([(40, 700), (3, 2000)], 2, 4, seed=11, k_scale=1.0, v_scale=1500.0)
    assert_chunk_close(c.call(), *c.reference())
    # scores ascend along the context, so every unit moves the maximum: q is a multiple of one direction, keys grow along it
    d = Chunk([(40, 0)], 1, 4, seed=12)
    u = np.random.default_rng(1).choice([-1.0, 1.0], 128)
    d.mu[:] = 0
    d.q = torch.from_numpy(np.broadcast_to(u, (40, 4, 128)).copy()).to(torch.bfloat16)
    d.k = torch.from_numpy((np.arange(40)[:, None, None] * 0.25 * u)).to(torch.bfloat16).expand(40, 1, 128).contiguous()
    assert_chunk_close(d.call(), *d.reference())


def test_zero_and_tiny_queries():
    c = Chunk([(9, 130)], 2, 4, seed=13)
    c.q[0] = 0
    c.q[1] = 1e-30
    c.q[2] *= 1e-4
    c.q[3, :, 5] = 2000.0
    c.q[3] *= 1e-3
    assert_chunk_close(c.call(), *c.reference())


@pytest.mark.parametrize("group", [32, 128])
def test_single_tokens_equal_the_decode(group):
    """One cached token a sequence: int2kv_decode, up to both sides' roundings (2e-3 of the row for the decode's bar)."""
    c = Chunk([(1, n) for n in (1, 16, 100, 900, 0)], 2, 4, group, True, seed=14)
    got = c.call().float().cpu().numpy().astype(np.float64)
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    cache = K.Int2KVCache(c.pool.shape[0], 2, pool=dev(c.pool), group_size=group)
    dec = K.int2kv_decode(cache, c.q.cuda(), dev(c.table), dev(c.lens), c.max_ctx, dev(c.R_k), dev(c.R_v)).cpu().numpy()
    ref, spread = c.reference()
    err = np.linalg.norm(got - dec, axis=-1)
    assert np.all(err <= 2.0 ** -7 * (np.linalg.norm(ref, axis=-1) + spread) + 2e-3 * np.sqrt(128) * np.linalg.norm(ref, axis=-1))


def test_repeats_bit_for_bit_on_any_stream_and_in_graphs():
    c = Chunk([(37, 900), (3, 4000), (100, 0)], 2, 4, seed=15)
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    cache = K.Int2KVCache(c.pool.shape[0], 2, pool=dev(c.pool), group_size=32)
    q, k, v = c.q.cuda(), c.k.cuda(), c.v.cuda()
    rest = (dev(c.table), dev(c.lens), c.max_ctx, dev(c.R_k), dev(c.R_v), k, v, dev(c.mu))
    starts = dev(c.starts)
    need = K.int2kv_chunk_attention_workspace_bytes(3, 8, 2, c.total, c.max_q, c.max_ctx)
    ws = [torch.full((need,), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(3)]
    outs = [torch.zeros((c.total, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    call = lambda i: K.int2kv_chunk_attention(cache, q, starts, c.max_q, *rest, out=outs[i], workspace=ws[i])  # noqa: E731
    first = call(0).clone()
    assert_chunk_close(first, *c.reference())
    ws[0].fill_(0xFF)
    assert torch.equal(call(0), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(1)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(outs[1], first)
    graphs = []
    for i in (1, 2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i)
        graphs.append(g)
    for turn in range(3):
        q.copy_(c.q.cuda() * (1 + turn))  # new inputs in place, an eager call beside the replays
        want = call(0).clone()
        outs[1].zero_(), outs[2].zero_()
        graphs[0].replay()
        graphs[1].replay()
        assert torch.equal(outs[1], want) and torch.equal(outs[2], want), turn
        torch.cuda.synchronize()


def test_far_pages():
    """Records beyond 2^32 bytes of the pool."""
    blocks = (1 << 32) // 1536 + 4000
    c = Chunk([(6, 100), (40, 60)], 1, 4, seed=16)
    small = torch.from_numpy(c.pool).cuda()
    pool = torch.zeros((blocks, 1, 1536), dtype=torch.uint8, device="cuda")
    pool[-c.pool.shape[0]:] = small
    ref = c.reference()
    c.table = np.where(c.table >= 0, c.table + (blocks - c.pool.shape[0]), -1).astype(np.int32)
    cache = K.Int2KVCache(blocks, 1, pool=pool)
    assert_chunk_close(c.call(cache=cache), *ref)


def test_many_sequences():
    """More sequences than a planning pass holds, lengths from nothing on."""
    rng = np.random.default_rng(17)
    seqs = [(int(rng.integers(0, 4)), int(rng.integers(0, 40))) for _ in range(700)]
    for cached in (False, True):
        c = Chunk(seqs, 1, 4, cached=cached, seed=18)
        assert_chunk_close(c.call(), *c.reference())


def test_overlapping_offsets_stay_in_bounds():
    """Offsets that descend or overlap are no valid batch: the call stays within its buffers and ends."""
    c = Chunk([(30, 50)] * 4, 1, 4, seed=19)
    c.starts = np.array([0, 120, 0, 120, -7], np.int32)
    c.call(max_q=120)
    c.starts = np.array([5, 5, 900, 3, 120], np.int32)
    c.call(max_q=120)
    torch.cuda.synchronize()
