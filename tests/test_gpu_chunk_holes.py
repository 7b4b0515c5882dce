"""Values that are not finite behind pages that do not exist: they reach every token that sees them, and no other."""
import numpy as np
import pytest

from _chunk import Chunk, assert_chunk_close
from test_gpu_chunk import _meta

pytestmark = pytest.mark.gpu

# name: sequences, tokens, cached tokens, KV heads, query heads per KV head. Many sequences, so that no tile is cut and a wave
# of the kernel of few rows has several 64-token units
BATCHES = {"few": (62, 2, 1500, 8, 4), "narrow": (40, 30, 700, 8, 4), "wide": (12, 130, 700, 8, 2), "listed": (66, 2, 1100, 8, 4)}


@pytest.mark.parametrize("cached", [False, True])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("name", BATCHES)
def test_values_behind_a_hole(name, group, cached):
    """A missing page in unit u of a sequence, an infinite value in unit u + 1 or u + 2, which every row sees all of."""
    B, n, ctx, heads, gq = BATCHES[name]
    print(f"\n[hole] {name} cached={cached} G={group}", flush=True)
    c = Chunk([(n, ctx)] * B, heads, gq, group, cached, seed=B)
    whole = (ctx - n) // 64  # units that all rows see all of
    struck = []
    _, v = _meta(c.pool, group)
    for b in range(B):
        u = b % (whole - 2)
        c.table[b, 4 * u + b % 4] = -1
        if b % 3:
            struck.append(b)
    ref, spread = c.reference()
    for b in struck:
        tok = 64 * (b % (whole - 2) + b % 3) + (7 * b) % 64
        v[c.table[b, tok // 16], :, 1, :, tok % 16] = np.inf
    got = c.call().float().cpu().numpy()
    hit = np.repeat(np.isin(np.arange(B), struck), n)
    assert_chunk_close(got[~hit], ref[~hit], spread[~hit])
    assert not np.isfinite(got[hit]).all(-1).any()
