"""Values of any size that the cache's parameters hold: averages over long contexts, far below and far above 1."""
import numpy as np
import pytest

from _chunk import Chunk, assert_chunk_close

pytestmark = pytest.mark.gpu

# name: sequences (new, cached), KV heads, query heads per KV head
BATCHES = {
    "few, cut": ([(5, 8000), (2, 300)], 1, 4),
    "few, whole": ([(2, 1500)] * 62, 8, 2),
    "narrow, cut": ([(24, 4000), (30, 10)], 2, 4),
    "narrow, whole": ([(30, 1200)] * 34, 8, 4),
    "wide, cut": ([(100, 6000)], 1, 4),
    "wide, whole": ([(140, 1200)] * 12, 8, 4),
}


@pytest.mark.parametrize("cached", [False, True])
@pytest.mark.parametrize("size", [1e-5, 1e-4, 1e-3, 2e4])
@pytest.mark.parametrize("name", BATCHES)
def test_value_sizes(name, size, cached):
    """The tolerance is relative to the row and its spread, so it does not know the values' size. (What the cache holds is
    exact at every size: code * s + z is a multiple of fp16's least number, and below 2^-13 fp16 holds every such multiple.)"""
    seqs, heads, gq = BATCHES[name]
    print(f"\n[small] {name} {size} cached={cached}", flush=True)
    c = Chunk(seqs, heads, gq, 128 if cached else 32, cached, seed=len(name), v_scale=size, blocks=211)
    worst = assert_chunk_close(c.call(), *c.reference(), what=f"{name} {size}")
    print(f"error {worst:.3f} of the tolerance", flush=True)


def test_rows_of_very_different_sizes():
    """Each row has its own size: a sequence of tiny values beside large ones, and rows of zeros."""
    a = Chunk([(9, 600), (9, 600), (9, 600)], 2, 4, cached=True, seed=5, spare=0)
    v = a.pool[..., 1024 + 64 * 4:].view(np.float16).reshape(a.pool.shape[0], 2, 2, 4, 16)
    for b, size in enumerate((1e-4, 1e4, 0.0)):
        v[a.table[b, :38]] = (v[a.table[b, :38]].astype(np.float64) * size).astype(np.float16)
    ref, spread = a.reference()
    got = a.call()
    assert_chunk_close(got[:18], ref[:18], spread[:18])
    assert bool((got[18:] == 0).all())
