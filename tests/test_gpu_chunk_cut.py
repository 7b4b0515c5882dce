"""Sequences and contexts that a call cuts (max_q, max_ctx, the table's width): what a token sees goes by the whole sequence
and the whole length, in both forms and in every kernel."""
import numpy as np
import pytest
import torch

from _chunk import PAGE, Chunk, assert_chunk_close

pytestmark = pytest.mark.gpu

# name: sequences (new, cached), KV heads, query heads per KV head, the call's max_q
CUTS = {
    "few": ([(20, 64), (7, 300), (3, 2), (30, 900)], 2, 4, 11),
    "few, a token": ([(3, 90), (1, 40), (9, 4000)], 2, 4, 1),
    "narrow": ([(60, 900), (20, 40), (45, 30)], 2, 4, 30),
    "narrow, tiles by their own length": ([(90, 700)], 2, 4, 50),
    "wide": ([(300, 2000), (90, 100)], 2, 4, 200),
    "listed": ([(2 + b % 7, 30 + 5 * b) for b in range(70)], 2, 4, 3),
    "listed, longer": ([(40 + b % 90, 10 + 9 * b) for b in range(70)], 1, 4, 77),
}


def _check(c, max_q, **kw):
    """The first max_q tokens of every sequence as the whole sequence has them, the others' rows as they were."""
    out = torch.full((c.total, c.Hq, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    c.call(out=out, max_q=max_q, **kw)
    ref, spread = c.reference()
    keep = np.concatenate([np.arange(n) < max_q for n, _ in c.seqs])
    assert_chunk_close(out[torch.from_numpy(keep).cuda()], ref[keep], spread[keep])
    assert bool((out[torch.from_numpy(~keep).cuda()] == 3.0).all())


@pytest.mark.parametrize("cached", [True, False])
@pytest.mark.parametrize("name", CUTS)
def test_sequences_beyond_max_q(name, cached):
    seqs, heads, gq, max_q = CUTS[name]
    print(f"\n[cut] {name} cached={cached} max_q={max_q}", flush=True)
    _check(Chunk(seqs, heads, gq, cached=cached, seed=len(name)), max_q)


@pytest.mark.parametrize("cached", [True, False])
@pytest.mark.parametrize("by", ["max_ctx", "table"])
@pytest.mark.parametrize("name", CUTS)
def test_contexts_beyond_the_bounds(name, by, cached):
    """A length beyond max_ctx or the table: its tokens are where the whole length puts them, what is beyond does not exist."""
    seqs, heads, gq, max_q = CUTS[name]
    print(f"\n[cut] {name} cached={cached} by {by}", flush=True)
    c = Chunk(seqs, heads, gq, 128, cached, seed=len(name))
    pages = max(1, c.max_ctx // (2 * PAGE))
    table = c.table.copy()
    c.table = table[:, :pages].copy() if by == "table" else table
    out = torch.full((c.total, c.Hq, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    c.call(out=out, **({"max_ctx": pages * PAGE} if by == "max_ctx" else {}))
    c.table = np.where(np.arange(table.shape[1]) < pages, table, -1).astype(np.int32)  # for the reference: pages that do not exist
    ref, spread = c.reference()
    assert_chunk_close(out, ref, spread)


def test_negative_and_huge_lengths():
    """Lengths outside every bound, in the cached form: nothing below zero, everything the table holds above."""
    c = Chunk([(4, 96), (5, 80), (2, 64)], 2, 4, cached=True, seed=3)
    ref, spread = c.reference()
    full = Chunk([(4, 96), (5, 80), (2, 64)], 2, 4, cached=True, seed=3)
    full.table = full.table[:, :6]
    full.table[1, 5] = full.table[2, 4] = full.table[2, 5] = -1
    full.lens = np.array([2 ** 31 - 1, -2 ** 31, 64], np.int32)
    got = full.call(max_ctx=2 ** 31 - 1)
    # every token of the first sequence sees all six pages: the same as tokens behind them
    first = Chunk([(4, 96 + 4)], 2, 4, cached=True, seed=3)
    first.pool, first.table, first.q, first.R_k, first.R_v = full.pool, np.pad(full.table[:1], ((0, 0), (0, 1)), constant_values=-1), full.q[:4], full.R_k, full.R_v
    r0, s0 = first.reference()
    assert_chunk_close(got[:4], r0, s0)
    assert bool((got[4:9] == 0).all())
    assert_chunk_close(got[9:], ref[9:], spread[9:])
