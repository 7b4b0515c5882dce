"""int2kv_token_weights with block tables that end before the lengths do: tokens behind them lie in no block. Their sums decay, and they
receive nothing."""
import numpy as np
import pytest
import torch

from _tokens import K, WeightsCall, assert_weights_close, dev

pytestmark = pytest.mark.gpu


# name: new and cached tokens, columns that are left, max_ctx: one launch, pieces, pieces of many sequences, many rows, in several chunks
FORMS = {
    "one launch": ([(1, 300), (2, 90), (0, 200), (1, 1)], 5, None),
    "one launch, one column": ([(1, 1000), (1, 7), (2, 17)], 1, None),
    "pieces": ([(1, 300), (2, 90), (0, 200), (1, 1)], 5, 2500),
    "pieces, long": ([(2, 5000), (1, 1400)], 70, None),
    "pieces, many sequences": ([(1, 2100 - 9 * i) for i in range(80)], 67, None),
    "many rows": ([(12, 300), (3, 90), (0, 200), (40, 40)], 5, None),
    "many rows, one column": ([(20, 600), (3, 8)], 1, None),
    "many rows, chunks": ([(200, 700), (64, 130)], 20, None),
    "no rows": ([(0, 100), (0, 40)], 3, None),
}


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("name", FORMS)
def test_tables_that_end_early(name, group):
    seqs, columns, max_ctx = FORMS[name]
    print(f"\n[table] {name} G={group}", flush=True)
    heads = 4 if "many sequences" in name else 1
    top = max(c for _, c in seqs)
    c = WeightsCall(seqs, heads, 4, group, seed=columns, wide=(max_ctx or top) - top)
    c.table[:, columns:] = -1
    ref, tol = c.reference()
    c.table = np.ascontiguousarray(c.table[:, :columns])
    for in_place in (False, True):
        w = dev(c.w)
        out = w if in_place else torch.full(c.shape, -3.0, device="cuda")
        c.call(max_ctx=max_ctx or top, weights=w, out=out)
        for b, (_, n) in enumerate(seqs):
            assert_weights_close(out[b, :, :n], ref[b, :, :n], tol[b, :, :n], f"{name}, {b}")
            assert torch.equal(out[b, :, n:], dev(c.w)[b, :, n:] if in_place else torch.full_like(out[b, :, n:], -3.0))


@pytest.mark.parametrize("n", [1, 30])
def test_selection_after_a_short_table(n):
    """What int2kv_select_tokens ranks are the decayed sums, not what an output held before."""
    c = WeightsCall([(n, 400)], 2, 4, seed=n)
    c.w[:, :, 200:] += 50.0
    c.table = np.ascontiguousarray(c.table[:, :10])
    out = c.call(decay=0.5)
    kept, lens = K.int2kv_select_tokens(out, dev(c.lens), 400, 200)
    assert int(lens[0]) == 200 and torch.equal(kept[0, 0].cpu(), torch.arange(200, 400, dtype=torch.int32))
