"""int2kv_select_tokens: lists that share memory with what the call reads, refused before any launch (CPU only). A work-group each reads
the length of its sequence and writes its list, so none may write what another still reads."""
import pytest

from paper_2608_02691_amd import int2kv as K

# two sequences, two KV heads: weights 4 lists of 64, kept 4 lists of 32 in strides of 40, lengths of two
W, KEPT, LENS, KLENS = 1 << 20, 2 << 20, 3 << 20, 4 << 20


def _select(w=W, kept=KEPT, lens=LENS, klens=KLENS, budget=32):
    st = K.load_library().int2kv_select_tokens(w, 64, 2, 2, lens, 64, budget, 4, 8, kept, 40, klens, None)
    return st, K.load_library().int2kv_last_error()


@pytest.mark.parametrize("kw", [
    dict(klens=LENS), dict(klens=LENS + 4), dict(klens=LENS - 4), dict(kept=LENS), dict(kept=LENS - 4 * (3 * 40 + 31)), dict(kept=LENS + 4),
    dict(kept=W), dict(kept=W + 4 * (3 * 64 + 63)), dict(kept=W - 4 * (3 * 40 + 31)), dict(klens=W + 64), dict(klens=W - 4), dict(klens=KEPT),
    dict(klens=KEPT + 4 * (3 * 40 + 31)), dict(klens=KEPT - 4)])
def test_outputs_over_inputs_are_refused(kw):
    st, msg = _select(**kw)
    assert st == K.INT2KV_EINVAL and b"overlap" in msg, msg


@pytest.mark.parametrize("kw", [
    dict(kept=W + 4 * 24), dict(kept=W + 4 * (64 - 1)), dict(kept=W - 4), dict(klens=W + 4 * 63), dict(klens=W + 4 * (64 + 39) - 4), dict(klens=W - 4)])
def test_lists_in_gaps_that_are_too_small(kw):
    """Lists of one stride, a list of new lengths: the weights' gaps do not hold them."""
    st = K.load_library().int2kv_select_tokens(W, 64, 2, 2, LENS, 40, 25, 4, 8, kw.get("kept", KEPT), 64, kw.get("klens", KLENS), None)
    assert st == K.INT2KV_EINVAL and b"overlap" in K.load_library().int2kv_last_error()
