"""The largest sizes that the operators around the decode step accept, and the first they refuse (CPU only): a launch holds
2^32 - 1 threads. Accepted sizes come with a pointer missing, so nothing is launched."""
import pytest

from paper_2608_02691_amd import int2kv as K

from test_abi_chunk import _read, _rope


@pytest.mark.parametrize("heads", [dict(hq=0, q=None, qo=None), dict(hk=0, k=None, ko=None), {}])
def test_rope_axes_fills_a_launch(heads):
    """Blocks of 256 threads take eight tokens: 2^24 - 1 blocks."""
    st, msg = _rope(n=(1 << 27) - 8, pos=None, **heads)
    assert st == K.INT2KV_EINVAL and b"NULL" in msg
    for n in ((1 << 27) - 7, (1 << 27) - 1):
        st, msg = _rope(n=n, pos=None, **heads)
        assert st == K.INT2KV_EUNSUPPORTED and b"num_tokens" in msg


@pytest.mark.parametrize("heads", [1, 2, 16])
def test_read_rows_fills_a_launch(heads):
    """Blocks of 256 threads take sixteen rows as stored: 2^24 - 1 blocks."""
    cache = K._Cache(16, 4, heads, 16, 128, 32)
    most = ((1 << 28) - 16) // heads
    st, msg = _read(cache=cache, n=most, slots=None)
    assert st == K.INT2KV_EINVAL and b"NULL" in msg
    for n in (most + 1, ((1 << 28) - 1) // heads):
        if n > most:
            st, msg = _read(cache=cache, n=n, slots=None)
            assert st == K.INT2KV_EUNSUPPORTED and b"num_tokens" in msg
