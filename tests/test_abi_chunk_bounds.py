"""The largest sizes that the operators around the decode step accept, and the first they refuse (CPU only): a launch holds
2^32 - 1 threads. Accepted sizes come with a pointer missing, so nothing is launched."""
import pytest

from paper_2608_02691_amd import int2kv as K

from test_abi_chunk import _rope


@pytest.mark.parametrize("heads", [dict(hq=0, q=None, qo=None), dict(hk=0, k=None, ko=None), {}])
def test_rope_axes_fills_a_launch(heads):
    """Blocks of 256 threads take eight tokens: 2^24 - 1 blocks."""
    st, msg = _rope(n=(1 << 27) - 8, pos=None, **heads)
    assert st == K.INT2KV_EINVAL and b"NULL" in msg
    for n in ((1 << 27) - 7, (1 << 27) - 1):
        st, msg = _rope(n=n, pos=None, **heads)
        assert st == K.INT2KV_EUNSUPPORTED and b"num_tokens" in msg
