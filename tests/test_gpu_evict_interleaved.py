"""int2kv_select_tokens on one buffer through the C entry point: weights, kept tokens and lengths of a list side by side, in strides of their own."""
import numpy as np
import pytest
import torch

from _tokens import K, dev, kept_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gap", [0, 5])
def test_lists_in_each_others_gaps(gap):
    """List i: weights, then its kept tokens; lengths, old and new, behind the first list's."""
    B, H, ctx, budget = 2, 3, 300, 100
    stride = ctx + budget + gap + 2 * B
    rng = np.random.default_rng(gap)
    host = np.full((B * H, stride), -7, np.int32)
    w = rng.random((B, H, ctx)).astype(np.float32)
    host[:, :ctx] = w.reshape(B * H, ctx).view(np.int32)
    lens = np.array([300, 80], np.int32)
    at = ctx + budget + gap
    host[0, at:at + B] = lens
    buf = dev(host)
    base = buf.data_ptr()
    st = K.load_library().int2kv_select_tokens(base, stride, B, H, base + 4 * at, ctx, budget, 4, 20, base + 4 * ctx, stride, base + 4 * (at + B),
                                               torch.cuda.current_stream().cuda_stream)
    assert st == K.INT2KV_OK, K.load_library().int2kv_last_error()
    torch.cuda.synchronize()
    got = buf.cpu().numpy()
    want = host.copy()
    want[0, at + B:at + 2 * B] = np.minimum(lens, budget)
    for b in range(B):
        for h in range(H):
            kept = kept_reference(w[b, h], int(lens[b]), budget, 4, 20)
            want[b * H + h, ctx:ctx + len(kept)] = kept
    assert np.array_equal(got, want)
