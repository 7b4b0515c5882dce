"""int2kv_token_weights where scores are so large that fp16's rounding of their first estimate is worth many powers of two: rows
keep their weight, which sums to one."""
import numpy as np
import pytest
import torch

from _tokens import WeightsCall, assert_weights_close
from test_gpu_chunk import _meta

pytestmark = pytest.mark.gpu

LOGIT2 = np.log2(np.e) / np.sqrt(128)


def flat_call(n, ctx, gq, group, q, zero):
    """Queries of one value, keys of one value, R_K the identity: every token's score is LOGIT2 128 q zero."""
    c = WeightsCall([(n, ctx), (1, 40)], 1, gq, group, seed=n, first=True)
    c.R_k = np.eye(128, dtype=np.float32)[None]
    c.q[:] = q
    k, _ = _meta(c.pool, group)
    k[..., 0], k[..., 1] = 0.0, zero
    return c, abs(LOGIT2 * 128 * q * zero)


# bf16 queries whose product with LOGIT2 fp16 rounds up by 0.90, down by 0.91 of 2^-11: with the zeros below the estimate lies 200 and
# 1,370 powers of two above every score of its row, or as far below it
@pytest.mark.parametrize("q", [15.9375, -15.9375, 15.875])
@pytest.mark.parametrize("zero", [1768.0, 12000.0])
@pytest.mark.parametrize("n,ctx,gq,group", [(1, 90, 4, 32), (12, 12, 4, 32), (12, 700, 4, 128), (12, 700, 1, 32), (70, 600, 4, 32), (300, 300, 4, 128)])
def test_estimates_far_from_the_scores(n, ctx, gq, group, zero, q):
    """Each row's weights are 1 / (tokens it sees). A score is the same number x in both passes; the row's base, a rounding of
    x, and its log sum are each off by half a step of x's size, 2^-24 |x|, so a weight is off by 2^(2^-23 |x|) of itself, and some
    roundings of its own; twice that is allowed."""
    c, x = flat_call(n, ctx, gq, group, q, zero if q > 0 else -zero)
    got = c.call().double().cpu().numpy()
    rel = 2.0 ** (2.0 ** -22 * x) - 1 + 2.0 ** -18
    for b, (m, length) in enumerate(c.seqs):
        want, lim = np.zeros(length), length - m + np.arange(m) + 1
        for i in lim:
            want[:i] += gq / i
        err = np.abs(got[b, 0, :length] - want) / want
        print(f"{n} of {ctx} x {gq}, {q}, {zero}: sequence {b} off by {err.max():.2e} of {rel:.2e}")
        assert err.max() <= rel
        assert abs(got[b].sum() - m * gq) <= rel * m * gq


@pytest.mark.parametrize("n", [3, 12, 64])
@pytest.mark.parametrize("group", [32, 128])
def test_scores_of_millions(n, group):
    """Drawn queries and zeros far apart: one token takes a row, and the rows' weights sum to one, by the tolerance above (that of
    the largest score)."""
    c = WeightsCall([(n, 25 + n), (n, 400)], 1, 4, group, seed=n + group, first=True, q_scale=60.0)
    k, _ = _meta(c.pool, group)
    k[..., 1] = (5000.0 * np.random.default_rng(n).standard_normal(k.shape[:-1])).astype(np.float16)
    ref, _ = c.reference()
    assert abs(ref.sum() - 8 * n) < 1e-6 * n
    top = max(float(np.abs(c.q.double().numpy()[a:e].reshape(-1, 128) @ c.R_k[0] @ (k[c.table[b, t // 16], 0, t % 16, :, 1].astype(np.float64).repeat(group))).max())
              for b, (a, e, length) in enumerate(zip(c.starts, c.starts[1:], c.lens)) for t in range(length)) * LOGIT2
    rel = 2.0 ** (2.0 ** -22 * top) - 1 + 2.0 ** -18
    got = c.call().double().cpu().numpy()
    total = got.sum(-1)
    print(f"{n}, {group}: largest score {top:.3g}, sums {total[:, 0] / (4 * n)}, allowed {rel:.2f}")
    assert np.isfinite(got).all() and np.all(np.abs(total - 4 * n) <= rel * 4 * n)


@pytest.mark.parametrize("n", [2, 20])
def test_ordinary_sizes_are_not_touched(n):
    c = WeightsCall([(n, 500)], 2, 4, seed=51, q_scale=30.0, k_scale=4.0)
    ref, tol = c.reference()
    assert_weights_close(c.call(), ref, tol, f"{n}")
