"""Rows read back from the INT2 cache against their fp64 definition."""
import numpy as np
import pytest
import torch

from paper_2608_02691_amd import int2kv as K

from _chunk import PAGE, haar, random_pool, stored_rows

pytestmark = pytest.mark.gpu


def _expected(pool, slots, R_k, R_v, mu):
    """fp64 rows of every slot (negative: zeros)."""
    k, v = stored_rows(pool, np.arange(pool.shape[0]), pool.shape[0] * PAGE)
    k, v = k[slots], v[slots]
    if R_k is not None:
        k = np.einsum("nhc,hdc->nhd", k, R_k.astype(np.float64)) + (0 if mu is None else mu.astype(np.float64))
    if R_v is not None:
        v = np.einsum("nhc,hdc->nhd", v, R_v.astype(np.float64))
    return k, v


def _slots(rng, n, blocks, order):
    if order == "pages":
        t = np.arange(n)
        return (rng.permutation(blocks)[t // PAGE] * PAGE + t % PAGE).astype(np.int32)
    return rng.integers(0, blocks * PAGE, n).astype(np.int32)  # repeats among them


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("n,heads,order", [(1, 1, "pages"), (16, 2, "pages"), (33, 3, "any"), (129, 8, "pages"), (1000, 2, "any")])
def test_model_basis(n, heads, order, group, dtype):
    """Tolerances, as row norms. bf16: the output's rounding 2^-8 |y|, under it one fp16 term of x^ (2^-11 of each value)
    and of R (2^-11 of each entry), 128 independent products each: sqrt(2) 2^-11 ||x^||. fp32: two fp16 terms each, 2^-22 of
    every value and entry, and fp32 sums of 384 products, with independent roundings below 20 * 2^-24 ||x^||; mu is added in
    fp32, 2^-24 of the result."""
    print(f"\n[read] n={n} H={heads} {order} G={group} {dtype}", flush=True)
    rng = np.random.default_rng(n + heads)
    blocks = -(-n // PAGE) + 2
    pool = random_pool(rng, blocks, heads, group)
    R_k, R_v, mu = haar(rng, heads), haar(rng, heads), (20 * rng.standard_normal((heads, 128))).astype(np.float32)
    slots = _slots(rng, n, blocks, order)
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    cache = K.Int2KVCache(blocks, heads, pool=dev(pool), group_size=group)
    k, v = K.int2kv_read_rows(cache, dev(slots), dev(R_k), dev(R_v), dev(mu), dtype=dtype)
    for got, ref, off in zip((k, v), _expected(pool, slots, R_k, R_v, mu), (mu, None)):
        assert got.dtype == dtype
        err = np.linalg.norm(got.double().cpu().numpy() - ref, axis=-1)
        size = np.linalg.norm(ref, axis=-1)
        turned = np.linalg.norm(ref - (0 if off is None else off.astype(np.float64)), axis=-1)
        tol = 2.0 ** -8 * size + 2.0 ** -10.5 * turned if dtype == torch.bfloat16 else 2.0 ** -24 * size + 24 * 2.0 ** -24 * turned
        assert np.all(err <= tol), float((err / tol).max())
    centered, _ = K.int2kv_read_rows(cache, dev(slots), dev(R_k), dev(R_v), dtype=torch.float32)
    ref = _expected(pool, slots, R_k, None, None)[0]
    assert np.all(np.linalg.norm(centered.double().cpu().numpy() - ref, axis=-1) <= 24 * 2.0 ** -24 * np.linalg.norm(ref, axis=-1))


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("n,heads", [(1, 1), (47, 3), (700, 8)])
def test_stored_rows_are_exact(n, heads, group):
    rng = np.random.default_rng(n)
    blocks = -(-n // PAGE) + 1
    pool = random_pool(rng, blocks, heads, group)
    slots = _slots(rng, n, blocks, "any")
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    cache = K.Int2KVCache(blocks, heads, pool=dev(pool), group_size=group)
    want = _expected(pool, slots, None, None, None)
    for dtype in (torch.float32, torch.bfloat16):
        for got, ref in zip(K.int2kv_read_rows(cache, dev(slots), dtype=dtype), want):
            once = torch.from_numpy(ref).float()  # code * s + z needs 13 bits past fp16's at most: one fp32 rounding
            assert torch.equal(got.cpu(), once.to(dtype))


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_skipped_slots_and_single_outputs(dtype, turned):
    rng = np.random.default_rng(4)
    n, heads, blocks = 70, 2, 9
    pool = random_pool(rng, blocks, heads, 32)
    R = torch.from_numpy(haar(rng, heads)).cuda()
    slots = _slots(rng, n, blocks, "any")
    slots[[0, 13, 31, 69]] = [-1, blocks * PAGE, -2 ** 31, 2 ** 31 - 1]
    s = torch.from_numpy(slots).cuda()
    cache = K.Int2KVCache(blocks, heads, pool=torch.from_numpy(pool).cuda())
    R_k, R_v = (R, R) if turned else (None, None)
    full = K.int2kv_read_rows(cache, s.clamp(0, blocks * PAGE - 1), R_k, R_v, dtype=dtype)
    mark = lambda: torch.full((n, heads, 128), 7.0, dtype=dtype, device="cuda")  # noqa: E731
    out = K.int2kv_read_rows(cache, s, R_k, R_v, k_out=mark(), v_out=mark())
    only_k, none = K.int2kv_read_rows(cache, s, R_k, R_v, k_out=mark())
    assert none is None
    _, only_v = K.int2kv_read_rows(cache, s, R_k, R_v, v_out=mark())
    mixed = K.int2kv_read_rows(cache, s, R_k, None, k_out=mark(), v_out=mark())
    skip = torch.zeros(n, dtype=torch.bool, device="cuda")
    skip[[0, 13, 31, 69]] = True
    for got, ref, alone in zip(out, full, (only_k, only_v)):
        assert bool((got[skip] == 7.0).all()) and torch.equal(got[~skip], ref[~skip]) and torch.equal(alone, got)
    assert torch.equal(mixed[0], out[0])
    assert torch.equal(mixed[1], K.int2kv_read_rows(cache, s, v_out=mark())[1])


def test_infinite_parameters_stay_in_their_rows():
    rng = np.random.default_rng(5)
    pool = random_pool(rng, 4, 2, 32)
    pool[1, :, 1024:1026] = np.frombuffer(np.float16(np.inf).tobytes(), np.uint8)  # key scale of token 0, group 0
    R = torch.from_numpy(haar(rng, 2)).cuda()
    cache = K.Int2KVCache(4, 2, pool=torch.from_numpy(pool).cuda())
    s = torch.arange(64, dtype=torch.int32, device="cuda")
    for dtype in (torch.bfloat16, torch.float32):
        k, v = K.int2kv_read_rows(cache, s, R, R, dtype=dtype)
        rows = torch.isfinite(k).all(-1).all(-1)
        assert not rows[16] and int(rows.sum()) == 63 and bool(torch.isfinite(v).all())


def test_far_slots_and_graphs():
    """Slots beyond 2^32 bytes of the pool; replays of a captured read with new slots."""
    rng = np.random.default_rng(6)
    small = random_pool(rng, 8, 1, 32)
    blocks = (1 << 32) // 1536 + 4000
    pool = torch.zeros((blocks, 1, 1536), dtype=torch.uint8, device="cuda")
    pool[-8:] = torch.from_numpy(small).cuda()
    R = torch.from_numpy(haar(rng, 1)).cuda()
    cache, near = K.Int2KVCache(blocks, 1, pool=pool), K.Int2KVCache(8, 1, pool=torch.from_numpy(small).cuda())
    s = torch.from_numpy(rng.integers(0, 128, 50).astype(np.int32)).cuda()
    far = s + (blocks - 8) * PAGE
    for Rx in (R, None):
        for a, b in zip(K.int2kv_read_rows(cache, far, Rx, Rx), K.int2kv_read_rows(near, s, Rx, Rx)):
            assert torch.equal(a, b)
    k, v = torch.zeros((2, 50, 1, 128), dtype=torch.bfloat16, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        K.int2kv_read_rows(near, s, R, R, k_out=k, v_out=v)
    for turn in range(3):
        s.copy_((s + 17 * turn) % 128)
        want = K.int2kv_read_rows(near, s, R, R)
        g.replay()
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
        torch.cuda.synchronize()
