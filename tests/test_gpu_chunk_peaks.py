"""Scores that rise, fall and peak along the context: the running maximum moves again and again, far more than the 2^8 that it
waits for, over INT2 units, over the chunk's own tokens behind them, and between the waves and pieces that are joined."""
import numpy as np
import pytest
import torch

from _chunk import D, Chunk, bf16, stored_rows
from test_gpu_chunk import _meta

pytestmark = pytest.mark.gpu


def _ragged(n, new, ctx, seed):
    rng = np.random.default_rng(seed)
    return [(int(rng.integers(*new)), int(rng.integers(*ctx))) for _ in range(n)]


# name: sequences (new, cached), KV heads, query heads per KV head: every kernel, its tiles cut and whole
PLANS = {
    "few, cut": ([(5, 3000), (3, 400), (8, 65)], 2, 4),
    "few, whole": (_ragged(60, (1, 8), (300, 1500), 2), 12, 4),
    "few, listed": (_ragged(70, (1, 4), (0, 1200), 3), 4, 4),
    "narrow, cut": ([(24, 2500), (30, 10)], 2, 4),
    "narrow, whole": (_ragged(40, (17, 33), (0, 900), 7), 8, 4),
    "wide, cut": ([(100, 3000)], 1, 4),
    "wide, whole": (_ragged(20, (180, 300), (0, 700), 11), 8, 4),
}

# Key sizes along a context of L tokens (t: token numbers); scores of N(0, 1) queries have this standard deviation
SHAPES = {
    "rising": lambda t, L: 0.1 + 25.0 * (t / max(L, 1)) ** 2,
    "falling": lambda t, L: 0.1 + 25.0 * (1.0 - t / max(L, 1)) ** 2,
    # many flat tokens, then some whose weights together are about as much
    "late": lambda t, L: np.where(t >= L - 40, 3.0, 0.05),
    "spikes": lambda t, L: np.where(t % 150 == 77, 4.0 + 8.0 * (t / max(L, 1)), 0.3),
}


def _shaped(seqs, heads, gq, group, cached, shape, own, seed):
    """A call whose cached keys have the shape's sizes and whose own keys have size `own` (and grow with their place)."""
    c = Chunk(seqs, heads, gq, group, cached, seed=seed)
    rng = np.random.default_rng(seed + 1)
    k, _ = _meta(c.pool, group)
    for b, (_, ctx) in enumerate(seqs):
        t = np.arange(ctx)
        f = shape(t, ctx)
        for page in range(-(-ctx // 16)):
            x = f[16 * page:16 * page + 16]
            k[c.table[b, page], :, :len(x)] *= x[None, :, None, None].astype(np.float16)
    grow = np.concatenate([own * (0.5 + np.arange(n) / max(n, 1)) for n, _ in seqs])
    c.k = bf16(grow[:, None, None] * rng.standard_normal(tuple(c.k.shape)) + c.mu)
    return c


def _reference(c):
    """fp64 outputs, and each row's tolerance.

    Beside 2^-7 (||o|| + spread) of unit-size rows (assert_chunk_close), the roundings of the INT2 scores grow with the keys:
    R_K, q' and k^ are off by half steps of 2^-11 each, three independent sums of 128 products, so a score is off by
    2^-11 sqrt(3) c ||q|| ||k_s|| / sqrt(128) in the root mean square at most, and hardly ever by four times that, d_s. A
    score's error d_s moves the output by p_s d_s (v_s - o); the sum of their norms is taken. Scores of the chunk's own tokens
    are exact products summed in fp32: q k_t of up to 128 products and q mu^T are off by 2^-20 of sum |q||k|, nothing here."""
    out, tol = np.zeros((c.total, c.Hq, D)), np.zeros((c.total, c.Hq))
    q, kn, vn = (x.double().numpy() for x in (c.q, c.k, c.v))
    for b, (n, ctx) in enumerate(c.seqs):
        if n == 0:
            continue
        kc, vc = stored_rows(c.pool, c.table[b], ctx) if ctx else (np.zeros((0, c.H, D)),) * 2
        at, i = c.starts[b], np.arange(n)
        for h in range(c.H):
            qh = q[at:at + n, h * c.gq:(h + 1) * c.gq].reshape(-1, D)
            keys, values = kc[:, h] @ c.R_k[h].astype(np.float64).T, vc[:, h] @ c.R_v[h].astype(np.float64).T
            off = np.linalg.norm(kc[:, h], axis=1)
            limit = ctx - n + i + 1 if c.cached else np.full(n, ctx)
            see = np.arange(ctx)[None] < limit[:, None]
            if not c.cached:
                keys = np.concatenate([keys, kn[at:at + n, h] - c.mu[h].astype(np.float64)])
                values = np.concatenate([values, vn[at:at + n, h]])
                see = np.concatenate([see, i[None] <= i[:, None]], 1)
                off = np.concatenate([off, np.zeros(n)])
            see = np.repeat(see, c.gq, 0)
            a = np.where(see, qh @ keys.T / np.sqrt(D), -np.inf)
            top = a.max(1, initial=-np.inf, keepdims=True)
            p = np.exp(a - np.where(np.isfinite(top), top, 0.0))
            den = p.sum(1, keepdims=True)
            p = np.divide(p, den, out=np.zeros_like(p), where=den > 0)
            o = p @ values
            size = np.linalg.norm(o, axis=1)
            spread = np.sqrt((p ** 2) @ (values ** 2).sum(1))
            away = np.sqrt(np.maximum((values ** 2).sum(1)[None] - 2 * o @ values.T + (size ** 2)[:, None], 0.0))
            d = 4 * np.sqrt(3) * 2.0 ** -11 / D * np.linalg.norm(qh, axis=1)[:, None] * off[None]
            slack = (p * np.minimum(d, 1.0) * away).sum(1)
            out[at:at + n, h * c.gq:(h + 1) * c.gq] = o.reshape(n, c.gq, D)
            tol[at:at + n, h * c.gq:(h + 1) * c.gq] = (2.0 ** -7 * (size + spread) + slack).reshape(n, c.gq)
    return out, tol


def _close(got, ref, tol, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    err = np.linalg.norm(got - ref, axis=-1)
    assert np.all(err[tol == 0] == 0), what
    worst = float((err[tol > 0] / tol[tol > 0]).max())
    assert worst <= 1.0, f"{what}: error {worst:.3f} of the tolerance"
    print(f"error {worst:.3f} of the tolerance", flush=True)


@pytest.mark.parametrize("cached", [True, False])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("name", PLANS)
def test_shapes(name, shape, cached):
    seqs, heads, gq = PLANS[name]
    group = 32 if (len(name) + len(shape)) % 2 else 128
    print(f"\n[peaks] {name} {shape} cached={cached} G={group}", flush=True)
    c = _shaped(seqs, heads, gq, group, cached, SHAPES[shape], 1.0, seed=len(name) + len(shape))
    _close(c.call(), *_reference(c), f"{name} {shape}")


@pytest.mark.parametrize("own", [0.05, 6.0, 30.0])
@pytest.mark.parametrize("name", ["few, cut", "narrow, cut", "wide, cut", "wide, whole"])
def test_own_tokens_above_and_below_the_cached_ones(name, own):
    """The maximum of the cached tokens, of a flat context, against the chunk's own: small, moving it once, moving it often."""
    seqs, heads, gq = PLANS[name]
    print(f"\n[peaks] {name} own keys {own}", flush=True)
    c = _shaped(seqs, heads, gq, 32, False, lambda t, L: np.full(t.shape, 0.5), own, seed=len(name))
    _close(c.call(), *_reference(c), f"{name} {own}")


@pytest.mark.parametrize("name", ["few, cut", "few, whole", "narrow, cut", "wide, cut", "wide, whole"])
def test_a_single_token_that_outweighs_all_others(name):
    """One cached token of each sequence, last of a unit's first half, first of its second or far behind: its value alone comes out."""
    seqs, heads, gq = PLANS[name]
    print(f"\n[peaks] {name} one token", flush=True)
    c = _shaped(seqs, heads, gq, 32, True, lambda t, L: np.full(t.shape, 0.2), 1.0, seed=len(name))
    c.q = torch.ones_like(c.q)
    k, _ = _meta(c.pool, 32)
    want = np.zeros((c.total, c.Hq, D))
    sure = np.zeros((c.total, c.Hq), bool)  # rows whose sequence and head have such a token
    for b, (n, ctx) in enumerate(seqs):
        if ctx <= n:
            continue
        tok = (31, 32, 0, ctx - n - 1)[b % 4]
        tok = min(tok, ctx - n - 1)
        # k^ R_K^T along the queries: a constant per group cannot do that, so the token takes scale 0 and the zero points that
        # lie closest to q's rotated direction, 64 times as large
        for h in range(heads):
            turned = np.ones(D) @ c.R_k[h].astype(np.float64)
            k[c.table[b, tok // 16], h, tok % 16, :, 0] = 0
            k[c.table[b, tok // 16], h, tok % 16, :, 1] = 600 * turned.reshape(4, 32).mean(1)
        kc, vc = stored_rows(c.pool, c.table[b], ctx)
        for h in range(heads):
            a = (kc[:, h] @ c.R_k[h].astype(np.float64).T).sum(1) / np.sqrt(D)
            lead = a[tok] - np.delete(a, tok).max()
            if lead > 40:
                rows = np.s_[c.starts[b]:c.starts[b] + n, h * gq:(h + 1) * gq]
                want[rows] = c.R_v[h].astype(np.float64) @ vc[tok, h]
                sure[rows] = True
    assert sure.any()
    got = c.call().double().cpu().numpy()[sure]
    want = want[sure]
    # the value's own rounding to fp16, R_V's and the output's
    assert np.all(np.linalg.norm(got - want, axis=-1) <= 2.0 ** -7 * np.linalg.norm(want, axis=-1))
