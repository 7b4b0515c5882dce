"""Inputs and fp64 references of the chunk operators' tests: caches with drawn codes and parameters, attention of several
new tokens per sequence, rows read back."""
from __future__ import annotations

import numpy as np
import torch

from oracle import int2kv_oracle as O
from paper_2608_02691_amd import int2kv as K

PAGE, D = 16, 128


def haar(rng, heads):
    q, r = np.linalg.qr(rng.standard_normal((heads, D, D)))
    return (q * np.sign(np.diagonal(r, axis1=1, axis2=2))[:, None, :]).astype(np.float32)


def bf16(x) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def random_pool(rng, blocks, heads, group, k_scale=1.0, v_scale=1.0):
    """A pool whose every slot holds drawn codes, with rows of about unit size times the given scales."""
    ng = D // group
    n = blocks * PAGE
    codes = lambda: rng.integers(0, 4, (n, heads, D)).astype(np.uint8)  # noqa: E731

    def params(scale):
        s = (rng.uniform(0.5, 1.1, (n, heads, ng)) * scale).astype(np.float16)
        z = (-1.5 * s.astype(np.float64) + rng.uniform(-0.3, 0.3, s.shape) * scale).astype(np.float16)
        return s, z

    pool = O.new_pool(blocks, heads, group)
    ks, kz = params(k_scale)
    vs, vz = params(v_scale)
    O.write_records(pool, np.arange(n), codes(), ks, kz, codes(), vs, vz)
    return pool


def stored_rows(pool, block_row, length):
    """Dequantized rows fp64 [length, H, 128] (keys, values); blocks outside the pool give zero rows."""
    row = np.asarray(block_row)
    safe = np.where((row >= 0) & (row < pool.shape[0]), row, 0)
    ks, vs = [], []
    for h in range(pool.shape[1]):
        kc, s, z, vc, s2, z2 = O.read_tokens(pool, safe, length, h)
        ks.append(O.dequantize(kc, s, z).astype(np.float64))
        vs.append(O.dequantize(vc, s2, z2).astype(np.float64))
    return np.stack(ks, 1), np.stack(vs, 1)


class Chunk:
    """One call's inputs. seqs: (new tokens, cached tokens) each; cached: the cache holds the new tokens too; blocks: the
    sequences draw their pages from so many, with repetition, instead of having their own."""

    def __init__(self, seqs, heads, gq, group=32, cached=False, seed=0, k_scale=1.0, v_scale=1.0, pad=0, fused=False,
                 spare=3, blocks=None):
        rng = np.random.default_rng(seed)
        self.seqs, self.H, self.gq, self.group, self.cached = seqs, heads, gq, group, cached
        self.Hq, self.total = heads * gq, sum(n for n, _ in seqs) + pad
        pages = [-(-c // PAGE) for _, c in seqs]
        if blocks is None:
            blocks = sum(pages) + spare
            perm = rng.permutation(blocks).astype(np.int32)
        else:
            perm = rng.integers(0, blocks, sum(pages)).astype(np.int32)
        self.table = np.full((len(seqs), max(1, max(pages)) + 1), -1, np.int32)
        at = 0
        for b, m in enumerate(pages):
            self.table[b, :m] = perm[at:at + m]
            at += m
        self.pool = random_pool(rng, blocks, heads, group, k_scale, v_scale)
        self.starts = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
        self.lens = np.array([c for _, c in seqs], np.int32)
        self.max_q, self.max_ctx = max(n for n, _ in seqs), max(c for _, c in seqs)
        self.R_k, self.R_v = haar(rng, heads), haar(rng, heads)
        self.mu = np.zeros((heads, D), np.float32)
        for h in range(heads):
            self.mu[h, rng.choice(D, 3, replace=False)] = rng.uniform(10, 30, 3)
        self.q = bf16(rng.standard_normal((self.total, self.Hq, D)))
        self.k = bf16(k_scale * rng.standard_normal((self.total, heads, D)) + self.mu)
        self.v = bf16(v_scale * rng.standard_normal((self.total, heads, D)))
        self.fused = fused

    def call(self, out=None, workspace=None, cache=None, **kw):
        dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
        q, k, v = self.q.cuda(), self.k.cuda(), self.v.cuda()
        if self.fused:  # views of one projection
            qkv = torch.cat([q, k, v], 1)
            q, k, v = qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + self.H], qkv[:, self.Hq + self.H:]
        if cache is None:
            cache = K.Int2KVCache(self.pool.shape[0], self.H, pool=dev(self.pool), group_size=self.group)
        if self.cached:
            own = (None, None, None)
        else:
            own = (k, v, dev(self.mu))
        args = dict(max_q=self.max_q, max_ctx=self.max_ctx)
        args.update(kw)
        return K.int2kv_chunk_attention(cache, q, dev(self.starts), args["max_q"], dev(self.table), dev(self.lens),
                                        args["max_ctx"], dev(self.R_k), dev(self.R_v), *own, out=out, workspace=workspace)

    def reference(self):
        """fp64 outputs [total, Hq, 128] and, per row, the norm sqrt(sum_s p_s^2 ||v_s||^2)."""
        out = np.zeros((self.total, self.Hq, D))
        spread = np.zeros((self.total, self.Hq))
        q, kn, vn = (x.double().numpy() for x in (self.q, self.k, self.v))
        for b, (n, ctx) in enumerate(self.seqs):
            if n == 0:
                continue
            kc, vc = stored_rows(self.pool, self.table[b], ctx) if ctx else (np.zeros((0, self.H, D)),) * 2
            real = np.repeat((self.table[b] >= 0) & (self.table[b] < self.pool.shape[0]), PAGE)[:ctx]
            at, i = self.starts[b], np.arange(n)
            for h in range(self.H):
                qh = q[at:at + n, h * self.gq:(h + 1) * self.gq].reshape(-1, D)
                keys = kc[:, h] @ self.R_k[h].astype(np.float64).T
                values = vc[:, h] @ self.R_v[h].astype(np.float64).T
                limit = ctx - n + i + 1 if self.cached else np.full(n, ctx)
                see = (np.arange(ctx)[None] < limit[:, None]) & real[None]
                if not self.cached:
                    keys = np.concatenate([keys, kn[at:at + n, h] - self.mu[h].astype(np.float64)])
                    values = np.concatenate([values, vn[at:at + n, h]])
                    see = np.concatenate([see, i[None] <= i[:, None]], 1)
                see = np.repeat(see, self.gq, 0)
                a = np.where(see, qh @ keys.T / np.sqrt(D), -np.inf)
                top = a.max(1, initial=-np.inf, keepdims=True)
                p = np.exp(a - np.where(np.isfinite(top), top, 0.0))
                den = p.sum(1, keepdims=True)
                p = np.divide(p, den, out=np.zeros_like(p), where=den > 0)
                o = (p @ values).reshape(n, self.gq, D)
                s = np.sqrt((p ** 2) @ (values ** 2).sum(1)).reshape(n, self.gq)
                out[at:at + n, h * self.gq:(h + 1) * self.gq] = o
                spread[at:at + n, h * self.gq:(h + 1) * self.gq] = s
        return out, spread


def assert_chunk_close(got, ref, spread, what=""):
    """Row norms of the error against the roundings of the call. With half steps of 2^-8 (bf16) and 2^-11 (fp16): the
    output's rounding is at most 2^-8 ||o||. A probability rounded to bf16 is off by at most 2^-8 p, with independent
    signs, so the sum of p_s eps_s v_s has a norm of about at most 2^-8 sqrt(sum p^2 ||v||^2) = 2^-8 spread. Rounded queries and keys
    (2^-11 each) move a score of unit-size rows by about 2^-11 * sqrt(2) * ||q|| ||k|| / sqrt(128)^2, i.e. below 2^-10 p, independent from
    token to token, values (2^-11) likewise: together below 2^-9 spread; R_V's rounding 2^-11 of ||o||. The sum stays below
    2^-7 ||o|| + 2^-7 spread."""
    got = np.asarray(got.detach().float().cpu().numpy() if isinstance(got, torch.Tensor) else got, dtype=np.float64)
    err, size = np.linalg.norm(got - ref, axis=-1), np.linalg.norm(ref, axis=-1)
    tol = 2.0 ** -7 * (size + spread)
    assert np.all(np.isfinite(got)), what
    zero = spread == 0
    assert np.all(got[zero] == 0), f"{what}: rows that see nothing must be zero"
    worst = float((err[~zero] / tol[~zero]).max()) if (~zero).any() else 0.0
    assert worst <= 1.0, f"{what}: error {worst:.3f} of the tolerance"
    return worst
