"""Inputs and fp64 references of the operators for drafted trees and for eviction: attention along paths, the weight that
cached tokens receive, the kept tokens, their rows."""
from __future__ import annotations

import numpy as np
import torch

from _chunk import D, PAGE, bf16, haar, random_pool, stored_rows
from paper_2608_02691_amd import int2kv as K


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def paged(rng, lens, spare=3, wide=1):
    """Block table int32 [B, pages + wide] (-1 behind a sequence's pages) and the number of blocks."""
    pages = [-(-c // PAGE) for c in lens]
    perm, at = rng.permutation(sum(pages) + spare).astype(np.int32), 0
    table = np.full((len(lens), max(1, max(pages)) + wide), -1, np.int32)
    for b, m in enumerate(pages):
        table[b, :m] = perm[at:at + m]
        at += m
    return table, sum(pages) + spare


def random_tree(rng, T, depth=None):
    """Parents of T tokens: anything before them, or -1 (`depth`: a chain of so many first)."""
    return np.array([-1 if t == 0 or (depth is None and rng.random() < 0.2) else t - 1 if depth and t < depth else rng.integers(-1, t)
                     for t in range(T)], np.int32)


def path_of(parents, t):
    """Tokens on the path of t, or None where it is absent."""
    path = []
    while t != -1:
        if t < 0 or t >= len(parents) or parents[t] >= t or parents[t] < -1:
            return None
        path.append(t)
        t = int(parents[t])
    return path


class TreeCall:
    """seqs: (queries, cached tokens, parents of the whole tree) each."""

    def __init__(self, seqs, heads, gq, group=32, seed=0, pad=0, fused=False, k_scale=1.0, v_scale=1.0, q_scale=1.0):
        rng = np.random.default_rng(seed)
        self.seqs, self.H, self.gq, self.group, self.fused = seqs, heads, gq, group, fused
        self.Hq, self.total, self.total_tree = heads * gq, sum(n for n, _, _ in seqs) + pad, sum(len(p) for _, _, p in seqs)
        self.lens = np.array([c for _, c, _ in seqs], np.int32)
        self.table, blocks = paged(rng, self.lens)
        self.pool = random_pool(rng, blocks, heads, group, k_scale, v_scale)
        self.starts = np.concatenate([[0], np.cumsum([n for n, _, _ in seqs])]).astype(np.int32)
        self.trees = np.concatenate([[0], np.cumsum([len(p) for _, _, p in seqs])]).astype(np.int32)
        self.parents = np.concatenate([np.asarray(p, np.int32) for _, _, p in seqs])
        self.max_q, self.max_ctx = max(n for n, _, _ in seqs), int(max(self.lens))
        self.max_tree = max(len(p) for _, _, p in seqs)
        self.R_k, self.R_v = haar(rng, heads), haar(rng, heads)
        self.mu = np.zeros((heads, D), np.float32)
        for h in range(heads):
            self.mu[h, rng.choice(D, 3, replace=False)] = rng.uniform(10, 30, 3)
        self.q = bf16(q_scale * rng.standard_normal((self.total, self.Hq, D)))
        self.k = bf16(k_scale * rng.standard_normal((self.total_tree, heads, D)) + self.mu)
        self.v = bf16(v_scale * rng.standard_normal((self.total_tree, heads, D)))

    def call(self, out=None, workspace=None, cache=None, **kw):
        q, k, v = self.q.cuda(), self.k.cuda(), self.v.cuda()
        if self.fused:  # views whose tokens lie apart
            kv = torch.cat([k, v], 1)
            k, v = kv[:, :self.H], kv[:, self.H:]
            q = torch.cat([q, q], 1)[:, :self.Hq]
        if cache is None:
            cache = K.Int2KVCache(self.pool.shape[0], self.H, pool=dev(self.pool), group_size=self.group)
        args = dict(max_q=self.max_q, max_ctx=self.max_ctx, max_tree=self.max_tree)
        args.update(kw)
        return K.int2kv_tree_attention(cache, q, dev(self.starts), args["max_q"], dev(self.parents), k, v, dev(self.mu), dev(self.table),
                                       dev(self.lens), args["max_ctx"], dev(self.R_k), dev(self.R_v), tree_starts=dev(self.trees),
                                       max_tree=args["max_tree"], out=out, workspace=workspace)

    def reference(self):
        """fp64 outputs [total, Hq, 128] and, per row, the norm sqrt(sum_s p_s^2 ||v_s||^2)."""
        out, spread = np.zeros((self.total, self.Hq, D)), np.zeros((self.total, self.Hq))
        q, kn, vn = (x.double().numpy() for x in (self.q, self.k, self.v))
        for b, (n, ctx, parents) in enumerate(self.seqs):
            kc, vc = stored_rows(self.pool, self.table[b], ctx) if ctx else (np.zeros((0, self.H, D)),) * 2
            real = np.repeat((self.table[b] >= 0) & (self.table[b] < self.pool.shape[0]), PAGE)[:ctx]
            for i in range(n):
                path = path_of(parents, len(parents) - n + i) if len(parents) - n + i >= 0 else None
                if path is None:
                    continue
                rows = self.trees[b] + np.array(path, int)
                for j in range(self.Hq):
                    h = j // self.gq
                    keys = np.concatenate([kc[real, h] @ self.R_k[h].astype(np.float64).T, kn[rows, h] - self.mu[h].astype(np.float64)])
                    values = np.concatenate([vc[real, h] @ self.R_v[h].astype(np.float64).T, vn[rows, h]])
                    a = keys @ q[self.starts[b] + i, j] / np.sqrt(D)
                    p = np.exp(a - a.max())
                    p /= p.sum()
                    out[self.starts[b] + i, j] = p @ values
                    spread[self.starts[b] + i, j] = np.sqrt((p ** 2) @ (values ** 2).sum(1))
        return out, spread


class WeightsCall:
    """seqs: (new tokens, cached tokens, the new ones among them) each."""

    def __init__(self, seqs, heads, gq, group=32, seed=0, pad=0, q_scale=2.0, k_scale=1.0, first=False, wide=0, fused=False):
        rng = np.random.default_rng(seed)
        self.seqs, self.H, self.gq, self.group, self.fused = seqs, heads, gq, group, fused
        self.Hq, self.total = heads * gq, sum(n for n, _ in seqs) + pad
        self.lens = np.array([c for _, c in seqs], np.int32)
        self.table, blocks = paged(rng, self.lens)
        self.pool = random_pool(rng, blocks, heads, group, k_scale)
        self.starts = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
        self.max_q, self.max_ctx = max(n for n, _ in seqs), int(max(self.lens))
        self.R_k = haar(rng, heads)
        self.q = bf16(q_scale * rng.standard_normal((max(1, self.total), self.Hq, D)))[:self.total]
        self.w = None if first else np.exp(rng.standard_normal((len(seqs), heads, self.max_ctx + wide))).astype(np.float32)
        self.shape = (len(seqs), heads, self.max_ctx + wide)

    def call(self, decay=0.75, out=None, workspace=None, cache=None, weights="own", **kw):
        if cache is None:
            cache = K.Int2KVCache(self.pool.shape[0], self.H, pool=dev(self.pool), group_size=self.group)
        q = self.q.cuda()
        if self.fused:
            q = torch.cat([q, q], 1)[:, self.Hq:]
        if isinstance(weights, str):
            weights = None if self.w is None else dev(self.w)
        args = dict(max_q=self.max_q, max_ctx=self.max_ctx)
        args.update(kw)
        return K.int2kv_token_weights(cache, q, dev(self.starts), args["max_q"], dev(self.table), dev(self.lens), args["max_ctx"],
                                      dev(self.R_k), weights=weights, decay=decay, out=out, workspace=workspace)

    def reference(self, decay=0.75):
        """fp64 sums and their tolerance [B, H, n]; both zero behind a length. With M = sum_g |s_g D_g| + |z_g Q_g| of a score
        (base 2), what the terms of its sum come to: a score is off by fewer than 16 roundings of partial sums of at most M,
        2^-24 each, and 2^-22 of the terms for the two-term queries, together below 2^-19 M; its row's log sum by as much and
        some roundings of its own size. A weight is then off by less than ln 2 (2^-18 M + 2^-21 |L|) of itself; sums over
        rows and the decayed part add a few roundings: 2^-20 of the result's parts. fp32's normal numbers end at 2^-126: a
        weight below that comes out as zero or as a multiple of 2^-149, off by at most 2^-126 a row that sees the token."""
        got, tol = np.zeros(self.shape), np.zeros(self.shape)
        q, ng = self.q.double().numpy(), D // self.group
        for b, (n, ctx) in enumerate(self.seqs):
            if ctx == 0:
                continue
            kc, _ = stored_rows(self.pool, self.table[b], ctx)
            real = np.repeat((self.table[b] >= 0) & (self.table[b] < self.pool.shape[0]), PAGE)[:ctx]
            base = 0.0 if self.w is None else decay * self.w[b, :, :ctx].astype(np.float64)
            got[b, :, :ctx] += base
            tol[b, :, :ctx] += 2.0 ** -20 * np.abs(base)
            limit = ctx - n + np.arange(n) + 1
            for h in range(self.H):
                z = self._zeros(b, ctx, h)
                for j in range(h * self.gq, (h + 1) * self.gq):
                    qr = q[self.starts[b]:self.starts[b] + n, j] @ self.R_k[h].astype(np.float64) / np.sqrt(D) * np.log2(np.e)
                    x = qr @ kc[:, h].T
                    M = np.zeros_like(x)
                    for g in range(ng):
                        c = slice(g * self.group, (g + 1) * self.group)
                        Q = qr[:, c].sum(1)[:, None] * z[None, :, g]
                        M += np.abs(qr[:, c] @ kc[:, h, c].T - Q) + np.abs(Q)
                    see = (np.arange(ctx)[None] < limit[:, None]) & real[None]
                    rows = see.any(1)
                    if not rows.any():
                        continue
                    x, M, see = x[rows], M[rows], see[rows]
                    x = np.where(see, x, -np.inf)
                    top = x.max(1, keepdims=True)
                    L = top + np.log2(np.exp2(x - top).sum(1, keepdims=True))
                    p = np.exp2(x - L)
                    worst = np.where(see, M, 0).max(1, keepdims=True)
                    got[b, h, :ctx] += p.sum(0)
                    tol[b, h, :ctx] += (p * (2.0 ** -18 * worst + 2.0 ** -21 * np.abs(L) + 2.0 ** -20)).sum(0) + 2.0 ** -126 * see.sum(0)
        return got, tol

    def _zeros(self, b, ctx, h):
        from oracle import int2kv_oracle as O
        row = np.where((self.table[b] >= 0) & (self.table[b] < self.pool.shape[0]), self.table[b], 0)
        return O.read_tokens(self.pool, row, ctx, h)[2].astype(np.float64)


def assert_weights_close(got, ref, tol, what=""):
    got = np.asarray(got.cpu().numpy() if isinstance(got, torch.Tensor) else got, np.float64)
    assert np.all(np.isfinite(got)), what
    err = np.abs(got - ref)
    assert np.all(err[tol == 0] == 0), f"{what}: tokens that receive nothing"
    worst = float((err[tol > 0] / tol[tol > 0]).max()) if (tol > 0).any() else 0.0
    assert worst <= 1.0, f"{what}: error {worst:.3f} of the tolerance"
    return worst


def kept_reference(w, length, budget, sink, recent):
    """Kept tokens of one list, in order: forced ones, then by weight, ties to the lower index, NaN below every number."""
    if length <= budget:
        return np.arange(length)
    t = np.arange(length)
    forced = (t < sink) | (t >= length - recent)
    rest = t[~forced]
    key = [(1, 0.0) if np.isnan(x) else (0, -float(x)) for x in w[rest]]
    order = sorted(range(len(rest)), key=lambda i: (key[i], rest[i]))
    return np.sort(np.concatenate([t[forced], rest[order[:budget - int(forced.sum())]]]))


def moved_pool(pool, table, kept, kept_lens, out_table, max_kept=None):
    """The pool after the move, token by token: every byte of a row by its place in the record."""
    new, nb, H = pool.copy(), pool.shape[0], pool.shape[1]
    group = 32 if pool.shape[2] == 1536 else 128
    meta = 512 // group

    def fields(t):
        yield np.arange(32 * t, 32 * t + 32)
        for m in range(16):
            yield np.arange(512 + 32 * m + 2 * t, 512 + 32 * m + 2 * t + 2)
        yield np.arange(1024 + meta * t, 1024 + meta * t + meta)
        for r in range(2 * (D // group)):
            yield np.arange(1024 + 16 * meta + 32 * r + 2 * t, 1024 + 16 * meta + 32 * r + 2 * t + 2)

    where = [np.concatenate(list(fields(t))) for t in range(PAGE)]
    for b in range(table.shape[0]):
        for h in range(H):
            for j in range(min(int(kept_lens[b]), kept.shape[2] if max_kept is None else max_kept)):
                old = int(kept[b, h, j])
                if old < 0 or old >= table.shape[1] * PAGE:
                    continue
                src, dst = int(table[b, old // PAGE]), int(out_table[b, j // PAGE])
                if 0 <= src < nb and 0 <= dst < nb:
                    new[dst, h, where[j % PAGE]] = pool[src, h, where[old % PAGE]]
    return new
