"""Inputs and plain 64-bit forms for the tests of the operators on a cache kept in pages."""
import math

import numpy as np
import torch


class Case:
    """One layer's cache with a few sequences.  Rows that belong to nobody, and the caches behind a sequence's last row, hold NaN."""

    def __init__(self, dtype, n_head, n_kv, d, page, new, lens, window=0, sinks=0, seed=0, spare=2, share=(), stale=float("nan")):
        self.dtype, self.n_head, self.n_kv, self.d, self.page, self.new, self.lens = dtype, n_head, n_kv, d, page, list(new), list(lens)
        self.window, self.sinks, self.group, self.T = window, sinks, n_head // n_kv, sum(new)
        rng = np.random.default_rng(seed)
        counts = [-(-n // page) for n in lens]
        self.n_pages = sum(counts) + spare
        order = rng.permutation(self.n_pages).astype(np.int32)
        self.table, at = [], 0
        for n in counts:
            self.table.append(order[at:at + n].tolist())
            at += n
        for a, b, n in share:                         # sequence a reads the first n pages of b
            self.table[a][:n] = self.table[b][:n]
        g = torch.Generator().manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=g)  # noqa: E731
        self.k, self.v = (torch.full((self.n_pages, n_kv, page, d), stale).to(dtype) for _ in range(2))
        for b, n in enumerate(lens):
            for p, pg in enumerate(self.table[b]):
                m = min(page, n - p * page)
                self.k[pg, :, :m] = randn(n_kv, m, d).to(dtype)
                self.v[pg, :, :m] = randn(n_kv, m, d).to(dtype)
        self.q = (1.5 * randn(self.T, n_head, d)).to(dtype)

    def plan(self, fl, **kw):
        args = dict(window=self.window, sinks=self.sinks)
        args.update(kw)
        return fl.PagedPlan(self.dtype, self.n_head, self.n_kv, self.d, self.page, self.n_pages, self.new, self.lens, self.table, **args)

    def rows(self, cache, b):
        """Cached rows of sequence b, [n_kv][position][d]."""
        mine = torch.cat([cache[p] for p in self.table[b]] or [cache[:0].reshape(self.n_kv, 0, self.d)], 1)
        return mine[:, :self.lens[b]]

    def seen(self, b):
        p = torch.arange(self.lens[b] - self.new[b], self.lens[b])[:, None]
        j = torch.arange(self.lens[b])[None]
        seen = j <= p
        if self.window:
            seen = seen & ((j > p - self.window) | (j < self.sinks))
        return seen

    def scores(self, b):
        """(scores, size of their terms) [head][new token][position] in 64 bits."""
        at = sum(self.new[:b])
        q = self.q[at:at + self.new[b]].double().transpose(0, 1)
        k = self.rows(self.k, b).double().repeat_interleave(self.group, 0)
        hidden = ~self.seen(b)
        s = torch.stack([q[h] @ k[h].T for h in range(self.n_head)]) / math.sqrt(self.d)
        terms = torch.stack([q[h].abs() @ k[h].abs().T for h in range(self.n_head)]) / math.sqrt(self.d)
        return s.masked_fill(hidden, -math.inf), terms.masked_fill(hidden, 0.0)

    def attention(self):
        """(out, lse, bound of out, bound of lse), [token][head]...; a key that is not seen takes no part.

        Bounds: a score is a sum of d terms and a scaling in fp32, off by (d + 8) 2^-24 of the terms' sum, which a weight feels twice
        (its own and the normaliser's), as it does the exponential's argument and result (2^-22 of 1 + |s|); sums of n terms are off by (n + 64)
        2^-24; a weight may be rounded to the 16-bit type once (half a step, and half the smallest step of fp16, 2^-25), the result is."""
        half = torch.finfo(self.dtype).eps / 2
        out = torch.zeros((self.T, self.n_head, self.d), dtype=torch.float64)
        lse, ob, lb = torch.zeros((self.T, self.n_head), dtype=torch.float64), torch.zeros_like(out), torch.zeros((self.T, self.n_head), dtype=torch.float64)
        for b in range(len(self.new)):
            n, at, L = self.new[b], sum(self.new[:b]), self.lens[b]
            if n == 0:
                continue
            s, terms = self.scores(b)
            z = torch.logsumexp(s, 2)
            p = torch.exp(s - z[..., None])
            v = self.rows(self.v, b).double().repeat_interleave(self.group, 0)
            seen = self.seen(b)
            es = (self.d + 8) * 2.0 ** -24 * terms.amax(2) + 2.0 ** -22 * (1 + s.masked_fill(~seen, 0).abs().amax(2))
            rel = 2 * es + 2.0 ** -20 + (L + 64) * 2.0 ** -24 + (half if self.dtype != torch.float32 else 0.0)
            for h in range(self.n_head):
                pv = p[h][:, :, None] * v[h][None]
                pv[~seen] = 0.0
                o, size = pv.sum(1), pv.abs().sum(1)
                floor = 2.0 ** -25 * (v[h].abs()[None] * seen[:, :, None]).nan_to_num(0.0, 0.0, 0.0).sum(1) if self.dtype == torch.float16 else 0.0
                out[at:at + n, h] = o
                ob[at:at + n, h] = half * o.abs() * 1.01 + rel[h][:, None] * size + floor + 1e-30
            lse[at:at + n] = z.T
            lb[at:at + n] = (es + (L + 64) * 2.0 ** -24 + 2.0 ** -22 * (1 + z.abs())).T
        return out, lse, ob, lb

    def weights(self, lse, old, decay):
        """(weights, bound): decay * old (0 for the new tokens' own rows) plus what the new tokens gave, with the given lse; errors as
        above, a weight's own once."""
        w, wb = old.double().clone(), torch.zeros(old.shape, dtype=torch.float64)
        for b in range(len(self.new)):
            n, at, L = self.new[b], sum(self.new[:b]), self.lens[b]
            w[b, :, :L - n] *= decay
            w[b, :, L - n:L] = 0.0
            wb[b, :, :L] = 2.0 ** -23 * w[b, :, :L].abs()
            if n == 0:
                continue
            s, terms = self.scores(b)
            z = lse[at:at + n].double().T[..., None]
            p = torch.exp(s - z)
            es = (self.d + 8) * 2.0 ** -24 * terms + 2.0 ** -22 * (2 + s.masked_fill(~self.seen(b), 0).abs() + z.abs())
            give = p.view(self.n_kv, self.group * n, L).sum(1)
            off = (p * es).view(self.n_kv, self.group * n, L).sum(1) + (n * self.group + 64) * 2.0 ** -24 * give
            w[b, :, :L] += give
            wb[b, :, :L] += off + 2.0 ** -23 * w[b, :, :L].abs() + 1e-30
        return w, wb

    def evicted(self, weights, budget, first, recent):
        """(k cache, v cache, rows kept [n_seq][n_kv] lists) from the definition."""
        k, v, kept = self.k.clone(), self.v.clone(), []
        for b, n in enumerate(self.lens):
            kept.append([])
            for h in range(self.n_kv):
                w = weights[b, h, :n].tolist()
                keep = list(range(n))
                if n > budget:
                    sure = set(range(first)) | set(range(n - recent, n))
                    rest = sorted((p for p in range(n) if p not in sure),
                                  key=lambda p: (math.isnan(w[p]), 0.0 if math.isnan(w[p]) else -w[p], p))
                    keep = sorted(sure | set(rest[:budget - len(sure)]))
                kept[b].append(keep)
                for r, p in enumerate(keep):
                    src, dst = self.table[b][p // self.page], self.table[b][r // self.page]
                    k[dst, h, r % self.page] = self.k[src, h, p % self.page]
                    v[dst, h, r % self.page] = self.v[src, h, p % self.page]
        return k, v, kept
