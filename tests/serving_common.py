"""Batches over a paged cache for the tests of the serving operators, and their tolerances."""
import numpy as np

from oracle import serving as ref


def half_step(dtype):
    """Largest relative error of one rounding to a type."""
    import torch
    return torch.finfo(dtype).eps / 2


class Batch:
    """Sequences of (new, before) tokens over a pool whose unused places hold NaN and whose page
    table's unused entries are no page ids."""

    def __init__(self, torch, seqs, heads, kv_heads, dim, page, dtype, seed=0, pad_rows=0, spare=3,
                 filled=True, q_scale=2.0, width=None, first_page=0):
        from paper_2607_09686_amd import KvCache  # noqa: F401
        rng = np.random.default_rng(seed)
        self.torch, self.seqs, self.dtype = torch, seqs, dtype
        self.heads, self.kv_heads, self.dim, self.page = heads, kv_heads, dim, page
        self.new, self.total = [n for n, _ in seqs], [n + p for n, p in seqs]
        counts = [-(-t // page) for t in self.total]
        self.n_pages = first_page + sum(counts) + spare
        self.width = width or max(counts + [1])
        ids = first_page + rng.permutation(sum(counts) + spare)
        self.table = np.full((len(seqs), self.width), 2 ** 30, np.int32)
        at = 0
        for s, c in enumerate(counts):
            self.table[s, :c] = ids[at:at + c]
            at += c
        self.n = sum(self.new) + pad_rows
        self.k = [rng.standard_normal((t, kv_heads, dim)) for t in self.total]
        self.v = [rng.standard_normal((t, kv_heads, dim)) for t in self.total]
        self.q = rng.standard_normal((self.n, heads, dim)) * q_scale
        self.k, self.v = [self.rounded(x) for x in self.k], [self.rounded(x) for x in self.v]
        self.q = self.rounded(self.q)
        front = (1, self.n_pages, kv_heads, page // 16)
        self.keys = torch.full(front + (dim // 8, 16, 8), float("nan"), dtype=dtype, device="cuda")
        self.values = torch.full(front + (2, dim, 8), float("nan"), dtype=dtype, device="cuda")
        self.pages = torch.from_numpy(self.table).cuda()
        self.starts = torch.tensor(np.cumsum([0] + self.new), dtype=torch.int32, device="cuda")
        self.lengths = torch.tensor(self.total, dtype=torch.int32, device="cuda")
        if filled:
            for s in range(len(seqs)):
                self.fill(s)

    def rounded(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x)).to(self.dtype).double().numpy()

    def fill(self, s, upto=None):
        """Writes sequence s's first tokens (all) to its pages."""
        n = self.total[s] if upto is None else upto
        if n == 0:
            return
        torch = self.torch
        t = np.arange(n)
        page, place = self.table[s, t // self.page], t % self.page
        k = torch.from_numpy(self.k[s][:n]).to(self.dtype).cuda()
        v = torch.from_numpy(self.v[s][:n]).to(self.dtype).cuda()
        page, place = torch.from_numpy(page).long().cuda(), torch.from_numpy(place).cuda()
        self.keys[0][page, :, place // 16, :, place % 16] = k.view(n, self.kv_heads, self.dim // 8, 8)
        self.values[0][page, :, place // 16, place // 8 % 2, :, place % 8] = v

    def cache(self, **kw):
        from paper_2607_09686_amd import KvCache
        return KvCache(1, self.heads, self.kv_heads, self.dim, self.page, self.n_pages, dtype=self.dtype,
                       keys=self.keys, values=self.values, **kw)

    def q_gpu(self):
        return self.torch.from_numpy(self.q).to(self.dtype).cuda()

    def rows(self, s):
        a = sum(self.new[:s])
        return slice(a, a + self.new[s])

    def positions(self, s):
        return np.arange(self.total[s] - self.new[s], self.total[s])

    def check(self, out, window=0, scale=None, skip=()):
        """`out` against the oracle.  A row's error: its rounding to the type, h |o|; each
        probability's, h p, so h sum p |v|; and the fp32 arithmetic's, relative to sum p |v|: a
        score off by ds changes probabilities by 2 ds (numerator and sum), ds being at most
        (dim + 8) roundings of the products' absolute sum (here at most the largest |q| |k|, by
        Cauchy's inequality) plus the exponential's and the sums' own, 2^-18 together."""
        h = half_step(self.dtype)
        scale = self.dim ** -0.5 if scale is None else scale
        tiny = float(self.torch.finfo(self.dtype).smallest_normal) * h
        got = out.double().cpu().numpy()
        worst = 0.0
        for s in range(len(self.seqs)):
            if not self.new[s] or s in skip:
                continue
            r = self.rows(s)
            want, weight = ref.attend(self.q[r], self.k[s], self.v[s], self.positions(s), scale, window)
            big = (np.linalg.norm(self.q[r], axis=2).max() * np.linalg.norm(self.k[s], axis=2).max() * scale)
            ds = (self.dim + 8) * 2.0 ** -24 * big
            tol = h * np.abs(want) + (h + 2 * ds + 2.0 ** -18) * (1 + h) * weight + 4 * tiny
            err = np.abs(got[r] - want)
            assert np.all(np.isfinite(got[r])), (s, self.seqs[s])
            worst = max(worst, float((err / tol).max()))
            assert np.all(err <= tol), (s, self.seqs[s], float((err / tol).max()),
                                        np.unravel_index(np.argmax(err / tol), err.shape))
        return worst
