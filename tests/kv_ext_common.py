"""Batches over a cache of 8 bits, and batches whose sequences begin with the same tokens."""
import numpy as np

from oracle import serving as ref
from serving_common import Batch

LIMITS = {"torch.bfloat16": (-100, 119), "torch.float16": (-15, 7)}  # of a scale's exponent


class ExtBatch(Batch):
    """As Batch; `held`: keys and values in 8 bits (k and v become what the numbers stand for; unused
    places hold NaN numbers and 255, which is no scale); `shared`: all sequences begin with the first
    one's first `shared` tokens, whole pages of which are the same pages."""

    def __init__(self, torch, seqs, heads, kv_heads, dim, page, dtype, held=True, shared=0, own_front=False, **kw):
        filled = kw.pop("filled", True)
        super().__init__(torch, seqs, heads, kv_heads, dim, page, dtype, filled=False, **kw)
        self.held, self.shared = held, shared
        front = shared // page
        for s in range(1, len(seqs)):
            if self.total[s] < shared:  # one without new tokens need not have them
                continue
            self.k[s][:shared], self.v[s][:shared] = self.k[0][:shared], self.v[0][:shared]
            if not own_front:
                self.table[s, :front] = self.table[0, :front]
        self.pages = torch.from_numpy(self.table).cuda()
        if shared:
            self.prefix = self.pages[0, :-(-shared // page)].clone()
            self.count = torch.tensor([shared], dtype=torch.int32, device="cuda")
        if held:
            limits = LIMITS[str(dtype)]
            self.codes = [[ref.hold(x[s], *limits) for s in range(len(seqs))] for x in (self.k, self.v)]
            for x, codes in ((self.k, self.codes[0]), (self.v, self.codes[1])):
                for s, (c, e) in enumerate(codes):
                    x[s] = c * 2.0 ** e[..., None].astype(np.float64)
            pool = (1, self.n_pages, kv_heads, page // 16)
            nan = lambda *s: torch.full(pool + s, 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)  # noqa: E731
            self.keys, self.values = nan(dim // 16, 16, 16), nan(2, dim, 8)
            none = lambda: torch.full((1, self.n_pages, kv_heads, page), 255, dtype=torch.uint8,  # noqa: E731
                                      device="cuda").view(torch.float8_e8m0fnu)
            self.key_scales, self.value_scales = none(), none()
        if filled:
            for s in range(len(seqs)):
                self.fill(s)

    def pools(self):
        """Every pool's bytes, to be compared or written at a place."""
        u8 = self.torch.uint8
        if not self.held:
            return [self.keys.view(self.torch.int16), self.values.view(self.torch.int16)]
        return [x.view(u8) for x in (self.keys, self.values, self.key_scales, self.value_scales)]

    def fill(self, s, upto=None):
        if not self.held:
            return super().fill(s, upto)
        n = self.total[s] if upto is None else upto
        if n == 0:
            return
        torch, t = self.torch, np.arange(n)
        page = torch.from_numpy(self.table[s, t // self.page]).long().cuda()
        at = torch.from_numpy(t % self.page).cuda()
        number = lambda c: torch.from_numpy(c[:n]).float().to(torch.float8_e4m3fn).view(torch.uint8).cuda()  # noqa: E731
        byte = lambda e: torch.from_numpy(e[:n] + 127).to(torch.uint8).cuda()  # noqa: E731
        keys, values, ks, vs = (x[0] for x in self.pools())
        (kc, ke), (vc, ve) = self.codes[0][s], self.codes[1][s]
        keys[page, :, at // 16, :, at % 16] = number(kc).view(n, self.kv_heads, self.dim // 16, 16)
        values[page, :, at // 16, at // 8 % 2, :, at % 8] = number(vc)
        ks[page, :, at], vs[page, :, at] = byte(ke), byte(ve)

    def cache(self, **kw):
        if not self.held:
            return super().cache(**kw)
        return super().cache(storage=self.torch.float8_e4m3fn, key_scales=self.key_scales,
                             value_scales=self.value_scales, **kw)

    def index(self):
        return self.pages, self.starts, self.lengths

    def front(self):
        return {"prefix": self.prefix, "shared": self.count} if self.shared else {}
