"""Plain forms of the operators on paged caches, in 64 bits on the CPU, and their inputs."""
import numpy as np
import torch

D = 128
STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}       # half a step, relative


class Cache:
    """A pool whose rows hold NaN where no row of a sequence stands, and a table whose entries behind the
    last page of a sequence are no pages."""

    def __init__(self, lens, Hkv, page, dtype=torch.bfloat16, seed=0, device="cpu", spare=2, width=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.Hkv, self.page, self.dtype = list(lens), Hkv, page, dtype
        each = [-(-n // page) for n in lens]
        total = sum(each) + spare
        perm = torch.randperm(total, generator=g)
        junk = torch.tensor([-1, total, 2 ** 31 - 1, -2 ** 31, total + 5])
        wide = max(1, max(each) + 1, width)
        table = junk[torch.randint(0, 5, (len(lens), wide), generator=g)]
        at = 0
        for s, n in enumerate(each):
            table[s, :n] = perm[at:at + n]
            at += n
        self.table = table.to(torch.int32)
        self.K = torch.full((total, Hkv, page, D), float("nan"), dtype=dtype)
        self.V = torch.full_like(self.K, float("nan"))
        self.rows_k, self.rows_v = [], []                             # [Hkv, n, D] of every sequence
        for s, n in enumerate(lens):
            k = (torch.randn(Hkv, n, D, generator=g) * 1.5).to(dtype)
            v = torch.randn(Hkv, n, D, generator=g).to(dtype)
            self.rows_k.append(k)
            self.rows_v.append(v)
            for r in range(n):
                self.K[self.table[s, r // page], :, r % page] = k[:, r]
                self.V[self.table[s, r // page], :, r % page] = v[:, r]
        self.device = device

    def write(self, s, h, r, k=None, v=None):
        p = self.table[s, r // self.page]
        for rows, pool, x in ((self.rows_k, self.K, k), (self.rows_v, self.V, v)):
            if x is not None:
                rows[s][h, r] = x
                pool[p, h, r % self.page] = x

    def kv(self):
        import paper_2412_03213_amd as ck
        dev = self.device
        return ck.PagedKV(self.K.to(dev), self.V.to(dev), self.table.to(dev))

    def there(self, s):
        """Which rows of a sequence are on a page."""
        p = self.table[s].long()[torch.arange(self.lens[s]) // self.page]
        return ((p >= 0) & (p < self.K.shape[0])).numpy()


def attend(q, K, V, seen, dtype, scale=D ** -0.5, p_step=0.0):
    """q [M, D], K, V [n, D], seen [M, n] (or counts of a row) -> (out, tol) [M, D] in 64 bits.

    tol bounds what an implementation with fp32 scores, maximum, sum and accumulators may be off by: scores by
    D roundings of their terms (and two of the scaling), which a probability takes over as a relative error, also
    in the sum; probabilities by p_step relative on top; sums over n rows by n roundings; the output by one
    rounding of the type."""
    q, K, V = (x.double().numpy() for x in (q, K, V))
    seen = np.asarray(seen, dtype=np.float64)
    out, tol = np.zeros((q.shape[0], D)), np.zeros((q.shape[0], D))
    for i in range(q.shape[0]):
        r = np.nonzero(seen[i])[0]
        if r.size == 0:
            continue
        w = seen[i, r]
        s = K[r] @ q[i] * scale
        e = w * np.exp(s - s.max())
        p = e / e.sum()
        out[i] = p @ V[r]
        ds = 2.0 ** -24 * (D * (np.abs(K[r]) @ np.abs(q[i])).max() * scale + 4 * np.abs(s).max() + 4)
        size = p @ np.abs(V[r])
        tol[i] = STEP[dtype] * np.abs(out[i]) * (1 + 2.0 ** -6) + size * (
            p_step + 2 * ds + (r.size + 8) * 2.0 ** -23) + 1e-30
    return out, tol


def seen_rows(n, p, n_sink, window):
    """Rows r < n that a query at row p sees."""
    r = np.arange(n)
    if window < 0:
        return r <= p
    return (r <= p) & ((r < n_sink) | (r > p - window))


def turn(x, pos, freqs, factor, adjacent):
    """x [.., D] turned at position pos -> (out, tol) in 64 bits: products and sum in fp32 with fp32 cosines, one
    rounding of the type."""
    y = x.double().numpy()
    w = np.asarray(freqs, dtype=np.float64)
    half = w.size
    a = pos * w
    c, s = np.cos(a) * factor, np.sin(a) * factor
    out, size = y.copy(), np.zeros_like(y)
    i = np.arange(half)
    j1, j2 = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
    x1, x2 = y[..., j1], y[..., j2]
    out[..., j1], out[..., j2] = x1 * c - x2 * s, x2 * c + x1 * s
    both = (np.abs(x1) + np.abs(x2)) * max(1.0, abs(factor))
    size[..., j1] = size[..., j2] = both
    # cosine and sine within 4 roundings (argument 2, function 2), factor, product and sum one each
    tol = STEP[x.dtype] * np.abs(out) * (1 + 2.0 ** -6) + size * 8 * 2.0 ** -24
    tol[size == 0] = 0.0
    return out, tol
