"""Inputs of the tests over caches of pages, and their tolerances.

Pages of a pool are owned in random order; page numbers behind a request's last page, slots behind its last token and pages that
nobody owns hold what must never be used: NaN, and page numbers out of range.
"""
import numpy as np
import torch

#: Half a step of a rounding, relative.
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class Pages:
    """A batch over a pool, on the CPU in fp64 (values of the stored dtype) and on the GPU."""

    def __init__(self, dtype, new, lens, Hq, Hkv, D, ps, seed=0, spare=3, wild=True, shift=0.0, tail=0):
        self.g = g = np.random.default_rng(seed)
        self.dtype, self.t = dtype, TYPES[dtype]
        self.new, self.lens, self.B, self.Hq, self.Hkv, self.D, self.ps = list(new), list(lens), len(lens), Hq, Hkv, D, ps
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.total = int(self.cu[-1]) + tail               # rows behind the last request
        pages = [-(-n // ps) for n in lens]
        self.num_pages = sum(pages) + spare
        order = g.permutation(self.num_pages)
        self.max_pages = max(max(pages), 1) + 1
        self.table = np.full((self.B, self.max_pages), 1 << 30 if wild else 0, np.int32)
        first = 0
        for b, k in enumerate(pages):
            self.table[b, :k] = order[first:first + k]
            first += k
        self.K, self.V = self.values(self.num_pages, ps, Hkv, D, shift=shift), self.values(self.num_pages, ps, Hkv, D)
        self.Q = self.values(self.total, Hq, D)
        self.W = g.random((self.num_pages, Hkv, ps)).astype(np.float32)
        if wild:                                           # NaN wherever no cached token lies
            owned = np.zeros((self.num_pages, ps), bool)
            for b, n in enumerate(lens):
                j = np.arange(n)
                owned[self.table[b, j // ps], j % ps] = True
            self.K[~owned], self.V[~owned] = np.nan, np.nan

    def values(self, *shape, shift=0.0):
        """Normal numbers, rounded to the stored dtype, as fp64."""
        x = torch.from_numpy(self.g.standard_normal(shape).astype(np.float32) + np.float32(shift)).to(self.t)
        return x.double().numpy()

    def dev(self, x):
        """fp64 values of the stored dtype -> device tensor of it; integers as they are."""
        t = torch.from_numpy(np.ascontiguousarray(x))
        return (t.to(self.t) if t.dtype == torch.float64 else t).cuda()

    def cache(self, seka, W=None, K=None, V=None):
        self.K_dev, self.V_dev = self.dev(self.K if K is None else K), self.dev(self.V if V is None else V)
        self.W_dev = None if W is None else torch.from_numpy(np.array(W, np.float32)).cuda()
        self.cu_dev = self.dev(self.cu)
        return seka.paged_cache(self.K_dev, self.V_dev, self.dev(self.table), self.dev(np.array(self.lens, np.int32)), W=self.W_dev)


def f64(t):
    return t.detach().double().cpu().numpy()


def score_error(size, D):
    """Bound of a score's error: D + 2 products and sums of fp32, each off by 2^-24 of the sum of the products' sizes, and the factor
    of the exponent (scale times log2 e, one more rounding each way)."""
    return (D + 6) * 2.0 ** -24 * size


def check_attention(O, L, ref, dtype, what, lse=True):
    """Probabilities are rounded to the operands' dtype before the product with V (bf16: half a step of every p_j |v_j|; fp32: none),
    and the result once.  Scores are off by score_error, which every exponential, and their sum, passes on; the exponential itself and
    sums of fp32 add 2^-20 of what is summed."""
    rO, rL, spread, size = ref
    D = O.shape[-1]
    e = 2 * score_error(size, D).T[..., None] + 2.0 ** -20
    bound = spread * ((HALF["bf16"] if dtype == "bf16" else 0.0) + e) + HALF[dtype] * np.abs(rO) * 1.01 + 1e-30
    off = np.abs(O - rO) - bound
    assert np.isfinite(O).all(), f"{what}: outputs that are not finite"
    assert (off <= 0).all(), f"{what}: O is off by {np.abs(O - rO).max():.3g}, {off.max():.3g} more than it may be"
    if lse:
        none = np.isneginf(rL)
        assert (np.isneginf(L) == none).all(), f"{what}: lse of rows that see nothing"
        far = np.abs(L[~none] - rL[~none]) - (score_error(size, D)[~none] + 2.0 ** -20 + 2.0 ** -23 * np.abs(rL[~none]))
        assert (far <= 0).all(), f"{what}: lse is {far.max():.3g} further off than it may be"
