"""Dense attention over packed sequences and over a paged cache, plainly and in 64 bits, with numpy on the host, and how far a kernel that
keeps fp32 sums and rounds weights and results to bf16 may be from it."""
import numpy as np
import torch

LOWEST, HIGHEST = -64, 63
LARGEST = 448.0
U = 2.0 ** -24    # rounding of one fp32 operation, relative
U16 = 2.0 ** -8   # of one to bf16
ALL = 2 ** 31 - 1

# values of the 128 codes without sign: 4 exponent bits of bias 7, 3 mantissa bits, the last code NaN
LEVELS = np.array([m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)])
LEVELS[127] = np.nan


def to64(t):
    """float64 numpy values of a tensor."""
    return t.detach().cpu().double().numpy()


def quantize(x):
    """Rows x [.., D] float64 -> codes [.., D], exponents [..].  A NaN gets code 127 and does not count, what is beyond the largest value becomes it."""
    size = np.abs(x)
    top = np.where(np.isnan(size), 0.0, size).max(axis=-1)
    e = np.full(top.shape, LOWEST)
    for power in range(LOWEST, HIGHEST):
        e = np.where(top > LARGEST * 2.0 ** power, power + 1, e)
    with np.errstate(over="ignore"):
        y = size / np.exp2(e)[..., None]
    codes = np.zeros(x.shape, dtype=np.int64)
    for c in range(1, 127):  # the nearest level; of two equally near ones the even code
        border = (LEVELS[c - 1] + LEVELS[c]) / 2
        codes = np.where((y > border) | ((y == border) & (c % 2 == 0)), c, codes)
    codes = np.where(np.isnan(y), 127, codes)
    return np.where(np.signbit(x), codes + 128, codes), e


def values(codes, exponents):
    v = LEVELS[codes & 127]
    return np.where(codes >= 128, -v, v) * np.exp2(exponents.astype(np.float64))[..., None]


def legal(t, rows, m, mask):
    if mask == 0:
        return rows
    return 0 if t < 0 else min(rows, (t + 1) // m)


def attend(q, K, V, position, m, mask, n_win, scale, there=None):
    """One sequence: q [S,H,D], K and V [T,H_kv,D] float64, position [S], there [T] (which rows there are, None: all).  Returns out, lse, and how far
    a kernel may be from either.

    A logit is a sum of D exact products: fp32 sums are within (D + 2) U of the sum of magnitudes; A is the largest such sum of a query, scaled.
    Reference, scaling and exponential add U of the exponent's size (at most A + |reference|, both at most A, in log2 units) and 2 U: a weight is off by
    eps relative to itself before it is rounded to bf16, U16 at most.  A sum over n weights adds n U, joining up to 64 parts as many steps of
    an exponential and a sum each (8 U a step), the quotient 2 U, the result's rounding U16.  A weight below 2^-126 of its reference may vanish, and
    one below 2^-133 of it, whose bf16 number does: the sum of weights is 2^-10 at least in these units where every reference is within 2^10 of the maximum."""
    S, H, D = q.shape
    T, H_kv = K.shape[:2]
    out, lse = np.zeros((S, H, D)), np.full((S, H), -np.inf)
    out_tol, lse_tol = np.zeros_like(out), np.zeros_like(lse)
    for i in range(S):
        n = legal(position[i], T, m, mask)
        rows = np.arange(max(0, n - n_win), n)
        if there is not None:
            rows = rows[there[rows]]
        if len(rows) == 0:
            continue
        for g in range(H):
            h = g // (H // H_kv)
            k, v = K[rows, h], V[rows, h]
            x = scale * (k @ q[i, g])
            top = x.max()
            lse[i, g] = top + np.log(np.exp(x - top).sum())
            p = np.exp(x - lse[i, g])
            out[i, g] = p @ v
            A = abs(scale) * (np.abs(k) @ np.abs(q[i, g])).max()
            eps = U * ((D + 2) * A + 2 * (2 * A + 16) + 4)
            steps = (len(rows) + 4 + 64 * 8) * U
            out_tol[i, g] = (U16 + 2 * eps + steps) * (p @ np.abs(v)) * (1 + U16) + U16 * np.abs(out[i, g]) + 2.0 ** -100 * np.abs(v).sum(axis=0)
            lse_tol[i, g] = eps + steps + 4 * U * abs(lse[i, g])
    return out, lse, out_tol, lse_tol


class Pages:
    """A cache whose pages are handed out in a shuffled order, `spare` of them to nobody; rows that no sequence holds, and pages of nobody, are filled with
    `filler`.  lengths: rows a sequence holds, of K and V [T,H,D] lists (float32 tensors, taken to what the cache holds)."""

    def __init__(self, seed, lengths, H, D, bits, page, shared=False, filler=float("nan"), wide=None, spare=2):
        g = torch.Generator().manual_seed(seed)
        used = [-(-n // page) for n in lengths]
        self.n_pages = sum(used) + spare
        wide = max(1, wide or max(used))
        order = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((len(lengths), wide), -1, dtype=torch.int32)
        self.K, self.V = torch.full((2, self.n_pages, H, page, D), filler).to(torch.bfloat16)
        self.k64, self.v64 = [], []
        at = 0
        for b, n in enumerate(lengths):
            self.table[b, :used[b]] = order[at:at + used[b]].to(torch.int32)
            for which, (pages, rows64) in enumerate(((self.K, self.k64), (self.V, self.v64))):
                x = torch.randn((n, H, D), generator=g) * torch.exp(0.5 * torch.randn((n, H, 1), generator=g)) + (0.4 if which else 0.0)
                x = x.to(torch.bfloat16)
                for i in range(used[b]):
                    part = x[i * page:(i + 1) * page]
                    pages[order[at + i], :, :len(part)] = part.transpose(0, 1)
                rows64.append(to64(x))
            at += used[b]
        self.k_scales = self.v_scales = None
        if bits == 8:
            self.k64 = [values(*quantize(x)) for x in self.k64]
            self.v64 = [values(*quantize(x)) for x in self.v64]
            (self.K, self.k_scales), (self.V, self.v_scales) = self._codes(self.K), self._codes(self.V)
        if shared:
            self.V, self.v_scales, self.v64 = None, None, self.k64

    @staticmethod
    def _codes(pages):
        codes, e = quantize(to64(pages))
        return torch.from_numpy(codes.astype(np.uint8)), torch.from_numpy((e + 127).astype(np.uint8))

    def to(self, dev):
        """table, K, V, k_scales, v_scales on the GPU."""
        return [None if t is None else t.to(dev) for t in (self.table, self.K, self.V, self.k_scales, self.v_scales)]
