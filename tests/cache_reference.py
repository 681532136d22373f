"""The operators of a cache held in 4 bits, plainly and in 64 bits, with numpy on the host, and how far a kernel that keeps
fp32 sums may be from them."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LOWEST, HIGHEST = -13, 13
U = 2.0 ** -24  # rounding of one fp32 operation, relative


def bf16_values(bits):
    """float64 values of bf16 bit patterns (uint16)."""
    with np.errstate(invalid="ignore"):  # signalling NaNs
        return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def quantize(x):
    """x [.., D] float64 -> codes [.., D] (0 .. 15), exponents [.., D / 32].  NaN: the largest code, not counted."""
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    top = np.where(np.isnan(blocks), 0.0, np.abs(blocks)).max(axis=-1)
    e = np.full(top.shape, LOWEST)
    for power in range(LOWEST, HIGHEST):
        e = np.where(top > 7.0 * 2.0 ** power, power + 1, e)
    y = np.abs(blocks) / np.exp2(e)[..., None]
    y = np.where(np.isnan(y), np.inf, y)
    # the nearest level; of two equally near ones the even code
    codes = np.zeros(blocks.shape, dtype=np.int64)
    for c in range(1, 8):
        border = (LEVELS[c - 1] + LEVELS[c]) / 2
        codes = np.where((y > border) | ((y == border) & (c % 2 == 0)), c, codes)
    codes = np.where(np.signbit(blocks), codes + 8, codes)
    return codes.reshape(x.shape), e


def pack(codes, e):
    c = codes.astype(np.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4), (e + 127).astype(np.uint8)


def values(codes, scales):
    """Packed codes [.., D / 2] and scale bytes [.., D / 32] -> float64 [.., D]."""
    c = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], -1)
    v = np.where(c >= 8, -LEVELS[c & 7], LEVELS[c & 7])
    return v * np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, axis=-1)


def held(lengths, b, T):
    return T if lengths is None else int(min(max(lengths[b], 0), T))


def selected(idx_row, t, n_held, m, mask, n_win):
    """U(t), ascending."""
    legal = n_held if mask == 0 else min(n_held, (t + 1) // m)
    rows = set(range(max(0, legal - n_win), legal))
    if idx_row is not None:
        rows |= {int(s) for s in idx_row if 0 <= s < n_held}
    return np.array(sorted(rows), dtype=np.int64)


def attend(q, V, lengths, idx, m, mask, n_win, scale):
    """q [B,S,H,D], V [B,T,D] float64.  Returns out, lse, given [B,T] (the softmax summed over queries and heads) and how far
    fp32 kernels may be from each of the three.

    A logit is a sum of D exact products: fp32 sums are within (D + 2) U of the sum of magnitudes; A is the largest such sum of a
    query and head, scaled.  Reference, scaling and exponential add U of the exponent's size (at most A + |reference|, both at most A, in
    log2 units) and 2 U.  So a weight is off by eps relative to itself; a sum over n of them adds n U, the quotient 2 U, and the split
    into two parts of 11 bits 2^-22.  The second part is an fp16 number, whose smallest step is 2^-24, and weights are held as 2^7 times
    exp2(logit - reference) where some row's logit was the reference: the sum of weights is at least 2^7, so each of the n weights is
    also off by up to 2^-25 / 2^7 = 2^-32 whatever its size."""
    B, S, H, D = q.shape
    T = V.shape[1]
    out, lse = np.zeros((B, S, H, D)), np.full((B, S, H), -np.inf)
    given = np.zeros((B, T))
    out_tol, lse_tol, given_tol = np.zeros_like(out), np.zeros_like(lse), np.zeros_like(given)
    for b in range(B):
        for t in range(S):
            U_t = selected(None if idx is None else idx[b, t], t, held(lengths, b, T), m, mask, n_win)
            if len(U_t) == 0:
                continue
            rows = V[b, U_t]
            x = scale * (q[b, t] @ rows.T)
            top = x.max(axis=1, keepdims=True)
            lse[b, t] = (top + np.log(np.exp(x - top).sum(axis=1, keepdims=True)))[:, 0]
            p = np.exp(x - lse[b, t][:, None])
            out[b, t] = p @ rows
            given[b, U_t] += p.sum(axis=0)
            A = abs(scale) * (np.abs(q[b, t]) @ np.abs(rows).T).max(axis=1)
            n = len(U_t)
            eps = U * ((D + 2) * A + 2 * (2 * A + 16) + 4)
            out_tol[b, t] = (2 * eps + (n + 4) * U + 2.0 ** -22)[:, None] * (p @ np.abs(rows)) + 2.0 ** -32 * np.abs(rows).sum(axis=0)
            lse_tol[b, t] = eps + (n + 4) * U + 4 * U * np.abs(lse[b, t])
            # with lse itself rounded: its U |lse|, that of its product with log2 e, then H sums, half a unit of 2^-32
            given_tol[b, U_t] += (p * (eps + 4 * U * np.abs(lse[b, t]) + (H + 4) * U)[:, None]).sum(axis=0) + 2.0 ** -33
    return out, lse, given, out_tol, lse_tol, given_tol


def evict(weights, lengths, n_keep, n_sink, n_recent):
    """weights [B,T] float32 -> per batch the rows that stay, ascending."""
    B, T = weights.shape
    stay = []
    for b in range(B):
        n = held(lengths, b, T)
        rank = [(s < n_sink or s >= n - n_recent, not np.isnan(weights[b, s]), 0.0 if np.isnan(weights[b, s]) else float(weights[b, s]), -s)
                for s in range(n)]
        best = sorted(range(n), key=lambda s: rank[s], reverse=True)[:n_keep]
        stay.append(sorted(best))
    return stay
