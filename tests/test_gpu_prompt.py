"""GPU tests of attention over packed prompts against 64-bit references."""
import numpy as np
import pytest
import torch

import paper_2605_02568_amd as P
from tests import dense_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NONE, CAUSAL = P.SI_MASK_NONE, P.SI_MASK_CAUSAL_BLOCK


def _ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def _offsets(lengths):
    return [0] + [int(x) for x in np.cumsum(lengths)]


def _inputs(seed, nq, nk, H, H_kv, D, shared):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((nq, H, D), generator=g).to(torch.bfloat16)
    K = (torch.randn((nk, H_kv, D), generator=g) * torch.exp(0.5 * torch.randn((nk, H_kv, 1), generator=g))).to(torch.bfloat16)
    V = None if shared else (torch.randn((nk, H_kv, D), generator=g) + 0.4).to(torch.bfloat16)
    return q, K, V


def _attend(q, K, V, qo, ko, first, m, mask, n_win, scale):
    out = torch.full(q.shape, 55.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full(q.shape[:2], 55.0, dtype=torch.float32, device=DEV)
    P.si_prompt_attention(q.to(DEV), K.to(DEV), None if V is None else V.to(DEV), _ints(qo), _ints(ko), _ints(first), m, mask, n_win, scale, out, lse)
    torch.cuda.synchronize()
    return out, lse


def _check(q, K, V, out, lse, qo, ko, first, m, mask, n_win, scale, some=None):
    """some: queries of each sequence that are looked at (all by default)."""
    V = K if V is None else V
    for b in range(len(qo) - 1):
        i = np.arange(qo[b + 1] - qo[b])
        if some is not None and len(i):
            i = np.unique(np.clip(some, 0, len(i) - 1))
        rows = slice(ko[b], ko[b + 1])
        at = qo[b] + i
        ro, rl, to, tl = R.attend(R.to64(q[at]), R.to64(K[rows]), R.to64(V[rows]), i + (0 if first is None else first[b]), m, mask, n_win, scale)
        got, got_lse = R.to64(out[at]), R.to64(lse[at])
        assert np.all(np.abs(got - ro) <= to), (b, np.nanmax(np.abs(got - ro) / np.maximum(to, 1e-300)))
        none = np.isneginf(rl)
        assert np.all(np.isneginf(got_lse[none]))
        assert np.all(np.abs(got_lse[~none] - rl[~none]) <= tl[~none]), b


CASES = [
    # queries, rows before, H, H_kv, D, mask, m, n_win
    ([1], [0], 8, 8, 128, CAUSAL, 1, R.ALL),
    ([130], [0], 16, 2, 128, CAUSAL, 1, R.ALL),
    ([33, 0, 1, 100, 64], [0, 0, 0, 0, 0], 64, 8, 128, CAUSAL, 1, R.ALL),
    ([65, 31], [0, 0], 64, 1, 128, CAUSAL, 1, R.ALL),
    ([90, 7, 200], [0, 150, 63], 33, 3, 64, CAUSAL, 1, R.ALL),
    ([100, 41], [3, 0], 8, 1, 64, CAUSAL, 4, R.ALL),
    ([300, 20], [0, 0], 5, 5, 64, CAUSAL, 1, 65),
    ([129], [500], 4, 2, 128, CAUSAL, 1, 128),
    ([70, 65], [10, 200], 6, 2, 128, NONE, 1, R.ALL),
    ([40, 30], [0, 90], 6, 2, 64, NONE, 1, 37),
    ([50], [0], 4, 4, 128, CAUSAL, 1, 0),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("shared", [False, True])
def test_attention(case, shared):
    lengths, before, H, H_kv, D, mask, m, n_win = case
    qo = _offsets(lengths)
    ko = _offsets([(n + p) // m for n, p in zip(lengths, before)])
    q, K, V = _inputs(3, qo[-1] + 5, max(1, ko[-1] + 3), H, H_kv, D, shared)  # rows behind the last sequence
    K[ko[-1]:] = float("nan")
    if V is not None:
        V[ko[-1]:] = float("nan")
    scale = 1.0 / np.sqrt(D)
    print(f"prompt {case} shared={shared}", flush=True)
    out, lse = _attend(q, K, V, qo, ko, before, m, mask, n_win, scale)
    _check(q, K, V, out, lse, qo, ko, before, m, mask, n_win, scale)
    assert bool((out[qo[-1]:] == 55.0).all()) and bool((lse[qo[-1]:] == 55.0).all())


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales(scale):
    q, K, V = _inputs(4, 90, 90, 4, 2, 64, False)
    out, lse = _attend(q, K, V, None, None, None, 1, CAUSAL, R.ALL, scale)
    _check(q, K, V, out, lse, [0, 90], [0, 90], None, 1, CAUSAL, R.ALL, scale)


def test_a_long_prompt():
    n = 5000
    q, K, V = _inputs(5, n, n, 8, 1, 128, False)
    out, lse = _attend(q, K, V, None, None, None, 1, CAUSAL, R.ALL, 0.09)
    _check(q, K, V, out, lse, [0, n], [0, n], None, 1, CAUSAL, R.ALL, 0.09, some=[0, 1, 31, 32, 63, 64, 1000, 2047, 2048, n - 2, n - 1])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_that_are_not_seen_may_hold_anything(bad, D):
    """Later rows, rows before the window, and rows of the next sequence."""
    lengths = [100, 90]
    qo = _offsets(lengths)
    q, K, V = _inputs(6, 190, 190, 4, 2, D, False)
    clean = _attend(q, K, V, qo, qo, None, 1, CAUSAL, 40, 0.1)
    K[50], V[51, 1, 3], V[130] = bad, bad, bad
    out, lse = _attend(q, K, V, qo, qo, None, 1, CAUSAL, 40, 0.1)
    t = np.concatenate([np.arange(n) for n in lengths])
    b = np.repeat([0, 1], lengths)
    for g in range(4):
        k_seen = (b == 0) & (t >= 50) & (t < 90)
        v_seen = ((b == 0) & (t >= 51) & (t < 91) & (g // 2 == 1)) | ((b == 1) & (t >= 30) & (t < 70))
        fine = torch.from_numpy(~(k_seen | v_seen)).to(DEV)
        assert torch.equal(out[fine, g], clean[0][fine, g])
        assert torch.equal(lse[fine, g], clean[1][fine, g])
        if bad != bad:
            assert bool(torch.isnan(lse[torch.from_numpy(k_seen).to(DEV), g]).all())
            assert bool(torch.isnan(out[torch.from_numpy(k_seen).to(DEV), g]).all())
        only = torch.from_numpy(v_seen & (b == 1)).to(DEV)
        assert bool((~torch.isfinite(out[only, g])).all())
