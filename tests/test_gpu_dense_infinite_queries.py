"""GPU tests of queries that hold an infinity where every logit that it makes is minus infinity: NaN in that head's result and lse wherever a row is seen, 0 and
minus infinity where none is, and nothing in any other head's."""
import numpy as np
import pytest
import torch

import paper_2605_02568_amd as P
from tests import dense_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NONE, CAUSAL = P.SI_MASK_NONE, P.SI_MASK_CAUSAL_BLOCK
AT = 3  # the coordinate with the infinity: keys are positive there, so all products with it have one sign


def _ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def _near(got, lse, want):
    ro, rl, to, tl = want
    none = np.isneginf(rl)
    lse = R.to64(lse)
    assert np.all(np.abs(R.to64(got) - ro) <= to)
    assert np.all(np.isneginf(lse[none])) and np.all(np.abs(lse[~none] - rl[~none]) <= tl[~none])


def _inputs(seed, T, H_kv, q_shape, D):
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn((T, H_kv, D), generator=g).to(torch.bfloat16) for _ in range(2))
    k[..., AT] = k[..., AT].abs() + 0.5
    return k, v, torch.randn((*q_shape, D), generator=g).to(torch.bfloat16)


# 16, 32 and 64 columns a workgroup; sequences that stay whole, and that are dealt out over the chip and joined
@pytest.mark.parametrize("H,H_kv", [(4, 2), (24, 1), (64, 1)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("wide", [40, 140])
@pytest.mark.parametrize("scale", [0.1, -0.1])
def test_over_pages(H, H_kv, D, bits, wide, scale):
    T, page, B = 600, 16, 4
    k, v, q = _inputs(H + D, T, H_kv, (B, 2, H), D)
    bad = q.clone()
    bad[:, :, 1, AT] = -np.sign(scale) * float("inf")
    n = -(-T // page)
    dtype = torch.bfloat16 if bits == 16 else torch.uint8
    K, V = torch.zeros((2, n, H_kv, page, D), dtype=dtype, device=DEV)
    scales = [None, None] if bits == 16 else list(torch.full((2, n, H_kv, page), 127, dtype=torch.uint8, device=DEV))
    whole = torch.full((1, wide), -1, dtype=torch.int32)
    whole[0, :n] = torch.arange(n)
    P.si_store_pages(k.to(DEV), v.to(DEV), None, None, whole.to(DEV), K, V, *scales)
    table = whole.repeat(B, 1)
    table[2, :] = -1      # no page is there
    table[3, :n - 1] = -1  # the last one only
    lengths, first = [T, 0, T, T], [T - 2, T - 2, T - 2, T - 2]
    ws = torch.empty(P.si_paged_workspace_bytes(B, 2, H, H_kv, D), dtype=torch.uint8, device=DEV)

    def attend(q, n_win, first):
        out, lse = torch.full(q.shape, 55.0, dtype=torch.bfloat16, device=DEV), torch.full(q.shape[:3], 55.0, device=DEV)
        P.si_paged_attention(q.to(DEV), table.to(DEV), K, V, *scales, _ints(lengths), _ints(first), 1, CAUSAL, n_win, scale, out, lse, ws)
        torch.cuda.synchronize()
        return out, lse

    print(f"pages H={H}/{H_kv} D={D} bits={bits} wide={wide} scale={scale}", flush=True)
    others = [h for h in range(H) if h != 1]
    for n_win in (R.ALL, 5, 0):
        for start in (first, [-1, -1, -2, 0]):  # with positions before the first row
            clean, clean_lse = attend(q, n_win, start)
            out, lse = attend(bad, n_win, start)
            assert torch.equal(out[:, :, others], clean[:, :, others]) and torch.equal(lse[:, :, others], clean_lse[:, :, others])
            sees = ~torch.isneginf(clean_lse[:, :, 1])  # a finite query's lse is finite where it sees a row
            assert bool(sees[0].any()) == (n_win != 0) and not bool(sees[1:3].any())
            assert bool(torch.isnan(out[:, :, 1][sees]).all()) and bool(torch.isnan(lse[:, :, 1][sees]).all())
            assert bool((out[:, :, 1][~sees] == 0).all()) and bool(torch.isneginf(lse[:, :, 1][~sees]).all())
    if bits == 16:
        clean, clean_lse = attend(q, R.ALL, first)
        _near(clean[0], clean_lse[0], R.attend(R.to64(q[0]), R.to64(k), R.to64(v), [T - 2, T - 1], 1, 1, R.ALL, scale))


# the four forms of the kernel: by queries, heads and rows
@pytest.mark.parametrize("S,T,H,H_kv,D", [(90, 90, 6, 2, 64), (300, 300, 16, 2, 128), (1200, 1200, 32, 4, 128), (2100, 2100, 32, 8, 128)])
@pytest.mark.parametrize("n_win", [R.ALL, 50])
@pytest.mark.parametrize("scale", [0.1, -0.1])
def test_over_packed_rows(S, T, H, H_kv, D, n_win, scale):
    k, v, q = _inputs(S, T, H_kv, (S, H), D)
    bad = q.clone()
    bad[:, 1, AT] = -np.sign(scale) * float("inf")

    def attend(q):
        out, lse = torch.full(q.shape, 55.0, dtype=torch.bfloat16, device=DEV), torch.full(q.shape[:2], 55.0, device=DEV)
        P.si_prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), None, None, _ints([-3]), 1, CAUSAL, n_win, scale, out, lse)  # the first three see nothing
        torch.cuda.synchronize()
        return out, lse

    print(f"prompt S={S} H={H}/{H_kv} D={D} n_win={n_win} scale={scale}", flush=True)
    clean, clean_lse = attend(q)
    out, lse = attend(bad)
    others = [h for h in range(H) if h != 1]
    assert torch.equal(out[:, others], clean[:, others]) and torch.equal(lse[:, others], clean_lse[:, others])
    assert bool(torch.isnan(out[3:, 1]).all()) and bool(torch.isnan(lse[3:, 1]).all())
    assert bool((out[:3, 1] == 0).all()) and bool(torch.isneginf(lse[:3, 1]).all())
    some = [0, 2, 3, 4, 40, S // 2, S - 1]
    want = R.attend(R.to64(q[some]), R.to64(k), R.to64(v), [i - 3 for i in some], 1, 1, n_win, scale)
    _near(clean[some], clean_lse[some], want)
