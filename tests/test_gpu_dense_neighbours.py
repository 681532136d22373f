"""GPU tests that a head's result does not depend, not by a bit, on the logits of the heads and positions that share its workgroup."""
import numpy as np
import pytest
import torch

import paper_2605_02568_amd as P
from tests import dense_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NONE, CAUSAL = P.SI_MASK_NONE, P.SI_MASK_CAUSAL_BLOCK


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _inputs(S, T, H, H_kv, D):
    """Queries, and the same with head 1 a thousand times as large in every third of them; rows that grow, so that its maxima rise again and again."""
    g = torch.Generator().manual_seed(S + D)
    q = torch.randn((S, H, D), generator=g).to(torch.bfloat16)
    k = (torch.randn((T, H_kv, D), generator=g) * torch.linspace(0.5, 1.5, T)[:, None, None]).to(torch.bfloat16)
    v = torch.randn((T, H_kv, D), generator=g).to(torch.bfloat16)
    large = q.clone()
    large[::3, 1] *= 1000
    same = torch.ones((S, H), dtype=torch.bool)
    same[::3, 1] = False
    return q, large, k, v, same.to(DEV)


@pytest.mark.parametrize("S,H,H_kv,D", [(300, 6, 2, 64), (300, 16, 2, 128), (1200, 32, 4, 128), (2100, 32, 8, 128)])  # the four forms of the kernel
@pytest.mark.parametrize("mask,n_win", [(CAUSAL, R.ALL), (CAUSAL, 200), (NONE, R.ALL)])
def test_prompts(S, H, H_kv, D, mask, n_win):
    q, large, k, v, same = _inputs(S, S, H, H_kv, D)
    print(f"neighbours S={S} H={H}/{H_kv} D={D} mask={mask} n_win={n_win}", flush=True)
    results = []
    for x in (q, large):
        out, lse = torch.full(q.shape, 55.0, dtype=torch.bfloat16, device=DEV), torch.full(q.shape[:2], 55.0, device=DEV)
        P.si_prompt_attention(x.to(DEV), k.to(DEV), v.to(DEV), None, None, None, 1, mask, n_win, 0.1, out, lse)
        torch.cuda.synchronize()
        results.append((out, lse))
    (out, lse), (out2, lse2) = results
    assert torch.equal(out[same], out2[same]) and torch.equal(lse[same], lse2[same])
    assert not torch.equal(lse, lse2)


@pytest.mark.parametrize("S,H,H_kv,D", [(4, 8, 2, 64), (4, 8, 1, 128), (4, 16, 1, 64), (4, 16, 1, 128)])  # 16, 32 and 64 columns
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("n_win", [R.ALL, 200])
def test_pages(S, H, H_kv, D, bits, n_win):
    T, page = 3000, 16
    q, large, k, v, same = _inputs(S, T, H, H_kv, D)
    n = -(-T // page)
    K, V = torch.zeros((2, n, H_kv, page, D), dtype=torch.bfloat16 if bits == 16 else torch.uint8, device=DEV)
    scales = [None, None] if bits == 16 else list(torch.full((2, n, H_kv, page), 127, dtype=torch.uint8, device=DEV))
    table = _ints([list(range(n))])
    P.si_store_pages(k.to(DEV), v.to(DEV), None, None, table, K, V, *scales)
    ws = torch.empty(P.si_paged_workspace_bytes(1, S, H, H_kv, D), dtype=torch.uint8, device=DEV)
    print(f"neighbours S={S} H={H}/{H_kv} D={D} bits={bits} n_win={n_win}", flush=True)
    results = []
    for x in (q, large):
        out, lse = torch.full((1, S, H, D), 55.0, dtype=torch.bfloat16, device=DEV), torch.full((1, S, H), 55.0, device=DEV)
        P.si_paged_attention(x.to(DEV)[None], table, K, V, *scales, _ints([T]), _ints([T - S]), 1, CAUSAL, n_win, 0.1, out, lse, ws)
        torch.cuda.synchronize()
        results.append((out[0], lse[0]))
    (out, lse), (out2, lse2) = results
    assert torch.equal(out[same], out2[same]) and torch.equal(lse[same], lse2[same])
    assert not torch.equal(lse, lse2)
    want = R.attend(R.to64(q), *([R.to64(k), R.to64(v)] if bits == 16 else [R.values(*R.quantize(R.to64(x))) for x in (k, v)]), range(T - S, T), 1, 1, n_win, 0.1)
    assert np.all(np.abs(R.to64(out) - want[0]) <= want[2]) and np.all(np.abs(R.to64(lse) - want[1]) <= want[3])
