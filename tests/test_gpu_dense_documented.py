"""GPU tests of calls of the paged cache and of packed prompts that their headers allow beside the ordinary ones: values alone, values that are not used, scales of
zero and below it for every number of columns and either width, values near the end of the stated range, a batch without any row."""
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


def _near(got, lse, want):
    ro, rl, to, tl = want
    got, lse = R.to64(got), R.to64(lse)
    assert np.all(np.abs(got - ro) <= to), np.nanmax(np.abs(got - ro) / np.maximum(to, 1e-300))
    none = np.isneginf(rl)
    assert np.all(np.isneginf(lse[none])) and np.all(np.abs(lse[~none] - rl[~none]) <= tl[~none])


def _paged(q, pages, lengths, first, mask, n_win, scale):
    B, S, H, D = q.shape
    table, K, V, ks, vs = pages.to(DEV)
    out = torch.full(q.shape, 55.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((B, S, H), 55.0, device=DEV)
    ws = torch.empty(P.si_paged_workspace_bytes(B, S, H, K.shape[1], D), dtype=torch.uint8, device=DEV)
    P.si_paged_attention(q.to(DEV), table, K, V, ks, vs, _ints(lengths), _ints(first), 1, mask, n_win, scale, out, lse, ws)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D,H,page,lengths", [(64, 5, 16, [70, 0, 33]), (128, 8, 64, [5000, 3000, 1500])])  # a row a thread, and four
def test_either_of_keys_and_values_alone(bits, D, H, page, lengths):
    pages = R.Pages(D, lengths, H, D, bits, page, filler=3.0)
    table, K, V, ks, vs = pages.to(DEV)
    off = _ints([0] + [int(x) for x in np.cumsum(lengths)])
    N = sum(lengths)
    print(f"load bits={bits} D={D} H={H} N={N}", flush=True)

    def load(k, v):
        k, v = (torch.full((N, H, D), 77.0, dtype=torch.bfloat16, device=DEV) if wanted else None for wanted in (k, v))
        P.si_load_pages(table, K, V, ks, vs, off, None, k, v)
        torch.cuda.synchronize()
        return k, v

    k, v = load(True, True)
    np.testing.assert_array_equal(R.to64(k), np.concatenate(pages.k64))
    np.testing.assert_array_equal(R.to64(v), np.concatenate(pages.v64))
    assert torch.equal(load(False, True)[1], v) and torch.equal(load(True, False)[0], k)


@pytest.mark.parametrize("bits", [16, 8])
def test_values_that_a_cache_of_keys_does_not_take(bits):
    H, D, page = 2, 64, 16
    x = torch.randn((40, H, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    K = torch.zeros((3, H, page, D), dtype=torch.bfloat16 if bits == 16 else torch.uint8, device=DEV)
    K2 = K.clone()
    ks = None if bits == 16 else torch.zeros((3, H, page), dtype=torch.uint8, device=DEV)
    ks2 = None if ks is None else ks.clone()
    table = _ints([[2, 0, 1]])
    P.si_store_pages(x, torch.full_like(x, float("nan")), None, None, table, K, None, ks, None)
    P.si_store_pages(x, None, None, None, table, K2, None, ks2, None)
    torch.cuda.synchronize()
    assert torch.equal(K.view(torch.uint8), K2.view(torch.uint8)) and bool((K != 0).any()) and (ks is None or torch.equal(ks, ks2))


@pytest.mark.parametrize("H,H_kv", [(6, 2), (24, 1), (64, 1)])  # 16, 32 and 64 columns a workgroup
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("wide", [None, 140])  # sequences that stay whole, and that are dealt out
@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales_of_pages(H, H_kv, D, bits, wide, scale):
    lengths = [300, 37]
    pages = R.Pages(2, lengths, H_kv, D, bits, 16, wide=wide)
    q = torch.randn((2, 1, H, D), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16)
    print(f"scales H={H}/{H_kv} D={D} bits={bits} wide={wide} scale={scale}", flush=True)
    out, lse = _paged(q, pages, lengths, None, NONE, R.ALL, scale)
    for b in range(2):
        _near(out[b], lse[b], R.attend(R.to64(q[b]), pages.k64[b], pages.v64[b], [0], 1, 0, R.ALL, scale))


@pytest.mark.parametrize("S,H,H_kv,D", [(90, 6, 2, 64), (300, 16, 2, 128), (1200, 32, 4, 128), (2100, 32, 8, 128)])  # the four forms of the kernel
@pytest.mark.parametrize("scale", [0.0, -0.3])
def test_scales_of_prompts(S, H, H_kv, D, scale):
    g = torch.Generator().manual_seed(S)
    q, k, v = (torch.randn((S, h, D), generator=g).to(torch.bfloat16) for h in (H, H_kv, H_kv))
    out, lse = torch.full(q.shape, 55.0, dtype=torch.bfloat16, device=DEV), torch.full(q.shape[:2], 55.0, device=DEV)
    print(f"scales S={S} H={H}/{H_kv} D={D} scale={scale}", flush=True)
    P.si_prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), None, None, None, 1, CAUSAL, R.ALL, scale, out, lse)
    torch.cuda.synchronize()
    some = np.unique([0, 1, 31, 32, 33, S // 2, S - 1])
    _near(out[some], lse[some], R.attend(R.to64(q[some]), R.to64(k), R.to64(v), some, 1, 1, R.ALL, scale))


@pytest.mark.parametrize("D,H,H_kv", [(64, 8, 2), (128, 8, 1), (128, 64, 1)])
def test_values_near_the_end_of_their_range(D, H, H_kv):
    """1,000 rows of values up to 2^107, all of one sign: rows times the largest is 2^117.  Logits rise by 30 or so from the first row to the last, so that references lag."""
    T, page = 1000, 16
    pages = R.Pages(D, [T], H_kv, D, 16, page, wide=140, filler=0.0)
    g = torch.Generator().manual_seed(H)
    k = (torch.randn((T, H_kv, D), generator=g) * 0.1).to(torch.bfloat16)
    v = ((torch.rand((T, H_kv, D), generator=g) * 0.5 + 0.5) * 2.0 ** 107).to(torch.bfloat16)
    q = torch.randn((40, H, D), generator=g).to(torch.bfloat16)
    k[..., 0] = torch.linspace(0, 30, T)[:, None].to(torch.bfloat16)
    q[..., 0] = 10.0
    table, K, V, _, _ = pages.to(DEV)
    P.si_store_pages(k.to(DEV), v.to(DEV), None, None, table, K, V)
    out = torch.full((1, 2, H, D), 55.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((1, 2, H), 55.0, device=DEV)
    ws = torch.empty(P.si_paged_workspace_bytes(1, 2, H, H_kv, D), dtype=torch.uint8, device=DEV)
    P.si_paged_attention(q[:2].to(DEV)[None], table, K, V, None, None, _ints([T]), None, 1, NONE, R.ALL, 0.1, out, lse, ws)
    out2, lse2 = torch.full(q.shape, 55.0, dtype=torch.bfloat16, device=DEV), torch.full(q.shape[:2], 55.0, device=DEV)
    P.si_prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), None, None, None, 1, NONE, R.ALL, 0.1, out2, lse2)
    torch.cuda.synchronize()
    want = R.attend(R.to64(q), R.to64(k), R.to64(v), range(40), 1, 0, R.ALL, 0.1)
    _near(out2, lse2, want)
    _near(out[0], lse[0], [x[:2] for x in want])


@pytest.mark.parametrize("D,H,H_kv", [(64, 3, 1), (128, 16, 2)])
def test_prompts_without_any_row(D, H, H_kv):
    """Prompts shorter than m: there is no compressed row yet; the one that the call wants belongs to nobody."""
    lengths = [3, 1, 2]
    qo, ko = _ints([0, 3, 4, 6]), _ints([0, 0, 0, 0])
    q = torch.randn((sum(lengths), H, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    k = torch.full((1, H_kv, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    out, lse = torch.full_like(q, 55.0), torch.full(q.shape[:2], 55.0, device=DEV)
    P.si_prompt_attention(q, k, None, qo, ko, None, 4, CAUSAL, R.ALL, 0.1, out, lse)
    torch.cuda.synchronize()
    assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())
