"""GPU: the 4-bit cache's attention and accumulated weights at the ends of what their arguments may be: values of a query far from one
another, products beyond fp32 that the softmax scale brings back, rows that receive little, every kernel that adds weights up."""
import numpy as np
import pytest
import torch

import paper_2605_02568_amd as P
from tests import cache_reference as R
from tests.test_gpu_cache import CAUSAL, DEV, NONE, _check, _gpu, _problem, _run

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------- values of a head far from one another
def _far_apart(seed, B, S, H, D, T, k, low, high, heads):
    """Queries of size 2^low with one value of 2^high in some heads, where the rows of the cache have zeros."""
    q, codes, scales, idx = _problem(seed, B, S, H, D, T, k, None, NONE, 1)
    at = D // 2 + 3
    q = (q.float() * 2.0 ** low).to(torch.bfloat16)
    q[:, :, heads, at] = 2.0 ** high
    codes[:, :, at // 2] &= 0x0F  # value `at` is odd: the high half
    return q, codes, scales, idx


@pytest.mark.parametrize("S,H,D", [(1, 64, 128), (3, 20, 64), (40, 64, 128), (300, 64, 128), (300, 40, 128), (300, 16, 128), (300, 33, 64),
                                   (300, 64, 64), (700, 9, 64), (300, 20, 128)])
@pytest.mark.parametrize("high", [31, 32, 36, 40, 126])
def test_a_value_far_above_the_others(S, H, D, high):
    """The logits consist of what lies far below a head's largest value: to the same tolerance as any others."""
    print(f"S={S} H={H} D={D} high={high}", flush=True)
    q, codes, scales, idx = _far_apart(high, 1, S, H, D, 150, 70, 0, high, slice(0, None, 3))
    _check(q, codes, scales, None, idx, 1, NONE, 33, 0.1)
    if high in (32, 126):
        _check(q, codes, scales, None, idx, 1, NONE, 33, -0.1)
        _check(q, codes, scales, None, idx, 1, NONE, 33, 0.0)


@pytest.mark.parametrize("S,H,D,T,k", [(1, 64, 128, 1700, 1600), (1, 20, 64, 1700, 1600), (40, 64, 128, 1700, 1600), (40, 64, 64, 1700, 1600),
                                       (40, 64, 64, 150, 70), (1, 5, 128, 40, 3)])
def test_a_value_far_above_the_others_of_few_queries(S, H, D, T, k):
    """Every number of waves and share of d that few queries come with."""
    print(f"S={S} H={H} D={D} T={T} k={k}", flush=True)
    q, codes, scales, idx = _far_apart(T + S, 1, S, H, D, T, k, 0, 50, slice(0, None, 5))
    _check(q, codes, scales, None, idx, 1, NONE, 3, 0.1)


@pytest.mark.parametrize("S,H,D", [(2, 33, 128), (400, 48, 64), (400, 33, 128)])
def test_values_far_apart_in_batches_that_hold_little(S, H, D):
    """Batches with all rows, none, some and one; queries without any; rising logits."""
    q, codes, scales, idx = _far_apart(S, 4, S, H, D, 150, 70, 4, 60, slice(0, None, 3))
    _check(q, codes, scales, [150, 0, 31, 1], idx, 1, NONE, 0, 0.3)
    _check(q, codes, scales, [150, 0, 31, 1], idx, 1, CAUSAL, 20, -0.3)


@pytest.mark.parametrize("S,H,D", [(2, 33, 128), (300, 64, 128), (300, 16, 64), (300, 48, 128)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_queries_that_are_not_finite_beside_values_far_apart(S, H, D, bad):
    """The head (not one of those with far values) has NaN, no other head of the block anything else than without it."""
    q, codes, scales, idx = _far_apart(S, 1, S, H, D, 150, 70, 0, 60, slice(0, None, 3))
    idx[0, S - 1] = np.arange(70)
    clean, clean_lse, _ = _run(q, codes, scales, None, idx, 1, NONE, 9, 0.1)
    q[0, S - 1, H - 2, 5] = bad
    out, lse, weights = _run(q, codes, scales, None, idx, 1, NONE, 9, 0.1)
    assert np.isnan(lse[0, S - 1, H - 2]) and np.all(np.isnan(out[0, S - 1, H - 2]))
    out[0, S - 1, H - 2], lse[0, S - 1, H - 2] = clean[0, S - 1, H - 2], clean_lse[0, S - 1, H - 2]
    assert np.array_equal(out, clean) and np.array_equal(lse, clean_lse)
    assert np.all(np.isfinite(weights))


@pytest.mark.parametrize("S,H,D", [(1, 64, 128), (300, 64, 128), (300, 40, 64), (300, 16, 128)])
@pytest.mark.parametrize("low,high,scale", [(-110, 0, 1e32), (-110, 100, 1e32), (-60, 60, 1e17), (60, 120, 1e-19), (100, 127, 1e-31), (-126, -80, 1e37),
                                            (-10, 126, 1e2)])
def test_values_far_apart_and_far_from_one(S, H, D, low, high, scale):
    print(f"S={S} H={H} D={D} low={low} high={high} scale={scale}", flush=True)
    q, codes, scales, idx = _far_apart(S, 1, S, H, D, 150, 70, low, high, slice(1, None, 2))
    _check(q, codes, scales, None, idx, 1, NONE, 33, scale)


@pytest.mark.parametrize("S", [1, 30, 300])
def test_denormal_values_that_the_scale_brings_back(S):
    """Queries of bf16's denormal numbers, alone and beside values that rows of zeros meet."""
    q, codes, scales, idx = _problem(3, 1, S, 20, 64, 150, 70, None, NONE, 1, q_size=2.0 ** -128)
    _check(q, codes, scales, None, idx, 1, NONE, 9, 2.0 ** 125)
    q[:, :, ::2, 5] = 2.0 ** -20
    codes[:, :, 2] &= 0x0F
    _check(q, codes, scales, None, idx, 1, NONE, 9, 2.0 ** 125)


@pytest.mark.parametrize("S", [1, 300])
def test_rows_of_zeros_under_the_largest_queries(S):
    """All logits are 0, whatever scale and query: every row counts alike."""
    q, codes, scales, idx = _problem(3, 1, S, 33, 128, 100, 40, None, NONE, 1, q_size=2.0 ** 120)
    codes[:] = 0x80  # zeros of either sign
    _check(q, codes, scales, None, idx, 1, NONE, 9, 2.0 ** 100)


# ---------------------------------------------------------------------------------- products that fp32 cannot hold
@pytest.mark.parametrize("S,H,D", [(1, 64, 128), (5, 20, 64), (200, 40, 128), (200, 20, 64)])
@pytest.mark.parametrize("q_size,spread,scale", [(1e34, 1e4, 1.2e-38), (-1e34, 1e4, -1.2e-38), (2e38, 1.0, 1.2e-38), (1e30, 1e4, 1e-33)])
def test_products_beyond_fp32(S, H, D, q_size, spread, scale):
    """Products of query and row beyond 2^128 whose logits are of an ordinary size: both calls take them."""
    print(f"S={S} H={H} D={D} q_size={q_size} spread={spread} scale={scale}", flush=True)
    q, codes, scales, idx = _problem(S, 1, S, H, D, 150, 70, None, NONE, 1, spread=spread)
    q = (q.double().clamp(-1.5, 1.5) * q_size).to(torch.bfloat16)
    assert bool(torch.isfinite(q.float()).all())
    _check(q, codes, scales, None, idx, 1, NONE, 33, scale)


# ---------------------------------------------------------------------------------- rows that receive little
def _weights(q, codes, scales, idx, scale):
    """weights of a call on nothing, with the library's own lse."""
    B, S, H, D = q.shape
    T = codes.shape[1]
    args = (q.to(DEV), _gpu(codes), _gpu(scales), None, _gpu(idx), 1, NONE, 0, scale)
    out, lse = torch.empty((B, S, H, D), device=DEV), torch.empty((B, S, H), device=DEV)
    P.si_quantized_attention(*args, out, lse)
    weights = torch.zeros((B, T), device=DEV)
    nbytes = P.si_accumulate_workspace_bytes(B, S, H, D, T)
    P.si_accumulate_weights(*args, lse, weights, torch.full((max(16, nbytes),), 0xAB, dtype=torch.uint8, device=DEV))
    return weights


@pytest.mark.parametrize("above", [20.0, 25.0, 30.0])
@pytest.mark.parametrize("B,S,H,T", [(1, 1, 64, 480), (1, 2, 64, 480), (1, 64, 64, 480), (1, 150, 64, 480), (2, 200, 20, 480), (1, 130, 64, 5000),
                                     (1, 40, 33, 16000)])
def test_rows_that_receive_little(B, S, H, T, above):
    """A row `above` over the others in every head takes nearly everything; what the others receive keeps the accuracy that ranking them
    needs, whatever the number of queries."""
    print(f"B={B} S={S} H={H} T={T} above={above}", flush=True)
    D, n = 64, 480
    g = torch.Generator().manual_seed(S)
    q = torch.randn((B, S, H, D), generator=g).to(torch.bfloat16)
    q[..., 0] = 1.0
    rows = 0.25 * torch.randn((B, T, D), generator=g)
    rows[..., :32] = 0.0
    rows[:, 7, :32] = 0.0
    rows[:, 7, 0] = above
    codes, scales = R.pack(*R.quantize(rows.to(torch.bfloat16).double().numpy()))
    idx = np.tile(np.arange(n, dtype=np.int32), (B, S, 1))
    weights = _weights(q, codes, scales, idx, 1.0)
    got = weights.double().cpu().numpy()
    _, _, given, _, _, tol = R.attend(q.double().numpy(), R.values(codes, scales), None, idx, 1, NONE, 0, 1.0)
    # The reference's tolerance has half a unit of 2^-32 a query.  A unit is S H / 2^63, its power of two rounded up, and S > 1 queries are
    # each rounded to half of one; the sum once to fp32.
    unit = 2.0 ** (np.ceil(np.log2(S * H)) - 63) if S > 1 else 0.0
    tol = tol[:, :n] - S * 2.0 ** -33 + S * unit / 2 + R.U * given[:, :n]
    off = np.abs(got[:, :n] - given[:, :n])
    assert np.all(off <= tol), float((off / tol).max())
    assert np.all(got[:, n:] == 0)
    assert np.all(off <= 2e-3 * given[:, :n]), float((off / given[:, :n]).max())
    # the rows that stay are those that the exact weights keep, but for rows that its tolerance cannot tell apart from the border
    n_keep = n // 2
    kept = torch.empty((B, n_keep), dtype=torch.int32, device=DEV)
    P.si_evict_rows(weights[:, :n].contiguous(), None, n_keep, 0, 0, [], kept, None,
                    torch.empty(P.si_evict_workspace_bytes(B, n), dtype=torch.uint8, device=DEV))
    for b in range(B):
        border = np.sort(given[b, :n])[n - n_keep]
        sure = np.flatnonzero(given[b, :n] - tol[b] > border + np.delete(tol[b], 7).max())
        assert len(sure) > 0.9 * n_keep
        assert np.isin(sure, kept[b].cpu().numpy()).all()


@pytest.mark.parametrize("S", [1, 7, 200])
def test_no_row_receives_more_than_all(S):
    """lse so large that its rounding is a matter of powers of two: a query gives a row at most 1 a head."""
    q, codes, scales, idx = _problem(8, 1, S, 40, 64, 90, 30, None, NONE, 1, q_size=1e6)
    weights = _weights(q, codes, scales, idx, 50.0).double().cpu().numpy()
    assert np.all(np.isfinite(weights)) and np.all(weights >= 0) and np.all(weights <= S * 40)


# ---------------------------------------------------------------------------------- every kernel that adds weights up
@pytest.mark.parametrize("T", [4096, 4097, 15360, 15361])
@pytest.mark.parametrize("H,D", [(64, 128), (33, 64), (32, 128), (5, 64)])
def test_weights_of_prompts_in_long_caches(T, H, D):
    """Around the lengths at which the sums of many queries are kept elsewhere."""
    print(f"T={T} H={H} D={D}", flush=True)
    q, codes, scales, idx = _problem(T + H, 1, 130, H, D, T, 40, [T - 1], NONE, 1)
    _check(q, codes, scales, [T - 1], idx, 1, NONE, 9, 1.0 / np.sqrt(D))


@pytest.mark.parametrize("B,S,H,D,T", [(70, 16, 20, 64, 100), (9, 127, 40, 128, 60), (64, 16, 33, 128, 4500), (63, 16, 8, 64, 300)])
def test_weights_of_short_prompts_in_batches(B, S, H, D, T):
    """Around the number of queries from which on the sums are kept in LDS."""
    print(f"B={B} S={S} H={H} D={D} T={T}", flush=True)
    q, codes, scales, idx = _problem(S + B, B, S, H, D, T, 24, None, CAUSAL, 1)
    _check(q, codes, scales, None, idx, 1, CAUSAL, 5, 1.0 / np.sqrt(D))


def test_weights_of_many_queries_in_a_long_cache():
    """More queries than waves fit the chip, whose sums go to the workspace at once."""
    B, S, H, D, T = 1, 2500, 4, 64, 15400
    q, codes, scales, idx = _problem(4, B, S, H, D, T, 33, None, NONE, 1)
    _check(q, codes, scales, None, idx, 1, NONE, 7, 0.125)
