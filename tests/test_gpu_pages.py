"""GPU tests of the paged cache: rows into and out of pages bit for bit, and attention over pages against 64-bit references."""
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
    return _ints([0] + list(np.cumsum(lengths)))


def _bits(t):
    return t.view(torch.int16 if t.dtype is torch.bfloat16 else torch.int32)


# ---------------------------------------------------------------------------------- rows in and out
@pytest.mark.parametrize("D,H,page", [(128, 8, 64), (64, 5, 16), (128, 1, 1024), (64, 33, 32)])
@pytest.mark.parametrize("bits", [16, 8])
def test_rows_in_and_out(D, H, page, bits):
    g = torch.Generator().manual_seed(D + H)
    lengths, start = [1, 70, 0, 17, 33], [5, 0, 9, 63, 16]
    N = sum(lengths) + 6  # six rows behind the last sequence
    rows = [(torch.randn((N, H, D), generator=g) * torch.exp(2 * torch.randn((N, H, 1), generator=g))).to(torch.bfloat16) for _ in range(2)]
    held = [s + n for s, n in zip(start, lengths)]
    pages = R.Pages(7, held, H, D, bits, page, filler=3.0, spare=4)
    table, K, V, ks, vs = pages.to(DEV)
    before = [None if t is None else t.clone() for t in (K, V, ks, vs)]
    off, st = _offsets(lengths), _ints(start)
    print(f"store D={D} H={H} page={page} bits={bits}", flush=True)
    P.si_store_pages(rows[0].to(DEV), rows[1].to(DEV), off, st, table, K, V, ks, vs)
    torch.cuda.synchronize()
    k_out = torch.full((N, H, D), 77.0, dtype=torch.bfloat16, device=DEV)
    v_out = k_out.clone()
    P.si_load_pages(table, K, V, ks, vs, off, st, k_out, v_out)
    torch.cuda.synchronize()
    n = sum(lengths)
    for out, x in ((k_out, rows[0]), (v_out, rows[1])):
        want = R.to64(x[:n]) if bits == 16 else R.values(*R.quantize(R.to64(x[:n])))
        np.testing.assert_array_equal(R.to64(out[:n]), want)
        assert bool((out[n:] == 77.0).all())
    # what no row went to is as it was
    written = torch.zeros((pages.n_pages, page), dtype=torch.bool)
    for b in range(len(lengths)):
        for s in range(start[b], held[b]):
            written[int(pages.table[b, s // page]), s % page] = True
    for now, was in zip((K, V, ks, vs), before):
        if now is not None:
            keep = (~written)[:, None, :].expand(-1, H, -1).to(DEV)
            assert torch.equal(now[keep].view(torch.uint8), was[keep].view(torch.uint8))


def test_rows_without_a_page_are_dropped_and_come_back_as_zeros():
    H, D, page = 2, 64, 16
    for bits in (16, 8):
        dtype = torch.bfloat16 if bits == 16 else torch.uint8
        K = torch.ones((3, H, page, D), dtype=dtype, device=DEV)
        V = K.clone()
        scales = [None, None] if bits == 16 else [torch.full((3, H, page), 127, dtype=torch.uint8, device=DEV) for _ in range(2)]
        table = _ints([[2, -1, 3, 0], [1, 2 ** 31 - 1, -2 ** 31, 7]])
        x = torch.full((2 * 70, H, D), 2.5, dtype=torch.bfloat16, device=DEV)
        P.si_store_pages(x, x, None, _ints([0, 0]), table, K, V, *scales)  # 70 rows each: the table has room for 64
        k, v = torch.full_like(x, 9.0), torch.full_like(x, 9.0)
        P.si_load_pages(table, K, V, *scales, None, None, k, v)
        torch.cuda.synchronize()
        want = torch.zeros((2, 70, H, D))
        want[0, :16] = want[0, 48:64] = want[1, :16] = 2.5
        assert torch.equal(k.cpu().float().view(2, 70, H, D), want) and torch.equal(v, k)
        # a start before the table or far behind it
        P.si_store_pages(x * 2, x * 2, None, _ints([-8, 2 ** 31 - 1]), table, K, V, *scales)
        torch.cuda.synchronize()
        P.si_load_pages(table, K, V, *scales, None, None, k, None)
        want[0, :16] = 5.0
        want[0, 48:62] = 5.0  # rows 0 .. 61 were stored, those of pages that there are
        assert torch.equal(k.cpu().float().view(2, 70, H, D), want)


def test_eight_bits_hold_every_kind_of_value():
    """Levels, ties, zeros of either sign, the smallest and the largest values, infinities and NaN."""
    D = 64
    rng = np.random.default_rng(3)
    rows = [np.resize(R.LEVELS[:127], D) * 2.0 ** e for e in (-64, -3, 0, 40, 63)]
    rows += [np.resize((R.LEVELS[:126] + R.LEVELS[1:127]) / 2, D), np.resize((R.LEVELS[62:126] + R.LEVELS[63:127]) / 2, D)]
    rows += [np.zeros(D), -np.zeros(D), np.full(D, 2.0 ** -120), np.full(D, 3.3e38), np.full(D, np.inf), np.full(D, np.nan)]
    for lead in (447.0, 448.0, 449.0, 464.0, 480.0, 1e30, np.inf, np.nan):
        row = rng.standard_normal(D)
        row[5] = lead
        rows.append(row)
        rows.append(-row)
    x = torch.tensor(np.array(rows), dtype=torch.float64).to(torch.bfloat16)[:, None, :].contiguous()
    n = len(rows)
    K = torch.zeros((4, 1, 16, D), dtype=torch.uint8, device=DEV)
    ks = torch.zeros((4, 1, 16), dtype=torch.uint8, device=DEV)
    table = _ints([[3, 1, 0, 2]])
    P.si_store_pages(x.to(DEV), None, None, None, table, K, None, ks, None)
    out = torch.empty_like(x, device=DEV)
    P.si_load_pages(table, K, None, ks, None, None, None, out, None)
    torch.cuda.synchronize()
    codes, e = R.quantize(R.to64(x))
    order = [3, 1, 0, 2]
    got = K.cpu().numpy()[order, 0].reshape(-1, D)[:n]
    nan = codes[:, 0] % 128 == 127
    np.testing.assert_array_equal(np.where(nan, 127, got % 128 + 0 * got), np.where(nan, 127, codes[:, 0] % 128))
    assert np.all(got[nan] % 128 == 127)
    np.testing.assert_array_equal((got >= 128)[~nan], (codes[:, 0] >= 128)[~nan])
    np.testing.assert_array_equal(ks.cpu().numpy()[order, 0].reshape(-1)[:n], e[:, 0] + 127)
    np.testing.assert_array_equal(R.to64(out)[:, 0], R.values(codes, e)[:, 0])


# ---------------------------------------------------------------------------------- attention
def _attend(pages, q, lengths, first, m, mask, n_win, scale, workspace=None):
    B, S, H, D = q.shape
    table, K, V, ks, vs = pages.to(DEV)
    out = torch.full(q.shape, 55.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((B, S, H), 55.0, dtype=torch.float32, device=DEV)
    ws = torch.empty(P.si_paged_workspace_bytes(B, S, H, K.shape[1], D), dtype=torch.uint8, device=DEV) if workspace is None else workspace
    P.si_paged_attention(q.to(DEV), table, K, V, ks, vs, _ints(lengths), _ints(first), m, mask, n_win, scale, out, lse, ws)
    torch.cuda.synchronize()
    return out, lse


def _check(pages, q, out, lse, lengths, first, m, mask, n_win, scale, there=None):
    B, S = q.shape[:2]
    for b in range(B):
        position = [(0 if first is None else first[b]) + i for i in range(S)]
        ro, rl, to, tl = R.attend(R.to64(q[b]), pages.k64[b][:lengths[b]], pages.v64[b][:lengths[b]], position, m, mask, n_win, scale,
                                  None if there is None else there[b][:lengths[b]])
        got, got_lse = R.to64(out[b]), R.to64(lse[b])
        assert np.all(np.abs(got - ro) <= to), (b, np.nanmax(np.abs(got - ro) / np.maximum(to, 1e-300)))
        none = np.isneginf(rl)
        assert np.all(np.isneginf(got_lse[none]))
        assert np.all(np.abs(got_lse[~none] - rl[~none]) <= tl[~none]), b


CASES = [
    # B, S, lengths, H, H_kv, D, page, mask, m, n_win
    (1, 1, [1], 8, 8, 128, 16, NONE, 1, R.ALL),
    (1, 1, [2048], 64, 8, 128, 64, NONE, 1, R.ALL),
    (5, 1, [31, 32, 33, 0, 500], 64, 8, 128, 16, NONE, 1, R.ALL),
    (3, 1, [257, 1000, 64], 64, 1, 128, 64, NONE, 1, R.ALL),
    (2, 1, [700, 129], 33, 1, 64, 32, NONE, 1, R.ALL),
    (2, 4, [77, 1203], 40, 8, 64, 16, CAUSAL, 1, R.ALL),
    (3, 7, [7, 300, 8], 33, 3, 128, 16, CAUSAL, 1, R.ALL),
    (2, 3, [40, 290], 5, 5, 64, 64, CAUSAL, 4, R.ALL),
    (2, 1, [4000, 2500], 8, 2, 128, 256, NONE, 1, 128),
    (2, 5, [900, 333], 16, 4, 64, 16, CAUSAL, 1, 100),
    (1, 2, [600], 4, 4, 128, 1024, NONE, 1, 0),
    (2, 1, [5000, 3], 24, 8, 64, 128, NONE, 1, R.ALL),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("room", [0, 2500])  # of the table: long sequences are dealt out over the chip
def test_attention(case, bits, shared, room):
    B, S, lengths, H, H_kv, D, page, mask, m, n_win = case
    pages = R.Pages(11, lengths, H_kv, D, bits, page, shared=shared, wide=max(-(-max(lengths) // page), -(-room // page)))  # NaN wherever no sequence has rows
    g = torch.Generator().manual_seed(5)
    q = torch.randn((B, S, H, D), generator=g).to(torch.bfloat16)
    first = [max(0, n - S) for n in lengths] if mask == CAUSAL else None
    if mask == CAUSAL and m > 1:
        first = [m * n // 2 - 2 for n in lengths]
    print(f"attention {case} bits={bits} shared={shared}", flush=True)
    out, lse = _attend(pages, q, lengths, first, m, mask, n_win, 1.0 / np.sqrt(D))
    _check(pages, q, out, lse, lengths, first, m, mask, n_win, 1.0 / np.sqrt(D))


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales(scale):
    lengths = [200, 37]
    pages = R.Pages(2, lengths, 2, 64, 16, 16)
    q = torch.randn((2, 1, 6, 64), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16)
    out, lse = _attend(pages, q, lengths, None, 1, NONE, R.ALL, scale)
    _check(pages, q, out, lse, lengths, None, 1, NONE, R.ALL, scale)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("D,bits", [(64, 16), (128, 16), (128, 8)])
def test_rows_that_are_not_seen_may_hold_anything(bad, D, bits):
    """Later positions' rows and rows before the window; what lies behind a length is NaN in all tests above."""
    S, lengths, n_win = 40, [100], 30
    pages = R.Pages(9, lengths, 2, D, bits, 16)
    q = torch.randn((1, S, 4, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    clean = _attend(pages, q, lengths, [50], 1, CAUSAL, n_win, 0.1)
    at = lambda s: (int(pages.table[0, s // 16]), slice(None), s % 16)  # noqa: E731
    if bits == 16:
        pages.K[at(60)], pages.V[at(70)], pages.K[at(95)] = bad, bad, bad
    else:  # a code that is NaN
        pages.K[at(60)], pages.V[at(70)], pages.K[at(95)] = 127, 255, 127
        bad = float("nan")
    out, lse = _attend(pages, q, lengths, [50], 1, CAUSAL, n_win, 0.1)
    t = 50 + np.arange(S)
    k_seen, v_seen = (t >= 60) & (t < 60 + n_win), (t >= 70) & (t < 70 + n_win)
    fine = torch.from_numpy(~(k_seen | v_seen)).to(DEV)
    assert int(fine.sum()) == 10
    assert torch.equal(out[0, fine], clean[0][0, fine]) and torch.equal(lse[0, fine], clean[1][0, fine])
    only = torch.from_numpy(v_seen & ~k_seen).to(DEV)
    assert torch.equal(lse[0, only], clean[1][0, only]) and not bool(torch.isfinite(out[0, only]).any())
    if bad != bad:
        assert bool(torch.isnan(lse[0, torch.from_numpy(k_seen).to(DEV)]).all())


def test_pages_that_are_not_there():
    """Pages taken out of the table: nobody sees their rows, wherever they lie in a tile or a window."""
    lengths = [600, 50, 40]
    pages = R.Pages(4, lengths, 2, 64, 16, 16)
    there = [np.ones(n, dtype=bool) for n in lengths]
    for b, page, number in ((0, 0, -1), (0, 7, pages.n_pages), (0, 8, 2 ** 31 - 1), (0, 20, -5), (0, 37, -1), (1, 1, -1), (2, 0, -1), (2, 1, -1), (2, 2, -1)):
        pages.table[b, page] = number
        there[b][page * 16:(page + 1) * 16] = False
    q = torch.randn((3, 2, 4, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    for n_win in (R.ALL, 13, 120):
        first = [n - 2 for n in lengths]
        out, lse = _attend(pages, q, lengths, first, 1, CAUSAL, n_win, 0.1)
        _check(pages, q, out, lse, lengths, first, 1, CAUSAL, n_win, 0.1, there)
    assert bool((out[2] == 0).all()) and bool(torch.isneginf(lse[2]).all())
