"""GPU tests of the paged cache and of packed prompts where their kernels change form or their numbers grow: every number of columns a workgroup takes,
more sequences than a wave has lanes or the chip has workgroups, chunks that outlast the page numbers a wave holds, arrays beyond 4 GB, positions at the
ends of their range, pages that several sequences share."""
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


def _near(got, lse, want, some=None):
    ro, rl, to, tl = want
    got, lse = R.to64(got), R.to64(lse)
    assert np.all(np.abs(got - ro) <= to), (some, np.nanmax(np.abs(got - ro) / np.maximum(to, 1e-300)))
    none = np.isneginf(rl)
    assert np.all(np.isneginf(lse[none])) and np.all(np.abs(lse[~none] - rl[~none]) <= tl[~none]), some


def _paged(q, table, K, V, ks, vs, lengths, first, m, mask, n_win, scale):
    B, S, H, D = q.shape
    out = torch.full(q.shape, 55.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((B, S, H), 55.0, device=DEV)
    ws = torch.empty(P.si_paged_workspace_bytes(B, S, H, K.shape[1], D), dtype=torch.uint8, device=DEV)
    P.si_paged_attention(q.to(DEV), table, K, V, ks, vs, _ints(lengths), _ints(first), m, mask, n_win, scale, out, lse, ws)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("S,H,H_kv", [(1, 16, 1), (1, 17, 1), (1, 32, 1), (1, 33, 1), (1, 64, 1), (1, 65, 1), (3, 43, 1), (2, 48, 3), (16, 8, 8), (130, 1, 1)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("n_win,wide", [(290, None), (R.ALL, None), (R.ALL, 140), (1300, 140)])
def test_columns_of_a_workgroup(S, H, H_kv, D, bits, n_win, wide):
    """Around 16, 32, 64 and 128 columns that share a head; sequences that stay whole, and, where the table has room for long ones, that are dealt out."""
    lengths = [301, 77] if n_win != 1300 else [2001, 1400]
    pages = R.Pages(S + H, lengths, H_kv, D, bits, 16, wide=wide)
    q = torch.randn((2, S, H, D), generator=torch.Generator().manual_seed(D)).to(torch.bfloat16)
    first = [max(0, n - S) for n in lengths]
    print(f"columns S={S} H={H}/{H_kv} D={D} bits={bits} n_win={n_win} wide={wide}", flush=True)
    out, lse = _paged(q, *pages.to(DEV), lengths, first, 1, CAUSAL, n_win, 0.1)
    for b, n in enumerate(lengths):
        _near(out[b], lse[b], R.attend(R.to64(q[b]), pages.k64[b], pages.v64[b], first[b] + np.arange(S), 1, 1, n_win, 0.1), b)


@pytest.mark.parametrize("B,H,H_kv,longest", [(70, 8, 8, 40), (300, 8, 4, 100), (700, 4, 2, 33), (130, 40, 1, 700)])
def test_many_sequences(B, H, H_kv, longest):
    rng = np.random.default_rng(B)
    lengths = [int(x) for x in rng.integers(0, longest + 1, B)]
    lengths[B // 2] = 20 * longest  # one far longer than the others
    pages = R.Pages(B, lengths, H_kv, 64, 16, 16)
    q = torch.randn((B, 1, H, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    print(f"sequences B={B} H={H}/{H_kv}", flush=True)
    out, lse = _paged(q, *pages.to(DEV), lengths, None, 1, NONE, R.ALL, 0.1)
    for b in range(B):
        _near(out[b], lse[b], R.attend(R.to64(q[b]), pages.k64[b], pages.v64[b], [0], 1, 0, R.ALL, 0.1), b)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D", [64, 128])
def test_more_tiles_than_page_numbers_a_wave_holds(bits, D):
    """So many heads that a sequence is one chunk: 70 tiles of each wave.  Pages of 16 rows, one of them not there."""
    H, L = 520, 9001
    wide = -(-L // 16)
    g = torch.Generator(device=DEV).manual_seed(6)
    table = torch.randperm(wide, generator=g, device=DEV).to(torch.int32).view(1, -1).contiguous()
    table[0, 77] = -1
    shape = (wide, H, 16, D)
    if bits == 16:
        K, V = (torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        ks = vs = None
    else:
        K, V = (torch.randint(0, 127, shape, generator=g, device=DEV, dtype=torch.uint8) for _ in range(2))
        K |= torch.randint(0, 2, shape, generator=g, device=DEV, dtype=torch.uint8) << 7
        ks, vs = (torch.randint(120, 123, shape[:3], generator=g, device=DEV, dtype=torch.uint8) for _ in range(2))
    q = torch.randn((1, 1, H, D), generator=g, device=DEV).to(torch.bfloat16)
    print(f"long chunks bits={bits} D={D}", flush=True)
    out, lse = _paged(q, table, K, V, ks, vs, [L], None, 1, NONE, R.ALL, 0.05)
    there = np.ones(L, dtype=bool)
    there[77 * 16:78 * 16] = False
    order = table[0].long().clamp(min=0)
    for h in (0, 1, 259, H - 1):
        rows = []
        for pages, scales in ((K, ks), (V, vs)):
            x = R.to64(pages[order, h].reshape(-1, D)[:L])
            rows.append(x[:, None] if bits == 16 else R.values(x.astype(np.int64), scales[order, h].reshape(-1)[:L].cpu().numpy().astype(np.int64) - 127)[:, None])
        _near(out[0, :, h:h + 1], lse[0, :, h:h + 1], R.attend(R.to64(q[0, :, h:h + 1]), *rows, [0], 1, 0, R.ALL, 0.05, there), h)


@pytest.mark.parametrize("bits", [16, 8])
def test_pages_beyond_4_gb(bits):
    """Rows in, out and attended to at the end of arrays whose offsets pass 32 bits."""
    H, page, D = 8, 1024, 128
    n_pages = 2100 if bits == 16 else 4200
    dtype = torch.bfloat16 if bits == 16 else torch.uint8
    K, V = (torch.zeros((n_pages, H, page, D), dtype=dtype, device=DEV) for _ in range(2))
    scales = [None, None] if bits == 16 else [torch.full((n_pages, H, page), 127, dtype=torch.uint8, device=DEV) for _ in range(2)]
    assert K.nbytes > 2 ** 32
    table = _ints([[n_pages - 1, 0], [n_pages - 2, n_pages - 3]])
    lengths = [1030, 900]
    N = sum(lengths)
    g = torch.Generator().manual_seed(8)
    k, v = ((torch.randn((N, H, D), generator=g) + 0.3 * i).to(torch.bfloat16) for i in range(2))
    offsets = _ints([0, 1030, 1930])
    print(f"beyond 4 GB bits={bits}", flush=True)
    P.si_store_pages(k.to(DEV), v.to(DEV), offsets, None, table, K, V, *scales)
    k_out, v_out = torch.empty((N, H, D), dtype=torch.bfloat16, device=DEV), torch.empty((N, H, D), dtype=torch.bfloat16, device=DEV)
    P.si_load_pages(table, K, V, *scales, offsets, None, k_out, v_out)
    torch.cuda.synchronize()
    k64, v64 = (R.to64(x) if bits == 16 else R.values(*R.quantize(R.to64(x))) for x in (k, v))
    np.testing.assert_array_equal(R.to64(k_out), k64)
    np.testing.assert_array_equal(R.to64(v_out), v64)
    q = torch.randn((2, 1, 2 * H, D), generator=g).to(torch.bfloat16)
    out, lse = _paged(q, table, K, V, *scales, lengths, None, 1, NONE, R.ALL, 0.1)
    for b, rows in enumerate((slice(0, 1030), slice(1030, 1930))):
        _near(out[b], lse[b], R.attend(R.to64(q[b]), k64[rows], v64[rows], [0], 1, 0, R.ALL, 0.1), b)


def test_sequences_that_share_pages():
    """Three requests with the same first 64 rows in the same pages, and rows of their own behind."""
    H, D, page = 2, 128, 16
    pages = R.Pages(3, [64, 37, 5, 20], H, D, 16, page)
    own = pages.table.clone()
    table = torch.full((3, 7), -1, dtype=torch.int32)
    k64, v64, lengths = [], [], []
    for b, n in enumerate((37, 5, 20)):
        table[b, :4] = own[0, :4]
        table[b, 4:4 + -(-n // page)] = own[b + 1, :-(-n // page)]
        k64.append(np.concatenate([pages.k64[0], pages.k64[b + 1]]))
        v64.append(np.concatenate([pages.v64[0], pages.v64[b + 1]]))
        lengths.append(64 + n)
    _, K, V, ks, vs = pages.to(DEV)
    q = torch.randn((3, 1, 4, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    out, lse = _paged(q, table.to(DEV), K, V, ks, vs, lengths, None, 1, NONE, R.ALL, 0.1)
    for b in range(3):
        _near(out[b], lse[b], R.attend(R.to64(q[b]), k64[b], v64[b], [0], 1, 0, R.ALL, 0.1), b)


@pytest.mark.parametrize("first", [-2 ** 31, -3, 0, 2 ** 31 - 1])
@pytest.mark.parametrize("m", [1, 3, 2 ** 31 - 1])
def test_positions_at_the_ends_of_their_range(first, m):
    """Both operators: positions that see nothing, everything, and what their block mask says."""
    S, H, D, T = 5, 4, 64, 50
    pages = R.Pages(1, [T], 2, D, 16, 16)
    q = torch.randn((1, S, H, D), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    t = [first + i for i in range(S)]
    want = R.attend(R.to64(q[0]), pages.k64[0], pages.v64[0], t, m, 1, 40, 0.1)
    out, lse = _paged(q, *pages.to(DEV), [T], [first], m, CAUSAL, 40, 0.1)
    _near(out[0], lse[0], want)
    k, v = (torch.tensor(x).to(torch.bfloat16).to(DEV) for x in (pages.k64[0], pages.v64[0]))
    o, e = torch.empty((S, H, D), dtype=torch.bfloat16, device=DEV), torch.empty((S, H), device=DEV)
    P.si_prompt_attention(q[0].to(DEV), k, v, None, None, _ints([first]), m, CAUSAL, 40, 0.1, o, e)
    torch.cuda.synchronize()
    _near(o, e, want)


def test_lengths_beyond_the_table_and_below_zero():
    pages = R.Pages(1, [64, 64], 2, 64, 16, 16)
    q = torch.randn((2, 1, 4, 64), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    out, lse = _paged(q, *pages.to(DEV), [2 ** 31 - 1, -7], None, 1, NONE, R.ALL, 0.1)
    _near(out[0], lse[0], R.attend(R.to64(q[0]), pages.k64[0], pages.v64[0], [0], 1, 0, R.ALL, 0.1))
    assert bool((out[1] == 0).all()) and bool(torch.isneginf(lse[1]).all())
    full, full_lse = _paged(q, *pages.to(DEV), None, None, 1, NONE, R.ALL, 0.1)
    assert torch.equal(full[0], out[0]) and torch.equal(full_lse[0], lse[0])
    _near(full[1], full_lse[1], R.attend(R.to64(q[1]), pages.k64[1], pages.v64[1], [0], 1, 0, R.ALL, 0.1))


@pytest.mark.parametrize("D", [64, 128])
def test_logits_far_from_zero(D):
    """References that have to rise and fall: rows whose logits grow along the sequence, all far below zero, or far above."""
    T, H = 900, 8
    g = torch.Generator().manual_seed(2)
    k = torch.zeros((T, 1, D))
    k[:, 0, 0] = torch.linspace(-1, 1, T)
    k[:, 0, 1:] = 0.01 * torch.randn((T, D - 1), generator=g)
    k, v = k.to(torch.bfloat16), torch.randn((T, 1, D), generator=g).to(torch.bfloat16)
    q = torch.zeros((1, 1, H, D))
    q[0, 0, :, 0] = torch.tensor([300.0, -300.0, 40.0, -40.0, 0.5, 0.0, 2000.0, -2000.0])
    q[0, 0, :, 1:] = torch.randn((H, D - 1), generator=g)
    q = q.to(torch.bfloat16)
    shifted = k.clone()
    shifted[:, 0, 0] = -3.0  # every logit of the first head about -900, of the second about 900
    for rows in (k, shifted):
        want = R.attend(R.to64(q[0]), R.to64(rows), R.to64(v), [0], 1, 0, R.ALL, 1.0)
        K, V = torch.zeros((2, 57, 1, 16, D), dtype=torch.bfloat16, device=DEV)
        table = _ints([list(range(56, -1, -1))])
        P.si_store_pages(rows.to(DEV), v.to(DEV), None, None, table, K, V)
        out, lse = _paged(q, table, K, V, None, None, [T], None, 1, NONE, R.ALL, 1.0)
        _near(out[0], lse[0], want)
        o, e = torch.empty((1, H, D), dtype=torch.bfloat16, device=DEV), torch.empty((1, H), device=DEV)
        P.si_prompt_attention(q[0].to(DEV), rows.to(DEV), v.to(DEV), None, None, None, 1, NONE, R.ALL, 1.0, o, e)
        torch.cuda.synchronize()
        _near(o, e, want)


# ---------------------------------------------------------------------------------- packed prompts
def _prompt(q, k, v, qo, ko, first, m, mask, n_win, scale):
    out, lse = torch.full(q.shape, 55.0, dtype=torch.bfloat16, device=DEV), torch.full(q.shape[:2], 55.0, device=DEV)
    P.si_prompt_attention(q.to(DEV), k.to(DEV), None if v is None else v.to(DEV), _ints(qo), _ints(ko), _ints(first), m, mask, n_win, scale, out, lse)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("H,H_kv,D,lengths,before,m,n_win", [
    (32, 4, 128, [2600, 1500, 317], [0, 700, 2000], 1, R.ALL),  # 256 columns a workgroup
    (32, 4, 128, [2600, 1500], [0, 700], 1, 2100),
    (64, 1, 128, [8300, 900], [5, 7400], 4, R.ALL),
    (64, 2, 128, [2500, 31, 1], [0, 2100, 2777], 1, 2049),
    (33, 3, 128, [3100, 2], [0, 3000], 1, R.ALL),
    (32, 4, 128, [2100, 0, 317], [0, 0, 200], 1, R.ALL),     # as many columns in all, but of few rows or in a window: 128 columns, tiles of 32 rows
    (32, 4, 128, [2100, 317], [0, 200], 1, 300),
    (33, 3, 128, [2500, 31, 1], [0, 0, 777], 1, R.ALL),
    (16, 2, 128, [1100, 700], [0, 60], 1, 129),              # few: 128 columns, tiles of 64 rows
    (16, 2, 128, [300, 130], [900, 0], 1, R.ALL),            # 128 columns, tiles of 64 rows
    (32, 4, 64, [1500, 200], [0, 99], 1, 64),
    (33, 3, 64, [1500, 0, 65, 1], [0, 0, 700, 3], 1, R.ALL),
])
def test_forms_of_the_prompt(H, H_kv, D, lengths, before, m, n_win):
    g = torch.Generator().manual_seed(H + D)
    qo = [0] + [int(x) for x in np.cumsum(lengths)]
    ko = [0] + [int(x) for x in np.cumsum([(n + p) // m for n, p in zip(lengths, before)])]
    q = torch.randn((qo[-1], H, D), generator=g).to(torch.bfloat16)
    k = (torch.randn((ko[-1], H_kv, D), generator=g) * torch.exp(torch.randn((ko[-1], H_kv, 1), generator=g))).to(torch.bfloat16)
    v = (torch.randn((ko[-1], H_kv, D), generator=g) + 0.3).to(torch.bfloat16)
    print(f"forms H={H}/{H_kv} D={D} {lengths} {before} m={m} n_win={n_win}", flush=True)
    out, lse = _prompt(q, k, v, qo, ko, before, m, CAUSAL, n_win, 0.1)
    for b, n in enumerate(lengths):
        if n == 0:
            continue
        some = np.unique(np.clip([0, 1, 2, 3, 31, 32, 33, 63, 64, 65, 255, 256, 500, n // 2, n - 33, n - 2, n - 1], 0, n - 1))
        rows = slice(ko[b], ko[b + 1])
        _near(out[qo[b] + some], lse[qo[b] + some],
              R.attend(R.to64(q[qo[b] + some]), R.to64(k[rows]), R.to64(v[rows]), before[b] + some, m, 1, n_win, 0.1), b)
    again = _prompt(q, k, v, qo, ko, before, m, CAUSAL, n_win, 0.1)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("n,H,H_kv,n_win,D", [(2600, 32, 4, 2050, 128), (2200, 32, 4, 100, 128), (1100, 16, 2, 100, 128), (300, 16, 2, 100, 128), (1100, 16, 2, 100, 64),
                                             (2600, 33, 3, 2050, 64)])
def test_rows_that_are_not_seen_in_every_form(n, H, H_kv, n_win, D):
    g = torch.Generator().manual_seed(n)
    q = torch.randn((n, H, D), generator=g).to(torch.bfloat16)
    k, v = (torch.randn((n, H_kv, D), generator=g).to(torch.bfloat16) for _ in range(2))
    clean = _prompt(q, k, v, None, None, None, 1, CAUSAL, n_win, 0.1)
    at = [0, 31, n - 140, n - 1] if n_win > 100 else [0, 31, 70, n - 140, n - 1]
    for s in at:
        v[s] = float("nan")
    out, lse = _prompt(q, k, v, None, None, None, 1, CAUSAL, n_win, 0.1)
    t = np.arange(n)
    seen = np.any([(t >= s) & (t < s + n_win) for s in at], axis=0)
    fine = torch.from_numpy(~seen).to(DEV)
    assert bool(fine.any()) and torch.equal(out[fine], clean[0][fine]) and torch.equal(lse, clean[1])
    assert bool(torch.isnan(out[~fine]).all())


def test_many_short_prompts():
    """More sequences than a search looks at in one step, many of them empty."""
    rng = np.random.default_rng(5)
    B, H, D = 5000, 4, 64
    lengths = rng.integers(0, 4, B) * rng.integers(0, 2, B)
    qo = np.concatenate([[0], np.cumsum(lengths)])
    N = int(qo[-1])
    g = torch.Generator().manual_seed(5)
    q = torch.randn((N, H, D), generator=g).to(torch.bfloat16)
    k, v = (torch.randn((N, 1, D), generator=g).to(torch.bfloat16) for _ in range(2))
    out, lse = _prompt(q, k, v, qo.tolist(), qo.tolist(), None, 1, CAUSAL, R.ALL, 0.1)
    for b in list(range(0, B, 97)) + [B - 1]:
        rows = slice(qo[b], qo[b + 1])
        if lengths[b]:
            _near(out[rows], lse[rows], R.attend(R.to64(q[rows]), R.to64(k[rows]), R.to64(v[rows]), list(range(lengths[b])), 1, 1, R.ALL, 0.1), b)
    # ... and the same rows into and out of pages
    K, V = torch.zeros((2, B, 1, 16, D), dtype=torch.bfloat16, device=DEV)
    table = torch.randperm(B, generator=g).to(torch.int32).view(B, 1).to(DEV)
    start, off = _ints(rng.integers(0, 13, B).tolist()), _ints(qo.tolist())
    P.si_store_pages(k.to(DEV), v.to(DEV), off, start, table, K, V)
    k_out, v_out = torch.empty_like(k, device=DEV), torch.empty_like(v, device=DEV)
    P.si_load_pages(table, K, V, None, None, off, start, k_out, v_out)
    torch.cuda.synchronize()
    assert torch.equal(k_out.cpu(), k) and torch.equal(v_out.cpu(), v)


def test_prompt_rows_beyond_4_gb():
    H_kv, D, far = 8, 128, 2 ** 21 + 1000
    k, v = (torch.zeros((far + 200, H_kv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    assert k.nbytes > 2 ** 32
    g = torch.Generator().manual_seed(4)
    rows = [torch.randn((200, H_kv, D), generator=g).to(torch.bfloat16) for _ in range(2)]
    k[far:], v[far:] = rows[0].to(DEV), rows[1].to(DEV)
    q = torch.randn((100, 16, D), generator=g).to(torch.bfloat16)
    out, lse = torch.empty((100, 16, D), dtype=torch.bfloat16, device=DEV), torch.empty((100, 16), device=DEV)
    P.si_prompt_attention(q.to(DEV), k, v, _ints([0, 0, 100]), _ints([0, far, far + 200]), _ints([0, 100]), 1, CAUSAL, R.ALL, 0.1, out, lse)
    torch.cuda.synchronize()
    _near(out, lse, R.attend(R.to64(q), R.to64(rows[0]), R.to64(rows[1]), 100 + np.arange(100), 1, 1, R.ALL, 0.1))


@pytest.mark.parametrize("n_below", [40, 200, 600])
@pytest.mark.parametrize("D,H,H_kv", [(64, 8, 1), (128, 16, 2), (128, 64, 1)])
def test_rows_whose_scores_are_minus_infinity(n_below, D, H, H_kv):
    """An infinite key takes a row's weight: the rows before the first finite one count for nothing, and for that head only."""
    T, S = 600, 300
    g = torch.Generator().manual_seed(n_below)
    k, v = (torch.randn((T, H_kv, D), generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((S, H, D), generator=g).to(torch.bfloat16)
    q[..., 3] = q[..., 3].abs() + 0.5
    finite = k.clone()
    k[:n_below, 0, 3] = float("-inf")
    G = H // H_kv
    out, lse = _prompt(q, k, v, None, None, None, 1, NONE, R.ALL, 0.1)
    pages_k, pages_v = torch.zeros((2, 40, H_kv, 16, D), dtype=torch.bfloat16, device=DEV)
    table = _ints([list(range(40))])
    P.si_store_pages(k.to(DEV), v.to(DEV), None, None, table, pages_k, pages_v)
    got, got_lse = _paged(q[:2].reshape(1, 2, H, D).contiguous(), table, pages_k, pages_v, None, None, [T], None, 1, NONE, R.ALL, 0.1)
    if n_below == T:
        for o, e in ((out, lse), (got[0], got_lse[0])):
            assert bool((o[:, :G] == 0).all()) and bool(torch.isneginf(e[:, :G]).all())
    else:
        want = R.attend(R.to64(q[:, :G]), R.to64(finite[n_below:, :1]), R.to64(v[n_below:, :1]), range(S), 1, 0, R.ALL, 0.1)
        _near(out[:, :G], lse[:, :G], want)
        _near(got[0, :, :G], got_lse[0, :, :G], [x[:2] for x in want])
    if H_kv > 1:
        want = R.attend(R.to64(q[:, G:]), R.to64(finite[:, 1:]), R.to64(v[:, 1:]), range(S), 1, 0, R.ALL, 0.1)
        _near(out[:, G:], lse[:, G:], want)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D,H", [(128, 16), (64, 33)])
@pytest.mark.parametrize("both", [True, False])
def test_rows_of_large_calls(bits, D, H, both):
    """64 MB of packed rows and more, of sequences with odd lengths, in and out."""
    lengths = [4099, 1, 0, 3000, 1200] if both else [9001, 1, 0, 7000, 1200]
    N, page = sum(lengths), 32
    assert N * H * D * (4 if both else 2) >= 64 << 20
    g = torch.Generator(device=DEV).manual_seed(9)
    k, v = (torch.randn((N, H, D), generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    wide = -(-(max(lengths) + 20) // page)
    n_pages = 5 * wide
    table = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32).view(5, wide)
    shape = (n_pages, H, page, D)
    K, V = (torch.full(shape, 7, dtype=torch.bfloat16 if bits == 16 else torch.uint8, device=DEV) for _ in range(2))
    scales = [None, None] if bits == 16 else [torch.full(shape[:3], 99, dtype=torch.uint8, device=DEV) for _ in range(2)]
    off, start = _ints([0] + [int(x) for x in np.cumsum(lengths)]), _ints([0, 13, 5, 19, 3])
    if not both:
        V, v, scales = None, None, [scales[0], None]
    print(f"large rows bits={bits} D={D} both={both}", flush=True)
    P.si_store_pages(k, v, off, start, table, K, V, *scales)
    k_out, v_out = torch.full_like(k, -3), None if v is None else torch.full_like(v, -3)
    P.si_load_pages(table, K, V, *scales, off, start, k_out, v_out)
    torch.cuda.synchronize()
    for x, got in ((k, k_out), (v, v_out)):
        if x is None:
            continue
        if bits == 16:
            assert torch.equal(got, x)
        else:
            for some in (slice(0, 300), slice(4000, 4300), slice(N - 300, N)):
                np.testing.assert_array_equal(R.to64(got[some]), R.values(*R.quantize(R.to64(x[some]))))
    # what no row went to is as it was
    used = torch.zeros((n_pages * page,), dtype=torch.bool, device=DEV)
    for b, n in enumerate(lengths):
        s = int(start[b]) + torch.arange(n, device=DEV)
        used[table[b, s // page].long() * page + s % page] = True
    left = K.permute(0, 2, 1, 3).reshape(n_pages * page, -1)[~used]
    assert bool((left == 7).all())


@pytest.mark.parametrize("B,S,H,H_kv,D,bits,longest", [(65, 1, 8, 8, 64, 16, 600), (1100, 1, 4, 1, 64, 8, 400), (1100, 2, 16, 8, 128, 16, 300), (5000, 1, 8, 2, 64, 16, 90),
                                                       (16384, 1, 2, 1, 64, 16, 40)])
def test_more_sequences_than_lanes(B, S, H, H_kv, D, bits, longest):
    """Mostly short ones, some empty, and three that are far longer than an even share; twice into the same workspace."""
    rng = np.random.default_rng(B + S)
    lengths = rng.integers(0, longest + 1, B)
    lengths[rng.integers(0, B, B // 7)] = 0
    far = [1, B // 2, B - 1]
    lengths[far] = [40 * longest, 33, 9 * longest + 1]
    page = 64
    wide = -(-int(lengths.max()) // page)
    first_page = np.concatenate([[0], np.cumsum(-(-lengths // page))])
    table = np.full((B, wide), -1, dtype=np.int32)
    for b in range(B):
        n = first_page[b + 1] - first_page[b]
        table[b, :n] = first_page[b] + np.arange(n)
    g = torch.Generator(device=DEV).manual_seed(B)
    shape = (int(first_page[-1]), H_kv, page, D)
    if bits == 16:
        K, V = (torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        ks = vs = None
    else:
        K, V = (torch.randint(0, 127, shape, generator=g, device=DEV, dtype=torch.uint8) for _ in range(2))
        ks, vs = (torch.randint(118, 121, shape[:3], generator=g, device=DEV, dtype=torch.uint8) for _ in range(2))
    q = torch.randn((B, S, H, D), generator=g, device=DEV).to(torch.bfloat16)
    first = [int(n) - S for n in lengths]
    print(f"sequences B={B} S={S} H={H}/{H_kv} D={D} bits={bits}", flush=True)
    out, lse = _paged(q, torch.from_numpy(table).to(DEV), K, V, ks, vs, lengths.tolist(), first, 1, CAUSAL, R.ALL, 0.05)
    again = _paged(q, torch.from_numpy(table).to(DEV), K, V, ks, vs, lengths.tolist(), first, 1, CAUSAL, R.ALL, 0.05)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    for b in far + sorted(rng.integers(0, B, 40).tolist()):
        n = int(lengths[b])
        rows = []
        for pages, scales in ((K, ks), (V, vs)):
            x = pages[int(first_page[b]):int(first_page[b + 1])].permute(0, 2, 1, 3).reshape(-1, H_kv, D)[:n]
            if bits == 8:
                e = scales[int(first_page[b]):int(first_page[b + 1])].permute(0, 2, 1).reshape(-1, H_kv)[:n].cpu().numpy().astype(np.int64) - 127
                rows.append(R.values(x.cpu().numpy().astype(np.int64), e))
            else:
                rows.append(R.to64(x))
        _near(out[b], lse[b], R.attend(R.to64(q[b]), *rows, range(first[b], first[b] + S), 1, 1, R.ALL, 0.05), b)
