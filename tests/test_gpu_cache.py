"""GPU parity of the operators of a cache held in 4 bits against the plain 64-bit reference (tests/cache_reference.py): rows in and
out, attention, accumulated weights, eviction, and a serving loop of all of them."""
import numpy as np
import pytest
import torch

import paper_2605_02568_amd as P
import workloads as W
from tests import cache_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gpu(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _bf16(a):
    """Tensor of bf16 bit patterns (uint16)."""
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16)


# ---------------------------------------------------------------------------------- rows in and out
def _all_patterns(D):
    """Every bf16 bit pattern, in blocks of one exponent and sign with others strewn in."""
    rng = np.random.default_rng(D)
    bits = np.arange(65536, dtype=np.uint16)
    mixed = rng.permutation(bits)
    near = (np.uint16(0x3F00) + rng.integers(0, 0x300, 65536).astype(np.uint16)) | (rng.integers(0, 2, 65536).astype(np.uint16) << 15)
    return np.concatenate([bits, mixed, near]).reshape(1, -1, D)


@pytest.mark.parametrize("D", [32, 64, 128])
def test_quantize_every_bf16_pattern(D):
    bits = _all_patterns(D)
    N = bits.shape[1]
    codes = torch.full((1, N, D // 2), 0xAA, dtype=torch.uint8, device=DEV)
    scales = torch.full((1, N, D // 32), 0xAA, dtype=torch.uint8, device=DEV)
    P.si_quantize_rows(_bf16(bits).to(DEV), None, codes, scales)
    torch.cuda.synchronize()
    x = R.bf16_values(bits)
    want, e = R.quantize(x)
    got = codes.cpu().numpy()
    got = np.stack([got & 15, got >> 4], axis=-1).reshape(x.shape)
    assert np.array_equal(scales.cpu().numpy().astype(np.int64) - 127, e)
    nan = np.isnan(x)
    assert np.array_equal(got[~nan], want[~nan])
    assert np.all((got[nan] & 7) == 7)
    # no finite value within the range is off by more than half a step
    v = R.values(codes.cpu().numpy(), scales.cpu().numpy())
    fine = ~nan & (np.abs(x) <= 7 * 2.0 ** 13)
    power = np.repeat(np.exp2(e), 32, axis=-1)
    assert np.all(np.abs(v - x)[fine] <= power[fine])
    small = fine & (np.abs(x) <= 2 * power)
    assert np.all(np.abs(v - x)[small] <= 0.25 * power[small])


@pytest.mark.parametrize("B,N,D,T,start", [
    (1, 1, 32, 1, None), (3, 1, 128, 7, [0, 6, 3]), (2, 5, 64, 9, [4, 0]), (5, 37, 128, 100, [0, 80, -5, 100, 63]),
    (2, 300, 32, 400, [-300, 399]), (2, 4, 64, 6, [2 ** 31 - 1, -2 ** 31]), (1, 1000, 128, 1000, None), (2, 10, 128, 4, None),
])
def test_rows_at_places(B, N, D, T, start):
    """Rows land at start[b] + n, those outside nowhere; reading back gives them and zeros outside; other rows stay."""
    print(f"rows B={B} N={N} D={D} T={T} start={start}", flush=True)
    g = torch.Generator().manual_seed(N * D)
    rows = (torch.randn((B, N, D), generator=g) * 3).to(torch.bfloat16)
    codes, scales = R.pack(*R.quantize(R.bf16_values(W.bf16_bits(rows))))
    want_c = np.full((B, T, D // 2), 0x5A, dtype=np.uint8)
    want_s = np.full((B, T, D // 32), 0x7B, dtype=np.uint8)
    back = np.zeros((B, N, D))
    for b in range(B):
        for n in range(N):
            at = n + (0 if start is None else start[b])
            if 0 <= at < T:
                want_c[b, at], want_s[b, at] = codes[b, n], scales[b, n]
                back[b, n] = R.values(codes[b, n], scales[b, n])
    c, s = torch.full((B, T, D // 2), 0x5A, dtype=torch.uint8, device=DEV), torch.full((B, T, D // 32), 0x7B, dtype=torch.uint8, device=DEV)
    at = None if start is None else torch.tensor(start, dtype=torch.int32, device=DEV)
    P.si_quantize_rows(rows.to(DEV), at, c, s)
    out = torch.full((B, N, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    P.si_dequantize_rows(c, s, at, out)
    torch.cuda.synchronize()
    # rows the call did not write keep 0x5A / 0x7B; written ones are equal up to the sign of a zero, which the codes carry
    assert np.array_equal(c.cpu().numpy(), want_c) and np.array_equal(s.cpu().numpy(), want_s)
    assert np.array_equal(out.double().cpu().numpy(), back)


@pytest.mark.parametrize("D", [32, 64, 128])
def test_dequantize_every_code_and_scale(D):
    rng = np.random.default_rng(1)
    codes = np.concatenate([np.arange(256, dtype=np.uint8), rng.integers(0, 256, 27 * D * 16 - 256, dtype=np.uint8)]).reshape(1, -1, D // 2)
    T = codes.shape[1]
    scales = np.resize(np.arange(114, 141, dtype=np.uint8), (1, T, D // 32))
    out = torch.full((1, T, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    P.si_dequantize_rows(_gpu(codes), _gpu(scales), None, out)
    torch.cuda.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), R.values(codes, scales))


def test_rows_beyond_4_gib():
    """Offsets beyond 32 bits, in a cache and in the rows of a call."""
    D, T = 128, 1 << 25  # 2 GiB of codes a batch, 4 GiB in all
    codes = torch.empty((3, T, D // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((3, T, D // 32), dtype=torch.uint8, device=DEV)
    g = torch.Generator().manual_seed(2)
    rows = torch.randn((3, 40, D), generator=g).to(torch.bfloat16)
    start = torch.tensor([5, T - 40, T - 39], dtype=torch.int32, device=DEV)
    P.si_quantize_rows(rows.to(DEV), start, codes, scales)
    out = torch.empty_like(rows, device=DEV)
    P.si_dequantize_rows(codes, scales, start, out)
    c, s = R.pack(*R.quantize(R.bf16_values(W.bf16_bits(rows))))
    want = R.values(c, s)
    want[2, 39] = 0  # fell outside
    assert np.array_equal(out.double().cpu().numpy(), want)
    big = torch.full((1, (1 << 24) + 77, D), 3.0, dtype=torch.bfloat16, device=DEV)  # rows of more than 4 GiB
    P.si_quantize_rows(big, None, codes[:1], scales[:1])
    n = big.shape[1]
    assert bool((codes[0, :n] == 0x77).all()) and bool((scales[0, :n] == 126).all())
    big.zero_()
    P.si_dequantize_rows(codes[:1], scales[:1], None, big)
    assert bool((big == 3.0).all())


# ---------------------------------------------------------------------------------- attention and weights
def _problem(seed, B, S, H, D, T, k, lengths, mask, m, spread=1.0, q_size=1.0):
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn((B, S, H, D), generator=g) * q_size).to(torch.bfloat16)
    rows = torch.randn((B, T, D), generator=g) * torch.exp(np.log(spread) * torch.rand((B, T, D // 32), generator=g)).repeat_interleave(32, dim=2)
    codes, scales = R.pack(*R.quantize(rows.to(torch.bfloat16).double().numpy()))
    idx = None
    if k:
        idx = np.full((B, S, k), -1, dtype=np.int32)
        for b in range(B):
            n_held = R.held(lengths, b, T)
            for t in range(S):
                L = n_held if mask == 0 else min(n_held, (t + 1) // m)
                n = [0, min(k, L), min(k, L) // 2, min(1, L)][int(rng.integers(0, 4))] if t else min(k, L)
                idx[b, t, rng.permutation(k)[:n]] = rng.choice(L, size=n, replace=False) if n else []
    return q, codes, scales, idx


def _run(q, codes, scales, lengths, idx, m, mask, n_win, scale):
    """out, lse, weights of the GPU, the last on top of 0.5 everywhere."""
    B, S, H, D = q.shape
    T = codes.shape[1]
    out = torch.full((B, S, H, D), float("nan"), device=DEV)
    lse = torch.full((B, S, H), float("nan"), device=DEV)
    weights = torch.full((B, T), 0.5, device=DEV)
    args = (q.to(DEV), _gpu(codes), _gpu(scales), None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV),
            _gpu(idx), m, mask, n_win, scale)
    P.si_quantized_attention(*args, out, lse)
    again = torch.full_like(out, float("nan"))
    P.si_quantized_attention(*args, again)  # without lse, and the same bits
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int32), again.view(torch.int32))
    nbytes = P.si_accumulate_workspace_bytes(B, S, H, D, T)
    ws = torch.full((nbytes,), 0xAB, dtype=torch.uint8, device=DEV) if nbytes else None
    P.si_accumulate_weights(*args, lse, weights, ws)
    second = torch.full((B, T), 0.5, device=DEV)
    P.si_accumulate_weights(*args, lse, second, ws)
    torch.cuda.synchronize()
    assert torch.equal(weights.view(torch.int32), second.view(torch.int32))
    return out.double().cpu().numpy(), lse.double().cpu().numpy(), weights.double().cpu().numpy()


def _check(q, codes, scales, lengths, idx, m, mask, n_win, scale):
    out, lse, weights = _run(q, codes, scales, lengths, idx, m, mask, n_win, scale)
    want, want_lse, given, tol, lse_tol, given_tol = R.attend(q.double().numpy(), R.values(codes, scales), lengths, idx, m, mask, n_win,
                                                              float(np.float32(scale)))
    assert np.all(np.isfinite(out))
    assert np.all(np.abs(out - want) <= tol), float((np.abs(out - want) / np.maximum(tol, 1e-300)).max())
    none = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(lse), none)
    assert np.all(np.abs(lse[~none] - want_lse[~none]) <= lse_tol[~none])
    untouched = given_tol == 0
    assert np.all(weights[untouched] == 0.5)
    # adding to 0.5 in fp32 rounds once
    assert np.all(np.abs(weights - 0.5 - given) <= given_tol + R.U * np.abs(weights))
    # all of a softmax is given away
    total = weights.sum() - 0.5 * weights.size
    assert abs(total - (~none).sum()) <= given_tol.sum() + R.U * np.abs(weights).sum()
    norm = np.linalg.norm(want)
    return float(np.linalg.norm(out - want) / norm) if norm else 0.0


NONE, CAUSAL = P.SI_MASK_NONE, P.SI_MASK_CAUSAL_BLOCK


@pytest.mark.parametrize("B,S,H,D,T,m,k,mask,n_win,lengths", [
    (1, 1, 1, 64, 1, 1, 1, NONE, 0, None),            # the smallest there is
    (1, 1, 1, 64, 1, 1, 0, NONE, 1, None),            # no list
    (1, 1, 64, 128, 33, 1, 0, NONE, 33, None),        # window only, a tile and a row
    (2, 1, 33, 128, 700, 1, 300, NONE, 17, [699, 400]),
    (4, 1, 64, 128, 1500, 1, 1024, NONE, 128, [0, 1, 1500, 9999]),  # nothing held, one row, all, more than there is
    (2, 2, 64, 64, 500, 1, 100, NONE, 40, [-3, 77]),
    (3, 45, 33, 128, 90, 1, 16, CAUSAL, 5, [90, 20, 0]),
    (1, 64, 8, 64, 16, 4, 8, CAUSAL, 3, None),
    (2, 70, 32, 64, 77, 3, 7, CAUSAL, 1, [10, 77]),
    (1, 40, 64, 128, 300, 1, 100, NONE, 0, None),
    (1, 30, 20, 128, 400, 2, 96, CAUSAL, 64, None),
    (1, 8, 64, 128, 4200, 1, 4096, NONE, 64, None),   # a list of several rounds
    (1, 3, 5, 64, 5000, 1, 4096, NONE, 4096, [4999]),  # the longest list there is
    (1, 300, 64, 128, 260, 1, 65, CAUSAL, 31, None),  # many queries
    (1, 530, 40, 64, 300, 2, 33, CAUSAL, 33, [200]),
    (600, 1, 33, 128, 40, 1, 20, NONE, 4, None),      # many batches of one query
    (37, 16, 32, 128, 64, 1, 40, NONE, 8, None),
    (40, 1, 64, 128, 1700, 1, 1600, NONE, 0, None),   # long lists of a middling number of queries
    (66, 1, 33, 64, 1650, 1, 1600, NONE, 30, None),
    (1, 200, 64, 128, 500, 1, 400, CAUSAL, 20, None),  # more workgroups than compute units, rows for each
    (130, 2, 64, 64, 450, 1, 390, NONE, 0, None),
    (9, 3, 16, 128, 800, 1, 700, NONE, 128, None),     # a number of queries that no eight divide
    (1, 700, 9, 128, 350, 2, 100, CAUSAL, 7, None),    # many queries whose last block of heads has up to 16
    (2, 400, 16, 64, 300, 1, 70, NONE, 0, [300, 31]),
    (1, 1100, 1, 64, 90, 12, 20, CAUSAL, 5, None),
    (1, 300, 48, 64, 300, 1, 64, CAUSAL, 32, None),
    (1, 520, 17, 128, 200, 3, 33, CAUSAL, 0, [150]),
])
def test_attention_and_weights(B, S, H, D, T, m, k, mask, n_win, lengths):
    print(f"attention B={B} S={S} H={H} D={D} T={T} m={m} k={k} mask={mask} n_win={n_win} lengths={lengths}", flush=True)
    q, codes, scales, idx = _problem(S + 7 * T, B, S, H, D, T, k, lengths, mask, m)
    rel = _check(q, codes, scales, lengths, idx, m, mask, n_win, 1.0 / np.sqrt(D))
    print(f"  relative error {rel:.2e}", flush=True)
    assert rel <= 2e-6  # rounding of logits of size 16 (log2 units) at random: 3e-7; of the weights' two parts: 1e-7


@pytest.mark.parametrize("S,H,D", [(3, 20, 128), (40, 64, 128), (5, 33, 64), (300, 10, 128)])
@pytest.mark.parametrize("scale", [-0.2, 0.0, -0.0, 1e-30, 3.0, 1e-3])
def test_scales_of_the_softmax(S, H, D, scale):
    q, codes, scales, idx = _problem(11, 2, S, H, D, 200, 90, None, NONE, 1)
    _check(q, codes, scales, None, idx, 1, NONE, 9, scale)


@pytest.mark.parametrize("q_size,spread,scale", [
    (1e-25, 1.0, 1e24), (1e25, 1.0, 1e-26), (1.0, 1e4, 1e-5), (1.0, 1e-4, 0.3), (0.0, 1.0, 1.0), (3e-39, 1.0, 1.0), (1e4, 1e4, 1e-9),
])
@pytest.mark.parametrize("S", [2, 50])
def test_sizes_of_values(S, q_size, spread, scale):
    """Queries and rows far from 1, blocks of a row far from one another, queries of zeros and of denormal numbers."""
    q, codes, scales, idx = _problem(13, 1, S, 40, 128, 150, 70, None, NONE, 1, spread=spread, q_size=q_size)
    _check(q, codes, scales, None, idx, 1, NONE, 33, scale)


@pytest.mark.parametrize("S", [1, 30, 550])
def test_rising_logits(S):
    """The reference maximum is raised late and often; the largest and the smallest exponents of a cache."""
    B, H, D, T = 1, 8, 64, 300
    g = torch.Generator().manual_seed(4)
    q = torch.randn((B, S, H, D), generator=g).to(torch.bfloat16)
    rows = torch.randn((B, T, D), generator=g) * torch.linspace(0.01, 4.0, T)[None, :, None]
    codes, scales = R.pack(*R.quantize(rows.to(torch.bfloat16).double().numpy()))
    up = np.tile(np.arange(T, dtype=np.int32), (B, S, 1))
    _check(q, codes, scales, None, up, 1, NONE, 0, 2.0)
    _check(q, codes, scales, None, up[:, :, ::-1], 1, NONE, 0, 2.0)
    _check(q, codes, np.full_like(scales, 140), None, up, 1, NONE, 0, 1e-6)
    _check(q, codes, np.full_like(scales, 114), None, up, 1, NONE, 0, 50.0)


@pytest.mark.parametrize("S", [1, 20])
def test_entries_outside_the_rows_held_are_skipped(S):
    q, codes, scales, idx = _problem(5, 2, S, 17, 128, 100, 40, None, NONE, 1)
    idx[:, :, ::3] = np.array([-1, -2 ** 31, 100, 2 ** 31 - 1, 60, 99, -7])[np.arange(2 * S * 14) % 7].reshape(2, S, 14)
    for b in range(2):  # distinct entries
        for t in range(S):
            seen = set()
            for j in range(40):
                if idx[b, t, j] in seen:
                    idx[b, t, j] = -1
                seen.add(idx[b, t, j])
    _check(q, codes, scales, [60, 100], idx, 1, NONE, 5, 0.1)


@pytest.mark.parametrize("S,H,D,k,n_win", [(1, 33, 128, 90, 9), (3, 20, 64, 40, 0), (260, 40, 128, 60, 5), (1, 64, 128, 140, 9), (260, 16, 64, 120, 0),
                                           (600, 64, 64, 120, 0), (600, 20, 128, 140, 9)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_queries_that_are_not_finite(S, H, D, k, n_win, bad):
    """The head has NaN, no other head or query anything else than without it; its query gives no row a weight."""
    B, T = 2, 150
    q, codes, scales, idx = _problem(17, B, S, H, D, T, k, None, NONE, 1)
    idx[1, S - 1, :] = np.arange(k)  # that query has rows
    clean, clean_lse, _ = _run(q, codes, scales, None, idx, 1, NONE, n_win, 0.1)
    spoilt = q.clone()
    spoilt[1, S - 1, H - 2, 5] = bad
    out, lse, weights = _run(spoilt, codes, scales, None, idx, 1, NONE, n_win, 0.1)
    assert np.isnan(lse[1, S - 1, H - 2]) and np.all(np.isnan(out[1, S - 1, H - 2]))
    out[1, S - 1, H - 2], lse[1, S - 1, H - 2] = clean[1, S - 1, H - 2], clean_lse[1, S - 1, H - 2]
    assert np.array_equal(out, clean) and np.array_equal(lse, clean_lse)
    if n_win == 0:  # the same as if that query's list were empty
        lists = idx.copy()
        lists[1, S - 1] = -1
        assert np.array_equal(weights, _run(q, codes, scales, None, lists, 1, NONE, n_win, 0.1)[2])
    assert np.all(np.isfinite(weights))
    if S == 1:
        assert np.all(weights[1] == 0.5)


def test_weights_of_many_queries_in_one_row():
    """One row that every query and head gives everything: sums that fp32 alone would lose count in."""
    B, S, H, D, T = 1, 5000, 64, 64, 3
    q = torch.zeros((B, S, H, D), dtype=torch.bfloat16, device=DEV)
    codes = torch.zeros((B, T, D // 2), dtype=torch.uint8, device=DEV)
    scales = torch.full((B, T, D // 32), 127, dtype=torch.uint8, device=DEV)
    idx = torch.full((B, S, 1), 1, dtype=torch.int32, device=DEV)
    out, lse = torch.empty((B, S, H, D), device=DEV), torch.empty((B, S, H), device=DEV)
    P.si_quantized_attention(q, codes, scales, None, idx, 1, NONE, 0, 1.0, out, lse)
    weights = torch.tensor([[1.0, 2.0, 3.0]], device=DEV)
    ws = torch.empty(P.si_accumulate_workspace_bytes(B, S, H, D, T), dtype=torch.uint8, device=DEV)
    P.si_accumulate_weights(q, codes, scales, None, idx, 1, NONE, 0, 1.0, lse, weights, ws)
    assert weights.tolist() == [[1.0, 2.0 + S * H, 3.0]]


@pytest.mark.parametrize("S", [1, 3])
def test_attention_in_a_cache_beyond_4_gib(S):
    B, H, D, T, k = 3, 40, 128, 1 << 25, 64
    g = torch.Generator().manual_seed(6)
    q = torch.randn((B, S, H, D), generator=g).to(torch.bfloat16)
    idx = torch.stack([torch.randperm(T, generator=g)[:k] for _ in range(B * S)]).view(B, S, k).to(torch.int32)
    codes = torch.zeros((B, T, D // 2), dtype=torch.uint8, device=DEV)
    scales = torch.full((B, T, D // 32), 127, dtype=torch.uint8, device=DEV)
    short_c = torch.randint(0, 256, (B, S, k, D // 2), generator=g, dtype=torch.uint8)
    rows = idx.reshape(B, S * k).long()
    for b in range(B):
        codes[b][rows[b].to(DEV)] = short_c[b].reshape(S * k, D // 2).to(DEV)
    out = torch.empty((B, S, H, D), device=DEV)
    P.si_quantized_attention(q.to(DEV), codes, scales, None, idx.to(DEV), 1, NONE, 0, 0.05, out)
    # the same rows in a short cache
    order = torch.arange(S * k, dtype=torch.int32).view(1, S, k).expand(B, S, k).contiguous()
    c = codes.new_empty((B, S * k, D // 2))
    for b in range(B):
        c[b] = codes[b][rows[b].to(DEV)]
    small = torch.empty_like(out)
    P.si_quantized_attention(q.to(DEV), c, scales[:, :S * k].contiguous(), None, order.to(DEV), 1, NONE, 0, 0.05, small)
    assert torch.equal(out.view(torch.int32), small.view(torch.int32))


# ---------------------------------------------------------------------------------- eviction
def _evict(weights, lengths, n_keep, n_sink, n_recent, arrays, alias=False):
    B, T = weights.shape
    kept = torch.full((B, n_keep), -5, dtype=torch.int32, device=DEV)
    held = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    new = held if alias else torch.full((B,), -5, dtype=torch.int32, device=DEV)
    ws = torch.full((P.si_evict_workspace_bytes(B, T),), 0xCD, dtype=torch.uint8, device=DEV)
    src = [a.to(DEV) for a in arrays]
    dst = [torch.full((B, n_keep, *a.shape[2:]), 77, dtype=a.dtype, device=DEV) for a in arrays]
    P.si_evict_rows(_gpu(weights), held, n_keep, n_sink, n_recent, list(zip(src, dst)), kept, new, ws)
    torch.cuda.synchronize()
    for a, s in zip(arrays, src):
        assert torch.equal(a, s.cpu())
    want = R.evict(weights, lengths, n_keep, n_sink, n_recent)
    assert new.tolist() == [len(w) for w in want]
    kept = kept.cpu()
    for b, w in enumerate(want):
        assert kept[b].tolist() == w + [-1] * (n_keep - len(w)), b
        for a, d in zip(arrays, dst):
            d = d.cpu()
            assert torch.equal(d[b, :len(w)], a[b, w])
            assert bool((d[b, len(w):] == 77).all())  # rows behind the last stay as they were


def _arrays(rng, B, T, widths):
    return [torch.from_numpy(rng.integers(0, 256, (B, T, n), dtype=np.uint8)) for n in widths]


@pytest.mark.parametrize("B,T,n_keep,n_sink,n_recent,lengths", [
    (1, 1, 1, 0, 0, None), (1, 1, 1, 1, 0, [0]), (2, 5, 2, 1, 1, [5, 1]), (3, 100, 99, 0, 0, None), (2, 100, 100, 3, 90, [100, 42]),
    (1, 255, 100, 0, 0, None), (1, 256, 100, 4, 20, None), (1, 257, 256, 4, 20, None), (2, 1000, 10, 0, 10, [1000, 9]),
    (2, 1000, 10, 10, 0, None), (5, 3000, 1800, 4, 128, [3000, 0, 1800, 1801, 5000]), (1, 9000, 4500, 1, 64, [-4]),
    (1, 70001, 50000, 4, 128, None), (2, 40000, 7, 3, 2, [39999, 40000]),
])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
def test_evict(B, T, n_keep, n_sink, n_recent, lengths, kind):
    print(f"evict B={B} T={T} n_keep={n_keep} n_sink={n_sink} n_recent={n_recent} lengths={lengths} {kind}", flush=True)
    rng = np.random.default_rng(T + n_keep)
    w = np.exp(3 * rng.standard_normal((B, T))).astype(np.float32)
    if kind == "ties":  # a few sizes, many rows that received nothing
        w = rng.choice(np.array([0.0, -0.0, 0.0, 1.0, 1.0 + 2.0 ** -23, 5.0], dtype=np.float32), (B, T))
    if kind == "odd":
        w = rng.choice(np.array([np.inf, -np.inf, np.nan, -np.nan, 0.0, -1.0, 1e-45, 3e38, -3e38], dtype=np.float32), (B, T))
    _evict(w, lengths, n_keep, n_sink, n_recent, _arrays(rng, B, T, (4, 64)), alias=lengths is not None and kind == "ties")


@pytest.mark.parametrize("B,T,n_keep,n_sink,n_recent,lengths", [
    (2, 4097, 4096, 0, 1, None), (1, 16385, 9000, 4, 128, None), (3, 32768, 20000, 0, 0, [32768, 20001, 16385]), (2, 32769, 3, 0, 0, [32769, 2]),
    (3, 50000, 30000, 1, 1, [0, 30001, 50000]), (3, 20000, 64, 60, 4, [20000, 65, 64]), (2, 40000, 64, 60, 4, [40000, 65]),
])
@pytest.mark.parametrize("kind", ["one", "spread", "near"])
def test_evict_sizes_of_each_kind(B, T, n_keep, n_sink, n_recent, lengths, kind):
    """Around the sizes where another kernel or another number of rows a thread begins; all weights alike, far apart, and of one exponent."""
    print(f"evict B={B} T={T} n_keep={n_keep} n_sink={n_sink} n_recent={n_recent} lengths={lengths} {kind}", flush=True)
    rng = np.random.default_rng(T)
    w = np.full((B, T), 2.5, dtype=np.float32)
    if kind == "spread":
        w = (rng.choice([-1.0, 1.0], (B, T)) * np.exp(15 * rng.standard_normal((B, T)))).astype(np.float32)
    if kind == "near":
        w = (1 + rng.integers(0, 5000, (B, T)) * 2.0 ** -23).astype(np.float32)
    _evict(w, lengths, n_keep, n_sink, n_recent, _arrays(rng, B, T, (4,)))


@pytest.mark.parametrize("T", [300, 3000, 20000, 40000])
@pytest.mark.parametrize("n_keep", [40, 200])
def test_evict_among_infinities(T, n_keep):
    """The border among the largest weights there can be, with NaN the smallest, beside rows that stay whatever theirs are."""
    rng = np.random.default_rng(T)
    w = rng.choice(np.array([np.inf, np.nan], dtype=np.float32), (2, T))
    _evict(w, None, n_keep, 4, 9, _arrays(rng, 2, T, (4,)))
    w[:, ::3] = np.finfo(np.float32).max
    w[:, 60:] = np.where(np.isinf(w[:, 60:]), np.float32(1), w[:, 60:])
    _evict(w, [T - 1, 299], n_keep, 4, 9, _arrays(rng, 2, T, (4,)))


@pytest.mark.parametrize("widths", [(), (1,), (2, 3), (16, 32, 48), (256, 64, 4, 4), (5, 6, 10, 12, 20, 100, 7, 260)])
def test_evict_row_sizes(widths):
    rng = np.random.default_rng(len(widths))
    w = rng.standard_normal((3, 700)).astype(np.float32)
    _evict(w, [700, 300, 650], 400, 2, 33, _arrays(rng, 3, 700, widths))


@pytest.mark.parametrize("B,T", [(1, 130), (1, 25000), (1, 25700), (7, 3500), (32, 4000), (33, 4096), (2, 32768), (512, 200), (513, 200)])
@pytest.mark.parametrize("alias", [False, True])
def test_evict_by_one_launch_and_by_two(B, T, alias):
    """Around the numbers of rows from which on another launch or another share of the arrays is taken; lengths rewritten or not."""
    print(f"evict B={B} T={T} alias={alias}", flush=True)
    rng = np.random.default_rng(B + T)
    w = np.where(rng.random((B, T)) < 0.3, 0, np.exp(2 * rng.standard_normal((B, T)))).astype(np.float32)
    lengths = rng.integers(0, T + 1, B).tolist()
    lengths[-1] = T
    _evict(w, lengths, max(1, T * 2 // 3), 4, 11, _arrays(rng, B, T, (16, 4, 1)), alias=alias)


def test_evict_moves_arrays_of_any_type():
    rng = np.random.default_rng(3)
    w = rng.standard_normal((2, 500)).astype(np.float32)
    _evict(w, None, 300, 0, 0, [torch.from_numpy(w), torch.from_numpy(w).double(), torch.from_numpy(w).to(torch.bfloat16),
                                torch.arange(1000, dtype=torch.int32).view(2, 500), torch.randn((2, 500, 3, 5)).to(torch.bfloat16)])


def test_evict_beyond_4_gib():
    B, T, n = 2, 1 << 22, 1 << 21
    g = torch.Generator(device=DEV).manual_seed(1)
    w = torch.rand((B, T), generator=g, device=DEV)
    src = torch.arange(B * T, device=DEV, dtype=torch.int32).view(B, T, 1).expand(B, T, 256).contiguous()  # 1 KiB a row: 8 GiB
    dst = torch.zeros((B, n, 256), device=DEV, dtype=torch.int32)
    kept = torch.empty((B, n), dtype=torch.int32, device=DEV)
    ws = torch.empty(P.si_evict_workspace_bytes(B, T), dtype=torch.uint8, device=DEV)
    P.si_evict_rows(w, None, n, 4, 128, [(src, dst)], kept, None, ws)
    rank = w.double()
    rank[:, :4] = 2.0
    rank[:, -128:] = 2.0
    want = torch.sort(torch.sort(rank, dim=1, descending=True, stable=True)[1][:, :n], dim=1)[0]
    assert torch.equal(kept.long(), want)
    assert torch.equal(dst[:, :, 0].long(), want + torch.arange(B, device=DEV)[:, None] * T)
    assert bool((dst == dst[:, :, :1]).all())


# ---------------------------------------------------------------------------------- together
def test_a_serving_loop():
    """Prompts enter the cache, decoding steps append, attend and accumulate, the cache is cut back, decoding goes on: against the
    reference at every step."""
    B, H, D, T, k, n_win, n_keep = 3, 33, 128, 96, 24, 8, 48
    g = torch.Generator().manual_seed(9)
    rng = np.random.default_rng(9)
    prompt = torch.randn((B, 60, D), generator=g).to(torch.bfloat16)
    codes = torch.zeros((B, T, D // 2), dtype=torch.uint8, device=DEV)
    scales = torch.full((B, T, D // 32), 127, dtype=torch.uint8, device=DEV)
    weights = torch.zeros((B, T), device=DEV)
    lengths = torch.tensor([60, 41, 5], dtype=torch.int32, device=DEV)  # ragged prompts: the rows behind are overwritten
    P.si_quantize_rows(prompt.to(DEV), None, codes, scales)
    want_w = np.zeros((B, T))
    slack = np.zeros((B, T))
    rounds = 30
    for step in range(rounds):
        new = torch.randn((B, 1, D), generator=g).to(torch.bfloat16)
        P.si_quantize_rows(new.to(DEV), lengths, codes, scales)
        lengths += 1
        q = torch.randn((B, 1, H, D), generator=g).to(torch.bfloat16)
        n_held = lengths.tolist()
        idx = np.full((B, 1, k), -1, dtype=np.int32)
        for b in range(B):
            n = min(k, n_held[b])
            idx[b, 0, :n] = rng.choice(n_held[b], size=n, replace=False)
        out, lse = torch.full((B, 1, H, D), float("nan"), device=DEV), torch.full((B, 1, H), float("nan"), device=DEV)
        P.si_quantized_attention(q.to(DEV), codes, scales, lengths, _gpu(idx), 1, NONE, n_win, 0.1, out, lse)
        P.si_accumulate_weights(q.to(DEV), codes, scales, lengths, _gpu(idx), 1, NONE, n_win, 0.1, lse, weights)
        V = R.values(codes.cpu().numpy(), scales.cpu().numpy())
        want, want_lse, given, tol, lse_tol, given_tol = R.attend(q.double().numpy(), V, n_held, idx, 1, NONE, n_win, float(np.float32(0.1)))
        assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
        assert np.all(np.abs(lse.double().cpu().numpy() - want_lse) <= lse_tol)
        want_w += given
        slack += given_tol + R.U * np.abs(want_w)
        got_w = weights.cpu().numpy()
        assert np.all(np.abs(got_w - want_w) <= slack)
        if max(n_held) >= 70:  # the bounded length
            kept = torch.empty((B, n_keep), dtype=torch.int32, device=DEV)
            ws = torch.empty(P.si_evict_workspace_bytes(B, T), dtype=torch.uint8, device=DEV)
            to = [torch.zeros((B, n_keep, *a.shape[2:]), dtype=a.dtype, device=DEV) for a in (codes, scales, weights)]
            stay = R.evict(got_w, n_held, n_keep, 2, n_win)
            P.si_evict_rows(weights, lengths, n_keep, 2, n_win, list(zip((codes, scales, weights), to)), kept, lengths, ws)
            assert [row[row >= 0].tolist() for row in kept.cpu()] == stay
            assert lengths.tolist() == [len(x) for x in stay]
            for a, d in zip((codes, scales, weights), to):
                a[:, :n_keep] = d
                a[:, n_keep:] = 0
            moved, moved_slack = np.zeros_like(want_w), np.zeros_like(slack)
            for b, rows in enumerate(stay):
                moved[b, :len(rows)], moved_slack[b, :len(rows)] = want_w[b, rows], slack[b, rows]
                assert np.array_equal(R.values(codes[b, :len(rows)].cpu().numpy(), scales[b, :len(rows)].cpu().numpy()), V[b, rows])
            want_w, slack = moved, moved_slack
            weights[:, n_keep:] = 0
    assert max(lengths.tolist()) < 70


def test_lists_from_the_indexer():
    """The real producer of the lists, and the bf16 consumer on the same values: both read the same rows."""
    B, S, H, D, m, k, n_win = 1, 512, 64, 128, 4, 64, 16
    T = S // m
    g = torch.Generator().manual_seed(5)
    q = torch.randn((B, S, H, D), generator=g).to(torch.bfloat16).to(DEV)
    K = torch.randn((B, T, D), generator=g).to(torch.bfloat16).to(DEV)
    w = (torch.randn((B, S, H), generator=g) / np.sqrt(H)).to(DEV)
    idx = torch.empty((B, S, k), dtype=torch.int32, device=DEV)
    score = torch.empty((B, S, k), device=DEV)
    P.si_indexer_topk(q, K, w, m, k, CAUSAL, idx, score, torch.empty(64 << 20, dtype=torch.uint8, device=DEV))
    codes = torch.empty((B, T, D // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((B, T, D // 32), dtype=torch.uint8, device=DEV)
    P.si_quantize_rows(K, None, codes, scales)
    values = torch.empty_like(K)
    P.si_dequantize_rows(codes, scales, None, values)
    out, ref = torch.empty((B, S, H, D), device=DEV), torch.empty((B, S, H, D), device=DEV)
    P.si_quantized_attention(q, codes, scales, None, idx, m, CAUSAL, n_win, 0.09, out)
    P.si_sparse_attention(q, values, idx, m, CAUSAL, n_win, 0.09, ref)
    torch.cuda.synchronize()
    # the bf16 consumer carries its weights with 16 bits: 2^-17 of a value's size, both sides' fp32 sums beside
    assert bool(((out - ref).abs() <= 2e-5 * (values.abs().amax() + 1)).all())


def _replays(call, outputs):
    """call(outputs, stream) eagerly, on a side stream and captured; every replay checked, with eager work and
    synchronisations of the program's own in between."""
    def fresh():
        return [torch.full_like(o, 9) for o in outputs]

    def same(a, b):
        return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))

    eager, on_side, captured = fresh(), fresh(), fresh()
    call(eager, None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(on_side, None)
    side.synchronize()
    assert same(eager, on_side)
    torch.cuda.synchronize()
    on_side = fresh()
    side.wait_stream(torch.cuda.current_stream())
    call(on_side, side)  # named, while another stream is the current one
    side.synchronize()
    assert same(eager, on_side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(captured, None)
    for replay in range(3):
        for o in captured:
            o.fill_(9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(eager, captured), f"replay {replay}"
        again = fresh()
        call(again, None)
        torch.cuda.synchronize()
        assert same(eager, again)


@pytest.mark.parametrize("B,S,H,D,T,k,n_win", [(5, 1, 64, 128, 700, 300, 17), (1, 400, 40, 64, 500, 60, 8), (2, 3, 20, 128, 300, 100, 0),
                                                  (2, 2, 8, 64, 40000, 50, 4), (40, 1, 16, 64, 3600, 40, 4), (1, 1, 64, 128, 3000, 1700, 64)])
def test_side_streams_and_replays(B, S, H, D, T, k, n_win):
    q, codes, scales, idx = _problem(21, B, S, H, D, T, k, None, NONE, 1)
    q, codes, scales, idx = q.to(DEV), _gpu(codes), _gpu(scales), _gpu(idx)
    lengths = torch.randint(T // 2, T + 1, (B,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).to(DEV)
    lse = torch.empty((B, S, H), device=DEV)
    _replays(lambda o, s: P.si_quantized_attention(q, codes, scales, lengths, idx, 1, NONE, n_win, 0.1, o[0], o[1], stream=s),
             (torch.empty((B, S, H, D), device=DEV), lse))
    P.si_quantized_attention(q, codes, scales, lengths, idx, 1, NONE, n_win, 0.1, torch.empty((B, S, H, D), device=DEV), lse)
    nbytes = P.si_accumulate_workspace_bytes(B, S, H, D, T)
    ws = torch.randint(0, 256, (max(nbytes, 16),), dtype=torch.uint8, device=DEV)
    _replays(lambda o, s: P.si_accumulate_weights(q, codes, scales, lengths, idx, 1, NONE, n_win, 0.1, lse, o[0], ws, stream=s),
             (torch.empty((B, T), device=DEV),))
    rows = torch.randn((B, T // 2, D), device=DEV).to(torch.bfloat16)
    _replays(lambda o, s: P.si_quantize_rows(rows, lengths, o[0], o[1], stream=s), (codes, scales))
    _replays(lambda o, s: P.si_dequantize_rows(codes, scales, lengths, o[0], stream=s), (rows,))
    w = torch.rand((B, T), device=DEV)
    ws = torch.randint(0, 256, (P.si_evict_workspace_bytes(B, T),), dtype=torch.uint8, device=DEV)
    n = T // 2
    _replays(lambda o, s: P.si_evict_rows(w, lengths, n, 4, 32, [(codes, o[0]), (w, o[1])], o[2], o[3], ws, stream=s),
             (torch.empty((B, n, D // 2), dtype=torch.uint8, device=DEV), torch.empty((B, n), device=DEV),
              torch.empty((B, n), dtype=torch.int32, device=DEV), torch.empty((B,), dtype=torch.int32, device=DEV)))


@pytest.mark.parametrize("B,S", [(1, (1 << 24) - 8), (2, (1 << 23) - 4), ((1 << 24) - 8, 1)])
def test_the_most_queries_a_call_takes(B, S):
    """Every query sees its batch's one row: that comes out, and receives a weight of 1 a query."""
    H, D, T = 1, 64, 1
    print(f"B={B} S={S}", flush=True)
    q = torch.ones((B, S, H, D), dtype=torch.bfloat16, device=DEV)
    codes = (torch.arange(B, device=DEV) % 251).to(torch.uint8).view(B, 1, 1).expand(B, T, D // 2).contiguous()
    scales = torch.full((B, T, D // 32), 127, dtype=torch.uint8, device=DEV)
    V = torch.empty((B, T, D), dtype=torch.bfloat16, device=DEV)
    P.si_dequantize_rows(codes, scales, None, V)
    out, lse = torch.full((B, S, H, D), float("nan"), device=DEV), torch.full((B, S, H), float("nan"), device=DEV)
    P.si_quantized_attention(q, codes, scales, None, None, 1, NONE, 1, 0.125, out, lse)
    # The one weight p is also its sum.  (hi + lo) V / p: the two parts are p to 2^-22 of it, their products with V exact; a rounding each
    # of their sum, of the quotient 1 / p and of the product with it.
    want = V.float().view(B, 1, 1, D)
    off = ((out - want).abs() / want.abs().clamp(min=0.5)).max().item()
    assert off <= 2.0 ** -22 + 4 * R.U, off
    # one row: its logit itself, whose products are exact; the factor to log2 and back round five times
    x = V.float().sum(dim=2).view(B, 1, 1) * 0.125
    assert bool(((lse - x).abs() <= 5 * R.U * x.abs() + 2.0 ** -20).all())
    weights = torch.zeros((B, T), device=DEV)
    nbytes = P.si_accumulate_workspace_bytes(B, S, H, D, T)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV) if nbytes else None
    P.si_accumulate_weights(q, codes, scales, None, None, 1, NONE, 1, 0.125, lse, weights, ws)
    # exp(logit - lse): both logits and what lse is off by, in units of a logit of up to 48
    assert bool(((weights - S).abs() <= S * 2.0 ** -16).all())


def test_the_most_batches_eviction_takes():
    B, T = (1 << 22) - 1, 2
    w = torch.zeros((B, T), device=DEV)
    w[::3, 1] = 1.0
    kept, new = torch.empty((B, 1), dtype=torch.int32, device=DEV), torch.empty((B,), dtype=torch.int32, device=DEV)
    src = torch.arange(2 * B, dtype=torch.int32, device=DEV).view(B, T)
    dst = torch.empty((B, 1), dtype=torch.int32, device=DEV)
    ws = torch.empty(P.si_evict_workspace_bytes(B, T), dtype=torch.uint8, device=DEV)
    P.si_evict_rows(w, None, 1, 0, 0, [(src, dst)], kept, new, ws)
    assert torch.equal(kept[:, 0], (w[:, 1] > 0).int()) and bool((new == 1).all())
    assert torch.equal(dst, src.gather(1, kept.long()))


@pytest.mark.parametrize("T", [700, 40000])
def test_two_calls_at_once(T):
    """Two streams, each with its own outputs and workspace, on the same inputs."""
    B, S, H, D, k, n = 3, 40, 40, 128, 200, 400
    q, codes, scales, idx = _problem(31, B, S, H, D, 700, k, None, NONE, 1)
    q, idx = q.to(DEV), _gpu(idx)
    codes = torch.cat([_gpu(codes), torch.zeros((B, T - 700, D // 2), dtype=torch.uint8, device=DEV)], dim=1)
    scales = torch.cat([_gpu(scales), torch.full((B, T - 700, D // 32), 127, dtype=torch.uint8, device=DEV)], dim=1)
    given = torch.rand((B, T), device=DEV)

    def outputs():
        return (torch.zeros((B, S, H, D), device=DEV), torch.zeros((B, S, H), device=DEV), torch.zeros((B, T), device=DEV),
                torch.zeros((B, n, D // 2), dtype=torch.uint8, device=DEV), torch.zeros((B, n), dtype=torch.int32, device=DEV),
                torch.randint(0, 256, (8 * B * T,), dtype=torch.uint8, device=DEV),
                torch.randint(0, 256, (P.si_evict_workspace_bytes(B, T),), dtype=torch.uint8, device=DEV))

    def run(o, stream):
        P.si_quantized_attention(q, codes, scales, None, idx, 1, NONE, 9, 0.1, o[0], o[1], stream=stream)
        P.si_accumulate_weights(q, codes, scales, None, idx, 1, NONE, 9, 0.1, o[1], o[2], o[5], stream=stream)
        P.si_evict_rows(given, None, n, 4, 32, [(codes, o[3])], o[4], None, o[6], stream=stream)

    alone = outputs()
    run(alone, None)
    sides, results = [torch.cuda.Stream() for _ in range(2)], [outputs() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for o, side in zip(results, sides):
            o[2].zero_()
        torch.cuda.synchronize()
        for o, side in zip(results, sides):
            run(o, side)
        torch.cuda.synchronize()
        for o in results:
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(alone[:5], o[:5]))


def test_refusals_of_the_binding():
    codes = torch.zeros((1, 8, 32), dtype=torch.uint8, device=DEV)
    scales = torch.full((1, 8, 2), 127, dtype=torch.uint8, device=DEV)
    q = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16, device=DEV)
    idx = torch.zeros((1, 2, 3), dtype=torch.int32, device=DEV)
    out, lse, w = torch.empty((1, 2, 4, 64), device=DEV), torch.empty((1, 2, 4), device=DEV), torch.zeros((1, 8), device=DEV)
    with pytest.raises(TypeError):
        P.si_quantized_attention(q.half(), codes, scales, None, idx, 1, NONE, 0, 1.0, out)
    with pytest.raises(TypeError):
        P.si_quantized_attention(q, codes, scales, None, idx.long(), 1, NONE, 0, 1.0, out)
    with pytest.raises(ValueError):
        P.si_quantized_attention(q, codes, scales, torch.zeros(2, dtype=torch.int32, device=DEV), idx, 1, NONE, 0, 1.0, out)
    with pytest.raises(ValueError):  # not contiguous
        P.si_quantized_attention(q.transpose(1, 2).contiguous().transpose(1, 2), codes, scales, None, idx, 1, NONE, 0, 1.0, out)
    with pytest.raises(P.StreamIndexError) as e:
        P.si_quantized_attention(q, codes, scales, None, idx, 1, NONE, 0, float("inf"), out)
    assert e.value.status == P.SI_ERR_INVALID_ARG
    with pytest.raises(P.StreamIndexError) as e:
        P.si_accumulate_weights(q, codes, scales, None, idx, 1, NONE, 0, 1.0, lse, w, torch.empty(63, dtype=torch.uint8, device=DEV))
    assert e.value.status == P.SI_ERR_WORKSPACE_TOO_SMALL
    kept = torch.empty((1, 4), dtype=torch.int32, device=DEV)
    with pytest.raises(P.StreamIndexError) as e:
        P.si_evict_rows(w, None, 4, 0, 0, [], kept, None, torch.empty(16, dtype=torch.uint8, device=DEV))
    assert e.value.status == P.SI_ERR_WORKSPACE_TOO_SMALL
    with pytest.raises(P.StreamIndexError) as e:  # dst inside src
        P.si_evict_rows(w, None, 4, 0, 0, [(w, w[:, :4].contiguous()), (codes, codes[:, :4])], kept, None,
                        torch.empty(4096, dtype=torch.uint8, device=DEV))
    assert e.value.status == P.SI_ERR_INVALID_ARG
