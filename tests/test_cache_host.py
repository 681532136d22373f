"""CPU-only: the 4-bit cache's entry points refuse what they cannot do before anything is launched (pointers are never used), their
sizes, the binding's checks, and the plain 64-bit reference against values worked by hand."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2605_02568_amd as P
from paper_2605_02568_amd import binding
from tests import cache_reference as R

A = ctypes.c_void_p


def _rows_call(rows=0x1000, codes=0x2000, scales=0x3000, dims=(2, 3, 1, 64, 5), start=None):
    lib, d = P.load(), binding.si_dims(*dims)
    return (lib.si_quantize_rows(A(rows), A(start), ctypes.byref(d), A(codes), A(scales), None),
            lib.si_dequantize_rows(A(codes), A(scales), A(start), ctypes.byref(d), A(rows), None))


@pytest.mark.parametrize("bad,status", [
    (dict(rows=None), P.SI_ERR_INVALID_ARG), (dict(codes=None), P.SI_ERR_INVALID_ARG), (dict(scales=None), P.SI_ERR_INVALID_ARG),
    (dict(rows=0x1008), P.SI_ERR_INVALID_ARG), (dict(codes=0x2004), P.SI_ERR_INVALID_ARG), (dict(scales=0x3001), P.SI_ERR_INVALID_ARG),
    (dict(start=0x4002), P.SI_ERR_INVALID_ARG),
    (dict(dims=(0, 3, 1, 64, 5)), P.SI_ERR_INVALID_ARG), (dict(dims=(2, 0, 1, 64, 5)), P.SI_ERR_INVALID_ARG),
    (dict(dims=(2, 3, 1, 64, 0)), P.SI_ERR_INVALID_ARG), (dict(dims=(2, 3, 1, 0, 5)), P.SI_ERR_INVALID_ARG),
    (dict(dims=(2, 3, 1, 96, 5)), P.SI_ERR_UNSUPPORTED_SHAPE), (dict(dims=(2, 3, 1, 256, 5)), P.SI_ERR_UNSUPPORTED_SHAPE),
])
def test_rows_refusals(bad, status):
    assert _rows_call(**bad) == (status, status)


GOOD = dict(qa=0x1000, codes=0x2000, scales=0x3000, lengths=0x4000, idx=0x5000, dims=(2, 3, 4, 64, 50), m=1, k=8, mask=0, n_win=4, scale=0.1,
            out=0x6000, lse=0x7000, weights=0x8000, ws=0x9000, ws_bytes=800)


def _attention_calls(**bad):
    a = {**GOOD, **bad}
    lib = P.load()
    d = None if a["dims"] is None else ctypes.byref(binding.si_dims(*a["dims"]))
    common = (A(a["qa"]), A(a["codes"]), A(a["scales"]), A(a["lengths"]), A(a["idx"]), d, a["m"], a["k"], a["mask"], a["n_win"], a["scale"])
    return (lib.si_quantized_attention(*common, A(a["out"]), A(a["lse"]), None),
            lib.si_accumulate_weights(*common, A(a["lse"]), A(a["weights"]), A(a["ws"]), a["ws_bytes"], None))


@pytest.mark.parametrize("bad,status", [
    (dict(qa=None), P.SI_ERR_INVALID_ARG), (dict(codes=None), P.SI_ERR_INVALID_ARG), (dict(scales=None), P.SI_ERR_INVALID_ARG),
    (dict(idx=None), P.SI_ERR_INVALID_ARG), (dict(dims=None), P.SI_ERR_INVALID_ARG),
    (dict(qa=0x1008), P.SI_ERR_INVALID_ARG), (dict(codes=0x2008), P.SI_ERR_INVALID_ARG), (dict(scales=0x3004), P.SI_ERR_INVALID_ARG),
    (dict(idx=0x5004), P.SI_ERR_INVALID_ARG), (dict(lse=0x7004), P.SI_ERR_INVALID_ARG),
    (dict(lengths=0x4001), P.SI_ERR_INVALID_ARG),
    (dict(m=0), P.SI_ERR_INVALID_ARG), (dict(k=-1), P.SI_ERR_INVALID_ARG), (dict(n_win=-1), P.SI_ERR_INVALID_ARG),
    (dict(mask=2), P.SI_ERR_INVALID_ARG), (dict(scale=float("nan")), P.SI_ERR_INVALID_ARG), (dict(scale=float("-inf")), P.SI_ERR_INVALID_ARG),
    (dict(scale=2.5e38), P.SI_ERR_INVALID_ARG), (dict(scale=-3e38), P.SI_ERR_INVALID_ARG),
    (dict(dims=(2, 3, 0, 64, 50)), P.SI_ERR_INVALID_ARG), (dict(dims=(2, 3, 4, 64, 0)), P.SI_ERR_INVALID_ARG),
    (dict(dims=(2, 3, 4, 32, 50)), P.SI_ERR_UNSUPPORTED_SHAPE), (dict(dims=(2, 3, 65, 64, 50)), P.SI_ERR_UNSUPPORTED_SHAPE),
    (dict(k=4097), P.SI_ERR_UNSUPPORTED_SHAPE), (dict(n_win=4097), P.SI_ERR_UNSUPPORTED_SHAPE),
    (dict(dims=(16, 1 << 20, 4, 64, 50)), P.SI_ERR_UNSUPPORTED_SHAPE),
    (dict(dims=(1, (1 << 24) - 7, 4, 64, 50)), P.SI_ERR_UNSUPPORTED_SHAPE),
    (dict(dims=(1, 1, 4, 64, (1 << 30) + 1)), P.SI_ERR_UNSUPPORTED_SHAPE),
])
def test_attention_and_weights_refusals(bad, status):
    assert _attention_calls(**bad) == (status, status)


@pytest.mark.parametrize("bad,status", [
    (dict(out=None), P.SI_ERR_INVALID_ARG), (dict(out=0x6004), P.SI_ERR_INVALID_ARG),
])
def test_attention_refusals(bad, status):
    assert _attention_calls(**{**bad, "weights": None})[0] == status


@pytest.mark.parametrize("bad,status", [
    (dict(lse=None), P.SI_ERR_INVALID_ARG), (dict(weights=None), P.SI_ERR_INVALID_ARG), (dict(weights=0x8004), P.SI_ERR_INVALID_ARG),
    (dict(ws=None), P.SI_ERR_INVALID_ARG), (dict(ws=0x9008), P.SI_ERR_INVALID_ARG), (dict(ws_bytes=799), P.SI_ERR_WORKSPACE_TOO_SMALL),
])
def test_weights_refusals(bad, status):
    assert _attention_calls(**{**bad, "out": None})[1] == status


def test_accumulate_workspace():
    assert P.si_accumulate_workspace_bytes(2, 3, 4, 64, 50) == 800
    assert P.si_accumulate_workspace_bytes(2, 1, 4, 64, 50) == 0  # one query a batch: nothing to add up
    assert P.si_accumulate_workspace_bytes(0, 3, 4, 64, 50) == 0


EVICT = dict(weights=0x10000, lengths=0x20000, B=2, T=1000, n_keep=600, n_sink=4, n_recent=100, moves=((0x100000, 0x200000, 68),),
             kept=0x30000, new_lengths=0x20000, ws=0x40000, ws_bytes=1 << 16)


def _evict_call(**bad):
    a = {**EVICT, **bad}
    moves = a["moves"]
    table = None
    if moves is not None:
        table = (binding.si_row_move * max(1, len(moves)))(*[binding.si_row_move(*x) for x in moves])
    return P.load().si_evict_rows(A(a["weights"]), A(a["lengths"]), a["B"], a["T"], a["n_keep"], a["n_sink"], a["n_recent"], table,
                                  len(moves) if moves is not None else 1, A(a["kept"]), A(a["new_lengths"]), A(a["ws"]), a["ws_bytes"], None)


@pytest.mark.parametrize("bad,status", [
    (dict(weights=None), P.SI_ERR_INVALID_ARG), (dict(kept=None), P.SI_ERR_INVALID_ARG), (dict(ws=None), P.SI_ERR_INVALID_ARG),
    (dict(moves=None), P.SI_ERR_INVALID_ARG), (dict(moves=((None, 0x200000, 4),)), P.SI_ERR_INVALID_ARG),
    (dict(moves=((0x100000, None, 4),)), P.SI_ERR_INVALID_ARG), (dict(moves=((0x100000, 0x200000, 0),)), P.SI_ERR_INVALID_ARG),
    (dict(moves=((0x100008, 0x200000, 4),)), P.SI_ERR_INVALID_ARG), (dict(moves=((0x100000, 0x200004, 4),)), P.SI_ERR_INVALID_ARG),
    (dict(moves=tuple((0x100000 * i, 0x1000000 * i, 4) for i in range(1, 10))), P.SI_ERR_INVALID_ARG),
    (dict(weights=0x10004), P.SI_ERR_INVALID_ARG), (dict(kept=0x30008), P.SI_ERR_INVALID_ARG), (dict(ws=0x40004), P.SI_ERR_INVALID_ARG),
    (dict(lengths=0x20002), P.SI_ERR_INVALID_ARG), (dict(new_lengths=0x20401), P.SI_ERR_INVALID_ARG),
    (dict(B=1 << 22, T=200, n_keep=100, n_sink=0, n_recent=0), P.SI_ERR_UNSUPPORTED_SHAPE),
    (dict(B=0), P.SI_ERR_INVALID_ARG), (dict(T=0), P.SI_ERR_INVALID_ARG), (dict(n_keep=0), P.SI_ERR_INVALID_ARG),
    (dict(n_keep=1001), P.SI_ERR_INVALID_ARG), (dict(n_sink=-1), P.SI_ERR_INVALID_ARG), (dict(n_recent=-1), P.SI_ERR_INVALID_ARG),
    (dict(n_sink=300, n_recent=301), P.SI_ERR_INVALID_ARG), (dict(n_sink=1, n_recent=2 ** 31 - 1), P.SI_ERR_INVALID_ARG),
    (dict(ws_bytes=63), P.SI_ERR_WORKSPACE_TOO_SMALL), (dict(T=(1 << 30) + 1), P.SI_ERR_UNSUPPORTED_SHAPE),
    # what is written overlaps what is read or written
    (dict(moves=((0x100000, 0x100000 + 68 * 999 * 2, 68),)), P.SI_ERR_INVALID_ARG),  # a move onto its own source's end
    (dict(moves=((0x100000, 0x10000, 4),)), P.SI_ERR_INVALID_ARG),                    # onto the weights
    (dict(moves=((0x10000, 0x10000, 4),)), P.SI_ERR_INVALID_ARG),                     # in place
    (dict(moves=((0x100000, 0x30000, 4),)), P.SI_ERR_INVALID_ARG),                    # onto kept
    (dict(moves=((0x100000, 0x40010, 4),)), P.SI_ERR_INVALID_ARG),                    # onto the workspace
    (dict(moves=((0x100000, 0x200000, 4), (0x180000, 0x200010, 4))), P.SI_ERR_INVALID_ARG),  # two onto the same place
    (dict(moves=((0x100000, 0x200000, 4), (0x180000, 0x100010, 4))), P.SI_ERR_INVALID_ARG),  # onto another one's source
    (dict(kept=0x11f30), P.SI_ERR_INVALID_ARG), (dict(ws=0x11f30), P.SI_ERR_INVALID_ARG), (dict(new_lengths=0x20004), P.SI_ERR_INVALID_ARG),
    (dict(new_lengths=0x10000), P.SI_ERR_INVALID_ARG), (dict(lengths=0x30000, new_lengths=None), P.SI_ERR_INVALID_ARG),
])
def test_evict_refusals(bad, status):
    assert _evict_call(**bad) == status


def test_evict_workspace_grows_with_rows_and_batches():
    one = P.si_evict_workspace_bytes(1, 1000)
    assert 0 < one < P.si_evict_workspace_bytes(1, 100000) <= 100000 + 65536
    assert P.si_evict_workspace_bytes(7, 1000) >= 7 * 16
    assert P.si_evict_workspace_bytes(0, 10) == 0 and P.si_evict_workspace_bytes(1, 0) == 0


def test_binding_checks_shapes_and_types_first(monkeypatch):
    class Untouchable:
        def __getattr__(self, name):
            raise AssertionError(f"library entry {name} was reached")

    monkeypatch.setattr(binding, "_lib", Untouchable())
    B, S, H, D, T, k, n = 2, 3, 4, 64, 10, 5, 6
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    rows, q = torch.zeros((B, S, D), dtype=torch.bfloat16), torch.zeros((B, S, H, D), dtype=torch.bfloat16)
    codes, scales, idx = u8(B, T, D // 2), u8(B, T, D // 32), torch.zeros((B, S, k), dtype=torch.int32)
    out, lse, w = torch.zeros((B, S, H, D)), torch.zeros((B, S, H)), torch.zeros((B, T))
    for c, s in ((u8(B, T, D), scales), (codes, u8(B, T, 1)), (u8(1, T, D // 2), scales), (codes, u8(B, T + 1, D // 32)), (u8(T, D // 2), scales)):
        with pytest.raises(ValueError):
            P.si_quantize_rows(rows, None, c, s)
        with pytest.raises(ValueError):
            P.si_dequantize_rows(c, s, None, rows)
        with pytest.raises(ValueError):
            P.si_quantized_attention(q, c, s, None, idx, 1, 0, 0, 1.0, out, lse)
        with pytest.raises(ValueError):
            P.si_accumulate_weights(q, c, s, None, idx, 1, 0, 0, 1.0, lse, w)
    with pytest.raises(ValueError):
        P.si_quantized_attention(q, codes, scales, None, idx[:, :2], 1, 0, 0, 1.0, out, lse)
    with pytest.raises(TypeError):  # host tensors
        P.si_quantize_rows(rows, None, codes, scales)
    with pytest.raises(TypeError):
        P.si_quantized_attention(q, codes, scales, None, idx, 1, 0, 0, 1.0, out, lse)
    kept, ws = torch.zeros((B, n), dtype=torch.int32), u8(1 << 16)
    for moves in ([(w, torch.zeros((B, n + 1)))], [(w, torch.zeros((B, n), dtype=torch.float64))], [(w[:, :3], w)], [(w, w)] * 9):
        with pytest.raises(ValueError):
            P.si_evict_rows(w, None, n, 0, 0, moves, kept, None, ws)
    with pytest.raises(ValueError):
        P.si_evict_rows(w, None, n, 0, 0, [], kept[:, :2], None, ws)
    with pytest.raises(ValueError):
        P.si_evict_rows(w[0], None, n, 0, 0, [], kept, None, ws)


def test_binding_refuses_sizes_beyond_int32():
    for sizes in ((2 ** 31, 1, 1, 64, 1), (1, 1, 1, 64, 2 ** 32 + 5)):
        with pytest.raises(ValueError):
            P.si_accumulate_workspace_bytes(*sizes)
    with pytest.raises(ValueError):
        P.si_evict_workspace_bytes(1, 2 ** 32 + 5)
    meta = lambda *s: torch.empty(s, device="meta", dtype=torch.uint8)  # noqa: E731
    with pytest.raises((ValueError, TypeError)):
        P.si_evict_rows(torch.empty((1, 2 ** 32 + 5), device="meta"), None, 4, 0, 0, [], meta(1, 4), None, meta(64))
    with pytest.raises(TypeError):  # not a tensor
        binding._ptr(None, torch.uint8, 0, "workspace")


def test_tensors_and_streams_of_another_gpu_are_refused(monkeypatch):
    class OnGpu(torch.Tensor):
        """A host tensor that says it is on a GPU: the checks come before any use of it."""
        gpu = 0

        def get_device(self):
            return self.gpu

    def at(gpu):
        t = torch.zeros(4).as_subclass(OnGpu)
        t.gpu = gpu
        return t

    class Stream:
        device, cuda_stream = torch.device("cuda", 1), 5

    monkeypatch.setattr(binding, "_current_gpu", lambda: 0)
    assert binding._gpu_of(at(0), "x") == 0
    with pytest.raises(ValueError):  # not the current GPU
        binding._gpu_of(at(1), "x")
    with pytest.raises(TypeError):
        binding._gpu_of(torch.zeros(4), "x")
    with pytest.raises((TypeError, ValueError)):  # another GPU than the call's first tensor
        binding._ptr(at(1), torch.float32, 0, "x")
    with pytest.raises(ValueError):
        binding._stream_on(Stream(), 0)
    assert binding._stream_on(Stream(), 1) == 5


def test_reference_by_hand():
    x = np.zeros((1, 32))
    x[0, :10] = [7.0, 5.0, 4.99, 2.5, -0.25, 0.26, -3.5, 0.75, 1.25, 1.75]
    c, e = R.quantize(x)
    assert e.tolist() == [[0]]
    assert c[0, :10].tolist() == [7, 6, 6, 4, 8, 1, 14, 2, 2, 4]  # 6 4 4 2 -0 .5 -4 1 1 2
    x[0, 0] = 7.01
    assert R.quantize(x)[1].tolist() == [[1]]
    x[0, 0] = 1e9
    c, e = R.quantize(x)
    assert e.tolist() == [[13]] and c[0, 0] == 7 and c[0, 1] == 0
    assert R.quantize(np.full((1, 32), 2.0 ** -16))[1].tolist() == [[-13]]
    codes, e = R.quantize(np.array([LV * s for LV in R.LEVELS for s in (1, -1, 1, -1)]).reshape(1, 32))
    packed, scale = R.pack(codes, e)
    assert R.values(packed, scale).tolist() == [[LV * s for LV in R.LEVELS for s in (1, -1, 1, -1)]]
    # one row: its own value whatever the query; two equal logits: the mean
    V = np.array([[[1.0] * 32, [3.0] * 32]])
    out, lse, given = R.attend(np.zeros((1, 1, 1, 32)), V, None, None, 1, 0, 2, 1.0)[:3]
    assert np.allclose(out, 2.0) and np.allclose(lse, np.log(2)) and np.allclose(given, 0.5)
    assert R.evict(np.array([[1, 5, 5, np.nan, -np.inf, 2]], dtype=np.float32), None, 3, 1, 0) == [[0, 1, 2]]
    assert R.evict(np.array([[1, 5, 5, np.nan, -np.inf, 2]], dtype=np.float32), [5], 4, 0, 1) == [[0, 1, 2, 4]]
