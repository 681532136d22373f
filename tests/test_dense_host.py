"""CPU-only: the paged cache's and the packed prompts' entry points refuse what they cannot do before anything is launched (pointers are never
used), the workspace, the binding's checks, and the plain 64-bit reference against values worked by hand."""
import ctypes
import threading

import numpy as np
import pytest
import torch

import paper_2605_02568_amd as P
from paper_2605_02568_amd import binding
from tests import dense_reference as R

A = ctypes.c_void_p
CACHE = dict(K=0x10000, V=0x20000, K_scales=0x30000, V_scales=0x40000, table=0x50004, B=2, table_pages=5, n_pages=9, page_rows=16, H_kv=2, D=64, bits=8)


def _cache(bad):
    fields = {**CACHE, **{k: v for k, v in bad.items() if k in CACHE}}
    return ctypes.byref(binding.si_paged_cache(*fields.values()))


def _rows_calls(**bad):
    a = {**dict(k=0x1000, v=0x2000, N=6, offsets=0x3004, start=0x4004), **bad}
    lib, c = P.load(), None if "cache" in bad else _cache(bad)
    return (lib.si_store_pages(A(a["k"]), A(a["v"]), a["N"], A(a["offsets"]), A(a["start"]), c, None),
            lib.si_load_pages(c, a["N"], A(a["offsets"]), A(a["start"]), A(a["k"]), A(a["v"]), None))


def _attention_call(**bad):
    a = {**dict(q=0x1000, S=3, H=4, lengths=0x6004, first=0x7004, m=1, mask=1, n_win=P.SI_ALL_ROWS, scale=0.1, out=0x8000, lse=0x9004, ws=0xA0000,
                ws_bytes=1 << 30), **bad}
    c = None if "cache" in bad else _cache(bad)
    return P.load().si_paged_attention(A(a["q"]), c, a["S"], a["H"], A(a["lengths"]), A(a["first"]), a["m"], a["mask"], a["n_win"], a["scale"], A(a["out"]),
                                       A(a["lse"]), A(a["ws"]), a["ws_bytes"], None)


BAD, NOT_DONE = P.SI_ERR_INVALID_ARG, P.SI_ERR_UNSUPPORTED_SHAPE


@pytest.mark.parametrize("bad,status", [
    (dict(cache=None), BAD), (dict(K=None), BAD), (dict(table=None), BAD), (dict(K_scales=None), BAD), (dict(V_scales=None), BAD),
    (dict(K=0x10008), BAD), (dict(V=0x20008), BAD), (dict(K_scales=0x30001), BAD), (dict(V_scales=0x40008), BAD), (dict(table=0x50002), BAD),
    (dict(B=0), BAD), (dict(table_pages=0), BAD), (dict(n_pages=0), BAD), (dict(page_rows=0), BAD), (dict(H_kv=0), BAD), (dict(D=0), BAD),
    (dict(bits=4), BAD), (dict(D=96), NOT_DONE), (dict(D=256), NOT_DONE), (dict(page_rows=8), NOT_DONE), (dict(page_rows=48), NOT_DONE),
    (dict(page_rows=2048), NOT_DONE), (dict(H_kv=1025, H=1025), NOT_DONE), (dict(B=(1 << 20) + 1, N=(1 << 20) + 1), NOT_DONE),
    (dict(table_pages=1 << 20, page_rows=1024 * 2), NOT_DONE), (dict(table_pages=(1 << 20) + 1, page_rows=1024), NOT_DONE),
])
def test_caches_that_are_refused(bad, status):
    assert _rows_calls(**bad) == (status, status)
    assert _attention_call(**bad) == status


@pytest.mark.parametrize("bad,status", [
    (dict(k=0x1008), BAD), (dict(v=0x2004), BAD), (dict(offsets=0x3001), BAD), (dict(start=0x4002), BAD), (dict(N=0), BAD), (dict(N=-1), BAD),
    (dict(offsets=None, N=5), BAD), (dict(N=(1 << 27) + 2), NOT_DONE), (dict(N=1 << 27, H_kv=1024, H=1024), NOT_DONE),
])
def test_rows_that_are_refused(bad, status):
    assert _rows_calls(**bad) == (status, status)


def test_rows_without_an_array():
    assert _rows_calls(k=None)[0] == BAD and _rows_calls(v=None)[0] == BAD  # both have to be stored
    assert _rows_calls(k=None, v=None)[1] == BAD  # either may be left in the cache
    assert _rows_calls(V=None)[1] == BAD  # values that there are not


@pytest.mark.parametrize("bad,status", [
    (dict(q=None), BAD), (dict(out=None), BAD), (dict(ws=None), BAD), (dict(q=0x1008), BAD), (dict(out=0x8008), BAD), (dict(ws=0xA0008), BAD),
    (dict(lengths=0x6001), BAD), (dict(first=0x7002), BAD), (dict(lse=0x9001), BAD), (dict(S=0), BAD), (dict(H=0), BAD), (dict(H=3), BAD),
    (dict(m=0), BAD), (dict(n_win=-1), BAD), (dict(mask=2), BAD), (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD),
    (dict(scale=2.5e38), BAD), (dict(H=1026), NOT_DONE), (dict(S=1 << 21, H=4), NOT_DONE), (dict(B=(1 << 14) + 1), NOT_DONE),
    (dict(ws_bytes=100), P.SI_ERR_WORKSPACE_TOO_SMALL),
    (dict(ws_bytes=lambda: P.si_paged_workspace_bytes(2, 3, 4, 2, 64) - 1), P.SI_ERR_WORKSPACE_TOO_SMALL),
])
def test_attention_that_is_refused(bad, status):
    assert _attention_call(**{k: v() if callable(v) else v for k, v in bad.items()}) == status


def test_workspace():
    # room for the parts of all sequences: each a result of fp32 and its two sums
    for B, S, H, H_kv, D in ((1, 1, 64, 8, 128), (64, 1, 64, 8, 128), (24, 4, 40, 8, 64), (1 << 14, 1, 1, 1, 64)):
        n = P.si_paged_workspace_bytes(B, S, H, H_kv, D)
        part = S * H * (D + 2) * 4
        assert (n - 8 * B) % part == 0 and (n - 8 * B) // part > B
        assert n <= 4 * (D + 4) * (131072 + 2 * B * S * H)
    for bad in ((0, 1, 4, 2, 64), (1, 0, 4, 2, 64), (1, 1, 5, 2, 64), (1, 1, 4, 0, 64), (1, 1, 4, 2, 0), ((1 << 14) + 1, 1, 4, 2, 64)):
        assert P.si_paged_workspace_bytes(*bad) == 0


PROMPT = dict(q=0x1000, K=0x2000, V=0x3000, dims=(2, 10, 20, 4, 2, 64), qo=0x4004, ko=0x5004, first=0x6004, m=1, mask=1, n_win=P.SI_ALL_ROWS, scale=0.1,
              out=0x7000, lse=0x8004)


@pytest.mark.parametrize("bad,status", [
    (dict(q=None), BAD), (dict(K=None), BAD), (dict(dims=None), BAD), (dict(out=None), BAD), (dict(q=0x1008), BAD), (dict(K=0x2008), BAD),
    (dict(V=0x3008), BAD), (dict(out=0x7004), BAD), (dict(qo=0x4001), BAD), (dict(ko=0x5002), BAD), (dict(first=0x6001), BAD), (dict(lse=0x8002), BAD),
    (dict(dims=(0, 10, 20, 4, 2, 64)), BAD), (dict(dims=(2, 0, 20, 4, 2, 64)), BAD), (dict(dims=(2, 10, 0, 4, 2, 64)), BAD),
    (dict(dims=(2, 10, 20, 0, 2, 64)), BAD), (dict(dims=(2, 10, 20, 4, 0, 64)), BAD), (dict(dims=(2, 10, 20, 5, 2, 64)), BAD),
    (dict(dims=(2, 10, 20, 4, 2, 0)), BAD), (dict(dims=(3, 10, 21, 4, 2, 64), qo=None), BAD), (dict(dims=(3, 12, 20, 4, 2, 64), ko=None), BAD),
    (dict(m=0), BAD), (dict(mask=2), BAD), (dict(n_win=-1), BAD), (dict(scale=float("nan")), BAD), (dict(scale=-3e38), BAD),
    (dict(dims=(2, 10, 20, 4, 2, 32)), NOT_DONE), (dict(dims=(2, 10, 20, 1026, 2, 64)), NOT_DONE), (dict(dims=(2, (1 << 30) + 1, 20, 1, 1, 64)), NOT_DONE),
    (dict(dims=(2, 10, (1 << 30) + 1, 1, 1, 64)), NOT_DONE), (dict(dims=((1 << 20) + 1, 10, 20, 1, 1, 64)), NOT_DONE),
    (dict(dims=(2, 1 << 20, 20, 1024, 1, 64)), NOT_DONE),
])
def test_prompts_that_are_refused(bad, status):
    a = {**PROMPT, **bad}
    d = None if a["dims"] is None else ctypes.byref(binding.si_packed_dims(*a["dims"]))
    got = P.load().si_prompt_attention(A(a["q"]), A(a["K"]), A(a["V"]), d, A(a["qo"]), A(a["ko"]), A(a["first"]), a["m"], a["mask"], a["n_win"], a["scale"],
                                       A(a["out"]), A(a["lse"]), None)
    assert got == status


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="on a machine with a GPU these calls would launch on addresses that are not memory")
@pytest.mark.parametrize("name,call", [
    ("store", lambda: _rows_calls()[0]), ("load", lambda: _rows_calls()[1]), ("attention", lambda: _attention_call()),
    ("prompt", lambda: P.load().si_prompt_attention(A(0x1000), A(0x2000), None, ctypes.byref(binding.si_packed_dims(2, 10, 20, 4, 2, 64)), None, None, None, 1,
                                                    0, 5, 0.1, A(0x7000), None, None)),
])
def test_a_failed_launch_is_named(name, call):
    seen = {}

    def run():  # in a thread of its own: the last error is a thread's, and a new thread has none
        seen["before"] = P.load().si_last_hip_error()
        seen["status"] = call()
        seen["after"] = P.load().si_last_hip_error()

    t = threading.Thread(target=run)
    t.start()
    t.join()
    assert seen["before"] == 0 and seen["status"] == P.SI_ERR_HIP and seen["after"] != 0


# ---------------------------------------------------------------------------------- the binding
def test_the_binding_wants_gpu_tensors_of_fitting_shapes():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    table = torch.zeros((2, 3), dtype=torch.int32)
    K = bf(5, 2, 16, 64)
    with pytest.raises(TypeError, match="table must be a GPU tensor"):
        P.si_store_pages(bf(4, 2, 64), bf(4, 2, 64), None, None, table, K, K)
    with pytest.raises(TypeError, match="q must be a GPU tensor"):
        P.si_prompt_attention(bf(4, 2, 64), bf(4, 1, 64), None, None, None, None, 1, 0, 5, 0.1, bf(4, 2, 64))
    with pytest.raises(ValueError, match="no scales"):
        P.si_store_pages(bf(4, 2, 64), None, None, None, table, K, None, torch.zeros(5, 2, 16, dtype=torch.uint8))
    with pytest.raises(ValueError, match="k_scales must be"):
        P.si_store_pages(bf(4, 2, 64), None, None, None, table, K.to(torch.uint8), None)
    with pytest.raises(ValueError, match="v_scales must be"):
        P.si_store_pages(bf(4, 2, 64), None, None, None, table, K.to(torch.uint8), K.to(torch.uint8), torch.zeros(5, 2, 16, dtype=torch.uint8))
    with pytest.raises(TypeError, match="bfloat16 or"):
        P.si_load_pages(table, K.float(), None, None, None, None, None, bf(4, 2, 64), None)
    with pytest.raises(ValueError, match="V must be"):
        P.si_load_pages(table, K, bf(5, 2, 16, 128), None, None, None, None, bf(4, 2, 64), None)
    with pytest.raises(ValueError, match="table must be"):
        P.si_load_pages(table[0], K, None, None, None, None, None, bf(4, 2, 64), None)
    with pytest.raises(ValueError, match="q must be"):
        P.si_prompt_attention(bf(4, 2, 64), bf(4, 1, 128), None, None, None, None, 1, 0, 5, 0.1, bf(4, 2, 64))
    with pytest.raises(ValueError, match="out must be"):
        P.si_prompt_attention(bf(4, 2, 64), bf(4, 1, 64), None, None, None, None, 1, 0, 5, 0.1, bf(4, 1, 64))
    with pytest.raises(ValueError, match="lse must be"):
        P.si_prompt_attention(bf(4, 2, 64), bf(4, 1, 64), None, None, None, None, 1, 0, 5, 0.1, bf(4, 2, 64), torch.zeros(2, 4))
    with pytest.raises(ValueError):
        P.si_paged_workspace_bytes(1, 2 ** 31, 1, 1, 64)


def test_the_packed_cache_is_the_header_s_struct():
    fields = tuple(range(1, 13))
    c = binding.si_paged_cache.from_buffer_copy(binding._cache_layout.pack(*fields))
    assert tuple(getattr(c, name) for name, _ in c._fields_) == fields
    assert binding._cache_layout.size == ctypes.sizeof(binding.si_paged_cache)


# ---------------------------------------------------------------------------------- the reference
def test_codes_by_hand():
    x = np.array([[448.0, 449.0 / 2, 1.0, -0.0625, 17.0, 19.0, 2.0 ** -9, 2.0 ** -10]])
    codes, e = R.quantize(x)
    assert e[0] == 0
    assert R.values(codes, e)[0].tolist() == [448.0, 224.0, 1.0, -0.0625, 16.0, 20.0, 2.0 ** -9, 0.0]  # ties to even codes
    codes, e = R.quantize(np.array([[449.0, 1.0, np.nan, 0.0]]))
    assert e[0] == 1 and codes[0].tolist()[2:] == [127, 0] and R.values(codes, e)[0, :2].tolist() == [448.0, 1.0]
    assert R.quantize(np.zeros((1, 4)))[1][0] == R.LOWEST and R.quantize(np.full((1, 4), np.inf))[1][0] == R.HIGHEST


def test_attention_by_hand():
    K = np.array([[[0.0, 0.0]], [[np.log(3.0), 0.0]], [[5.0, 5.0]]])
    V = np.array([[[4.0, 0.0]], [[0.0, 8.0]], [[100.0, 100.0]]])
    q = np.array([[[1.0, 0.0]], [[1.0, 0.0]]])
    out, lse, _, _ = R.attend(q, K, V, [0, 1], 1, 1, R.ALL, 1.0)
    np.testing.assert_allclose(out[:, 0], [[4.0, 0.0], [1.0, 6.0]], rtol=1e-12)
    np.testing.assert_allclose(lse[:, 0], [0.0, np.log(4.0)], rtol=1e-12, atol=1e-12)
    out, lse, _, _ = R.attend(q, K, V, [-1, 1], 1, 1, 1, 1.0)  # nothing, and a window of one row
    np.testing.assert_allclose(out[:, 0], [[0.0, 0.0], [0.0, 8.0]], rtol=1e-12)
    assert np.isneginf(lse[0, 0])
    assert [R.legal(t, 5, 4, 1) for t in (-1, 0, 2, 3, 19, 30)] == [0, 0, 0, 1, 5, 5]
