"""CPU-only: whole numbers beyond an int32 are refused by the cache's calls, not cut to their lowest 32 bits."""
import pytest
import torch

import paper_2605_02568_amd as P
from paper_2605_02568_amd import binding


class _Library:
    """Takes every call and notes it."""
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return P.SI_OK
        return call


@pytest.fixture
def library(monkeypatch):
    lib = _Library()
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_gpu_of", lambda t, name: 0)  # host tensors pass for ones of the GPU
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype, gpu, name: 0x1000)
    monkeypatch.setattr(binding, "_stream_on", lambda stream, gpu: 0)
    return lib


B, S, H, D, T, K, N = 2, 3, 4, 64, 10, 5, 6
Q = torch.zeros((B, S, H, D), dtype=torch.bfloat16)
CODES, SCALES = torch.zeros((B, T, D // 2), dtype=torch.uint8), torch.zeros((B, T, D // 32), dtype=torch.uint8)
IDX = torch.zeros((B, S, K), dtype=torch.int32)
LSE, WEIGHTS = torch.zeros((B, S, H)), torch.zeros((B, T))
WS, KEPT = torch.zeros(1 << 12, dtype=torch.uint8), torch.zeros((B, N), dtype=torch.int32)


def _attention(m=1, mask=0, n_win=0):
    P.si_quantized_attention(Q, CODES, SCALES, None, IDX, m, mask, n_win, 1.0, torch.zeros((B, S, H, D)), LSE)


def _weights(m=1, mask=0, n_win=0):
    P.si_accumulate_weights(Q, CODES, SCALES, None, IDX, m, mask, n_win, 1.0, LSE, WEIGHTS, WS)


def _evict(n_sink=0, n_recent=0):
    P.si_evict_rows(WEIGHTS, None, N, n_sink, n_recent, [], KEPT, None, WS)


@pytest.mark.parametrize("number", [2 ** 31, 2 ** 32 + 1, -2 ** 31 - 1, -2 ** 32 + 1])
@pytest.mark.parametrize("call,name", [(_attention, "m"), (_attention, "mask"), (_attention, "n_win"), (_weights, "m"), (_weights, "mask"),
                                       (_weights, "n_win"), (_evict, "n_sink"), (_evict, "n_recent")])
def test_numbers_beyond_int32_are_refused(library, call, name, number):
    call()
    assert len(library.calls) == 1
    with pytest.raises(ValueError):
        call(**{name: number})
    assert len(library.calls) == 1
