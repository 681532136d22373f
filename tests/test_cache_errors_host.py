"""CPU-only: a HIP call that fails in an entry point of the cache or of the attention is what si_last_hip_error() then names."""
import ctypes
import threading

import pytest
import torch

import paper_2605_02568_amd as P
from paper_2605_02568_amd import binding

A = ctypes.c_void_p

CALLS = {
    "si_quantize_rows": lambda lib, d: lib.si_quantize_rows(A(0x1000), None, d, A(0x2000), A(0x3000), None),
    "si_dequantize_rows": lambda lib, d: lib.si_dequantize_rows(A(0x2000), A(0x3000), None, d, A(0x1000), None),
    "si_quantized_attention": lambda lib, d: lib.si_quantized_attention(A(0x1000), A(0x2000), A(0x3000), None, None, d, 1, 0, 0, 4, 0.1, A(0x6000),
                                                                        None, None),
    "si_accumulate_weights": lambda lib, d: lib.si_accumulate_weights(A(0x1000), A(0x2000), A(0x3000), None, None, d, 1, 0, 0, 4, 0.1, A(0x7000),
                                                                      A(0x8000), A(0x9000), 800, None),
    "si_evict_rows": lambda lib, d: lib.si_evict_rows(A(0x10000), None, 2, 1000, 600, 4, 100, None, 0, A(0x30000), None, A(0x40000), 1 << 16, None),
    "si_sparse_attention": lambda lib, d: lib.si_sparse_attention(A(0x1000), A(0x2000), A(0x3000), d, 1, 8, 0, 4, 0.1, A(0x6000), None),
}


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="on a machine with a GPU these calls would launch on addresses that are not memory")
@pytest.mark.parametrize("name", CALLS)
def test_a_failed_launch_is_named(name):
    seen = {}

    def call():  # in a thread of its own: the last error is a thread's, and a new thread has none
        lib = P.load()
        seen["before"] = lib.si_last_hip_error()
        seen["status"] = CALLS[name](lib, ctypes.byref(binding.si_dims(2, 3, 4, 64, 50)))
        seen["after"] = lib.si_last_hip_error()

    t = threading.Thread(target=call)
    t.start()
    t.join()
    assert seen["before"] == 0
    assert seen["status"] == P.SI_ERR_HIP
    assert seen["after"] != 0
