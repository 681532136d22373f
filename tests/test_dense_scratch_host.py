"""CPU-only: no kernel of the paged cache or of packed prompts keeps anything in scratch memory.  Their loops have loads on the way to LDS, and a
register that comes back from scratch memory waits for all of them."""
import pytest

from tests.test_cache_scratch_host import scratch_bytes  # noqa: F401

KERNELS = {"store_pages_kernel": 12, "load_pages_kernel": 12, "paged_attention_kernel": 12, "join_chunks_kernel": 4, "deal_chunks_kernel": 1, "prompt_attention_kernel": 4}


@pytest.mark.parametrize("kernel,forms", KERNELS.items())
def test_no_kernel_uses_scratch(scratch_bytes, kernel, forms):  # noqa: F811
    found = {name: n for name, n in scratch_bytes.items() if f"{len(kernel)}{kernel}" in name}
    assert len(found) == forms and not any(found.values()), found
