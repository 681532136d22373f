"""GPU: the 4-bit cache's attention and accumulated weights at the ends of what their arguments may be."""
import pytest
import torch

from tests.test_gpu_cache import NONE, _check, _problem

pytestmark = pytest.mark.gpu


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
