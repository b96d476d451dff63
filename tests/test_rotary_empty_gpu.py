"""Rotations of no tokens through the binding."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_queries_and_keys_of_no_tokens(dtype):
    from paper_2605_09681_gb300 import Rotary
    rotary = Rotary(head_dim=64, axes=(20, 12))
    pos = torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    q, k = (torch.zeros(0, h, 64, dtype=dtype, device="cuda") for h in (6, 2))
    a, b = rotary.rotate(pos, q, k)
    assert a.shape == q.shape and b.shape == k.shape and a.dtype == b.dtype == dtype
    assert rotary.rotate(pos, q, k, inverse=True, Q_out=q, K_out=k) == (q, k)
    wide = torch.zeros(5, 10, 64, dtype=dtype, device="cuda")
    a, b = rotary.rotate(pos, wide[2:2, :6], wide[2:2, 6:8], stream=torch.cuda.Stream())
    assert a.shape == (0, 6, 64) and b.shape == (0, 2, 64)
    torch.cuda.synchronize()
