"""The example's layer refuses more tokens than it was made for, before anything is
indexed by them on the GPU."""
import os
import sys

import pytest
import torch

from tests.kv4_cases import DEV

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_more_tokens_than_the_layer_holds():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from sparse_decode import SparseLayer, fp8
    layer = SparseLayer(2, 20, q_heads=4, kv_heads=2, head_dim=64, K=8, page=16)

    def prompt(n):
        q, k = torch.randn((2 * n, 4, 64), device=DEV).bfloat16(), torch.randn((2 * n, 2, 64), device=DEV).bfloat16()
        return layer.prompt(q, k, k, fp8((2 * n, 128), DEV))

    with pytest.raises(ValueError):
        prompt(21)
    assert prompt(15).shape == (30, 4, 64) and torch.isfinite(prompt(5)).all()
    before = layer.cache.clone()
    with pytest.raises(ValueError):
        prompt(1)
    assert torch.equal(layer.cache, before) and layer.length.tolist() == [20, 20]
