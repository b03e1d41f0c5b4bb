"""Attention over the paged cache at the edges of its numbers."""
import math

import pytest
import torch

from test_verifier_gpu import _attend, _setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def Bn():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_03819_gb300 import binding
    binding.load_library()
    return binding


# new tokens per sequence: kernels for few rows and for many (groups of four rows per token)
FEW_AND_MANY = [1, 4, 17, 40]


@pytest.mark.parametrize("n", FEW_AND_MANY)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_a_query_that_is_not_finite_gives_nan_in_its_row_alone(Bn, n, dtype, value):
    # its scores are infinities of both signs: cached keys have either, and the new tokens' keys are made to score -inf
    c = _setup(Bn, lens=[37, 300], n=n, heads=8, kv_heads=2, hd=64, page=16, dtype=dtype, seed=21, mask="causal")
    d = c["dims"]
    c["qkv"][:, :, d.heads, 5] = -1.0 if value == math.inf else 1.0
    want, want_lse, _ = _attend(Bn, c)
    assert want.isfinite().all()
    i = n - 1
    c["qkv"][:, i, 2, 5] = value                              # head 2 reads the keys' head 0
    out, lse, status = _attend(Bn, c)
    assert not status.any()
    assert out[:, i, 2].isnan().all() and lse[:, i, 2].isnan().all()
    rest = torch.ones_like(lse, dtype=torch.bool)
    rest[:, i, 2] = False
    assert torch.equal(out[rest], want[rest]) and torch.equal(lse[rest], want_lse[rest])
