"""Cache plans at the largest tables that the dimensions allow."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def Bn():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_03819_gb300 import binding
    binding.load_library()
    return binding


def test_pages_asked_for_are_added_up_beyond_32_bits(Bn):
    # 17 sequences of 2^27 - 64 pages each ask for more than 2^31 together: all of them are refused, and so are those behind them
    page, most, n_pages = 16, (1 << 27) - 64, 64
    b = 19
    dims = Bn.CacheDims(batch=b, heads=1, kv_heads=1, head_dim=16, page=page, n_pages=n_pages, max_pages=most)
    t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.full((b, most), -1, dtype=torch.int32, device="cuda")
    free, count = torch.arange(n_pages, dtype=torch.int32, device="cuda"), t([n_pages])
    lens, status = t([0] * b), t([9] * b)
    delta = t([2 * page] + [most * page] * (b - 2) + [1])
    Bn.tf_cache_plan(dims, lens, delta, 0, table, free, count, None, lens, status)
    torch.cuda.synchronize()
    assert status.tolist() == [0] + [Bn.TF_DEV_POOL_EMPTY] * (b - 1)
    assert lens.tolist() == [2 * page] + [0] * (b - 1)
    assert count.item() == n_pages - 2 and free.tolist() == list(range(n_pages))
    assert table[0, :3].tolist() == [n_pages - 1, n_pages - 2, -1]
    assert all(int((row >= 0).sum()) == (2 if s == 0 else 0) for s, row in enumerate(table))
