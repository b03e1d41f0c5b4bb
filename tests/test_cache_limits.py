"""Limits of the paged cache that the host checks before any GPU work, and the binding's treatment of what it is given."""
import pytest


@pytest.fixture(scope="module")
def Bn():
    import os
    from paper_2606_03819_gb300 import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2606_03819_gb300 import build
        build.build()
    binding.load_library()
    return binding


@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_lengths_leave_room_for_rounding_up_to_tiles(Bn, page):
    # the kernels form (length + 127) and look two tiles of 128 tokens ahead in 32 bits
    dims = lambda most: Bn.CacheDims(batch=1, heads=1, kv_heads=1, head_dim=64, page=page, n_pages=8, max_pages=most)  # noqa: E731
    most = (2 ** 31 - 1024) // page
    assert Bn.tf_attention_workspace_size(dims(most), 1) > 0
    for more in (most + 1, (2 ** 31 - 1) // page):
        with pytest.raises(Bn.TreeFlashError) as e:
            Bn.tf_attention_workspace_size(dims(more), 1)
        assert e.value.status == Bn.TF_ERR_UNSUPPORTED
