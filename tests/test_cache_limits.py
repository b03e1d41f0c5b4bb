"""Limits of the paged cache that the host checks before any GPU work, and the binding's treatment of what it is given."""
import pytest
import torch


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


class OnGpu(torch.Tensor):
    """A tensor that says it lies on some GPU."""
    gpu = 0

    def get_device(self):
        return self.gpu


def _calls(Bn):
    """(function, its arguments in good order as {name: value}) of the four calls."""
    d = Bn.CacheDims(batch=2, heads=4, kv_heads=2, head_dim=64, page=16, n_pages=8, max_pages=4)
    z = lambda *s, dt=torch.int32: torch.zeros(*s, dtype=dt).as_subclass(OnGpu)  # noqa: E731
    f32, u8, bf = torch.float32, torch.uint8, torch.bfloat16
    pools = lambda: dict(k_cache=z(8, 2, 16, 64, dt=u8), v_cache=z(8, 2, 16, 64, dt=u8), k_scale=z(8, 2, dt=f32), v_scale=z(8, 2, dt=f32))  # noqa: E731
    kv = lambda: dict(k=z(2, 3, 2, 64, dt=bf), v=z(2, 3, 2, 64, dt=bf))  # noqa: E731
    return {
        "plan": (Bn.tf_cache_plan, dict(dims=d, seq_len=z(2), delta=z(2), extra=0, block_table=z(2, 4), free_list=z(8), free_count=z(1),
                                        slot_map=z(2, 5), new_len=z(2), dev_status=z(2))),
        "append": (Bn.tf_cache_append, dict(dims=d, **kv(), slot_map=z(2, 3), src=z(2, 3), **pools(), dev_status=z(2))),
        "attention": (Bn.tf_tree_attention, dict(dims=d, q=z(2, 3, 4, 64, dt=bf), **kv(), **pools(), block_table=z(2, 4), seq_len=z(2),
                                                 mask=z(2, 3, 3, dt=u8), scale=1.0, out=z(2, 3, 4, 64, dt=bf), lse=z(2, 3, 4, dt=f32),
                                                 dev_status=z(2), ws=z(64, dt=u8))),
        "sample": (Bn.tf_sample, dict(logits=z(4, 10, dt=f32), u=z(4, dt=f32), tok=z(4), logp=z(4, dt=f32), temperature=z(2, dt=f32), top_k=z(2),
                                      top_p=z(2, dt=f32), min_p=z(2, dt=f32), rows_per_seq=2)),
    }


@pytest.mark.parametrize("name", ["plan", "append", "attention", "sample"])
def test_tensors_on_the_host_or_another_gpu_are_refused(Bn, name, monkeypatch):
    reached = []

    class Lib:
        def __getattr__(self, fn):
            return lambda *a: reached.append(fn) or 0

    class Null:
        cuda_stream = None

    monkeypatch.setattr(Bn, "load_library", Lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    f, args = _calls(Bn)[name]
    f(**args, stream=Null)
    assert len(reached) == 1
    tensors = [k for k, x in args.items() if torch.is_tensor(x)]
    for key in tensors:
        for gpu in (-1, 1):
            bad = dict(args)
            bad[key] = args[key].clone().as_subclass(OnGpu)
            bad[key].gpu = gpu
            with pytest.raises(ValueError, match=f"^{key}: .*current CUDA device"):
                f(**bad, stream=Null)
    for x in args.values():                                   # all of them on another GPU than the current one
        if torch.is_tensor(x):
            x.gpu = 1
    with pytest.raises(ValueError, match="current CUDA device"):
        f(**args, stream=Null)
    assert len(reached) == 1


def test_bits_that_two_e4m3_parts_keep_of_a_query():
    # a row's largest element lies in [2^7, 2^8); hi is the nearest e4m3 number, lo that of the rest: every bf16 number (8 bits) below it
    import numpy as np
    from oracle import verifier_oracle as VO
    worst = 0.0
    for top in np.arange(128, 256) * 2.0 ** 7 / 128:
        x = (np.arange(128, 256)[:, None] / 128 * 2.0 ** np.arange(-24, 8)[None, :]).ravel()
        x = x[x <= top]
        hi = VO.from_e4m3(VO.to_e4m3(x))
        lo = VO.from_e4m3(VO.to_e4m3(x - hi))
        off = np.abs(x - hi - lo)
        assert not off[x >= top * 2.0 ** -9].any()
        worst = max(worst, float((off / top).max()))
    assert worst == 2.0 ** -17


def test_a_single_row_may_have_any_stride(Bn):
    # the first token of a buffer whose rows are 516 elements apart: the distance to a next row, which there is not, does not matter
    bf = torch.bfloat16
    x = torch.zeros(1, 3, 516, dtype=bf)[..., :512].unflatten(2, (8, 64))
    assert Bn._take_rows("q", x[:, :1], bf, 1, 8, 64) == (1, 512)
    assert Bn._take_rows("q", x, bf, 1, 8, 64) == (3, 516)          # (refused by the library)
    assert Bn._take_rows("q", torch.zeros(1, 1, 8, 64, dtype=bf), bf, 1, 8, 64) == (1, 512)
    y = torch.zeros(2, 3, 1024, dtype=bf)[..., :512].unflatten(2, (8, 64))
    assert Bn._take_rows("q", y[:, :1], bf, 2, 8, 64) == (1, 3072)
    assert Bn._take_rows("q", torch.zeros(2, 1, 8, 64, dtype=bf), bf, 2, 8, 64) == (1, 512)
