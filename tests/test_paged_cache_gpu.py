"""PagedCache on the GPU: streams other than the current one, refusals, and what its calls leave behind."""
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


def _cache(Bn, **kw):
    from paper_2606_03819_gb300 import PagedCache
    base = dict(batch=3, heads=8, kv_heads=2, head_dim=64, page=16, n_pages=40, max_pages=12)
    base.update(kw)
    return PagedCache(Bn.CacheDims(**base), layers=2, n_max=9)


def test_a_side_stream_while_the_current_one_is_busy(Bn):
    g = torch.Generator(device="cuda").manual_seed(0)
    i32 = dict(dtype=torch.int32, device="cuda")
    steps, width = 6, 9
    qkv = [torch.randn(3, width, 12, 64, generator=g, device="cuda").to(torch.bfloat16) for _ in range(steps)]
    delta = [torch.randint(0, width + 1, (3,), generator=g, **i32) for _ in range(steps)]
    which = [torch.rand(3, generator=g, device="cuda") < 0.4 for _ in range(steps)]
    busy = torch.randn(4096, 4096, generator=g, device="cuda").to(torch.bfloat16)

    def decode(cache, stream, between):
        outs = []
        for i in range(steps):
            between()
            q, k, v = qkv[i].split([8, 2, 2], 2)
            outs.append(cache.attend(0, q, k, v, stream=stream))
            slots = cache.grow(delta[i], width=width, stream=stream)
            cache.append(0, k, v, slots, stream=stream)
            outs.append(slots)
            cache.release(which[i], stream=stream)
        return outs

    plain, other = _cache(Bn), _cache(Bn)
    want = decode(plain, None, lambda: None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()

    def work():
        for _ in range(40):
            torch.mm(busy, busy)
        torch.zeros(3, width, **i32)                          # the current stream's pool is asked for tensors of the same size
        torch.full((3, width, 8, 64), 5.0, dtype=torch.bfloat16, device="cuda")

    have = decode(other, s, work)
    assert other.status(stream=s) == 0 == plain.status()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, have))
    for name in ("seq_len", "block_table", "free_count", "k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(plain, name), getattr(other, name)), name
    n = plain.free_count.item()
    assert torch.equal(plain.free_list[:n], other.free_list[:n])


def test_a_refusal_is_kept_until_it_is_cleared(Bn):
    cache = _cache(Bn, n_pages=5)
    t = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache.grow(t(40, 16, 1), width=40)                        # 3 + 1 pages; the fifth is the last one's
    assert cache.status() == 0
    cache.grow(t(1, 1, 16), width=16)                         # a page each for the second and the third: none is left
    assert cache.plan_status.tolist() == [0, Bn.TF_DEV_POOL_EMPTY, Bn.TF_DEV_POOL_EMPTY]
    assert cache.seq_len.tolist() == [41, 16, 1]
    cache.grow(t(0, 0, 0))
    cache.grow(t(1, 0, 200), width=16)                        # longer than the slot map
    cache.release(torch.tensor([True, False, False], device="cuda"))
    assert cache.plan_status.tolist() == [0, 0, 0]
    assert cache.dev_status.tolist() == [0, Bn.TF_DEV_POOL_EMPTY, Bn.TF_DEV_POOL_EMPTY | Bn.TF_DEV_BAD_LENGTH]
    assert cache.status() == Bn.TF_DEV_POOL_EMPTY | Bn.TF_DEV_BAD_LENGTH
    cache.clear_status()
    assert cache.status() == 0
    cache.grow(t(1, 1, 16), width=16)                         # the released pages serve them now
    assert cache.status() == 0 and cache.seq_len.tolist() == [1, 17, 17]
