"""PagedCache's own part of its calls, without a GPU: the C entry points are replaced by recorders."""
from contextlib import contextmanager

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


@pytest.fixture
def cache(Bn):
    from paper_2606_03819_gb300 import PagedCache
    dims = Bn.CacheDims(batch=3, heads=4, kv_heads=2, head_dim=64, page=16, n_pages=12, max_pages=6)
    return PagedCache(dims, layers=2, n_max=4, device="cpu")


class Stream:
    cuda_stream = 4711


def test_what_a_call_makes_itself_is_made_on_the_stream_it_is_given(Bn, cache, monkeypatch):
    current, made, ran = [None], [], []

    @contextmanager
    def as_current(stream):
        current.append(stream)
        yield
        current.pop()

    def noting(f):
        def g(*a, **kw):
            made.append(current[-1])
            return f(*a, **kw)
        return g

    monkeypatch.setattr(torch.cuda, "stream", as_current)
    for name in ("empty", "where", "cat"):
        monkeypatch.setattr(torch, name, noting(getattr(torch, name)))
    for name in ("tf_cache_plan", "tf_tree_attention"):
        monkeypatch.setattr(Bn, name, lambda *a, **kw: ran.append(a))
    s = Stream()
    q, k = torch.zeros(3, 2, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 2, 64, dtype=torch.bfloat16)
    for call in (lambda **kw: cache.grow(torch.zeros(3, dtype=torch.int32), width=4, **kw),
                 lambda **kw: cache.release(torch.ones(3, dtype=torch.bool), **kw), lambda **kw: cache.attend(1, q, k, k, **kw),
                 lambda **kw: cache.status(**kw)):
        for kw, want in ((dict(stream=s), s), (dict(), None)):
            made.clear()
            call(**kw)
            assert made and all(x is want for x in made) and current == [None]
    assert len(ran) == 6 and all(a[-1] is s for a in ran[::2]) and all(a[-1] is None for a in ran[1::2])


def test_every_refusal_stays_in_the_status(Bn, cache, monkeypatch):
    # a plan overwrites its words: here the first one refuses two sequences, those after it none
    words = iter([[0, Bn.TF_DEV_POOL_EMPTY, Bn.TF_DEV_BAD_LENGTH], [0, 0, 0], [0, 0, 0]])
    monkeypatch.setattr(Bn, "tf_cache_plan", lambda *a: a[9].copy_(torch.tensor(next(words), dtype=torch.int32)))
    cache.grow(torch.zeros(3, dtype=torch.int32))
    cache.grow(torch.zeros(3, dtype=torch.int32))
    cache.release(torch.ones(3, dtype=torch.bool))
    assert cache.status() == Bn.TF_DEV_POOL_EMPTY | Bn.TF_DEV_BAD_LENGTH
    cache.clear_status()
    assert cache.status() == 0
