"""PagedCache's refusals of caches that it cannot use, without a GPU."""
import pytest
from torch._subclasses.fake_tensor import FakeTensor

from test_attention_boundary import BF, I32, new  # noqa: F401  (a fixture)
from paper_1908_11263_gb300 import qnn


def batch(new):  # noqa: F811
    return new(3, 4, dtype=I32), new(3, dtype=I32)


def test_a_cache_without_heads_is_refused(new):  # noqa: F811
    cache = qnn.PagedCache(new(9, 0, 16, 64), new(9, 0, 16, 64))
    with pytest.raises(ValueError, match="heads"):
        cache.attend(new(3, 8, 64), *batch(new))


def test_tensors_are_not_replaced_behind_the_cache(new):  # noqa: F811
    cache = qnn.PagedCache(new(9, 2, 16, 64), new(9, 2, 16, 64))
    for name in ("k", "v"):
        with pytest.raises(AttributeError):
            setattr(cache, name, new(20, 2, 16, 64))


@pytest.mark.parametrize("moved", ["k", "v"])
def test_tensors_that_have_moved_are_refused(new, monkeypatch, moved):  # noqa: F811
    """Memory that the cache's tensors have given up (their storage was replaced or resized) is neither read nor written."""
    places = {}
    monkeypatch.setattr(FakeTensor, "data_ptr", lambda t: places.get(id(t), 4096), raising=False)
    cache = qnn.PagedCache(new(9, 2, 16, 64), new(9, 2, 16, 64))
    call = {"append": lambda: cache.append(new(3, 2, 64), new(3, 2, 64), *batch(new)),
            "attend": lambda: cache.attend(new(3, 8, 64), *batch(new))}
    for f in call.values():
        with pytest.raises(AssertionError, match="was reached"):
            f()
    places[id(getattr(cache, moved))] = 8192
    for f in call.values():
        with pytest.raises(ValueError, match="moved"):
            f()
